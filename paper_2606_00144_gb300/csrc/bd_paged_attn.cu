// Verify blocks, and decoding one token, over a paged cache (bd_paged_verify_attn): n_q queries per head at positions
// T .. T + n_q - 1 over the keys of [0, T + i] whose pages are there.
//
//   o_i = sum_k 2^(s_ik - M) v_k / sum_k 2^(s_ik - M),  s = q k log2(e) / sqrt(d)
//
// One pass over K and V with a running maximum and sum.  The (unit, 64-key tile) pairs of all (sequence, KV head)
// units form one list, cut into contiguous ranges of equal cost, one per CTA; each piece of a unit ("segment") ends in
// a normalised partial, and row-merge joins the segments of units that span CTAs.
//   warp 4      producer: a tile is 64 / (rows of a box) pages' pieces of K and of V, each one TMA box (rows x both
//               64-column halves), one lane each, which looked its page up a tile ahead.  Pieces whose page is not there, or that
//               lie past the sequence's block, are not read.
//   warps 0..3  16 keys of a tile each on mma.sync (bd_attn_warp.cuh), the query rows on the N side.
// The pieces of a tile lie one behind the other, so a warp's 16 keys are in one piece (pages hold at least 16 rows).
#include <algorithm>

#include "bd_attn_warp.cuh"
#include "bd_internal.h"
#include "bd_paged.cuh"
#include "bd_verify.cuh"

namespace bd {

constexpr int kPvKeys = 64;           // keys of a tile
constexpr int kPvWarps = 4;           // consumer warps
constexpr int kPvThreads = 160;       // + one producer warp
constexpr int kPvStages = 5;
constexpr int kPvMaxRows = 24;        // query rows of a unit; more go to the tcgen05 kernel,
constexpr int kPvTcMaxRows = 256;     // which takes this many: two M tiles

struct PagedVerifyParams {
  const __nv_bfloat16* q;             // [kv units][rows_total][D]
  __nv_bfloat16* o;
  float* lse;
  float* o_part;                      // [units][max_seg][nq_rows][D]
  float* lse_part;                    // [units][max_seg][nq_rows]
  int* nseg;                          // [units]
  int* status;
  const int32_t* seq_lens;
  PageTable pages;
  int box_shift;                      // log2 of a box's rows
  int batch, h_kv, n_q, nq_rows, rows_total, row_chunks, t_ctx;
  int max_seg, seg_cost, tiles_per_unit, vtiles_per_cta;
  float scale_log2;
};

template <int D, int NT>
struct PagedSmem {
  static constexpr int NQC = 8 * NT;
  static constexpr uint32_t TILE = kPvKeys * D * 2;
  static constexpr uint32_t STAGE = 2 * TILE;                      // K, V
  static constexpr size_t kMerge = (size_t)(2 * kPvWarps * NQC) * 4 + (size_t)kPvWarps * NQC * (D + 4) * 4;
  // alignment, barriers and the poison table, stages, merge scratch; then the sequences' table
  static constexpr size_t kTotal = 1024 + 1024 + (size_t)kPvStages * STAGE + kMerge;
};

template <int D, int NT>
__global__ void __launch_bounds__(kPvThreads) paged_verify_kernel(const __grid_constant__ PagedVerifyParams p,
                                                                  const __grid_constant__ CUtensorMap kmap,
                                                                  const __grid_constant__ CUtensorMap vmap) {
  using L = PagedSmem<D, NT>;
  constexpr int NQC = L::NQC, STAGES = kPvStages, NCT = 32 * kPvWarps;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem);
  uint64_t* empty_bar = full_bar + STAGES;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(empty_bar + STAGES);
  int* stop_flag = const_cast<int*>(abort_flag) + 1;
  int* hide_s = stop_flag + 1;                             // [STAGES] 16-key sub-tiles that are not there
  int* nan_from = reinterpret_cast<int*>(smem + 512);      // [D] first row of the block (from 1 on) whose V is no number there
  uint8_t* stage_base = smem + 1024;
  float* m_s = reinterpret_cast<float*>(stage_base + STAGES * L::STAGE);
  float* l_s = m_s + kPvWarps * NQC;
  float* o_s = l_s + kPvWarps * NQC;
  int* pref = reinterpret_cast<int*>(reinterpret_cast<uint8_t*>(m_s) + L::kMerge);   // [batch + 1]

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], kPvWarps);
    }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_map(&kmap);
    tma_prefetch_map(&vmap);
  }
  if (tid < D) nan_from[tid] = INT_MAX;
  grid_dependency_wait();
  allow_dependent_launch();
  PagedMap map{nullptr, p.tiles_per_unit + p.seg_cost, p.seg_cost, p.h_kv * p.row_chunks, p.batch, p.vtiles_per_cta};
  if (p.seq_lens) {
    map.lay_out<kPvThreads, kPvKeys>(p.seq_lens, p.t_ctx, p.n_q, p.vtiles_per_cta, reinterpret_cast<int*>(smem + 256), pref);
  } else {
    __syncthreads();
  }
  const int v_total = map.seq_base(p.batch);
  const int v0 = min(v_total, (int)blockIdx.x * map.vtpc), v1 = min(v_total, v0 + map.vtpc);
  if (v0 >= v1) return;
  const int u_first = map.unit_of(v0), u_last = map.unit_of(v1 - 1);

  if (warp == kPvWarps) {
    // ------------------------------------------------------------------ producer
    fence_proxy_async_global();
    // A tile is n_box pieces (a page's rows, or 64 of them) of K and of V; lane (tensor, piece) fetches one.  The entries of 32
    // pieces are looked up at once, the next 32 while these are used: one tile's at a time, a CTA's first tiles came a
    // round trip to memory apart.
    const int n_box = kPvKeys >> p.box_shift, piece = lane & (n_box - 1), which = lane / n_box;
    const uint32_t piece_bytes = (uint32_t)D * 2 << p.box_shift;
    const int page_mask = (1 << p.pages.shift) - 1;
    int issued = 0;
    bool ok = true;
    for (int unit = u_first; unit <= u_last && ok; ++unit) {
      const int tb = map.first_tile(unit, v0), n = map.end_tile(unit, v1) - tb;
      if (n <= 0) continue;
      const int seq = map.seq_of(unit), head = unit / p.row_chunks - seq * p.h_kv;
      const int end = paged_context(p.seq_lens, seq, p.t_ctx, nullptr) + p.n_q;   // rows of the sequence, its block's among them
      auto look_up = [&](int first) {                      // entry of the segment's piece first + lane
        const int at = first + lane, key = tb * kPvKeys + (at << p.box_shift);
        return at < n * n_box && key < end ? p.pages.entry(seq, key) : -1;
      };
      int now = look_up(0), then = look_up(32);
      for (int i = 0; i < n; ++i) {
        const int at = i * n_box;
        if (i > 0 && (at & 31) == 0) {
          now = then;
          then = look_up(at + 32);
        }
        const int entry = __shfl_sync(0xffffffffu, now, (at & 31) + piece);
        const int s = issued % STAGES;
        if (issued >= STAGES) ok = mbar_wait_warp(&empty_bar[s], ((issued / STAGES) & 1) ^ 1, p.status, abort_flag);
        if (!ok) break;
        const bool there = p.pages.there(entry);
        if (entry >= p.pages.n_pages) record_error(p.status, BD_ERR_INVALID_ARG);
        const uint32_t pieces = __ballot_sync(0xffffffffu, there) & ((1u << n_box) - 1);
        if (lane == 0) {
          int hide = 0;
#pragma unroll
          for (int sub = 0; sub < kPvWarps; ++sub) hide |= (int)(~pieces >> (16 * sub >> p.box_shift) & 1) << sub;
          hide_s[s] = hide;
          if (pieces) mbar_arrive_expect_tx(&full_bar[s], 2 * __popc(pieces) * piece_bytes);
          else mbar_arrive(&full_bar[s]);
        }
        __syncwarp();
        if (there && which < 2)
          tma_load_page(stage_base + s * L::STAGE + which * L::TILE + piece * piece_bytes, which ? &vmap : &kmap, &full_bar[s],
                        ((tb + i) * kPvKeys + (piece << p.box_shift)) & page_mask, 0, head, entry);
        __syncwarp();
        ++issued;
      }
    }
    if (*abort_flag && lane == 0) {      // never leave a copy in flight behind an aborted CTA
      for (int t = max(0, issued - STAGES); t < issued; ++t)
        mbar_wait(&full_bar[t % STAGES], (t / STAGES) & 1, p.status, nullptr);
    }
    return;
  }

  // -------------------------------------------------------------------- consumers
  const int gid = lane >> 2, tig = lane & 3;
  // where this warp's 16 keys lie in a tile
  const uint32_t half_bytes = 128u << p.box_shift;
  const int my_piece = 16 * warp >> p.box_shift;
  const uint32_t sub_off = my_piece * ((uint32_t)D * 2 << p.box_shift) + (16 * warp - (my_piece << p.box_shift)) * 128;
  uint32_t bq[NT][D / 16][2];
  auto load_q = [&](int unit) {
    const int kv_unit = unit / p.row_chunks, row_base = (unit - kv_unit * p.row_chunks) * p.nq_rows;
    const int rows = min(p.nq_rows, p.rows_total - row_base);
    const __nv_bfloat16* q = p.q + ((size_t)kv_unit * p.rows_total + row_base) * D;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = 8 * nt + gid;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          bq[nt][ks][h] = row < rows ? __ldcg(reinterpret_cast<const uint32_t*>(q + row * D + 16 * ks + 2 * tig + 8 * h)) : 0u;
    }
  };
  auto next_unit = [&](int u) {
    while (u <= u_last && map.first_tile(u, v0) >= map.end_tile(u, v1)) ++u;
    return u;
  };
  int lim[NT][2];                                          // last visible key of each of this thread's columns
  bool alive = true;
  int t = 0;
  int unit = next_unit(u_first);
  if (unit <= u_last) load_q(unit);
  while (unit <= u_last) {
    const int tb = map.first_tile(unit, v0), te = map.end_tile(unit, v1);
    const int kv_unit = unit / p.row_chunks, row_base = (unit - kv_unit * p.row_chunks) * p.nq_rows;
    const int rows = min(p.nq_rows, p.rows_total - row_base);
    const int t_unit = paged_context(p.seq_lens, map.seq_of(unit), p.t_ctx, tid == 0 ? p.status : nullptr);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int col = 8 * nt + 2 * tig + e;
        lim[nt][e] = col < rows ? t_unit + (row_base + col) % p.n_q : -1;
      }
    WarpAttn<D, NT> wa;
    wa.init();
    for (int tile = tb; tile < te; ++tile, ++t) {
      const int s = t % STAGES;
      if (!mbar_wait(&full_bar[s], (t / STAGES) & 1, p.status, abort_flag)) {
        alive = false;
        break;
      }
      const int key_base = tile * kPvKeys + 16 * warp, last = t_unit + p.n_q - 1 - key_base;   // last: the sub-tile's last row of the block
      if (!(hide_s[s] >> warp & 1) && last >= 0) {
        const uint32_t kbase = smem_u32(stage_base + s * L::STAGE) + sub_off, vbase = kbase + L::TILE;
        // rows of the block behind its first one, which its first query does not see
        const int block0 = max(0, t_unit + 1 - key_base);
        if (block0 <= min(last, 15)) scrub_rows<D>(vbase, p.box_shift, block0, min(last, 15) + 1, key_base + block0 - t_unit, nan_from, lane);
        wa.step(kbase, vbase, half_bytes, 0, bq, p.scale_log2, lane, [&](int ko, int nt, int e) { return key_base + ko <= lim[nt][e]; },
                last);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty_bar[s]);
    }
    // the next unit's queries arrive while this segment closes
    const int next = next_unit(unit + 1);
    if (next <= u_last && alive) load_q(next);
    wa.finish_rows();

    // ---------------------------------------------------------------- end of a segment
    wa.store(m_s, l_s, o_s, warp, NQC, 0, lane);
    named_bar(1, NCT);
    const int c_first = map.owner(unit, 0), n_seg = map.owner(unit, map.tiles(unit) - 1) - c_first + 1;
    const bool whole = n_seg == 1;
    if (p.max_seg > 1 && (int)blockIdx.x == c_first && tid == 0) p.nseg[unit] = n_seg;
    const size_t slot = ((size_t)unit * p.max_seg + ((int)blockIdx.x - c_first)) * p.nq_rows;
    const size_t orow = (size_t)kv_unit * p.rows_total + row_base;
    for (int i = tid; i < rows * (D / 4); i += NCT) {
      const int r = i / (D / 4), d = i % (D / 4) * 4;
      float mw[kPvWarps], M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kPvWarps; ++w) {
        mw[w] = m_s[w * NQC + r];
        M = fmaxf(M, mw[w]);
      }
      const float M_use = M == -INFINITY ? 0.f : M;
      float sum = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kPvWarps; ++w) {
        const float f = fast_exp2(mw[w] - M_use);
        const float4 v = *reinterpret_cast<const float4*>(o_s + (size_t)(w * NQC + r) * (D + 4) + d);
        sum = fmaf(f, l_s[w * NQC + r], sum);
        a[0] = fmaf(f, v.x, a[0]);
        a[1] = fmaf(f, v.y, a[1]);
        a[2] = fmaf(f, v.z, a[2]);
        a[3] = fmaf(f, v.w, a[3]);
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;      // (a NaN stays one)
      const int qi = (row_base + r) % p.n_q;
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = qi >= nan_from[d + e] ? NAN : a[e] * inv;
      const float lse = sum == 0.f ? -INFINITY : (M_use + log2f(sum)) * kLn2;
      if (whole) {
        *reinterpret_cast<uint2*>(p.o + (orow + r) * D + d) = make_uint2(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]));
        if (d == 0 && p.lse) p.lse[orow + r] = lse;
      } else {
        *reinterpret_cast<float4*>(p.o_part + (slot + r) * D + d) = make_float4(a[0], a[1], a[2], a[3]);
        if (d == 0) p.lse_part[slot + r] = lse;
      }
    }
    named_bar(1, NCT);                                     // scratch and poison free for the next segment
    if (tid < D) nan_from[tid] = INT_MAX;
    if (tid == 0) *stop_flag = *abort_flag;
    named_bar(1, NCT);
    if (*stop_flag) break;
    unit = next;
  }
}

// ============================================================================ host side

namespace {

struct PvInfo {
  const void* fn;
  size_t smem;
};
PvInfo pv_kernel(int d, int nt) {
#define BD_PV(DD, N) \
  if (d == DD && nt == N) return {reinterpret_cast<const void*>(&paged_verify_kernel<DD, N>), PagedSmem<DD, N>::kTotal};
  BD_PV(64, 1) BD_PV(64, 3) BD_PV(128, 1) BD_PV(128, 3)
#undef BD_PV
  return {nullptr, 0};
}

// CTAs an SM holds, by shared memory (228 KB, a CTA taking 1 KB more than it asks for).
int pv_per_sm(size_t smem) { return std::max(1, (int)(228 * 1024 / (smem + 1024))); }

// Which kernel takes this many query rows of a KV head, and in which chunks.
void pv_rows(int rows, bool tc, PagedVerifyPlan* plan) {
  const int most = tc ? kPvTcMaxRows : kPvMaxRows;
  plan->chunks = (rows + most - 1) / most;
  plan->nq_rows = (rows + plan->chunks - 1) / plan->chunks;
  plan->q_tiles = tc ? (plan->nq_rows > 128 ? 2 : 1) : 0;
  plan->nt = tc ? 0 : plan->nq_rows <= 8 ? 1 : 3;
}
size_t pv_smem(const bd_shape& s, const PagedVerifyPlan& plan) {
  return plan.q_tiles ? verify_tc_smem(s.head_dim, plan.q_tiles) + (16 + s.head_dim) * 4 : pv_kernel(s.head_dim, plan.nt).smem;
}
long pv_ctas(const PagedVerifyPlan& plan, size_t smem) {
  return (long)std::max(1, current_sm_count()) * (plan.q_tiles ? 1 : pv_per_sm(smem));
}

}  // namespace

bool paged_verify_plan(const bd_shape& s, int rows, int n_q, PagedVerifyPlan* plan) {
  const bool tc = rows > kPvMaxRows;
  pv_rows(rows, tc, plan);
  plan->smem = pv_smem(s, *plan);
  const int keys = tc ? kVTcKeys : kPvKeys;
  const long units = (long)s.batch * s.h_kv * plan->chunks, ctas = pv_ctas(*plan, plan->smem);
  const long tpu = ((long)s.t_ctx + n_q + keys - 1) / keys;
  // A segment's end and the next one's start cost about 5 us of streaming (as in verify_plan), charged as virtual tiles.
  const double tile_us = (double)keys * s.head_dim * 4 / (6.5e6 / std::max(1, current_sm_count()));
  const long a = (long)std::min(16.0, std::max(0.0, 5.0 / tile_us + 0.5));
  const long vtotal = units * (tpu + a);
  if (vtotal >= 1L << 30) return false;
  const long least = (tpu + a + kVMaxSeg - 2) / (kVMaxSeg - 1);     // <= kVMaxSeg segments
  const long vtpc = std::max((vtotal + ctas - 1) / ctas, least);
  plan->tiles_per_unit = (int)tpu;
  plan->seg_cost = (int)a;
  plan->grid = (int)((vtotal + vtpc - 1) / vtpc);
  if (s.seq_lens) {
    // the kernel cuts the ranges itself over the actual tiles
    plan->tiles_per_cta = (int)least;
    plan->max_seg = kVMaxSeg;
    plan->smem += align_up((size_t)(s.batch + 1) * 4, 16);
    return plan->smem <= kMaxSmem;
  }
  plan->tiles_per_cta = (int)vtpc;
  // a run of tpu tiles crosses no more borders than this; none where every range holds whole units
  plan->max_seg = vtpc % (tpu + a) == 0 ? 1 : (int)std::min<long>(kVMaxSeg, (tpu + vtpc - 2) / vtpc + 1);
  return true;
}

size_t paged_verify_bytes(const bd_shape& s, const PagedVerifyPlan& plan) {
  if (plan.max_seg <= 1) return 0;
  const size_t units = (size_t)s.batch * s.h_kv * plan.chunks, rows = units * plan.max_seg * plan.nq_rows;
  return align_up(rows * s.head_dim * 4, 256) + align_up(rows * 4, 256) + align_up(units * 4, 256);
}

size_t paged_verify_room(const bd_shape& s, int rows) {
  // A unit's tpu tiles lie in at most ceil((tpu - 1) / vtpc) + 1 ranges of vtpc >= units (tpu + a) / ctas.
  PagedVerifyPlan plan = {};
  pv_rows(rows, rows > kPvMaxRows, &plan);
  const long units = (long)s.batch * s.h_kv * plan.chunks, ctas = pv_ctas(plan, pv_smem(s, plan));
  plan.max_seg = s.seq_lens ? kVMaxSeg : (int)std::min<long>(kVMaxSeg, (ctas + units - 1) / units + 1);
  return paged_verify_bytes(s, plan);
}

cudaError_t launch_paged_verify(const bd_shape& s, const PagedVerifyPlan& plan, int rows, int n_q, const void* q,
                                const bd_paged_cache& c, const int32_t* table, int table_pages, void* o_out, float* lse_out,
                                void* ws_region, int* status, cudaStream_t stream) {
  const bool tc = plan.q_tiles != 0;
  // (tcgen05: a K tile's operand is halves of 128 rows, so a box is one half of a piece's rows.  Boxes of 16 rows so are too
  // many: 64 units of 16K, 32 rows, d 128 112.9 us in pages of 16, 93.4 in larger ones.  Those take both halves.)
  const bool box16 = tc && c.page_size == 16 && s.head_dim == 128;
  const int box = std::min<int>(c.page_size, tc ? kVTcKeys : kPvKeys), halves = tc && !box16 ? 1 : s.head_dim / 64;
  CUtensorMap kmap, vmap;
  cudaError_t err = make_paged_map(&kmap, c.k, c.k_strides, s.head_dim, s.h_kv, c.page_size, c.n_pages, box, halves);
  if (err == cudaSuccess) err = make_paged_map(&vmap, c.v, c.v_strides, s.head_dim, s.h_kv, c.page_size, c.n_pages, box, halves);
  if (err != cudaSuccess) return err;
  const PageTable pages = {table, table_pages, c.n_pages, page_shift(c)};
  int box_shift = 0;
  while (1 << box_shift < box) ++box_shift;
  const int units = s.batch * s.h_kv * plan.chunks;
  const size_t part_rows = (size_t)units * plan.max_seg * plan.nq_rows;
  // what the two kernels' parameters have in common
  auto fill = [&](auto& p) {
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.o = static_cast<__nv_bfloat16*>(o_out);
    p.lse = lse_out;
    p.o_part = static_cast<float*>(ws_region);
    p.lse_part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws_region) + align_up(part_rows * s.head_dim * 4, 256));
    p.nseg = reinterpret_cast<int*>(reinterpret_cast<uint8_t*>(p.lse_part) + align_up(part_rows * 4, 256));
    p.status = status;
    p.seq_lens = s.seq_lens;
    p.pages = pages;
    p.box_shift = box_shift;
    p.batch = s.batch;
    p.h_kv = s.h_kv;
    p.n_q = n_q;
    p.nq_rows = plan.nq_rows;
    p.rows_total = rows;
    p.row_chunks = plan.chunks;
    p.t_ctx = s.t_ctx;
    p.max_seg = plan.max_seg;
    p.seg_cost = plan.seg_cost;
    p.tiles_per_unit = plan.tiles_per_unit;
    p.vtiles_per_cta = plan.tiles_per_cta;
    p.scale_log2 = kLog2e / sqrtf((float)s.head_dim);
  };
  if (tc) {
    PagedTcParams p;
    fill(p);
    p.counters = nullptr;
    p.units = units;
    p.tile_rows = plan.q_tiles == 2 ? (plan.nq_rows + 1) / 2 : plan.nq_rows;
    CUtensorMap qmap;
    err = make_rows_map(&qmap, q, (long long)s.batch * s.h_kv * rows, s.head_dim, 128);
    const void* fn = paged_tc_fn(s.head_dim, plan.q_tiles, box16);
    if (err == cudaSuccess) err = allow_shared_memory(fn);
    if (err != cudaSuccess) return err;
    void* args[] = {&p, &kmap, &vmap, &qmap};
    err = launch_kernel(fn, dim3(plan.grid), dim3(kVTcThreads), plan.smem, stream, args, 0);
    if (err != cudaSuccess || plan.max_seg <= 1) return err;
    return launch_verify_tc_merge(s.head_dim, units, p, stream, true);
  }
  PagedVerifyParams p;
  fill(p);
  const PvInfo k = pv_kernel(s.head_dim, plan.nt);
  err = allow_shared_memory(k.fn);
  if (err != cudaSuccess) return err;
  void* args[] = {&p, &kmap, &vmap};
  err = launch_kernel(k.fn, dim3(plan.grid), dim3(kPvThreads), plan.smem, stream, args, 0);
  if (err != cudaSuccess || plan.max_seg <= 1) return err;
  return launch_row_merge(s.head_dim, {p.o_part, p.lse_part, p.nseg, plan.max_seg, plan.nq_rows, rows, plan.chunks, units, o_out, lse_out}, stream);
}

}  // namespace bd
