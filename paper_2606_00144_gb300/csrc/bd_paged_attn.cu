// Verify blocks, and decoding one token, over a paged cache (bd_paged_verify_attn): n_q queries per head at positions
// T .. T + n_q - 1 over the keys of [0, T + i] whose pages are there.
//
//   o_i = sum_k 2^(s_ik - M) v_k / sum_k 2^(s_ik - M),  s = q k log2(e) / sqrt(d)
//
// One pass over K and V with a running maximum and sum, in 64-key tiles.  Two producer warps fetch a tile's pieces of K and of
// V (a page's rows of the tile, each one TMA box of whole rows); the consumer warps take 16 keys of it each on mma.sync
// (bd_attn_warp.cuh), the query rows on the N side.  The pieces of a tile lie one behind the other, so a warp's 16 keys are in
// one piece (pages hold at least 16 rows).  Pieces whose page is not there, or that lie past the sequence's block, are not
// fetched, and their keys are passed over.
//   cluster  a unit's tiles (a unit: a sequence's KV head, and up to 8 of its query rows) are taken in turn by the CTAs
//            of a cluster, or go to one CTA.  For short units, and for many, which the hardware deals out.
//   stream   the (unit, tile) pairs of all units form one list, cut into contiguous ranges of equal cost, one per CTA; each
//            piece of a unit ("segment") ends in a partial, and a second kernel joins those of units that span CTAs.  For
//            few long units.
// More than 8 query rows of long units (24 at d 64) are the tcgen05 kernel's (bd_verify_tc.cu, PAGED).
//
// Bound by HBM where there is enough to read: 256 units of 1.6K to 8K (630 MB) take 92 us (6.8 TB/s), 256 of 4K 78 (6.9), 8
// of 128K 83.1 (6.5: a start of some 5 us, of which the page's look-up and the first tile are 4, and an end of 5), in pages of
// 16 as in larger ones.  Short calls are a chain of latencies: 8 units of 1K 5.3 us, 2 of 1K (d 64) 3.9.
#include <cooperative_groups.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "bd_attn_warp.cuh"
#include "bd_internal.h"
#include "bd_paged.cuh"
#include "bd_verify.cuh"

namespace cg = cooperative_groups;

namespace bd {

constexpr int kPvKeys = 64;           // keys of a tile
constexpr int kPvSubs = kPvKeys / 16; // a warp's sub-tiles
constexpr int kPvStages = 5;          // tiles in flight of a stream
constexpr int kPvMaxStages = 12;      // and at most
constexpr int kPvCluster = 8;         // most CTAs of a cluster (the portable size)
constexpr int kPvTcMaxRows = 256;     // query rows of a unit of the tcgen05 kernel: two M tiles

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
  int stages;                         // of a cluster's CTA
  float scale_log2;
};

// A cluster's unit: its CTAs take its tiles in turn, so that what is left of a context behind a window is spread over all of them.
struct ClusterMap {
  int per_seq;
  __device__ __forceinline__ int stride() const { return gridDim.x; }
  __device__ __forceinline__ int seq_of(int u) const { return u / per_seq; }
  __device__ __forceinline__ int first_tile(int, int v0) const { return v0; }
  __device__ __forceinline__ int end_tile(int, int v1) const { return v1; }
};

template <int D, int NT, bool CLUSTER>
struct PagedSmem {
  static constexpr int NQC = 8 * NT;
  static constexpr int WARPS = CLUSTER ? 6 : 4, THREADS = 32 * WARPS + 64;   // consumers, and two producers
  static constexpr uint32_t TILE = kPvKeys * D * 2;
  static constexpr uint32_t STAGE = 2 * TILE;                      // K, V
  static constexpr uint32_t kMerge = (2 * WARPS * NQC) * 4 + WARPS * NQC * (D + 4) * 4;
  // the stages and the warps' states (CLUSTER: the latter over the former)
  __host__ __device__ static constexpr uint32_t area(int stages) {
    return CLUSTER ? (stages * STAGE > kMerge ? stages * STAGE : kMerge) : stages * STAGE + kMerge;
  }
  // alignment, barriers and the poison table, the area; then the sequences' table, or the cluster's parts
  static size_t bytes(int stages) { return 1024 + 1024 + area(stages); }
  // CLUSTER: CTA k of a unit's C merges rows k, k + C, ... of every CTA's part
  __host__ __device__ static constexpr int slot_rows(int C) { return (NQC + C - 1) / C; }
  static size_t slots(int C) { return (size_t)C * slot_rows(C) * (D + 1) * 4; }
};

// CLUSTER: a unit's tiles are split over the CTAs of a cluster, which meet in shared memory: no partials, no second launch; six
// warps take the sub-tiles in turn.
template <int D, int NT, bool CLUSTER>
__global__ void __launch_bounds__(PagedSmem<D, NT, CLUSTER>::THREADS, CLUSTER || D == 64 ? 2 : 1)
    paged_verify_kernel(const __grid_constant__ PagedVerifyParams p, const __grid_constant__ CUtensorMap kmap,
                        const __grid_constant__ CUtensorMap vmap) {
  using L = PagedSmem<D, NT, CLUSTER>;
  constexpr int NQC = L::NQC, WARPS = L::WARPS, NCT = 32 * WARPS;
  constexpr bool kSkips = CLUSTER || NT > 1;               // tiles that are not there are passed over
  const int stages = CLUSTER ? p.stages : kPvStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem);
  uint64_t* empty_bar = full_bar + kPvMaxStages;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(empty_bar + kPvMaxStages);
  int* stop_flag = const_cast<int*>(abort_flag) + 1;
  int* hide_s = stop_flag + 1;                             // [stages] 16-key sub-tiles that are not there; the tiles passed over before
  int* nan_from = reinterpret_cast<int*>(smem + 512);      // [D] first row of the block (from 1 on) whose V is no number there
  uint8_t* stage_base = smem + 1024;
  float* m_s = reinterpret_cast<float*>(stage_base + (CLUSTER ? 0 : stages * L::STAGE));
  float* l_s = m_s + WARPS * NQC;
  float* o_s = l_s + WARPS * NQC;
  int* pref = reinterpret_cast<int*>(stage_base + L::area(stages));   // [batch + 1]

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (CLUSTER) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // this CTA has started
  if (tid == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(&full_bar[s], 2);
      mbar_init(&empty_bar[s], WARPS);
    }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_map(&kmap);
    tma_prefetch_map(&vmap);
  }
  if (tid < D) nan_from[tid] = INT_MAX;
  if (CLUSTER) {   // the sequence's entries and the queries on their way into L2 while the kernel before ends
    const int seq = (int)blockIdx.y / (p.h_kv * p.row_chunks), pages = min(p.pages.pages, ((p.t_ctx + p.n_q - 1) >> p.pages.shift) + 1);
    prefetch_lines_l2(p.pages.table + (size_t)seq * p.pages.pages, min(pages, 2048) * sizeof(int32_t), tid, L::THREADS);
    prefetch_lines_l2(p.q + (size_t)(blockIdx.y / p.row_chunks) * p.rows_total * D, (size_t)p.rows_total * D * 2, tid, L::THREADS);
  }
  using Map = std::conditional_t<CLUSTER, ClusterMap, PagedMap>;
  using Walk = PageWalk<kPvKeys, Map, PagedVerifyParams>;
  Map map;
  int v0, v1, u_first, u_last;                             // this CTA's range of tiles, its units
  typename Walk::Segment seg{};                            // the producers' first
  auto plan = [&] {
    if constexpr (CLUSTER) {
      u_first = u_last = blockIdx.y;
      map.per_seq = p.h_kv * p.row_chunks;
      const int t = paged_context(p.seq_lens, map.seq_of(u_first), p.t_ctx, nullptr);
      v0 = blockIdx.x;
      v1 = (t + p.n_q + kPvKeys - 1) / kPvKeys;
    } else {
      map = PagedMap{nullptr, p.tiles_per_unit + p.seg_cost, p.seg_cost, p.h_kv * p.row_chunks, p.batch, p.vtiles_per_cta};
      if (p.seq_lens) map.template lay_out<L::THREADS, kPvKeys>(p.seq_lens, p.t_ctx, p.n_q, p.vtiles_per_cta, reinterpret_cast<int*>(smem + 256), pref);
      const int v_total = map.seq_base(p.batch);
      v0 = min(v_total, (int)blockIdx.x * map.vtpc);
      v1 = min(v_total, v0 + map.vtpc);
      if (v0 < v1) {
        u_first = map.unit_of(v0);
        u_last = map.unit_of(v1 - 1);
      }
    }
    if ((CLUSTER || v0 < v1) && warp >= WARPS) seg = Walk{map, p, u_last, v0, v1}.from(u_first);
  };
  if (!p.seq_lens) plan();                                 // (as much as can be before the wait)
  __syncthreads();
  grid_dependency_wait();
  allow_dependent_launch();
  if (p.seq_lens) plan();
  if (!CLUSTER && v0 >= v1) return;
  // the producers' first look-ups, whose round trip is the longest thing before the first tile
  const Walk walk{map, p, u_last, v0, v1};
  int now = -1, then = -1;
  if (warp >= WARPS) {
    now = walk.entry(seg, 0, lane);
    then = walk.entry(seg, 32, lane);
  }

  if (warp >= WARPS) {
    // ------------------------------------------------------------------ producers: K, V
    fence_proxy_async_global();
    // A tile is n_box pieces of K and of V; a lane fetches one, which takes a warp some 130 cycles a piece, so K and V have a warp
    // each (both in one: 0.55 us a tile in pages of 16, whatever the consumers do).  Entries are looked up 32 pieces, and the
    // next segment's, ahead: a tile at a time, a CTA's first tiles came a round trip to memory apart.
    const int which = warp - WARPS, n_box = kPvKeys >> p.box_shift, piece = lane & (n_box - 1);
    const uint32_t piece_bytes = (uint32_t)D * 2 << p.box_shift;
    const int page_mask = (1 << p.pages.shift) - 1;
    const CUtensorMap* my_map = which ? &vmap : &kmap;
    int issued = 0, s = 0;
    uint32_t phase = 1;                                    // of the stage's last use (its first waits for none)
    bool ok = true;
    while (seg.unit <= u_last && ok) {
      auto next = seg;
      int next_now = -1, next_then = -1, skipped = 0;
      for (int i = 0; i < seg.n; ++i) {
        const int at = i * n_box & 31;
        if (i > 0 && at == 0) {
          now = then;
          then = walk.entry(seg, i * n_box + 32, lane);
        }
        const int entry = __shfl_sync(0xffffffffu, now, at + piece);
        const uint32_t pieces = __ballot_sync(0xffffffffu, p.pages.there(now)) >> at & ((1u << n_box) - 1);
        if (entry >= p.pages.n_pages) record_error(p.status, BD_ERR_INVALID_ARG);
        // Nothing of it is there (a segment's last tile stands for its end).  256 units of 8K behind a window of 1K, one row: 39.3 us,
        // 57 without; 64 of 16K, d 64, 16 rows, a window of 500: 20.4 / 27.9.  Not in a stream of few rows, whose ranges hold as many
        // tiles with a window as without: 8 units of 64K, a window of 4K 34.1 / 33.6, and the check costs 4 % at d 64.
        if (kSkips && pieces == 0 && i + 1 < seg.n) {
          ++skipped;
          continue;
        }
        if (issued >= stages) ok = mbar_wait_warp(&empty_bar[s], phase, p.status, abort_flag);
        if (!ok) break;
        if (lane == 0) {
          if (which == 0) {
            int hide = 0;
#pragma unroll
            for (int sub = 0; sub < kPvSubs; ++sub) hide |= (int)(~pieces >> (16 * sub >> p.box_shift) & 1) << sub;
            hide_s[s] = skipped << kPvSubs | hide;
          }
          if (pieces) mbar_arrive_expect_tx(&full_bar[s], __popc(pieces) * piece_bytes);
          else mbar_arrive(&full_bar[s]);
        }
        __syncwarp();
        if (p.pages.there(entry) && lane < n_box)
          tma_load_page(1, smem_u32(stage_base + s * L::STAGE + which * L::TILE) + piece * piece_bytes, my_map, &full_bar[s],
                        ((seg.tb + i * map.stride()) * kPvKeys + (piece << p.box_shift)) & page_mask, 0, seg.head, entry);
        __syncwarp();
        skipped = 0;
        ++issued;
        if (++s == stages) s = 0, phase ^= 1;
        if (next.unit == seg.unit) {                       // (behind the first tile)
          if (CLUSTER) {
            next.unit = u_last + 1;
          } else {
            next = walk.from(seg.unit + 1);
            next_now = walk.entry(next, 0, lane);
            next_then = walk.entry(next, 32, lane);
          }
        }
      }
      seg = next;
      now = next_now;
      then = next_then;
    }
    if (*abort_flag && lane == 0) {      // never leave a copy in flight behind an aborted CTA
      for (int t = max(0, issued - stages); t < issued; ++t)
        mbar_wait_for(&full_bar[t % stages], (t / stages) & 1, p.status, nullptr, 20000000);   // (the other producer may have stopped before)
    }
    if constexpr (CLUSTER) {             // (its part in the consumers' two barriers)
      __syncwarp();
      asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
      asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    return;
  }

  // -------------------------------------------------------------------- consumers
  const int gid = lane >> 2, tig = lane & 3;
  const uint32_t half_bytes = 128u << p.box_shift;
  auto offset_of = [&](int sub) {                          // where a sub-tile lies in a tile
    const int at = 16 * sub >> p.box_shift;
    return at * ((uint32_t)D * 2 << p.box_shift) + (16 * sub - (at << p.box_shift)) * 128;
  };
  const uint32_t own_off = offset_of(warp);                // (a stream's warp always takes the same one)
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
  auto next_unit = [&](int u) {                            // (CLUSTER: the unit, also where this CTA has no tile of it)
    while (!CLUSTER && u <= u_last && map.first_tile(u, v0) >= map.end_tile(u, v1)) ++u;
    return u;
  };
  int lim[NT][2];                                          // last visible key of each of this thread's columns
  bool alive = true;
  int s = 0;                                               // the next tile's stage, and its phase
  uint32_t phase = 0;
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
    for (int tile = tb, nth = 0; tile < te; ++nth, tile += map.stride()) {
      if (!mbar_wait(&full_bar[s], phase, p.status, abort_flag)) {
        alive = false;
        break;
      }
      // CLUSTER: sub-tiles go round the warps, at most one of a tile to each; some warps have none
      const int sub = CLUSTER ? (warp - kPvSubs * nth % WARPS + WARPS) % WARPS : warp, hide = hide_s[s];
      if (kSkips) tile += (hide >> kPvSubs) * map.stride();
      const int key_base = tile * kPvKeys + 16 * sub, last = t_unit + p.n_q - 1 - key_base;   // last: the sub-tile's last row of the block
      if ((!CLUSTER || sub < kPvSubs) && !(hide >> sub & 1) && last >= 0) {
        const uint32_t kbase = smem_u32(stage_base + s * L::STAGE) + (CLUSTER ? offset_of(sub) : own_off), vbase = kbase + L::TILE;
        // rows of the block behind its first one, which its first query does not see
        const int block0 = max(0, t_unit + 1 - key_base);
        if (block0 <= min(last, 15)) scrub_rows<D>(vbase, p.box_shift, block0, min(last, 15) + 1, key_base + block0 - t_unit, nan_from, lane);
        wa.step(kbase, vbase, half_bytes, 0, bq, p.scale_log2, lane, [&](int ko, int nt, int e) { return key_base + ko <= lim[nt][e]; },
                last);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty_bar[s]);
      if (++s == stages) s = 0, phase ^= 1;
    }
    // the next unit's queries arrive while this segment closes
    const int next = next_unit(unit + 1);
    if (next <= u_last && alive) load_q(next);
    wa.finish_rows();

    // ---------------------------------------------------------------- end of a segment
    if (CLUSTER) named_bar(1, NCT);                        // (every tile has been read)
    wa.store(m_s, l_s, o_s, warp, NQC, 0, lane);
    named_bar(1, NCT);
    bool whole = CLUSTER && gridDim.x == 1;
    size_t slot = 0;
    if constexpr (!CLUSTER) {
      const int c_first = map.owner(unit, 0), n_seg = map.owner(unit, map.tiles(unit) - 1) - c_first + 1;
      whole = n_seg == 1;
      if (p.max_seg > 1 && (int)blockIdx.x == c_first && tid == 0) p.nseg[unit] = n_seg;
      slot = ((size_t)unit * p.max_seg + ((int)blockIdx.x - c_first)) * p.nq_rows;
    }
    const int C = gridDim.x, slot_rows = L::slot_rows(C);
    float* slots = reinterpret_cast<float*>(pref);         // CLUSTER: [C][slot_rows][D], then [C][slot_rows] lse
    float* lses = slots + (size_t)C * slot_rows * D;
    if constexpr (CLUSTER) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");   // every CTA is running
    const size_t orow = (size_t)kv_unit * p.rows_total + row_base;
    for (int i = tid; i < rows * (D / 4); i += NCT) {
      const int r = i / (D / 4), d = i % (D / 4) * 4;
      float mw[WARPS], M = -INFINITY;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        mw[w] = m_s[w * NQC + r];
        M = fmaxf(M, mw[w]);
      }
      const float M_use = M == -INFINITY ? 0.f : M;
      float sum = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
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
      } else if constexpr (CLUSTER) {
        const int at = (int)blockIdx.x * slot_rows + r / C;
        cg::cluster_group cluster = cg::this_cluster();
        *reinterpret_cast<float4*>(cluster.map_shared_rank(slots + (size_t)at * D + d, r % C)) = make_float4(a[0], a[1], a[2], a[3]);
        if (d == 0) *cluster.map_shared_rank(lses + at, r % C) = lse;
      } else {
        *reinterpret_cast<float4*>(p.o_part + (slot + r) * D + d) = make_float4(a[0], a[1], a[2], a[3]);
        if (d == 0) p.lse_part[slot + r] = lse;
      }
    }
    if constexpr (CLUSTER) {
      __syncwarp();
      asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");   // all parts have landed
      for (int i = tid; !whole && i < slot_rows * (D / 4); i += NCT) {
        const int at = i / (D / 4), r = at * C + (int)blockIdx.x, d = i % (D / 4) * 4;
        if (r >= rows) break;
        float ls[kPvCluster], mx = -INFINITY, sum = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kPvCluster; ++k) {
          ls[k] = k < C ? lses[k * slot_rows + at] : -INFINITY;
          mx = fmaxf(mx, ls[k]);
        }
#pragma unroll
        for (int k = 0; k < kPvCluster; ++k) {
          if (k >= C || ls[k] == -INFINITY) continue;      // (a NaN stays one)
          const float f = fast_exp2((ls[k] - mx) * kLog2e);
          const float4 v = *reinterpret_cast<const float4*>(slots + ((size_t)k * slot_rows + at) * D + d);
          sum += f;
          a[0] = fmaf(f, v.x, a[0]);
          a[1] = fmaf(f, v.y, a[1]);
          a[2] = fmaf(f, v.z, a[2]);
          a[3] = fmaf(f, v.w, a[3]);
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<uint2*>(p.o + (orow + r) * D + d) = make_uint2(pack_bf16x2(a[0] * inv, a[1] * inv), pack_bf16x2(a[2] * inv, a[3] * inv));
        if (d == 0 && p.lse) p.lse[orow + r] = sum == 0.f ? -INFINITY : mx + logf(sum);
      }
      return;
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
  int threads;
  size_t (*bytes)(int stages);
  size_t (*slots)(int cluster);
  std::atomic<uint64_t>* allowed;
};
template <int D, int NT, bool CLUSTER>
PvInfo pv_one() {
  using L = PagedSmem<D, NT, CLUSTER>;
  static std::atomic<uint64_t> allowed{0};
  return {reinterpret_cast<const void*>(&paged_verify_kernel<D, NT, CLUSTER>), L::THREADS, &L::bytes, &L::slots, &allowed};
}
PvInfo pv_kernel(int d, int nt, bool cluster) {
  if (d == 64) return cluster ? pv_one<64, 1, true>() : nt == 1 ? pv_one<64, 1, false>() : pv_one<64, 3, false>();
  return cluster ? pv_one<128, 1, true>() : pv_one<128, 1, false>();
}

// A cluster's CTA: tiles in flight where it shares the SM with another one (96 KB).
int pv_half(int d) { return d == 128 ? 3 : 6; }

// Clusters of c CTAs that the device holds at once, one or two CTAs to an SM (a GPC's SMs are shared out by whole clusters).
// Asked once per instance and c; the device, once a plan (asked 24 times a plan, it was 0.7 of a call of 7 us).
class PvClusters {
 public:
  PvClusters(int d, int sms) : d_(d), sms_(sms) {
    static thread_local int cache_dev = -1;
    static thread_local int cache[2][2][kPvCluster + 1];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) {
      (void)cudaGetLastError();
      return;
    }
    if (dev != cache_dev) {
      std::fill_n(&cache[0][0][0], sizeof(cache) / sizeof(int), -1);
      cache_dev = dev;
    }
    held_ = cache[d == 128];
  }
  long operator()(int c, bool alone) const {
    const long guess = (alone ? 1L : 2L) * sms_ / c;
    if (!held_) return guess;
    int& held = held_[alone][c];
    if (held < 0) {
      const PvInfo k = pv_kernel(d_, 1, true);
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(c);
      cfg.blockDim = dim3(k.threads);
      cfg.dynamicSmemBytes = k.bytes(pv_half(d_) * (alone ? 2 : 1)) + k.slots(c);
      cudaLaunchAttribute at;
      at.id = cudaLaunchAttributeClusterDimension;
      at.val.clusterDim.x = (unsigned)c;
      at.val.clusterDim.y = at.val.clusterDim.z = 1;
      cfg.attrs = &at;
      cfg.numAttrs = 1;
      int n = 0;
      if (allow_shared_memory_once(k.fn, 0, k.allowed) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, k.fn, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();
        n = (int)guess;
      }
      held = n;
    }
    return held;
  }

 private:
  int d_, sms_;
  int (*held_)[kPvCluster + 1] = nullptr;
};

// CTAs an SM holds, by shared memory (228 KB, a CTA taking 1 KB more than it asks for).
int pv_per_sm(size_t smem) { return std::max(1, (int)(228 * 1024 / (smem + 1024))); }

// The kernel that takes this many query rows of a KV head as a stream, and in which chunks.  More than 8 rows are the tcgen05
// kernel's at head_dim 128 (64 units of 16K, 16 rows: 94.9 us, three n8 tiles 104.5; 24 rows 94.8 / 104.7; 256 units of 4K, 24
// rows 100 / 115), more than 24 at 64 (32 units of 1.6K to 8K each of 8 heads, 20 rows: 79 / 108; 64 units of 16K, 16 rows 59).
void pv_stream_rows(const bd_shape& s, int rows, PagedVerifyPlan* plan) {
  const int small = s.head_dim == 128 ? 8 : 24;
  const bool tc = rows > small;
  const int most = tc ? kPvTcMaxRows : small;
  plan->chunks = (rows + most - 1) / most;
  plan->nq_rows = (rows + plan->chunks - 1) / plan->chunks;
  plan->q_tiles = tc ? (plan->nq_rows > 128 ? 2 : 1) : 0;
  plan->nt = tc ? 0 : plan->nq_rows <= 8 ? 1 : 3;
  plan->cluster = plan->stages = 0;
  plan->smem = tc ? verify_tc_smem(s.head_dim, plan->q_tiles) + (16 + s.head_dim) * 4
                  : pv_kernel(s.head_dim, plan->nt, false).bytes(kPvStages);
  if (s.seq_lens) plan->smem += align_up((size_t)(s.batch + 1) * 4, 16);
}
long pv_ctas(const PagedVerifyPlan& plan) {
  return (long)std::max(1, current_sm_count()) * (plan.q_tiles ? 1 : pv_per_sm(plan.smem));
}

// Estimates of both routes in us, fitted to d 64 and 128, pages of 16, 1 to 64 sequences of 256 to 16K, 1 to 48 rows, equal and
// unequal lengths (those within a tenth or two).
//   stream   a start and an end, what a CTA's change of units costs, the bytes at the rate it reaches
//   cluster  4.2 for a wave's start and end; a tile is 0.48 (0.44) where a CTA has the SM to itself, 0.88 where two share it; the
//            SM's tiles, the bytes
// cluster / stream, d 128, one row: 8 units of 1K 5.6 / 7.5, of 8K 12.6 / 13.9; 32 units of 4K 15.7 / 17.7; 128 of 8K 81.2 / 88.0;
// 256 of 4K 82.2 / 89.3; 512 units of 0.4K to 4K 88.5 / 97.3; 16 rows, 8 units of 1K 6.3 / 11.3, 32 of 4K 19.9 / 24.4; 24 rows, 64
// units of 1K 17.3 / 21.4, of 4K 49.5 / 36.1.
struct PvWork {
  long units, tiles;           // (sequence, KV head) units; tiles of the longest
  double mb, share;            // MB of K and V at most; how much of it there is likely to be
};
PvWork pv_work(const bd_shape& s, int n_q) {
  PvWork w;
  w.units = (long)s.batch * s.h_kv;
  w.tiles = ((long)s.t_ctx + n_q + kPvKeys - 1) / kPvKeys;
  w.mb = (double)w.units * w.tiles * kPvKeys * s.head_dim * 4e-6;
  // (the host does not know the lengths.  Where they are all alike half is wrong, and the lay-out waits for them: 256 units of 4K 82.7 us,
  // 80.7 without lengths; 8 of 8K 15.4 / 11.8; 32 of 8K 28.2 / 24.2.)
  w.share = s.seq_lens ? 0.5 : 1.0;
  return w;
}
double pv_stream_us(const bd_shape& s, int rows, const PvWork& w) {
  const double per_sm = (double)w.units / current_sm_count(), mb = w.mb * w.share;
  const bool wide = s.head_dim == 128;
  if (rows <= 8) return 6.8 + 0.6 * per_sm + mb / (wide ? 6.2 : 5.5);
  if (!wide && rows <= 24) return 11.5 + 2.0 * per_sm + mb / 5.0;
  return 12.0 + 10.0 * per_sm * ((rows + kPvTcMaxRows - 1) / kPvTcMaxRows) + mb / (wide ? 6.2 : 4.2);
}

bool pv_cluster(const bd_shape& s, int rows, int n_q, PagedVerifyPlan* plan) {
  const PvWork w = pv_work(s, n_q);
  const long chunks = (rows + 7) / 8, groups = w.units * chunks, sms = std::max(1, current_sm_count());
  if (groups > 65535) return false;
  const double tile = s.head_dim == 128 ? 0.48 : 0.44;
  const PvClusters clusters_held(s.head_dim, (int)sms);
  double best = pv_stream_us(s, rows, w);
  int c = 0, stages = 0;
  for (int n = (int)std::min<long>(kPvCluster, w.tiles); n >= 1; --n) {
    const bool alone = groups <= clusters_held(n, true);
    const long held = clusters_held(n, false);
    if (held < 1) continue;
    const long waves = (groups + held - 1) / held;
    if (waves > 1 && n > 2) continue;
    const long per = (w.tiles + n - 1) / n;
    const double sm_tiles = (double)groups * n * per / sms * w.share * tile;
    const double us = 4.2 + (waves - 1) * (groups == w.units && n == 1 ? 2.5 : 4.2) +
                      std::max({per * (alone ? tile : 0.88), sm_tiles, w.mb * w.share / 6.6});
    if (us >= best) continue;
    best = us;
    c = n;
    stages = (int)std::min<long>(per, pv_half(s.head_dim) * (alone ? 2 : 1));
  }
  if (c == 0) return false;
  const PvInfo k = pv_kernel(s.head_dim, 1, true);
  plan->q_tiles = 0;
  plan->nt = 1;
  plan->chunks = (int)chunks;
  plan->nq_rows = (int)((rows + chunks - 1) / chunks);
  plan->cluster = c;
  plan->stages = stages;
  plan->smem = k.bytes(stages) + k.slots(c);
  plan->tiles_per_unit = (int)w.tiles;
  plan->tiles_per_cta = plan->seg_cost = plan->grid = 0;
  plan->max_seg = 1;
  return true;
}

}  // namespace

bool paged_verify_plan(const bd_shape& s, int rows, int n_q, PagedVerifyPlan* plan) {
  if (pv_cluster(s, rows, n_q, plan)) return true;
  pv_stream_rows(s, rows, plan);
  if (plan->smem > kMaxSmem) return false;
  const int keys = plan->q_tiles ? kVTcKeys : kPvKeys;
  const long units = (long)s.batch * s.h_kv * plan->chunks, ctas = pv_ctas(*plan);
  const long tpu = ((long)s.t_ctx + n_q + keys - 1) / keys;
  // A segment's end and the next one's start cost about 5 us of streaming (as in verify_plan), charged as virtual tiles.
  const double tile_us = (double)keys * s.head_dim * 4 / (6.5e6 / std::max(1, current_sm_count()));
  const long a = (long)std::min(16.0, std::max(0.0, 5.0 / tile_us + 0.5));
  const long vtotal = units * (tpu + a);
  if (vtotal >= 1L << 30) return false;
  // <= kVMaxSeg segments, as many as the merges hold the weights of: few long units do not fill the GPU (one of 128K, d 128, has
  // 32 CTAs: 38.4 us, 4 times what its bytes take; two 39.8, four 48.2, eight 83.1), and pv_stream_us does not know it.
  const long least = (tpu + a + kVMaxSeg - 2) / (kVMaxSeg - 1);
  const long vtpc = std::max((vtotal + ctas - 1) / ctas, least);
  plan->tiles_per_unit = (int)tpu;
  plan->seg_cost = (int)a;
  plan->grid = (int)((vtotal + vtpc - 1) / vtpc);
  if (s.seq_lens) {
    // the kernel cuts the ranges itself over the actual tiles
    plan->tiles_per_cta = (int)least;
    plan->max_seg = kVMaxSeg;
    return true;
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
  // (as a stream: a cluster needs none)  A unit's tpu tiles lie in at most ceil((tpu - 1) / vtpc) + 1 ranges of vtpc >= units (tpu + a) / ctas.
  PagedVerifyPlan plan = {};
  pv_stream_rows(s, rows, &plan);
  const long units = (long)s.batch * s.h_kv * plan.chunks, ctas = pv_ctas(plan);
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
    err = launch_kernel(fn, dim3(plan.grid), dim3(kPagedTcThreads), plan.smem, stream, args, 0);
    if (err != cudaSuccess || plan.max_seg <= 1) return err;
    return launch_verify_tc_merge(s.head_dim, units, p, stream, true);
  }
  PagedVerifyParams p;
  fill(p);
  p.stages = plan.stages;
  const PvInfo k = pv_kernel(s.head_dim, plan.nt, plan.cluster > 0);
  err = allow_shared_memory_once(k.fn, 0, k.allowed);
  if (err != cudaSuccess) return err;
  void* args[] = {&p, &kmap, &vmap};
  if (plan.cluster) return launch_kernel(k.fn, dim3(plan.cluster, units), dim3(k.threads), plan.smem, stream, args, plan.cluster);
  err = launch_kernel(k.fn, dim3(plan.grid), dim3(k.threads), plan.smem, stream, args, 0);
  if (err != cudaSuccess || plan.max_seg <= 1) return err;
  return launch_row_merge(s.head_dim, {p.o_part, p.lse_part, p.nseg, plan.max_seg, plan.nq_rows, rows, plan.chunks, units, o_out, lse_out}, stream);
}

}  // namespace bd
