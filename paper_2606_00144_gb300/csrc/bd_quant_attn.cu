// Attention over a 4-bit cache on mma.sync: the drafter's pass over a sparse view
// (bd_quant_draft_attn), and verify blocks (bd_quant_verify_attn).
//
// A warp takes tiles of 32 entries of its CTA's slice; K is the A operand (16 entries x 16 elements), the
// query rows the n8 side, as in the bf16 kernels, and the codes become fp16 operands by a mask and an FMA (bd_quant.cuh):
//   D_g   = sum over group g of (c - 8) q          exact products of a 4-bit and an 8-bit number;
//   S     = sum_g scale_g D_g                      fp32;
//   P_g   = 2^(S - M + e) ns_g                     fp16, ns_g the row's V scale of group g over 2^e
//                                                  (scale_exponent, kWeightExponent): 11 bits, where bf16 would keep 8; a
//                                                  weight below 2^-30 of the largest is lost;
//   O^T_g += (V_codes - 8)^T P_g                   both centred before the MMA (one FMA for two codes), which aligns
//                                                  a subnormal as if its leading zeros counted: with the codes
//                                                  as such and 8 times the rest subtracted, an element whose
//                                                  heavy rows hold zeros is what is left of a cancellation, to
//                                                  2^-17 of the weights, and a score is off by 2^-21 of
//                                                  sum |q k| (2^-24 so).
// ldmatrix lays a row's 16-byte group out as the A operand of S (a 32-bit word a lane), its transposed form as the
// A operand of O^T (16-bit units of two rows in a word), so neither side needs a shuffle.
// M is a running maximum of S + e that may trail by 2^8; each warp keeps its own, and the warps, then the CTAs
// of a unit, are merged at the end.
//
// A pass is a chain of latencies, not bandwidth (64 units of 512 entries read 5 MB, 0.7 us of HBM), so as few round trips as
// there are: the view's first indices are fetched beside its count, every warp has a tile or two, and the CTAs of a unit
// are a cluster that meets in shared memory (long views of few units: several clusters, whose parts the last CTA to
// arrive merges from global memory, in order).  64 units of 512 entries take 6.6 us, of 2048 13.8, 2 of 256 (d 64) 3.6.
#include <cooperative_groups.h>

#include <algorithm>

#include "bd_internal.h"
#include "bd_quant.cuh"

namespace cg = cooperative_groups;

namespace bd {

constexpr int kQaTile = 32;          // entries of a warp's tile
constexpr int kQaCluster = 8;        // most CTAs of a cluster (the portable size)
constexpr int kQaMaxParts = 8;       // clusters of a unit
constexpr float kQaSlack = 8.f;      // log2 of how far the running maximum may trail
constexpr float kQaLift = 6.f;       // weights are kept 2^6 higher: fp16's range is wider above 1 than P needs

struct QuantAttnParams {
  const uint8_t* kc;           // [units][t_cap][D / 2]
  const uint16_t* ks;          // [units][t_cap][D / 32]
  const uint8_t* vc;
  const uint16_t* vs;
  const __nv_bfloat16* q;      // [units][rows][D]: rows = query heads of a KV head x n_q
  __nv_bfloat16* o;
  float* lse;                  // or null
  float* o_part;               // [units][clusters][rows][D], normalised
  float* lse_part;             // [units][clusters][rows]
  int* counters;               // [units]
  int* status;
  const int32_t* seq_lens;
  const int32_t* idx;          // drafter pass: [units][budget]
  const int32_t* count;
  int h_kv, t_ctx, t_cap, n_q, rows, budget, step_j;
  int per_split, cluster, clusters;   // entries of a CTA; CTAs of a cluster; clusters of a unit
  bool early;                  // BD_DRAFT_VIEW_READY
  float scale_log2;            // log2(e) / sqrt(D)
};

template <int D>
struct QaStage {
  static constexpr int CODES = kQaTile * D / 2;                  // bytes of a tile's codes
  static constexpr int SCALES = kQaTile * D / kQGroup * 2;
  static constexpr int BYTES = 2 * (CODES + SCALES);
};
// Byte offset of 16-byte group g of row r in a tile of codes: groups rotate so that eight rows' reads of one
// group fall into different banks.
template <int D>
__device__ __forceinline__ uint32_t code_offset(int r, int g) {
  return D == 128 ? r * 64 + ((g ^ (r >> 1 & 3)) << 4) : r * 32 + ((g ^ (r >> 2 & 1)) << 4);
}

// Ones in the half of each number that is negative.
__device__ __forceinline__ uint32_t signs(float lo, float hi) {
  uint32_t r;
  asm("prmt.b32 %0, %1, %2, 0xffbb;" : "=r"(r) : "r"(__float_as_uint(lo)), "r"(__float_as_uint(hi)));
  return r;
}

// WARPS: 4 with three tiles in flight each, or 8 with two for slices of more than a tile a warp.
template <int D, int NT, int WARPS>
struct QaSmem {
  static constexpr int kStages = WARPS == 4 ? 3 : 2;
  static constexpr size_t kRing = (size_t)WARPS * kStages * QaStage<D>::BYTES;
  static constexpr size_t kMerge = (size_t)WARPS * 8 * NT * (D + 4 + 2) * 4;
  static constexpr size_t kArea = kRing > kMerge ? kRing : kMerge;
  // A cluster's parts: CTA k merges rows k, k + cluster, ... of every CTA, so that the slots of all are little more than
  // one CTA's rows (all of them in the first CTA took 33 (66) KB of each, which halved the CTAs of an SM).
  __host__ __device__ static constexpr int slot_rows(int cluster) { return (8 * NT + cluster - 1) / cluster; }
  static size_t bytes(int cluster) { return kArea + (cluster > 1 ? (size_t)cluster * slot_rows(cluster) * (D + 1) * 4 : 0); }
};

__device__ __forceinline__ int quant_context(const int32_t* seq_lens, int b, int t_ctx, int* status) {
  if (seq_lens == nullptr) return t_ctx;
  int t = seq_lens[b];
  if (t < 0 || t > t_ctx) {
    if (status) record_error(status, BD_ERR_INVALID_ARG);
    t = min(max(t, 0), t_ctx);
  }
  return t;
}

// NT: n8 tiles of query rows; GATHER: entries come from idx (and the drafted rows), else entry = cache row.
template <int D, int NT, bool GATHER, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, NT == 1 ? 16 / WARPS : 1) quant_attn_kernel(const __grid_constant__ QuantAttnParams p) {
  using ST = QaStage<D>;
  constexpr int kQaWarps = WARPS, kQaThreads = 32 * WARPS, kQaStages = QaSmem<D, NT, WARPS>::kStages;
  constexpr int G = D / 32, NQC = 8 * NT;
  extern __shared__ __align__(128) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
  const int split = blockIdx.x, unit = blockIdx.y, row0 = blockIdx.z * NQC;
  const int rows = min(p.rows - row0, NQC);
  const int b = unit / p.h_kv;
  if (!p.early) {
    grid_dependency_wait();
    allow_dependent_launch();
  }
  if (p.cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // this CTA has started

  // slices by what a view can hold: the first tiles' indices need not wait for the count
  const int e_begin = split * p.per_split;
  const int32_t* iunit = GATHER ? p.idx + (size_t)unit * p.budget : nullptr;
  auto index = [&](int tile) {                 // idx of entry `lane` of a tile, if it may be one
    const int e = e_begin + tile * kQaTile + lane;
    return GATHER && e < p.budget && tile * kQaTile + lane < p.per_split ? __ldg(iunit + e) : 0;
  };
  int spec[kQaStages];
#pragma unroll
  for (int i = 0; i < kQaStages; ++i) spec[i] = index(warp + i * kQaWarps);
  int* status = tid == 0 ? p.status : nullptr;
  int cnt = 0;
  if (GATHER) {
    cnt = __ldg(p.count + unit);
    if (cnt < 0 || cnt > p.budget) {
      if (status) record_error(status, BD_ERR_INVALID_ARG);
      cnt = min(max(cnt, 0), p.budget);
    }
  }
  const int t_unit = quant_context(p.seq_lens, b, p.t_ctx, status);
  const int n_entries = GATHER ? cnt + p.step_j + 1 : t_unit + p.n_q;
  const int e_end = min(n_entries, e_begin + p.per_split);
  const int n_tiles = e_end > e_begin ? (e_end - e_begin + kQaTile - 1) / kQaTile : 0;

  const size_t base = (size_t)unit * p.t_cap;
  uint8_t* ring = smem + (size_t)warp * kQaStages * ST::BYTES;

  // entry `lane` of a tile: its cache row, or -1 (r: its index, where it has one)
  auto entry_row = [&](int tile, int r) {
    const int e = e_begin + tile * kQaTile + lane;
    if (e >= e_end) return -1;
    if (!GATHER) return e;
    if (e >= cnt) return t_unit + (e - cnt);
    if (r < 0 || r >= t_unit) {
      record_error(p.status, BD_ERR_INVALID_ARG);
      return -1;
    }
    return r;
  };
  // Scales come through L1 (a cp.async of 4 or 8 bytes has no other way), a line of many rows'.  A row whose line may also
  // hold a drafted row's (the context's last rows; the first ones, next to the unit before) must not bring that line in
  // before the drafted rows are there, or their scales could be read stale: it is asked for with the drafted rows.
  constexpr int kNear = 128 / (2 * G);         // rows of a line's scales
  auto late = [&](int row) { return row < kNear || row + kNear > t_unit; };
  // row: this lane's entry_row; returns which of the tile's entries are there (the rest are zero-filled).
  // part 0: rows that are not late; 1: those that are, and what is zero-filled; 2: all
  auto fetch = [&](int row, int slot, int part) {
    uint8_t* st = ring + slot * ST::BYTES;
    constexpr int PER = 32 / G;                // rows a pass of the warp covers, G 16-byte groups each
#pragma unroll
    for (int it = 0; it < G; ++it) {
      const int r = it * PER + lane / G, g = lane % G;
      const int src_row = __shfl_sync(0xffffffffu, row, r);
      if (part != 2 && (part == 1) != late(src_row)) continue;
      const size_t src = (base + max(src_row, 0)) * (D / 2) + 16 * g;
      const uint32_t off = code_offset<D>(r, g);
      cp_async16_zfill(st + off, p.kc + src, src_row >= 0);
      cp_async16_zfill(st + ST::CODES + off, p.vc + src, src_row >= 0);
    }
    if (part == 2 || (part == 1) == late(row)) {
      const size_t src = (base + max(row, 0)) * G;
      cp_async_small<2 * G>(st + 2 * ST::CODES + lane * 2 * G, p.ks + src, row >= 0);
      cp_async_small<2 * G>(st + 2 * ST::CODES + ST::SCALES + lane * 2 * G, p.vs + src, row >= 0);
    }
    return __ballot_sync(0xffffffffu, row >= 0);
  };

  // this warp's tiles: warp, warp + kQaWarps, ...
  const int mine = n_tiles > warp ? (n_tiles - warp + kQaWarps - 1) / kQaWarps : 0;
  uint32_t live[kQaStages] = {};               // of this iteration's tile and the next ones
  int at_row[kQaStages];
#pragma unroll
  for (int i = 0; i < kQaStages; ++i) at_row[i] = i < mine ? entry_row(warp + i * kQaWarps, spec[i]) : -1;
  if (p.early) {                               // the view is older than the kernel before; the drafted rows are not
#pragma unroll
    for (int i = 0; i < kQaStages - 1; ++i)
      if (i < mine) fetch(at_row[i], i, 0);
    grid_dependency_wait();
    allow_dependent_launch();
  }
#pragma unroll
  for (int i = 0; i < kQaStages - 1; ++i) {
    if (i < mine) live[i] = fetch(at_row[i], i, p.early ? 1 : 2);
    cp_async_commit();
  }
  int next_row = at_row[kQaStages - 1];

  // ---- the query rows as B operands: fp16 over a power of two of their own
  uint32_t bq[NT][G][4];
  float mult[NT][2];
  int lim[NT][2];                              // last visible entry of this lane's columns
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = 8 * nt + gid;                // B column gid
    uint4 w[G];
#pragma unroll
    for (int g = 0; g < G; ++g)
      w[g] = r < rows ? *reinterpret_cast<const uint4*>(p.q + ((size_t)unit * p.rows + row0 + r) * D + 32 * g + 8 * tig)
                      : make_uint4(0u, 0u, 0u, 0u);
    uint32_t top = 0;                          // largest exponent of the row's finite elements
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint32_t x[4] = {w[g].x, w[g].y, w[g].z, w[g].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo = x[e] >> 7 & 0xffu, hi = x[e] >> 23 & 0xffu;
        top = max(top, max(lo == 255 ? 0u : lo, hi == 255 ? 0u : hi));
      }
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int qe = min(max((int)top - 127, -100), 100);        // the row's elements are below 2^(qe + 1)
    const float down = pow2i(13 - qe);                         // to fp16: below 2^14
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint32_t x[4] = {w[g].x, w[g].y, w[g].z, w[g].w};
      float f[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(x[e] << 16) * down;
        f[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u) * down;
      }
      // element pairs (0, 4), (1, 5), (2, 6), (3, 7): the codes that one mask of a word leaves
      bq[nt][g][0] = pack_half2(f[0], f[4]);
      bq[nt][g][1] = pack_half2(f[1], f[5]);
      bq[nt][g][2] = pack_half2(f[2], f[6]);
      bq[nt][g][3] = pack_half2(f[3], f[7]);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {              // this lane's accumulator columns
      const int src = 4 * (2 * tig + e), col = 8 * nt + 2 * tig + e;
      // S over the codes' 2^-10 and the row's own power of two, in log2 units
      mult[nt][e] = p.scale_log2 * pow2i(__shfl_sync(0xffffffffu, qe, src) - 3);
      lim[nt][e] = GATHER || col >= rows ? 0x7fffffff : t_unit + (row0 + col) % p.n_q;
    }
  }

  float o[2 * G][NT][4], m[NT][2], l[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt][0] = m[nt][1] = -INFINITY;
    l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
    for (int mt = 0; mt < 2 * G; ++mt)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[mt][nt][c] = 0.f;
  }

  for (int i = 0; i < mine; ++i) {
    const int tile = warp + i * kQaWarps;
    // the tile two further on, its rows looked up an iteration ago
    if (i + kQaStages - 1 < mine) live[kQaStages - 1] = fetch(next_row, (i + kQaStages - 1) % kQaStages, 2);
    cp_async_commit();
    if (i + kQaStages < mine) next_row = entry_row(tile + kQaStages * kQaWarps, index(tile + kQaStages * kQaWarps));
    cp_async_wait<kQaStages - 1>();
    __syncwarp();
    const uint8_t* st = ring + (i % kQaStages) * ST::BYTES;
    const uint32_t kbase = smem_u32(st), vbase = kbase + ST::CODES;
    const uint16_t* ksm = reinterpret_cast<const uint16_t*>(st + 2 * ST::CODES);
    const uint16_t* vsm = reinterpret_cast<const uint16_t*>(st + 2 * ST::CODES + ST::SCALES);
    const int e0 = e_begin + tile * kQaTile;

    // ---------------------------------------------------------------- S of two 16-entry sub-tiles
    // scores; of rows gid, gid + 8: V's exponents e, 2^-u (u = max(e, kWeightExponent)), V scales over 2^u
    float s[2][NT][4], ve[2][2], un[2][2], vn[2][2][G];
    bool low = false;                           // some u is above its e
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      uint32_t kw[2 * G];                       // [group][row half]
#pragma unroll
      for (int gp = 0; gp < G; gp += 2) {
        uint32_t r4[4];
        const int r = 16 * sub + (lane & 15), g = gp + (lane >> 4);
        ldmatrix_x4(r4, kbase + code_offset<D>(r, g));
        kw[2 * gp] = r4[0], kw[2 * gp + 1] = r4[1], kw[2 * gp + 2] = r4[2], kw[2 * gp + 3] = r4[3];
      }
      float kscale[2][G];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = 16 * sub + 8 * h + gid;
        RowScales<D> ks, vs;
        ks.load_shared(ksm + r * G);
        vs.load_shared(vsm + r * G);
        const int e = vs.exponent();
        ve[sub][h] = (float)e;
        un[sub][h] = pow2i(-max(e, kWeightExponent));
        low |= e < kWeightExponent;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          kscale[h][g] = ks.scale(g);
          vn[sub][h][g] = vs.scale(g) * un[sub][h];
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int c = 0; c < 4; ++c) s[sub][nt][c] = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const uint32_t w0 = kw[2 * g], w1 = kw[2 * g + 1], x0 = w0 >> 8, x1 = w1 >> 8;
          float d[4] = {0.f, 0.f, 0.f, 0.f};
          mma_16816_f16(d, centred0(w0), centred0(w1), centred1(w0), centred1(w1), bq[nt][g][0], bq[nt][g][1]);
          mma_16816_f16(d, centred0(x0), centred0(x1), centred1(x0), centred1(x1), bq[nt][g][2], bq[nt][g][3]);
#pragma unroll
          for (int c = 0; c < 4; ++c) s[sub][nt][c] = fmaf(d[c], kscale[c >> 1][g], s[sub][nt][c]);
        }
      }
    }

    // ---------------------------------------------------------------- weights
    const bool masked = live[0] != 0xffffffffu || (!GATHER && e0 + kQaTile - 1 > t_unit);
    bool grow = false;
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float y = s[sub][nt][c] * mult[nt][c & 1] + ve[sub][c >> 1];
          if (masked) {
            const int r = 16 * sub + 8 * (c >> 1) + gid;
            if ((live[0] >> r & 1) == 0 || (!GATHER && e0 + r > lim[nt][c & 1])) y = -INFINITY;
          }
          s[sub][nt][c] = y;
          grow |= y > m[nt][c & 1] + kQaSlack;
        }
    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = fmaxf(fmaxf(s[0][nt][e], s[0][nt][e + 2]), fmaxf(s[1][nt][e], s[1][nt][e + 2]));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          mx = fmaxf(mx, m[nt][e]);
          const float root = mx == -INFINITY ? 1.f : fast_exp2(0.5f * (m[nt][e] - mx)), alpha = root * root;
          m[nt][e] = mx;
          l[nt][e] = l[nt][e] * root * root;
#pragma unroll
          for (int mt = 0; mt < 2 * G; ++mt) {
            o[mt][nt][e] *= alpha;
            o[mt][nt][e + 2] *= alpha;
          }
        }
    }
    if (__any_sync(0xffffffffu, low)) {         // (rare)
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float rest = fmaxf(ve[sub][h], kWeightExponent) - ve[sub][h];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            s[sub][nt][2 * h] += rest;
            s[sub][nt][2 * h + 1] += rest;
          }
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float nm = kQaLift - (m[nt][e] == -INFINITY ? 0.f : m[nt][e]);
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float w = fast_exp2(s[sub][nt][2 * h + e] + nm);
            if (!GATHER && masked && s[sub][nt][2 * h + e] == -INFINITY) w = -0.f;   // hidden (below)
            s[sub][nt][2 * h + e] = w;
            l[nt][e] = fmaf(w, un[sub][h], l[nt][e]);
          }
      }

    // ---------------------------------------------------------------- O^T += V^T P^T
    uint32_t vw[2][2 * G];                      // [sub][group][entry half]
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int gp = 0; gp < G; gp += 2) {
        uint32_t r4[4];
        const int r = 16 * sub + (lane & 15), g = gp + (lane >> 4);
        ldmatrix_x4_trans(r4, vbase + code_offset<D>(r, g));
        vw[sub][2 * gp] = r4[0], vw[sub][2 * gp + 1] = r4[1], vw[sub][2 * gp + 2] = r4[2], vw[sub][2 * gp + 3] = r4[3];
      }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int g = 0; g < G; ++g) {
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          const float* w = s[sub][nt];
          uint32_t b0 = pack_half2(w[0] * vn[sub][0][g], w[1] * vn[sub][0][g]);
          uint32_t b1 = pack_half2(w[2] * vn[sub][1][g], w[3] * vn[sub][1][g]);
          if (!GATHER) {                        // a hidden entry's weight is -0: its product is 0, also with a scale that is no number
            b0 &= ~signs(w[0], w[1]);
            b1 &= ~signs(w[2], w[3]);
          }
          b0 = movmatrix_trans(b0);
          b1 = movmatrix_trans(b1);
          const uint32_t w0 = vw[sub][2 * g], w1 = vw[sub][2 * g + 1], x0 = w0 >> 8, x1 = w1 >> 8;
          mma_16816_f16(o[2 * g][nt], centred0(w0), centred1(w0), centred0(w1), centred1(w1), b0, b1);
          mma_16816_f16(o[2 * g + 1][nt], centred0(x0), centred1(x0), centred0(x1), centred1(x1), b0, b1);
        }
      }
    __syncwarp();                               // the slot is free
#pragma unroll
    for (int k = 0; k + 1 < kQaStages; ++k) live[k] = live[k + 1];
  }
  cp_async_wait<0>();
  __syncthreads();                              // every warp's ring is free: the merge area

  // ---------------------------------------------------------------- the warps' states
  constexpr int OP = D + 4;
  float* o_s = reinterpret_cast<float*>(smem);                 // [warp][NQC][OP]
  float* m_s = o_s + kQaWarps * NQC * OP;                      // [warp][NQC]
  float* l_s = m_s + kQaWarps * NQC;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float sum = l[nt][e];
      sum += __shfl_xor_sync(0xffffffffu, sum, 4);
      sum += __shfl_xor_sync(0xffffffffu, sum, 8);
      sum += __shfl_xor_sync(0xffffffffu, sum, 16);
      const int at = warp * NQC + 8 * nt + 2 * tig + e;
      if (gid == 0) {
        m_s[at] = m[nt][e] == -INFINITY ? -INFINITY : m[nt][e] - kQaLift;
        l_s[at] = sum;
      }
      // four adjacent elements 32 g + 4 gid ..
#pragma unroll
      for (int g = 0; g < G; ++g)
        *reinterpret_cast<float4*>(o_s + (size_t)at * OP + 32 * g + 4 * gid) =
            make_float4(o[2 * g][nt][e] * 0x1p10f, o[2 * g][nt][e + 2] * 0x1p10f, o[2 * g + 1][nt][e] * 0x1p10f,
                        o[2 * g + 1][nt][e + 2] * 0x1p10f);
    }
  __syncthreads();
  const size_t out0 = (size_t)unit * p.rows + row0;
  const int C = p.cluster, part = split / C;
  const int slot_rows = QaSmem<D, NT, WARPS>::slot_rows(C);
  float* slots = reinterpret_cast<float*>(smem + QaSmem<D, NT, WARPS>::kArea);   // [C][slot_rows][D], then [C][slot_rows] lse
  float* lses = slots + (size_t)C * slot_rows * D;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = C > 1 ? (int)cluster.block_rank() : 0;
  if (C > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // every CTA is running
  // a row's final values, or with several clusters its part's
  auto emit = [&](int r, int d, float4 a, float lse) {
    if (p.clusters == 1) {
      *reinterpret_cast<uint2*>(p.o + (out0 + r) * D + d) = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
      if (d == 0 && p.lse) p.lse[out0 + r] = lse;
    } else {
      const size_t at = ((size_t)unit * p.clusters + part) * p.rows + row0 + r;
      *reinterpret_cast<float4*>(p.o_part + at * D + d) = a;
      if (d == 0) p.lse_part[at] = lse;
    }
  };
  for (int i = tid; i < rows * (D / 4); i += kQaThreads) {
    const int r = i / (D / 4), d = i % (D / 4) * 4;
    float mx = -INFINITY, tot = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kQaWarps; ++w) mx = fmaxf(mx, m_s[w * NQC + r]);
#pragma unroll
    for (int w = 0; w < kQaWarps; ++w) {
      const float mw = m_s[w * NQC + r], lw = l_s[w * NQC + r];
      if (mw == -INFINITY && lw == 0.f) continue;              // a warp without entries for this row
      const float root = fast_exp2(0.5f * (mw - mx)), f = root * root;
      const float4 v = *reinterpret_cast<const float4*>(o_s + (size_t)(w * NQC + r) * OP + d);
      tot = fmaf(root * lw, root, tot);
      a.x = fmaf(f, v.x, a.x);
      a.y = fmaf(f, v.y, a.y);
      a.z = fmaf(f, v.z, a.z);
      a.w = fmaf(f, v.w, a.w);
    }
    const float inv = tot == 0.f ? 0.f : 1.f / tot;            // (a NaN stays one)
    a.x *= inv, a.y *= inv, a.z *= inv, a.w *= inv;
    const float lse = tot == 0.f ? -INFINITY : (mx + log2f(tot)) * kLn2;
    if (C == 1) {
      emit(r, d, a, lse);
    } else {
      const int to = r % C, at = rank * slot_rows + r / C;
      *reinterpret_cast<float4*>(cluster.map_shared_rank(slots + (size_t)at * D + d, to)) = a;
      if (d == 0) *cluster.map_shared_rank(lses + at, to) = lse;
    }
  }
  if (C > 1) {
    // ---------------------------------------------------------------- the cluster's parts of this CTA's rows
    __syncwarp();
    cluster.sync();                            // all have landed
    for (int i = tid; i < slot_rows * (D / 4); i += kQaThreads) {
      const int at = i / (D / 4), r = at * C + rank, d = i % (D / 4) * 4;
      if (r >= rows) break;
      float ls[kQaCluster], mx = -INFINITY, tot = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kQaCluster; ++k) {
        ls[k] = k < C ? lses[k * slot_rows + at] : -INFINITY;
        mx = fmaxf(mx, ls[k]);
      }
#pragma unroll
      for (int k = 0; k < kQaCluster; ++k) {
        if (k >= C || ls[k] == -INFINITY) continue;            // (an empty part's slot holds zeros; a NaN stays one)
        const float f = fast_exp2((ls[k] - mx) * kLog2e);
        const float4 v = *reinterpret_cast<const float4*>(slots + ((size_t)k * slot_rows + at) * D + d);
        tot += f;
        a.x = fmaf(f, v.x, a.x);
        a.y = fmaf(f, v.y, a.y);
        a.z = fmaf(f, v.z, a.z);
        a.w = fmaf(f, v.w, a.w);
      }
      const float inv = tot == 0.f ? 0.f : 1.f / tot;
      a.x *= inv, a.y *= inv, a.z *= inv, a.w *= inv;
      emit(r, d, a, tot == 0.f ? -INFINITY : mx + logf(tot));
    }
  }
  if (p.clusters == 1) return;

  // ---------------------------------------------------------------- the unit's last CTA to arrive merges
  __shared__ int last;
  __threadfence();
  __syncthreads();
  if (tid == 0) last = atomicAdd(&p.counters[unit], 1) == (int)(gridDim.x * gridDim.z) - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  const float* parts = p.o_part + (size_t)unit * p.clusters * p.rows * D;
  const float* part_lse = p.lse_part + (size_t)unit * p.clusters * p.rows;
  for (int i = tid; i < p.rows * (D / 4); i += kQaThreads) {
    const int r = i / (D / 4), d = i % (D / 4) * 4;
    float ls[kQaMaxParts], mx = -INFINITY, tot = 0.f;
    float4 v[kQaMaxParts], a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kQaMaxParts; ++k) {    // every part requested at once
      const size_t at = (size_t)k * p.rows + r;
      ls[k] = k < p.clusters ? __ldcg(part_lse + at) : -INFINITY;
      v[k] = k < p.clusters ? __ldcg(reinterpret_cast<const float4*>(parts + at * D + d)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int k = 0; k < kQaMaxParts; ++k) mx = fmaxf(mx, ls[k]);
#pragma unroll
    for (int k = 0; k < kQaMaxParts; ++k) {
      if (ls[k] == -INFINITY) continue;
      const float f = fast_exp2((ls[k] - mx) * kLog2e);
      tot += f;
      a.x = fmaf(f, v[k].x, a.x);
      a.y = fmaf(f, v[k].y, a.y);
      a.z = fmaf(f, v[k].z, a.z);
      a.w = fmaf(f, v[k].w, a.w);
    }
    const float inv = tot == 0.f ? 0.f : 1.f / tot;
    *reinterpret_cast<uint2*>(p.o + ((size_t)unit * p.rows + r) * D + d) =
        make_uint2(pack_bf16x2(a.x * inv, a.y * inv), pack_bf16x2(a.z * inv, a.w * inv));
    if (d == 0 && p.lse) p.lse[(size_t)unit * p.rows + r] = tot == 0.f ? -INFINITY : mx + logf(tot);
  }
  if (tid == 0) p.counters[unit] = 0;
}

// ============================================================================ host side

namespace {

struct QaInfo {
  const void* fn;
  int id;                      // 0 .. 11
  size_t (*smem)(int cluster);
  std::atomic<uint64_t>* allowed;
};
template <int D, int NT, bool GATHER, int WARPS>
QaInfo qa_one() {
  static std::atomic<uint64_t> allowed{0};
  constexpr int id = (D == 128 ? 6 : 0) + (GATHER ? 3 : 0) + (NT == 2 ? 2 : WARPS == 8);
  return {reinterpret_cast<const void*>(&quant_attn_kernel<D, NT, GATHER, WARPS>), id, &QaSmem<D, NT, WARPS>::bytes, &allowed};
}
template <int D, bool GATHER>
QaInfo qa_info(int nt, int warps) {
  return nt == 2 ? qa_one<D, 2, GATHER, 4>() : warps == 4 ? qa_one<D, 1, GATHER, 4>() : qa_one<D, 1, GATHER, 8>();
}
QaInfo qa_kernel(int d, int nt, int warps, bool gather) {
  if (d == 64) return gather ? qa_info<64, true>(nt, warps) : qa_info<64, false>(nt, warps);
  return gather ? qa_info<128, true>(nt, warps) : qa_info<128, false>(nt, warps);
}

// Clusters of c CTAs that the device holds at once (a GPC's SMs are shared out by whole clusters).  Asked once per instance
// and c.
long clusters_held(const QaInfo& k, int warps, int c) {
  static thread_local int cache_dev = -1;
  static thread_local int cache[12][kQaCluster + 1];
  int dev = 0;
  const long guess = 2L * current_sm_count() / c;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    (void)cudaGetLastError();
    return guess;
  }
  if (dev != cache_dev) {
    std::fill_n(&cache[0][0], sizeof(cache) / sizeof(int), -1);
    cache_dev = dev;
  }
  int& held = cache[k.id][c];
  if (held < 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(c);
    cfg.blockDim = dim3(32 * warps);
    cfg.dynamicSmemBytes = k.smem(c);
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)c;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    int n = 0;
    if (allow_shared_memory_once(k.fn, 128, k.allowed) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, k.fn, &cfg) != cudaSuccess) {
      (void)cudaGetLastError();
      n = (int)guess;
    }
    held = n;
  }
  return held;
}

}  // namespace

bool quant_attn_plan(const bd_shape& s, int rows, long entries, bool gather, QuantAttnPlan* plan) {
  const long units = (long)s.batch * s.h_kv;
  long blocks = 0;             // units x chunks
  auto tiles = [&](int nt) {
    plan->nt = nt;
    plan->chunks = (rows + 8 * nt - 1) / (8 * nt);
    blocks = units * plan->chunks;
  };
  tiles(rows <= 8 ? 1 : 2);
  if (units > 65535 || plan->chunks > 65535) return false;
  // A tile for every one of four warps, eight warps where a slice is longer, as long as one wave holds the CTAs: a second
  // one repeats the whole chain of latencies (32 units of 1024 entries, 16 rows: 23.7 us in clusters of eight that waited for
  // another's end, 12.3; 40 units, 8 rows 12.3 / 9.3).
  const long slots = std::max(1L, 2L * current_sm_count() / blocks);
  const int most = (int)std::min<long>(kQaCluster, (entries + 4 * kQaTile - 1) / (4 * kQaTile));
  auto take = [&](int cluster, int clusters) {
    const long ctas = (long)cluster * clusters;
    plan->cluster = cluster;
    plan->clusters = clusters;
    plan->per_split = (int)(((entries + ctas - 1) / ctas + 15) / 16 * 16);
    plan->warps = plan->nt == 1 && plan->per_split > 4 * kQaTile ? 8 : 4;
    // (above seven eighths of what the device holds, launches of 16 rows do take a second wave: 96 of 97 clusters 14.5 us,
    // 10.8 as pairs; 32 of 36 12.3)
    const long held = clusters_held(qa_kernel(s.head_dim, plan->nt, plan->warps, gather), plan->warps, cluster);
    return plan->one_wave = blocks * clusters <= (plan->nt == 2 ? held * 7 / 8 : held);
  };
  plan->most_clusters = (int)std::min<long>(kQaMaxParts, (slots + kQaCluster - 1) / kQaCluster);
  // Several clusters of a unit cost a merge through global memory, as long as some 320 entries of a CTA.
  auto cut = [&] {
    const long room = std::max(1L, 2L * current_sm_count() / blocks);
    const long want = std::min(room, (entries + 4 * kQaTile - 1) / (4 * kQaTile));
    int clusters = (int)std::min<long>(kQaMaxParts, (want + kQaCluster - 1) / kQaCluster);
    if (entries / kQaCluster - entries / want <= 320) clusters = 1;
    plan->one_wave = false;
    for (; clusters > 1 && !plan->one_wave; --clusters) take((int)std::min<long>(kQaCluster, (want + clusters - 1) / clusters), clusters);
    for (int c = most; c > 0 && !plan->one_wave; --c) take(c, 1);
  };
  // Chunks of 8 rows while the device holds them all at once, else of 16.  A CTA's chain is a third shorter with one n8 tile, and
  // what the chunks read again is in L2 (2 units of 1K, d 64, 24 rows: 6.3 us as chunks of 16, 4.2; 64 units of 0.5K, 24 rows 12.1 / 9.9;
  // drafter pass of 8 units of 1024, 16 rows 8.2 / 6.7).
  tiles(1);
  cut();
  if (rows > 8 && !plan->one_wave) {
    tiles(2);
    cut();
  }
  return true;
}

size_t quant_attn_bytes(const bd_shape& s, int rows, const QuantAttnPlan& plan) {
  const size_t part_rows = (size_t)s.batch * s.h_kv * plan.most_clusters * rows;
  return plan.most_clusters > 1 ? align_up(part_rows * s.head_dim * 4, 256) + align_up(part_rows * 4, 256) : 0;
}

cudaError_t launch_quant_attn(const bd_shape& s, const QuantAttnPlan& plan, const QuantAttnCall& c, const bd_quant_cache& cache,
                              void* ws_region, int* counters, int* status, cudaStream_t stream) {
  QuantAttnParams p;
  p.kc = static_cast<const uint8_t*>(cache.k_codes);
  p.ks = static_cast<const uint16_t*>(cache.k_scales);
  p.vc = static_cast<const uint8_t*>(cache.v_codes);
  p.vs = static_cast<const uint16_t*>(cache.v_scales);
  p.q = static_cast<const __nv_bfloat16*>(c.q);
  p.o = static_cast<__nv_bfloat16*>(c.o_out);
  p.lse = c.lse_out;
  p.rows = c.rows;
  const size_t part_rows = (size_t)s.batch * s.h_kv * plan.clusters * c.rows;
  p.o_part = static_cast<float*>(ws_region);
  p.lse_part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws_region) + align_up(part_rows * s.head_dim * 4, 256));
  p.counters = counters;
  p.status = status;
  p.seq_lens = s.seq_lens;
  p.idx = c.idx;
  p.count = c.count;
  p.h_kv = s.h_kv;
  p.t_ctx = s.t_ctx;
  p.t_cap = s.t_cap;
  p.n_q = c.n_q;
  p.budget = c.budget;
  p.step_j = c.step_j;
  p.per_split = plan.per_split;
  p.cluster = plan.cluster;
  p.clusters = plan.clusters;
  p.early = c.view_ready;
  p.scale_log2 = kLog2e / sqrtf((float)s.head_dim);
  const QaInfo k = qa_kernel(s.head_dim, plan.nt, plan.warps, c.idx != nullptr);
  cudaError_t err = allow_shared_memory_once(k.fn, 128, k.allowed);
  if (err != cudaSuccess) return err;
  void* args[] = {&p};
  return launch_kernel(k.fn, dim3(plan.cluster * plan.clusters, s.batch * s.h_kv, plan.chunks), dim3(32 * plan.warps),
                       k.smem(plan.cluster), stream, args, plan.cluster > 1 ? plan.cluster : 0);
}

}  // namespace bd
