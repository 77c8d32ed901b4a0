// Verify blocks and single-token decoding over a 4-bit cache on the 5th-generation tensor cores.
//
// A 4-bit cache halves the bytes of an 8-bit one and moves the work to the codes' unpacking, so the kernel is built
// around it: both MMAs take the unpacked cache as their A operand from TENSOR MEMORY, written there straight
// from the registers it is unpacked in, and the few query rows are the N side.
//   S^T = K Q^T      M = 128 keys, N = 32 (64) query rows, K = D.  A thread unpacks a key's row: lane = key.
//   P^T = 2^(S^T - M + e), one thread per key; e the exponent of the key's V scales (scale_exponent, kWeightExponent)
//   O^T += V^T P^T   M = D, N = query rows, K = 128 keys.  ldmatrix.trans lays a group's 32 channels of two keys
//                    out as the 16-lane halves of a 16x128b store: lane = channel, column = key pair.
// Unpacking is a mask and one packed FMA for two codes (bd_quant.cuh): c * 2^-k * scale + (-8 scale 2^-j), rounded
// once.  Each row's scales are divided by a power of two of its own, which joins the scores (K) or the weights (V), so that
// the row's largest fits fp16 whatever it is; a value is off by 2^-19 of that at most, and not at all where its own group's
// scale is at least 2^-8 of it.  (Exact down to 2^-23, with c - 8 formed before it is multiplied: 24 rows of 64 units of 16K
// 47.5 us for 43.0, one row 42.1 for 37.3; codes 0 and 2 left where they lie in K, with 2^-16 in place of 2^-19: 42.5, 36.8.)
//
// Four warpgroups take the tiles in turn, each through the whole chain with buffers of its own: unpack K, start S,
// unpack V while S runs (into K's columns once it is done), softmax, start P V.  Roles of their own (K, V, softmax
// warps, with two buffers between them) left every warp a chain of waits: 1700 cycles a tile, of which its work
// was 600.  As it is a tile takes some 1240 cycles of an SM, of which each scheduler issues in some 780 (64 units of 16K,
// 24 rows: 43.7 us, 3.5 TB/s; one row 37.5 us, 4.0 TB/s).  No unit is full (the issue slots 62 %, the ALU pipe 47 %, DRAM
// 44 %): the rest is waiting along each group's chain, where V takes K's columns once S is done and the next K V's once P V
// is.  A fifth group of the same chain (up to 8 rows, 96 registers a thread: 38.4 us for 36.2) did not fill it.
// Blocks of more than 32 query rows run on two groups of two warpgroups: those share a tile's unpacking and halve its
// columns, so that K and V are unpacked once for up to 96 rows (16 units of 16K, 168 rows in two chunks: 48 us, 68 on
// four groups, when that was tried; 51 now; 64 units, 64 rows 73 us, 84 rows 86).
// Work is cut as in verify_kernel (bd_verify.cuh): one list of (unit, 128-key tile) pairs in equal ranges, one CTA
// per SM, partials merged by quant_merge_kernel.
#include <algorithm>

#include "bd_internal.h"
#include "bd_quant.cuh"
#include "bd_verify.cuh"

namespace bd {

constexpr int kQtKeys = 128;          // keys of a tile
constexpr int kQtThreads = 512;
constexpr int kQtStages = 2;          // tiles of codes in flight for each group
constexpr float kQtSlack = 8.f;       // log2 of how far a running maximum may trail
constexpr float kQtScale = 0x1p15f;                  // where a row's largest scale is put in fp16, whose end is 2^16,
constexpr float kQtOperand = kQtScale * 0x1p-21f;    // and where that leaves a code of 1 times it
constexpr float kQtLift = 6.f;        // weights are kept 2^6 higher (fp16 reaches further above 1 than P needs)

struct QuantTcParams {
  const uint16_t* ks;          // [units][t_cap][D / 32]
  const uint16_t* vs;
  const __nv_bfloat16* q;      // [units][rows_total][D]
  __nv_bfloat16* o;
  float* lse;                  // or null
  float* o_part;               // [units x chunks][max_seg][nq_rows][D], normalised
  float* lse_part;             // [units x chunks][max_seg][nq_rows]
  int* nseg;                   // [units x chunks] segments
  int* status;
  const int32_t* seq_lens;
  int h_kv, n_q, nq_rows, rows_total, row_chunks, t_ctx, t_cap, units;
  int tiles_per_unit, max_seg, seg_cost, vtiles_per_cta;
  float scale_log2;            // log2(e) / sqrt(D)
};

// H warpgroups a group, each of which takes NC columns of query rows.
template <int D, int NC, int H>
struct QuantTcSmem {
  static constexpr int N = H == 1 ? 32 : H * NC;               // the MMAs' N side
  static constexpr int GROUPS = 4 / H;
  static constexpr uint32_t TILE = kQtKeys * D / 2;            // codes of one tensor
  static constexpr uint32_t Q_BYTES = N * D * 2, P_BYTES = kQtKeys * N * 2;
  static constexpr uint32_t FIXED = 2048;                      // the CTA's flags, places of the query rows; then its queries
  // A group's area, everything at a constant offset from its start: barriers and loads, exchange, a tile's V scales
  // (4 groups x 128 keys, fp16), weights, codes.
  static constexpr uint32_t EXCHANGE = 256, SCALES = 4096, WEIGHTS = 5120, CODES = WEIGHTS + P_BYTES;
  static constexpr uint32_t GROUP = CODES + kQtStages * 2 * TILE;
  static constexpr size_t kTotal = 1024 + FIXED + Q_BYTES + GROUPS * GROUP;
};

template <int N>
__device__ __forceinline__ void tc_ld_cols(uint32_t taddr, float (&v)[N]);
__device__ __forceinline__ void tc_ld_8(uint32_t taddr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
template <>
__device__ __forceinline__ void tc_ld_cols<8>(uint32_t taddr, float (&v)[8]) {
  tc_ld_8(taddr, v);
}
template <>
__device__ __forceinline__ void tc_ld_cols<24>(uint32_t taddr, float (&v)[24]) {
  tc_ld_16cols(taddr, *reinterpret_cast<float(*)[16]>(&v[0]));
  tc_ld_8(taddr + 16, v + 16);
}
template <>
__device__ __forceinline__ void tc_ld_cols<32>(uint32_t taddr, float (&v)[32]) {
  tc_ld_32cols(taddr, v);
}
__device__ __forceinline__ void tc_st_8(uint32_t taddr, const float* v) {
  const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// 16 lanes x 32 columns: register 2 i (2 i + 1) of lane l is TMEM lane l / 4 (+ 8), column 4 i + l % 4.
__device__ __forceinline__ void tc_st_16x128b_8(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ void tc_st_16x128b(uint32_t taddr, const uint32_t (&r)[16]) { tc_st_16x128b_8(taddr, r); }
__device__ __forceinline__ void tc_st_16x128b(uint32_t taddr, const uint32_t (&r)[8]) {   // 16 columns
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// MMA with A in tensor memory, B in shared memory; desc_hi: B's high descriptor word.
__device__ __forceinline__ void tc_mma_ts_hi(uint32_t lead, uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi,
                                             uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\t"
      "setp.ne.b32 q, %0, 0;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 db, {%3, %6};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%1], [%2], db, %4, p;\n\t}" ::"r"(lead),
      "r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(b_hi)
      : "memory");
}
// Instruction descriptor: kind::f16 with fp16 A and B, fp32 D, K-major operands.
__host__ __device__ constexpr uint32_t umma_idesc_f16(int m, int n) {
  return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}

// Whether any of n threads says so; a barrier over them.
__device__ __forceinline__ bool bar_any(int id, int n, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.or.pred q, %2, %3, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)x), "r"(id), "r"(n)
      : "memory");
  return r != 0;
}

// Floats as integers of the same order (NaN above all).
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }

__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}

__device__ __forceinline__ int quant_tc_context(const int32_t* seq_lens, int b, int t_ctx, int* status) {
  if (seq_lens == nullptr) return t_ctx;
  int t = seq_lens[b];
  if (t < 0 || t > t_ctx) {
    if (status) record_error(status, BD_ERR_INVALID_ARG);
    t = min(max(t, 0), t_ctx);
  }
  return t;
}

// A thread's columns of query rows: NB blocks of BC.
template <int D, int BC, int NB, int H>
__global__ void __launch_bounds__(kQtThreads, 1) quant_tc_kernel(const __grid_constant__ QuantTcParams p,
                                                                const __grid_constant__ CUtensorMap kmap,
                                                                const __grid_constant__ CUtensorMap vmap) {
  constexpr int NC = BC * NB;
  using L = QuantTcSmem<D, NC, H>;
  constexpr int N = L::N, G = D / 32, ST = kQtStages, GROUPS = L::GROUPS, GT = 128 * H;
  constexpr uint32_t TILE = L::TILE;
  // B of P V: MN-major, 32 weights of a key in one row of a 64-byte swizzle atom of 8 keys, blocks of 32 one after another
  constexpr uint32_t P_PITCH = 64, P_ATOM = 8 * P_PITCH, P_BLOCK = kQtKeys * P_PITCH;
  constexpr uint32_t kPDescHi = (P_ATOM >> 4) | (1u << 14) | (4u << 29);
  constexpr uint32_t TM = 512 / GROUPS;                    // TMEM columns of a group: K's, then V's operand (64), S (N), O (N)
  static_assert(64 + 2 * N <= TM, "a group's tensor memory");
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* qtop = reinterpret_cast<int*>(smem + 64);           // [16]
  int* wtot = reinterpret_cast<int*>(smem + 128);          // [16]
  int* nan_from = reinterpret_cast<int*>(smem + 192);      // [4] first row of the block (from 1 on) whose V is no number, by group
  int* lifted = reinterpret_cast<int*>(smem + 208);        // whether some query row has a power of two of its own,
  int* qpos = reinterpret_cast<int*>(smem + 1024);         // [N] a query row's place in its block
  float* qdown = reinterpret_cast<float*>(smem + 1536);    // [N] and what that takes its scores by
  static_assert(N <= 128, "a row's place and factor");
  uint8_t* qbuf = smem + L::FIXED;
  uint8_t* groups = qbuf + L::Q_BYTES;
  int* pref = reinterpret_cast<int*>(groups + GROUPS * L::GROUP);
  static_assert(L::Q_BYTES % 1024 == 0 && L::P_BYTES % 1024 == 0 && L::GROUP % 1024 == 0, "aligned tiles");
  static_assert(L::EXCHANGE + N * 16 + N * 8 <= L::SCALES, "exchange");

  const int tid = threadIdx.x, warp = uniform_warp(), lane = tid & 31, quad = warp & 3, set = warp >> 2;
  const int grp = set / H, half = set % H;                 // the warpgroup's group, and which of its columns and unpacking
  // a group's barriers
  auto k_full = [&](int g, int st) { return reinterpret_cast<uint64_t*>(groups + g * L::GROUP) + st; };   // codes of K,
  auto v_full = [&](int g, int st) { return k_full(g, ST + st); };                                        // of V have arrived
  auto s_done = [&](int g) { return k_full(g, 2 * ST); };          // S is in TMEM, K's columns are free
  auto pv_done = [&](int g) { return k_full(g, 2 * ST + 1); };     // O is up to date, V's columns and P are free
  auto drain = [&](int g) { return k_full(g, 2 * ST + 2); };
  if (tid == 0) {
    for (int g = 0; g < GROUPS; ++g)
      for (int i = 0; i < 2 * ST + 3; ++i) mbar_init(k_full(g, i), 1);
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_map(&kmap);
    tma_prefetch_map(&vmap);
  }
  // Branches that single lanes take end in a __syncwarp() where an instruction for whole warps follows (tcgen05.alloc, .ld,
  // .st, bar): nothing else promises that the lanes are together again.
  __syncwarp();
  if (warp == 0) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  // P's columns past the query rows are never written again
  for (uint32_t i = tid % GT; i < L::P_BYTES / 16; i += GT)
    reinterpret_cast<uint4*>(groups + grp * L::GROUP + L::WEIGHTS)[i] = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, lanes = (uint32_t)(quad * 32) << 16;
  const uint32_t t_kv = tmem + TM * grp, t_s = t_kv + 64, t_o = t_s + N;

  grid_dependency_wait();
  allow_dependent_launch();
  VerifyMap map{nullptr, p.tiles_per_unit, p.seg_cost, p.units, p.vtiles_per_cta};
  if (p.seq_lens) {
    int last_u = -1, last = 0;               // (asked for twice; a thread has one unit as a rule)
    lay_out_spans<kQtThreads>(p.units, [&](int u) {
      if (u != last_u) last = (quant_tc_context(p.seq_lens, u / p.row_chunks / p.h_kv, p.t_ctx, nullptr) + p.n_q + kQtKeys - 1) / kQtKeys + p.seg_cost;
      last_u = u;
      return last;
    }, wtot, pref);
    map.pref = pref;
    map.vtpc = max((pref[p.units] + (int)gridDim.x - 1) / (int)gridDim.x, p.vtiles_per_cta);
  }
  const int v_total = map.vbase(p.units);
  const int v0 = min(v_total, (int)blockIdx.x * map.vtpc), v1 = min(v_total, v0 + map.vtpc);
  const int u_first = v0 < v1 ? map.unit_of(v0) : 0;
  int u_last = v0 < v1 ? u_first : -1;       // (a unit more or two)
  while (u_last >= 0 && u_last + 1 < p.units && map.vbase(u_last + 1) < v1) ++u_last;
  bool alive = true;      // false once a wait gave up

  // ---- the group's MMAs and its loads are started by a warp each (other groups' on other SMSPs).  Local tile i is job
  // grp + GROUPS i of the CTA's list of tiles.
  const bool issuer = quad == grp && half == 0, loader = quad == (grp ^ 2) && half == H - 1;
  const uint32_t lead = elect_leader();
  uint8_t* mine = groups + grp * L::GROUP;
  uint8_t* my_ring = mine + L::CODES;
  int* issued = reinterpret_cast<int*>(mine + 128);        // K's, V's loads so far (for a CTA that gives up)
  // Job j's K or V into stage s: u is a unit of the list, its segment the tiles tb, .. of which the first is job `from`;
  // j lies in it or, seldom, further on.
  auto load = [&](int which, int s, int j, int u, int kv_unit, int tb, int n, int from) {
    while (j >= from + n) {
      if (u >= u_last) return;
      from += n;
      ++u;
      kv_unit = u / p.row_chunks;
      tb = map.first_tile(u, v0);
      n = max(0, map.end_tile(u, v1) - tb);
    }
    if (lead) {
      uint64_t* full = which ? v_full(grp, s) : k_full(grp, s);
      mbar_arrive_expect_tx(full, TILE);
      tma_load_3d(my_ring + (2 * s + which) * TILE, which ? &vmap : &kmap, full, 0, (tb + j - from) * kQtKeys, kv_unit);
      issued[which] = j / GROUPS + 1;
    }
    __syncwarp();
  };
  if (loader && lead) issued[0] = issued[1] = 0;

  const int row = quad * 32 + lane, tig = lane & 3;   // this thread's key of a tile
  const int col0 = half * NC;                         // and its columns of query rows
  const bool has_rows = quad < G;                     // this warp has channels of V (and of O)
  uint8_t* my_scales = mine + L::SCALES;                   // [4][4][16][2] fp16
  uint8_t* my_p = mine + L::WEIGHTS;
  auto red_of = [&](int g) { return reinterpret_cast<int*>(groups + g * L::GROUP + L::EXCHANGE); };   // [N][4] a column's maximum
  auto nm_of = [&](int g) { return reinterpret_cast<float*>(red_of(g) + 4 * N); };   // (or sum) in each warp; [N] lift - running
  int* my_red = red_of(grp) + 4 * col0;                    // maximum (1e30: none yet); [N] the root of what its last rise scales by
  float* my_nm = nm_of(grp) + col0;
  float* my_alpha = my_nm + N;
  const int bar = 1 + grp;
  constexpr uint32_t idesc_s = umma_idesc_f16(128, N), idesc_o = idesc_s | kIdescBMnMajor;

  // A wait that has usually been over for long: one poll and a vote.  Once one has given up the warp goes on without
  // waiting (every address stays in bounds and every barrier meets), starts no MMA and writes no output.
  auto wait = [&](uint64_t* b, uint32_t parity) {
    if (!__all_sync(0xffffffffu, mbar_test(smem_u32(b), parity))) alive = alive && mbar_wait_warp(b, parity, p.status, abort_flag);
  };
  int job = 0, i = 0;     // tiles of the CTA before the segment; this warpgroup's tiles so far
  for (int unit = u_first; unit <= u_last; ++unit) {
    const int tb = map.first_tile(unit, v0), n = map.end_tile(unit, v1) - tb;
    if (n <= 0) continue;
    const int kv_unit = unit / p.row_chunks;
    const int t_unit = quant_tc_context(p.seq_lens, kv_unit / p.h_kv, p.t_ctx, tid == 0 ? p.status : nullptr);
    const int row_base = (unit - kv_unit * p.row_chunks) * p.nq_rows;
    const int rows = min(p.nq_rows, p.rows_total - row_base);
    const int end = t_unit + p.n_q;
    // the first tile's scales, on their way while the queries are laid out
    const int row0 = kv_unit * p.t_cap;        // (a cache has fewer than 2^31 rows)
    const int t_first = (grp - job) & (GROUPS - 1);   // this group's tiles of the segment: t_first, t_first + GROUPS, ...
    RowScales<D> kn, vn;
    {
      const int key = (tb + t_first) * kQtKeys + row;
      kn.load(p.ks + (size_t)(row0 + key) * G, t_first < n && key < end);
      vn.load(p.vs + (size_t)(row0 + key) * G, t_first < n && key < end);
    }
    // ---- the query rows as B of S: fp16 over one power of two, in the order the codes are unpacked in.  A row whose largest
    // is below 2^-12 of the block's has its own besides, which its scores are multiplied by: one row's size costs no other
    // its digits.
    float base;
    bool own_sizes;
    {
      constexpr int CH = D / 8, PER = (N * CH + kQtThreads - 1) / kQtThreads, STEP = kQtThreads / CH;
      const int r0 = tid / CH, c = tid % CH;
      uint4 w[PER];
      uint32_t top = 0, row_top[PER];
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int r = r0 + k * STEP;
        w[k] = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows) w[k] = __ldg(reinterpret_cast<const uint4*>(p.q + ((size_t)kv_unit * p.rows_total + row_base + r) * D + 8 * c));
      }
      if (job == 0 && loader) {                // the first tiles, while the queries and scales arrive
#pragma unroll 1
        for (int k = 0; k < 2 * ST; ++k) load(k & 1, k >> 1, grp + GROUPS * (k >> 1), unit, kv_unit, tb, n, 0);
      }
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const uint32_t x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
        row_top[k] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t lo = x[e] >> 7 & 0xffu, hi = x[e] >> 23 & 0xffu;
          row_top[k] = max(row_top[k], max(lo == 255 ? 0u : lo, hi == 255 ? 0u : hi));
        }
#pragma unroll
        for (int off = 1; off < CH; off *= 2) row_top[k] = max(row_top[k], __shfl_xor_sync(0xffffffffu, row_top[k], off));
        top = max(top, row_top[k]);
      }
      top = __reduce_max_sync(0xffffffffu, top);
      if (job > 0) __syncthreads();            // (the segment before has read its own)
      if (lane == 0) qtop[warp] = (int)top;
      if (tid < 4) nan_from[tid] = 0x7fffffff;
      if (tid == 0) *lifted = 0;
      if (tid < N) qpos[tid] = tid < rows ? (row_base + tid) % p.n_q : 0x7fffffff;
      if (tid < N)
        for (int g = 0; g < GROUPS; ++g) nm_of(g)[tid] = 1e30f;
      __syncthreads();
      int t = 0;
#pragma unroll
      for (int k = 0; k < 16; ++k) t = max(t, qtop[k]);
      const int qe = min(max(t - 127, -100), 100);
      // S over the queries' power of two and the operand's, in log2 units (the key's own power comes with it)
      base = p.scale_log2 / kQtOperand * pow2i(qe - 13);
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int r = r0 + k * STEP;
        const int below = qe - ((int)row_top[k] - 127), lift = row_top[k] > 0 && below > 12 ? min(below, min(126, 114 + qe)) : 0;
        const float down = pow2i(13 - qe + lift);
        if (c == 0 && r < N) qdown[r] = pow2i(-lift);
        if (lift > 0) *lifted = 1;
        const uint32_t x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
        float f[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f[2 * e] = __uint_as_float(x[e] << 16) * down;
          f[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u) * down;
        }
        if (r < N)
          *reinterpret_cast<uint4*>(qbuf + (c >> 3) * (N * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) =
              make_uint4(pack_half2(f[0], f[4]), pack_half2(f[1], f[5]), pack_half2(f[2], f[6]), pack_half2(f[3], f[7]));
      }
      fence_proxy_async_smem();
      __syncthreads();
      own_sizes = *lifted != 0;
    }

    float l[NC];                               // sums of this thread's keys' weights
#pragma unroll
    for (int c = 0; c < NC; ++c) l[c] = 0.f;
    for (int t = t_first; t < n; t += GROUPS, ++i) {
      const int s = i & 1, ph = (i >> 1) & 1, key = (tb + t) * kQtKeys + row;
      const uint32_t stage = s * 2 * TILE;
      // this thread's places in shared memory: its row of codes of a tile, its V scales, its weights (with several blocks of
      // columns worked out anew in every tile: their sums need the registers)
      int at_row = row;
      if (NB > 1) asm volatile("" : "+r"(at_row));
      const uint32_t sw = D == 128 ? at_row >> 1 & 3 : at_row >> 2 & 1, p_sw = (at_row >> 1 & 3) << 4;
      const uint8_t* k_row = my_ring + at_row * (D / 2);
      const uint32_t v_rows = smem_u32(my_ring) + TILE + (at_row & 31) * (D / 2) + ((quad ^ (D == 128 ? at_row >> 1 & 3 : at_row >> 2 & 1)) << 4);
      uint8_t* scale_at = my_scales + (at_row >> 1 & 3) * 64 + (at_row >> 3) * 4 + (at_row & 1) * 2;
      uint8_t* p_row = my_p + at_row * P_PITCH;
      const bool masked = (tb + t + 1) * kQtKeys - 1 > t_unit;
      const float a = fminf(base * pow2i(kn.exponent()), 3e38f);
      const int ev = vn.exponent();
      // ---- K: this thread's key into its TMEM lane
      {
        const float down = pow2i(-kn.exponent()) * kQtScale;
        constexpr int KG = G / H;              // groups of 32 elements that this warpgroup unpacks
        uint32_t s0[KG];
#pragma unroll
        for (int g = 0; g < KG; ++g) {
          const float ns = kn.scale(half * KG + g) * down;
          s0[g] = pack_half2(ns, ns);
        }
        // the keys' V scales, laid out by (group, lane of a quad, key pair)
        const float vdown = pow2i(-ev) * kQtScale;
#pragma unroll
        for (int g = 0; g < KG; ++g)
          *reinterpret_cast<__half*>(scale_at + (half * KG + g) * 256) = __float2half_rn(vn.scale(half * KG + g) * vdown);
        if (masked && key > t_unit) {          // (rare: one tile or two of a unit)
          // A row of the block that is no number may be hidden from some of the queries, to whom 0 times it would be NaN: it
          // counts as zeros here, and the queries that see it have NaN written at the segment's end.
#pragma unroll
          for (int g = 0; g < KG; ++g)
            if (!(vn.scale(half * KG + g) < INFINITY)) {
              *reinterpret_cast<uint16_t*>(scale_at + (half * KG + g) * 256) = 0;
              atomicMin(nan_from + half * KG + g, key - t_unit);
            }
        }
        if (masked) __syncwarp();
        const int next = key + GROUPS * kQtKeys;   // the next tile's, a tile ahead (84 rows, 64 units of 16K, d 64: 81 us, 94 without)
        kn.load(p.ks + (size_t)(row0 + next) * G, next < end && t + GROUPS < n);
        vn.load(p.vs + (size_t)(row0 + next) * G, next < end && t + GROUPS < n);
        wait(k_full(grp, s), ph);
        uint4 w[KG];                           // (with several blocks of columns read where they are used: 93 us for 86.5 at 84 rows)
        auto read = [&](int g) { w[g] = *reinterpret_cast<const uint4*>(k_row + stage + (((half * KG + g) ^ sw) << 4)); };
#pragma unroll
        for (int g = 0; g < KG; ++g)
          if (NB == 1) read(g);
        // (the columns' last reader was the P V before)
        if (i > 0) wait(pv_done(grp), (i - 1) & 1);
        tc_fence_after();
#pragma unroll
        for (int g = 0; g < KG; ++g) {
            const uint32_t s1 = mul_half2(s0[g], 0x2c002c00u);       // 2^-4
            const uint32_t c = mul_half2(s0[g], 0x80408040u);        // -2^-18: -8 of 2^-21
            if (NB > 1) read(g);
            const uint32_t x[4] = {w[g].x, w[g].y, w[g].z, w[g].w};
            uint32_t out[16];                                        // element pairs (0, 4), (1, 5), (2, 6), (3, 7) of eight
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t lo = x[k] << 3, hi = x[k] >> 5;
              out[4 * k] = fma_half2(lo & 0x00780078u, s0[g], c);    // c 2^-21 * s
              out[4 * k + 1] = fma_half2(lo & 0x07800780u, s1, c);   // c 2^-17 * s / 16
              out[4 * k + 2] = fma_half2(hi & 0x00780078u, s0[g], c);
              out[4 * k + 3] = fma_half2(hi & 0x07800780u, s1, c);
            }
            tc_st_16cols(t_kv + lanes + 16 * (half * KG + g), out);
        }
        tc_wait_st();
      }
      tc_fence_before();
      named_bar(bar, GT);
      if (issuer && alive) {
        tc_fence_after();
        const uint32_t b_lo = desc_k(smem_u32(qbuf));
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
          tc_mma_ts_hi(lead, t_s, t_kv + 8 * ks, b_lo + ((ks >> 2) * (N * 128) + (ks & 3) * 32) / 16, kDescHi, idesc_s, ks > 0 ? 1u : 0u);
        tc_commit(lead, s_done(grp));
      }
      if (loader) load(0, s, job + t + GROUPS * ST, unit, kv_unit, tb, n, job);

      // ---- V: a warp unpacks a group's 32 channels, while S runs
      wait(v_full(grp, s), ph);
      {
        constexpr int VK = NB > 1 ? 4 : 8;    // key pairs of a lane at a time (four where the sums leave few registers)
#pragma unroll
        for (int hh = 0; hh < 16 / (VK * H); ++hh) {
          const int h = H == 1 ? hh : half * (16 / (VK * H)) + hh;
          uint32_t w[VK], sp[VK];
          if (has_rows) {
#pragma unroll
            for (int k = 0; k < VK / 4; ++k) {
              ldmatrix_x4_trans(*reinterpret_cast<uint32_t(*)[4]>(&w[4 * k]), v_rows + stage + (8 * VK * h + 32 * k) * (D / 2));
              *reinterpret_cast<uint4*>(&sp[4 * k]) = *reinterpret_cast<const uint4*>(my_scales + quad * 256 + tig * 64 + 4 * VK * h + 16 * k);
            }
          }
          if (hh == 0) {
            wait(s_done(grp), i & 1);
            tc_fence_after();
          }
          if (has_rows) {
            uint32_t lo[2 * VK], hi[2 * VK];  // lanes 0-15: codes 0 and 1 of a unit; 16-31: codes 2 and 3
#pragma unroll
            for (int k = 0; k < VK; ++k) {
              const uint32_t s0 = sp[k], s1 = mul_half2(s0, 0x2c002c00u);   // 2^-4
              const uint32_t c = mul_half2(s0, 0x80408040u);                // -2^-18
              const uint32_t x = w[k] << 3, y = w[k] >> 5;
              lo[2 * k] = fma_half2(x & 0x00780078u, s0, c);
              lo[2 * k + 1] = fma_half2(x & 0x07800780u, s1, c);
              hi[2 * k] = fma_half2(y & 0x00780078u, s0, c);
              hi[2 * k + 1] = fma_half2(y & 0x07800780u, s1, c);
            }
            tc_st_16x128b(t_kv + lanes + 4 * VK * h, lo);
            tc_st_16x128b(t_kv + lanes + 4 * VK * h + (16u << 16), hi);
          }
        }
      }

      // ---- softmax: this thread's key, NC query rows
      // (rare; asked of shared memory anew where the sums leave no register for it)
      if (NB > 1 ? *reinterpret_cast<volatile int*>(lifted) != 0 : own_sizes) {
#pragma unroll 1
        for (int c = 0; c < NC; c += 8) {
          float z[8];
          tc_ld_8(t_s + lanes + col0 + c, z);
          tc_wait_ld();
#pragma unroll
          for (int k = 0; k < 8; ++k) z[k] *= qdown[col0 + c + k];
          tc_st_8(t_s + lanes + col0 + c, z);
        }
        tc_wait_st();
      }
      const int eu = max(ev, kWeightExponent);  // what joins the weights before their sum (a row below may raise maxima in vain)
      const float e = (float)eu;
      float ys[NB > 1 ? 2 : 1][BC];            // (of several blocks the next is on its way while one is worked on)
      auto fetch = [&](int nb) { tc_ld_cols<BC>(t_s + lanes + col0 + BC * nb, ys[nb & 1]); };
      // a block of the tile's scores plus e less the running maximum, in log2 units
      auto scores = [&](int nb, float& mx) {
        const int c0 = BC * nb;
        float* y = ys[nb & 1];
        tc_wait_ld();
        if (nb + 1 < NB) fetch(nb + 1);
#pragma unroll
        for (int c = 0; c < BC; c += 2) {
          const float2 r = ffma2(make_float2(y[c], y[c + 1]), make_float2(a, a), make_float2(e, e));
          y[c] = r.x;
          y[c + 1] = r.y;
        }
        if (masked) {
#pragma unroll
          for (int c = 0; c < BC; ++c) y[c] = key - t_unit <= qpos[col0 + c0 + c] ? y[c] : -INFINITY;
        }
#pragma unroll
        for (int c = 0; c < BC; c += 4) {
          const float4 m = *reinterpret_cast<const float4*>(my_nm + c0 + c);
          const float2 r0 = fadd2(make_float2(y[c], y[c + 1]), make_float2(m.x, m.y));
          const float2 r1 = fadd2(make_float2(y[c + 2], y[c + 3]), make_float2(m.z, m.w));
          y[c] = r0.x;
          y[c + 1] = r0.y;
          y[c + 2] = r1.x;
          y[c + 3] = r1.y;
          mx = fmaxf(fmaxf(mx, y[c]), y[c + 1]);
          mx = fmaxf(fmaxf(mx, y[c + 2]), y[c + 3]);
        }
      };
      // (one copy of that code for one block: once maxima have been raised it runs again, and only once: a
      // row that holds a NaN may still be above the slack)
#pragma unroll 1
      for (int pass = 0; pass < 2; ++pass) {
        float mx = -INFINITY;
        fetch(0);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) scores(nb, mx);
        if (pass == 1 || !bar_any(bar, GT, mx > kQtSlack + kQtLift)) break;
        // ---- some row's maximum grows by more than the slack: all rows take theirs
#pragma unroll 1
        for (int c = 0; c < NC; c += 8) {
          float z[8];
          int top = 0;
          tc_ld_8(t_s + lanes + col0 + c, z);
          tc_wait_ld();
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float x = masked && key - t_unit > qpos[col0 + c + k] ? -INFINITY : fmaf(z[k], a, (float)ev);
            const int r = __reduce_max_sync(0xffffffffu, ordered(x));
            top = lane == k ? r : top;
          }
          if (lane < 8) my_red[4 * (c + lane) + quad] = top;
          __syncwarp();
        }
        named_bar(bar, GT);
        if (quad == 0) {
          for (int c = lane; c < NC; c += 32) {
            const int4 r = *reinterpret_cast<const int4*>(my_red + 4 * c);
            const float top = unordered(max(max(r.x, r.y), max(r.z, r.w))), old = my_nm[c];
            const float m = fminf(old, top == -INFINITY ? 1e30f : kQtLift - top);   // (a NaN score is passed over: its row is NaN all the same)
            my_nm[c] = m;
            my_alpha[c] = fast_exp2(0.5f * (m - old));
          }
          __syncwarp();                        // (lanes leave the loop apart)
        }
        named_bar(bar, GT);
#pragma unroll
        for (int c = 0; c < NC; ++c) l[c] = l[c] * my_alpha[c] * my_alpha[c];
        if (t > t_first && has_rows) {         // O holds the group's earlier tiles of the segment
#pragma unroll 1
          for (int c = 0; c < NC; c += 8) {
            float o[8];
            tc_ld_8(t_o + lanes + col0 + c, o);
            tc_wait_ld();
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] *= my_alpha[c + k] * my_alpha[c + k];
            tc_st_8(t_o + lanes + col0 + c, o);
          }
          tc_wait_st();
        }
      }
      {
        const float el = pow2i(-eu), rest = pow2i(ev - eu);   // (the rest of ev: multiplied in always, a branch around it took longer)
        if (NB > 1) fetch(0);                  // (a single block is still there)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float mx = 0.f;
          if (NB > 1) scores(nb, mx);
          const float* y = ys[nb & 1];
#pragma unroll
          for (int c = 0; c < BC; c += 8) {
            uint32_t h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float* lc = l + BC * nb + c + 2 * k;
              const float x0 = fast_exp2(y[c + 2 * k]), x1 = fast_exp2(y[c + 2 * k + 1]);
              const float2 z = ffma2(make_float2(x0, x1), make_float2(el, el), make_float2(lc[0], lc[1]));
              lc[0] = z.x;
              lc[1] = z.y;
              const float2 w = fmul2(make_float2(x0, x1), make_float2(rest, rest));
              h[k] = pack_half2(w.x, w.y);
            }
            const int at = col0 + BC * nb + c;
            *reinterpret_cast<uint4*>(p_row + (H == 1 ? c * 2 ^ p_sw : (at >> 5) * P_BLOCK + ((at & 31) * 2 ^ p_sw))) =
                make_uint4(h[0], h[1], h[2], h[3]);
          }
        }
        tc_wait_st();
      }
      fence_proxy_async_smem();
      tc_fence_before();
      named_bar(bar, GT);
      if (issuer && alive) {
        tc_fence_after();
        const uint32_t b_lo = desc_mn(smem_u32(my_p), P_BLOCK);
#pragma unroll
        for (int ks = 0; ks < kQtKeys / 16; ++ks)
          tc_mma_ts_hi(lead, t_o, t_kv + 8 * ks, b_lo + ks * (2 * P_ATOM / 16), kPDescHi, idesc_o, t > t_first || ks > 0 ? 1u : 0u);
        tc_commit(lead, pv_done(grp));
      }
      if (loader) load(1, s, job + t + GROUPS * ST, unit, kv_unit, tb, n, job);
    }

    // ---------------------------------------------------------------- end of the segment
    job += n;
    // the rows' sums over this warp's keys: lane c ends with column 32 k + c (their maxima were read before the last barrier)
#pragma unroll
    for (int c0 = 0; c0 < NC; c0 += 32) {
      float sum[32];
#pragma unroll
      for (int c = 0; c < 32; ++c) sum[c] = c0 + c < NC ? l[c0 + c < NC ? c0 + c : 0] : 0.f;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1)
#pragma unroll
        for (int k = 0; k < off; ++k) {
          const bool upper = (lane & off) != 0;
          const float send = upper ? sum[k] : sum[k + off], keep = upper ? sum[k + off] : sum[k];
          sum[k] = keep + __shfl_xor_sync(0xffffffffu, send, off);
        }
      if (c0 + lane < NC) my_red[4 * (c0 + lane) + quad] = __float_as_int(sum[0]);
    }
    __syncwarp();
    // Every group's last P V: its own warps wait for it (a parity does not tell another group's phases apart), the barrier
    // passes that on, and the fence behind the barrier orders the reads of the groups' O below.
    if (t_first < n) wait(pv_done(grp), (i - 1) & 1);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const int c_first = map.owner(unit, 0), n_seg = map.owner(unit, map.tiles(unit) - 1) - c_first + 1;
    const bool whole = n_seg == 1;
    const size_t slot = (size_t)unit * p.max_seg + ((int)blockIdx.x - c_first), orow0 = (size_t)kv_unit * p.rows_total + row_base;
    if ((int)blockIdx.x == c_first && tid == 0 && p.max_seg > 1) p.nseg[unit] = n_seg;
    const int ch = 32 * quad + 4 * (lane & 7) + (lane >> 3);   // this lane's channel
    const int no_number = nan_from[quad];
    // the groups' states merged, eight columns at a time, the blocks dealt out over the warpgroups: lane k has column c + k
#pragma unroll 1
    for (int c = 8 * set; c < rows; c += 32) {
      const int mc = c + (lane & 7);
      float f[GROUPS], tot = 0.f, nm = nm_of(0)[mc];
#pragma unroll
      for (int g = 1; g < GROUPS; ++g) nm = fminf(nm, nm_of(g)[mc]);
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int4 r = *reinterpret_cast<const int4*>(red_of(g) + 4 * mc);
        f[g] = fast_exp2(0.5f * (nm - nm_of(g)[mc]));
        tot += f[g] * (f[g] * ((__int_as_float(r.x) + __int_as_float(r.y)) + (__int_as_float(r.z) + __int_as_float(r.w))));
        f[g] *= f[g];
      }
      const float inv = tot == 0.f ? 0.f : 1.f / (kQtOperand * tot);   // (a NaN stays one)
      if (!alive) continue;
      if (quad == 0 && lane < 8 && mc < rows) {
        const float lse = tot == 0.f ? -INFINITY : (log2f(tot) - nm) * kLn2;
        if (!whole) p.lse_part[slot * p.nq_rows + mc] = lse;
        else if (p.lse) p.lse[orow0 + mc] = lse;
      }
      __syncwarp();
      if (!has_rows) continue;
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = 0.f;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int done = (job - g + GROUPS - 1) / GROUPS;
        if (g + GROUPS * (done - 1) < job - n) continue;       // no tiles, O holds nothing
        float o[8];
        tc_ld_8(tmem + TM * g + 64 + N + lanes + c, o);
        tc_wait_ld();
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = fmaf(o[k], __shfl_sync(0xffffffffu, f[g] * inv, k), x[k]);
      }
      if (no_number != 0x7fffffff) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = qpos[c + k] >= no_number ? NAN : x[k];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int r = c + k;
        if (r < rows) {
          if (whole) p.o[(orow0 + r) * D + ch] = __float2bfloat16_rn(x[k]);
          else p.o_part[(slot * p.nq_rows + r) * D + ch] = x[k];
        }
      }
    }
    tc_fence_before();                                         // (the next segment's barrier comes before its P V)
  }
  if (*abort_flag) {   // no copy may land in shared memory, no MMA write to TMEM after the CTA exits
    if (loader)
      for (int w = 0; w < 2; ++w)
        for (int k = max(0, issued[w] - ST); k < issued[w]; ++k)
          mbar_wait(w ? v_full(grp, k % ST) : k_full(grp, k % ST), (k / ST) & 1, p.status, nullptr);
    if (issuer) {
      tc_commit(lead, drain(grp));
      mbar_wait(drain(grp), 0, p.status, nullptr);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) tmem_dealloc(tmem, 512);
}

// Merge of the segments' partials, one warp per query row of a unit (a unit of one segment was written by
// quant_tc_kernel itself).  A lane takes four adjacent channels (at D 64 half of the segments).
template <int D>
__global__ void __launch_bounds__(128) quant_merge_kernel(const float* o_part, const float* lse_part, const int* nseg, int max_seg,
                                                          int nq_rows, int rows_total, int row_chunks, __nv_bfloat16* o, float* lse) {
  // lanes of a row's channels; segment groups; a group's parts at a time, and those asked for before their number is known
  constexpr int Q = D / 4, NG = 32 / Q, AT = 16, AHEAD = 4;
  grid_dependency_wait();
  allow_dependent_launch();
  const int unit = blockIdx.x, r = blockIdx.y * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int kv_unit = unit / row_chunks, row_base = (unit - kv_unit * row_chunks) * nq_rows;
  if (r >= min(nq_rows, rows_total - row_base)) return;
  const size_t base = (size_t)unit * max_seg;
  const int q = lane % Q, g = lane / Q;
  const float* lp = lse_part + base * nq_rows + r;
  const float4* op = reinterpret_cast<const float4*>(o_part + (base * nq_rows + r) * D) + q;
  // one round trip for the segments' number, their lse and the first parts (what lies past the number is not used): 64 units of
  // 16K 44.3 -> 43.0 us; all 16 parts so: 40 units of 84 rows 36.8 -> 39.4
  auto part = [&](int s, int end) { return s < end ? __ldcg(op + (size_t)s * nq_rows * Q) : make_float4(0.f, 0.f, 0.f, 0.f); };
  float4 v[AT];
#pragma unroll
  for (int i = 0; i < AT; ++i) v[i] = part(i * NG + g, i < AHEAD ? max_seg : 0);
  float l0 = lane < max_seg ? __ldcg(lp + (size_t)lane * nq_rows) : -INFINITY;
  float l1 = lane + 32 < max_seg ? __ldcg(lp + (size_t)(lane + 32) * nq_rows) : -INFINITY;
  const int n = min(__ldcg(nseg + unit), max_seg);
  if (n <= 1) return;
  l0 = lane < n ? l0 : -INFINITY;
  l1 = lane + 32 < n ? l1 : -INFINITY;
  float mx = fmaxf(l0, l1);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
  // (empty parts weigh nothing; a NaN stays one)
  const float w0 = l0 == -INFINITY ? 0.f : fast_exp2((l0 - mx) * kLog2e), w1 = l1 == -INFINITY ? 0.f : fast_exp2((l1 - mx) * kLog2e);
  float tot = w0 + w1;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) tot += __shfl_xor_sync(0xffffffffu, tot, off);
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = 0; s0 < n; s0 += AT * NG) {
    if (s0 > 0 || n > AHEAD * NG) {
#pragma unroll
      for (int i = 0; i < AT; ++i)
        if (s0 > 0 || i >= AHEAD) v[i] = part(s0 + i * NG + g, n);
    }
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const int s = s0 + i * NG + g;
      const float wl = __shfl_sync(0xffffffffu, w0, s & 31), wh = __shfl_sync(0xffffffffu, w1, s & 31);
      const float w = s < 32 ? wl : wh;
      if (s < n) {                             // (an empty part holds zeros; a NaN stays one however little its part weighs)
        a.x = fmaf(w, v[i].x, a.x);
        a.y = fmaf(w, v[i].y, a.y);
        a.z = fmaf(w, v[i].z, a.z);
        a.w = fmaf(w, v[i].w, a.w);
      }
    }
  }
  if (NG == 2) {
    a.x += __shfl_xor_sync(0xffffffffu, a.x, Q);
    a.y += __shfl_xor_sync(0xffffffffu, a.y, Q);
    a.z += __shfl_xor_sync(0xffffffffu, a.z, Q);
    a.w += __shfl_xor_sync(0xffffffffu, a.w, Q);
  }
  const float inv = tot == 0.f ? 0.f : 1.f / tot;
  const size_t orow = (size_t)kv_unit * rows_total + row_base + r;
  if (g == 0)
    *reinterpret_cast<uint2*>(o + orow * D + 4 * q) = make_uint2(pack_bf16x2(a.x * inv, a.y * inv), pack_bf16x2(a.z * inv, a.w * inv));
  if (lane == 0 && lse) lse[orow] = tot == 0.f ? -INFINITY : mx + logf(tot);
}

// ============================================================================ host side

namespace {

struct QtInfo {
  const void* fn;
  size_t smem;
  std::atomic<uint64_t>* allowed;
};
template <int D, int BC, int NB, int H>
QtInfo qt_info() {
  static std::atomic<uint64_t> allowed{0};
  return {reinterpret_cast<const void*>(&quant_tc_kernel<D, BC, NB, H>), QuantTcSmem<D, BC * NB, H>::kTotal, &allowed};
}
template <int D>
QtInfo qt_kernel(int rows) {
  return rows <= 8 ? qt_info<D, 8, 1, 1>() : rows <= 24 ? qt_info<D, 24, 1, 1>() : rows <= 32 ? qt_info<D, 32, 1, 1>()
         : rows <= 64 ? qt_info<D, 32, 1, 2>() : qt_info<D, 8, 6, 2>();
}
QtInfo qt_kernel(int d, int rows) { return d == 64 ? qt_kernel<64>(rows) : qt_kernel<128>(rows); }

constexpr int kQtMaxRows = 96;        // query rows of a unit

}  // namespace

static void cut_rows(int rows, QuantTcPlan* plan) {
  plan->chunks = (rows + kQtMaxRows - 1) / kQtMaxRows;
  plan->nq_rows = (rows + plan->chunks - 1) / plan->chunks;
}

bool quant_tc_plan(const bd_shape& s, int rows, int n_q, QuantTcPlan* plan) {
  cut_rows(rows, plan);
  plan->smem = qt_kernel(s.head_dim, plan->nq_rows).smem;
  plan->tiles_per_unit = (int)(((long)s.t_ctx + n_q + kQtKeys - 1) / kQtKeys);
  const long units = (long)s.batch * s.h_kv * plan->chunks, ctas = std::max(1, current_sm_count());
  // a: what a segment's start and end cost, in tiles (3, 6, 8, 11: 64 units of 16K, 24 rows 47.7, 46.5, 46.3, 46.0 us; 64
  // units of 4K 24.1, 22.9, 22.5, 22.6)
  const int tpu = plan->tiles_per_unit, a = 8;
  const long vtotal = units * (tpu + a);
  if (vtotal >= (1L << 31)) return false;
  long vtpc = (vtotal + ctas - 1) / ctas;
  vtpc = std::max<long>(vtpc, (tpu + a + kVMaxSeg - 2) / (kVMaxSeg - 1));   // <= kVMaxSeg segments
  plan->seg_cost = a;
  plan->tiles_per_cta = (int)vtpc;
  plan->grid = (int)((vtotal + vtpc - 1) / vtpc);
  int max_seg = 1;
  for (long u = 0; u < std::min(units, vtpc); ++u) {   // (units' offsets in the CTA ranges repeat after vtpc units)
    const int c0 = tile_owner((int)(u * tpu), tpu, a, (int)vtpc);
    const int c1 = tile_owner((int)(u * tpu + tpu - 1), tpu, a, (int)vtpc);
    max_seg = std::max(max_seg, c1 - c0 + 1);
  }
  if (max_seg > kVMaxSeg) return false;
  plan->max_seg = max_seg;
  if (s.seq_lens) {
    plan->tiles_per_cta = (int)((tpu + a + kVMaxSeg - 2) / (kVMaxSeg - 1));
    plan->max_seg = kVMaxSeg;
    plan->smem += align_up((size_t)(units + 1) * 4, 16);
    if (plan->smem > kMaxSmem) return false;
  }
  return true;
}

size_t quant_tc_bytes(const bd_shape& s, const QuantTcPlan& plan) {
  if (plan.max_seg <= 1) return 0;
  const size_t units = (size_t)s.batch * s.h_kv * plan.chunks, rows = units * plan.max_seg * plan.nq_rows;
  return align_up(rows * s.head_dim * 4, 256) + align_up(rows * 4, 256) + align_up(units * 4, 256);
}

// The mma.sync kernel starts in a third of the time and streams up to one n8 tile of rows as fast; every chunk of 8 rows
// reads the cache and unpacks it anew, several clusters of a unit meet in global memory.  So it takes short slices, and of
// more rows what an SM is soon done with.  mma.sync / tcgen05, us, d 128, 4 rows: 8 units of 1K 5.3 / 8.2, 64 of 4K 16.3 / 17.9, of
// 8K 25.6 / 24.3, 256 of 2K 24.8 / 30.6, 8 of 8K (four clusters) 11.3 / 10.6; 16 rows: 64 of 1K 11.3 / 13.6, of 4K 25.4 / 21.0, 8 of
// 8K 14.2 / 12.9; 24 rows: 8 of 1K 6.9 / 10.1, 64 of 0.5K 10.1 / 12.8, of 1K 14.8 / 14.1; 84 rows: 8 of 1K 9.0 / 15.5, 32 of 1K
// 21.4 / 18.8; d 64: 64 of 16K, 4 rows 28.0 / 32.8, of 4K, 16 rows 16.6 / 19.7, 24 rows 26.8 / 20.1, 8 of 2K, 84 rows 8.7 / 15.9, of
// 16K, 16 rows 13.4 / 12.6.
static bool warps_suit(const bd_shape& s, int rows, int n_q, const QuantAttnPlan& w) {
  const bool wide = s.head_dim == 128, one = w.clusters == 1;
  const long keys = (long)s.t_ctx + n_q;
  if (rows <= 8) return wide ? one && keys <= 6144 : w.per_split <= 5120;
  const long most = wide ? (one ? 1100 : 450) : (one ? 2700 : 1300);      // keys x chunks of an SM
  return w.one_wave && (long)s.batch * s.h_kv * ((rows + 7) / 8) * keys <= most * current_sm_count();
}

bool quant_verify_plan(const bd_shape& s, int rows, int n_q, QuantVerifyPlan* plan) {
  const bool w = quant_attn_plan(s, rows, (long)s.t_ctx + n_q, false, &plan->warps);
  plan->on_tc = !(w && warps_suit(s, rows, n_q, plan->warps)) && quant_tc_plan(s, rows, n_q, &plan->tc);
  if (!plan->on_tc && !w) return false;
  plan->bytes = plan->on_tc ? quant_tc_bytes(s, plan->tc) : quant_attn_bytes(s, rows, plan->warps);
  return true;
}

size_t quant_verify_room(const bd_shape& s, int rows) {
  // A unit's tpu tiles lie in at most ceil(tpu / vtpc) + 1 ranges of vtpc >= units (tpu + a) / ctas.
  QuantTcPlan tc = {};
  cut_rows(rows, &tc);
  const long units = (long)s.batch * s.h_kv * tc.chunks, ctas = std::max(1, current_sm_count());
  tc.max_seg = s.seq_lens ? kVMaxSeg : (int)std::min<long>(kVMaxSeg, (ctas + units - 1) / units + 1);
  QuantAttnPlan w;
  const bool on_warps = quant_attn_plan(s, rows, 1, false, &w);   // (its partials do not depend on the entries)
  return std::max(quant_tc_bytes(s, tc), on_warps ? quant_attn_bytes(s, rows, w) : 0);
}

cudaError_t launch_row_merge(int head_dim, const RowMerge& m, cudaStream_t stream) {
  const float* op = m.o_part;
  const float* lp = m.lse_part;
  const int* ns = m.nseg;
  int max_seg = m.max_seg, nq = m.nq_rows, total = m.rows_total, chunks = m.row_chunks;
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(m.o);
  float* l = m.lse;
  void* args[] = {&op, &lp, &ns, &max_seg, &nq, &total, &chunks, &o, &l};
  const void* fn = head_dim == 64 ? reinterpret_cast<const void*>(&quant_merge_kernel<64>) : reinterpret_cast<const void*>(&quant_merge_kernel<128>);
  return launch_kernel(fn, dim3(m.units, (nq + 3) / 4), dim3(128), 0, stream, args, 0);
}

cudaError_t launch_quant_tc(const bd_shape& s, const QuantTcPlan& plan, const QuantAttnCall& c, const bd_quant_cache& cache,
                            void* ws_region, int* status, cudaStream_t stream) {
  const int kv_units = s.batch * s.h_kv;
  CUtensorMap kmap, vmap;
  cudaError_t err = make_codes_map(&kmap, cache.k_codes, kv_units, s.t_cap, s.t_ctx + c.n_q, s.head_dim, kQtKeys);
  if (err == cudaSuccess) err = make_codes_map(&vmap, cache.v_codes, kv_units, s.t_cap, s.t_ctx + c.n_q, s.head_dim, kQtKeys);
  if (err != cudaSuccess) return err;
  QuantTcParams p;
  p.ks = static_cast<const uint16_t*>(cache.k_scales);
  p.vs = static_cast<const uint16_t*>(cache.v_scales);
  p.q = static_cast<const __nv_bfloat16*>(c.q);
  p.o = static_cast<__nv_bfloat16*>(c.o_out);
  p.lse = c.lse_out;
  p.units = kv_units * plan.chunks;
  const size_t rows = (size_t)p.units * plan.max_seg * plan.nq_rows;
  p.o_part = static_cast<float*>(ws_region);
  p.lse_part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws_region) + align_up(rows * s.head_dim * 4, 256));
  p.nseg = reinterpret_cast<int*>(reinterpret_cast<uint8_t*>(p.lse_part) + align_up(rows * 4, 256));
  p.status = status;
  p.seq_lens = s.seq_lens;
  p.h_kv = s.h_kv;
  p.n_q = c.n_q;
  p.nq_rows = plan.nq_rows;
  p.rows_total = c.rows;
  p.row_chunks = plan.chunks;
  p.t_ctx = s.t_ctx;
  p.t_cap = s.t_cap;
  p.tiles_per_unit = plan.tiles_per_unit;
  p.max_seg = plan.max_seg;
  p.seg_cost = plan.seg_cost;
  p.vtiles_per_cta = plan.tiles_per_cta;
  p.scale_log2 = kLog2e / sqrtf((float)s.head_dim);
  const QtInfo k = qt_kernel(s.head_dim, plan.nq_rows);
  err = allow_shared_memory_once(k.fn, 0, k.allowed);
  if (err != cudaSuccess) return err;
  void* args[] = {&p, &kmap, &vmap};
  err = launch_kernel(k.fn, dim3(plan.grid), dim3(kQtThreads), plan.smem, stream, args, 0);
  if (err != cudaSuccess || plan.max_seg <= 1) return err;
  return launch_row_merge(s.head_dim, {p.o_part, p.lse_part, p.nseg, plan.max_seg, plan.nq_rows, c.rows, plan.chunks, p.units, p.o, p.lse}, stream);
}

}  // namespace bd
