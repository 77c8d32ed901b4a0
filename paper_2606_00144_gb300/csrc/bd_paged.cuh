// What the kernels over a paged cache (include/budgetdraft.h, bd_paged_cache) share.
#pragma once

#include "bd_common.cuh"
#include "bd_verify.cuh"

namespace bd {

// One tensor of the pool: elements from a page, a KV head and a row to the next.
struct PagedTensor {
  __nv_bfloat16* base;
  long long sp, sh, sn;
};

// The pages of the batch's positions.
struct PageTable {
  const int32_t* table;        // [batch][pages]
  int pages;                   // entries of a sequence
  int n_pages;                 // of the pool
  int shift;                   // log2 of a page's rows
  __device__ __forceinline__ int entry(int seq, int pos) const { return __ldcg(table + (long long)seq * pages + (pos >> shift)); }
  __device__ __forceinline__ bool there(int e) const { return (unsigned)e < (unsigned)n_pages; }
};

// Context length of sequence `seq`; one outside [0, t_ctx] is recorded as an argument error and clamped.
__device__ __forceinline__ int paged_context(const int32_t* seq_lens, int seq, int t_ctx, int* status) {
  if (seq_lens == nullptr) return t_ctx;
  int t = __ldcg(seq_lens + seq);
  if (t < 0 || t > t_ctx) {
    if (status) record_error(status, BD_ERR_INVALID_ARG);
    t = min(max(t, 0), t_ctx);
  }
  return t;
}

// Boxes of the pool's tensor map (make_paged_map): 64 columns x rows x halves x head x page.  Issued by the lane with lead
// != 0 of a whole warp whose operands are alike (see tc_mma_ss).
__device__ __forceinline__ void tma_load_page(uint32_t lead, uint32_t dst, const CUtensorMap* map, uint64_t* bar, int row, int half, int head, int page) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %0, 0;\n\t"
      "@q cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%1], [%2, {%3, %4, %5, %6, %7}], [%8];\n\t}" ::"r"(lead),
      "r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(half), "r"(head), "r"(page), "r"(smem_u32(bar))
      : "memory");
}
// What other kernels wrote is read through the async proxy from here on (after the dependency wait).
__device__ __forceinline__ void fence_proxy_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }


// The virtual tile list of a verify block (as VerifyMap): unit u's `a` virtual tiles, then its real ones.  A sequence's units
// (KV heads x chunks) are alike, so the table for per-sequence lengths, pref, only says where each sequence's units begin
// (null: every unit has span0 - a tiles).
struct PagedMap {
  const int* pref;
  int span0, a, per_seq, batch, vtpc;
  __device__ __forceinline__ static constexpr int stride() { return 1; }   // from a segment's tile to its next one
  __device__ __forceinline__ int seq_of(int u) const { return u / per_seq; }
  __device__ __forceinline__ int seq_base(int b) const { return pref ? pref[b] : b * per_seq * span0; }
  __device__ __forceinline__ int span(int b) const { return pref ? (pref[b + 1] - pref[b]) / per_seq : span0; }
  __device__ __forceinline__ int real_base(int u) const {    // the unit's first real tile
    const int b = seq_of(u);
    return seq_base(b) + (u - b * per_seq) * span(b) + a;
  }
  __device__ __forceinline__ int tiles(int u) const { return span(seq_of(u)) - a; }
  __device__ __forceinline__ int first_tile(int u, int v0) const { return max(0, v0 - real_base(u)); }
  __device__ __forceinline__ int end_tile(int u, int v1) const { return min(tiles(u), v1 - real_base(u)); }
  __device__ __forceinline__ int owner(int u, int tile) const { return (real_base(u) + tile) / vtpc; }
  __device__ __forceinline__ int unit_of(int v) const {
    int b = 0;
    if (!pref) {
      b = v / (per_seq * span0);
    } else {
      int hi = batch - 1;
      while (b < hi) {
        const int mid = (b + hi + 1) >> 1;
        if (pref[mid] <= v) b = mid;
        else hi = mid - 1;
      }
    }
    return b * per_seq + (v - seq_base(b)) / span(b);
  }
  // Lays the sequences out in `table` (shared, batch + 1 ints) and cuts the list anew over their tiles.
  template <int NTHREADS, int KEYS>
  __device__ __forceinline__ void lay_out(const int32_t* seq_lens, int t_ctx, int n_q, int least, int* wtot, int* table) {
    auto tiles_of = [&](int b) { return per_seq * ((paged_context(seq_lens, b, t_ctx, nullptr) + n_q + KEYS - 1) / KEYS + a); };
    lay_out_spans<NTHREADS>(batch, tiles_of, wtot, table);
    pref = table;
    vtpc = max((table[batch] + (int)gridDim.x - 1) / (int)gridDim.x, least);
  }
};

// A producer warp's walk over its CTA's segments (a segment: the tiles of a unit in the CTA's range), and the pages of a
// segment's pieces (a piece: a page's rows of a tile, or the whole tile), 32 looked up at once, a lane each.
template <int KEYS, typename Map, typename Params>
struct PageWalk {
  const Map& map;
  const Params& p;
  int u_last, v0, v1;
  struct Segment {
    int unit, tb, n, seq, head, end;   // n tiles, the first tb; end: rows of the sequence, its block's among them (unit > u_last: none)
  };
  __device__ __forceinline__ Segment from(int unit) const {
    Segment s{unit, 0, 0, 0, 0, 0};
    for (; s.unit <= u_last; ++s.unit) {
      s.tb = map.first_tile(s.unit, v0);
      s.n = (map.end_tile(s.unit, v1) - s.tb + map.stride() - 1) / map.stride();
      if (s.n <= 0) continue;
      s.seq = map.seq_of(s.unit);
      s.head = s.unit / p.row_chunks - s.seq * p.h_kv;
      s.end = paged_context(p.seq_lens, s.seq, p.t_ctx, nullptr) + p.n_q;
      return s;
    }
    s.n = 0;
    return s;
  }
  // The entry of the segment's piece first + lane (nothing looks at it here, so that the load is on its way while others are
  // used); negative past the segment and the sequence's rows.
  __device__ __forceinline__ int entry(const Segment& s, int first, int lane) const {
    const int at = first + lane, n_box = KEYS >> p.box_shift, i = at << p.box_shift & ~(KEYS - 1);   // (the tiles before, in keys)
    const int key = s.tb * KEYS + i * map.stride() + ((at << p.box_shift) - i);
    return at < s.n * n_box && key < s.end ? p.pages.entry(s.seq, key) : -1;
  }
};

// A verify block on the tcgen05 kernel, which has a second producer warp then.
constexpr int kPagedTcThreads = kVTcThreads + 32;
struct PagedTcParams : VerifyParams {
  PageTable pages;
  int box_shift;       // log2 of a box's rows
  int batch;
};
// Its instance for q_tiles M tiles of query rows per unit, and for boxes of 16 rows and both halves of a row (head_dim 128) or
// of a half; it takes 16 + head_dim ints of shared memory beside the sequences' table.
const void* paged_tc_fn(int head_dim, int q_tiles, bool box16);

// Rows [r0, r1) of a V tile in shared memory are hidden from some of the block's queries, to whom 0 times a NaN would be
// NaN: elements that are no finite number become zero, and from[column] the first row of the block that has one there (the
// queries that see it have NaN written at the end).  first: row r0's index in the block; the tile's rows lie in pieces of 2^ps
// rows, each [half][row][128 B].
template <int D>
__device__ __noinline__ void scrub_rows(uint32_t tile, int ps, int r0, int r1, int first, int* from, int lane) {
  constexpr int CH = D / 8;
  bool any = false;
  for (int i = lane; i < (r1 - r0) * CH; i += 32) {
    const int r = r0 + i / CH, col = i % CH * 8;
    const uint32_t at = tile + ((uint32_t)(r >> ps) * (2 * D) << ps) + sw128_offset(r & ((1 << ps) - 1), col, 128u << ps);
    uint32_t w[4];
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if ((w[e] & 0x7f80u) == 0x7f80u) atomicMin(from + col + 2 * e, first + r - r0), w[e] &= 0xffff0000u, odd = true;
      if ((w[e] & 0x7f800000u) == 0x7f800000u) atomicMin(from + col + 2 * e + 1, first + r - r0), w[e] &= 0xffffu, odd = true;
    }
    if (odd) asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    any |= odd;
  }
  if (__any_sync(0xffffffffu, any)) fence_proxy_async_smem();      // (before the next copy into this stage)
  __syncwarp();
}

}  // namespace bd
