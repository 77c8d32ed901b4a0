// What the kernels over a paged cache (include/budgetdraft.h, bd_paged_cache) share.
#pragma once

#include "bd_common.cuh"

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

// Boxes of the pool's tensor map (make_paged_map): 64 columns x rows x halves x head x page.
__device__ __forceinline__ void tma_load_page(void* dst, const CUtensorMap* map, uint64_t* bar, int row, int half, int head, int page) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(half), "r"(head), "r"(page), "r"(smem_u32(bar))
      : "memory");
}
// What other kernels wrote is read through the async proxy from here on (after the dependency wait).
__device__ __forceinline__ void fence_proxy_async_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }

}  // namespace bd
