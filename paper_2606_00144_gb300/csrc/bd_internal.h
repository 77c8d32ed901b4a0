// Host-side plumbing shared by the translation units of libbudgetdraft: launch plans,
// workspace layout, tensor-map encoding and per-kernel launchers.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

#include "budgetdraft.h"

namespace bd {

// ---------------------------------------------------------------------------- device facts
int current_sm_count();   // SMs of the current device (cached per device)

// Launch with programmatic dependent launch allowed (the kernel may be scheduled while
// its predecessor finishes; every kernel of this library waits on the grid dependency before it
// writes anything or reads what the predecessor may have written, and some read older rows of the
// caches sooner) and, when cluster_x > 0, as clusters of cluster_x CTAs.
cudaError_t launch_kernel(const void* fn, dim3 grid, dim3 block, size_t smem, cudaStream_t stream,
                          void** args, int cluster_x);

// Shared memory a CTA may have, and permission for `fn` to ask for all of it beside static_bytes of its
// own.  The permission belongs to the function, not to a launch: set to each launch's own size, a thread
// could lower it between another one's setting and launching.
constexpr size_t kMaxSmem = 227 * 1024;
inline cudaError_t allow_shared_memory(const void* fn, size_t static_bytes = 0) {
  return cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kMaxSmem - static_bytes));
}
// The same, asked for once a device (`done`: the function's own, a bit for each device below 64).
inline cudaError_t allow_shared_memory_once(const void* fn, size_t static_bytes, std::atomic<uint64_t>* done) {
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done->load(std::memory_order_relaxed) & bit) return cudaSuccess;
  err = allow_shared_memory(fn, static_bytes);
  if (err == cudaSuccess) done->fetch_or(bit, std::memory_order_relaxed);
  return err;
}

// ---------------------------------------------------------------------------- workspace
// [0, 256): status word; [256, 256 + units*4 rounded to 256): per-unit arrival counters;
// then the op-specific region.
size_t ws_counters_offset();
size_t ws_region_offset(int units);

// ---------------------------------------------------------------------------- verify
struct VerifyPlan {
  int nq_rows;          // query rows per unit (a chunk of the group * n_q rows of a KV head)
  int rows_total;       // group * n_q
  int row_chunks;       // chunks of a (sequence, KV head): units = batch * h_kv * row_chunks
  int q_tiles;          // M tiles of query rows of verify_tc_kernel, 0: verify_kernel (mma.sync)
  int nt;               // verify_kernel: n8 tiles of query rows
  int tiles_per_unit;   // 64-key (verify_tc_kernel: 128-key) tiles over [0, t_ctx + n_q)
  int tiles_per_cta;    // contiguous range of the virtual tile list per CTA
  int seg_cost;         // virtual tiles before each unit's tiles (the cost of starting a unit)
  int grid;
  int max_seg;          // most CTAs that share one unit
  size_t smem_bytes;
  bool wide;            // more segments per unit than one staged merge round holds
};
bool verify_plan(const bd_shape& s, int n_q, VerifyPlan* plan);
// What a workspace for blocks of up to n_q queries holds beside its header.  A shorter block may need more
// partials than a longer one: on either side of 24 query rows the kernels differ, past 256 and 512 rows
// there are more, smaller units with fewer segments each, and at a tile's end the ranges are cut anew.
size_t verify_region_bytes(const bd_shape& s, int n_q);
size_t verify_partials_bytes(const bd_shape& s, const VerifyPlan& plan);
// q/o/lse as in bd_verify_attn; ws_region points at the op region, counters/status into ws.
cudaError_t launch_verify(const bd_shape& s, const VerifyPlan& plan, int n_q, const void* q,
                          const void* k_cache, const void* v_cache, void* o_out, float* lse_out,
                          void* ws_region, int* counters, int* status, cudaStream_t stream);

// ---------------------------------------------------------------------------- draft
struct DraftPlan {
  int n_split;          // CTAs of a cluster
  int n_clusters;       // clusters of a (sequence, KV head)
  int rows_per_split;   // entries of a CTA's slice
  bool longs;           // the LONG kernel instance
};
// room: bytes of the op region; a plan that needs more is not made.
bool draft_plan(const bd_shape& s, int budget, int n_steps, size_t room, DraftPlan* plan);
size_t draft_region_bytes(const bd_shape& s);
size_t draft_partials_bytes(const bd_shape& s, const DraftPlan& plan);
cudaError_t launch_draft(const bd_shape& s, const DraftPlan& plan, const void* q, const void* k_cache,
                         const void* v_cache, const int32_t* idx, const int32_t* count, int budget,
                         int step_j, unsigned flags, void* o_out, float* lse_out, void* ws_region,
                         int* counters, int* status, cudaStream_t stream);

// Allocation-free variant: scratch in a file-scope device array of this many bytes.
size_t draft_static_scratch_bytes();
cudaError_t draft_static_status(int* out, cudaStream_t stream);
cudaError_t launch_draft_static(const bd_shape& s, const DraftPlan& plan, const void* q, const void* k_cache,
                                const void* v_cache, const int32_t* idx, const int32_t* count, int budget,
                                int step_j, void* o_out, float* lse_out, cudaStream_t stream);

// ---------------------------------------------------------------------------- row normalisers
// Softmax normalisers of the last `window` positions' queries over their causal prefixes of a
// t_ctx-row cache: the selection's self mode, and bd_verify_attn without an output (whose
// block is the last n_q positions of a context of t_ctx + n_q).
struct LsePlan {
  int nq_rows;             // group * window query rows per KV head, at most 128
  int tiles_per_unit, total_tiles, tiles_per_cta, grid, max_seg;
  size_t smem_bytes, part_bytes;
};
bool lse_plan(const bd_shape& s, int window, LsePlan* plan);
// The context whose last n_q positions are the block's rows.
inline bd_shape block_context(const bd_shape& s, int n_q) {
  bd_shape ls = s;
  ls.t_ctx = s.t_ctx + n_q;
  return ls;
}
// The same for a block without an output of up to n_q queries behind a context of s.t_ctx.
size_t lse_region_bytes(const bd_shape& s, int n_q);
// len_offset is added to every sequence's length (seq_lens); part: plan.part_bytes of scratch.
cudaError_t launch_lse(const bd_shape& s, const LsePlan& plan, const void* k_cache, const void* q, int window,
                       int len_offset, bool window_ready, bool hide_nan, float* lse_out, void* part, int* counters,
                       int* status, cudaStream_t stream);

// ---------------------------------------------------------------------------- select
struct SelectPlan {
  bool keep_all;        // budget >= t_ctx
  bool need_scores;     // some middle position (chunk) must be ranked
  int nq_rows, nq_pad;  // window query rows per KV head (padded to 16)
  int n_mid, n_mid_pad;
  int tiles_per_unit, total_tiles, grid, tiles_per_cta;
  int stages;           // K tiles in flight
  int nqb;              // window-query tile buffers
  int n_acc;            // TMEM accumulators
  uint32_t tmem_cols;
  size_t smem_bytes;
  size_t score_bytes, lse_bytes;
  bool self_mode;       // the window LSE can be computed here (at most 128 window rows per KV head)
  LsePlan lse;
};
bool select_plan(const bd_shape& s, int window, int budget, int n_sink, int n_recent, int chunk,
                 SelectPlan* plan);
size_t select_region_bytes(const bd_shape& s, const SelectPlan& plan);
cudaError_t launch_select(const bd_shape& s, const SelectPlan& plan, const void* k_cache,
                          const void* q_window, const float* window_lse, int window, int budget,
                          int n_sink, int n_recent, int chunk, unsigned flags, int32_t* idx_out, int32_t* count_out,
                          void* ws_region, int* counters, int* status, cudaStream_t stream);

// ---------------------------------------------------------------------------- combine
// Largest part count of bd_combine: one row's merge weights (n_split floats) must fit the
// 48 KB of dynamic shared memory a launch gets without opting in.
constexpr int kCombineMaxSplit = 12288;
cudaError_t launch_combine(const float* o_part, const float* lse_part, int n_split, int rows,
                           int head_dim, void* o_out, float* lse_out, cudaStream_t stream);
int combine_rows_per_block(int n_split);
cudaError_t launch_wait_probe(int* status, long long limit_us, cudaStream_t stream);

// ---------------------------------------------------------------------------- acceptance
int argmax_cluster(int rows, int vocab);   // CTAs per row
cudaError_t launch_argmax(const void* logits, bool bf16, int rows, int vocab, int32_t* ids_out,
                          cudaStream_t stream);
cudaError_t launch_accept(int batch, int gamma, const int32_t* draft_tokens, const int32_t* verify_tokens,
                          int32_t* n_accept, int32_t* emit, cudaStream_t stream);
size_t advance_smem(int window, int head_dim);
cudaError_t launch_write_rows(const bd_shape& s, int n_rows, const void* k_rows, const void* v_rows, void* k_cache,
                              void* v_cache, cudaStream_t stream);
cudaError_t launch_advance(const bd_shape& s, int window, int n_q, const int32_t* n_accept, const void* q_verify,
                           const float* verify_lse, void* q_window, float* window_lse, int32_t* idx, int32_t* count,
                           int capacity, int32_t* advance_out, cudaStream_t stream);

// ---------------------------------------------------------------------------- 4-bit caches
struct QuantTensor {    // one tensor's rows of a write or a read: strides in elements; rows null: not this tensor
  void* rows;
  long long sb, sh, sn;
};
cudaError_t launch_quant_write(const bd_shape& s, int n_rows, int dtype, const bd_quant_cache& c, const QuantTensor& k,
                               const QuantTensor& v, cudaStream_t stream);
// first_row < 0: the rows behind each sequence's length.
cudaError_t launch_quant_read(const bd_shape& s, int first_row, int n_rows, int dtype, const bd_quant_cache& c,
                              const QuantTensor& k, const QuantTensor& v, cudaStream_t stream);

struct QuantAttnCall {
  const void* q;        // [units][rows][head_dim]
  void* o_out;
  float* lse_out;
  int rows;             // query rows of a KV head: group * n_q
  int n_q;              // queries per head (a drafter pass: 1)
  const int32_t* idx;   // a drafter pass's view (null: a verify block)
  const int32_t* count;
  int budget, step_j;
  bool view_ready;      // BD_DRAFT_VIEW_READY
};
struct QuantAttnPlan {
  int nt, chunks;       // n8 tiles of a CTA's query rows; chunks of a KV head's rows
  int per_split, warps; // entries and warps of a CTA
  int cluster, clusters;   // CTAs of a cluster, clusters of a unit
  int most_clusters;    // the most that any number of entries takes
  bool one_wave;        // the device holds every CTA at once
};
// entries: the most that a unit attends to; gather: they come from a view
bool quant_attn_plan(const bd_shape& s, int rows, long entries, bool gather, QuantAttnPlan* plan);
// Op region for any number of entries with this many query rows.
size_t quant_attn_bytes(const bd_shape& s, int rows, const QuantAttnPlan& plan);
cudaError_t launch_quant_attn(const bd_shape& s, const QuantAttnPlan& plan, const QuantAttnCall& c, const bd_quant_cache& cache,
                              void* ws_region, int* counters, int* status, cudaStream_t stream);

// Verify blocks on the tcgen05 kernel.
struct QuantTcPlan {
  int chunks, nq_rows;  // chunks of a KV head's query rows, rows of one: units = batch * h_kv * chunks
  int tiles_per_unit, tiles_per_cta, seg_cost, grid, max_seg;   // as in VerifyPlan, of 128 keys
  size_t smem;
};
bool quant_tc_plan(const bd_shape& s, int rows, int n_q, QuantTcPlan* plan);
size_t quant_tc_bytes(const bd_shape& s, const QuantTcPlan& plan);
cudaError_t launch_quant_tc(const bd_shape& s, const QuantTcPlan& plan, const QuantAttnCall& c, const bd_quant_cache& cache,
                            void* ws_region, int* status, cudaStream_t stream);

// Which kernel takes a verify block, and its plan.
struct QuantVerifyPlan {
  bool on_tc;
  QuantTcPlan tc;
  QuantAttnPlan warps;
  size_t bytes;         // op region
};
bool quant_verify_plan(const bd_shape& s, int rows, int n_q, QuantVerifyPlan* plan);
// Op region for this many query rows behind any context: the kernel that takes them and how a unit is cut follow the context.
size_t quant_verify_room(const bd_shape& s, int rows);

// Merge of partials laid out [units][max_seg][nq_rows][head_dim] (lse_part [units][max_seg][nq_rows]), nseg[unit] of them,
// into the rows of units that have more than one.
struct RowMerge {
  const float* o_part;
  const float* lse_part;
  const int* nseg;
  int max_seg, nq_rows, rows_total, row_chunks, units;
  void* o;
  float* lse;
};
cudaError_t launch_row_merge(int head_dim, const RowMerge& m, cudaStream_t stream);

// ---------------------------------------------------------------------------- paged caches
using RowTensor = QuantTensor;
inline int page_shift(const bd_paged_cache& c) {
  int n = 0;
  while (1 << n < c.page_size) ++n;
  return n;
}
cudaError_t launch_paged_append(const bd_shape& s, int n_rows, int dtype, const RowTensor& q, const RowTensor& k, const RowTensor& v,
                                const int32_t* row_starts, const bd_rope* rope, const bd_paged_cache& c, const int32_t* table,
                                int table_pages, const RowTensor& q_out, cudaStream_t stream);
cudaError_t launch_paged_read(const bd_shape& s, int first_row, int n_rows, const bd_paged_cache& c, const int32_t* table,
                              int table_pages, const RowTensor& k, const RowTensor& v, bool nan_absent, cudaStream_t stream);

cudaError_t launch_paged_draft(const bd_shape& s, const DraftPlan& plan, const void* q, const bd_paged_cache& c,
                               const int32_t* table, int table_pages, const int32_t* idx, const int32_t* count, int budget,
                               int step_j, unsigned flags, void* o_out, float* lse_out, void* ws_region, int* counters,
                               int* status, cudaStream_t stream);

// Verify blocks.
struct PagedVerifyPlan {
  int q_tiles;          // M tiles of a unit's query rows on the tcgen05 kernel, 0: the mma.sync kernel
  int nt;               // mma.sync: n8 tiles of a unit's query rows
  int cluster;          // mma.sync: CTAs of a unit, as a cluster; 0: ranges of the tile list
  int stages;           // a cluster's CTA: tiles in flight
  int chunks, nq_rows;  // chunks of a KV head's query rows, rows of one: units = batch * h_kv * chunks
  int tiles_per_unit, tiles_per_cta, seg_cost, grid, max_seg;   // as in VerifyPlan
  size_t smem;
};
bool paged_verify_plan(const bd_shape& s, int rows, int n_q, PagedVerifyPlan* plan);
size_t paged_verify_bytes(const bd_shape& s, const PagedVerifyPlan& plan);
// Op region for this many query rows behind any context.
size_t paged_verify_room(const bd_shape& s, int rows);
cudaError_t launch_paged_verify(const bd_shape& s, const PagedVerifyPlan& plan, int rows, int n_q, const void* q,
                                const bd_paged_cache& c, const int32_t* table, int table_pages, void* o_out, float* lse_out,
                                void* ws_region, int* status, cudaStream_t stream);

// ---------------------------------------------------------------------------- TMA maps
// 5-D map over one tensor of a pool: 64 columns x rows of a page x 64-column halves of a row x KV heads x pages, 128-byte
// swizzle.  Box = 64 columns x box_rows rows x box_halves halves; pages that the pool has not read as zero.
cudaError_t make_paged_map(CUtensorMap* map, const void* base, const int64_t* strides, int head_dim, int h_kv, int page_size,
                           int n_pages, int box_rows, int box_halves);
// 3-D map over a [units, rows_total (stride t_cap), head_dim] bf16 cache: only rows
// [0, n_rows) of each unit are addressable (the rest reads as zero).  Box = 64 columns x
// box_rows rows x 1 unit, 128-byte swizzle.
cudaError_t make_cache_map(CUtensorMap* map, const void* base, int units, int t_cap, int n_rows,
                           int head_dim, int box_rows);
// 3-D map over a [units, n_rows (stride t_cap), head_dim / 2] array of 4-bit codes, rows past n_rows reading as zero.
// Box = a whole row x box_rows rows x 1 unit, swizzled over the row's 64 (32) bytes.
cudaError_t make_codes_map(CUtensorMap* map, const void* base, int units, int t_cap, int n_rows, int head_dim, int box_rows);
// 2-D map over a dense [n_rows, head_dim] bf16 matrix; box = 64 columns x box_rows rows,
// 128-byte swizzle; rows past n_rows read as zero.
cudaError_t make_rows_map(CUtensorMap* map, const void* base, long long n_rows, int head_dim, int box_rows);

}  // namespace bd
