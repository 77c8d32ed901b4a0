// Rows that join a paged cache with their position rotation (bd_paged_append), and rows read back (bd_paged_read).
//
//   (x, y) -> s (x cos a - y sin a, x sin a + y cos a),  a = 2 pi frac(p f) for pair j's turns f a position
//
// The angle is exact for any position: f is held as 64 bits after the point, so that p f modulo 2^64 is one integer
// multiplication, and what is left of a full turn becomes the argument of sincospif.  A token's sines are worked out once
// by its CTA and shared by all its heads (a thread that worked them out for its own elements would spend more on them than on
// the rows).  Both kernels move each byte once.
#include <algorithm>

#include "bd_internal.h"
#include "bd_paged.cuh"

namespace bd {

constexpr int kPgThreads = 256;
constexpr int kPgTokens = 4;     // tokens of an append CTA

struct AppendRows {              // one source: element strides of a sequence, a head, a row
  const void* rows;
  long long sb, sh, sn;
};

struct AppendParams {
  AppendRows q, k, v;
  __nv_bfloat16* q_out;
  long long ob, oh, on;
  PagedTensor pk, pv;
  PageTable pages;
  const int32_t* seq_lens;
  const int32_t* row_starts;     // packed rows, or null
  const uint64_t* turns;
  int rot, interleaved;          // rotated elements of a row (0: none)
  float scale;
  int batch, t_ctx, t_cap, n_rows;
  long long total;               // tokens: batch * n_rows, or the packed rows
  int nq, nk, nv;                // rows of a token: heads of q, k, v (0: not this tensor)
  int rows_per_cta;              // rows of a token that a CTA takes (blockIdx.y: which)
  bool wide;                     // every source row is 32-byte aligned (fp32)
};

// Eight adjacent elements as floats.
template <typename T>
__device__ __forceinline__ void load8(const T* p, bool wide, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else if (wide) {
    asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                 : "l"(p));
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 v = reinterpret_cast<const float4*>(p)[i];
      x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
    }
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// The sequence that packed row r belongs to, by a whole warp: the last one that starts at or before it (32 probes a round).
__device__ __forceinline__ int sequence_of(const int32_t* starts, int batch, long long r, int lane) {
  int lo = 0, n = batch;
  while (n > 1) {
    const int step = (n + 31) / 32, at = lane * step;
    const uint32_t before = __ballot_sync(0xffffffffu, at < n && __ldcg(starts + lo + at) <= r);
    const int last = max(0, 31 - __clz(before));             // (starts ascend: the lanes that vote are the first ones)
    lo += last * step;
    n = min(step, n - last * step);
  }
  return lo;
}

struct Token {                   // a token's place, in shared memory
  long long src_row, out_row;    // its row among its sequence's (packed: among all)
  int seq, pos, page, row;       // page < 0: not written;  pos < 0: no token
};

template <int D, typename T>
__global__ void __launch_bounds__(kPgThreads) paged_append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int CH = D / 16, SLOTS = kPgThreads / CH;          // threads of a row; rows at a time
  __shared__ Token tok[kPgTokens];
  __shared__ float2 sc[kPgTokens][D / 2];                      // (cos, sin) of each pair, scaled
  grid_dependency_wait();
  allow_dependent_launch();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long t0 = (long long)blockIdx.x * kPgTokens;
  if (warp < kPgTokens) {                                      // a warp places a token
    const long long r = t0 + warp;
    Token k;
    k.pos = k.page = -1;
    k.seq = k.row = 0;
    k.src_row = 0;
    if (r < p.total) {
      long long i;
      bool mine = true;
      if (p.row_starts) {
        k.seq = sequence_of(p.row_starts, p.batch, r, lane);
        const int first = __ldcg(p.row_starts + k.seq);
        mine = r >= first && r < __ldcg(p.row_starts + k.seq + 1);
        i = r - first;
        k.src_row = r;
      } else {
        k.seq = (int)(r / p.n_rows);
        i = k.src_row = r - (long long)k.seq * p.n_rows;
      }
      const long long pos = paged_context(p.seq_lens, k.seq, p.t_ctx, nullptr) + i;
      if (mine && pos < p.t_cap) {
        k.pos = (int)pos;
        const int e = p.pages.entry(k.seq, k.pos);
        if (p.pages.there(e)) k.page = e;
        k.row = k.pos & ((1 << p.pages.shift) - 1);
      }
    }
    if (lane == 0) tok[warp] = k;
    // the angle as a signed part of a half turn, rounded once
    for (int j = lane; j < p.rot / 2; j += 32) {
      const long long phase = (long long)((unsigned long long)k.pos * __ldcg(reinterpret_cast<const unsigned long long*>(p.turns) + j));
      float s, c;
      sincospif((float)phase * 0x1p-63f, &s, &c);
      sc[warp][j] = make_float2(c * p.scale, s * p.scale);
    }
  }
  __syncthreads();

  const int c = tid % CH, half = p.rot / 2;
  const int row_end = min(p.nq + p.nk + p.nv, ((int)blockIdx.y + 1) * p.rows_per_cta), rows0 = blockIdx.y * p.rows_per_cta;
  const int rows = row_end - rows0;
  // this thread's 16 elements of a row: of a rotated one with its pairs' halves apart, two times eight
  const bool apart = !p.interleaved && 16 * c < p.rot;
  const int e0 = apart ? 8 * c : 16 * c, e1 = apart ? half + 8 * c : 16 * c + 8;
  for (int item = tid / CH; item < kPgTokens * rows; item += SLOTS) {
    const int ti = item / rows, r = rows0 + item - ti * rows;
    const Token k = tok[ti];
    if (k.pos < 0) continue;
    const int seq = p.row_starts ? 0 : k.seq;
    const bool is_q = r < p.nq, is_k = !is_q && r < p.nq + p.nk;
    const int head = is_q ? r : is_k ? r - p.nq : r - p.nq - p.nk;
    const AppendRows& s = is_q ? p.q : is_k ? p.k : p.v;
    if (!is_q && k.page < 0) continue;
    const T* src = static_cast<const T*>(s.rows) + seq * s.sb + head * s.sh + k.src_row * s.sn;
    float x[8], y[8];
    load8(src + e0, p.wide, x);
    load8(src + e1, p.wide, y);
    if ((is_q || is_k) && 16 * c < p.rot) {
      const float2* t = sc[ti] + 8 * c;
      if (apart) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 w = t[i];
          const float a = x[i], b = y[i];
          x[i] = fmaf(a, w.x, -(b * w.y));
          y[i] = fmaf(a, w.y, b * w.x);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 w = t[i], u = t[4 + i];
          const float a = x[2 * i], b = x[2 * i + 1], e = y[2 * i], f = y[2 * i + 1];
          x[2 * i] = fmaf(a, w.x, -(b * w.y));
          x[2 * i + 1] = fmaf(a, w.y, b * w.x);
          y[2 * i] = fmaf(e, u.x, -(f * u.y));
          y[2 * i + 1] = fmaf(e, u.y, f * u.x);
        }
      }
    }
    __nv_bfloat16* dst;
    if (is_q) {
      dst = p.q_out + seq * p.ob + head * p.oh + k.src_row * p.on;
    } else {
      const PagedTensor& to = is_k ? p.pk : p.pv;
      dst = to.base + k.page * to.sp + head * to.sh + k.row * to.sn;
    }
    store8(dst + e0, x);
    store8(dst + e1, y);
  }
  // the rows are in L2, for the copy engines' proxy too, before the CTA ends: an attention that follows reads them there
  fence_proxy_async_global();
  __threadfence();
}

// ---------------------------------------------------------------------------- rows read back

struct ReadTensor {
  __nv_bfloat16* out;
  long long sb, sh, sn;
  PagedTensor pool;
};
struct ReadParams {
  ReadTensor t[2];
  PageTable pages;
  const int32_t* seq_lens;
  int t_ctx, first, n_rows, h_kv, units;   // first < 0: the rows behind each sequence's length
  int blocks;                              // CTAs of a unit's rows
  bool wide;                               // 32-byte aligned everywhere
};
constexpr int kPgPasses = 4;               // rows of a thread

struct Half16 {                            // 16 elements as they lie
  uint32_t w[8];
  __device__ __forceinline__ void load(const void* p, bool wide) {
    if (wide) {
      asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                   : "l"(p));
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4 v = static_cast<const uint4*>(p)[i];
        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
      }
    }
  }
  __device__ __forceinline__ void store(void* p, bool wide) const {
    if (wide) {
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                   "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                   : "memory");
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) static_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
  }
};

// (No early trigger, and the rows in L2 for every proxy before the CTA ends: the selection and the contiguous verify block
// may stream context rows before their own dependency wait.)
template <int D>
__global__ void __launch_bounds__(kPgThreads) paged_read_kernel(const __grid_constant__ ReadParams p) {
  constexpr int CH = D / 16, STEP = kPgThreads / CH;
  grid_dependency_wait();
  const unsigned u = blockIdx.x / (unsigned)p.blocks, b = blockIdx.x - u * (unsigned)p.blocks;
  const int which = u >= (unsigned)p.units, unit = (int)u - which * p.units;
  const int seq = unit / p.h_kv, head = unit - seq * p.h_kv;
  const ReadTensor& t = p.t[which];
  const int len = paged_context(p.seq_lens, seq, p.t_ctx, nullptr);
  const int first = p.first < 0 ? len : p.first;
  const int n = p.first < 0 ? p.n_rows : min(p.n_rows, len - first);   // (may be negative)
  const int c = threadIdx.x % CH, row0 = (int)b * STEP * kPgPasses + threadIdx.x / CH;
  int e[kPgPasses];
#pragma unroll
  for (int i = 0; i < kPgPasses; ++i) {
    const int r = row0 + i * STEP;
    e[i] = r < n ? p.pages.entry(seq, first + r) : -1;
  }
  const __nv_bfloat16* pool = t.pool.base + head * t.pool.sh + 16 * c;
  Half16 x[kPgPasses] = {};
#pragma unroll
  for (int i = 0; i < kPgPasses; ++i) {
    const int in_page = (first + row0 + i * STEP) & ((1 << p.pages.shift) - 1);
    if (p.pages.there(e[i])) x[i].load(pool + e[i] * t.pool.sp + in_page * t.pool.sn, p.wide);
  }
  __nv_bfloat16* out = t.out + seq * t.sb + head * t.sh + 16 * c;
#pragma unroll
  for (int i = 0; i < kPgPasses; ++i) {
    const int r = row0 + i * STEP;
    if (r < n) x[i].store(out + (long long)r * t.sn, p.wide);
  }
  fence_proxy_async_global();
  __threadfence();
}

// ============================================================================ host side

static PagedTensor pool_tensor(void* base, const int64_t* st) { return {static_cast<__nv_bfloat16*>(base), st[0], st[1], st[2]}; }

cudaError_t launch_paged_append(const bd_shape& s, int n_rows, int dtype, const RowTensor& q, const RowTensor& k, const RowTensor& v,
                                const int32_t* row_starts, const bd_rope* rope, const bd_paged_cache& c, const int32_t* table,
                                int table_pages, const RowTensor& q_out, cudaStream_t stream) {
  AppendParams p;
  const int e = dtype == BD_DTYPE_F32 ? 4 : 2;
  p.wide = true;
  auto rows = [&](const RowTensor& t) {
    if (t.rows)
      p.wide &= reinterpret_cast<uintptr_t>(t.rows) % 32 == 0 && t.sb * e % 32 == 0 && t.sh * e % 32 == 0 && t.sn * e % 32 == 0;
    return AppendRows{t.rows, t.sb, t.sh, t.sn};
  };
  p.q = rows(q);
  p.k = rows(k);
  p.v = rows(v);
  p.q_out = static_cast<__nv_bfloat16*>(q_out.rows);
  p.ob = q_out.sb;
  p.oh = q_out.sh;
  p.on = q_out.sn;
  p.pk = pool_tensor(c.k, c.k_strides);
  p.pv = pool_tensor(c.v, c.v_strides);
  p.pages = {table, table_pages, c.n_pages, page_shift(c)};
  p.seq_lens = s.seq_lens;
  p.row_starts = row_starts;
  p.turns = rope ? rope->turns : nullptr;
  p.rot = rope ? rope->dim : 0;
  p.interleaved = rope ? rope->interleaved : 0;
  p.scale = rope ? rope->scale : 1.f;
  p.batch = s.batch;
  p.t_ctx = s.t_ctx;
  p.t_cap = s.t_cap;
  p.n_rows = n_rows;
  p.total = row_starts ? n_rows : (long long)s.batch * n_rows;
  p.nq = q.rows ? s.h_q : 0;
  p.nk = k.rows ? s.h_kv : 0;
  p.nv = v.rows ? s.h_kv : 0;
  const int all = p.nq + p.nk + p.nv, at_once = kPgThreads / (s.head_dim / 16);
  const long long blocks = (p.total + kPgTokens - 1) / kPgTokens;
  // few tokens: a token's rows spread over CTAs, a pass of rows each
  int split = 1;
  while (split < 64 && blocks * split < current_sm_count() && all * kPgTokens > at_once * split) split *= 2;
  p.rows_per_cta = (all + split - 1) / split;
  const void* fn = nullptr;
#define BD_PA(D, CODE, T) \
  if (s.head_dim == D && dtype == CODE) fn = reinterpret_cast<const void*>(&paged_append_kernel<D, T>);
  BD_PA(64, BD_DTYPE_BF16, __nv_bfloat16) BD_PA(128, BD_DTYPE_BF16, __nv_bfloat16)
  BD_PA(64, BD_DTYPE_F32, float) BD_PA(128, BD_DTYPE_F32, float)
#undef BD_PA
  void* args[] = {&p};
  return launch_kernel(fn, dim3((unsigned)blocks, (unsigned)((all + p.rows_per_cta - 1) / p.rows_per_cta)), dim3(kPgThreads), 0, stream,
                       args, 0);
}

cudaError_t launch_paged_read(const bd_shape& s, int first_row, int n_rows, const bd_paged_cache& c, const int32_t* table,
                              int table_pages, const RowTensor& k, const RowTensor& v, cudaStream_t stream) {
  ReadParams p;
  int n = 0;
  p.wide = true;
  for (int i = 0; i < 2; ++i) {
    const RowTensor& r = i ? v : k;
    if (!r.rows) continue;
    ReadTensor& t = p.t[n++];
    t = {static_cast<__nv_bfloat16*>(r.rows), r.sb, r.sh, r.sn, i ? pool_tensor(c.v, c.v_strides) : pool_tensor(c.k, c.k_strides)};
    for (long long st : {t.sb, t.sh, t.sn, t.pool.sp, t.pool.sh, t.pool.sn}) p.wide &= st % 16 == 0;
    p.wide &= reinterpret_cast<uintptr_t>(t.out) % 32 == 0 && reinterpret_cast<uintptr_t>(t.pool.base) % 32 == 0;
  }
  if (n == 1) p.t[1] = p.t[0];
  p.pages = {table, table_pages, c.n_pages, page_shift(c)};
  p.seq_lens = s.seq_lens;
  p.t_ctx = s.t_ctx;
  p.first = first_row;
  p.n_rows = n_rows;
  p.h_kv = s.h_kv;
  p.units = s.batch * s.h_kv;
  const int rows = kPgThreads / (s.head_dim / 16) * kPgPasses;
  p.blocks = (n_rows + rows - 1) / rows;
  const long long grid = (long long)p.blocks * p.units * n;
  if (grid >= (1LL << 31)) return cudaErrorInvalidConfiguration;
  const void* fn = s.head_dim == 64 ? reinterpret_cast<const void*>(&paged_read_kernel<64>) : reinterpret_cast<const void*>(&paged_read_kernel<128>);
  void* args[] = {&p};
  return launch_kernel(fn, dim3((unsigned)grid), dim3(kPgThreads), 0, stream, args, 0);
}

}  // namespace bd
