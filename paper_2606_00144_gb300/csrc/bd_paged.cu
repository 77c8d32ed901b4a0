// Rows that join a paged cache with their position rotation (bd_paged_append), and rows read back (bd_paged_read, bd_paged_keys).
//
//   (x, y) -> s (x cos a - y sin a, x sin a + y cos a),  a = 2 pi frac(p f) for pair j's turns f a position
//
// The angle is exact for any position: f is held as 64 bits after the point, so that p f modulo 2^64 is one integer
// multiplication, and what is left of a full turn becomes the argument of sincospif.  A token's sines are worked out once
// by its CTA and shared by all its heads (a thread that worked them out for its own elements would spend more on them than on
// the rows).  Both kernels move each byte once and are bound by HBM where there is enough: 4 x 8192 tokens of 48 rows of 128
// (805 MB) are appended in 128 us (6.3 TB/s), the keys of 8 x 16K positions of 8 heads (537 MB) read in 82 (6.5 TB/s).
#include <algorithm>

#include "bd_internal.h"
#include "bd_paged.cuh"

namespace bd {

constexpr int kPgThreads = 256;
constexpr int kPgTokens = 32;    // most tokens of an append CTA: a warp places four
constexpr int pg_ahead(int elem_bytes) { return elem_bytes == 2 ? 2 : 1; }   // (4 and 2: 3 % and 8 % longer, in fewer warps or spilled)

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
  int total;                     // tokens: batch * n_rows, or the packed rows
  int nq, nk, nv;                // rows of a token: heads of q, k, v (0: not this tensor)
  int tokens;                    // of a CTA
  int row_shift;                 // log2 of the rows of a token that a CTA walks side by side
  int rows_per_cta;              // rows of a token that a CTA takes (blockIdx.y: which)
  bool wide;                     // every source row is 32-byte aligned (fp32)
};

// Eight adjacent elements as they lie.
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, bool) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
};
template <>
struct Eight<float> {
  float w[8];
  __device__ __forceinline__ void load(const float* p, bool wide) {
    if (wide) {
      asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=f"(w[0]), "=f"(w[1]), "=f"(w[2]), "=f"(w[3]), "=f"(w[4]), "=f"(w[5]), "=f"(w[6]), "=f"(w[7])
                   : "l"(p));
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 v = reinterpret_cast<const float4*>(p)[i];
        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
      }
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = w[i];
  }
};
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// The sequence that packed row r belongs to, by a whole warp: the last one that starts at or before it, found with 32 probes a
// round; probe: the first round's, starts[lane * ceil(batch / 32)].
__device__ __forceinline__ int sequence_of(const int32_t* starts, int batch, int probe, int r, int lane) {
  int lo = 0, n = batch;
  while (n > 1) {
    const int step = (n + 31) / 32, at = lane * step;
    if (n < batch && at < n) probe = __ldcg(starts + lo + at);
    const uint32_t before = __ballot_sync(0xffffffffu, at < n && probe <= r);
    const int last = max(0, 31 - __clz(before));             // (starts ascend: the lanes that vote are the first ones)
    lo += last * step;
    n = min(step, n - last * step);
  }
  return lo;
}

struct Token {                   // a token of a CTA, in shared memory; q, k, v:
  long long src[3], dst[3];      // where its rows of head 0 lie in the sources, in q_out and the pool
  int live;                      // 1: its query is written, 2: its key and value are
};

// A thread keeps its place in a row and walks the CTA's tokens, several in flight, so that what it costs to find a row is an
// addition.  A CTA's threads take so many rows side by side that they divide a token's, and as many tokens as that leaves.  The
// first rows are asked for before their tokens' places are known.
template <int D, typename T>
__global__ void __launch_bounds__(kPgThreads, 4) paged_append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int CH = D / 16, SLOTS = kPgThreads / CH;          // threads of a row; rows at a time
  constexpr int AHEAD = pg_ahead(sizeof(T));                   // tokens in flight of a thread
  __shared__ Token tok[kPgTokens];
  __shared__ float2 sc[kPgTokens][D / 2];                      // (cos, sin) of each pair, scaled
  grid_dependency_wait();
  allow_dependent_launch();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int t0 = blockIdx.x * p.tokens, tokens = min(p.tokens, p.total - t0);
  if (tid < tokens) {
    const int g = t0 + tid, s = p.row_starts ? 0 : g / p.n_rows;
    const long long seq = s, at = g - s * p.n_rows;
    tok[tid].src[0] = seq * p.q.sb + at * p.q.sn;
    tok[tid].src[1] = seq * p.k.sb + at * p.k.sn;
    tok[tid].src[2] = seq * p.v.sb + at * p.v.sn;
    tok[tid].dst[0] = seq * p.ob + at * p.on;
  }
  __syncthreads();

  const int rows = min(p.nq + p.nk + p.nv, ((int)blockIdx.y + 1) * p.rows_per_cta);
  const int c = tid % CH, slot = tid / CH, half = p.rot / 2;
  const int row_slots = 1 << p.row_shift, tok_slots = SLOTS >> p.row_shift, first_tok = slot >> p.row_shift;
  // this thread's 16 elements of a row: of a rotated one with its pairs' halves apart, two times eight
  const bool turned = 16 * c < p.rot, apart = !p.interleaved && turned;
  const int e0 = apart ? 8 * c : 16 * c, step = apart ? half : 8;
  Eight<T> x[AHEAD], y[AHEAD];
  int row = (int)blockIdx.y * p.rows_per_cta + (slot & (row_slots - 1)), kind = 0;
  if (first_tok >= tokens) row = rows;
  const T* src = nullptr;
  __nv_bfloat16* dst = nullptr;
  auto start_row = [&] {
    kind = row < p.nq ? 0 : row < p.nq + p.nk ? 1 : 2;
    const int head = row - (kind > 0 ? p.nq : 0) - (kind > 1 ? p.nk : 0);
    const AppendRows& s = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
    src = static_cast<const T*>(s.rows) + head * s.sh + e0;
    dst = (kind == 0 ? p.q_out + head * p.oh : kind == 1 ? p.pk.base + head * p.pk.sh : p.pv.base + head * p.pv.sh) + e0;
  };
  auto load = [&](int t) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (t + i * tok_slots < tokens) {
        const T* from = src + tok[t + i * tok_slots].src[kind];
        x[i].load(from, p.wide);
        y[i].load(from + step, p.wide);
      }
  };
  if (row < rows) {
    start_row();
    load(first_tok);
  }

  // a warp places the tokens warp, warp + 8, ..., lane k the k-th of them
  constexpr int WARPS = kPgThreads / 32;
  unsigned long long turns[D / 64];                            // of this lane's pairs
#pragma unroll
  for (int j = 0; j < D / 64; ++j)
    turns[j] = lane + 32 * j < half ? __ldcg(reinterpret_cast<const unsigned long long*>(p.turns) + lane + 32 * j) : 0;
  long long my_pos = 0;
  {
    int seq = 0, i = 0;
    bool mine = false;
    const int probe = p.row_starts && lane * ((p.batch + 31) / 32) < p.batch ? __ldcg(p.row_starts + lane * ((p.batch + 31) / 32)) : 0;
    for (int k = 0; warp + k * WARPS < tokens; ++k) {
      const int r = t0 + warp + k * WARPS;
      if (p.row_starts) {
        const int found = sequence_of(p.row_starts, p.batch, probe, r, lane);
        if (lane == k) seq = found, i = r, mine = true;
      } else if (lane == k) {
        seq = r / p.n_rows;
        i = r - seq * p.n_rows;
        mine = true;
      }
    }
    if (mine) {
      if (p.row_starts) {
        const int first = __ldcg(p.row_starts + seq);
        mine = first >= 0 && i >= first && i < __ldcg(p.row_starts + seq + 1);
        i -= first;
      }
      my_pos = (long long)paged_context(p.seq_lens, seq, p.t_ctx, nullptr) + i;
      const bool live = mine && my_pos < p.t_cap;
      const int e = live ? p.pages.entry(seq, (int)my_pos) : -1;
      const bool there = p.pages.there(e);
      const long long page = there ? e : 0, in_page = my_pos & ((1 << p.pages.shift) - 1);
      Token& k = tok[warp + lane * WARPS];
      k.dst[1] = page * p.pk.sp + in_page * p.pk.sn;
      k.dst[2] = page * p.pv.sp + in_page * p.pv.sn;
      k.live = (live ? 1 : 0) | (there ? 2 : 0);
    }
  }
  for (int k = 0; warp + k * WARPS < tokens; ++k) {
    const unsigned long long pos = (unsigned long long)__shfl_sync(0xffffffffu, my_pos, k);
    // the angle as a signed part of a half turn, rounded once
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      float s, c;
      sincospif((float)(long long)(pos * turns[j]) * 0x1p-63f, &s, &c);
      if (lane + 32 * j < half) sc[warp + k * WARPS][lane + 32 * j] = make_float2(c * p.scale, s * p.scale);
    }
  }
  __syncthreads();

  for (int t = first_tok; row < rows;) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int ti = t + i * tok_slots;
      if (ti >= tokens) break;
      const Token& k = tok[ti];
      if (!(k.live & (kind == 0 ? 1 : 2))) continue;
      __nv_bfloat16* to = dst + k.dst[kind];
      if constexpr (sizeof(T) == 2) {
        if (kind == 2 || !turned) {                            // as they are
          *reinterpret_cast<uint4*>(to) = x[i].w;
          *reinterpret_cast<uint4*>(to + step) = y[i].w;
          continue;
        }
      }
      float a[8], b[8];
      x[i].get(a);
      y[i].get(b);
      if (kind < 2 && turned) {
        const float4* v = reinterpret_cast<const float4*>(sc[ti] + 8 * c);   // two pairs' (cos, sin)
        if (apart) {
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const float4 w = v[e / 2];
            const float a0 = a[e], a1 = a[e + 1], b0 = b[e], b1 = b[e + 1];
            a[e] = fmaf(a0, w.x, -(b0 * w.y));
            b[e] = fmaf(a0, w.y, b0 * w.x);
            a[e + 1] = fmaf(a1, w.z, -(b1 * w.w));
            b[e + 1] = fmaf(a1, w.w, b1 * w.z);
          }
        } else {
          auto pairs = [](float (&z)[8], const float4* v) {
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
              const float4 w = v[e / 4];
              const float z0 = z[e], z1 = z[e + 1], z2 = z[e + 2], z3 = z[e + 3];
              z[e] = fmaf(z0, w.x, -(z1 * w.y));
              z[e + 1] = fmaf(z0, w.y, z1 * w.x);
              z[e + 2] = fmaf(z2, w.z, -(z3 * w.w));
              z[e + 3] = fmaf(z2, w.w, z3 * w.z);
            }
          };
          pairs(a, v);
          pairs(b, v + 2);
        }
      }
      store8(to, a);
      store8(to + step, b);
    }
    t += AHEAD * tok_slots;
    if (t >= tokens) {
      t = first_tok;
      row += row_slots;
      if (row < rows) start_row();
    }
    if (row < rows) load(t);
  }
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
  uint32_t absent;                         // two elements of a row whose page is not there
  bool wide;                               // 32-byte aligned everywhere
};
constexpr int kPgPasses = 4;               // rows of a thread

struct Half16 {                            // 16 elements as they lie
  uint32_t w[8];
  __device__ __forceinline__ void fill(uint32_t two) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = two;
  }
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
  Half16 x[kPgPasses];
#pragma unroll
  for (int i = 0; i < kPgPasses; ++i) {
    x[i].fill(p.absent);
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
  p.total = row_starts ? n_rows : s.batch * n_rows;
  p.nq = q.rows ? s.h_q : 0;
  p.nk = k.rows ? s.h_kv : 0;
  p.nv = v.rows ? s.h_kv : 0;
  const int all = p.nq + p.nk + p.nv, at_once = kPgThreads / (s.head_dim / 16), sms = current_sm_count();
  // few tokens: a token's rows spread over CTAs, a pass of rows each
  int split = 1;
  while (split < 64 && (long)p.total * split < sms && all > at_once * split) split *= 2;
  p.rows_per_cta = (all + split - 1) / split;
  // rows side by side: as many as divide a token's, or nearly; tokens: up to four of a thread and row, while there are enough.  (A
  // start, the look-ups and sines, costs a CTA some 2 us.  Two of a thread / four / eight, bf16, and one / four, fp32: 4 x 8192 tokens of 48
  // rows 133 / 129 / 138 us, 188 / 178; of 40 rows 111 / 115 / 118; 2 x 2048 tokens of 48 rows 22.6 / 20.8 / 20.8, 28.9 / 26.5.)
  p.row_shift = 0;
  for (int k = 1; 1 << k <= at_once && 1 << k < 2 * p.rows_per_cta; ++k)
    if (((p.rows_per_cta + (1 << k) - 1) >> k << k) * 8 <= p.rows_per_cta * 9) p.row_shift = k;
  const int room = std::min(kPgTokens, 4 * (at_once >> p.row_shift));
  p.tokens = 1;
  while (2 * p.tokens <= room && p.total >= 6L * sms * p.tokens) p.tokens *= 2;
  const unsigned blocks = ((unsigned)p.total + p.tokens - 1) / p.tokens;
  const void* fn = nullptr;
#define BD_PA(D, CODE, T) \
  if (s.head_dim == D && dtype == CODE) fn = reinterpret_cast<const void*>(&paged_append_kernel<D, T>);
  BD_PA(64, BD_DTYPE_BF16, __nv_bfloat16) BD_PA(128, BD_DTYPE_BF16, __nv_bfloat16)
  BD_PA(64, BD_DTYPE_F32, float) BD_PA(128, BD_DTYPE_F32, float)
#undef BD_PA
  void* args[] = {&p};
  return launch_kernel(fn, dim3(blocks, (unsigned)((all + p.rows_per_cta - 1) / p.rows_per_cta)), dim3(kPgThreads), 0, stream,
                       args, 0);
}

cudaError_t launch_paged_read(const bd_shape& s, int first_row, int n_rows, const bd_paged_cache& c, const int32_t* table,
                              int table_pages, const RowTensor& k, const RowTensor& v, bool nan_absent, cudaStream_t stream) {
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
  p.absent = nan_absent ? 0x7fc07fc0u : 0u;
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
