// Writing rows into a 4-bit cache and reading them back (bd_quant_write, bd_quant_read).
//
//   scale = bf16(max |x| / 7) over a group of 32, code = clamp(round(x / scale), -7, 7) + 8,
//   value = (code - 8) * scale
//
// Both are one pass over the rows with nothing to reuse, bound by HBM: a thread takes eight adjacent
// elements of a row (16 bytes of bf16, one 32-bit word of codes), so that a warp's accesses are
// contiguous on both sides; the four threads of a group find its largest magnitude with two shuffles.
#include <algorithm>

#include "bd_internal.h"
#include "bd_quant.cuh"

namespace bd {

constexpr int kQThreads = 256;

struct QuantRows {            // one tensor of a call
  void* rows;                 // bf16 or fp32 rows (source or destination), element strides:
  long long sb, sh, sn;       // of a sequence, a KV head, a row
  uint8_t* codes;             // [units][t_cap][D / 2]
  uint16_t* scales;           // [units][t_cap][D / 32]
};

struct QuantParams {
  QuantRows t[2];
  const int32_t* seq_lens;    // rows start at each sequence's length (or null: at first)
  int first;                  // first row of every unit; with seq_lens the bound of the lengths
  int n_rows, h_kv, t_cap;
  long long items;            // (row, eight elements) pairs of one tensor
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]);
template <>
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) {
  const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
template <>
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                            pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Where item i of a tensor lies: its row's offset among the caller's rows (elements), and its cache row.
struct ItemPlace {
  long long at;    // first of the item's eight elements
  long long row;   // cache row
  int chunk;       // which eight of the row
};
template <int D>
__device__ __forceinline__ ItemPlace place(const QuantParams& p, const QuantRows& t, long long i) {
  constexpr int CH = D / 8;
  ItemPlace r;
  r.chunk = (int)(i % CH);
  const unsigned rr = (unsigned)(i / CH);      // (a cache has fewer than 2^31 rows)
  const unsigned unit = rr / (unsigned)p.n_rows, n = rr - unit * (unsigned)p.n_rows;
  const unsigned b = unit / (unsigned)p.h_kv, h = unit - b * (unsigned)p.h_kv;
  int first = p.first;
  if (p.seq_lens) first = min(max(p.seq_lens[b], 0), p.first);
  r.at = b * t.sb + h * t.sh + n * t.sn + 8 * r.chunk;
  r.row = (long long)unit * p.t_cap + first + n;
  return r;
}

template <int D, typename T>
__global__ void __launch_bounds__(kQThreads) quant_write_kernel(const __grid_constant__ QuantParams p) {
  grid_dependency_wait();
  allow_dependent_launch();
  const QuantRows& t = p.t[blockIdx.y];
  // (items come in whole rows of at least eight, and a group's four threads are adjacent lanes: a
  // group is wholly inside or outside of the range)
  for (long long i = (long long)blockIdx.x * kQThreads + threadIdx.x; i < p.items; i += (long long)gridDim.x * kQThreads) {
    const ItemPlace at = place<D>(p, t, i);
    float x[8];
    load8(static_cast<const T*>(t.rows) + at.at, x);
    float top = 0.f;
    bool odd = false;                         // a NaN or an infinity among them
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      top = fmaxf(top, fabsf(x[e]));
      odd |= !(fabsf(x[e]) < INFINITY);
    }
    const unsigned four = 0xfu << (threadIdx.x & 28);   // the lanes of the group
    top = fmaxf(top, __shfl_xor_sync(four, top, 1));
    top = fmaxf(top, __shfl_xor_sync(four, top, 2));
    odd = (__ballot_sync(four, odd) & four) != 0;
    const __nv_bfloat16 sb = __float2bfloat16_rn(__fdiv_rn(top, 7.f));
    const float s = __bfloat162float(sb);
    uint32_t word = 0x88888888u;
    if (!odd && s > 0.f) {
      word = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float r = fminf(fmaxf(rintf(__fdiv_rn(x[e], s)), -7.f), 7.f);
        word |= (uint32_t)((int)r + 8) << (4 * e);
      }
    }
    *reinterpret_cast<uint32_t*>(t.codes + at.row * (D / 2) + 4 * at.chunk) = word;
    if ((at.chunk & 3) == 0)
      t.scales[at.row * (D / kQGroup) + at.chunk / 4] = odd ? 0x7fffu : __bfloat16_as_ushort(sb);
  }
}

// The rows may be what the next kernel on the stream streams before its own dependency wait (the
// selection and the verify block do that with context rows): no early trigger here, and every thread's
// rows are in L2, for the copy engines' proxy too, before it ends.
template <int D, typename T>
__global__ void __launch_bounds__(kQThreads) quant_read_kernel(const __grid_constant__ QuantParams p) {
  grid_dependency_wait();
  const QuantRows& t = p.t[blockIdx.y];
  for (long long i = (long long)blockIdx.x * kQThreads + threadIdx.x; i < p.items; i += (long long)gridDim.x * kQThreads) {
    const ItemPlace at = place<D>(p, t, i);
    const uint32_t word = __ldcs(reinterpret_cast<const uint32_t*>(t.codes + at.row * (D / 2) + 4 * at.chunk));
    const float s = bf16_bits_to_float(t.scales[at.row * (D / kQGroup) + at.chunk / 4]);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)((int)((word >> (4 * e)) & 15u) - 8) * s;
    store8(static_cast<T*>(t.rows) + at.at, x);
  }
  asm volatile("fence.proxy.async.global;" ::: "memory");
  __threadfence();
}

static cudaError_t launch_rows(const bd_shape& s, bool write, const int32_t* seq_lens, int first, int n_rows, int dtype,
                               const bd_quant_cache& c, const QuantTensor& k, const QuantTensor& v, cudaStream_t stream) {
  QuantParams p;
  int n = 0;
  for (int i = 0; i < 2; ++i) {
    const QuantTensor& t = i ? v : k;
    if (!t.rows) continue;
    QuantRows& r = p.t[n++];
    r.rows = t.rows;
    r.sb = t.sb;
    r.sh = t.sh;
    r.sn = t.sn;
    r.codes = static_cast<uint8_t*>(i ? c.v_codes : c.k_codes);
    r.scales = static_cast<uint16_t*>(i ? c.v_scales : c.k_scales);
  }
  if (n == 1) p.t[1] = p.t[0];
  p.seq_lens = seq_lens;
  p.first = first;
  p.n_rows = n_rows;
  p.h_kv = s.h_kv;
  p.t_cap = s.t_cap;
  p.items = (long long)s.batch * s.h_kv * n_rows * (s.head_dim / 8);
  const long long blocks = (p.items + kQThreads - 1) / kQThreads;
  const int most = current_sm_count() * 8;
  const void* fn = nullptr;
#define BD_QR(D, CODE, T)                 \
  if (s.head_dim == D && dtype == CODE)   \
    fn = write ? reinterpret_cast<const void*>(&quant_write_kernel<D, T>) : reinterpret_cast<const void*>(&quant_read_kernel<D, T>);
  BD_QR(64, BD_DTYPE_BF16, __nv_bfloat16) BD_QR(128, BD_DTYPE_BF16, __nv_bfloat16)
  BD_QR(64, BD_DTYPE_F32, float) BD_QR(128, BD_DTYPE_F32, float)
#undef BD_QR
  void* args[] = {&p};
  return launch_kernel(fn, dim3((unsigned)std::min<long long>(blocks, most), n), dim3(kQThreads), 0, stream, args, 0);
}

cudaError_t launch_quant_write(const bd_shape& s, int n_rows, int dtype, const bd_quant_cache& c, const QuantTensor& k,
                               const QuantTensor& v, cudaStream_t stream) {
  return launch_rows(s, true, s.seq_lens, s.t_ctx, n_rows, dtype, c, k, v, stream);
}

cudaError_t launch_quant_read(const bd_shape& s, int first_row, int n_rows, int dtype, const bd_quant_cache& c,
                              const QuantTensor& k, const QuantTensor& v, cudaStream_t stream) {
  const bool behind = first_row < 0;          // the rows behind each sequence's length
  return launch_rows(s, false, behind ? s.seq_lens : nullptr, behind ? s.t_ctx : first_row, n_rows, dtype, c, k, v, stream);
}

}  // namespace bd
