// Writing rows into a 4-bit cache and reading them back (bd_quant_write, bd_quant_read).
//
//   scale = bf16(max |x| / 7) over a group of 32, code = clamp(round(x / scale), -7, 7) + 8,
//   value = (code - 8) * scale
//
// Both are one pass over the rows with nothing to reuse, bound by HBM: 8 x 16K rows of K and V (690 MB) are written in
// 109 us (6.3 TB/s) and read back in 100 (6.9 TB/s).  The write is as fast only because a quotient takes three packed
// FMAs and its code comes off the sum's last bits: with a division and a conversion an element it took 383 us.
// A thread takes 16 adjacent elements of a row, half a group: 32 bytes of bf16, an 8-byte word of codes; a warp's
// accesses are contiguous on both sides and the two threads of a group meet in one shuffle.
#include <algorithm>

#include "bd_internal.h"
#include "bd_quant.cuh"

namespace bd {

constexpr int kQThreads = 256;
constexpr int kQPasses = 4;   // row blocks of a CTA

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
  int n_rows, h_kv, units, t_cap;
  int blocks;                 // CTAs of a unit's rows
  bool wide;                  // every row is 32-byte aligned
};

// 32 bytes at once, or as two halves where the rows are not 32-byte aligned.  As two halves every access covers half of
// each 32-byte sector of what a warp touches: reading 8 x 16K rows took 133 us so, 100 as one.
__device__ __forceinline__ void load32(const void* p, bool wide, uint32_t* w) {
  if (wide) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 v = __ldcs(static_cast<const uint4*>(p) + i);
      w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
  }
}
__device__ __forceinline__ void store32(void* p, bool wide, const uint32_t* w) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) static_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
}

// 16 elements as they lie.
template <typename T>
struct Sixteen;
template <>
struct Sixteen<__nv_bfloat16> {
  uint32_t w[8];
  __device__ __forceinline__ void load(const __nv_bfloat16* p, bool wide) { load32(p, wide, w); }
  // the largest magnitude's bits as a float's (a NaN's are above infinity's); one instruction for two elements, their signs
  // left to the end (with a mask and an integer maximum 8 x 16K rows took 111 us, 109 so)
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = w[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i]));
    return max(m << 16 & 0x7fff0000u, m & 0x7fff0000u);
  }
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)); }
};
template <>
struct Sixteen<float> {
  float x[16];
  __device__ __forceinline__ void load(const float* p, bool wide) {
    load32(p, wide, reinterpret_cast<uint32_t*>(x));
    load32(p + 8, wide, reinterpret_cast<uint32_t*>(x) + 8);
  }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(x[2 * i], x[2 * i + 1]); }
};

// Codes and scale of a group's half; top: the group's largest magnitude, as bits.
template <typename T>
__device__ __forceinline__ uint2 quantise(const Sixteen<T>& x, uint32_t top, uint16_t* scale) {
  const float t = __uint_as_float(top);
  uint32_t word[2];
  if (top - 0x12800000u < 0x7f800000u - 0x12800000u) {   // 2^-90 <= t, finite: nothing below underflows
    // Quotients a / b as q + (a - q b) y with y = 1 / b and q = a y, both rounded (Markstein 1990): the rounded quotient.
    constexpr float kSeventh = 1.f / 7.f;
    const float q7 = t * kSeventh;
    const __nv_bfloat16 sb = __float2bfloat16_rn(fmaf(fmaf(-q7, 7.f, t), kSeventh, q7));
    const float s = __bfloat162float(sb), y = __frcp_rn(s);
    *scale = __bfloat16_as_ushort(sb);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // 1.5 2^23 + 8 + the quotient, rounded half to even, has the code in its last four bits (|quotient| <= 7 / (1 - 2^-8),
      // so none needs the clamp); what the sum below carries of the rest is a constant
      uint32_t sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 a = x.pair(4 * h + i), yy = make_float2(y, y), q = fmul2(a, yy);
        const float2 r = ffma2(q, make_float2(-s, -s), a);
        const float2 c = fadd2(ffma2(r, yy, q), make_float2(12582920.f, 12582920.f));
        sum += __float_as_uint(c.x) << (8 * i);
        sum += __float_as_uint(c.y) << (8 * i + 4);
      }
      constexpr uint32_t kBias = 0x4b400000u;
      word[h] = sum - (kBias + (kBias << 4) + (kBias << 8) + (kBias << 12) + (kBias << 16) + (kBias << 20) + (kBias << 24) + (kBias << 28));
    }
    return make_uint2(word[0], word[1]);
  }
  // tiny groups, zeros, and groups that are not numbers
  const bool odd = top >= 0x7f800000u;
  const __nv_bfloat16 sb = __float2bfloat16_rn(__fdiv_rn(t, 7.f));
  const float s = __bfloat162float(sb);
  *scale = odd ? 0x7fffu : __bfloat16_as_ushort(sb);
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {
    word[0] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 a = h ? x.pair(4 + i) : x.pair(i);
      const bool live = !odd && s > 0.f;
      const int c0 = live ? (int)fminf(fmaxf(rintf(__fdiv_rn(a.x, s)), -7.f), 7.f) : 0;
      const int c1 = live ? (int)fminf(fmaxf(rintf(__fdiv_rn(a.y, s)), -7.f), 7.f) : 0;
      word[0] |= (uint32_t)(c0 + 8) << (8 * i) | (uint32_t)(c1 + 8) << (8 * i + 4);
    }
    if (h == 0) word[1] = word[0];
  }
  return make_uint2(word[1], word[0]);
}

// A CTA's place: its tensor, unit and first row.
struct Place {
  const QuantRows* t;
  long long at, cache_row;     // the unit's offset among the caller's rows; the cache row of its row 0
  int row;
};
template <int D>
__device__ __forceinline__ Place place(const QuantParams& p) {
  constexpr int ROWS = kQThreads / (D / 16) * kQPasses;
  const unsigned u = blockIdx.x / (unsigned)p.blocks, b = blockIdx.x - u * (unsigned)p.blocks;
  const int which = u >= (unsigned)p.units, unit = (int)u - which * p.units;
  const int seq = unit / p.h_kv, head = unit - seq * p.h_kv;
  int first = p.first;
  if (p.seq_lens) first = min(max(p.seq_lens[seq], 0), p.first);
  Place r;
  r.t = &p.t[which];
  r.at = seq * r.t->sb + head * r.t->sh;
  r.cache_row = (long long)unit * p.t_cap + first;
  r.row = (int)b * ROWS + threadIdx.x / (D / 16);
  return r;
}

template <int D, typename T>
__global__ void __launch_bounds__(kQThreads) quant_write_kernel(const __grid_constant__ QuantParams p) {
  constexpr int CH = D / 16, STEP = kQThreads / CH;   // threads of a row; rows at a time
  constexpr int AHEAD = sizeof(T) == 2 ? 4 : 2;       // rows in flight: 128 bytes a thread (bf16 with 64: 1.1 times the time; fp32 with 256: 95 us for 86)
  grid_dependency_wait();
  allow_dependent_launch();
  const Place at = place<D>(p);
  const QuantRows& t = *at.t;
  const int c = threadIdx.x % CH;
  const T* src = static_cast<const T*>(t.rows) + at.at + 16 * c;
#pragma unroll 1
  for (int k = 0; k < kQPasses; k += AHEAD) {
    if (at.row + k * STEP - (int)threadIdx.x / CH >= p.n_rows) break;      // (the whole CTA's rows are past the end)
    Sixteen<T> x[AHEAD] = {};
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      const int row = at.row + (k + e) * STEP;
      if (row < p.n_rows) x[e].load(src + (long long)row * t.sn, p.wide);
    }
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      const int row = at.row + (k + e) * STEP;
      uint32_t top = x[e].top();
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      if (row < p.n_rows) {
        uint16_t scale;
        const long long to = at.cache_row + row;
        *reinterpret_cast<uint2*>(t.codes + to * (D / 2) + 8 * c) = quantise(x[e], top, &scale);
        if ((c & 1) == 0) t.scales[to * (D / kQGroup) + c / 2] = scale;
      }
    }
  }
}

__device__ __forceinline__ uint32_t bf16x2_add(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t bf16x2_mul(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// The eight values of a word of codes, as they are written.
__device__ __forceinline__ void values(uint32_t w, uint32_t scale, uint32_t (&out)[4]) {
  // 128 + c is a bf16 with c in its last bits; less 136 it is c - 8, exactly, and the product is rounded once
  const uint32_t s2 = scale | scale << 16;
  uint32_t v[4];                                  // element pairs (0, 4), (1, 5), (2, 6), (3, 7)
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = bf16x2_mul(bf16x2_add((w >> (4 * i) & kNibble0) | 0x43004300u, 0xc308c308u), s2);
  out[0] = __byte_perm(v[0], v[1], 0x5410);
  out[1] = __byte_perm(v[2], v[3], 0x5410);
  out[2] = __byte_perm(v[0], v[1], 0x7632);
  out[3] = __byte_perm(v[2], v[3], 0x7632);
}
__device__ __forceinline__ void values(uint32_t w, uint32_t scale, uint32_t (&out)[8]) {
  const float s = bf16_bits_to_float(scale);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {                // 2^23 + c, less 2^23 + 8
    const float2 c = fadd2(make_float2(__uint_as_float((w >> (4 * i) & 15u) | 0x4b000000u), __uint_as_float((w >> (4 * i + 4) & 15u) | 0x4b000000u)),
                           make_float2(-8388616.f, -8388616.f));
    const float2 x = fmul2(c, make_float2(s, s));
    out[i] = __float_as_uint(x.x);
    out[i + 1] = __float_as_uint(x.y);
  }
}

// The rows may be what the next kernel on the stream streams before its own dependency wait (the
// selection and the verify block do that with context rows): no early trigger here, and every thread's
// rows are in L2, for the copy engines' proxy too, before it ends.
template <int D, typename T>
__global__ void __launch_bounds__(kQThreads) quant_read_kernel(const __grid_constant__ QuantParams p) {
  constexpr int CH = D / 16, STEP = kQThreads / CH;
  grid_dependency_wait();
  const Place at = place<D>(p);
  const QuantRows& t = *at.t;
  const int c = threadIdx.x % CH;
  T* dst = static_cast<T*>(t.rows) + at.at + 16 * c;
  uint2 w[kQPasses];
  uint32_t s[kQPasses];
#pragma unroll
  for (int k = 0; k < kQPasses; ++k) {
    const int row = at.row + k * STEP;
    const long long from = at.cache_row + row;
    if (row < p.n_rows) {
      w[k] = __ldcs(reinterpret_cast<const uint2*>(t.codes + from * (D / 2) + 8 * c));
      s[k] = __ldg(t.scales + from * (D / kQGroup) + c / 2);
    }
  }
#pragma unroll
  for (int k = 0; k < kQPasses; ++k) {
    const int row = at.row + k * STEP;
    if (row < p.n_rows) {
      T* to = dst + (long long)row * t.sn;
      constexpr int WORDS = sizeof(T) * 2;       // of eight elements
      uint32_t out[2][WORDS];
      values(w[k].x, s[k], out[0]);
      values(w[k].y, s[k], out[1]);
#pragma unroll
      for (int i = 0; i < 2 * WORDS; i += 8) store32(to + i * 4 / sizeof(T), p.wide, &out[0][0] + i);
    }
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
  p.wide = true;
  for (int i = 0; i < n; ++i) {
    const long long e = dtype == BD_DTYPE_F32 ? 4 : 2;
    const QuantRows& r = p.t[i];
    p.wide &= reinterpret_cast<uintptr_t>(r.rows) % 32 == 0 && r.sb * e % 32 == 0 && r.sh * e % 32 == 0 && r.sn * e % 32 == 0;
  }
  p.seq_lens = seq_lens;
  p.first = first;
  p.n_rows = n_rows;
  p.h_kv = s.h_kv;
  p.units = s.batch * s.h_kv;
  p.t_cap = s.t_cap;
  const int rows = kQThreads / (s.head_dim / 16) * kQPasses;
  p.blocks = (n_rows + rows - 1) / rows;
  const long long grid = (long long)p.blocks * p.units * n;
  if (grid >= (1LL << 31)) return cudaErrorInvalidConfiguration;   // (fewer than 2^31 rows in a cache: never)
  const void* fn = nullptr;
#define BD_QR(D, CODE, T)                 \
  if (s.head_dim == D && dtype == CODE)   \
    fn = write ? reinterpret_cast<const void*>(&quant_write_kernel<D, T>) : reinterpret_cast<const void*>(&quant_read_kernel<D, T>);
  BD_QR(64, BD_DTYPE_BF16, __nv_bfloat16) BD_QR(128, BD_DTYPE_BF16, __nv_bfloat16)
  BD_QR(64, BD_DTYPE_F32, float) BD_QR(128, BD_DTYPE_F32, float)
#undef BD_QR
  void* args[] = {&p};
  return launch_kernel(fn, dim3((unsigned)grid), dim3(kQThreads), 0, stream, args, 0);
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
