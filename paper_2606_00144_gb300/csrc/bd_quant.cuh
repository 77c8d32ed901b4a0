// What the kernels over a 4-bit cache (include/budgetdraft.h, bd_quant_cache) share.
//
// A row of D elements is D/2 bytes of 4-bit codes (element 2 j in the low half of byte j) and one bf16
// scale for every group of 32 elements; code c of group g stands for (c - 8) * scale[g].
//
// Codes reach the tensor cores without a conversion: a code in the low bits of an fp16's mantissa
// is the subnormal c * 2^-24, exactly, and the next one, left where it lies four bits higher, 16 c *
// 2^-24.  One AND of a 32-bit word that holds two 16-bit units and one packed FMA, which brings them
// to normal numbers less the offset of 8, so make two operands.
#pragma once

#include <cuda_fp16.h>

#include "bd_common.cuh"

namespace bd {

constexpr int kQGroup = 32;                  // elements of a scale's group
constexpr uint32_t kNibble0 = 0x000f000fu;   // codes 0 of a word's two 16-bit units, as c * 2^-24
constexpr uint32_t kNibble1 = 0x00f000f0u;   // codes 1, as 16 c * 2^-24

__device__ __forceinline__ float bf16_bits_to_float(uint32_t bits) { return __uint_as_float(bits << 16); }

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// 2^e for -126 <= e <= 127.
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }

__device__ __forceinline__ float2 fmul2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
      "mul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}

__device__ __forceinline__ void mma_16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Codes 0, codes 1 of a word's two 16-bit units as (c - 8) * 2^-10, exactly.
__device__ __forceinline__ uint32_t fma_half2(uint32_t a, uint32_t b, uint32_t c) {
  const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b),
                            *reinterpret_cast<const __half2*>(&c));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t centred0(uint32_t w) {   // c 2^-24 * 2^14 - 2^-7
  return fma_half2(w & kNibble0, 0x74007400u, 0xa000a000u);
}
__device__ __forceinline__ uint32_t centred1(uint32_t w) {   // 16 c 2^-24 * 2^10 - 2^-7
  return fma_half2(w & kNibble1, 0x64006400u, 0xa000a000u);
}

// 4- and 8-byte cp.async (through L1), zero bytes where !valid.
template <int BYTES>
__device__ __forceinline__ void cp_async_small(void* dst, const void* src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(smem_u32(dst)), "l"(src), "n"(BYTES),
               "r"(valid ? BYTES : 0)
               : "memory");
}

// The exponent that normalises a cache row's V scales: floor(log2) of the largest, within [-100, 126].
// Scales are taken to fp16 as scale * 2^-e (the largest in [1, 2)) and 2^e joins the row's softmax
// weight, so that V of any size keeps its precision in fp16.  A row of zeros (or smaller than
// 2^-90) has -90.
__device__ __forceinline__ int scale_exponent(int largest_bits) { return min(max((largest_bits >> 7) - 127, -90), 126); }
// The normaliser counts a key by its score alone, 2^S: a row of zeros whose exponent of -90 went into the weight's would be
// flushed (ex2 ends at 2^-126) beside rows of 2^40 although it may have the highest score.  So only what is above
// kWeightExponent joins the weight before the sum:
//   t = 2^(S - M + max(e, -16)),  sum += t 2^-max(e, -16),  weight = t 2^min(e + 16, 0)
// With V up to 2^92 no key is lost to the sum whose 2^S is above 2^-24 of the largest key's; a sum stays below 2^128 for
// 2^24 keys of zeros that all trail the maximum by the slack (2^14 2^90 each).  A factor between two maxima may span as
// much, so it is applied to a sum as two halves.
constexpr int kWeightExponent = -16;

// A cache row's scales as they lie: D / 32 bf16.
template <int D>
struct RowScales {
  uint32_t w[D / 64];
  // from global memory, zero where there is no row
  __device__ __forceinline__ void load(const uint16_t* p, bool valid) {
    if constexpr (D == 128) {
      const uint2 v = valid ? __ldg(reinterpret_cast<const uint2*>(p)) : make_uint2(0u, 0u);
      w[0] = v.x;
      w[1] = v.y;
    } else {
      w[0] = valid ? __ldg(reinterpret_cast<const uint32_t*>(p)) : 0u;
    }
  }
  __device__ __forceinline__ void load_shared(const uint16_t* p) {
    if constexpr (D == 128) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x;
      w[1] = v.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
  }
  // scale_exponent of the largest that is a number: one that is not makes its own group NaN and says nothing about the
  // others (a unit more in the exponent takes it below all numbers, as a signed 16-bit value)
  __device__ __forceinline__ int exponent() const {
    uint32_t t = (w[0] & 0x7fff7fffu) + 0x00800080u;
    if constexpr (D == 128) asm("max.s16x2 %0, %0, %1;" : "+r"(t) : "r"((w[D / 64 - 1] & 0x7fff7fffu) + 0x00800080u));
    return scale_exponent(max((int)t >> 16, (int)(int16_t)t) - 0x80);
  }
  __device__ __forceinline__ float scale(int g) const {
    const uint32_t x = g < 2 ? w[0] : w[D / 64 - 1];
    return __uint_as_float(g & 1 ? x & 0xffff0000u : x << 16);
  }
};

}  // namespace bd
