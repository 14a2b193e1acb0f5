// e4m3 codes with a power of two for every few tokens of a page and head.  A code times that power has four bits of mantissa, so
// it is exact in bf16; the conversion that multiplies by it takes two values at the rate of an addition, and of the scale only the
// exponent.
#pragma once

#include "ff_attn_plan.h"

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;

// the lower or upper two of four codes -> a pair of bf16
template <bool UPPER>
__device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, UPPER));
}
__device__ __forceinline__ u32x2_t decode4(uint32_t codes, float scale) { return u32x2_t{decode2<false>(codes, scale), decode2<true>(codes, scale)}; }
__device__ __forceinline__ u32x4_t decode8(uint32_t a, uint32_t b, float scale) {
  return u32x4_t{decode2<false>(a, scale), decode2<true>(a, scale), decode2<false>(b, scale), decode2<true>(b, scale)};
}

// Two values -> two codes in the lower or upper half of `old`.  The conversion rounds to nearest even and gives NaN from 464 on: finite
// values beyond 448 (of a block whose scale would exceed its limit) become 448 before it, infinities and NaN are NaN.
template <bool UPPER>
__device__ __forceinline__ uint32_t encode2(float a, float b, uint32_t old) {
  const float x = fabsf(a) < INFINITY ? __builtin_amdgcn_fmed3f(a, -448.f, 448.f) : NAN;
  const float y = fabsf(b) < INFINITY ? __builtin_amdgcn_fmed3f(b, -448.f, 448.f) : NAN;
  return __builtin_amdgcn_cvt_pk_fp8_f32(x, y, old, UPPER);
}
// two pairs of bf16, times a factor -> four codes
__device__ __forceinline__ uint32_t encode4(uint32_t lo, uint32_t hi, float factor) {
  const uint32_t w = encode2<false>(__uint_as_float(lo << 16) * factor, __uint_as_float(lo & 0xffff0000u) * factor, 0);
  return encode2<true>(__uint_as_float(hi << 16) * factor, __uint_as_float(hi & 0xffff0000u) * factor, w);
}
