// Shared by the kernels of the 4-bit cache: codes and scales.
//
// A code is a sign, two bits of exponent and one of mantissa: 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives.  The scale of a row's values is the least 2^e
// with max|x| <= 7 * 2^e: then nothing, the largest value either, is off by more than half a step of the topmost codes (5 .. 7 are 6).  It is held as the
// byte e + 127, 255 for "not a number".  x / scale is exact, so a code is one rounding.
#pragma once
#include "k8_dev.hpp"

namespace k4 {

using namespace k8;

using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;

constexpr int kNone = 255;     // byte of a scale that is not a number
constexpr int kGroup = 32;     // dims of K under one scale
constexpr int kCodeBytes(int D) { return kBlock * D / 2; }  // of a block of K, or of V

// The byte of the scale of values whose largest magnitude has these bits; 7 = 1.75 * 2^2.
__device__ inline int scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return kNone;
  const int x = (int)(amax_bits >> 23) - 127;  // (a subnormal magnitude comes out below kEMin anyway)
  const int e = x - 2 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kEMin), kEMax) + 127;
}

__device__ inline float inverse_scale(int byte) { return byte == kNone ? 0.f : __uint_as_float((uint32_t)(254 - byte) << 23); }

// Eight values in units of their scale -> eight codes, the first in the lowest bits; nearest, ties to the even code, at most 6.
__device__ inline uint32_t encode8(const float* x) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], 1.f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], 1.f, 3);
  return w;
}

// Eight codes -> their values, times a power of two.
__device__ inline void decode8(uint32_t w, float scale, float (&x)[8]) {
  const float2v a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1),
                c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
}

}  // namespace k4
