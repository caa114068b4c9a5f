// Codes and scales of the 4-bit cache, device side.
#pragma once
#include "ncache.hpp"
#include "qcode.hpp"

namespace arckv {

constexpr int kNMinExp = -100, kNMaxExp = 125;   // of a scale: every stored value is zero or a normal number

// Exponent of a group's scale from its largest magnitude (float bits, finite): the smallest power of two that brings
// it to 6 = 1.5 * 2^2 or below.
__device__ inline int nscale_exp(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23) - 127 - 2 + ((amax_bits & 0x7fffffu) > 0x400000u);
  return min(max(e, kNMinExp), kNMaxExp);
}

// A scale byte as a number: 2^(byte - 127), NaN for 255 (0, which no write leaves, is 0).
__device__ inline float nscale(uint32_t byte) { return byte == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(byte << 23); }

// Four numbers to codes: e2m1 of x / scale, to nearest even, magnitudes above 6 to 6; eight.
__device__ inline uint32_t npack4(float a, float b, float c, float d, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, scale, 0), c, d, scale, 1);
}
__device__ inline uint32_t npack8(const float *x, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

}  // namespace arckv
