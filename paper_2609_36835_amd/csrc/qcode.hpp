// Codes and scales of the 8-bit cache, device side.
#pragma once
#include "common.hpp"
#include "qcache.hpp"

namespace arckv {

constexpr int kQMinExp = -100;      // least exponent of a scale: every stored value is zero or a normal number

// FMT is an arckv_qformat.  Codes are e4m3 (4 exponent bits, 3 mantissa bits, largest value 448, no infinity) or
// two's complement int8 in [-127, 127].
template <int FMT> struct QCode;

template <> struct QCode<ARCKV_E4M3> {
  static constexpr int kExpBits = 8;                    // 448 = 1.75 * 2^8
  static constexpr uint32_t kTopMantissa = 0x600000u;   // of 1.75
  // rounded to nearest even
  __device__ static inline uint32_t pack4(float a, float b, float c, float d) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
  }
  __device__ static inline void unpack4(uint32_t w, float (&x)[4]) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0];
    x[1] = lo[1];
    x[2] = hi[0];
    x[3] = hi[1];
  }
};

template <> struct QCode<ARCKV_INT8> {
  static constexpr int kExpBits = 6;                    // 127 = 1.984375 * 2^6
  static constexpr uint32_t kTopMantissa = 0x7e0000u;   // of 1.984375
  __device__ static inline uint32_t pack4(float a, float b, float c, float d) {
    const int ia = (int)rintf(a), ib = (int)rintf(b), ic = (int)rintf(c), id = (int)rintf(d);
    return ((uint32_t)ia & 255u) | (((uint32_t)ib & 255u) << 8) | (((uint32_t)ic & 255u) << 16) | ((uint32_t)id << 24);
  }
  __device__ static inline void unpack4(uint32_t w, float (&x)[4]) {
    x[0] = (float)(int8_t)w;
    x[1] = (float)(int8_t)(w >> 8);
    x[2] = (float)(int8_t)(w >> 16);
    x[3] = (float)(int8_t)(w >> 24);
  }
};

// Bounds-checked reads of `bytes` from p on (wave-uniform): zero behind them.
__device__ inline __amdgpu_buffer_rsrc_t buffer(const void *p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00020000);
}
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
constexpr int kStreamed = 2;   // a load's or store's aux bits: not kept in the caches

// Reduction over the four 16-lane rows of a wave, every lane with the result.
template <typename F> __device__ inline float over_rows(float x, F f) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// 2^e for e in [-126, 127]
__device__ inline float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Exponent of the smallest power of two that brings a largest magnitude (its float bits) into the codes' range.
template <int FMT> __device__ inline int qscale_exp(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23) - 127 - QCode<FMT>::kExpBits + ((amax_bits & 0x7fffffu) > QCode<FMT>::kTopMantissa);
  return max(e, kQMinExp);
}

__device__ inline int clip_len(const int32_t *len, int p, int most) {
  return len ? min(max(len[p], 0), most) : most;
}

}  // namespace arckv
