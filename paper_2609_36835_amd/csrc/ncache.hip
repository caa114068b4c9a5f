// The 4-bit cache: rows written into it and rows read back.
//
// A row stands on its own: each of its four groups of 32 channels has the power of two as scale that brings its largest
// magnitude to 6, and a code is x / scale rounded to the nearest, ties to even.  Powers of two make the division exact,
// so the codes are the same however they are computed, and a stored value (scale times code) is exact in bf16.
#include <type_traits>

#include "ncode.hpp"

namespace arckv {

// pairs lie over a grid's y and z, whose extents are limited
constexpr int kGridY = 32768;

// ---------------------------------------------------------------- write
// HBM-bound: 2 (or 4) bytes in and 17 / 32 out per element, once.  Sixteen lanes take a row, 16 bytes of whole lines at a
// time, a thread one row of float32 and up to four of bf16, and a wave consecutive rows, whose scales go out as one piece.
// Codes are written as streams.  64 pairs of 1024 to 2048 bf16 rows take 12.3 us, 256 of 3277 float32 rows 150 us (6.5 TB/s;
// 193 with a group per thread, 179 with four rows and half lines per load, 164 kept in the caches).
template <int ROWS> constexpr int kNwTile = 4 * 4 * ROWS;   // rows of a workgroup of four waves, ROWS to a thread
// Source bytes of bf16 up to which a thread takes one row.  us with one, two and four: 512 pairs of one row 2.5, 2.9, 3.1; 8 of
// 2048 (8 MB) 3.3, 3.3, 3.5; 64 of 500 (16 MB) 4.6, 4.4, 4.7; of 2048 (67 MB) 14.8, 13.7, 12.8.
constexpr int64_t kNwFew = (int64_t)16 << 20;
// Source bytes above which rows are read as streams that the caches do not keep: 64 pairs of 2048 bf16 rows (67 MB) take 14.7 us
// kept and 15.7 streamed, of 4096 30.7 and 28.7.  Streams of bf16 take two rows a thread: with two and with four 256 pairs of
// 2048 54.2 and 55.1, 8 of 131072 104.8 and 109.7, 512 of 3277 170 and 185.
constexpr int64_t kNwKept = (int64_t)96 << 20;

// The largest of four lanes' values, in all of them; of eight.
__device__ inline uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true));   // neighbours in twos
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true));
}
__device__ inline uint32_t oct_max(uint32_t x) {
  x = quad_max(x);
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true));   // mirrored in eights
}
template <int BY> __device__ inline uint32_t or_turned(uint32_t x) {   // a row's lanes turned by BY
  return x | (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + BY, 0xf, 0xf, true);
}

// A group's scale from its largest magnitude, as a byte and as a number.
struct Scale {
  uint32_t byte;
  float value;
  bool finite;
  __device__ inline explicit Scale(uint32_t amax) {
    finite = amax < 0x7f800000u;   // a NaN or an infinity is larger than every number
    const int e = nscale_exp(finite ? amax : 0u);
    byte = finite ? (uint32_t)(e + 127) : 255u;
    value = pow2f(e);
  }
};

__device__ inline uint32_t largest4(u32x4 w) {
  return max(max(w[0] & 0x7fffffffu, w[1] & 0x7fffffffu), max(w[2] & 0x7fffffffu, w[3] & 0x7fffffffu));
}

// A lane's part of a row: 16 bytes at a time of 16 lanes' whole lines.  Returns word `at` of the row's codes, and all its
// scales in every lane.
__device__ inline uint32_t encode(const u32x4 (&w)[1], int r, int &at, uint32_t &scales) {   // bf16: channels 8 r ..
  float x[8];
  uint32_t amax = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = __uint_as_float(e & 1 ? w[0][e / 2] & 0xffff0000u : w[0][e / 2] << 16);
    amax = max(amax, __float_as_uint(x[e]) & 0x7fffffffu);
  }
  const Scale s(quad_max(amax));
  scales = or_turned<8>(or_turned<4>(s.byte << 8 * (r >> 2)));
  at = r;
  return s.finite ? npack8(x, s.value) : 0u;
}
__device__ inline uint32_t encode(const u32x4 (&w)[2], int r, int &at, uint32_t &scales) {   // f32: channels 4 r .. and 64 + 4 r ..
  uint32_t code[2];
  scales = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const Scale s(oct_max(largest4(w[h])));
    scales |= s.byte << (16 * h + 8 * (r >> 3));
    code[h] = s.finite ? npack4(__uint_as_float(w[h][0]), __uint_as_float(w[h][1]), __uint_as_float(w[h][2]), __uint_as_float(w[h][3]), s.value)
                       : 0u;
  }
  scales = or_turned<8>(scales);
  // even lanes take the first half's words, odd ones the second's
  const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(r & 1 ? code[0] : code[1]), 0xb1, 0xf, 0xf, true);
  at = (r & 1) * 8 + (r >> 1);
  return r & 1 ? other | code[1] << 16 : code[0] | other << 16;
}

template <typename T, int ROWS, bool STREAM>
__global__ void __launch_bounds__(256) k_ncache_write(NCache c, int n, const T *__restrict__ K, const T *__restrict__ V,
                                                      const int32_t *__restrict__ starts,
                                                      const int32_t *__restrict__ counts) {
  constexpr int LOADS = sizeof(T) / 2;
  const int p = (blockIdx.z >> 1) * gridDim.y + blockIdx.y;
  if (p >= c.P) return;
  const int start = clip_len(starts, p, starts ? c.rows : 0);
  const int count = min(clip_len(counts, p, n), c.rows - start);
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int i0 = blockIdx.x * kNwTile<ROWS> + (threadIdx.x >> 6) * 4 * ROWS;   // the wave's rows i0 + 4 k + g
  if (i0 >= count) return;
  const T *src = (blockIdx.z & 1 ? V : K) + ((int64_t)p * n + i0) * kHeadDim;
  const int64_t row0 = (int64_t)p * c.rows + start + i0;
  uint8_t *codes = (blockIdx.z & 1 ? c.V : c.K) + row0 * kNRow;
  const int held = min(count - i0, 4 * ROWS);
  u32x4 w[ROWS][LOADS];
#pragma unroll
  for (int k = 0; k < ROWS; ++k)   // rows past the end are the last one again, and not stored
#pragma unroll
    for (int h = 0; h < LOADS; ++h) {
      const u32x4 *from = reinterpret_cast<const u32x4 *>(src + min(4 * k + g, held - 1) * kHeadDim) + 16 * h + r;
      w[k][h] = STREAM ? __builtin_nontemporal_load(from) : *from;
    }
  uint32_t scale = 0;   // of row i0 + 4 r + g, in the lanes r < ROWS
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    int at;
    uint32_t scales;
    const uint32_t code = encode(w[k], r, at, scales);
    scale = r == k ? scales : scale;
    if (4 * k + g < held) __builtin_nontemporal_store(code, reinterpret_cast<uint32_t *>(codes + (4 * k + g) * kNRow) + at);
  }
  if (r < ROWS && 4 * r + g < held) (blockIdx.z & 1 ? c.Vs : c.Ks)[row0 + 4 * r + g] = scale;
}

hipError_t launch_ncache_write(int dtype, const NCache &c, int n, const void *K, const void *V, const int32_t *start,
                               const int32_t *count, hipStream_t s) {
  auto go = [&](auto kern, auto rows, auto *k, auto *v) {
    const int tile = kNwTile<decltype(rows)::value>;
    const dim3 grid((unsigned)((n + tile - 1) / tile), (unsigned)min(c.P, kGridY), (unsigned)(2 * ((c.P + kGridY - 1) / kGridY)));
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, c, n, k, v, start, count);
    return hipGetLastError();
  };
  constexpr std::integral_constant<int, 1> one{};
  constexpr std::integral_constant<int, 2> two{};
  constexpr std::integral_constant<int, 4> four{};
  const int64_t bytes = (int64_t)c.P * n * 2 * kHeadDim * (dtype == ARCKV_BF16 ? 2 : 4);
  if (dtype == ARCKV_BF16) {
    const bf16 *k = (const bf16 *)K, *v = (const bf16 *)V;
    return bytes <= kNwFew    ? go(k_ncache_write<bf16, 1, false>, one, k, v)
           : bytes <= kNwKept ? go(k_ncache_write<bf16, 4, false>, four, k, v)
                              : go(k_ncache_write<bf16, 2, true>, two, k, v);
  }
  return bytes <= kNwKept ? go(k_ncache_write<float, 1, false>, one, (const float *)K, (const float *)V)
                          : go(k_ncache_write<float, 1, true>, one, (const float *)K, (const float *)V);
}

// ---------------------------------------------------------------- read
// HBM-bound.  A thread turns 8 (bf16 out) or 4 (float32 out) codes of each of two rows into 16 bytes, written as a stream: 8
// pairs of 32768 rows to bf16 take 24.4 us (7.0 TB/s; 34.3 where the caches keep what is written), 32 of 4567 to float32 24.1
// (39.5; 26.6 with four rows a thread).
constexpr int kNrRows = 2;
template <typename T>
__global__ void __launch_bounds__(256) k_ncache_read(NCache c, int first, int n, const int32_t *__restrict__ length,
                                                     T *__restrict__ K, T *__restrict__ V) {
  constexpr int PER = 16 / sizeof(T), LANES = kHeadDim / PER, STEP = 256 / LANES;   // codes per thread; threads per row; rows at a time
  const int p = (blockIdx.z >> 1) * gridDim.y + blockIdx.y;
  if (p >= c.P) return;
  const int piece = threadIdx.x % LANES, i0 = blockIdx.x * (kNrRows * STEP) + threadIdx.x / LANES;
  const int len = clip_len(length, p, c.rows);
  const uint8_t *codes = (blockIdx.z & 1 ? c.V : c.K) + (int64_t)p * c.rows * kNRow;
  const uint8_t *scales = reinterpret_cast<const uint8_t *>((blockIdx.z & 1 ? c.Vs : c.Ks) + (int64_t)p * c.rows);
  T *out = (blockIdx.z & 1 ? V : K) + (int64_t)p * n * kHeadDim + PER * piece;
  uint32_t w[kNrRows];
  float s[kNrRows];
#pragma unroll
  for (int k = 0; k < kNrRows; ++k) {
    if (len == 0) break;   // nothing to read
    const int64_t at = min(first + i0 + k * STEP, len - 1);   // rows past the end are not used
    if constexpr (PER == 8)
      w[k] = reinterpret_cast<const uint32_t *>(codes + at * kNRow)[piece];
    else
      w[k] = reinterpret_cast<const uint16_t *>(codes + at * kNRow)[piece];
    s[k] = nscale(scales[4 * at + piece * PER / kNGroup]);
  }
#pragma unroll
  for (int k = 0; k < kNrRows; ++k) {
    const int i = i0 + k * STEP;
    if (i >= n) continue;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (first + i < len) {
      if constexpr (PER == 8) {
        v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], s[k], 0));
        v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], s[k], 1));
        v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], s[k], 2));
        v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[k], s[k], 3));
      } else {
        const f32x2 a = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[k], s[k], 0)),
                    b = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[k], s[k], 1));
        v = u32x4{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])};
      }
    }
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(out + (int64_t)i * kHeadDim));
  }
}

hipError_t launch_ncache_read(int dtype, const NCache &c, int first, int n, const int32_t *length, void *K, void *V,
                              hipStream_t s) {
  const int per_wg = kNrRows * 256 / (kHeadDim / (dtype == ARCKV_BF16 ? 8 : 4));
  const dim3 grid((unsigned)((n + per_wg - 1) / per_wg), (unsigned)min(c.P, kGridY),
                  (unsigned)(2 * ((c.P + kGridY - 1) / kGridY)));
  if (dtype == ARCKV_BF16)
    hipLaunchKernelGGL(k_ncache_read<bf16>, grid, dim3(256), 0, s, c, first, n, length, (bf16 *)K, (bf16 *)V);
  else
    hipLaunchKernelGGL(k_ncache_read<float>, grid, dim3(256), 0, s, c, first, n, length, (float *)K, (float *)V);
  return hipGetLastError();
}

}  // namespace arckv
