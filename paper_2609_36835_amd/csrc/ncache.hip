// The 4-bit cache: rows written into it and rows read back.
//
// A row stands on its own: each of its four groups of 32 channels has the power of two as scale that brings its largest
// magnitude to 6, and a code is x / scale rounded to the nearest, ties to even.  Powers of two make the division exact,
// so the codes are the same however they are computed, and a stored value (scale times code) is exact in bf16.
#include "ncode.hpp"

namespace arckv {

// pairs lie over a grid's y and z, whose extents are limited
constexpr int kGridY = 32768;

// ---------------------------------------------------------------- write
// A thread takes a group.
template <typename T>
__global__ void __launch_bounds__(256) k_ncache_write(NCache c, int n, const T *__restrict__ K, const T *__restrict__ V,
                                                      const int32_t *__restrict__ starts,
                                                      const int32_t *__restrict__ counts) {
  const int p = (blockIdx.z >> 1) * gridDim.y + blockIdx.y;
  if (p >= c.P) return;
  const int start = clip_len(starts, p, starts ? c.rows : 0);
  const int count = min(clip_len(counts, p, n), c.rows - start);
  const int i = blockIdx.x * 64 + threadIdx.x / 4, group = threadIdx.x % 4;
  if (i >= count) return;
  const T *src = (blockIdx.z & 1 ? V : K) + ((int64_t)p * n + i) * kHeadDim + kNGroup * group;
  const int64_t row = (int64_t)p * c.rows + start + i;
  float x[kNGroup];
  uint32_t amax = 0;
  for (int e = 0; e < kNGroup; ++e) {
    x[e] = to_f(src[e]);
    amax = max(amax, __float_as_uint(x[e]) & 0x7fffffffu);
  }
  const bool finite = amax < 0x7f800000u;   // a NaN or an infinity is larger than every number
  const int ex = nscale_exp(finite ? amax : 0u);
  uint32_t *codes = reinterpret_cast<uint32_t *>((blockIdx.z & 1 ? c.V : c.K) + row * kNRow) + 4 * group;
  for (int e = 0; e < 4; ++e) codes[e] = finite ? npack8(x + 8 * e, pow2f(ex)) : 0u;
  reinterpret_cast<uint8_t *>((blockIdx.z & 1 ? c.Vs : c.Ks) + row)[group] = finite ? (uint8_t)(ex + 127) : 255;
}

hipError_t launch_ncache_write(int dtype, const NCache &c, int n, const void *K, const void *V, const int32_t *start,
                               const int32_t *count, hipStream_t s) {
  const dim3 grid((unsigned)((n + 63) / 64), (unsigned)min(c.P, kGridY), (unsigned)(2 * ((c.P + kGridY - 1) / kGridY)));
  if (dtype == ARCKV_BF16)
    hipLaunchKernelGGL(k_ncache_write<bf16>, grid, dim3(256), 0, s, c, n, (const bf16 *)K, (const bf16 *)V, start, count);
  else
    hipLaunchKernelGGL(k_ncache_write<float>, grid, dim3(256), 0, s, c, n, (const float *)K, (const float *)V, start, count);
  return hipGetLastError();
}

// ---------------------------------------------------------------- read
// A thread turns 8 codes.
template <typename T>
__global__ void __launch_bounds__(256) k_ncache_read(NCache c, int first, int n, const int32_t *__restrict__ length,
                                                     T *__restrict__ K, T *__restrict__ V) {
  const int p = (blockIdx.z >> 1) * gridDim.y + blockIdx.y;
  if (p >= c.P) return;
  const int i = blockIdx.x * 16 + threadIdx.x / 16, piece = threadIdx.x % 16;
  if (i >= n) return;
  float x[8] = {};
  if (first + i < clip_len(length, p, c.rows)) {
    const int64_t row = (int64_t)p * c.rows + first + i;
    const uint32_t w = reinterpret_cast<const uint32_t *>((blockIdx.z & 1 ? c.V : c.K) + row * kNRow)[piece];
    nunpack8(w, nscale(reinterpret_cast<const uint8_t *>((blockIdx.z & 1 ? c.Vs : c.Ks) + row)[piece / 4]), x);
  }
  T *out = (blockIdx.z & 1 ? V : K) + ((int64_t)p * n + i) * kHeadDim + 8 * piece;
  for (int e = 0; e < 8; ++e) out[e] = (T)x[e];
}

hipError_t launch_ncache_read(int dtype, const NCache &c, int first, int n, const int32_t *length, void *K, void *V,
                              hipStream_t s) {
  const dim3 grid((unsigned)((n + 15) / 16), (unsigned)min(c.P, kGridY), (unsigned)(2 * ((c.P + kGridY - 1) / kGridY)));
  if (dtype == ARCKV_BF16)
    hipLaunchKernelGGL(k_ncache_read<bf16>, grid, dim3(256), 0, s, c, first, n, length, (bf16 *)K, (bf16 *)V);
  else
    hipLaunchKernelGGL(k_ncache_read<float>, grid, dim3(256), 0, s, c, first, n, length, (float *)K, (float *)V);
  return hipGetLastError();
}

}  // namespace arckv
