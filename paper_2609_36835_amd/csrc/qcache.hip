// The 8-bit cache: rows written into it, rows read back, and the choice of the
// blocks that a decode step attends to.
//
// A block is 64 consecutive tokens of one pair.  With A the largest magnitude
// among its keys (its values), the block's scale is the smallest power of two
// that brings A into the codes' range, and a code is x / scale rounded to the
// nearest, ties to even.  Powers of two make the division exact, so the codes
// are the same however they are computed, a stored value (scale times code) is
// exact in bf16, and writing a stored value again changes nothing.
#include "qcode.hpp"

namespace arckv {

hipError_t launch_select(const float *scores, int B, int T, int t, int32_t *anchors, hipStream_t s);

// ---------------------------------------------------------------- write
// One workgroup per (block, pair, keys or values).  Thread (row group, 8 dims)
// holds four of the block's rows in registers: the kept rows before `start`
// from the cache, the new ones from the source, so that a block's scale is that
// of all it holds.  One pass over memory: 2 (or 4) bytes in, 1 out per element.
template <int FMT, typename T, bool BOUNDS>
__device__ inline void write_block(uint8_t *codes, float *scales, uint8_t *bounds, const T *src, int p, int b, int rows,
                                   int nblk, int n, int start, int end) {
  __shared__ uint32_t s_amax[4];
  __shared__ float s_bound[4][2][kHeadDim];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int dim = 8 * (tid & 15), row0 = b * kQBlock + (tid >> 4);   // this thread's rows: row0 + 16 i
  float x[4][8];
  bool held[4];
  const float old_scale = b * kQBlock < start ? scales[(int64_t)p * nblk + b] : 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = row0 + 16 * i;
    held[i] = row < end;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = 0.0f;
    if (row < start) {
      const uint2 c = *reinterpret_cast<const uint2 *>(codes + ((int64_t)p * rows + row) * kHeadDim + dim);
      float y[2][4];
      QCode<FMT>::unpack4(c.x, y[0]);
      QCode<FMT>::unpack4(c.y, y[1]);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = y[e / 4][e % 4] * old_scale;
    } else if (row < end) {
      const T *from = src + ((int64_t)p * n + (row - start)) * kHeadDim + dim;
      if constexpr (sizeof(T) == 2) {
        const bf16x8 v = *reinterpret_cast<const bf16x8 *>(from);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = (float)v[e];
      } else {
        const float4 a = *reinterpret_cast<const float4 *>(from), c = *reinterpret_cast<const float4 *>(from + 4);
        x[i][0] = a.x; x[i][1] = a.y; x[i][2] = a.z; x[i][3] = a.w;
        x[i][4] = c.x; x[i][5] = c.y; x[i][6] = c.z; x[i][7] = c.w;
      }
    }
  }
  // largest magnitude as float bits: a NaN or an infinity is larger than every number
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(x[i][e]) & 0x7fffffffu);
  for (int m = 32; m >= 1; m >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, m, 64));
  if (lane == 0) s_amax[wave] = amax;
  if constexpr (BOUNDS) {
    // extremes before the scaling: rounding keeps the order, so the extremes' codes are the codes' extremes
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float lo = INFINITY, hi = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (held[i]) {
          lo = fminf(lo, x[i][e]);
          hi = fmaxf(hi, x[i][e]);
        }
#pragma unroll
      for (int m = 16; m <= 32; m <<= 1) {
        lo = fminf(lo, __shfl_xor(lo, m, 64));
        hi = fmaxf(hi, __shfl_xor(hi, m, 64));
      }
      if (lane < 16) {
        s_bound[wave][0][dim + e] = lo;
        s_bound[wave][1][dim + e] = hi;
      }
    }
  }
  __syncthreads();
  amax = max(max(s_amax[0], s_amax[1]), max(s_amax[2], s_amax[3]));
  const bool finite = amax < 0x7f800000u;
  const int ex = qscale_exp<FMT>(finite ? amax : 0u);
  const float inv = pow2f(-ex);
  if (tid == 0) scales[(int64_t)p * nblk + b] = finite ? pow2f(ex) : __uint_as_float(0x7fc00000u);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (!held[i]) continue;
    uint2 c;
    c.x = QCode<FMT>::pack4(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv);
    c.y = QCode<FMT>::pack4(x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv);
    if (!finite) c.x = c.y = 0u;
    *reinterpret_cast<uint2 *>(codes + ((int64_t)p * rows + row0 + 16 * i) * kHeadDim + dim) = c;
  }
  if constexpr (BOUNDS) {
    if (tid < 64) {
      const int which = tid >> 5, d4 = 4 * (tid & 31);
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a = s_bound[0][which][d4 + e], c = s_bound[1][which][d4 + e], f = s_bound[2][which][d4 + e],
                    g = s_bound[3][which][d4 + e];
        v[e] = (which ? fmaxf(fmaxf(a, c), fmaxf(f, g)) : fminf(fminf(a, c), fminf(f, g))) * inv;
      }
      const uint32_t w = finite ? QCode<FMT>::pack4(v[0], v[1], v[2], v[3]) : 0u;
      *reinterpret_cast<uint32_t *>(bounds + (((int64_t)p * nblk + b) * 2 + which) * kHeadDim + d4) = w;
    }
  }
}

template <int FMT, typename T>
__global__ void __launch_bounds__(256) k_qcache_write(QCache c, int n, const T *__restrict__ K, const T *__restrict__ V,
                                                      const int32_t *__restrict__ starts,
                                                      const int32_t *__restrict__ counts) {
  for (int p = blockIdx.y; p < c.P; p += gridDim.y) {
    const int start = starts ? min(max(starts[p], 0), c.rows) : 0;
    const int end = min(start + clip_len(counts, p, n), c.rows);
    const int b = start / kQBlock + blockIdx.x;
    if (end > start && b * kQBlock < end) {
      if (blockIdx.z)
        write_block<FMT, T, false>(c.V, c.Vs, nullptr, V, p, b, c.rows, c.nblk, n, start, end);
      else if (c.bounds)
        write_block<FMT, T, true>(c.K, c.Ks, c.bounds, K, p, b, c.rows, c.nblk, n, start, end);
      else
        write_block<FMT, T, false>(c.K, c.Ks, nullptr, K, p, b, c.rows, c.nblk, n, start, end);
    }
    __syncthreads();   // the next pair's block uses the same LDS
  }
}

hipError_t launch_qcache_write(int fmt, int dtype, const QCache &c, int n, const void *K, const void *V,
                               const int32_t *start, const int32_t *count, hipStream_t s) {
  // blocks that n rows can touch: one more than their number where they may begin inside a block
  const int spans = min(start ? (n + kQBlock - 2) / kQBlock + 1 : (n + kQBlock - 1) / kQBlock, c.nblk);
  const dim3 grid((unsigned)spans, (unsigned)min(c.P, 65535), 2);
  auto go = [&](auto kern, auto *k, auto *v) {
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, c, n, k, v, start, count);
    return hipGetLastError();
  };
  if (dtype == ARCKV_BF16)
    return fmt == ARCKV_E4M3 ? go(k_qcache_write<ARCKV_E4M3, bf16>, (const bf16 *)K, (const bf16 *)V)
                             : go(k_qcache_write<ARCKV_INT8, bf16>, (const bf16 *)K, (const bf16 *)V);
  return fmt == ARCKV_E4M3 ? go(k_qcache_write<ARCKV_E4M3, float>, (const float *)K, (const float *)V)
                           : go(k_qcache_write<ARCKV_INT8, float>, (const float *)K, (const float *)V);
}

// ---------------------------------------------------------------- read
// A thread turns 8 (bf16 out) or 4 (float32 out) codes of a row into 16 bytes.
template <int FMT, typename T>
__global__ void __launch_bounds__(256) k_qcache_read(QCache c, int first, int n, const int32_t *__restrict__ length,
                                                     T *__restrict__ K, T *__restrict__ V) {
  constexpr int PER = 16 / sizeof(T), LANES = kHeadDim / PER;   // codes per thread, threads per row
  const uint8_t *codes = blockIdx.z ? c.V : c.K;
  const float *scales = blockIdx.z ? c.Vs : c.Ks;
  T *out = blockIdx.z ? V : K;
  const int dim = PER * (threadIdx.x % LANES);
  const int i = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (i >= n) return;
  const int row = first + i;
  for (int p = blockIdx.y; p < c.P; p += gridDim.y) {
    float x[PER];
    if (row < clip_len(length, p, c.rows)) {
      const float s = scales[(int64_t)p * c.nblk + row / kQBlock];
      const uint32_t *from = reinterpret_cast<const uint32_t *>(codes + ((int64_t)p * c.rows + row) * kHeadDim + dim);
#pragma unroll
      for (int k = 0; k < PER / 4; ++k) {
        float y[4];
        QCode<FMT>::unpack4(from[k], y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * k + e] = y[e] * s;
      }
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e) x[e] = 0.0f;
    }
    T *to = out + ((int64_t)p * n + i) * kHeadDim + dim;
    if constexpr (sizeof(T) == 2) {
      bf16x8 v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (bf16)x[e];
      *reinterpret_cast<bf16x8 *>(to) = v;
    } else {
      *reinterpret_cast<float4 *>(to) = make_float4(x[0], x[1], x[2], x[3]);
    }
  }
}

hipError_t launch_qcache_read(int fmt, int dtype, const QCache &c, int first, int n, const int32_t *length, void *K,
                              void *V, hipStream_t s) {
  const int per_wg = 256 / (kHeadDim / (dtype == ARCKV_BF16 ? 8 : 4));
  const dim3 grid((unsigned)((n + per_wg - 1) / per_wg), (unsigned)min(c.P, 65535), 2);
  auto go = [&](auto kern, auto *k, auto *v) {
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, c, first, n, length, k, v);
    return hipGetLastError();
  };
  if (dtype == ARCKV_BF16)
    return fmt == ARCKV_E4M3 ? go(k_qcache_read<ARCKV_E4M3, bf16>, (bf16 *)K, (bf16 *)V)
                             : go(k_qcache_read<ARCKV_INT8, bf16>, (bf16 *)K, (bf16 *)V);
  return fmt == ARCKV_E4M3 ? go(k_qcache_read<ARCKV_E4M3, float>, (float *)K, (float *)V)
                           : go(k_qcache_read<ARCKV_INT8, float>, (float *)K, (float *)V);
}

// ---------------------------------------------------------------- block scores
// s_b = max_g [ scale * kappa_b * sum_d max(q_gd lo_bd, q_gd hi_bd) ] (+ max beta of
// the block's tokens): no logit of the block's stored keys exceeds it.  The
// order of blocks decides what a step attends to, so it must not hang on the
// rounding of a sum: the products of an 8-bit significand and a code are exact
// in float32, and their sum is taken in float64, where it is exact for queries
// whose channels span less than about 2^30.  Four lanes share a block, 32 channels each.
template <int FMT>
__global__ void __launch_bounds__(256) k_block_scores(QCache c, int G, double scale, const bf16 *__restrict__ Q,
                                                      const float *__restrict__ beta,
                                                      const int32_t *__restrict__ length,
                                                      float *__restrict__ scores) {
  __shared__ float sQ[16][4][36];   // a part's 32 channels, padded so that the four parts lie in different banks
  const int tid = threadIdx.x, part = tid & 3;
  const int b = blockIdx.x * 64 + (tid >> 2);
  for (int p = blockIdx.y; p < c.P; p += gridDim.y) {
    __syncthreads();
    for (int i = tid; i < G * kHeadDim; i += 256)
      sQ[i / kHeadDim][(i % kHeadDim) / 32][i % 32] = (float)Q[(int64_t)p * G * kHeadDim + i];
    __syncthreads();
    const int len = clip_len(length, p, c.rows);
    if (b >= c.nblk) continue;
    if (b * kQBlock >= len) {
      if (part == 0) scores[(int64_t)p * c.nblk + b] = -INFINITY;
      continue;
    }
    const uint8_t *bd = c.bounds + ((int64_t)p * c.nblk + b) * 2 * kHeadDim + 32 * part;
    float lo[32], hi[32];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint4 l = *reinterpret_cast<const uint4 *>(bd + 16 * k), h = *reinterpret_cast<const uint4 *>(bd + kHeadDim + 16 * k);
      const uint32_t lw[4] = {l.x, l.y, l.z, l.w}, hw[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float y[4], z[4];
        QCode<FMT>::unpack4(lw[j], y);
        QCode<FMT>::unpack4(hw[j], z);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[16 * k + 4 * j + e] = y[e];
          hi[16 * k + 4 * j + e] = z[e];
        }
      }
    }
    double best = -INFINITY;
    bool nan = false;
    for (int g = 0; g < G; ++g) {
      double sum = 0.0;
#pragma unroll
      for (int d = 0; d < 32; ++d) {
        const float q = sQ[g][part][d];
        sum += (double)(q * (q >= 0.0f ? hi[d] : lo[d]));
      }
      sum += __shfl_xor(sum, 1, 64);
      sum += __shfl_xor(sum, 2, 64);
      nan |= sum != sum;
      best = fmax(best, sum);
    }
    double score = best * (scale * (double)c.Ks[(int64_t)p * c.nblk + b]);
    if (beta) {
      const float *row = beta + (int64_t)p * c.rows + b * kQBlock;
      float top = -INFINITY;
      for (int j = part; j < min(kQBlock, len - b * kQBlock); j += 4) {
        nan |= row[j] != row[j];
        top = fmaxf(top, row[j]);
      }
      top = fmaxf(top, __shfl_xor(top, 1, 64));
      top = fmaxf(top, __shfl_xor(top, 2, 64));
      score = top == -INFINITY ? -INFINITY : score + (double)top;
    }
    int bad = nan;
    bad |= __shfl_xor(bad, 1, 64);
    bad |= __shfl_xor(bad, 2, 64);
    if (part == 0) scores[(int64_t)p * c.nblk + b] = bad ? __uint_as_float(0x7fc00000u) : (float)score;
  }
}

hipError_t launch_select_blocks(int fmt, const QCache &c, int G, double scale, const void *Q, const float *beta,
                                const int32_t *length, int k, float *scores, int32_t *blocks, hipStream_t s) {
  const dim3 grid((unsigned)((c.nblk + 63) / 64), (unsigned)min(c.P, 65535));
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, c, G, scale, (const bf16 *)Q, beta, length, scores);
    return hipGetLastError();
  };
  const hipError_t e = fmt == ARCKV_E4M3 ? go(k_block_scores<ARCKV_E4M3>) : go(k_block_scores<ARCKV_INT8>);
  return e != hipSuccess ? e : launch_select(scores, c.P, c.nblk, k, blocks, s);
}

}  // namespace arckv
