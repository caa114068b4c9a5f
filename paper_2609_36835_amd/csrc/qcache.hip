// The 8-bit cache: rows written into it, rows read back, and the choice of the
// blocks that a decode step attends to.
//
// A block is 64 consecutive tokens of one pair.  With A the largest magnitude
// among its keys (its values), the block's scale is the smallest power of two
// that brings A into the codes' range, and a code is x / scale rounded to the
// nearest, ties to even.  Powers of two make the division exact, so the codes
// are the same however they are computed, a stored value (scale times code) is
// exact in bf16, and writing a stored value again changes nothing.
#include <type_traits>

#include "qcode.hpp"

namespace arckv {

hipError_t launch_select(const float *scores, int B, int T, int t, int32_t *anchors, hipStream_t s);

// pairs lie over a grid's y and z, whose extents are limited
constexpr int kGridY = 32768;

// ---------------------------------------------------------------- write
// One workgroup per (block, pair, keys or values).  Thread (row group, 8 dims)
// holds four of the block's rows in registers: the kept rows before `start`
// from the cache, the new ones from the source, so that a block's scale is that
// of all it holds.  One pass over memory: 2 (or 4) bytes in, 1 out per element,
// both as streams.  Loads go through the bounds-checked path, which gives zeros
// for rows of the other kind, so none waits in a branch.
template <int FMT, typename T, bool BOUNDS>
__device__ inline void write_block(uint8_t *codes, float *scales, uint8_t *bounds, const T *src, int p, int b, int rows,
                                   int nblk, int n, int start, int end) {
  __shared__ uint32_t s_amax[4];
  __shared__ float s_bound[4][2][kHeadDim];
  constexpr int kRow = kHeadDim * sizeof(T), kOutside = 1 << 30;   // an offset behind every block
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int dim = 8 * (tid & 15), r0 = tid >> 4;        // this thread's rows of the block: r0 + 16 i
  const int row0 = b * kQBlock;
  // the same in every lane, which a median instruction hides from the compiler
  const int kept = __builtin_amdgcn_readfirstlane(min(max(start - row0, 0), kQBlock)),
            held = __builtin_amdgcn_readfirstlane(min(end - row0, kQBlock));
  uint8_t *block = codes + ((int64_t)p * rows + row0) * kHeadDim;
  float x[4][8];
  {
    const __amdgpu_buffer_rsrc_t from = buffer(src + ((int64_t)p * n + row0 + kept - start) * kHeadDim, (held - kept) * kRow);
    u32x4 v[4][sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = r0 + 16 * i < kept ? kOutside : (r0 + 16 * i - kept) * kRow + dim * (int)sizeof(T);
#pragma unroll
      for (int h = 0; h < (int)sizeof(T) / 2; ++h)
        v[i][h] = __builtin_amdgcn_raw_buffer_load_b128(from, at + 16 * h, 0, kStreamed);
    }
    if (kept > 0) {
      const float old = scales[(int64_t)p * nblk + b];
      const __amdgpu_buffer_rsrc_t before = buffer(block, kept * kHeadDim);
      u32x2 c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = __builtin_amdgcn_raw_buffer_load_b64(before, (r0 + 16 * i) * kHeadDim + dim, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y[2][4];
        QCode<FMT>::unpack4(c[i][0], y[0]);
        QCode<FMT>::unpack4(c[i][1], y[1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = y[e / 4][e % 4] * old;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = sizeof(T) == 2 ? __uint_as_float(e & 1 ? v[i][0][e / 2] & 0xffff0000u : v[i][0][e / 2] << 16)
                                       : __uint_as_float(v[i][(e / 4) % (sizeof(T) / 2)][e % 4]);
        x[i][e] = r0 + 16 * i < kept ? x[i][e] : y;
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
      for (int i = 0; i < 4; ++i) {
        lo = r0 + 16 * i < held ? fminf(lo, x[i][e]) : lo;
        hi = r0 + 16 * i < held ? fmaxf(hi, x[i][e]) : hi;
      }
      lo = over_rows(lo, [](float a, float c) { return fminf(a, c); });
      hi = over_rows(hi, [](float a, float c) { return fmaxf(a, c); });
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
    u32x2 c;
    c[0] = QCode<FMT>::pack4(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv);
    c[1] = QCode<FMT>::pack4(x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv);
    if (!finite) c = u32x2{0u, 0u};
    if (r0 + 16 * i < held)
      __builtin_nontemporal_store(c, reinterpret_cast<u32x2 *>(block + (r0 + 16 * i) * kHeadDim + dim));
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
  const int p = (blockIdx.z >> 1) * gridDim.y + blockIdx.y;
  if (p >= c.P) return;
  const int start = starts ? __builtin_amdgcn_readfirstlane(min(max(starts[p], 0), c.rows)) : 0;
  const int end = __builtin_amdgcn_readfirstlane(min(start + clip_len(counts, p, n), c.rows));
  const int b = start / kQBlock + blockIdx.x;
  if (end <= start || b * kQBlock >= end) return;
  if (blockIdx.z & 1)
    write_block<FMT, T, false>(c.V, c.Vs, nullptr, V, p, b, c.rows, c.nblk, n, start, end);
  else if (c.bounds)
    write_block<FMT, T, true>(c.K, c.Ks, c.bounds, K, p, b, c.rows, c.nblk, n, start, end);
  else
    write_block<FMT, T, false>(c.K, c.Ks, nullptr, K, p, b, c.rows, c.nblk, n, start, end);
}

hipError_t launch_qcache_write(int fmt, int dtype, const QCache &c, int n, const void *K, const void *V,
                               const int32_t *start, const int32_t *count, hipStream_t s) {
  // blocks that n rows can touch: one more than their number where they may begin inside a block
  const int spans = min(start ? (n + kQBlock - 2) / kQBlock + 1 : (n + kQBlock - 1) / kQBlock, c.nblk);
  const dim3 grid((unsigned)spans, (unsigned)min(c.P, kGridY), (unsigned)(2 * ((c.P + kGridY - 1) / kGridY)));
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
// A thread turns 8 (bf16 out) or 4 (float32 out) codes of each of four rows into
// 16 bytes, written as a stream.
constexpr int kReadRows = 4;
template <int FMT, typename T>
__global__ void __launch_bounds__(256) k_qcache_read(QCache c, int first, int n, const int32_t *__restrict__ length,
                                                     T *__restrict__ K, T *__restrict__ V) {
  constexpr int PER = 16 / sizeof(T), LANES = kHeadDim / PER, STEP = 256 / LANES;   // codes per thread; threads per row; rows at a time
  const int p = (blockIdx.z >> 1) * gridDim.y + blockIdx.y;
  if (p >= c.P) return;
  const uint8_t *codes = blockIdx.z & 1 ? c.V : c.K;
  const float *scales = (blockIdx.z & 1 ? c.Vs : c.Ks) + (int64_t)p * c.nblk;
  T *out = (blockIdx.z & 1 ? V : K) + (int64_t)p * n * kHeadDim;
  const int dim = PER * (threadIdx.x % LANES), i0 = blockIdx.x * (kReadRows * STEP) + threadIdx.x / LANES;
  const int len = clip_len(length, p, c.rows);
  uint32_t w[kReadRows][PER / 4];
  float s[kReadRows];
#pragma unroll
  for (int k = 0; k < kReadRows; ++k) {
    const int row = first + i0 + k * STEP, at = max(min(row, len - 1), 0);   // in range always; rows past the end are not used
    s[k] = row < len ? scales[at / kQBlock] : 0.0f;
    __builtin_memcpy(w[k], codes + ((int64_t)p * c.rows + at) * kHeadDim + dim, PER);
  }
#pragma unroll
  for (int k = 0; k < kReadRows; ++k) {
    const int i = i0 + k * STEP;
    float x[PER];
#pragma unroll
    for (int h = 0; h < PER / 4; ++h) {
      float y[4];
      QCode<FMT>::unpack4(w[k][h], y);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * h + e] = first + i < len ? y[e] * s[k] : 0.0f;
    }
    if (i >= n) continue;
    u32x4 v;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_perm(__float_as_uint(x[2 * e + 1]), __float_as_uint(x[2 * e]), 0x07060302u);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(x[e]);
    }
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(out + (int64_t)i * kHeadDim + dim));
  }
}

hipError_t launch_qcache_read(int fmt, int dtype, const QCache &c, int first, int n, const int32_t *length, void *K,
                              void *V, hipStream_t s) {
  const int per_wg = kReadRows * 256 / (kHeadDim / (dtype == ARCKV_BF16 ? 8 : 4));
  const dim3 grid((unsigned)((n + per_wg - 1) / per_wg), (unsigned)min(c.P, kGridY),
                  (unsigned)(2 * ((c.P + kGridY - 1) / kGridY)));
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
// the block's tokens): no logit of the block's stored keys exceeds it but by its
// roundings.  The order of blocks decides what a step attends to, so it must not
// hang on the order of a sum: the parts below are exact sums, four of them a
// query row, and meet in float64 (exactly for int8, 48 bits; 57 in e4m3) before
// the one rounding to float32.
//
// The sum is (q+ . hi) + (q- . lo) with the positive and negative parts of q, a
// product of matrices, and MFMA's float32 sums are exact if every product is a
// whole number of units and their sum stays below 2^24 of them.  So a query row
// enters as four planes of 8 bits each below its largest magnitude 2^E,
//   q = sum_t D_t 2^(E - 8 (t + 1)), D_t whole, |D_t| < 256
// (exact for channels down to 2^(E - 24); smaller ones lose what lies below
// 2^(E - 32)), four query rows times four planes filling the 16 columns, and
// codes as they are (int8: |c| <= 127, units of 1) or as nearest whole numbers
// and the rests in units of 2^-9 (e4m3: both at most 448 and 256 units): at
// most 448 * 255 * 128 < 2^24.
constexpr int kBsTile = 16;   // blocks per wave and step

// max and sum over lanes of a 16-lane row by DPP moves of a double's halves
template <int CTRL> __device__ inline double dpp(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0u, (uint32_t)u, CTRL, 0xf, 0xf, true),
                 hi = __builtin_amdgcn_update_dpp(0u, (uint32_t)(u >> 32), CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
constexpr int kDppXor1 = 0xb1, kDppXor2 = 0x4e, kDppRor4 = 0x124, kDppRor8 = 0x128;
__device__ inline f32x4 mfma_f16(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight codes as fp16: whole numbers and, for e4m3, rests.
template <int FMT> __device__ inline void code_parts(uint32_t w0, uint32_t w1, f16x8 &whole, f16x8 &rest) {
  uint32_t out[4], low[4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w = i ? w1 : w0;
    if constexpr (FMT == ARCKV_INT8) {
      // a byte u below fp16's exponent of 1024 is 1024 + u; with the code's sign bit flipped u is code + 128
      const f16x2 off = {(f16)-1152.0f, (f16)-1152.0f};
      const uint32_t u = w ^ 0x80808080u;
      out[2 * i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off);
      out[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f16x2 big = {(f16)1536.0f, (f16)1536.0f};   // fp16 steps by 1 here
        const f16x2 x = __builtin_bit_cast(f16x2, h ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true)
                                                    : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
        const f16x2 n = (x + big) - big;
        out[2 * i + h] = __builtin_bit_cast(uint32_t, n);
        low[2 * i + h] = __builtin_bit_cast(uint32_t, x - n);
      }
    }
  }
  __builtin_memcpy(&whole, out, 16);
  if constexpr (FMT == ARCKV_E4M3) __builtin_memcpy(&rest, low, 16);
}

// A pair's query planes in LDS and their exponents.  CT: tiles of 16 columns, four query rows each.
constexpr int kNoQuery = INT32_MIN, kBadQuery = INT32_MAX;   // in the place of an exponent: no row; a non-finite one
template <int CT> struct Planes {
  f16 d[2][16 * CT][kHeadDim + 8];   // of q+ and q-, row = column 4 g + t; padded for the banks
  int e[4 * CT];
};

// A wave a query row, two channels a lane; the workgroup meets afterwards.
template <int CT> __device__ inline void make_planes(const bf16 *Q, int G, Planes<CT> &pl) {
  const int lane = threadIdx.x & 63;
  uint32_t word[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int g = 4 * ct + (threadIdx.x >> 6);
    word[ct] = g < G ? reinterpret_cast<const uint32_t *>(Q + g * kHeadDim)[lane] : 0u;
  }
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int g = 4 * ct + (threadIdx.x >> 6);
    const float q[2] = {__uint_as_float(word[ct] << 16), __uint_as_float(word[ct] & 0xffff0000u)};
    uint32_t amax = max(__float_as_uint(q[0]) & 0x7fffffffu, __float_as_uint(q[1]) & 0x7fffffffu);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, m, 64));
    const bool finite = amax < 0x7f800000u;
    int E = 0;
    if (finite && amax) E = __builtin_amdgcn_frexp_expf(__uint_as_float(amax));   // amax < 2^E
    if (lane == 0) pl.e[g] = g >= G ? kNoQuery : finite ? E : kBadQuery;
    float x[2] = {ldexpf(q[0], 8 - E), ldexpf(q[1], 8 - E)};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f16x2 plus, minus;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float n = finite ? truncf(x[e]) : 0.0f;
        plus[e] = (f16)fmaxf(n, 0.0f);
        minus[e] = (f16)fminf(n, 0.0f);
        x[e] = (x[e] - n) * 256.0f;
      }
      *reinterpret_cast<f16x2 *>(&pl.d[0][4 * g + t][2 * lane]) = plus;
      *reinterpret_cast<f16x2 *>(&pl.d[1][4 * g + t][2 * lane]) = minus;
    }
  }
  __syncthreads();
}

// The tile's bounds that a lane needs: block r's, bytes 64 kk + 16 kg .. + 15.
struct TileBounds {
  uint4 lo[2], hi[2];
};
__device__ inline TileBounds load_bounds(const QCache &c, int p, int tile) {
  const int lane = threadIdx.x & 63, b = min(tile * kBsTile + (lane & 15), c.nblk - 1);
  const uint8_t *row = c.bounds + ((int64_t)p * c.nblk + b) * 2 * kHeadDim + 16 * (lane >> 4);
  TileBounds t;
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    t.lo[kk] = *reinterpret_cast<const uint4 *>(row + 64 * kk);
    t.hi[kk] = *reinterpret_cast<const uint4 *>(row + kHeadDim + 64 * kk);
  }
  return t;
}

// A wave's scores of the tile's 16 blocks: lane 16 kg + j (j < 4) returns block 4 kg + j's.
template <int FMT, int CT, bool BETA>
__device__ inline float tile_scores(const QCache &c, const TileBounds &t, int p, int tile, int len, int G, double scale,
                                    const float *beta, const Planes<CT> &pl) {
  const int lane = threadIdx.x & 63, kg = lane >> 4, r = lane & 15, b0 = tile * kBsTile;
  if (b0 * kQBlock >= len) return -INFINITY;
  const int b = b0 + 4 * kg + (r & 3);   // this lane's output
  const bool there = b < c.nblk && b * kQBlock < len;
  const double kscale = there ? scale * (double)c.Ks[(int64_t)p * c.nblk + b] : 0.0;
  float top = -INFINITY;
  if constexpr (BETA) {
    // four lanes a block, 16 biases each; a NaN wins
    const int j0 = (b0 + (lane >> 2)) * kQBlock + 16 * (lane & 3), j1 = min(j0 + 16, len);
    for (int j = j0; j < j1; ++j) {
      const float x = beta[(int64_t)p * c.rows + j];
      top = x > top || x != x ? x : top;
    }
#pragma unroll
    for (int m = 1; m <= 2; m <<= 1) {
      const float x = __shfl_xor(top, m, 64);
      top = x > top || x != x ? x : top;
    }
    top = __shfl(top, 4 * (4 * kg + (r & 3)), 64);
  }
  f32x4 acc[CT][2] = {};
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    // channels 64 kk + 16 kg + 8 h .. + 7, as the codes were read
    const int kk = ks / 2, h = ks % 2, d = 64 * kk + 16 * kg + 8 * h;
    f16x8 hn, hr, ln, lr;
    code_parts<FMT>(h ? t.hi[kk].z : t.hi[kk].x, h ? t.hi[kk].w : t.hi[kk].y, hn, hr);
    code_parts<FMT>(h ? t.lo[kk].z : t.lo[kk].x, h ? t.lo[kk].w : t.lo[kk].y, ln, lr);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const f16x8 qp = *reinterpret_cast<const f16x8 *>(&pl.d[0][16 * ct + r][d]),
                  qn = *reinterpret_cast<const f16x8 *>(&pl.d[1][16 * ct + r][d]);
      acc[ct][0] = mfma_f16(ln, qn, mfma_f16(hn, qp, acc[ct][0]));
      if constexpr (FMT == ARCKV_E4M3) acc[ct][1] = mfma_f16(lr, qn, mfma_f16(hr, qp, acc[ct][1]));
    }
  }
  double best = 0.0, weight[CT];
  bool bad = false;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int e = pl.e[4 * ct + (r >> 2)];
    weight[ct] = e == kNoQuery ? 0.0 : ldexp(1.0, e - 8 * ((r & 3) + 1));
    bad |= e == kBadQuery;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {   // blocks 4 kg + j
    double m = -INFINITY;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      double x = (double)acc[ct][0][j];
      if constexpr (FMT == ARCKV_E4M3) x += (double)acc[ct][1][j];
      x *= weight[ct];
      x += dpp<kDppXor1>(x);
      x += dpp<kDppXor2>(x);
      m = fmax(m, weight[ct] > 0.0 ? x : -INFINITY);   // a row that is not there never is the largest
    }
    m = fmax(m, dpp<kDppRor4>(m));
    m = fmax(m, dpp<kDppRor8>(m));
    best = (r & 3) == j ? m : best;
  }
  if (__any(bad)) best = __longlong_as_double(0x7ff8000000000000ll);   // a non-finite query gives NaN scores
  double score = best * kscale;
  if constexpr (BETA) score = top == -INFINITY ? -INFINITY : score + (double)top;
  return there ? (float)score : -INFINITY;
}

// A wave per tile of 16 blocks and step.  The next tile's bounds are asked for before this one's scores, but do not stay in
// flight: loads return in order, and the wait for this tile's scales (the queries', for the first tile) is for them too.
template <int FMT, int CT, bool BETA>
__global__ void __launch_bounds__(256) k_block_scores(QCache c, int G, double scale, const bf16 *__restrict__ Q,
                                                      const float *__restrict__ beta,
                                                      const int32_t *__restrict__ length,
                                                      float *__restrict__ scores) {
  __shared__ __align__(16) Planes<CT> pl;
  const int p = blockIdx.z * gridDim.y + blockIdx.y, lane = threadIdx.x & 63;
  if (p >= c.P) return;
  int tile = blockIdx.x * 4 + (threadIdx.x >> 6);
  TileBounds t = load_bounds(c, p, tile);
  const int len = clip_len(length, p, c.rows);
  make_planes<CT>(Q + (int64_t)p * G * kHeadDim, G, pl);
  while (tile * kBsTile < c.nblk) {
    const int next = tile + 4 * gridDim.x;
    const TileBounds ahead = load_bounds(c, p, next);
    const float score = tile_scores<FMT, CT, BETA>(c, t, p, tile, len, G, scale, beta, pl);
    const int b = tile * kBsTile + 4 * (lane >> 4) + (lane & 15);
    if ((lane & 15) < 4 && b < c.nblk) scores[(int64_t)p * c.nblk + b] = score;
    t = ahead;
    tile = next;
  }
}

// The k largest of a pair's n scores in launch_select's order: larger first, ties to the lower index, NaN below every
// number.  WAVES of a workgroup (one: each wave a pair of its own) hold up to 64 KEYS keys each, lane l of wave w the keys
// (64 w + l) per .. + per - 1, so indices ascend with the lanes.  The k-th largest key is found two bits at a time from
// the top, by counting (ballots) the keys at or above the three candidates; then every lane writes the indices of its keys
// above it, and of those equal to it as many as are still wanted.  Each key's load stands under its own condition and is waited
// for before the next.
template <int WAVES, int KEYS>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) k_pick_blocks(const float *__restrict__ scores, int P, int n,
                                                                               int k, int32_t *__restrict__ blocks) {
  __shared__ uint64_t s_count[2][WAVES];   // three counts of 21 bits
  __shared__ uint32_t s_sum[WAVES];
  const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : threadIdx.x >> 6;
  const int p = WAVES == 1 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (p >= P) return;
  const int per = (n + 64 * WAVES - 1) / (64 * WAVES), at0 = (64 * wave + lane) * per;
  uint32_t key[KEYS];   // a key that is not there is 0, below every candidate but the NaNs' own, 0, which is not counted
#pragma unroll
  for (int i = 0; i < KEYS; ++i) key[i] = i < per && at0 + i < n ? score_key(scores[(int64_t)p * n + at0 + i]) : 0u;
  uint32_t kth = 0;
  for (int shift = 30, buf = 0; shift >= 0; shift -= 2, buf ^= 1) {
    int count[3] = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < KEYS; ++i)
#pragma unroll
      for (int d = 0; d < 3; ++d) count[d] += __popcll(__ballot(key[i] >= (kth | (uint32_t)(d + 1) << shift)));
    if constexpr (WAVES > 1) {
      if (lane == 0) s_count[buf][wave] = (uint64_t)count[2] << 42 | (uint64_t)count[1] << 21 | (uint64_t)count[0];
      __syncthreads();
      uint64_t all = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) all += s_count[buf][w];
#pragma unroll
      for (int d = 0; d < 3; ++d) count[d] = (int)(all >> 21 * d & 0x1fffff);
    }
    kth |= (uint32_t)(count[2] >= k ? 3 : count[1] >= k ? 2 : count[0] >= k ? 1 : 0) << shift;
  }
  uint32_t above = 0, equal = 0;
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    const bool in = i < per && at0 + i < n;
    above += in && key[i] > kth;
    equal += in && key[i] == kth;
  }
  const uint32_t both = above << 16 | equal;   // at most 2048 each
  uint32_t sum = both;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t x = __shfl_up(sum, off, 64);
    sum += lane >= off ? x : 0u;
  }
  uint32_t before = sum - both, total = __shfl(sum, 63, 64);
  if constexpr (WAVES > 1) {
    if (lane == 63) s_sum[wave] = sum;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      before += w < wave ? s_sum[w] : 0u;
      total += s_sum[w];
    }
  }
  const uint32_t wanted = (uint32_t)k - (total >> 16);   // of the equal ones
  uint32_t seen = before & 0xffffu, at = (before >> 16) + min(seen, wanted);
  int32_t *out = blocks + (int64_t)p * k;
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    const bool in = i < per && at0 + i < n, eq = in && key[i] == kth;
    if (in && (key[i] > kth || (eq && seen < wanted))) out[at++] = at0 + i;
    seen += eq;
  }
}

hipError_t launch_select_blocks(int fmt, const QCache &c, int G, double scale, const void *Q, const float *beta,
                                const int32_t *length, int k, float *scores, int32_t *blocks, hipStream_t s) {
  const unsigned py = (unsigned)min(c.P, kGridY), pz = (unsigned)((c.P + kGridY - 1) / kGridY);
  // two tiles a wave where that leaves the CUs four workgroups each: the planes are made once for both
  const int by4 = (c.nblk + 4 * kBsTile - 1) / (4 * kBsTile);
  const dim3 grid((unsigned)((int64_t)c.P * by4 > 2048 - 1 ? (by4 + 2 - 1) / 2 : by4), py, pz);
  auto by_tiles = [&](auto fm, auto ct, auto bt) {
    constexpr int FMT = decltype(fm)::value, CT = decltype(ct)::value;
    constexpr bool BETA = decltype(bt)::value;
    hipLaunchKernelGGL((k_block_scores<FMT, CT, BETA>), grid, dim3(256), 0, s, c, G, scale, (const bf16 *)Q, beta, length,
                       scores);
    return hipGetLastError();
  };
  auto by_rows = [&](auto fm, auto bt) {
    return G <= 4 ? by_tiles(fm, std::integral_constant<int, 1>{}, bt)
                  : G <= 8 ? by_tiles(fm, std::integral_constant<int, 2>{}, bt) : by_tiles(fm, std::integral_constant<int, 4>{}, bt);
  };
  auto by_beta = [&](auto fm) { return beta ? by_rows(fm, std::true_type{}) : by_rows(fm, std::false_type{}); };
  const hipError_t e = fmt == ARCKV_E4M3 ? by_beta(std::integral_constant<int, ARCKV_E4M3>{})
                                         : by_beta(std::integral_constant<int, ARCKV_INT8>{});
  if (e != hipSuccess) return e;
  auto pick = [&](auto kern, int per_wg, int threads) {
    hipLaunchKernelGGL(kern, dim3((unsigned)((c.P + per_wg - 1) / per_wg)), dim3((unsigned)threads), 0, s, scores, c.P, c.nblk,
                       k, blocks);
    return hipGetLastError();
  };
  // a wave per pair up to 256 blocks (512 pairs of 256 4.3 us, 10.7 in k_select_topt), four up to 1024 (the call for 64
  // pairs of 1024 14.1 us, 16.1), eight up to 2048 (for 64 pairs 19.4 us, 20.1)
  if (c.nblk <= 256) return pick(k_pick_blocks<1, 4>, 4, 256);
  if (c.nblk <= 1024) return pick(k_pick_blocks<4, 4>, 1, 256);
  if (c.nblk <= 2048) return pick(k_pick_blocks<8, 4>, 1, 512);
  return launch_select(scores, c.P, c.nblk, k, blocks, s);
}

}  // namespace arckv
