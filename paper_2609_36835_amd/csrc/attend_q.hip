// Decode attention over the 8-bit cache, optionally over listed blocks of it
// only, followed by an uncompressed bf16 tail.  For pair p and each of its G
// query rows q:
//   o = softmax([s q K^T + beta, s q K_f^T]) [V; V_f],  K = scale * code
// over the rows below the pair's lengths whose bias is not -inf; a pair with
// none of them gets zeros.
//
// HBM-bound: 256 bytes of codes per token.  Split-key in two kernels:
//   k_attendq_partial  a wave takes one block of 64 tokens (so one key scale
//                      and one value scale), or 32 rows of the tail.  Codes
//                      become bf16 in registers, where they are exact, and feed
//                      MFMA 16x16x32: keys as rows and queries as columns for
//                      the logits, then the lane that holds a query's
//                      probabilities is the one that feeds them to P V.  The
//                      block's scales multiply the logits and the sums.  Eight
//                      waves' (max, sum, o) are merged in LDS.
//   k_attendq_combine  merges the partials of a pair; a call of one chunk per
//                      pair needs none.
#include "qcode.hpp"

namespace arckv {

namespace {
constexpr int kAqW = 8;               // waves per workgroup
constexpr int kAqTail = 32;           // tail rows per wave

__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

union Frag {
  uint32_t w[4];
  bf16x8 v;
};

__device__ inline uint32_t upper_halves(uint32_t first, uint32_t second) {
  return __builtin_amdgcn_perm(second, first, 0x07060302u);
}
__device__ inline uint32_t lower_halves(uint32_t first, uint32_t second) {
  return __builtin_amdgcn_perm(second, first, 0x05040100u);
}

// Four codes as two words of two bf16 each; every code is exact in bf16.
template <int FMT> __device__ inline void to_bf16x4(uint32_t w, uint32_t &first, uint32_t &second) {
  float y[4];
  QCode<FMT>::unpack4(w, y);
  first = upper_halves(__float_as_uint(y[0]), __float_as_uint(y[1]));
  second = upper_halves(__float_as_uint(y[2]), __float_as_uint(y[3]));
}

// Probabilities of 8 keys as three bf16 terms (truncated, so all of one sign) that
// sum to them exactly.
__device__ inline void split_p(const float *p, Frag &h, Frag &m, Frag &l) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t a[2], b[2], c[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float x = p[2 * k + i];
      a[i] = __float_as_uint(x) & 0xffff0000u;
      const float x1 = x - __uint_as_float(a[i]);
      b[i] = __float_as_uint(x1) & 0xffff0000u;
      c[i] = __float_as_uint(x1 - __uint_as_float(b[i]));
    }
    h.w[k] = upper_halves(a[0], a[1]);
    m.w[k] = upper_halves(b[0], b[1]);
    l.w[k] = upper_halves(c[0], c[1]);
  }
}

// Softmax of a wave's logits per query (columns r, keys over the lane's N and over g):
// probabilities in place, maximum and sum returned.  -inf marks keys left out.
template <int N> __device__ inline void wave_softmax(float (&sv)[N], float &m, float &l) {
  m = sv[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, sv[i]);
  m = fmaxf(m, __shfl_xor(m, 16, 64));
  m = fmaxf(m, __shfl_xor(m, 32, 64));
  const float mref = m == -INFINITY ? 0.0f : m;
  l = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sv[i] = __expf(sv[i] - mref);
    l += sv[i];
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
}
}  // namespace

struct AttendQ {
  QCache c;
  int G, F;
  float scale;
  const bf16 *Q;
  const float *beta;          // [P][rows] or null
  const int32_t *length;      // [P] or null
  const int32_t *blocks;      // [P][nsel] or null: every block
  int nsel;                   // list entries (blocks given), else c.nblk
  const bf16 *Kf, *Vf;
  const int32_t *length_f;
  float *part_o, *part_ml, *out;
  int nq, nch;                // chunks over the cache; with the tail's
};

// A block of 64 tokens, `live` of them in use (1..64).
template <int FMT>
__device__ inline void attend_block(const AttendQ &a, int p, int b, int live, const bf16 *Q, float &m, float &l,
                                    f32x4 (&o)[8]) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int64_t row0 = (int64_t)p * a.c.rows + (int64_t)b * kQBlock;
  // keys as MFMA rows; a contraction step pairs bytes 64 kk + 16 g + 8 h .. + 7 of keys and queries, so that a lane
  // reads 16 bytes at a time
  uint4 kc[4][2];
#pragma unroll
  for (int kt = 0; kt < 4; ++kt) {
    const uint8_t *row = a.c.K + (row0 + min(16 * kt + r, live - 1)) * kHeadDim + 16 * g;
    kc[kt][0] = *reinterpret_cast<const uint4 *>(row);
    kc[kt][1] = *reinterpret_cast<const uint4 *>(row + 64);
  }
  bf16x8 qf[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
    qf[ks] = *reinterpret_cast<const bf16x8 *>(Q + (int64_t)min(r, a.G - 1) * kHeadDim + 64 * (ks / 2) + 16 * g + 8 * (ks % 2));
  const float kscale = a.c.Ks[(int64_t)p * a.c.nblk + b] * a.scale, vscale = a.c.Vs[(int64_t)p * a.c.nblk + b];
  // values: the lane of keys 16 (i / 4) + 4 g + i % 4 (those of its logits) and dims 8 r .. 8 r + 7
  uint2 vc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i)
    vc[i] = *reinterpret_cast<const uint2 *>(a.c.V + (row0 + min(16 * (i / 4) + 4 * g + i % 4, live - 1)) * kHeadDim + 8 * r);
  float bv[16];
#pragma unroll
  for (int i = 0; i < 16; ++i)
    bv[i] = a.beta ? a.beta[row0 + min(16 * (i / 4) + 4 * g + i % 4, live - 1)] : 0.0f;
  float sv[16];
#pragma unroll
  for (int kt = 0; kt < 4; ++kt) {
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      const uint4 c = kc[kt][ks / 2];
      Frag k;
      to_bf16x4<FMT>(ks % 2 ? c.z : c.x, k.w[0], k.w[1]);
      to_bf16x4<FMT>(ks % 2 ? c.w : c.y, k.w[2], k.w[3]);
      acc = mfma16(k.v, qf[ks], acc);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = 4 * kt + j;
      const bool held = 16 * kt + 4 * g + j < live && bv[i] != -INFINITY;
      sv[i] = held ? fmaf(kscale, acc[j], bv[i]) : -INFINITY;
      if (!held) vc[i] = make_uint2(0u, 0u);   // its probability is zero, but zero times a NaN code is not
    }
  }
  wave_softmax(sv, m, l);
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    Frag ph, pm, pl, vb[8];
    split_p(sv + 8 * half, ph, pm, pl);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint2 x = vc[8 * half + 2 * k], y = vc[8 * half + 2 * k + 1];
#pragma unroll
      for (int dd = 0; dd < 2; ++dd) {
        // bytes of two keys side by side: dims 4 dd, 4 dd + 1, then 4 dd + 2, 4 dd + 3
        const uint32_t u = dd ? x.y : x.x, w = dd ? y.y : y.x;
        to_bf16x4<FMT>(__builtin_amdgcn_perm(w, u, 0x05010400u), vb[4 * dd].w[k], vb[4 * dd + 1].w[k]);
        to_bf16x4<FMT>(__builtin_amdgcn_perm(w, u, 0x07030602u), vb[4 * dd + 2].w[k], vb[4 * dd + 3].w[k]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = mfma16(ph.v, vb[e].v, mfma16(pm.v, vb[e].v, mfma16(pl.v, vb[e].v, o[e])));
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] *= vscale;
}

// 32 rows of the tail from row0 on, `live` of them in use (1..32).
__device__ inline void attend_tail(const AttendQ &a, int p, int row0, int live, const bf16 *Q, float &m, float &l,
                                   f32x4 (&o)[8]) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const int64_t first = (int64_t)p * a.F + row0;
  bf16x8 kf[2][4], qf[4];
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
      kf[kt][ks] = *reinterpret_cast<const bf16x8 *>(a.Kf + (first + min(16 * kt + r, live - 1)) * kHeadDim + 32 * ks + 8 * g);
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
    qf[ks] = *reinterpret_cast<const bf16x8 *>(Q + (int64_t)min(r, a.G - 1) * kHeadDim + 32 * ks + 8 * g);
  Frag vf[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    vf[i].v = *reinterpret_cast<const bf16x8 *>(a.Vf + (first + min(16 * (i / 4) + 4 * g + i % 4, live - 1)) * kHeadDim + 8 * r);
  float sv[8];
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) acc = mfma16(kf[kt][ks], qf[ks], acc);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = 4 * kt + j;
      const bool held = 16 * kt + 4 * g + j < live;
      sv[i] = held ? a.scale * acc[j] : -INFINITY;
      if (!held) vf[i] = Frag{};   // zero times an infinite value is not zero
    }
  }
  wave_softmax(sv, m, l);
  Frag ph, pm, pl;
  split_p(sv, ph, pm, pl);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    Frag b;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      b.w[k] = e & 1 ? upper_halves(vf[2 * k].w[e / 2], vf[2 * k + 1].w[e / 2])
                     : lower_halves(vf[2 * k].w[e / 2], vf[2 * k + 1].w[e / 2]);
    // the first term has products of its own, which alone carry an infinite value (0 times it in the others is NaN)
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    const f32x4 first_term = mfma16(ph.v, b.v, zero), rest = mfma16(pm.v, b.v, mfma16(pl.v, b.v, zero));
#pragma unroll
    for (int j = 0; j < 4; ++j) o[e][j] = fabsf(first_term[j]) < INFINITY ? first_term[j] + rest[j] : first_term[j];
  }
}

// GP: the query rows that the LDS has room for, G <= GP <= 16.
template <int FMT, int GP>
__global__ void __launch_bounds__(64 * kAqW) k_attendq_partial(AttendQ a) {
  __shared__ __align__(16) float sO[kAqW][GP][kHeadDim];
  __shared__ float sM[kAqW][GP], sL[kAqW][GP];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, r = lane & 15;
  const int ch = blockIdx.x;
  for (int p = blockIdx.y; p < a.c.P; p += gridDim.y) {
    const int len = clip_len(a.length, p, a.c.rows), len_f = clip_len(a.length_f, p, a.F);
    const int G = a.G;
    float m = -INFINITY, l = 0.0f;
    f32x4 o[8] = {};
    const bf16 *Q = a.Q + (int64_t)p * G * kHeadDim;
    bool used;   // whether the combine reads this chunk
    if (ch < a.nq) {
      const int idx = ch * kAqW + wave;
      used = a.blocks || ch * kAqW * kQBlock < len;
      int b = idx < a.nsel ? idx : -1;
      if (a.blocks && b >= 0) b = a.blocks[(int64_t)p * a.nsel + idx];
      const int live = b >= 0 && b < a.c.nblk ? min(len - b * kQBlock, kQBlock) : 0;
      if (live > 0) attend_block<FMT>(a, p, b, live, Q, m, l, o);
    } else {
      const int row0 = ((ch - a.nq) * kAqW + wave) * kAqTail;
      used = (ch - a.nq) * kAqW * kAqTail < len_f;
      const int live = min(len_f - row0, kAqTail);
      if (live > 0) attend_tail(a, p, row0, live, Q, m, l, o);
    }
    if (!used && a.nch > 1) continue;   // the whole workgroup
    if (g == 0 && r < G) {
      sM[wave][r] = m;
      sL[wave][r] = l;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (4 * g + j < G) {
        float *to = &sO[wave][4 * g + j][8 * r];
        *reinterpret_cast<float4 *>(to) = make_float4(o[0][j], o[1][j], o[2][j], o[3][j]);
        *reinterpret_cast<float4 *>(to + 4) = make_float4(o[4][j], o[5][j], o[6][j], o[7][j]);
      }
    __syncthreads();
    // one partial (max, sum, o) per query for the chunk; the result itself where there is one chunk
    for (int idx = tid; idx < G * kHeadDim; idx += 64 * kAqW) {
      const int q = idx / kHeadDim, dim = idx % kHeadDim;
      float M = sM[0][q];
#pragma unroll
      for (int w = 1; w < kAqW; ++w) M = fmaxf(M, sM[w][q]);
      float acc = 0.0f, lsum = 0.0f;
#pragma unroll
      for (int w = 0; w < kAqW; ++w) {
        if (sM[w][q] == -INFINITY) continue;   // no key in use; its o may be zero times a NaN scale
        const float f = __expf(sM[w][q] - M);
        acc = fmaf(f, sO[w][q][dim], acc);
        lsum = fmaf(f, sL[w][q], lsum);
      }
      if (a.nch == 1) {
        a.out[((int64_t)p * G + q) * kHeadDim + dim] = lsum == 0.0f ? 0.0f : acc / lsum;
      } else {
        const int64_t at = ((int64_t)p * a.nch + ch) * G + q;
        a.part_o[at * kHeadDim + dim] = acc;
        if (dim == 0) {
          a.part_ml[2 * at] = M;
          a.part_ml[2 * at + 1] = lsum;
        }
      }
    }
    __syncthreads();   // the next pair's chunk uses the same LDS
  }
}

// One workgroup per (query, pair): thread = dim merges the pair's partials.
__global__ void __launch_bounds__(kHeadDim) k_attendq_combine(AttendQ a) {
  const int q = blockIdx.x, dim = threadIdx.x;
  for (int p = blockIdx.y; p < a.c.P; p += gridDim.y) {
    const int len = clip_len(a.length, p, a.c.rows), len_f = clip_len(a.length_f, p, a.F);
    const int n0 = a.blocks ? a.nq : (len + kAqW * kQBlock - 1) / (kAqW * kQBlock);
    const int n1 = (len_f + kAqW * kAqTail - 1) / (kAqW * kAqTail);
    const int64_t base = (int64_t)p * a.nch * a.G + q;
    auto at = [&](int c) { return base + (int64_t)(c < n0 ? c : a.nq + c - n0) * a.G; };
    float M = -INFINITY;
#pragma unroll 8
    for (int c = 0; c < n0 + n1; ++c) M = fmaxf(M, a.part_ml[2 * at(c)]);
    float acc = 0.0f, lsum = 0.0f;
#pragma unroll 8
    for (int c = 0; c < n0 + n1; ++c) {
      const float mc = a.part_ml[2 * at(c)];
      const float f = mc == -INFINITY ? 0.0f : __expf(mc - M);
      acc = fmaf(f, a.part_o[at(c) * kHeadDim + dim], acc);
      lsum = fmaf(f, a.part_ml[2 * at(c) + 1], lsum);
    }
    a.out[((int64_t)p * a.G + q) * kHeadDim + dim] = lsum == 0.0f ? 0.0f : acc / lsum;
  }
}

// Chunks over the cache's blocks (or the list's) and over the tail.
int attendq_chunks(int nsel, int F, int *nq) {
  *nq = (nsel + kAqW - 1) / kAqW;
  return *nq + (F + kAqW * kAqTail - 1) / (kAqW * kAqTail);
}

hipError_t launch_attendq(int fmt, const QCache &c, int G, int F, float scale, const void *Q, const float *beta,
                          const int32_t *length, const int32_t *blocks, int nsel, const void *Kf, const void *Vf,
                          const int32_t *length_f, float *part_o, float *part_ml, float *out, hipStream_t s) {
  AttendQ a{c, G, F, scale, (const bf16 *)Q, beta, length, blocks, blocks ? nsel : c.nblk, (const bf16 *)Kf,
            (const bf16 *)Vf, length_f, part_o, part_ml, out, 0, 0};
  a.nch = attendq_chunks(a.nsel, F, &a.nq);
  const unsigned py = (unsigned)min(c.P, 65535);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3((unsigned)a.nch, py), dim3(64 * kAqW), 0, s, a);
    return hipGetLastError();
  };
  hipError_t e;
  if (fmt == ARCKV_E4M3)
    e = G <= 4 ? go(k_attendq_partial<ARCKV_E4M3, 4>)
               : G <= 8 ? go(k_attendq_partial<ARCKV_E4M3, 8>) : go(k_attendq_partial<ARCKV_E4M3, 16>);
  else
    e = G <= 4 ? go(k_attendq_partial<ARCKV_INT8, 4>)
               : G <= 8 ? go(k_attendq_partial<ARCKV_INT8, 8>) : go(k_attendq_partial<ARCKV_INT8, 16>);
  if (e != hipSuccess || a.nch == 1) return e;
  hipLaunchKernelGGL(k_attendq_combine, dim3((unsigned)G, py), dim3(kHeadDim), 0, s, a);
  return hipGetLastError();
}

}  // namespace arckv
