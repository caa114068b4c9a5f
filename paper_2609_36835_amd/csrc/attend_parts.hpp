// Parts that the attention kernels over a quantised cache share: a step of a running softmax, probabilities as bf16 terms,
// the uncompressed bf16 tail, and the joining of partial results.
#pragma once
#include "qcode.hpp"

namespace arckv {

constexpr int kAttendTail = 32;       // tail rows per wave and step

namespace {

__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// LDS that only one wave uses: what its lanes wrote before is there for all of them (LDS takes a wave's accesses in order,
// so this holds back the compiler alone).
__device__ inline void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
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

// The word that lane r + FROM (mod 16) of the lane's row holds.
template <int FROM> __device__ inline uint32_t from_lane(uint32_t x) {
  return __builtin_amdgcn_update_dpp(0u, x, 0x120 + (16 - FROM), 0xf, 0xf, true);   // rotate right by 16 - FROM
}
template <int FROM> __device__ inline float from_lane(float x) { return __uint_as_float(from_lane<FROM>(__float_as_uint(x))); }

// One step of a running softmax per query: turns the lane's N logits into probabilities times 2^SHIFT, takes them (without
// 2^SHIFT) up in m and l, and returns what the earlier sums have to be multiplied by.  OWN: the probabilities are relative
// to the step's own largest logit, which fp16 terms need where it lies far below the largest of all, and `now` is what this
// step's sums have to be multiplied by; else they are relative to the new maximum and `now` is not used.  A query's logits lie
// in the lanes of its column r of the four rows, and, PARTS > 1, of the columns r + 16 / PARTS, ....  -inf marks keys left
// out; any: whether there is one that is not.
template <int N, int PARTS, int SHIFT, bool OWN>
__device__ inline float softmax_step(float (&sv)[N], float &m, float &l, bool &any, float &now) {
  auto larger = [](float x, float y) { return fmaxf(x, y); };
  auto plus = [](float x, float y) { return x + y; };
  float top = sv[0];
#pragma unroll
  for (int i = 1; i < N; ++i) top = fmaxf(top, sv[i]);
  if constexpr (PARTS == 4) top = fmaxf(top, from_lane<4>(top));
  if constexpr (PARTS >= 2) top = fmaxf(top, from_lane<8>(top));
  top = over_rows(top, larger);
  any = top != -INFINITY;
  const float own = any ? top : 0.0f;
  top = fmaxf(top, m);
  const float all = top == -INFINITY ? 0.0f : top, ref = OWN ? own : all;
  const float keep = __builtin_amdgcn_exp2f((m - all) * 1.44269504f);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sv[i] = __builtin_amdgcn_exp2f(fmaf(sv[i] - ref, 1.44269504f, (float)SHIFT));
    sum += sv[i];
  }
  if constexpr (PARTS == 4) sum += from_lane<4>(sum);
  if constexpr (PARTS >= 2) sum += from_lane<8>(sum);
  sum = over_rows(sum, plus);
  if constexpr (OWN) {
    now = any ? __builtin_amdgcn_exp2f((own - all) * 1.44269504f) : 0.0f;
    sum *= now;
  }
  m = top;
  l = fmaf(l, keep, sum * (1.0f / (1 << SHIFT)));
  return keep;
}

// 32 rows of the tail, `live` of them in use: what a wave has in flight of them.  The contraction steps are the blocks',
// so a lane reads 32 bytes at a time of a key.
template <typename A>
__device__ inline void load_tail_keys(const A &a, int64_t row0, int live, u32x4 (&k)[2][4]) {
  const int lane = threadIdx.x & 63, at = (lane & 15) * 2 * kHeadDim + 32 * (lane >> 4);
  const __amdgpu_buffer_rsrc_t kb = buffer(a.Kf + row0 * kHeadDim, live * 2 * kHeadDim);
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
      k[kt][ks] = __builtin_amdgcn_raw_buffer_load_b128(kb, at + 128 * (ks / 2) + 16 * (ks % 2), 32 * kHeadDim * kt, 0);
}

template <int NT, typename A>
__device__ inline void load_tail_values(const A &a, int64_t row0, int live, u32x4 (&v)[8]) {
  const int lane = threadIdx.x & 63, at = 4 * (lane >> 4) * 2 * kHeadDim + 16 * (lane & 15);
  const __amdgpu_buffer_rsrc_t vb = buffer(a.Vf + row0 * kHeadDim, live * 2 * kHeadDim);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    v[i] = __builtin_amdgcn_raw_buffer_load_b128(vb, at + 2 * kHeadDim * (i % 4), 32 * kHeadDim * (i / 4), NT);
}

// The tail's units of 32 rows first, first + W, ... below end, a wave's share of a chunk (ONE: one at most).  The queries
// stand in the first COLS of the 16 columns; sums in the others, whose maximum goes along, only keep up with it.  Probabilities
// enter the product, not their sum, times `down`.
template <int W, bool ONE, bool STREAM, int COLS, typename A>
__device__ inline void attend_tail(const A &a, int p, int first, int end, int len, const bf16x8 *s_q, float &m,
                                   float &l, f32x4 (&o)[8], float down = 1.0f) {
  constexpr int NTV = STREAM ? kStreamed : 0;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int64_t pr = (int64_t)p * a.F;
  auto live_at = [&](int idx) { return __builtin_amdgcn_readfirstlane(idx < end ? max(0, min(len - idx * kAttendTail, kAttendTail)) : 0); };
  int live = live_at(first);
  u32x4 k[2][4], v[8];
  load_tail_keys(a, pr + first * kAttendTail, live, k);
  load_tail_values<NTV>(a, pr + first * kAttendTail, live, v);
  for (int idx = first; idx < end; idx += W) {
    const int nlive = live_at(idx + W);
    const int64_t next = pr + (idx + W) * kAttendTail;
    float sv[8];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) acc = mfma16(__builtin_bit_cast(bf16x8, k[kt][ks]), s_q[ks * 64 + lane], acc);
#pragma unroll
      for (int j = 0; j < 4; ++j) sv[4 * kt + j] = 16 * kt + 4 * g + j < live ? a.scale * acc[j] : -INFINITY;
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!ONE) load_tail_keys(a, next, nlive, k);
    __builtin_amdgcn_sched_barrier(0);
    bool any;
    float now;
    const float keep = softmax_step<8, 1, 0, false>(sv, m, l, any, now);
#pragma unroll
    for (int i = 0; i < 8; ++i) sv[i] *= down;
    Frag ph, pm, pl;
    split_p(sv, ph, pm, pl);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      Frag b;
#pragma unroll
      for (int n = 0; n < 4; ++n)
        b.w[n] = e & 1 ? upper_halves(v[2 * n][e / 2], v[2 * n + 1][e / 2]) : lower_halves(v[2 * n][e / 2], v[2 * n + 1][e / 2]);
      // the first term has products of its own, which alone carry an infinite value (0 times it in the others is NaN)
      const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
      const f32x4 lead = mfma16(b.v, ph.v, zero), rest = mfma16(b.v, pm.v, mfma16(b.v, pl.v, zero));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float sum = fmaf(o[e][j], keep, fabsf(lead[j]) < INFINITY ? lead[j] + rest[j] : lead[j]);
        o[e][j] = COLS == 16 || (lane & 15) < COLS ? sum : o[e][j] * keep;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (ONE) return;
    load_tail_values<NTV>(a, next, nlive, v);
    __builtin_amdgcn_sched_barrier(0);
    live = nlive;
  }
}

// One workgroup per (query, pair): four groups of threads, thread = dim, take every fourth of the pair's partials, four
// loads at a time, and meet in LDS: 86 chunks of 8 pairs take 4.2 us (9.8 us with one group).
constexpr int kCombineGroups = 4, kCombineAhead = 4;
template <typename A, int GROUPS> __global__ void __launch_bounds__(GROUPS *kHeadDim) k_attend_combine(A a) {
  __shared__ float sM[GROUPS], sL[GROUPS], sA[GROUPS][kHeadDim];
  const int q = blockIdx.x, dim = threadIdx.x % kHeadDim, group = threadIdx.x / kHeadDim, p = blockIdx.z * gridDim.y + blockIdx.y;
  if (p >= a.c.P) return;
  const float *ml = a.part_ml + ((int64_t)p * a.nch * a.G + q) * 2;
  const float *po = a.part_o + ((int64_t)p * a.nch * a.G + q) * kHeadDim + dim;
  float M = -INFINITY, lsum = 0.0f, acc = 0.0f;
  for (int c0 = group; c0 < a.nch; c0 += GROUPS * kCombineAhead) {
    float m[kCombineAhead], l[kCombineAhead], o[kCombineAhead], top = M;
#pragma unroll
    for (int i = 0; i < kCombineAhead; ++i) {
      const int c = c0 + GROUPS * i;
      const int64_t at = (int64_t)min(c, a.nch - 1) * a.G;
      m[i] = ml[2 * at];
      l[i] = ml[2 * at + 1];
      o[i] = po[at * kHeadDim];
      if (c >= a.nch) m[i] = -INFINITY, l[i] = o[i] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kCombineAhead; ++i) top = fmaxf(top, m[i]);
    const float ref = top == -INFINITY ? 0.0f : top, keep = __expf(M - ref);
    lsum *= keep;
    acc *= keep;
#pragma unroll
    for (int i = 0; i < kCombineAhead; ++i) {
      const float f = __expf(m[i] - ref);   // a chunk without a key in use: zero, as its sums are
      lsum = fmaf(f, l[i], lsum);
      acc = fmaf(f, o[i], acc);
    }
    M = top;
  }
  if constexpr (GROUPS == 1) {
    a.out[((int64_t)p * a.G + q) * kHeadDim + dim] = lsum == 0.0f ? 0.0f : acc / lsum;
    return;
  }
  if (dim == 0) {
    sM[group] = M;
    sL[group] = lsum;
  }
  sA[group][dim] = acc;
  __syncthreads();
  if (group) return;
#pragma unroll
  for (int i = 1; i < GROUPS; ++i) M = fmaxf(M, sM[i]);
  const float ref = M == -INFINITY ? 0.0f : M;
  acc = lsum = 0.0f;
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const float f = __expf(sM[i] - ref);
    lsum = fmaf(f, sL[i], lsum);
    acc = fmaf(f, sA[i][dim], acc);
  }
  a.out[((int64_t)p * a.G + q) * kHeadDim + dim] = lsum == 0.0f ? 0.0f : acc / lsum;
}

}  // namespace

}  // namespace arckv
