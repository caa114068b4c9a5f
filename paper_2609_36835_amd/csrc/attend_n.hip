// Decode attention over the 4-bit cache, followed by an uncompressed bf16 tail.
// For pair p and each of its G query rows q:
//   o = softmax([s q K^T + beta, s q K_f^T]) [V; V_f],  K = scale * code
// over the rows below the pair's lengths whose bias is not -inf; a pair with
// none of them gets zeros.
//
// One workgroup per query row: a wave takes every fourth row, a lane two channels, with a running softmax; the waves
// meet in LDS.
#include "ncode.hpp"

namespace arckv {

struct AttendN {
  NCache c;
  int G, F;
  float scale;
  const bf16 *Q;
  const float *beta;          // [P][rows] or null
  const int32_t *length;      // [P] or null
  const bf16 *Kf, *Vf;
  const int32_t *length_f;
  float *part_o, *part_ml, *out;
};

__global__ void __launch_bounds__(256) k_attendn(AttendN a) {
  __shared__ float sM[4], sL[4], sO[4][kHeadDim];
  const int q = blockIdx.x, p = blockIdx.z * gridDim.y + blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (p >= a.c.P) return;
  const bf16 *Q = a.Q + ((int64_t)p * a.G + q) * kHeadDim + 2 * lane;
  const float q0 = (float)Q[0], q1 = (float)Q[1];
  const int len = clip_len(a.length, p, a.c.rows), len_f = clip_len(a.length_f, p, a.F);
  float m = -INFINITY, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
  auto take = [&](float k0, float k1, float v0, float v1, float bias) {
    const float logit = fmaf(a.scale, wave_sum(fmaf(q0, k0, q1 * k1)), bias);
    const float top = fmaxf(m, logit), keep = m == top ? 1.0f : __expf(m - top), w = logit == top ? 1.0f : __expf(logit - top);
    l = fmaf(l, keep, w);
    o0 = fmaf(o0, keep, w * v0);
    o1 = fmaf(o1, keep, w * v1);
    m = top;
  };
  for (int i = wave; i < len; i += 4) {
    const int64_t row = (int64_t)p * a.c.rows + i;
    const float bias = a.beta ? a.beta[row] : 0.0f;
    if (bias == -INFINITY) continue;
    float k[8], v[8];
    nunpack8(a.c.K[row * kNRow + lane], nscale(a.c.Ks[row] >> (8 * (lane >> 4)) & 255u), k);
    nunpack8(a.c.V[row * kNRow + lane], nscale(a.c.Vs[row] >> (8 * (lane >> 4)) & 255u), v);
    take(k[0], k[1], v[0], v[1], bias);
  }
  for (int i = wave; i < len_f; i += 4) {
    const int64_t at = ((int64_t)p * a.F + i) * kHeadDim + 2 * lane;
    take((float)a.Kf[at], (float)a.Kf[at + 1], (float)a.Vf[at], (float)a.Vf[at + 1], 0.0f);
  }
  sO[wave][2 * lane] = o0;
  sO[wave][2 * lane + 1] = o1;
  if (lane == 0) {
    sM[wave] = m;
    sL[wave] = l;
  }
  __syncthreads();
  if (threadIdx.x >= kHeadDim) return;
  float M = -INFINITY, acc = 0.0f, sum = 0.0f;
  for (int w = 0; w < 4; ++w) M = fmaxf(M, sM[w]);
  for (int w = 0; w < 4; ++w) {
    const float f = sM[w] == M ? 1.0f : __expf(sM[w] - M);
    acc = fmaf(f, sO[w][threadIdx.x], acc);
    sum = fmaf(f, sL[w], sum);
  }
  a.out[((int64_t)p * a.G + q) * kHeadDim + threadIdx.x] = sum == 0.0f ? 0.0f : acc / sum;
}

int attendn_chunks(int P, int rows, int F) { return 1; }

hipError_t launch_attendn(const NCache &c, int G, int F, float scale, const void *Q, const float *beta,
                          const int32_t *length, const void *Kf, const void *Vf, const int32_t *length_f, float *part_o,
                          float *part_ml, float *out, hipStream_t s) {
  AttendN a{c, G, F, scale, (const bf16 *)Q, beta, length, (const bf16 *)Kf, (const bf16 *)Vf, length_f, part_o, part_ml, out};
  const unsigned py = (unsigned)min(c.P, 32768), pz = (unsigned)((c.P + 32767) / 32768);
  hipLaunchKernelGGL(k_attendn, dim3((unsigned)G, py, pz), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace arckv
