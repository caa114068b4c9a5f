// Rotary positions: pairs of channels turned by position * frequency.
//
// One workgroup per token, a thread a pair of channels; the angle's sine and cosine serve all heads.
#include "common.hpp"
#include "rotary.hpp"

namespace arckv {

template <typename T> __global__ void __launch_bounds__(256) k_rotary(Rotary a) {
  const int64_t n = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (n >= a.N) return;
  const int i = threadIdx.x % 64;   // a pair, or two channels behind the pairs
  float c = 1.0f, s = 0.0f;
  if (i < a.half) {
    // whole turns leave in float64: a position has up to 31 bits and the angle's remainder needs 24 more
    const double turns = (double)(a.positions ? a.positions[n] : (int)n) * a.freq[i] * 0.15915494309189533577;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    s *= a.sign * a.factor;
    c *= a.factor;
  }
  const int u = i < a.half ? (a.neighbours ? 2 * i : i) : 2 * i, v = i < a.half && !a.neighbours ? i + a.half : u + 1;
  for (int h = threadIdx.x / 64; h < a.heads[0] + a.heads[1]; h += 4) {
    const int t = h >= a.heads[0], hh = h - (t ? a.heads[0] : 0);
    const RotaryRows &r = a.r[t];
    const T *x = (const T *)r.x + n * r.x_token + hh * r.x_head;
    T *y = (T *)r.y + n * r.y_token + hh * r.y_head;
    const T xu = x[u], xv = x[v];
    y[u] = i < a.half ? (T)(to_f(xu) * c - to_f(xv) * s) : xu;
    y[v] = i < a.half ? (T)(to_f(xu) * s + to_f(xv) * c) : xv;
  }
}

hipError_t launch_rotary(int dtype, const Rotary &a, hipStream_t s) {
  const dim3 grid((unsigned)min(a.N, 65536), (unsigned)((a.N + 65535) / 65536));
  if (dtype == ARCKV_BF16)
    hipLaunchKernelGGL(k_rotary<bf16>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(k_rotary<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace arckv
