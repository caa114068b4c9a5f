// Rotary positions: pairs of channels turned by position * frequency.
//
// HBM-bound: every row is read and written once.  A row is cut into pieces of 16 bytes, and a thread takes the two that
// belong together (channels c .. and c + half .., or neighbours) of one row or two, all loaded before the angles are
// formed: a workgroup's rows follow each other through tokens and heads, so it needs the angles of few tokens, each formed
// once, by one thread, for all its heads, and handed out through LDS.  Halves that end inside a piece have their rows in LDS
// too, where a channel finds its mate at any distance.
// 32768 tokens of 40 bf16 heads, out of a fused projection, take 113 us (5.9 TB/s), 4093 of 20 float32 heads 13.5 (6.2); a thread
// a pair of channels took 274 and 22.9.  16384 of 40 heads with 34 channels turned take 71 us in halves, 60 as neighbours.
#include <type_traits>

#include "common.hpp"
#include "qcode.hpp"
#include "rotary.hpp"

namespace arckv {

namespace {
constexpr int kRotThreads = 256;
// Bytes above which rows are read as streams that the caches do not keep.  us kept and streamed: 4096 tokens of 40 bf16 heads (42
// MB in) 14.0 and 17.4, 8000 (82 MB) 27.3 and 30.5, 9500 (97 MB) 34.8 and 35.8, 12000 (123 MB) 45.6 and 44.1, 32768 (336 MB) 123
// and 113.
constexpr int64_t kRotKept = (int64_t)96 << 20;
// Bytes above which, if not streamed, a thread takes two rows instead of one, where tokens have more than one head (one head's rows
// need as many angles as there are channels).  us with one, two and four: 64 tokens of 40 bf16 heads 2.8, 3.2, 3.9; 1000 (10 MB)
// 4.9, 5.0, 5.7; 2000 (20 MB) 8.3, 7.8, 7.9; 4096 (42 MB) 15.7, 13.9, 13.2; 4093 of 20 float32 heads (42 MB) 15.1, 13.7, 13.4;
// 65536 of 5 (84 MB) 30.9, 27.2, 27.5; 131072 of one (34 MB) 18.4, 20.6, 25.8; 32768 of 40, streamed, 113.0 with one, 123.1 with four.
constexpr int64_t kRotFew = (int64_t)16 << 20;
template <typename T> constexpr int kRotPer = 16 / (int)sizeof(T);                     // channels of a piece
template <typename T> constexpr int kRotSlots = kRotThreads * 2 * kRotPer<T> / kHeadDim;  // rows that threads take at a time
template <typename T, int ROWS> constexpr int kRotTile = kRotSlots<T> * ROWS;             // and a workgroup in all

// Turns per position of a pair.
__device__ inline double turns_of(const Rotary &a, int i) { return a.freq[i] * 0.15915494309189533577; }

__device__ inline void angle(const Rotary &a, int64_t n, double per_position, float &c, float &s) {
  // whole turns leave in float64: a position has up to 31 bits and the angle's remainder needs 24 more
  const double turns = (double)(a.positions ? a.positions[n] : (int)n) * per_position;
  sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
  s *= a.sign * a.factor;
  c *= a.factor;
}

template <typename T> struct Piece;
template <> struct Piece<float> {
  __device__ static inline void unpack(u32x4 w, float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(w[e]);
  }
  __device__ static inline u32x4 pack(const float (&x)[4]) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
};
template <> struct Piece<bf16> {
  __device__ static inline void unpack(u32x4 w, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
  __device__ static inline u32x4 pack(const float (&x)[8]) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)x[2 * e], (bf16)x[2 * e + 1]});
    return w;
  }
};

}  // namespace

enum RotaryMode { kHalves, kNeighbours, kUnevenHalves };

template <typename T, int MODE, int ROWS, bool STREAM> __global__ void __launch_bounds__(kRotThreads) k_rotary(Rotary a) {
  constexpr int PER = kRotPer<T>, THREADS = kHeadDim / (2 * PER), SLOTS = kRotSlots<T>, TILE = kRotTile<T, ROWS>;
  extern __shared__ __align__(16) float s_angle[];   // [token][cos, sin][64]
  __shared__ __align__(16) T s_row[MODE == kUnevenHalves ? TILE : 1][kHeadDim];
  const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  const int H = a.heads[0] + a.heads[1];
  const int64_t row0 = block * TILE, rows = (int64_t)a.N * H;
  if (row0 >= rows) return;
  const int64_t n0 = H == 1 ? row0 : row0 / H;
  const int first = (int)(row0 - n0 * H), count = (int)min((int64_t)TILE, rows - row0);   // row of token n0; rows of this workgroup
  const int c = threadIdx.x % THREADS, slot = threadIdx.x / THREADS;
  // the thread's pieces: two that are pairs (halves), any two (of neighbours, of a row in LDS), or two that are copied;
  // neighbouring threads have neighbouring pieces, so that streamed stores fill lines
  const int turned = a.half / PER;
  const bool pairs = MODE == kHalves && c < turned;
  const int pu = MODE != kHalves || pairs ? c : c + turned, pv = pairs ? c + turned : c + THREADS;
  u32x4 u[ROWS], v[ROWS];
  T *y[ROWS];
  int token[ROWS];
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    const int i = min(slot + SLOTS * k, count - 1) + first;   // rows past the end load the last one and store nothing
    // i < TILE + H: a token further at most where H is a tile or more, else exact for i < 2 TILE
    token[k] = H >= TILE ? (i >= H) : (int)(((uint32_t)i * a.by_heads) >> 16);
    const int h = i - token[k] * H, t = h >= a.heads[0];
    const RotaryRows &r = a.r[t];
    const int64_t n = n0 + token[k], hh = h - (t ? a.heads[0] : 0);
    const T *x = (const T *)r.x + n * r.x_token + hh * r.x_head;
    y[k] = (T *)r.y + n * r.y_token + hh * r.y_head;
    if constexpr (STREAM) {
      u[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(x + pu * PER));
      v[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(x + pv * PER));
    } else {
      u[k] = *reinterpret_cast<const u32x4 *>(x + pu * PER);
      v[k] = *reinterpret_cast<const u32x4 *>(x + pv * PER);
    }
    if constexpr (MODE == kUnevenHalves) {
      *reinterpret_cast<u32x4 *>(&s_row[slot + SLOTS * k][pu * PER]) = u[k];
      *reinterpret_cast<u32x4 *>(&s_row[slot + SLOTS * k][pv * PER]) = v[k];
    }
  }
  const int last = (count - 1 + first) / H;
  const int f = threadIdx.x % 64;
  if (f < a.half) {
    const double per_position = turns_of(a, f);
    for (int t = threadIdx.x / 64; t <= last; t += kRotThreads / 64)
      angle(a, n0 + t, per_position, s_angle[t * 128 + f], s_angle[t * 128 + 64 + f]);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    const float *cs = s_angle + token[k] * 128;
    if (pairs) {
      float xu[PER], xv[PER], yu[PER], yv[PER];
      Piece<T>::unpack(u[k], xu);
      Piece<T>::unpack(v[k], xv);
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const float co = cs[PER * c + e], si = cs[64 + PER * c + e];
        yu[e] = xu[e] * co - xv[e] * si;
        yv[e] = xu[e] * si + xv[e] * co;
      }
      u[k] = Piece<T>::pack(yu);
      v[k] = Piece<T>::pack(yv);
    }
    if constexpr (MODE == kNeighbours) {
      auto turn = [&](u32x4 &w, int piece) {   // words whose pairs are turned; the others stay
        float x[PER], z[PER];
        Piece<T>::unpack(w, x);
#pragma unroll
        for (int e = 0; e < PER / 2; ++e) {
          const float co = cs[PER / 2 * piece + e], si = cs[64 + PER / 2 * piece + e];
          z[2 * e] = x[2 * e] * co - x[2 * e + 1] * si;
          z[2 * e + 1] = x[2 * e] * si + x[2 * e + 1] * co;
        }
        const u32x4 y = Piece<T>::pack(z);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (PER * piece + PER / 4 * e) / 2 < a.half ? y[e] : w[e];
      };
      turn(u[k], pu);
      turn(v[k], pv);
    }
    if constexpr (MODE == kUnevenHalves) {
      const T *row = s_row[slot + SLOTS * k];
      auto turn = [&](u32x4 &w, int piece) {
        float x[PER], z[PER];
        Piece<T>::unpack(w, x);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
          const int ch = PER * piece + e;
          const bool lower = ch < a.half, in = ch < 2 * a.half;
          const int i = lower ? ch : in ? ch - a.half : 0;   // its pair
          const float mate = to_f(row[lower ? ch + a.half : i]), si = cs[64 + i];
          z[e] = x[e] * cs[i] + mate * (lower ? -si : si);
        }
        const u32x4 y = Piece<T>::pack(z);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = PER * piece + PER / 4 * e < 2 * a.half ? y[e] : w[e];
      };
      turn(u[k], pu);
      turn(v[k], pv);
    }
    if (slot + SLOTS * k < count) {
      __builtin_nontemporal_store(u[k], reinterpret_cast<u32x4 *>(y[k] + pu * PER));
      __builtin_nontemporal_store(v[k], reinterpret_cast<u32x4 *>(y[k] + pv * PER));
    }
  }
}

template <typename T> static hipError_t launch_rotary_of(Rotary a, hipStream_t s) {
  const int H = a.heads[0] + a.heads[1];
  a.by_heads = (65536 + H - 1) / H;   // used where H is below a workgroup's rows: exact for i < TILE + H
  const int64_t bytes = (int64_t)a.N * H * kHeadDim * (int)sizeof(T);
  auto go = [&](auto kern, int64_t tile) {
    const int64_t blocks = ((int64_t)a.N * H + tile - 1) / tile;
    const dim3 grid((unsigned)min(blocks, (int64_t)65536), (unsigned)((blocks + 65535) / 65536));
    const int64_t tokens = min((int64_t)a.N, H == 1 ? tile : (tile + H - 2) / H + 1);
    hipLaunchKernelGGL(kern, grid, dim3(kRotThreads), tokens * 128 * sizeof(float), s, a);
    return hipGetLastError();
  };
  auto by_rows = [&](auto mode) {
    constexpr int MODE = decltype(mode)::value;
    if (bytes > kRotKept) return go(k_rotary<T, MODE, 1, true>, kRotTile<T, 1>);
    if constexpr (MODE != kUnevenHalves)
      if (bytes > kRotFew && H > 1) return go(k_rotary<T, MODE, 2, false>, kRotTile<T, 2>);
    return go(k_rotary<T, MODE, 1, false>, kRotTile<T, 1>);
  };
  if (a.neighbours) return by_rows(std::integral_constant<int, kNeighbours>{});
  return a.half % kRotPer<T> == 0 ? by_rows(std::integral_constant<int, kHalves>{}) : by_rows(std::integral_constant<int, kUnevenHalves>{});
}

hipError_t launch_rotary(int dtype, const Rotary &a, hipStream_t s) {
  return dtype == ARCKV_BF16 ? launch_rotary_of<bf16>(a, s) : launch_rotary_of<float>(a, s);
}

}  // namespace arckv
