// Decode attention over the 8-bit cache, optionally over listed blocks of it
// only, followed by an uncompressed bf16 tail.  For pair p and each of its G
// query rows q:
//   o = softmax([s q K^T + beta, s q K_f^T]) [V; V_f],  K = scale * code
// over the rows below the pair's lengths whose bias is not -inf; a pair with
// none of them gets zeros.
//
// HBM-bound: 256 bytes of codes per token.  Split-key in two kernels:
//   k_attendq_partial  a workgroup takes a share of the pair's blocks and of its
//                      tail, a wave one block of 64 tokens (so one key scale and
//                      one value scale) or 32 rows of the tail at a time, with a
//                      running softmax.  Codes become bf16 (keys) and fp16
//                      (values) in registers, where they are exact, and feed MFMA
//                      16x16x32: keys as rows and queries as columns for the
//                      logits, then the lane that holds a query's probabilities
//                      feeds them to (P V)^T, whose columns are the queries again,
//                      so the sums sit with their maximum.  The next block's keys
//                      are loaded once this one's are used up, and so are its
//                      values: 168 registers, three waves on a SIMD, 8 to 16 KB
//                      in flight each.  The waves' (max, sum, o) are merged in LDS.
//   k_attendq_combine  merges the partials of a pair; a call of one chunk per
//                      pair needs none.
// 512 pairs of 3277 int8 rows with bias and 256 tail rows take 74 us (6.6 TB/s; 77 us
// with half lines of keys per load, 93 us with one block per wave and the tail in
// workgroups of its own, 145 us with loads under branches), of 8192 to 16384 e4m3 rows
// 261 us (6.2 TB/s; 272, 314, 495).  Reading alone reaches 6.9 TB/s.
#include <type_traits>

#include "qcode.hpp"

namespace arckv {

namespace {
constexpr int kAqW = 4;               // waves per workgroup
constexpr int kAqWide = 16;           // of one that takes a whole pair of a small call, one unit per wave
constexpr int kAqSlots = 768;         // workgroups that run at a time: three on each of 256 CUs
constexpr int kAqStart = 6;           // cost of a workgroup beside its blocks, in blocks per wave
constexpr int kAqTail = 32;           // tail rows per wave
// Bytes of codes above which keys and values are read as streams that the caches do not keep: a quarter of the last-level
// cache, which a decode step's other layers pass through before a layer's turn comes again.  Three caches in turn, kept and
// streamed (values alone): 64 pairs of 4096 rows (67 MB) 16.1 and 16.5 us, of 6000 23.5 and 22.7, of 8192 31.8 and 27.8.
constexpr int64_t kAttendKept = (int64_t)64 << 20;

__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ inline f32x4 mfma16h(bf16x8 a, bf16x8 b, f32x4 c) {   // fp16 values in the fragments
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
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

// Codes as MFMA operands, two to a word: four of a key as bf16 (the queries' type); those of four dims of two tokens
// side by side, dim by dim, as fp16.  Every code is exact in both.
template <int FMT> struct Operand;

template <> struct Operand<ARCKV_E4M3> {
  __device__ static inline void keys(uint32_t w, uint32_t &first, uint32_t &second) {
    first = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
    second = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  }
  __device__ static inline void values(uint32_t x, uint32_t y, uint32_t (&dim)[4]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t w = __builtin_amdgcn_perm(y, x, h ? 0x07030602u : 0x05010400u);   // x, y, x, y
      dim[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false));
      dim[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true));
    }
  }
};

template <> struct Operand<ARCKV_INT8> {
  __device__ static inline void keys(uint32_t w, uint32_t &first, uint32_t &second) {
    float y[4];
    QCode<ARCKV_INT8>::unpack4(w, y);
    first = upper_halves(__float_as_uint(y[0]), __float_as_uint(y[1]));
    second = upper_halves(__float_as_uint(y[2]), __float_as_uint(y[3]));
  }
  // a byte u below fp16's exponent of 1024 is 1024 + u; with the code's sign bit flipped u is code + 128
  __device__ static inline void values(uint32_t x, uint32_t y, uint32_t (&dim)[4]) {
    const f16x2 off = {(f16)-1152.0f, (f16)-1152.0f};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t w = __builtin_amdgcn_perm(y, x, 0x0c040c00u + 0x10001u * e) ^ 0x64806480u;   // 0x0c: a zero byte
      dim[e] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, w) + off);
    }
  }
};

// Probabilities, times 2^kPShift, as two fp16 terms: 22 bits of the large ones, and 2^-39 of the block's largest where
// they are small.
constexpr int kPShift = 15;
__device__ inline void split_p_f16(float p0, float p1, uint32_t &h, uint32_t &l) {
  const f32x2 x = {p0, p1};
  const f16x2 hi = __builtin_convertvector(x, f16x2);
  const f32x2 rest = {x[0] - (float)hi[0], x[1] - (float)hi[1]};
  h = __builtin_bit_cast(uint32_t, hi);
  l = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, f16x2));
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
  int iters, nch;             // units (blocks, 32 tail rows) per wave of a chunk; chunks per pair
};

// What a wave has in flight of a block of 64 tokens.  Keys feed MFMA as rows, where a contraction step pairs bytes
// 64 kk + 16 g + 8 h .. + 7 of keys and queries; values are the lane's of keys 16 (i / 4) + 4 g + i % 4 (those of its
// logits) and dims 8 r .. 8 r + 7.  MFMA gives a key row to four lanes, so its 128 bytes would take two loads of half a
// line each; as a stream a line is then fetched twice.  LINES: a load takes 8 whole rows, 16 bytes a lane in order, and
// the rows find their lanes through LDS that only this wave uses: 512 pairs of 8192 to 16384 rows 261 us instead of 272.
struct Keys {
  u32x4 c[4][2];   // LINES: c[i / 2][i % 2] is row 8 i + lane / 8, piece lane % 8
  float scale, bias;
};
struct Values {
  u32x2 c[16];
  float scale;
};

// Loads of block b of pair p, `live` of its tokens in use (both the wave's); none where live is 0, and zeros behind them.
template <bool BETA, bool LINES, int NT>
__device__ inline void load_keys(const AttendQ &a, int64_t pair_block, int64_t row0, int live, Keys &k) {
  const int lane = threadIdx.x & 63, at = LINES ? 16 * lane : (lane & 15) * kHeadDim + 16 * (lane >> 4);
  const __amdgpu_buffer_rsrc_t kb = buffer(a.c.K + row0 * kHeadDim, live * kHeadDim);
#pragma unroll
  for (int kt = 0; kt < 4; ++kt)
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
      k.c[kt][kk] = __builtin_amdgcn_raw_buffer_load_b128(kb, at + 16 * kHeadDim * (kt % 2) + (LINES ? 8 * kHeadDim : 64) * kk,
                                                          4096 * (kt / 2), LINES ? NT : 0);
  k.scale = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(buffer(a.c.Ks + pair_block, live ? 4 : 0), 0, 0, 0));
  if constexpr (BETA)
    k.bias = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(buffer(a.beta + row0, live * 4), 4 * lane, 0, 0));
}

// Rows in order to LDS; the 16-byte pieces of row n lie at piece ^ (n / 2 % 8), so that the lanes of a key column, 16 rows
// apart in nothing but the row, meet different banks.
__device__ inline void put_keys(const Keys &k, u32x4 *s_k) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = 8 * i + (lane >> 3);
    s_k[row * 8 + ((lane & 7) ^ (row >> 1 & 7))] = k.c[i / 2][i % 2];
  }
  wave_exchange();
}
__device__ inline u32x4 get_keys(const u32x4 *s_k, int kt, int kk) {
  const int lane = threadIdx.x & 63, row = 16 * kt + (lane & 15);
  return s_k[row * 8 + ((4 * kk + (lane >> 4)) ^ (row >> 1 & 7))];
}

template <int NT>
__device__ inline void load_values(const AttendQ &a, int64_t pair_block, int64_t row0, int live, Values &v) {
  const int lane = threadIdx.x & 63, at = 4 * (lane >> 4) * kHeadDim + 8 * (lane & 15);
  const __amdgpu_buffer_rsrc_t vb = buffer(a.c.V + row0 * kHeadDim, live * kHeadDim);
#pragma unroll
  for (int i = 0; i < 16; ++i)
    v.c[i] = __builtin_amdgcn_raw_buffer_load_b64(vb, at + 16 * kHeadDim * (i / 4 % 2) + kHeadDim * (i % 4), 4096 * (i / 8), NT);
  v.scale = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(buffer(a.c.Vs + pair_block, live ? 4 : 0), 0, 0, 0));
}

// A wave's query operands go to LDS, [step][lane]: a block's 16 products would hold 16 registers for them.
__device__ inline void put_queries(const bf16x8 (&qf)[4], bf16x8 *s_q) {
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) s_q[ks * 64 + (threadIdx.x & 63)] = qf[ks];
  wave_exchange();
}

// The blocks first, first + W, ... below end of the list (or of the cache), a wave's share of a chunk.
template <int W, int FMT, int GP, bool BETA, bool STREAM>
__device__ inline void attend_blocks(const AttendQ &a, int p, int first, int end, int len, float *s_bias,
                                     const bf16x8 (&qf0)[4], bf16x8 *s_q, u32x4 *s_k, float &m, float &l,
                                     f32x4 (&o)[8]) {
  constexpr int NTV = STREAM ? kStreamed : 0;
  constexpr bool LINES = W != kAqWide;   // 16 waves have no room in LDS
  const int lane = threadIdx.x & 63, g = lane >> 4;
  // block and live tokens of list entry idx; none past the end
  auto block_at = [&](int idx, int &b, int &live) {
    b = idx < end ? idx : -1;
    if (a.blocks && idx < end) b = __builtin_amdgcn_readfirstlane(a.blocks[(int64_t)p * a.nsel + idx]);
    const bool in = b >= 0 && b < a.c.nblk;
    live = __builtin_amdgcn_readfirstlane(in ? max(0, min(len - b * kQBlock, kQBlock)) : 0);
    b = in ? b : 0;
  };
  int b, live;
  block_at(first, b, live);
  Keys k;
  Values v;
  const int64_t pb = (int64_t)p * a.c.nblk, pr = (int64_t)p * a.c.rows;
  load_keys<BETA, LINES, NTV>(a, pb + b, pr + (int64_t)b * kQBlock, live, k);
  load_values<NTV>(a, pb + b, pr + (int64_t)b * kQBlock, live, v);
  __builtin_amdgcn_sched_barrier(0);
  put_queries(qf0, s_q);
  for (int idx = first; idx < end; idx += W) {
    int nb, nlive;
    block_at(idx + W, nb, nlive);
    // ---- logits: keys 16 kt + 4 g + j (j < 4) of query r % GP, all four kt in every lane; the columns beyond the GP
    // queries hold them again, and each of the 16 / GP copies goes on with its own share of the keys
    constexpr int PARTS = 16 / GP, N = 16 / PARTS;
    const int part = (lane & 15) / GP;
    bf16x8 qf[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) qf[ks] = s_q[ks * 64 + lane];
    if constexpr (LINES) put_keys(k, s_k);
    f32x4 dots[4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
      f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        const u32x4 c = LINES ? get_keys(s_k, kt, ks / 2) : k.c[kt][ks / 2];
        Frag f;
        Operand<FMT>::keys(c[2 * (ks % 2)], f.w[0], f.w[1]);
        Operand<FMT>::keys(c[2 * (ks % 2) + 1], f.w[2], f.w[3]);
        acc = mfma16(f.v, qf[ks], acc);
      }
      dots[kt] = acc;
    }
    const float kscale = k.scale * a.scale;
    float sv[N];
    uint64_t hidden = 0;   // tokens in use with a bias of -inf, a bit each
    if constexpr (BETA) {
      // one bias per lane, spread to the lanes of a key's logits through LDS that only this wave uses
      const float bias = lane < live ? k.bias : -INFINITY;
      hidden = __ballot(lane < live && bias == -INFINITY);
      s_bias[lane] = bias;
      wave_exchange();
    }
#pragma unroll
    for (int t = 0; t < N / 4; ++t) {
      const int key0 = 16 * (part * (N / 4) + t) + 4 * g;
      f32x4 d = dots[t];
#pragma unroll
      for (int s = 1; s < PARTS; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] = part == s ? dots[s * (N / 4) + t][j] : d[j];
      if constexpr (BETA) {
        const float4 x = *reinterpret_cast<const float4 *>(s_bias + key0);
        const float bv[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) sv[4 * t + j] = bv[j] != -INFINITY ? fmaf(kscale, d[j], bv[j]) : -INFINITY;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) sv[4 * t + j] = key0 + j < live ? kscale * d[j] : -INFINITY;
      }
    }
    if constexpr (BETA || LINES) wave_exchange();   // the next block's keys and biases take the place of what was read here
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (W != kAqWide) load_keys<BETA, LINES, NTV>(a, pb + nb, pr + (int64_t)nb * kQBlock, nlive, k);
    __builtin_amdgcn_sched_barrier(0);
    bool any;
    float now;
    const float keep = softmax_step<N, PARTS, kPShift, true>(sv, m, l, any, now);
    if constexpr (BETA && FMT == ARCKV_E4M3) {
      // the probability of a token left out is zero, but zero times a NaN code is not (int8 has none)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t keeps = ~((uint32_t)(hidden >> 16 * t) >> 4 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t mask = (uint32_t)((int32_t)(keeps << (31 - j)) >> 31);
          v.c[4 * t + j][0] &= mask;
          v.c[4 * t + j][1] &= mask;
        }
      }
    }
    // ---- (P V)^T: the probabilities of column r, query r, are the B operand with the lane's keys as contraction slots, and
    // its values row r of eight A operands, one per dim 8 r + e: the sums of query r end up with its maximum
    Frag ph[2], pl[2];   // of tokens 0..31 and 32..63; lane r collects the shares from the copies of its column
    {
      uint32_t h[N / 2], lo[N / 2];
#pragma unroll
      for (int i = 0; i < N / 2; ++i) split_p_f16(sv[2 * i], sv[2 * i + 1], h[i], lo[i]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (PARTS == 4) {
          ph[0].w[i] = h[i];
          pl[0].w[i] = lo[i];
          ph[0].w[2 + i] = from_lane<4>(h[i]);
          pl[0].w[2 + i] = from_lane<4>(lo[i]);
          ph[1].w[i] = from_lane<8>(h[i]);
          pl[1].w[i] = from_lane<8>(lo[i]);
          ph[1].w[2 + i] = from_lane<12>(h[i]);
          pl[1].w[2 + i] = from_lane<12>(lo[i]);
        } else {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            ph[0].w[2 * u + i] = h[2 * u + i];
            pl[0].w[2 * u + i] = lo[2 * u + i];
            ph[1].w[2 * u + i] = PARTS == 2 ? from_lane<8>(h[2 * u + i]) : h[(4 + 2 * u + i) % (N / 2)];
            pl[1].w[2 * u + i] = PARTS == 2 ? from_lane<8>(lo[2 * u + i]) : lo[(4 + 2 * u + i) % (N / 2)];
          }
        }
      }
    }
    // without the probabilities' 2^kPShift; the scale of a block that is left out whole may be NaN
    const float vscale = any ? v.scale * (1.0f / (1 << kPShift)) * now : 0.0f;
#pragma unroll
    for (int dd = 0; dd < 2; ++dd) {
      f32x4 acc[4] = {};
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        Frag vf[4];
#pragma unroll
        for (int kq = 0; kq < 4; ++kq) {
          const uint32_t x = v.c[8 * half + 2 * kq][dd], y = v.c[8 * half + 2 * kq + 1][dd];
          uint32_t w[4];
          Operand<FMT>::values(x, y, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) vf[e].w[kq] = w[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = mfma16h(vf[e].v, ph[half].v, mfma16h(vf[e].v, pl[half].v, acc[e]));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[4 * dd + e][j] = fmaf(vscale, acc[e][j], o[4 * dd + e][j] * keep);
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (W == kAqWide) return;   // its only block
    load_values<NTV>(a, pb + nb, pr + (int64_t)nb * kQBlock, nlive, v);
    __builtin_amdgcn_sched_barrier(0);
    live = nlive;
  }
}

// 32 rows of the tail, `live` of them in use: what a wave has in flight of them.  The contraction steps are the blocks',
// so a lane reads 32 bytes at a time of a key.
__device__ inline void load_tail_keys(const AttendQ &a, int64_t row0, int live, u32x4 (&k)[2][4]) {
  const int lane = threadIdx.x & 63, at = (lane & 15) * 2 * kHeadDim + 32 * (lane >> 4);
  const __amdgpu_buffer_rsrc_t kb = buffer(a.Kf + row0 * kHeadDim, live * 2 * kHeadDim);
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
      k[kt][ks] = __builtin_amdgcn_raw_buffer_load_b128(kb, at + 128 * (ks / 2) + 16 * (ks % 2), 32 * kHeadDim * kt, 0);
}

template <int NT> __device__ inline void load_tail_values(const AttendQ &a, int64_t row0, int live, u32x4 (&v)[8]) {
  const int lane = threadIdx.x & 63, at = 4 * (lane >> 4) * 2 * kHeadDim + 16 * (lane & 15);
  const __amdgpu_buffer_rsrc_t vb = buffer(a.Vf + row0 * kHeadDim, live * 2 * kHeadDim);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    v[i] = __builtin_amdgcn_raw_buffer_load_b128(vb, at + 2 * kHeadDim * (i % 4), 32 * kHeadDim * (i / 4), NT);
}

// The tail's units of 32 rows first, first + W, ... below end, a wave's share of a chunk.
template <int W, bool STREAM>
__device__ inline void attend_tail(const AttendQ &a, int p, int first, int end, int len, const bf16x8 *s_q, float &m,
                                   float &l, f32x4 (&o)[8]) {
  constexpr int NTV = STREAM ? kStreamed : 0;
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int64_t pr = (int64_t)p * a.F;
  auto live_at = [&](int idx) { return __builtin_amdgcn_readfirstlane(idx < end ? max(0, min(len - idx * kAqTail, kAqTail)) : 0); };
  int live = live_at(first);
  u32x4 k[2][4], v[8];
  load_tail_keys(a, pr + first * kAqTail, live, k);
  load_tail_values<NTV>(a, pr + first * kAqTail, live, v);
  for (int idx = first; idx < end; idx += W) {
    const int nlive = live_at(idx + W);
    const int64_t next = pr + (idx + W) * kAqTail;
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
    if constexpr (W != kAqWide) load_tail_keys(a, next, nlive, k);
    __builtin_amdgcn_sched_barrier(0);
    bool any;
    float now;
    const float keep = softmax_step<8, 1, 0, false>(sv, m, l, any, now);
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
      for (int j = 0; j < 4; ++j) o[e][j] = fmaf(o[e][j], keep, fabsf(lead[j]) < INFINITY ? lead[j] + rest[j] : lead[j]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (W == kAqWide) return;
    load_tail_values<NTV>(a, next, nlive, v);
    __builtin_amdgcn_sched_barrier(0);
    live = nlive;
  }
}

// GP: the query rows that LDS and operands have room for, G <= GP <= 16.
template <int W, int FMT, int GP, bool BETA, bool STREAM>
__global__ void __launch_bounds__(64 * W, W == kAqW ? 3 : 4) k_attendq_partial(AttendQ a) {
  // a wave's query operands, [step][lane], and a block's keys; in their place its sums once they are complete
  union Own {
    struct {
      bf16x8 q[4 * 64];
      u32x4 k[W == kAqWide ? 1 : kQBlock * kHeadDim / 16];
    };
    float o[GP][kHeadDim];
  };
  __shared__ __align__(16) Own sOwn[W];
  __shared__ float sM[W][GP], sL[W][GP];
  __shared__ __align__(16) float sB[BETA ? W : 1][kQBlock];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, r = lane & 15;
  const int ch = blockIdx.x, p = blockIdx.z * gridDim.y + blockIdx.y, G = a.G;
  if (p >= a.c.P) return;
  bf16x8 qf[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
    qf[ks] = *reinterpret_cast<const bf16x8 *>(a.Q + ((int64_t)p * G + min(r % GP, G - 1)) * kHeadDim + 64 * (ks / 2) + 16 * g +
                                               8 * (ks % 2));
  float m = -INFINITY, l = 0.0f;
  f32x4 o[8] = {};
  // units: the blocks (or list entries), then the tail's 32-row pieces; this chunk's, wave by wave
  const int first = ch * a.iters * W + wave, end = ch * a.iters * W + a.iters * W;
  const int len = clip_len(a.length, p, a.c.rows);
  const int bend = min(end, a.blocks ? a.nsel : (len + kQBlock - 1) / kQBlock);
  if (first < bend)
    attend_blocks<W, FMT, GP, BETA, STREAM>(a, p, first, bend, len, sB[BETA ? wave : 0], qf, sOwn[wave].q, sOwn[wave].k, m, l, o);
  else
    put_queries(qf, sOwn[wave].q);
  if (end > a.nsel) {
    const int len_f = clip_len(a.length_f, p, a.F);
    const int skip = first < a.nsel ? (a.nsel - first + W - 1) / W * W : 0;   // this wave's blocks
    const int tfirst = first + skip - a.nsel, tend = min(end - a.nsel, (len_f + kAqTail - 1) / kAqTail);
    if (tfirst < tend) attend_tail<W, STREAM>(a, p, tfirst, tend, len_f, sOwn[wave].q, m, l, o);
  }
  if (g == 0 && r < G) {
    sM[wave][r] = m;
    sL[wave][r] = l;
  }
  wave_exchange();
  if (r < G)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float *to = &sOwn[wave].o[r][8 * (4 * g + j)];
      *reinterpret_cast<float4 *>(to) = make_float4(o[0][j], o[1][j], o[2][j], o[3][j]);
      *reinterpret_cast<float4 *>(to + 4) = make_float4(o[4][j], o[5][j], o[6][j], o[7][j]);
    }
  __syncthreads();
  // one partial (max, sum, o) per query for the chunk; the result itself where there is one chunk
  for (int idx = tid; idx < G * kHeadDim; idx += 64 * W) {
    const int q = idx / kHeadDim, dim = idx % kHeadDim;
    float M = sM[0][q];
#pragma unroll
    for (int w = 1; w < W; ++w) M = fmaxf(M, sM[w][q]);
    const float ref = M == -INFINITY ? 0.0f : M;
    float acc = 0.0f, lsum = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = __expf(sM[w][q] - ref);   // a wave without a key in use: zero, as its sums are
      acc = fmaf(f, sOwn[w].o[q][dim], acc);
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
}

// One workgroup per (query, pair): four groups of threads, thread = dim, take every fourth of the pair's partials, four
// loads at a time, and meet in LDS: 86 chunks of 8 pairs take 4.2 us (9.8 us with one group).
constexpr int kCombineGroups = 4, kCombineAhead = 4;
__global__ void __launch_bounds__(kCombineGroups *kHeadDim) k_attendq_combine(AttendQ a) {
  __shared__ float sM[kCombineGroups], sL[kCombineGroups], sA[kCombineGroups][kHeadDim];
  const int q = blockIdx.x, dim = threadIdx.x % kHeadDim, group = threadIdx.x / kHeadDim, p = blockIdx.z * gridDim.y + blockIdx.y;
  if (p >= a.c.P) return;
  const float *ml = a.part_ml + ((int64_t)p * a.nch * a.G + q) * 2;
  const float *po = a.part_o + ((int64_t)p * a.nch * a.G + q) * kHeadDim + dim;
  float M = -INFINITY, lsum = 0.0f, acc = 0.0f;
  for (int c0 = group; c0 < a.nch; c0 += kCombineGroups * kCombineAhead) {
    float m[kCombineAhead], l[kCombineAhead], o[kCombineAhead], top = M;
#pragma unroll
    for (int i = 0; i < kCombineAhead; ++i) {
      const int c = c0 + kCombineGroups * i;
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
  if (dim == 0) {
    sM[group] = M;
    sL[group] = lsum;
  }
  sA[group][dim] = acc;
  __syncthreads();
  if (group) return;
#pragma unroll
  for (int i = 1; i < kCombineGroups; ++i) M = fmaxf(M, sM[i]);
  const float ref = M == -INFINITY ? 0.0f : M;
  acc = lsum = 0.0f;
#pragma unroll
  for (int i = 0; i < kCombineGroups; ++i) {
    const float f = __expf(sM[i] - ref);
    lsum = fmaf(f, sL[i], lsum);
    acc = fmaf(f, sA[i][dim], acc);
  }
  a.out[((int64_t)p * a.G + q) * kHeadDim + dim] = lsum == 0.0f ? 0.0f : acc / lsum;
}

// Whether a call is small: one wide workgroup per pair takes its units in one step, and no second launch joins what it
// leaves: 8 pairs of 819 + 37 rows take 10.5 us, 6.7 and 3.3 us in two launches, and 11.8 us a call against 15.9.
static bool attendq_small(int P, int nsel, int F) {
  return P <= 256 && nsel + (F + kAqTail - 1) / kAqTail <= kAqWide;
}

// Chunks per pair, and the units (blocks and 32-row pieces of the tail) per wave of one.  Workgroups run kAqSlots at a
// time, so a call takes as many rounds as they fill, of a workgroup's units and its start each; the number of chunks with
// the least sum is taken: 512 pairs of 3277 + 256 rows in one chunk each took 80 us where three took 96; 8192 to 16384
// rows go in three.
int attendq_chunks(int P, int nsel, int F, int *iters) {
  const int units = nsel + (F + kAqTail - 1) / kAqTail;
  if (attendq_small(P, nsel, F)) {
    *iters = 1;
    return 1;
  }
  const int n = (units + kAqW - 1) / kAqW;
  *iters = 1;
  if ((int64_t)P * n > kAqSlots) {
    int64_t least = INT64_MAX;
    for (int c = 1; c <= n && (int64_t)P * (c - 1) < 4 * kAqSlots; ++c) {
      const int it = (n + c - 1) / c;
      const int64_t cost = ((int64_t)P * c + kAqSlots - 1) / kAqSlots * (it + kAqStart);
      if (cost < least) {
        least = cost;
        *iters = it;
      }
    }
  }
  return (n + *iters - 1) / *iters;
}

hipError_t launch_attendq(int fmt, const QCache &c, int G, int F, float scale, const void *Q, const float *beta,
                          const int32_t *length, const int32_t *blocks, int nsel, const void *Kf, const void *Vf,
                          const int32_t *length_f, float *part_o, float *part_ml, float *out, hipStream_t s) {
  AttendQ a{c, G, F, scale, (const bf16 *)Q, beta, length, blocks, blocks ? nsel : c.nblk, (const bf16 *)Kf,
            (const bf16 *)Vf, length_f, part_o, part_ml, out, 0, 0};
  a.nch = attendq_chunks(c.P, a.nsel, F, &a.iters);
  // pairs over y and z: a grid's y extent is limited
  const unsigned py = (unsigned)min(c.P, 32768), pz = (unsigned)((c.P + 32767) / 32768);
  const bool stream = (int64_t)c.P * a.nsel * kQBlock * 2 * kHeadDim > kAttendKept;
  const bool small = attendq_small(c.P, a.nsel, F);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3((unsigned)a.nch, py, pz), dim3(64 * (small ? kAqWide : kAqW)), 0, s, a);
    return hipGetLastError();
  };
  auto by_stream = [&](auto fm, auto gp, auto bt) {
    constexpr int FMT = decltype(fm)::value, GP = decltype(gp)::value;
    constexpr bool BETA = decltype(bt)::value;
    if (small) return go(k_attendq_partial<kAqWide, FMT, GP, BETA, false>);
    return stream ? go(k_attendq_partial<kAqW, FMT, GP, BETA, true>) : go(k_attendq_partial<kAqW, FMT, GP, BETA, false>);
  };
  auto by_beta = [&](auto fm, auto gp) {
    return beta ? by_stream(fm, gp, std::true_type{}) : by_stream(fm, gp, std::false_type{});
  };
  auto by_rows = [&](auto fm) {
    return G <= 4 ? by_beta(fm, std::integral_constant<int, 4>{})
                  : G <= 8 ? by_beta(fm, std::integral_constant<int, 8>{}) : by_beta(fm, std::integral_constant<int, 16>{});
  };
  const hipError_t e = fmt == ARCKV_E4M3 ? by_rows(std::integral_constant<int, ARCKV_E4M3>{})
                                         : by_rows(std::integral_constant<int, ARCKV_INT8>{});
  if (e != hipSuccess || a.nch == 1) return e;
  hipLaunchKernelGGL(k_attendq_combine, dim3((unsigned)G, py, pz), dim3(kCombineGroups * kHeadDim), 0, s, a);
  return hipGetLastError();
}

}  // namespace arckv
