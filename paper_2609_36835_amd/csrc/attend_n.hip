// Decode attention over the 4-bit cache, followed by an uncompressed bf16 tail.
// For pair p and each of its G query rows q:
//   o = softmax([s q K^T + beta, s q K_f^T]) [V; V_f],  K = scale * code
// over the rows below the pair's lengths whose bias is not -inf; a pair with
// none of them gets zeros.
//
// HBM-bound: 136 bytes per token.  Split-key in two kernels:
//   k_attendn_partial  a workgroup takes a share of the pair's units (blocks of 64 rows, 32 rows of the tail) as its lengths
//                      say, a wave a unit at a time, with a running softmax.  The next block's keys are loaded once this
//                      one's are used up, and so are its values: 144 to 168 registers and three waves on a SIMD in workgroups
//                      of four; 144 to 172 in those of eight, which have a CU to themselves, two on a SIMD.
//   k_attend_combine   merges the partials of a pair; a call of one chunk per pair needs none.
// 512 pairs of 3277 rows with bias and 256 tail rows take 49 us (5.9 TB/s), of 8192 to 16384 rows 140 us (6.2), of 32768 rows
// 330 (6.9); with the loads alone, at the same places, the first two take 48.4 and 137.3.  256 of 4096-8192 rows for 16 queries take
// 49 us (4.5 TB/s), one workgroup a CU; vector units are busy 37% of that, matrix units 25%.  8 pairs of 819 + 37 rows take 8 us: a
// start of 3.5, a little over 1 for each of a wave's units, and the waves' join.  A wave loads its first rows of the tail once its
// blocks are done, so there the way to memory counts twice.
//
// Logits.  Keys go to MFMA 16x16x128 as they are held, codes and scales, so that nothing is unpacked.  Its other operand
// is 8-bit, and it aligns the products of neighbouring channels to the largest of them, 13 bits below which it cuts.  So a
// query enters as four planes, q = sum_t p_t 2^(E - 5 t), with 2^E above the magnitudes of its 32 channels and each p_t the
// nearest e4m3 number to what the planes before it left, in magnitude at most 2, in units of 2^-9: products with codes (units
// of 0.5, at most 6) are whole numbers of 2^-10 and stay within the 13 bits, so every sum is exact up to its float32 rounding,
// and what the four planes leave is below 2^(E - 25).  2^(E - 5 t) is the operand's scale.  The planes are columns beside the
// queries (up to 4 queries fill 16 columns), or products of their own (more queries).
//
// Values become bf16, scale included, in registers (exact); probabilities enter (P V)^T as three bf16 terms that sum to
// them exactly, as columns beside the queries again where there is room.  The columns of both products are the same queries,
// so a query's sums sit with its running maximum.  P V is held times 2^-S, 2^S > 2 (rows + F): probabilities are at most 1, so
// sums over the largest values stay below float32's end, and a mean that is finite comes out so.  A power of two costs no
// bit where nothing falls below 2^-126; the scales of a block's values take it, a tail's probabilities, and once the sum of
// probabilities that divides.
#include <type_traits>

#include "attend_parts.hpp"
#include "ncode.hpp"

namespace arckv {

namespace {
constexpr int kAnBlock = 64;          // rows of a unit
constexpr int kAnW = 4;               // waves per workgroup
constexpr int kAnMore = 8;            // of one that has a whole pair, and a CU, to itself
constexpr int kAnCus = 256;
constexpr int kAnSlots = 3 * kAnCus;  // workgroups that run at a time
constexpr int kAnPlanes = 4;
// How far the reference of the exponentials is set above the largest logit when one passes it: the largest probability stays
// between 2^-8 or so and 1, and sums are rescaled a few times in a call instead of at every block.
constexpr float kAnLead = 5.5451774f;
// Bytes above which codes are read as streams that the caches do not keep: 64 pairs of 8192 rows (71 MB) take 18.2 us kept and
// 19.2 streamed, of 12000 24.8 and 24.5, of 16384 31.7 and 29.2, three caches in turn.
constexpr int64_t kAnKept = (int64_t)96 << 20;

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
}  // namespace

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
  int nch;                    // chunks per pair
  float down;                 // 2^-S
};

namespace {

// A pair's query planes, the scales of plane 0 as bytes, and the rows themselves as the tail's operands.
template <int GP> struct Queries {
  uint32_t plane[kAnPlanes][GP][kHeadDim / 4 + 4];   // padded for the banks, as what follows
  uint32_t scale[GP];
  bf16x8 tail[4 * 64];
};

// A thread's share of a pair's queries, two channels at a time; queries beyond G are copies of the last.
template <int W, int GP> struct QueryWords {
  static constexpr int N = (GP + W - 1) / W;
  uint32_t w[N];
  __device__ inline void load(const AttendN &a, int p) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      w[k] = reinterpret_cast<const uint32_t *>(a.Q + ((int64_t)p * a.G + min((int)threadIdx.x / 64 + W * k, a.G - 1)) *
                                                          kHeadDim)[threadIdx.x % 64];
  }
};

// The largest of a row's 16 lanes, in all of them.
__device__ inline uint32_t row_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true));    // neighbours in twos
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, true));   // turned by 4, by 8
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true));
}

// 32 channels stand in 16 lanes of a row.
template <int W, int GP>
__device__ inline void make_queries(const AttendN &a, int p, const QueryWords<W, GP> &words, Queries<GP> &s) {
#pragma unroll
  for (int k = 0; k < QueryWords<W, GP>::N; ++k) {
    const int q = threadIdx.x / 64 + W * k, piece = threadIdx.x % 64;
    if (q >= GP) break;
    const uint32_t w = words.w[k];
    const float x[2] = {__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
    const uint32_t amax = row_max(max(__float_as_uint(x[0]) & 0x7fffffffu, __float_as_uint(x[1]) & 0x7fffffffu));
    const bool finite = amax < 0x7f800000u;
    // magnitudes below 2^(E + 1) at the type's end, below 2^E elsewhere; planes reach the least subnormal at the other
    const int E = finite ? min(max((int)(amax >> 23) - 126, -111), 127) : 0;
    float r[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) r[e] = finite ? ldexpf(x[e], -E) : 0.0f;
#pragma unroll
    for (int t = 0; t < kAnPlanes; ++t) {
      const int c = __builtin_amdgcn_cvt_pk_fp8_f32(r[0], r[1], 0, false);
      reinterpret_cast<uint16_t *>(s.plane[t][q])[piece] = (uint16_t)c;
      const f32x2 got = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_pk_f32_fp8(c, false));
#pragma unroll
      for (int e = 0; e < 2; ++e) r[e] = (r[e] - got[e]) * 32.0f;
    }
    if (piece % 16 == 0) reinterpret_cast<uint8_t *>(&s.scale[q])[piece / 16] = finite ? (uint8_t)(E + 127) : 255;
  }
  if (a.F > 0)
    for (int i = threadIdx.x; i < 4 * 64; i += 64 * W) {
      const int ks = i / 64, lane = i % 64, g = lane >> 4, r = lane & 15;
      u32x4 w = *reinterpret_cast<const u32x4 *>(a.Q + ((int64_t)p * a.G + min(r % GP, a.G - 1)) * kHeadDim + 64 * (ks / 2) +
                                                 16 * g + 8 * (ks % 2));
      // An infinite channel enters as NaN, as it does over the blocks: its logits could all be -inf, which marks rows left out.
      // Adding 0x80 carries into a half's top bit from the largest exponent alone.
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] |= (((w[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 9;
      s.tail[i] = __builtin_bit_cast(bf16x8, w);
    }
}

// A wave's own part of LDS.  Rows stand in the order of the lanes that use them: row 16 kt + 4 j + g of a block, whose
// logits are element j of the lanes of row g, at 16 kt + 4 g + j.
template <int GP> struct WaveLds {
  uint32_t ks[kAnBlock];                   // four scale bytes
  float vs[kHeadDim / kNGroup][kAnBlock + 16];   // scales of a group as numbers
  float bias[kAnBlock];
  uint32_t p[4][GP < 16 ? 32 * GP + 4 : 4];      // [term][row g of lanes, query, tokens in pairs]; the fourth term is zero
  __device__ inline uint32_t *terms_of(int term, int g, int q) { return &p[term][8 * (GP * g + q)]; }
};

// What a wave has in flight of a block.  Keys: row r' = 4 (r % 4) + r / 4 of each 16, so that element j of the logits of
// lane row g is row 4 j + g and a load of values takes four rows in order: whole lines, which a streamed load that takes half
// of one fetches twice.
struct BlockData {
  u32x4 k[4];        // lane (g, r): bytes 16 g .. 16 g + 15 of row 16 kt + r'
  uint32_t v[16];    // bytes 4 r .. 4 r + 3 of row 16 (i / 4) + 4 (i % 4) + g
  uint32_t ks, vs;   // of row `lane`
  float bias;
};

template <bool BETA, int NT> __device__ inline void load_keys(const AttendN &a, int64_t row0, int live, BlockData &d) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const __amdgpu_buffer_rsrc_t kb = buffer(a.c.K + row0 * kNRow, live * kNRow);
#pragma unroll
  for (int kt = 0; kt < 4; ++kt)
    d.k[kt] = __builtin_amdgcn_raw_buffer_load_b128(kb, (4 * (r & 3) + (r >> 2)) * kNRow + 16 * g, 16 * kNRow * kt, NT);
  d.ks = __builtin_amdgcn_raw_buffer_load_b32(buffer(a.c.Ks + row0, live * 4), 4 * lane, 0, NT);
  d.vs = __builtin_amdgcn_raw_buffer_load_b32(buffer(a.c.Vs + row0, live * 4), 4 * lane, 0, NT);
  if constexpr (BETA)
    d.bias = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(buffer(a.beta + row0, live * 4), 4 * lane, 0, 0));
}

template <int NT> __device__ inline void load_values(const AttendN &a, int64_t row0, int live, BlockData &d) {
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
  const __amdgpu_buffer_rsrc_t vb = buffer(a.c.V + row0 * kNRow, live * kNRow);
#pragma unroll
  for (int i = 0; i < 16; ++i)
    d.v[i] = __builtin_amdgcn_raw_buffer_load_b32(vb, g * kNRow + 4 * r, 4 * kNRow * i, NT);
}

// A float's bf16 terms: its upper half and the upper halves of what is left, one below the other.
__device__ inline void terms(float x, uint32_t (&t)[3]) {
  t[0] = __float_as_uint(x) & 0xffff0000u;
  const float x1 = x - __uint_as_float(t[0]);
  t[1] = __float_as_uint(x1) & 0xffff0000u;
  t[2] = __float_as_uint(x1 - __uint_as_float(t[1]));
}

// Two dims (byte B of x and y) of two tokens as bf16, scales included, dim by dim.
template <int B> __device__ inline void value_pairs(uint32_t x, uint32_t y, float sx, float sy, uint32_t &even, uint32_t &odd) {
  const uint32_t xx = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, sx, B)),
                 yy = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(y, sy, B));
  even = lower_halves(xx, yy);
  odd = upper_halves(xx, yy);
}

// The blocks first, first + W, ... below end, a wave's share of a chunk, the first of them on its way in d.
template <int W, int GP, bool BETA, bool STREAM>
__device__ inline void attend_blocks(const AttendN &a, int p, int first, int end, int len, const Queries<GP> &sq,
                                     WaveLds<GP> &s, BlockData &d, float &m, float &l, f32x4 (&o)[8]) {
  constexpr int NT = STREAM ? kStreamed : 0;
  constexpr int C = 16 / GP;                      // columns of a query
  constexpr int NQ = kAnPlanes / C;               // products for its planes
  constexpr int NP = (3 + C - 1) / C;             // and for its probabilities' terms
  constexpr int N = 16 / C;                       // logits of a lane's share
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15, q = r % GP, part = r / GP;
  const int place = (lane & 48) + 4 * (lane & 3) + ((lane & 15) >> 2);   // of row `lane` in LDS
  const int64_t pr = (int64_t)p * a.c.rows;
  auto live_at = [&](int idx) { return __builtin_amdgcn_readfirstlane(idx < end ? min(len - idx * kAnBlock, kAnBlock) : 0); };
  int live = live_at(first);
  // the planes of this lane's column: bytes 16 g .. and 64 + 16 g ..; one scale for channels 32 g ..
  i32x8 qf[NQ];
  int qscale[NQ];
  auto load_planes = [&] {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const u32x4 *plane = reinterpret_cast<const u32x4 *>(&sq.plane[i * C + part][q][4 * g]);
      const u32x4 lo = plane[0], hi = plane[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        qf[i][e] = (int)lo[e];
        qf[i][4 + e] = (int)hi[e];
      }
    }
  };
  if constexpr (NQ == 1) load_planes();   // more of them stay in LDS
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int byte = (int)(sq.scale[q] >> 8 * g & 255u);
    qscale[i] = byte == 255 ? 255 : byte - 5 * (i * C + part);
  }
  if constexpr (C > 1) {   // no fourth term
    u32x4 *none = reinterpret_cast<u32x4 *>(s.terms_of(3, g, q));
    none[0] = none[1] = u32x4{0u, 0u, 0u, 0u};
  }
  for (int idx = first; idx < end; idx += W) {
    const int nlive = live_at(idx + W);
    const int64_t next = pr + (int64_t)(nlive ? idx + W : idx) * kAnBlock;
    {
      // zero times NaN is not zero: a row left out is finite.  (255, a NaN's byte, becomes an infinity, which converts to NaN.)
      const uint32_t vs = BETA && d.bias == -INFINITY ? 0x7f7f7f7fu : d.vs;
      s.ks[place] = d.ks;
      s.vs[0][place] = __uint_as_float((vs & 255u) << 23) * a.down;
      s.vs[1][place] = __uint_as_float((vs >> 8 & 255u) << 23) * a.down;
      s.vs[2][place] = __uint_as_float((vs >> 16 & 255u) << 23) * a.down;
      s.vs[3][place] = __uint_as_float(vs >> 24 << 23) * a.down;
      if constexpr (BETA) s.bias[place] = lane < live ? d.bias : -INFINITY;
    }
    wave_exchange();
    if constexpr (NQ > 1) load_planes();
    // ---- logits: rows 16 kt + 4 j + g of query q, a plane's part in each column
    float sv[N];
    {
      f32x4 dots[4];
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        i32x8 kf;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          kf[e] = (int)d.k[kt][e];
          kf[4 + e] = 0;
        }
        const int kscale = (int)reinterpret_cast<const uint8_t *>(s.ks)[4 * (16 * kt + r) + g];
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = NQ - 1; i >= 0; --i)
          acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, qf[i], acc, 4, 0, 0, kscale, 0, qscale[i]);
        dots[kt] = acc;
      }
      // the planes' parts meet; each of the C copies of a column goes on with its own share of the rows
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (C >= 2) dots[kt][j] += from_lane<8>(dots[kt][j]);
          if constexpr (C == 4) dots[kt][j] += from_lane<4>(dots[kt][j]);
        }
#pragma unroll
      for (int t = 0; t < N / 4; ++t) {
        f32x4 x = dots[t];
#pragma unroll
        for (int c = 1; c < C; ++c)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = part == c ? dots[c * (N / 4) + t][j] : x[j];
        const int kt = part * (N / 4) + t;
        if constexpr (BETA) {
          const float4 b = *reinterpret_cast<const float4 *>(&s.bias[16 * kt + 4 * g]);
          const float bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) sv[4 * t + j] = bv[j] != -INFINITY ? fmaf(a.scale, x[j], bv[j]) : -INFINITY;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) sv[4 * t + j] = 16 * kt + 4 * j + g < live ? a.scale * x[j] : -INFINITY;
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // the scales of this block's values leave LDS before the next block's come
    f32x4 vs[4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) vs[kt] = *reinterpret_cast<const f32x4 *>(&s.vs[r >> 2][16 * kt + 4 * g]);
    load_keys<BETA, NT>(a, next, nlive, d);
    __builtin_amdgcn_sched_barrier(0);
    // ---- probabilities relative to a reference m at or above every logit so far
    {
      float top = sv[0];
#pragma unroll
      for (int i = 1; i < N; ++i) top = fmaxf(top, sv[i]);
      if (__any(top > m)) {
        auto larger = [](float x, float y) { return fmaxf(x, y); };
        if constexpr (C == 4) top = fmaxf(top, from_lane<4>(top));
        if constexpr (C >= 2) top = fmaxf(top, from_lane<8>(top));
        top = over_rows(top, larger);
        const float to = top > m ? top + kAnLead : m, keep = m == to ? 1.0f : __builtin_amdgcn_exp2f((m - to) * 1.44269504f);
        l *= keep;
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[e][j] *= keep;
        m = to;
      }
      const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        sv[i] = __builtin_amdgcn_exp2f((sv[i] - ref) * 1.44269504f);
        l += sv[i];
      }
    }
    // ---- terms of the probabilities, to the lanes whose columns they are
    Frag pf[NP][2];   // of tokens 0 .. 31 and 32 .. 63
    if constexpr (C == 1) {
      split_p(sv, pf[0][0], pf[1][0], pf[2][0]);
      split_p(sv + 8, pf[0][1], pf[1][1], pf[2][1]);
    } else {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        uint32_t t[4][3];
#pragma unroll
        for (int j = 0; j < 4; ++j) terms(sv[4 * i + j], t[j]);
#pragma unroll
        for (int k = 0; k < 3; ++k)
          *reinterpret_cast<u32x2 *>(s.terms_of(k, g, q) + 2 * (part * (N / 4) + i)) =
              u32x2{upper_halves(t[0][k], t[1][k]), upper_halves(t[2][k], t[3][k])};
      }
      wave_exchange();
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          pf[i][h].v = *reinterpret_cast<const bf16x8 *>(s.terms_of(C * i + part, g, q) + 4 * h);
    }
    // ---- (P V)^T: values as rows, one dim 8 r + e of the lane's tokens to each of eight operands
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int eh = 0; eh < 2; ++eh) {
        Frag vf[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int kt = 2 * h + w / 2, j = 2 * (w % 2);
          eh ? value_pairs<2>(d.v[4 * kt + j], d.v[4 * kt + j + 1], vs[kt][j], vs[kt][j + 1], vf[0].w[w], vf[1].w[w])
             : value_pairs<0>(d.v[4 * kt + j], d.v[4 * kt + j + 1], vs[kt][j], vs[kt][j + 1], vf[0].w[w], vf[1].w[w]);
          eh ? value_pairs<3>(d.v[4 * kt + j], d.v[4 * kt + j + 1], vs[kt][j], vs[kt][j + 1], vf[2].w[w], vf[3].w[w])
             : value_pairs<1>(d.v[4 * kt + j], d.v[4 * kt + j + 1], vs[kt][j], vs[kt][j + 1], vf[2].w[w], vf[3].w[w]);
        }
#pragma unroll
        for (int i = NP - 1; i >= 0; --i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[4 * eh + e] = mfma16(vf[e].v, pf[i][h].v, o[4 * eh + e]);
      }
    __builtin_amdgcn_sched_barrier(0);
    load_values<NT>(a, next, nlive, d);
    wave_exchange();   // the next block's scales and terms take the place of what was read here
    __builtin_amdgcn_sched_barrier(0);
    live = nlive;
  }
  // each lane's share of the sum of probabilities meets the others
  if constexpr (C == 4) l += from_lane<4>(l);
  if constexpr (C >= 2) l += from_lane<8>(l);
  l = over_rows(l, [](float x, float y) { return x + y; });
}

// GP: the query rows that LDS and operands have room for, G <= GP <= 16.  W waves.
template <int W, int GP, bool BETA, bool STREAM>
__global__ void __launch_bounds__(64 * W, W == kAnW ? 3 : 2) k_attendn_partial(AttendN a) {
  constexpr int C = 16 / GP;
  __shared__ __align__(16) Queries<GP> sQ;
  union Own {
    WaveLds<GP> work;
    float o[GP][kHeadDim + 4];   // in its place the wave's sums once they are complete
  };
  __shared__ __align__(16) Own sOwn[W];
  __shared__ float sM[W][GP], sL[W][GP];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, r = lane & 15;
  const int ch = blockIdx.x, p = blockIdx.z * gridDim.y + blockIdx.y, G = a.G;
  if (p >= a.c.P) return;
  // units: blocks, then the tail's 32-row pieces; each chunk an equal share of those the pair has, wave by wave
  const int len = clip_len(a.length, p, a.c.rows), len_f = clip_len(a.length_f, p, a.F);
  const int blocks = (len + kAnBlock - 1) / kAnBlock, units = blocks + (len_f + kAttendTail - 1) / kAttendTail;
  const int iters = ((units + W - 1) / W + a.nch - 1) / a.nch;
  const int first = ch * iters * W + wave, end = min(units, (ch + 1) * iters * W);
  const int bend = min(end, blocks);
  QueryWords<W, GP> words;
  words.load(a, p);
  __builtin_amdgcn_sched_barrier(0);
  BlockData d;
  if (first < bend) {   // on their way while the queries are made ready
    constexpr int NT = STREAM ? kStreamed : 0;
    const int64_t row0 = (int64_t)p * a.c.rows + (int64_t)first * kAnBlock;
    const int live = __builtin_amdgcn_readfirstlane(min(len - first * kAnBlock, kAnBlock));
    load_keys<BETA, NT>(a, row0, live, d);
    load_values<NT>(a, row0, live, d);
    __builtin_amdgcn_sched_barrier(0);
  }
  make_queries<W, GP>(a, p, words, sQ);
  __syncthreads();
  float m = -INFINITY, l = 0.0f;
  f32x4 o[8] = {};
  if (first < bend) attend_blocks<W, GP, BETA, STREAM>(a, p, first, bend, len, sQ, sOwn[wave].work, d, m, l, o);
  if (end > blocks) {
    const int skip = first < blocks ? (blocks - first + W - 1) / W * W : 0;   // this wave's blocks
    const int tfirst = first + skip - blocks, tend = end - blocks;
    if (tfirst < tend) attend_tail<W, false, STREAM, GP>(a, p, tfirst, tend, len_f, sQ.tail, m, l, o, a.down);
  }
  // the terms' sums meet
  if constexpr (C > 1)
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        o[e][j] += from_lane<8>(o[e][j]);
        if constexpr (C == 4) o[e][j] += from_lane<4>(o[e][j]);
      }
  if (g == 0 && r < G) {
    sM[wave][r] = m;
    sL[wave][r] = l * a.down;   // as the sums beside it are
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

int units_of(int rows, int F) { return (rows + kAnBlock - 1) / kAnBlock + (F + kAttendTail - 1) / kAttendTail; }

// Waves of a workgroup.  A pair that is one workgroup's and has a CU to itself takes eight, two to a SIMD, where four would
// go round more than once.  us with 4 and with 8: 8 pairs of 819 + 37 rows 8.4 and 7.9, of 300 5.8 and 5.6; 64 of 1500 9.1 and 8.6;
// 200 of 600 + 64 for 16 queries 10.8 and 9.5; 256 of 4000 26.5 and 24.7.  Where four do not go round, more only wait: 300 of 60
// 5.2 and 7.5; of several chunks too: 8 of 2000 7.5 and 9.7.
int waves_of(int P, int units, int nch) { return nch == 1 && P <= kAnCus && units > kAnW ? kAnMore : kAnW; }

}  // namespace

// Chunks per pair, by the time that a call of as many takes, in ns: up to three workgroups run at a time on each of 256 CUs
// (the fullest ends the call), which share the memory's rate but need a wave's latency for each unit all the same; a
// workgroup's start, beside others on its CU; the second launch, which joins.  One chunk that eight waves take is priced as such
// where that is less.
// us per call by chunks: 512 pairs of 3277 + 256 rows 1: 49.3, 2: 50.5, 3: 52.2; of 8192-16384 rows 1: 139.2, 2: 148.1, 3: 144.3;
// eight waves' one chunk and others': 256 of 4500-9000 1: 43.4, 2: 45.8, 3: 44.6; of 4000 1: 24.9, 2: 27.4; 200 of 6621 1: 34.2, 2:
// 38.4, for 16 queries 40.5 and 45.7; 160 of 2500 1: 13.3, 2: 16.9, 3: 15.2; of 46849 1: 202, 2: 216, 3: 165; 64 of 2500 1: 11.6, 2: 11.6,
// 4: 10.8, 8: 12.6; 8 of 4000 1: 15.2, 4: 10.5, 16: 10.2; of 819 + 37 1: 8.2, 2: 10.0, 4: 9.9; 8 of 131072 21: 39.2, 32: 30.0, 64: 29.6,
// 86: 30.5; one of 131072 32: 20.6, 64: 15.1, 128: 14.0, 256: 17.1.
int attendn_chunks(int P, int rows, int F) {
  constexpr int64_t kAlone = 1000, kLatency = 1600, kShare = 1400, kStart = 3500, kMore = 1000, kJoin = 3000, kJoinChunk = 30,
                    kEight = 1600;   // eight waves' units: their latency, and the pairs' share of the memory's rate
  const int units = units_of(rows, F);
  const int n = (units + kAnW - 1) / kAnW;
  int best = 1;
  int64_t least = INT64_MAX;
  // of the numbers that give a wave as many units the least is best
  for (int c = 1; c <= n && (int64_t)P * (c - 1) < 2 * kAnSlots;) {
    const int units_each = (n + c - 1) / c;
    const int64_t wgs = (int64_t)P * c, rounds = (wgs + kAnSlots - 1) / kAnSlots;
    const int64_t on_cu = min((wgs + kAnCus - 1) / kAnCus, kAnSlots / kAnCus);
    int64_t blocks = units_each * (wgs <= kAnCus / 2 ? kAlone : max(kLatency, kShare * on_cu));
    if (waves_of(P, units, c) == kAnMore) blocks = min(blocks, (units + kAnMore - 1) / kAnMore * (kEight + kShare * P / kAnCus));
    const int64_t cost = rounds * (blocks + kStart + kMore * (on_cu - 1)) + (c > 1 ? kJoin + kJoinChunk * c : 0);
    if (cost < least) {
      least = cost;
      best = c;
    }
    if (units_each == 1) break;
    c = (n + units_each - 2) / (units_each - 1);
  }
  return best;
}

hipError_t launch_attendn(const NCache &c, int G, int F, float scale, const void *Q, const float *beta,
                          const int32_t *length, const void *Kf, const void *Vf, const int32_t *length_f, float *part_o,
                          float *part_ml, float *out, int nch, hipStream_t s) {
  AttendN a{c, G, F, scale, (const bf16 *)Q, beta, length, (const bf16 *)Kf, (const bf16 *)Vf, length_f, part_o, part_ml, out, nch,
            ldexpf(1.0f, -2 - (63 - __builtin_clzll((int64_t)c.rows + F)))};
  // pairs over y and z: a grid's y extent is limited
  const unsigned py = (unsigned)min(c.P, 32768), pz = (unsigned)((c.P + 32767) / 32768);
  const bool stream = (int64_t)c.P * c.rows * 2 * kNRow > kAnKept;
  const int waves = waves_of(c.P, units_of(c.rows, F), nch);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3((unsigned)a.nch, py, pz), dim3(64 * waves), 0, s, a);
    return hipGetLastError();
  };
  auto by_stream = [&](auto gp, auto bt) {
    constexpr int GP = decltype(gp)::value;
    constexpr bool BETA = decltype(bt)::value;
    if (waves == kAnMore)
      return stream ? go(k_attendn_partial<kAnMore, GP, BETA, true>) : go(k_attendn_partial<kAnMore, GP, BETA, false>);
    return stream ? go(k_attendn_partial<kAnW, GP, BETA, true>) : go(k_attendn_partial<kAnW, GP, BETA, false>);
  };
  auto by_beta = [&](auto gp) { return beta ? by_stream(gp, std::true_type{}) : by_stream(gp, std::false_type{}); };
  const hipError_t e = G <= 4 ? by_beta(std::integral_constant<int, 4>{})
                              : G <= 8 ? by_beta(std::integral_constant<int, 8>{}) : by_beta(std::integral_constant<int, 16>{});
  if (e != hipSuccess || a.nch == 1) return e;
  if (a.nch <= kCombineAhead)   // one group's loads
    hipLaunchKernelGGL((k_attend_combine<AttendN, 1>), dim3((unsigned)G, py, pz), dim3(kHeadDim), 0, s, a);
  else
    hipLaunchKernelGGL((k_attend_combine<AttendN, kCombineGroups>), dim3((unsigned)G, py, pz), dim3(kCombineGroups * kHeadDim), 0, s, a);
  return hipGetLastError();
}

}  // namespace arckv
