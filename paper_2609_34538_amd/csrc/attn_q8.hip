// Policy attention (Eq. (2)-(3)) over a cache held in 8 bits: e4m3 codes with one
// power-of-two scale per 8 tokens and KV head (das_attn_q8).
//
// A unit is one (sequence, KV head); its 32-token tiles, the draft block's first,
// then the prefix's, are cut into chunks of chunk_tiles, one workgroup of four
// waves each. RW of the waves hold different query rows (16 * NQ each), the other
// 4 / RW take a chunk's tiles in turn, each with its own running maximum, sum and
// output; they merge through LDS, and where a unit has several chunks these leave
// records that a second kernel merges. Up to 16 * NQ rows a wave has tiles of its own,
// from memory into registers, two on the way; waves that share a tile get it from LDS.
//
// Bound by HBM for few rows (32 x 55 heads x 32 rows, dh 96, 2.1 GB: 350 us, 6.1 TB/s) or
// by the longest unit's workgroup (24 x 8 KV heads x 1-4099 tokens, one query token, dh 128:
// 25 us, 4.0 TB/s), for many by the vector and matrix work of a tile, which two waves per
// SIMD do not overlap wholly (4 x 8 KV heads x 128 rows, dh 128, 137 MB: 60 us, 575
// TFLOP/s; 32 matrix instructions and 140 others on vectors a tile and wave). fp32 calls are
// bound by the fp32 matrix rate for many rows (4 x 8 KV heads x 128 rows x 4096 tokens, dh
// 128: 99 us, 87 TFLOP/s; 16 x 55 heads x 16 rows x 512-4096, dh 96: 119 us, 105 TFLOP/s).
//
// Both products take the key / value tile as the A operand, as in mfma_tile.h:
//   S^T (tokens x rows) = K . Q^T,   O^T (dh x rows) += V^T . P^T
// The page layouts give every lane its operands in 16-byte pieces: a key piece is
// 8 dims of the two tokens 8 G + n % 4 and + 4 that its two S^T tiles want, a value
// piece the 8 tokens of two neighbouring dims, which become rows of two O^T tiles.
// A wave's load is four runs of 256 bytes. Codes become bf16 keys and fp16 values
// in one instruction per two (v_cvt_scalef32_pk_*_fp8) that applies the scale and
// is exact.
//
// P.V of bf16 calls runs in fp16: e4m3 values are exact there and probabilities
// keep 11 bits instead of 8 (error against 64 bits then is the output's rounding).
// Values are held relative to the largest exponent that the wave
// has met (vref, per wave), which like the running maximum rescales the output
// when it grows, by a power of two. Draft-block values are bf16 with bf16's range:
// their probabilities enter as a bf16 and its remainder, two products. Sums are in units of
// 2^vref / 2^9, of 2^-73 or more after a block, which a value past 2^40 could take past the
// largest fp32: those, as what is not finite, are left out of the products and added one by
// one at the end, when the sums are plain, to the rows that see them (kLate). Waves without
// a block start in units of 2^-111, and one whose block lies under 2^-40 and which has met no
// scale over 2^-64 goes through its tiles again so: caches of the smallest scales keep their
// values.
// fp32 calls use v_mfma_f32_16x16x4_f32 for both products; reduction slots may be
// numbered freely as long as both operands agree, so the same pieces serve: step i
// takes a lane's i-th dim or token.

#include "mfma_tile.h"
#include "q8_internal.h"

namespace das {
namespace {

typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kTile = 32;
constexpr int kTilesPerPage = kPage / kTile;
constexpr int kWavesQ8 = 4;
// Probabilities are held relative to a reference that a row's logits may pass by
// kSlack binary orders before it moves; bf16 calls hold them times 2^kProbShift, so
// that the largest fit fp16 and those down to 2^-23 of the reference are normal there. Plain
// sums, and all of fp32 calls', are relative to the reference plus kSlack: no probability is
// over 1, so that a sum passes the largest fp32 only where the values' does.
constexpr float kSlack = 6.f;
constexpr float kProbShift = 9.f;
// Exponent of a wave's units at first: probabilities of 2^15 in them fit fp32, and the
// smallest codes of the smallest scale, 2^-9 * 2^-126, are 2^-24 of it, fp16's smallest.
constexpr int kLowUnit = -111;
constexpr float kBySlack = 0x1p-6f, kFromSlack = 0x1p6f;  // 2^-kSlack, 2^kSlack
constexpr float kNoRef = 3e38f;  // in place of shift - reference: nothing seen yet
// A reference past this (in base-2 units) is far: the rounding of reference * scale would be
// a factor of its own in every probability, past fp16's range from 2^27 on. A wave that has
// met one goes through its tiles again, in a form that takes the references off the logits
// (5 x 32 heads x 4 x 29 rows x 2005 tokens: 43.6 us without, 44.6 so, 46.7 with that form
// in the steps themselves).
constexpr float kFar = 0x1p20f;
constexpr float kLowest = -3.402823466e38f;  // as a reference of that form: nothing seen yet

__device__ __forceinline__ f32x4 mfma_f16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, a),
                                                __builtin_bit_cast(h16x8, b), c, 0, 0, 0);
}

// 8 codes (two words) times `scale`, a power of two.
__device__ __forceinline__ u32x4 codes_to_bf16(uint32_t lo, uint32_t hi, float scale) {
  return u32x4{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true))};
}
__device__ __forceinline__ u32x4 codes_to_f16(uint32_t lo, uint32_t hi, float scale) {
  return u32x4{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true))};
}
__device__ __forceinline__ void codes_to_f32(uint32_t lo, uint32_t hi, float scale, float (&x)[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(lo, scale, false);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(lo, scale, true);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, scale, false);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, scale, true);
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
  x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
}

// A tile as loaded: pieces of keys and values, and the exponent bytes of its four
// token groups (the same words in every lane).
template <int DH>
struct Raw {
  u32x4 k[DH / 32], v[DH / 32];
  uint32_t ke, ve;
};

// One wave's running result: neg = shift - reference (far form: the reference, before the
// scale), a lane's share of the sum l and the output o, in units of 2^vref for bf16 calls,
// both times 2^shift.
template <int DH, int NQ>
struct Acc {
  float neg[NQ], l[NQ];
  f32x4 o[NQ][DH / 16];
  int vref;
};

// The Q operand of a 16-row tile: bf16 one piece per 32 dims, fp32 two.
template <typename T, int DH>
struct QFrag {
  u32x4 x[DH / 32][sizeof(T) / 2];
};

// Softmax step of a tile: logits s[qt][e][v] (token 8 g + 4 e + v of the tile, row n)
// become probabilities in place, the lane's share of the sum is added. The reference
// (the same in a row's four lanes) moves to the row's maximum only when a logit passes it
// by more than kSlack, which after the first tiles is rare: most tiles need no reduction
// over lanes and no rescaling. E / 2 tiles at once; BLOCK: a row sees tokens up to its cap.
// F32: an fp32 call's. FAR: the far form; otherwise `far` receives the lanes of rows whose reference is far.
template <int DH, int NQ, int E, bool BLOCK, bool FAR, bool F32>
__device__ __forceinline__ void softmax_step(Acc<DH, NQ> &st, uint64_t &far, f32x4 (&s)[NQ][E], const int (&cap)[NQ],
                                             const int (&limit)[E / 2], float scale, float shift, int lg) {
  bool full = !BLOCK;
#pragma unroll
  for (int j = 0; j < E / 2; ++j) full = full && limit[j] >= kTile;
  float mx[NQ];
  bool moves = false;
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    if (!full) {
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int t = 8 * lg + 4 * (e % 2) + v;
          s[qt][e][v] = ((t < limit[e / 2]) & (!BLOCK | (t <= cap[qt]))) ? s[qt][e][v] : kNegInf;
        }
    }
    mx[qt] = kNegInf;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int v = 0; v < 4; ++v) mx[qt] = fmaxf(mx[qt], s[qt][e][v]);
    if constexpr (FAR) moves = true;
    else moves |= __builtin_fmaf(mx[qt], scale, st.neg[qt]) > shift + kSlack;
  }
  if (__builtin_amdgcn_ballot_w64(moves) != 0) {
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      float neg, alpha;
      if constexpr (FAR) {
        const float top = group_max(mx[qt]);
        neg = (top - st.neg[qt]) * scale > kSlack ? top : st.neg[qt];
        alpha = __builtin_amdgcn_exp2f((st.neg[qt] - neg) * scale);
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int v = 0; v < 4; ++v) s[qt][e][v] -= neg;
      } else {
        const float m = group_max(mx[qt]) * scale;
        // rows with nothing visible, and those that stay within their slack, keep theirs
        neg = m + st.neg[qt] > shift + kSlack ? shift - m : st.neg[qt];
        alpha = __builtin_amdgcn_exp2f(neg - st.neg[qt]);  // 0 from kNoRef
        far |= __builtin_amdgcn_ballot_w64(fabsf(neg) > kFar && neg != kNoRef);
      }
      st.neg[qt] = neg;
      st.l[qt] *= alpha;
      // a lane's accumulators of row tile qt all belong to one row
#pragma unroll
      for (int dt = 0; dt < DH / 16; ++dt) st.o[qt][dt] *= alpha;
    }
  }
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qt][e][v], scale, FAR ? shift : st.neg[qt]));
        if constexpr (F32) p *= kBySlack;
        s[qt][e][v] = p;
        st.l[qt] += p;
      }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const bf16x2 h = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
  return __builtin_bit_cast(uint32_t, h);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const h16x2 h = {static_cast<_Float16>(a), static_cast<_Float16>(b)};
  return __builtin_bit_cast(uint32_t, h);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Codes of a tile's values with those of invisible tokens cleared, and the exponent byte
// of their group, 1 where none of it is visible: whatever the page holds there adds nothing.
// On the codes and in a branch: masks on the converted values took 32 of the 235 vector
// instructions of every tile.
template <int N>
__device__ __forceinline__ void clear_invisible(u32x4 (&v)[N], uint32_t &vexp, int limit, int lg) {
  const int seen = min(max(limit - 8 * lg, 0), 8);
  const uint32_t lo = seen >= 4 ? ~0u : (1u << 8 * seen) - 1;
  const uint32_t hi = seen >= 8 ? ~0u : seen <= 4 ? 0u : (1u << 8 * (seen - 4)) - 1;
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] &= u32x4{lo, hi, lo, hi};
  if (seen == 0) vexp = 1;
}
// The largest exponent of the groups with a visible token, as a wave-uniform value.
__device__ __forceinline__ int most_exponent(uint32_t ve, int limit) {
  uint32_t w = __builtin_amdgcn_readfirstlane(ve);
  if (limit < kTile) w &= limit > 24 ? ~0u : limit > 16 ? 0xffffffu : limit > 8 ? 0xffffu : limit > 0 ? 0xffu : 0u;
  return max(max(static_cast<int>(w & 255), static_cast<int>(w >> 8 & 255)),
             max(static_cast<int>(w >> 16 & 255), static_cast<int>(w >> 24))) - 127;
}
// Output in units of 2^vref from now on.
template <int DH, int NQ>
__device__ __forceinline__ void raise_vref(Acc<DH, NQ> &st, int vref) {
  if (vref <= st.vref) return;
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
    for (int dt = 0; dt < DH / 16; ++dt)
#pragma unroll
      for (int v = 0; v < 4; ++v) st.o[qt][dt][v] = __builtin_amdgcn_ldexpf(st.o[qt][dt][v], st.vref - vref);
  st.vref = vref;
}
// Scale of a group's values in units of 2^vref.
__device__ __forceinline__ float scale_of(uint32_t vexp, int vref) {
  return __uint_as_float(static_cast<uint32_t>(max(static_cast<int>(vexp) - vref, 0)) << 23);
}
// A tile of the prefix through both products. `limit`: visible tokens.
template <typename T, int DH, int NQ, bool FAR = false>
__device__ __forceinline__ void prefix_tile(Acc<DH, NQ> &st, uint64_t &far, Raw<DH> &t,
                                            const QFrag<T, DH> (&qf)[NQ], int limit, float scale,
                                            int ln, int lg) {
  const bool full = limit >= kTile;
  const float ks = __uint_as_float(__builtin_amdgcn_ubfe(t.ke, 8 * (ln >> 2), 8) << 23);
  f32x4 s[NQ][2], odd[NQ][2];  // odd: fp32's second chains, half the roundings each
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt)
    s[qt][0] = s[qt][1] = odd[qt][0] = odd[qt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < DH / 32; ++k) {
    if constexpr (sizeof(T) == 2) {
      const u32x4 a0 = codes_to_bf16(t.k[k][0], t.k[k][1], ks);
      const u32x4 a1 = codes_to_bf16(t.k[k][2], t.k[k][3], ks);
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
        s[qt][0] = mfma16x16x32(a0, qf[qt].x[k][0], s[qt][0]);
        s[qt][1] = mfma16x16x32(a1, qf[qt].x[k][0], s[qt][1]);
      }
    } else {
      float a0[8], a1[8];
      codes_to_f32(t.k[k][0], t.k[k][1], ks, a0);
      codes_to_f32(t.k[k][2], t.k[k][3], ks, a1);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) {
          const uint32_t b = qf[qt].x[k][i / 4][i % 4];
          f32x4 &c0 = i % 2 ? odd[qt][0] : s[qt][0], &c1 = i % 2 ? odd[qt][1] : s[qt][1];
          c0 = mfma16x16x4(__float_as_uint(a0[i]), b, c0);
          c1 = mfma16x16x4(__float_as_uint(a1[i]), b, c1);
        }
    }
  }
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) s[qt][0] += odd[qt][0], s[qt][1] += odd[qt][1];
  }
  const int none[NQ] = {}, limits[1] = {limit};
  softmax_step<DH, NQ, 2, false, FAR, sizeof(T) == 4>(st, far, s, none, limits, scale, sizeof(T) == 2 ? kProbShift : 0.f, lg);

  uint32_t vexp = __builtin_amdgcn_ubfe(t.ve, 8 * lg, 8);
  if (!full) clear_invisible(t.v, vexp, limit, lg);
  if constexpr (sizeof(T) == 2) {
    raise_vref(st, most_exponent(t.ve, limit));
    const float vs = scale_of(vexp, st.vref);
    u32x4 pf[NQ];
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt)
      pf[qt] = u32x4{pack_f16(s[qt][0][0], s[qt][0][1]), pack_f16(s[qt][0][2], s[qt][0][3]),
                     pack_f16(s[qt][1][0], s[qt][1][1]), pack_f16(s[qt][1][2], s[qt][1][3])};
#pragma unroll
    for (int k = 0; k < DH / 32; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x4 a = codes_to_f16(t.v[k][2 * i], t.v[k][2 * i + 1], vs);
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) st.o[qt][2 * k + i] = mfma_f16(a, pf[qt], st.o[qt][2 * k + i]);
      }
  } else {
    const float vs = __uint_as_float(vexp << 23);
#pragma unroll
    for (int k = 0; k < DH / 32; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float a[8];
        codes_to_f32(t.v[k][2 * i], t.v[k][2 * i + 1], vs, a);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
          for (int qt = 0; qt < NQ; ++qt)
            st.o[qt][2 * k + i] = mfma16x16x4(__float_as_uint(a[j]), __float_as_uint(s[qt][j / 4][j % 4]),
                                              st.o[qt][2 * k + i]);
        }
      }
  }
}

// A bf16 call's N tiles, `stride` bytes apart, from their converted fragments in LDS: 2 KB
// per 32 dims of keys, then of values, of which a lane takes 16 bytes twice. Values are in
// units of 2^st.vref. One softmax step for all of them: fewer branches, and products of one
// tile while another's probabilities are made.
constexpr int kConvBytes = 2048;
template <int DH, int NQ, int N>
__device__ __forceinline__ void shared_tiles(Acc<DH, NQ> &st, uint64_t &far, const uint8_t *tiles, int stride,
                                             const QFrag<bf16_t, DH> (&qf)[NQ], const int (&limit)[N], float scale,
                                             int lane) {
  constexpr int KS = DH / 32;
  auto part = [&](int t, int f, int i) {
    return *reinterpret_cast<const u32x4 *>(tiles + t * stride + f * kConvBytes + i * kFragBytes + 16 * lane);
  };
  f32x4 s[NQ][2 * N];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
    for (int e = 0; e < 2 * N; ++e) s[qt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const u32x4 a = part(t, k, e);
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) s[qt][2 * t + e] = mfma16x16x32(a, qf[qt].x[k][0], s[qt][2 * t + e]);
      }
  const int none[NQ] = {};
  softmax_step<DH, NQ, 2 * N, false, false, false>(st, far, s, none, limit, scale, kProbShift, lane >> 4);
#pragma unroll
  for (int t = 0; t < N; ++t) {
    u32x4 pf[NQ];
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt)
      pf[qt] = u32x4{pack_f16(s[qt][2 * t][0], s[qt][2 * t][1]), pack_f16(s[qt][2 * t][2], s[qt][2 * t][3]),
                     pack_f16(s[qt][2 * t + 1][0], s[qt][2 * t + 1][1]),
                     pack_f16(s[qt][2 * t + 1][2], s[qt][2 * t + 1][3])};
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x4 a = part(t, KS + k, i);
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) st.o[qt][2 * k + i] = mfma_f16(a, pf[qt], st.o[qt][2 * k + i]);
      }
  }
}

// The bits of the smallest block value that is added late: 2^40 in bf16 calls (probabilities
// reach 2^15 in units of 2^-64, and a block has 64 positions: 2^125 at most), in fp32 calls
// infinity.
template <typename T>
constexpr uint32_t kLate = sizeof(T) == 2 ? (127u + 40) << 7 : 0x7f800000u;
// A word of block values (two bf16 or one fp32) with those of them replaced by 0.
template <typename T>
__device__ __forceinline__ uint32_t without_late(uint32_t w) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t lo = (w & 0x7fffu) >= kLate<T> ? 0u : w & 0xffffu;
    return (w >> 16 & 0x7fffu) >= kLate<T> ? lo : lo | (w & 0xffff0000u);
  } else {
    return (w & 0x7fffffffu) >= kLate<T> ? 0u : w;
  }
}
template <typename T>
__device__ __forceinline__ bool is_late(float x) {
  return (__float_as_uint(x) & 0x7fffffffu) >= (sizeof(T) == 2 ? kLate<T> << 16 : kLate<T>);
}

// A draft-block tile as loaded, in the call's type, straight from the token-major rows:
// a lane's pieces of its two key tokens, and its 8 tokens of value dims 32 k + 2 n, + 1.
// Rows past the block's last repeat it and are masked.
template <typename T, int DH>
struct Block {
  static constexpr int W = sizeof(T) / 2;
  u32x4 k[2][DH / 32][W];
  uint32_t v[DH / 32][8][W];
};
template <typename T, int DH>
__device__ __forceinline__ void load_block(Block<T, DH> &t, const AttnQ8Params &p, int b, int kvh, int u, int ln,
                                           int lg) {
  const size_t row_elems = static_cast<size_t>(p.hkv) * DH;
  const size_t base = (static_cast<size_t>(b) * p.w * p.hkv + kvh) * DH;
  const T *kb = static_cast<const T *>(p.kb) + base, *vb = static_cast<const T *>(p.vb) + base;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int tok = min(kTile * u + 8 * (ln >> 2) + (ln & 3) + 4 * e, p.w - 1);
    const T *row = kb + tok * row_elems + 8 * lg;
#pragma unroll
    for (int k = 0; k < DH / 32; ++k)
#pragma unroll
      for (int h = 0; h < Block<T, DH>::W; ++h) t.k[e][k][h] = reinterpret_cast<const u32x4 *>(row + 32 * k)[h];
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const T *row = vb + min(kTile * u + 8 * lg + j, p.w - 1) * row_elems + 2 * ln;
#pragma unroll
    for (int k = 0; k < DH / 32; ++k) {
      if constexpr (sizeof(T) == 2) {
        t.v[k][j][0] = *reinterpret_cast<const uint32_t *>(row + 32 * k);
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(row + 32 * k);
        t.v[k][j][0] = x[0], t.v[k][j][1] = x[1];
      }
    }
  }
}

// Logits of tile u of the draft block.
template <typename T, int DH, int NQ>
__device__ __forceinline__ void block_logits(f32x4 (&s)[NQ][2], const Block<T, DH> &t, const QFrag<T, DH> (&qf)[NQ]) {
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) s[qt][0] = s[qt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < DH / 32; ++k)
#pragma unroll
    for (int h = 0; h < Block<T, DH>::W; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int qt = 0; qt < NQ; ++qt) s[qt][e] = mfma16x16x32(t.k[e][k][0], qf[qt].x[k][0], s[qt][e]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) s[qt][e] = mfma16x16x4(t.k[e][k][h][i], qf[qt].x[k][h][i], s[qt][e]);
        }
      }
}

// Tile u of the draft block through both products. What its values are: kHasLate, some are
// left to late_values; kHasLarge, some are 2^-40 or more (bf16 calls).
constexpr uint32_t kHasLate = 1, kHasLarge = 2;
template <typename T, int DH, int NQ, bool FAR = false>
__device__ __forceinline__ uint32_t block_tile(Acc<DH, NQ> &st, uint64_t &far, Block<T, DH> &t,
                                               const AttnQ8Params &p, int u, const QFrag<T, DH> (&qf)[NQ],
                                               const int (&row_pos)[NQ], int lg) {
  constexpr int KS = DH / 32;
  f32x4 s[NQ][2];
  block_logits<T, DH, NQ>(s, t, qf);
  int cap[NQ];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) cap[qt] = row_pos[qt] - kTile * u;
  const int limits[1] = {p.w - kTile * u};
  softmax_step<DH, NQ, 2, true, FAR, sizeof(T) == 4>(st, far, s, cap, limits, p.scale_log2,
                                                     sizeof(T) == 2 ? kProbShift : 0.f, lg);

  // the largest magnitude's bits tell whether any is late
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 most = {0, 0};
  uint32_t most32 = 0;
#pragma unroll
  for (int k = 0; k < KS; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (sizeof(T) == 2)
        most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, t.v[k][j][0] & 0x7fff7fffu));
      else
        most32 = max(most32, max(t.v[k][j][0] & 0x7fffffffu, t.v[k][j][1] & 0x7fffffffu));
    }
  if constexpr (sizeof(T) == 2) most32 = max(most[0], most[1]);
  const bool any_late = __builtin_amdgcn_ballot_w64(most32 >= kLate<T>) != 0;
  if (any_late) {
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int h = 0; h < Block<T, DH>::W; ++h) t.v[k][j][h] = without_late<T>(t.v[k][j][h]);
  }
  if constexpr (sizeof(T) == 2) {
    u32x4 hi[NQ], lo[NQ];
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a = __builtin_amdgcn_ldexpf(s[qt][j / 2][2 * (j % 2)], -st.vref);
        const float c = __builtin_amdgcn_ldexpf(s[qt][j / 2][2 * (j % 2) + 1], -st.vref);
        hi[qt][j] = pack_bf16(a, c);
        lo[qt][j] = pack_bf16(a - bf16_lo(hi[qt][j]), c - bf16_hi(hi[qt][j]));
      }
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      u32x4 a0, a1;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t x = t.v[k][2 * j][0], y = t.v[k][2 * j + 1][0];
        a0[j] = __builtin_amdgcn_perm(y, x, 0x05040100);
        a1[j] = __builtin_amdgcn_perm(y, x, 0x07060302);
      }
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
        st.o[qt][2 * k] = mfma16x16x32(a0, lo[qt], st.o[qt][2 * k]);
        st.o[qt][2 * k + 1] = mfma16x16x32(a1, lo[qt], st.o[qt][2 * k + 1]);
        st.o[qt][2 * k] = mfma16x16x32(a0, hi[qt], st.o[qt][2 * k]);
        st.o[qt][2 * k + 1] = mfma16x16x32(a1, hi[qt], st.o[qt][2 * k + 1]);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int qt = 0; qt < NQ; ++qt)
            st.o[qt][2 * k + h] = mfma16x16x4(t.v[k][j][h], __float_as_uint(s[qt][j / 4][j % 4]), st.o[qt][2 * k + h]);
  }
  constexpr uint32_t kLarge = (127u - 40) << 7;  // bits of 2^-40
  return (any_late ? kHasLate : 0) | (__builtin_amdgcn_ballot_w64(most32 >= kLarge) != 0 ? kHasLarge : 0);
}

// The late values of tile u of the draft block, for the rows that see them (in a product
// 0 * NaN would reach the rows that do not). Of st, sums are plain here and m their
// references in base-2 units; probs: the wave's place in LDS for the tile's probabilities,
// [row tile][row][token].
template <typename T, int DH, int NQ>
__device__ __forceinline__ void late_values(Acc<DH, NQ> &st, bool far, const float (&m)[NQ], const AttnQ8Params &p,
                                            int b, int kvh, int u, const QFrag<T, DH> (&qf)[NQ],
                                            const int (&row_pos)[NQ], float *probs, int ln, int lg) {
  Block<T, DH> t;
  load_block<T, DH>(t, p, b, kvh, u, ln, lg);
  f32x4 s[NQ][2];
  block_logits<T, DH, NQ>(s, t, qf);
  __builtin_amdgcn_wave_barrier();  // the tile before has been read
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    f32x4 *dst = reinterpret_cast<f32x4 *>(probs + (16 * qt + ln) * kTile + 8 * lg);
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float x = far ? s[qt][e][v] - st.neg[qt] : s[qt][e][v];
        s[qt][e][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(x, p.scale_log2, far ? 0.f : -m[qt])) * kBySlack;
      }
    dst[0] = s[qt][0], dst[1] = s[qt][1];
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const size_t row_elems = static_cast<size_t>(p.hkv) * DH;
  const T *vb = static_cast<const T *>(p.vb) + (static_cast<size_t>(b) * p.w * p.hkv + kvh) * DH;
#pragma unroll
  for (int k = 0; k < DH / 32; ++k) {
#pragma unroll 1
    for (int i = 0; i < kTile && kTile * u + i < p.w; ++i) {
      const T *src = vb + (kTile * u + i) * row_elems + 32 * k + 8 * lg;
#pragma unroll
      for (int qt = 0; qt < NQ; ++qt) {
        const float pt = probs[(16 * qt + ln) * kTile + i];
#pragma unroll
        for (int j = 0; j < 8; ++j) {  // tile 2 k + j % 2 holds dim 32 k + 8 g + j
          const float x = to_f32<T>(src[j]);
          if (is_late<T>(x) && kTile * u + i <= row_pos[qt]) st.o[qt][2 * k + j % 2][j / 2] += pt * x;
        }
      }
    }
  }
}

// Eight neighbouring results of a lane: tiles 2 k and 2 k + 1 hold dims 32 k + 8 g + 2 v and + 1.
template <int DH>
__device__ __forceinline__ void eight(const f32x4 (&o)[DH / 16], int k, float scale, f32x4 &lo, f32x4 &hi) {
  const f32x4 x = o[2 * k] * scale, y = o[2 * k + 1] * scale;
  lo = f32x4{x[0], y[0], x[1], y[1]};
  hi = f32x4{x[2], y[2], x[3], y[3]};
}
// A row's record (write_piece_row's form) and its output, by its four lanes.
template <typename T, int DH>
__device__ __forceinline__ void write_record_row(uint8_t *rec, int rows, int row, int lg,
                                                 const f32x4 (&o)[DH / 16], float m, float l) {
  float q = 1.f, sc = 1.f;
  if constexpr (sizeof(T) == 2) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    float amax = 0.f;
#pragma unroll
    for (int dt = 0; dt < DH / 16; ++dt)
#pragma unroll
      for (int v = 0; v < 4; ++v) amax = fmaxf(amax, fabsf(o[dt][v]));
    amax = group_max(amax) * inv;
    const int e = record_exponent(amax);
    sc = __builtin_amdgcn_ldexpf(inv, -e);
    q = __builtin_amdgcn_ldexpf(l, e);
  }
#pragma unroll
  for (int k = 0; k < DH / 32; ++k) {
    f32x4 lo, hi;
    eight<DH>(o, k, sc, lo, hi);
    uint8_t *dst = rec + (static_cast<size_t>(row) * DH + 32 * k + 8 * lg) * rec_elem_bytes(sizeof(T));
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x4 *>(dst) =
          u32x4{pack_f16(lo[0], lo[1]), pack_f16(lo[2], lo[3]), pack_f16(hi[0], hi[1]), pack_f16(hi[2], hi[3])};
    } else {
      reinterpret_cast<f32x4 *>(dst)[0] = lo;
      reinterpret_cast<f32x4 *>(dst)[1] = hi;
    }
  }
  if (lg == 0)
    *reinterpret_cast<f32x4 *>(rec + static_cast<size_t>(rows) * DH * rec_elem_bytes(sizeof(T)) + row * 16) =
        f32x4{m, l, q, 0.f};
}
template <typename T, int DH>
__device__ __forceinline__ void write_output_row(const AttnQ8Params &p, int b, int kvh, int row, int lg,
                                                 const f32x4 (&o)[DH / 16], float m, float l) {
  const int pos = row / p.group, h = kvh * p.group + row % p.group;
  T *out = static_cast<T *>(p.out) + ((static_cast<size_t>(b) * p.w + pos) * p.hq + h) * DH;
  const float inv = 1.f / l;
#pragma unroll
  for (int k = 0; k < DH / 32; ++k) {
    f32x4 lo, hi;
    eight<DH>(o, k, inv, lo, hi);
    store_out4(out + 32 * k + 8 * lg, lo);
    store_out4(out + 32 * k + 8 * lg + 4, hi);
  }
  if (lg == 0 && p.lse)
    p.lse[(static_cast<size_t>(b) * p.hq + h) * p.w + pos] = (m + log2f(l * kFromSlack)) * 0.69314718055994530942f;
}

// Shared memory of a workgroup.
// RW == 1: the merge area of one row tile, before that a block tile's probabilities for its
// late values.
// RW > 1, bf16: two steps of IW * TPS converted tiles; afterwards, in the second one's place,
// the probabilities, and then, with IW > 1, the merge area.
// RW > 1, fp32: a ring of NB steps of IW * TPS tiles of codes, their exponents per wave, and
// the probabilities; afterwards the merge area.
template <typename T, int DH, int NQ, int RW>
struct Lds {
  static constexpr bool CONV = RW > 1 && sizeof(T) == 2;
  static constexpr int IW = kWavesQ8 / RW;             // waves that share a chunk's tiles
  static constexpr int TPS = RW == 4 ? 2 : 1;          // tiles of a wave and step
  static constexpr int NB = RW == 1 ? 0 : CONV ? 2 : 3;  // steps held
  static constexpr int TILE = CONV ? 2 * (DH / 32) * kConvBytes : 2 * kTile * DH;  // bytes of a tile
  static constexpr int STEP = IW * TPS * TILE;
  static constexpr int RS = DH + 4;                    // row stride of the merge area (floats)
  static constexpr int EXPS = NB * STEP;
  static constexpr int PROBS = CONV ? STEP : EXPS + NB * TPS * kWavesQ8 * 8;
  static constexpr int PROB_STRIDE = RW == 1 ? 16 * RS * 4 : 16 * NQ * kTile * 4;
  static constexpr int MERGE = IW == 1 ? 0 : kWavesQ8 * 16 * RS * 4;
  static constexpr int WITH_PROBS = PROBS + kWavesQ8 * PROB_STRIDE;
  static constexpr int HELD = EXPS > WITH_PROBS ? EXPS : WITH_PROBS;
  static constexpr int BYTES = HELD > MERGE ? HELD : MERGE;
  static_assert(PROB_STRIDE >= 16 * NQ * kTile * 4 && PROBS % 16 == 0, "a tile's probabilities fit");
};

template <typename T, int DH, int NQ, int RW>
__global__ __launch_bounds__(64 * kWavesQ8) __attribute__((amdgpu_waves_per_eu(2)))
void attn_q8_kernel(AttnQ8Params p, int n_rg) {
  using L = Lds<T, DH, NQ, RW>;
  constexpr int IW = L::IW;
  constexpr int RS = L::RS;
  constexpr int KS = DH / 32;
  __shared__ __attribute__((aligned(16))) uint8_t smem[L::BYTES];
  float(*part)[16 * RS] = reinterpret_cast<float(*)[16 * RS]>(smem);
  __shared__ float sm[kWavesQ8][16 * NQ], sl[kWavesQ8][16 * NQ], sa[kWavesQ8][16 * NQ];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ln = lane & 15, lg = lane >> 4;
  const int rw = wave % RW, iw = wave / RW;
  // every unit's first chunk comes before any second one
  const int units = p.batch * p.hkv;
  const int rg = blockIdx.x % n_rg, grp = blockIdx.x / n_rg;
  const int unit = grp % units, chunk = grp / units;
  const int b = unit / p.hkv, kvh = unit % p.hkv;
  const int row0 = rg * (16 * NQ * RW) + rw * (16 * NQ);
  const int nb = (p.w + kTile - 1) / kTile;
  const int g0 = chunk * p.chunk_tiles + iw;  // this wave's first tile of the unit

  const int s_raw = p.prefix_len[b];
  QFrag<T, DH> qf[NQ];
  int row_pos[NQ];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    // rows past the last are clamped; their outputs are never written
    const int row = min(row0 + qt * 16 + ln, p.rows - 1);
    const int i = row / p.group, g = row % p.group;
    row_pos[qt] = i;
    const T *qrow = static_cast<const T *>(p.q) +
                    ((static_cast<size_t>(b) * p.w + i) * p.hq + kvh * p.group + g) * DH;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int h = 0; h < static_cast<int>(sizeof(T)) / 2; ++h)
        qf[qt].x[k][h] = reinterpret_cast<const u32x4 *>(qrow + 32 * k + 8 * lg)[h];
  }
  // page ids: lane i holds the page of this wave's (window + i)-th tile
  auto load_window = [&](int first) {
    const int pg = (g0 + IW * (first + lane) - nb) / kTilesPerPage;
    return g0 + IW * (first + lane) >= nb && pg < p.max_pages
               ? p.block_table[static_cast<size_t>(b) * p.max_pages + pg] : 0;
  };
  int window = load_window(0);
  // draft-block tiles come first: tiles 0 .. nb - 1 of chunk 0
  Block<T, DH> blk;
  const bool has_block = g0 < nb;
  if (has_block) load_block<T, DH>(blk, p, b, kvh, g0, ln, lg);

  bool bad;
  const int S = clamp_prefix(s_raw, p.max_pages, &bad);
  if (bad && kvh == 0 && rg == 0 && chunk == 0 && threadIdx.x == 0)
    report_error(p.dev_error, DAS_DEVERR_PREFIX);
  const int ntile = nb + (S + kTile - 1) / kTile;
  const int nsb = (ntile + p.chunk_tiles - 1) / p.chunk_tiles;  // chunks of this unit
  if (chunk >= nsb) return;
  const int g_end = min(ntile, (chunk + 1) * p.chunk_tiles);
  const int n = g_end > g0 ? (g_end - g0 + IW - 1) / IW : 0;  // this wave's tiles

  Acc<DH, NQ> st;
  uint64_t far = 0;  // lanes of rows that have met a far reference
  auto clear = [&](float neg, int vref) {
    st.vref = vref;
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      st.neg[qt] = neg;
      st.l[qt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DH / 16; ++dt) st.o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  clear(kNoRef, has_block ? kQ8MinExp : kLowUnit);

  const uint32_t lane_k = (ln >> 2) * 8 * DH + lg * 64 + (ln & 3) * 16;
  const uint32_t lane_v = lg * 8 * DH + ln * 16;
  // Where the wave's i-th tile lies, and the number of its visible tokens. An out-of-range
  // page id is reported and read as page 0 (its tile is masked out).
  auto locate = [&](int i, size_t &off, size_t &eoff) {
    if (i >= 64 && i % 64 == 0) {
      window = load_window(i);
      wait_vmcnt<0>();  // here: otherwise every use of it waits for all loads under way
    }
    const int page_raw = __builtin_amdgcn_readlane(window, i & 63);
    const bool ok = page_raw >= 0 && page_raw < p.num_pages;
    if (!ok && i < n) report_error(p.dev_error, DAS_DEVERR_PAGE);
    const int page = ok ? page_raw : 0;
    const int tile = g0 + IW * i - nb, half = tile % kTilesPerPage;
    off = (static_cast<size_t>(kvh) * p.num_pages + page) * (kPage * DH) + half * kTile * DH;
    eoff = (static_cast<size_t>(page) * p.hkv + kvh) * kQ8GroupsPerPage + 4 * half;
    return ok ? min(kTile, S - kTile * tile) : 0;
  };
  const int n_block = g0 < nb ? min((nb - g0 + IW - 1) / IW, n) : 0;  // the wave's block tiles
  uint32_t block = 0;                                                 // what they hold

  // The wave's i-th tile into registers. Past the last tile the loads go to empty buffers:
  // they are always issued, so that the compiler can count them, and waits for one tile leave
  // the next under way.
  auto load = [&](int i, Raw<DH> &t) {
    size_t off, eoff;
    const int visible = locate(i, off, eoff);
    const int bytes = i < n ? kTile * DH : 0;
    const auto rk = buffer_of(p.k_layer + off, bytes), rv = buffer_of(p.v_layer + off, bytes);
#pragma unroll
    for (int k = 0; k < KS; ++k)
      t.k[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, lane_k, 256 * k, kNonTemporal));
#pragma unroll
    for (int k = 0; k < KS; ++k)
      t.v[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, lane_v, 256 * k, kNonTemporal));
    t.ke = __builtin_amdgcn_raw_buffer_load_b32(buffer_of(p.k_exp + eoff, bytes ? 4 : 0), 0, 0, kCached);
    t.ve = __builtin_amdgcn_raw_buffer_load_b32(buffer_of(p.v_exp + eoff, bytes ? 4 : 0), 0, 0, kCached);
    return visible;
  };

  if constexpr (RW == 1) {
    // two tiles in flight, the first of the prefix before the block's are worked on
    Raw<DH> ta, tb;
    int i = n_block;
    int la = load(i, ta);
    if (has_block) {
      block = block_tile<T, DH, NQ>(st, far, blk, p, g0, qf, row_pos, lg);
      for (int k = 1; k < n_block; ++k) {
        load_block<T, DH>(blk, p, b, kvh, g0 + IW * k, ln, lg);
        block |= block_tile<T, DH, NQ>(st, far, blk, p, g0 + IW * k, qf, row_pos, lg);
      }
    }
    int lb = load(i + 1, tb);
    for (; i < n; i += 2) {
      prefix_tile<T, DH, NQ>(st, far, ta, qf, la, p.scale_log2, ln, lg);
      la = load(i + 2, ta);
      if (i + 1 < n) prefix_tile<T, DH, NQ>(st, far, tb, qf, lb, p.scale_log2, ln, lg);
      lb = load(i + 3, tb);
    }
  } else if constexpr (L::CONV) {
    // Waves that share a tile share its conversion: each brings every RW-th fragment's codes
    // into registers, a step ahead, and writes them converted to LDS, from where all multiply.
    // One barrier a step publishes step s and frees the slot of step s - 1, which step s + 1
    // takes. All know the exponents, and with them the same vref. Codes in LDS, converted by
    // every wave, took 250 vector instructions a tile instead of 170, its 32 matrix ones
    // included (128 rows 64 -> 59 us, dh 64 49 -> 43); three waves per SIMD spill (133 us).
    constexpr int TPS = L::TPS, LPW = (2 * KS + RW - 1) / RW;
    const int np = n - n_block;  // this wave's prefix tiles
    const int steps = (g_end - chunk * p.chunk_tiles + IW * TPS - 1) / (IW * TPS);  // of every wave
    u32x4 raw[TPS][LPW];
    uint32_t ke[TPS], ve[TPS];
    int limit[TPS], ahead[TPS];
    int vref = st.vref;
    // always issued, past the last tile from empty buffers
    auto load = [&](int step) {
#pragma unroll
      for (int t = 0; t < TPS; ++t) {
        const int i = n_block + TPS * step + t;
        size_t off, eoff;
        const int visible = locate(i, off, eoff);
        ahead[t] = i < n ? visible : 0;
        const int bytes = i < n ? kTile * DH : 0;
        const auto rk = buffer_of(p.k_layer + off, bytes), rv = buffer_of(p.v_layer + off, bytes);
#pragma unroll
        for (int c = 0; c < LPW; ++c) {
          const int f = min(rw + RW * c, 2 * KS - 1);  // the last may be loaded by several
          const bool key = f < KS;
          raw[t][c] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
              key ? rk : rv, key ? lane_k : lane_v, 256 * (key ? f : f - KS), kNonTemporal));
        }
        ke[t] = __builtin_amdgcn_raw_buffer_load_b32(buffer_of(p.k_exp + eoff, bytes ? 4 : 0), 0, 0, kCached);
        ve[t] = __builtin_amdgcn_raw_buffer_load_b32(buffer_of(p.v_exp + eoff, bytes ? 4 : 0), 0, 0, kCached);
      }
    };
    auto convert = [&](int step) {
      uint8_t *slot = smem + (step % 2) * L::STEP + iw * L::TILE + 16 * lane;
#pragma unroll
      for (int t = 0; t < TPS; ++t) vref = max(vref, most_exponent(ve[t], ahead[t]));
#pragma unroll
      for (int t = 0; t < TPS; ++t) {
        limit[t] = ahead[t];
        const float ks = __uint_as_float(__builtin_amdgcn_ubfe(ke[t], 8 * (ln >> 2), 8) << 23);
#pragma unroll
        for (int c = 0; c < LPW; ++c) {
          const int f = rw + RW * c;
          if (f >= 2 * KS) continue;
          u32x4 x, y;
          if (f < KS) {
            x = codes_to_bf16(raw[t][c][0], raw[t][c][1], ks);
            y = codes_to_bf16(raw[t][c][2], raw[t][c][3], ks);
          } else {
            uint32_t vexp = __builtin_amdgcn_ubfe(ve[t], 8 * lg, 8);
            u32x4 v[1] = {raw[t][c]};
            if (limit[t] < kTile) clear_invisible(v, vexp, limit[t], lg);
            const float vs = scale_of(vexp, vref);
            x = codes_to_f16(v[0][0], v[0][1], vs);
            y = codes_to_f16(v[0][2], v[0][3], vs);
          }
          uint8_t *to = slot + t * IW * L::TILE + f * kConvBytes;
          *reinterpret_cast<u32x4 *>(to) = x;
          *reinterpret_cast<u32x4 *>(to + kFragBytes) = y;
        }
      }
    };
    for (int k = 0; k < n_block; ++k) {
      if (k > 0) load_block<T, DH>(blk, p, b, kvh, g0 + IW * k, ln, lg);
      block |= block_tile<T, DH, NQ>(st, far, blk, p, g0 + IW * k, qf, row_pos, lg);
    }
    load(0);  // not ahead of the block: registers
    convert(0);
    load(1);
#pragma unroll 1
    for (int step = 0; step < steps; ++step) {
      __syncthreads();
      int now[TPS];
      const int units_of = vref;
#pragma unroll
      for (int t = 0; t < TPS; ++t) now[t] = limit[t];
      convert(step + 1);
      load(step + 2);
      raise_vref(st, units_of);
      const uint8_t *slot = smem + (step % 2) * L::STEP + iw * L::TILE;
      // a last step's missing tile: zeros of an empty buffer, none of them visible
      if (TPS * step < np) shared_tiles<DH, NQ, TPS>(st, far, slot, IW * L::TILE, qf, now, p.scale_log2, lane);
    }
    __syncthreads();  // the tiles have been read
  } else {
    // Step s: every wave's s-th tiles, all from the ring. A wave fetches its share of the
    // tiles that it works on with the other row waves (whole fragments, straight into LDS),
    // and for itself the tiles' exponents; one barrier a step publishes step s and frees
    // the slot of step s - 1, which step s - 1 + NB takes. Codes, as fp32 elements are four
    // times as many bytes and their matrix instructions cost far more than conversions.
    constexpr int NB = L::NB, TPS = L::TPS, LPW = (2 * KS + RW - 1) / RW;
    const int steps = (g_end - chunk * p.chunk_tiles + IW * TPS - 1) / (IW * TPS);  // of every wave
    uint64_t visible = 0;  // of the tiles of the last NB issued steps, 8 bits each
    auto issue = [&](int s) {
#pragma unroll
      for (int t = 0; t < TPS; ++t) {
        const int i = TPS * s + t, at = (s % NB) * TPS + t;
        visible <<= 8;
        if (i < n_block || i >= n) continue;
        size_t off, eoff;
        visible |= locate(i, off, eoff);
        const auto rk = buffer_of(p.k_layer + off, kTile * DH), rv = buffer_of(p.v_layer + off, kTile * DH);
        uint8_t *slot = smem + (at * IW + iw) * L::TILE;
#pragma unroll
        for (int c = 0; c < LPW; ++c) {
          const int f = (rw * LPW + c) % (2 * KS);  // the last wave's may come twice
          const bool key = f < KS;
          dma16<kNonTemporal>(key ? rk : rv, key ? lane_k : lane_v, 256 * (key ? f : f - KS), slot + f * kFragBytes);
        }
        if (lane < 2)
          __builtin_amdgcn_global_load_lds(
              (__attribute__((address_space(1))) void *)(lane == 0 ? p.k_exp + eoff : p.v_exp + eoff),
              (__attribute__((address_space(3))) void *)(smem + L::EXPS + (at * kWavesQ8 + wave) * 8), 4, 0, 0);
      }
    };
    // steps of block tiles need no ring: they are done while its first loads are under way
    for (int s = 0; s < NB - 1; ++s) issue(s);
    for (int s = 0; s < n_block; ++s) {
      if (s > 0) load_block<T, DH>(blk, p, b, kvh, g0 + IW * s, ln, lg);
      block |= block_tile<T, DH, NQ>(st, far, blk, p, g0 + IW * s, qf, row_pos, lg);
    }
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
      // tiles that may still be under way: those of the later steps
      wait_tiles<LPW + 1>(min(n, TPS * (s + NB - 1)) - TPS * (s + 1));
      __syncthreads();
      issue(s + NB - 1);
#pragma unroll
      for (int t = 0; t < TPS; ++t) {
        const int i = TPS * s + t, at = (s % NB) * TPS + t;
        if (i < n_block || i >= n) continue;
        const uint8_t *slot = smem + (at * IW + iw) * L::TILE + 16 * lane;
        Raw<DH> x;
#pragma unroll
        for (int k = 0; k < KS; ++k) x.k[k] = *reinterpret_cast<const u32x4 *>(slot + k * kFragBytes);
#pragma unroll
        for (int k = 0; k < KS; ++k) x.v[k] = *reinterpret_cast<const u32x4 *>(slot + (KS + k) * kFragBytes);
        const u32x2 e = *reinterpret_cast<const u32x2 *>(smem + L::EXPS + (at * kWavesQ8 + wave) * 8);
        x.ke = e[0];
        x.ve = e[1];
        prefix_tile<T, DH, NQ>(st, far, x, qf, static_cast<int>(visible >> (8 * (TPS * NB - 1 - t)) & 255), p.scale_log2, ln, lg);
      }
    }
    __syncthreads();  // the ring has been read
  }

  // far references, or values of small scales alone: the wave by itself, one tile after the other
  const bool low = sizeof(T) == 2 && !(block & kHasLarge);
  const bool again = far != 0 || (low && st.vref == kQ8MinExp && n_block > 0 && n > n_block);
  if (again) {
    clear(kLowest, low ? kLowUnit : kQ8MinExp);
    for (int k = 0; k < n_block; ++k) {
      load_block<T, DH>(blk, p, b, kvh, g0 + IW * k, ln, lg);
      block |= block_tile<T, DH, NQ, true>(st, far, blk, p, g0 + IW * k, qf, row_pos, lg);
    }
    window = load_window(0);
#pragma unroll 1
    for (int i = n_block; i < n; ++i) {
      Raw<DH> t;
      const int visible = load(i, t);
      prefix_tile<T, DH, NQ, true>(st, far, t, qf, visible, p.scale_log2, ln, lg);
    }
  }
  // From here on l and o are the plain ones, unnormalised, without shifts but kSlack.
  constexpr float kShift = sizeof(T) == 2 ? kProbShift : 0.f;
  float m[NQ];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    m[qt] = again ? (st.neg[qt] == kLowest ? kNegInf : st.neg[qt] * p.scale_log2)
            : st.neg[qt] == kNoRef ? kNegInf : kShift - st.neg[qt];
    st.l[qt] = group_sum(st.l[qt]);
    if constexpr (sizeof(T) == 2) {
      st.l[qt] *= 0x1p-15f;
      static_assert(kProbShift + kSlack == 15.f, "the shift that is taken back");
#pragma unroll
      for (int dt = 0; dt < DH / 16; ++dt)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          st.o[qt][dt][v] = __builtin_amdgcn_ldexpf(st.o[qt][dt][v], st.vref - 15);
    }
  }
  if (block & kHasLate) {
    float *probs = reinterpret_cast<float *>(smem + L::PROBS + wave * L::PROB_STRIDE);
    for (int k = 0; k < n_block; ++k)
      late_values<T, DH, NQ>(st, again, m, p, b, kvh, g0 + IW * k, qf, row_pos, probs, ln, lg);
  }
  uint8_t *rec = p.ws + (static_cast<size_t>(unit) * p.nsplit + chunk) * p.piece_stride;
  if constexpr (IW == 1) {  // a row's result is one wave's
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      const int row = row0 + 16 * qt + ln;
      if (row >= p.rows) continue;  // a row's four lanes together
      if (nsb > 1) write_record_row<T, DH>(rec, p.rows, row, lg, st.o[qt], m[qt], st.l[qt]);
      else write_output_row<T, DH>(p, b, kvh, row, lg, st.o[qt], m[qt], st.l[qt]);
    }
    return;
  }
  // Merge of the waves' results: every row's maxima and sums first, then, one
  // 16-row tile at a time, the outputs scaled to the common maximum.
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    float amax = 0.f;
    if (sizeof(T) == 2 && nsb > 1) {
#pragma unroll
      for (int dt = 0; dt < DH / 16; ++dt)
#pragma unroll
        for (int v = 0; v < 4; ++v) amax = fmaxf(amax, fabsf(st.o[qt][dt][v]));
      amax = group_max(amax);
    }
    if (lg == 0) {
      sm[wave][16 * qt + ln] = m[qt];
      sl[wave][16 * qt + ln] = st.l[qt];
      sa[wave][16 * qt + ln] = amax;
    }
  }
  __syncthreads();
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    float mx = kNegInf;
#pragma unroll
    for (int k = 0; k < IW; ++k) mx = fmaxf(mx, sm[k * RW + rw][16 * qt + ln]);
    // no visible position in the whole chunk (an unreadable page): outputs are 0
    const float ref = mx == kNegInf ? 0.f : mx;
    const float sc = __builtin_amdgcn_exp2f(m[qt] - ref);
    if (qt > 0) __syncthreads();  // the previous row tile has been summed
    // tile 2 k + i of a lane holds dims 32 k + 8 g + 2 v + i
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const f32x4 x = st.o[qt][2 * k] * sc, y = st.o[qt][2 * k + 1] * sc;
      float *dst = &part[wave][ln * RS + 32 * k + 8 * lg];
      *reinterpret_cast<f32x4 *>(dst) = f32x4{x[0], y[0], x[1], y[1]};
      *reinterpret_cast<f32x4 *>(dst + 4) = f32x4{x[2], y[2], x[3], y[3]};
    }
    __syncthreads();
    constexpr int CG = DH / 4;
    for (int item = threadIdx.x; item < RW * 16 * CG; item += 64 * kWavesQ8) {
      const int wr = item / (16 * CG), r = item / CG % 16, c = 4 * (item % CG);
      const int row = rg * (16 * NQ * RW) + wr * (16 * NQ) + 16 * qt + r;
      if (row >= p.rows) continue;
      float m2 = kNegInf;
#pragma unroll
      for (int k = 0; k < IW; ++k) m2 = fmaxf(m2, sm[k * RW + wr][16 * qt + r]);
      const float ref2 = m2 == kNegInf ? 0.f : m2;
      float den = 0.f, bound = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < IW; ++k) {
        const int src = k * RW + wr;
        const float sck = __builtin_amdgcn_exp2f(sm[src][16 * qt + r] - ref2);
        den += sck * sl[src][16 * qt + r];
        bound += sck * sa[src][16 * qt + r];
        o += *reinterpret_cast<const f32x4 *>(&part[src][r * RS + c]);
      }
      if (nsb > 1) {
        write_piece_item<T, DH>(rec, p.rows, row, c, o, m2, den, bound);
        continue;
      }
      const int pos = row / p.group, h = kvh * p.group + row % p.group;
      store_out4(static_cast<T *>(p.out) + ((static_cast<size_t>(b) * p.w + pos) * p.hq + h) * DH + c,
                 o * (1.f / den));
      if (p.lse && c == 0)
        p.lse[(static_cast<size_t>(b) * p.hq + h) * p.w + pos] =
            (m2 + log2f(den * kFromSlack)) * 0.69314718055994530942f;
    }
  }
}

// Merge of the chunks of a unit: a lane per (row, 4 columns), every fourth record per wave,
// the waves' results through LDS. A wave's first kEagerQ8 records are loaded at once,
// together with the prefix length, so that up to 32 chunks cost one round trip (30 of them,
// merged one by one past the eighth, took 11 us longer).
constexpr int kEagerQ8 = 8;

template <typename T, int DH>
__global__ __launch_bounds__(64 * kWavesQ8) void attn_q8_combine_kernel(AttnQ8Params p) {
  constexpr int CG = DH / 4, RB = rec_elem_bytes(sizeof(T));
  typedef typename RecVec<T>::type Ov;
  __shared__ float sm[kWavesQ8][64], sl[kWavesQ8][64];
  __shared__ f32x4 so[kWavesQ8][64];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int unit = blockIdx.x, b = unit / p.hkv, kvh = unit % p.hkv;
  const int item = min(static_cast<int>(blockIdx.y) * 64 + lane, p.rows * CG - 1);  // the last may repeat
  const int row = item / CG, c = 4 * (item % CG);
  const size_t stride = static_cast<size_t>(p.piece_stride);
  const uint8_t *rec = p.ws + static_cast<size_t>(unit) * p.nsplit * stride;
  const uint8_t *orow = rec + (row * DH + c) * RB, *mrow = rec + p.rows * DH * RB + row * 16;
  const int s_raw = p.prefix_len[b];
  float mx = kNegInf, den = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  int ns = p.nsplit;
  for (int k0 = wave; k0 < ns; k0 += kWavesQ8 * kEagerQ8) {
    f32x4 meta[kEagerQ8];
    Ov ov[kEagerQ8];
#pragma unroll
    for (int k = 0; k < kEagerQ8; ++k) {
      const int r = k0 + kWavesQ8 * k;
      if (r < ns) {
        meta[k] = *reinterpret_cast<const f32x4 *>(mrow + r * stride);
        ov[k] = *reinterpret_cast<const Ov *>(orow + r * stride);
      }
    }
    if (k0 == wave) {  // chunks of this sequence
      bool bad;
      const int S = clamp_prefix(s_raw, p.max_pages, &bad);
      const int ntile = (p.w + kTile - 1) / kTile + (S + kTile - 1) / kTile;
      ns = (ntile + p.chunk_tiles - 1) / p.chunk_tiles;
    }
    float most = mx;
#pragma unroll
    for (int k = 0; k < kEagerQ8; ++k) most = k0 + kWavesQ8 * k < ns ? fmaxf(most, meta[k][0]) : most;
    const float ref = most == kNegInf ? 0.f : most;  // nothing visible in any of them
    const float a = exp2f(mx - ref);
    mx = most;
    den *= a;
    o *= a;
#pragma unroll
    for (int k = 0; k < kEagerQ8; ++k) {
      if (k0 + kWavesQ8 * k < ns) {
        const float sc = exp2f(meta[k][0] - ref), wt = sc * meta[k][2];
        den += sc * meta[k][1];
#pragma unroll
        for (int v = 0; v < 4; ++v) o[v] += wt * static_cast<float>(ov[k][v]);
      }
    }
  }
  sm[wave][lane] = mx;
  sl[wave][lane] = den;
  so[wave][lane] = o;
  __syncthreads();
  // one chunk: the attention kernel wrote the output
  const int mine = blockIdx.y * 64 + lane;
  bool bad;
  const int S = clamp_prefix(s_raw, p.max_pages, &bad);
  const int ntile = (p.w + kTile - 1) / kTile + (S + kTile - 1) / kTile;
  if (wave > 0 || ntile <= p.chunk_tiles || mine >= p.rows * CG) return;
#pragma unroll
  for (int k = 1; k < kWavesQ8; ++k) mx = fmaxf(mx, sm[k][lane]);
  // the first chunk holds the block's diagonal, so mx is finite
  den = 0.f;
  o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kWavesQ8; ++k) {
    const float sc = exp2f(sm[k][lane] - mx);
    den += sc * sl[k][lane];
    o += so[k][lane] * sc;
  }
  const int pos = row / p.group, h = kvh * p.group + row % p.group;
  store_out4(static_cast<T *>(p.out) + ((static_cast<size_t>(b) * p.w + pos) * p.hq + h) * DH + c,
             o * (1.f / den));
  if (p.lse && c == 0)
    p.lse[(static_cast<size_t>(b) * p.hq + h) * p.w + pos] = (mx + log2f(den * kFromSlack)) * 0.69314718055994530942f;
}

template <typename T, int DH, int NQ, int RW>
hipError_t launch_shape(const AttnQ8Params &p, hipStream_t s) {
  constexpr int GR = 16 * NQ * RW;
  const int n_rg = (p.rows + GR - 1) / GR;
  const dim3 grid(static_cast<unsigned>(p.batch) * p.hkv * p.nsplit * n_rg);
  return launch_kernel(attn_q8_kernel<T, DH, NQ, RW>, grid, dim3(64 * kWavesQ8), s, p, n_rg);
}

template <typename T, int DH>
hipError_t launch_dh(const AttnQ8Params &p, hipStream_t s) {
  constexpr int ES = sizeof(T);
  const int nq = q8_row_tiles(p.rows, DH, ES), rw = q8_row_waves(p.rows, DH, ES);
  hipError_t e = hipErrorInvalidValue;
  if (nq == 1 && rw == 1) e = launch_shape<T, DH, 1, 1>(p, s);
  if constexpr (ES == 4 && DH == 128) {
    if (rw == 2) e = launch_shape<T, DH, 1, 2>(p, s);
    if (rw == 4) e = launch_shape<T, DH, 1, 4>(p, s);
  } else {
    if (nq == 2 && rw == 1) e = launch_shape<T, DH, 2, 1>(p, s);
    if constexpr (ES == 4 && DH == 96) {
      if (rw == 4) e = launch_shape<T, DH, 1, 4>(p, s);
    } else {
      if (rw == 2) e = launch_shape<T, DH, 2, 2>(p, s);
      if (rw == 4) e = launch_shape<T, DH, 2, 4>(p, s);
    }
  }
  if (e != hipSuccess || p.nsplit == 1) return e;
  const dim3 merge(static_cast<unsigned>(p.batch) * p.hkv, (p.rows * (DH / 4) + 63) / 64);
  return launch_kernel(attn_q8_combine_kernel<T, DH>, merge, dim3(256), s, p);
}

}  // namespace

hipError_t launch_attn_q8(const AttnQ8Params &p, int dtype, int dh, hipStream_t s) {
  if (dtype == DAS_F32) {
    if (dh == 64) return launch_dh<float, 64>(p, s);
    if (dh == 96) return launch_dh<float, 96>(p, s);
    return launch_dh<float, 128>(p, s);
  }
  if (dh == 64) return launch_dh<bf16_t, 64>(p, s);
  if (dh == 96) return launch_dh<bf16_t, 96>(p, s);
  return launch_dh<bf16_t, 128>(p, s);
}

}  // namespace das
