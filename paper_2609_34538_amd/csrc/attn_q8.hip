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

#include "attn_coded.h"

namespace das {
namespace {
// Exponent of a wave's units at first: probabilities of 2^15 in them fit fp32, and the
// smallest codes of the smallest scale, 2^-9 * 2^-126, are 2^-24 of it, fp16's smallest.
constexpr int kLowUnit = -111;

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
// Tile u of the draft block through both products. What its values are: kHasLate, some are
// left to late_values; kHasLarge, some are 2^-40 or more (bf16 calls).
constexpr uint32_t kHasLate = 1, kHasLarge = 2;
template <typename T, int DH, int NQ, bool FAR = false>
__device__ __forceinline__ uint32_t block_tile(Acc<DH, NQ> &st, uint64_t &far, Block<T, DH> &t,
                                               const AttnQ8Params &p, int u, const QFrag<T, DH> (&qf)[NQ],
                                               const int (&row_pos)[NQ], int lg) {
  constexpr int KS = DH / 32;
  f32x4 s[NQ][2];
  block_logits(s, t, qf);
  int cap[NQ];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) cap[qt] = row_pos[qt] - kTile * u;
  const int limits[1] = {p.w - kTile * u};
  softmax_step<DH, NQ, 2, true, FAR, sizeof(T) == 4>(st, far, s, cap, limits, p.scale_log2,
                                                     sizeof(T) == 2 ? kProbShift : 0.f, lg);

  // the largest magnitude's bits tell whether any is late
  const uint32_t most32 = most_value(t);
  const bool any_late = __builtin_amdgcn_ballot_w64(most32 >= kLate<T>) != 0;
  if (any_late) drop_late<T, DH, kLate<T>>(t);
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
      late_values<T, DH, NQ, kLate<T>>(st, again, m, p, b, kvh, g0 + IW * k, qf, row_pos, probs, ln, lg);
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
  merge_waves<T, DH, NQ, RW>(p, st, m, part, sm, sl, sa, rec, nsb, rg, b, kvh, wave, ln, lg);
}

template <typename T, int DH>
__global__ __launch_bounds__(64 * kWavesQ8) void attn_q8_combine_kernel(AttnQ8Params p) {
  combine_chunks<T, DH, kTile>(p);
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
