// Policy attention (Eq. (2)-(3)) over a cache held in 4 bits: e2m1 codes with one
// power-of-two scale per token, KV head and 32 dims (das_attn_q4).
//
// A unit is one (sequence, KV head); its 64-token tiles, the draft block's first, then a
// page each, are cut into chunks of chunk_tiles, one workgroup of four waves each. Up to 32
// query rows (RW == 1) the waves take a chunk's pages in turn, from memory into registers, one
// ahead; with more (RW == 4) each has rows of its own and all four share the conversion of a
// page through LDS. Each wave has its own running maximum, sum and output; with RW == 1 they
// merge through LDS, and where a unit has several chunks these leave records that a second
// kernel merges.
//
// Both products take the key / value tile as the A operand, as in mfma_tile.h:
//   S^T (tokens x rows) = K . Q^T,   O^T (dh x rows) += V^T . P^T
// v_cvt_scalef32_pk_bf16_fp4 makes two bf16 of a byte and applies the scale, which is exact;
// of the scale's register only the exponent field counts, so that one shift of a word of four
// exponent bytes makes it. A byte holds neighbouring dims, which share their scale: for keys
// four bytes are a lane's 8 dims of a token, an operand at once; for values the two dims are
// rows of two O^T tiles, and the conversions of 8 tokens are sorted into two operands by
// eight byte permutations (a byte of two tokens of one dim would need as many
// multiplications by their scales).
// Probabilities of bf16 calls are rounded to bf16 for the cached values (the normaliser sums
// them in fp32), and enter as a bf16 and its remainder for the draft block's. fp32 calls take
// queries, probabilities and the block's elements in three bf16 parts each, which hold all 24
// bits, and sum their products with the codes, exact, in fp32: three times the bf16 matrix
// work, where fp32 instructions would take sixteen times.
//
// Measured (bf16): 32 sequences x 55 heads, dh 96, 4096-8192 tokens: 4 rows 178 us, 6.2 TB/s of
// page bytes, 16 rows 189 us, 5.9, both near what this card's memory gives; 32 rows 224 us, 5.1:
// vector instructions, some 400 a page (204 of them the conversion, 180 the softmax). 192 units of
// 4 rows, 1-8191 tokens, dh 128: 26.6 us, the longest units and the second launch. 32 units of 128
// rows, 32768 tokens, dh 128: 90 us, 760 TFLOP/s, vector and matrix instructions in turn. One
// sequence of 2048 tokens, 55 heads, 8 rows: 9.4 us, two launches and their round trips.
// Measured and not kept: pages through a ring of three in LDS in place of registers (226 -> 235
// us, 28.8 -> 32); the sum of the rounded probabilities by the matrix unit (226 -> 222 us, and
// a less exact log-sum-exp); no maximum unless a sum overflows (spills, 453 us); a page in two
// halves at dh 96 (the same; at dh 128 with two row tiles it is what keeps them in registers).

#include <type_traits>

#include "attn_coded.h"
#include "q4_internal.h"

namespace das {
namespace {

constexpr int kTokens = kPage;    // of a tile
constexpr float kShift = -kSlack; // probabilities relative to the reference plus kSlack: at most 1
constexpr uint32_t kInf16 = 0x7f80u, kInf32 = 0x7f800000u;
template <typename T>
constexpr uint32_t kLate4 = sizeof(T) == 2 ? kInf16 : kInf32;  // block values added late: what is not finite

// bf16 operands that make up an element of T.
template <typename T>
constexpr int kParts = sizeof(T) == 2 ? 1 : 3;

// The Q operand of a 16-row tile.
template <typename T, int DH>
struct QParts {
  u32x4 x[DH / 32][kParts<T>];
};

// The upper 16 bits of two words: bf16s by truncation.
__device__ __forceinline__ uint32_t upper(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
}
__device__ __forceinline__ float truncated(float a) { return __uint_as_float(__float_as_uint(a) & 0xffff0000u); }
// Eight fp32 as three bf16 each, by truncation: 8 bits a part, exact.
// KEYS: an infinity is in the first part alone; of a NaN the second is one, whatever its upper
// bits are. QUERIES: parts that would be 0 are 2^-40 of the element instead, which no fp32 sum
// notices, so that the products of an infinite key with them are infinities and not NaN (but with
// a query of 0, or under 2^-93).
enum Split { FINITE, KEYS, QUERIES };
template <Split KIND>
__device__ __forceinline__ void split3(const float (&a)[8], u32x4 (&part)[3]) {
  float x[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) part[0][j] = upper(a[2 * j], a[2 * j + 1]);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    x[j] = a[j] - truncated(a[j]);
    if (KIND == KEYS) x[j] = fabsf(a[j]) == __builtin_huge_valf() ? 0.f : x[j];
    if (KIND == QUERIES) x[j] = x[j] == 0.f ? a[j] * 0x1p-40f : x[j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) part[1][j] = upper(x[2 * j], x[2 * j + 1]);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    x[j] -= truncated(x[j]);
    if (KIND == QUERIES) x[j] = x[j] == 0.f ? a[j] * 0x1p-40f : x[j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) part[2][j] = upper(x[2 * j], x[2 * j + 1]);
}
__device__ __forceinline__ void eight_floats(const u32x4 &lo, const u32x4 &hi, float (&a)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] = __uint_as_float(lo[j]), a[4 + j] = __uint_as_float(hi[j]);
}

// A scale from byte `i` of a word of exponent bytes; the bits beside the exponent field do
// not count.
__device__ __forceinline__ float scale_of(uint32_t w, int i) {
  return __uint_as_float(i == 0 ? w << 23 : i == 1 ? w << 15 : i == 2 ? w << 7 : w >> 1);
}
template <int I>
__device__ __forceinline__ uint32_t two_codes(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, I));
}
// The K operand of a word: 8 dims of a token.
__device__ __forceinline__ u32x4 key_operand(uint32_t w, float scale) {
  return u32x4{two_codes<0>(w, scale), two_codes<1>(w, scale), two_codes<2>(w, scale), two_codes<3>(w, scale)};
}
// The V operands of dims 32 k + 2 n and + 1: the words of tokens 0-3 and 4-7, their exponents.
__device__ __forceinline__ void value_operands(uint32_t w0, uint32_t w1, uint32_t e0, uint32_t e1, u32x4 &even,
                                               u32x4 &odd) {
  uint32_t c[8];
  c[0] = two_codes<0>(w0, scale_of(e0, 0)), c[1] = two_codes<1>(w0, scale_of(e0, 1));
  c[2] = two_codes<2>(w0, scale_of(e0, 2)), c[3] = two_codes<3>(w0, scale_of(e0, 3));
  c[4] = two_codes<0>(w1, scale_of(e1, 0)), c[5] = two_codes<1>(w1, scale_of(e1, 1));
  c[6] = two_codes<2>(w1, scale_of(e1, 2)), c[7] = two_codes<3>(w1, scale_of(e1, 3));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    even[j] = __builtin_amdgcn_perm(c[2 * j + 1], c[2 * j], 0x05040100);
    odd[j] = __builtin_amdgcn_perm(c[2 * j + 1], c[2 * j], 0x07060302);
  }
}
// The exponents of 8 values tokens with those of tokens from `seen` on cleared: whatever the
// page holds there is finite then, and its probability 0.
__device__ __forceinline__ void clear_unseen(uint32_t &e0, uint32_t &e1, int seen) {
  e0 &= seen >= 4 ? ~0u : (1u << 8 * max(seen, 0)) - 1;
  e1 &= seen >= 8 ? ~0u : seen <= 4 ? 0u : (1u << 8 * (seen - 4)) - 1;
}

// A page as loaded: pieces of keys and values, the exponent bytes of the lane's key tokens
// (word (2 t + e) * dh / 32 + s in words of four) and of its value tokens.
template <int DH>
struct Page {
  u32x4 k[DH / 32], v[DH / 32], ve[DH / 32];
  uint32_t ke[DH / 32];
};

// The P operands of a 32-token tile, from its probabilities.
template <typename T>
__device__ __forceinline__ void prob_operands(const f32x4 &a, const f32x4 &b, u32x4 (&pf)[kParts<T>]) {
  if constexpr (sizeof(T) == 2) {
    pf[0] = u32x4{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3])};
  } else {
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    split3<FINITE>(x, pf);
  }
}

// E / 2 tiles of 32 tokens of a page, from tile T0 on, through both products.
// `limit`: visible tokens of the page; keys_taken is called when t's keys are.
template <typename T, int DH, int NQ, int T0, int E, bool FAR, typename Then>
__device__ __forceinline__ void prefix_tiles(Acc<DH, NQ> &st, uint64_t &far, Page<DH> &t,
                                             const QParts<T, DH> (&qf)[NQ], int limit, float scale, int lg,
                                             Then keys_taken) {
  constexpr int KS = DH / 32;
  f32x4 s[NQ][E];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
    for (int e = 0; e < E; ++e) s[qt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const int at = (2 * T0 + e) * KS + k;
      const u32x4 a = key_operand(t.k[at / 4][at % 4], scale_of(t.ke[at / 4], at % 4));
#pragma unroll
      for (int i = kParts<T> - 1; i >= 0; --i)
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) s[qt][e] = mfma16x16x32(a, qf[qt].x[k][i], s[qt][e]);
    }
  keys_taken();
  const int none[NQ] = {};
  int limits[E / 2];
#pragma unroll
  for (int j = 0; j < E / 2; ++j) limits[j] = limit - kTile * (T0 + j);
  softmax_step<DH, NQ, E, false, FAR, false>(st, far, s, none, limits, scale, kShift, lg);
#pragma unroll
  for (int j = 0; j < E / 2; ++j) {
    u32x4 pf[NQ][kParts<T>];
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) prob_operands<T>(s[qt][2 * j], s[qt][2 * j + 1], pf[qt]);
    const int w = 2 * (T0 + j);
    if (limits[j] < kTile) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t e0 = t.ve[k][w], e1 = t.ve[k][w + 1];
        clear_unseen(e0, e1, limits[j] - 8 * lg);
        t.ve[k][w] = e0, t.ve[k][w + 1] = e1;
      }
    }
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      u32x4 even, odd;
      value_operands(t.v[k][w], t.v[k][w + 1], t.ve[k][w], t.ve[k][w + 1], even, odd);
#pragma unroll
      for (int i = kParts<T> - 1; i >= 0; --i)
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) {
          st.o[qt][2 * k] = mfma16x16x32(even, pf[qt][i], st.o[qt][2 * k]);
          st.o[qt][2 * k + 1] = mfma16x16x32(odd, pf[qt][i], st.o[qt][2 * k + 1]);
        }
    }
  }
}

// N tiles of 32 tokens from their converted operands in LDS: per tile 2 * dh / 32 of keys
// (index 2 s + e), then as many of values (2 k + i), a lane's 16 bytes each.
template <typename T, int DH, int NQ, int N>
__device__ __forceinline__ void shared_tiles4(Acc<DH, NQ> &st, uint64_t &far, const uint8_t *tiles,
                                              const QParts<T, DH> (&qf)[NQ], const int (&limit)[N], float scale,
                                              int lane) {
  constexpr int KS = DH / 32;
  auto part = [&](int t, int f) {
    return *reinterpret_cast<const u32x4 *>(tiles + (t * 4 * KS + f) * kFragBytes + 16 * lane);
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
        const u32x4 a = part(t, 2 * k + e);
#pragma unroll
        for (int i = kParts<T> - 1; i >= 0; --i)
#pragma unroll
          for (int qt = 0; qt < NQ; ++qt) s[qt][2 * t + e] = mfma16x16x32(a, qf[qt].x[k][i], s[qt][2 * t + e]);
      }
  const int none[NQ] = {};
  softmax_step<DH, NQ, 2 * N, false, false, false>(st, far, s, none, limit, scale, kShift, lane >> 4);
#pragma unroll
  for (int t = 0; t < N; ++t) {
    u32x4 pf[NQ][kParts<T>];
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) prob_operands<T>(s[qt][2 * t], s[qt][2 * t + 1], pf[qt]);
#pragma unroll
    for (int k = 0; k < 2 * KS; ++k) {
      const u32x4 a = part(t, 2 * KS + k);
#pragma unroll
      for (int i = kParts<T> - 1; i >= 0; --i)
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) st.o[qt][k] = mfma16x16x32(a, pf[qt][i], st.o[qt][k]);
    }
  }
}

// Logits of a tile of the draft block. fp32: the eight largest products of the parts, which
// are below 2^-7 and 2^-14 of the element; the ninth is below 2^-28.
template <typename T, int DH, int NQ>
__device__ __forceinline__ void block_logits(f32x4 (&s)[NQ][2], const Block<T, DH> &t, const QParts<T, DH> (&qf)[NQ]) {
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) s[qt][0] = s[qt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < DH / 32; ++k)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) s[qt][e] = mfma16x16x32(t.k[e][k][0], qf[qt].x[k][0], s[qt][e]);
      } else {
        float x[8];
        u32x4 a[3];
        eight_floats(t.k[e][k][0], t.k[e][k][1], x);
        split3<KEYS>(x, a);
#pragma unroll
        for (int sum = 3; sum >= 0; --sum)
#pragma unroll
          for (int i = max(sum - 2, 0); i <= min(sum, 2); ++i)
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) s[qt][e] = mfma16x16x32(a[i], qf[qt].x[k][sum - i], s[qt][e]);
      }
    }
}

// Tile u of the draft block through both products; whether some of its values are left to
// late_values.
template <typename T, int DH, int NQ, bool FAR>
__device__ __forceinline__ bool block_tile4(Acc<DH, NQ> &st, uint64_t &far, Block<T, DH> &t, const AttnQ8Params &p,
                                            int u, const QParts<T, DH> (&qf)[NQ], const int (&row_pos)[NQ], int lg) {
  constexpr int KS = DH / 32;
  f32x4 s[NQ][2];
  block_logits(s, t, qf);
  int cap[NQ];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) cap[qt] = row_pos[qt] - kTile * u;
  const int limits[1] = {p.w - kTile * u};
  softmax_step<DH, NQ, 2, true, FAR, false>(st, far, s, cap, limits, p.scale_log2, kShift, lg);
  const bool any_late = __builtin_amdgcn_ballot_w64(most_value(t) >= kLate4<T>) != 0;
  if (any_late) drop_late<T, DH, kLate4<T>>(t);
  if constexpr (sizeof(T) == 2) {
    u32x4 hi[NQ], lo[NQ];
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a = s[qt][j / 2][2 * (j % 2)], c = s[qt][j / 2][2 * (j % 2) + 1];
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
    u32x4 pf[NQ][3];
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) prob_operands<T>(s[qt][0], s[qt][1], pf[qt]);
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[8];
        u32x4 a[3];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(t.v[k][j][h]);
        split3<FINITE>(x, a);
#pragma unroll
        for (int sum = 3; sum >= 0; --sum)
#pragma unroll
          for (int i = max(sum - 2, 0); i <= min(sum, 2); ++i)
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt)
              st.o[qt][2 * k + h] = mfma16x16x32(a[i], pf[qt][sum - i], st.o[qt][2 * k + h]);
      }
  }
  return any_late;
}

// Shared memory of a workgroup.
// RW == 1: the merge area of one row tile, before that a block tile's probabilities for its
// late values.
// RW == 4: two converted pages; afterwards, in the second one's place, the probabilities.
template <int DH, int NQ, int RW>
struct Lds4 {
  static constexpr int RS = DH + 4;  // row stride of the merge area (floats)
  static constexpr int STEP = RW == 1 ? 0 : 8 * (DH / 32) * kFragBytes;
  static constexpr int MERGE = RW == 4 ? 0 : kWavesQ8 * 16 * RS * 4;
  static constexpr int PROBS = STEP;
  static constexpr int PROB_STRIDE = RW == 1 ? 16 * RS * 4 : 16 * NQ * kTile * 4;
  static constexpr int HELD = 2 * STEP;
  static constexpr int BYTES = HELD > MERGE ? HELD : MERGE;
  static_assert(PROB_STRIDE >= 16 * NQ * kTile * 4 && PROBS + kWavesQ8 * PROB_STRIDE <= BYTES,
                "a tile's probabilities fit");
};

template <typename T, int DH, int NQ, int RW>
__global__ __launch_bounds__(64 * kWavesQ8) __attribute__((amdgpu_waves_per_eu(2)))
void attn_q4_kernel(AttnQ8Params p, int n_rg) {
  using L = Lds4<DH, NQ, RW>;
  constexpr int KS = DH / 32;
  static_assert(RW == 1 || RW == kWavesQ8, "waves with rows of their own: none or all");
  constexpr int STRIDE = RW == 1 ? kWavesQ8 : 1;  // from a wave's tile to its next
  __shared__ __attribute__((aligned(16))) uint8_t smem[L::BYTES];
  __shared__ float sm[kWavesQ8][16 * NQ], sl[kWavesQ8][16 * NQ], sa[kWavesQ8][16 * NQ];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ln = lane & 15, lg = lane >> 4;
  const int rw = RW == 1 ? 0 : wave;
  // every unit's first chunk comes before any second one
  const int units = p.batch * p.hkv;
  const int rg = blockIdx.x % n_rg, grp = blockIdx.x / n_rg;
  const int unit = grp % units, chunk = grp / units;
  const int b = unit / p.hkv, kvh = unit % p.hkv;
  const int row0 = rg * (16 * NQ * RW) + rw * (16 * NQ);
  const int g0 = chunk * p.chunk_tiles + (RW == 1 ? wave : 0);  // this wave's first tile of the unit

  const int s_raw = p.prefix_len[b];
  QParts<T, DH> qf[NQ];
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
    for (int k = 0; k < KS; ++k) {
      const u32x4 *src = reinterpret_cast<const u32x4 *>(qrow + 32 * k + 8 * lg);
      if constexpr (sizeof(T) == 2) {
        qf[qt].x[k][0] = src[0];
      } else {
        float x[8];
        eight_floats(src[0], src[1], x);
        split3<QUERIES>(x, qf[qt].x[k]);
      }
    }
  }
  // page ids: lane i holds the page of this wave's (window + i)-th tile
  auto load_window = [&](int first) {
    const int pg = g0 + STRIDE * (first + lane) - 1;
    return pg >= 0 && pg < p.max_pages ? p.block_table[static_cast<size_t>(b) * p.max_pages + pg] : 0;
  };
  int window = load_window(0);
  // The draft block is tile 0 of chunk 0, one or two tiles of 32 tokens.
  Block<T, DH> blk;
  const int n_block = g0 == 0 ? 1 : 0;
  const int u_end = n_block ? min((p.w + kTile - 1) / kTile, 2) : 0;
  const bool has_block = u_end > 0;
  // not ahead where its registers are those of the first page
  constexpr bool AHEAD = sizeof(T) == 2 && (DH < 128 || NQ == 1);
  if (AHEAD && has_block) load_block<T, DH>(blk, p, b, kvh, 0, ln, lg);

  bool bad;
  const int S = clamp_prefix(s_raw, p.max_pages, &bad);
  if (bad && kvh == 0 && rg == 0 && chunk == 0 && threadIdx.x == 0)
    report_error(p.dev_error, DAS_DEVERR_PREFIX);
  const int ntile = 1 + (S + kTokens - 1) / kTokens;
  const int nsb = (ntile + p.chunk_tiles - 1) / p.chunk_tiles;  // chunks of this unit
  if (chunk >= nsb) return;
  const int g_end = min(ntile, (chunk + 1) * p.chunk_tiles);
  const int n = g_end > g0 ? (g_end - g0 + STRIDE - 1) / STRIDE : 0;  // this wave's tiles

  Acc<DH, NQ> st;
  uint64_t far = 0;  // lanes of rows that have met a far reference
  auto clear = [&](float neg) {
    st.vref = 0;
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      st.neg[qt] = neg;
      st.l[qt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DH / 16; ++dt) st.o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  clear(kNoRef);

  // Which page the wave's i-th tile is, and the number of its visible tokens. An out-of-range
  // page id is reported and read as page 0 (its tokens are masked out).
  auto locate = [&](int i, size_t &page_head) {
    if (i >= 64 && i % 64 == 0) {
      window = load_window(i);
      wait_vmcnt<0>();  // here: otherwise every use of it waits for all loads under way
    }
    const int page_raw = __builtin_amdgcn_readlane(window, i & 63);
    const bool ok = page_raw >= 0 && page_raw < p.num_pages;
    if (!ok && i < n) report_error(p.dev_error, DAS_DEVERR_PAGE);
    page_head = static_cast<size_t>(kvh) * p.num_pages + (ok ? page_raw : 0);
    return ok ? min(kTokens, S - kTokens * (g0 + STRIDE * i - 1)) : 0;
  };

  // The keys and the values of the wave's i-th tile into registers. Past the last tile the loads
  // go to empty buffers: they are always issued, so that the compiler can count them, and waits
  // for some leave the others under way.
  auto load_keys = [&](int i, size_t at, Page<DH> &t) {
    const auto rk = buffer_of(p.k_layer + at * q4_page_bytes(DH), i < n ? q4_page_bytes(DH) : 0);
    const auto rke = buffer_of(p.k_exp + at * q4_page_exps(DH), i < n ? q4_page_exps(DH) : 0);
    if constexpr (KS == 2) {
      const u32x2 e = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rke, ln * 4 * KS, 0, kCached));
      t.ke[0] = e[0], t.ke[1] = e[1];
    } else if constexpr (KS == 3) {
      typedef uint32_t u32x3 __attribute__((ext_vector_type(3)));
      const u32x3 e = __builtin_bit_cast(u32x3, __builtin_amdgcn_raw_buffer_load_b96(rke, ln * 4 * KS, 0, kCached));
      t.ke[0] = e[0], t.ke[1] = e[1], t.ke[2] = e[2];
    } else {
      const u32x4 e = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rke, ln * 4 * KS, 0, kCached));
      t.ke[0] = e[0], t.ke[1] = e[1], t.ke[2] = e[2], t.ke[3] = e[3];
    }
#pragma unroll
    for (int k = 0; k < KS; ++k)
      t.k[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, 16 * lane, 1024 * k, kNonTemporal));
  };
  auto load_values = [&](int i, size_t at, Page<DH> &t) {
    const auto rv = buffer_of(p.v_layer + at * q4_page_bytes(DH), i < n ? q4_page_bytes(DH) : 0);
    const auto rve = buffer_of(p.v_exp + at * q4_page_exps(DH), i < n ? q4_page_exps(DH) : 0);
#pragma unroll
    for (int k = 0; k < KS; ++k)
      t.ve[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rve, lg * 16 * KS, 16 * k, kCached));
#pragma unroll
    for (int k = 0; k < KS; ++k)
      t.v[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, 16 * lane, 1024 * k, kNonTemporal));
  };
  auto load = [&](int i, Page<DH> &t) {
    size_t at;
    const int visible = locate(i, at);
    load_keys(i, at, t);
    load_values(i, at, t);
    return visible;
  };

  bool late = false;  // whether the block has values that are added late
  auto work_block = [&](auto far_form) {
    for (int u = 0; u < u_end; ++u) {
      if (!AHEAD || decltype(far_form)::value || u > 0) load_block<T, DH>(blk, p, b, kvh, u, ln, lg);
      late |= block_tile4<T, DH, NQ, decltype(far_form)::value>(st, far, blk, p, u, qf, row_pos, lg);
    }
  };
  if constexpr (RW == 1) {
    if (!AHEAD && has_block) work_block(std::false_type{});
    constexpr bool WHOLE = sizeof(T) == 2 && (DH < 128 || NQ == 1);  // a page's logits fit the registers
    if constexpr (WHOLE && (DH > 64 || NQ == 2)) {
      // The next page's keys are asked for when the page's have been taken, its values likewise.
      // Two pages in turn, as below, are slower (192 units of 4 rows, dh 128: 28.7 against 26.6
      // us; 32 rows, dh 96: 224.7 against 223.4; at dh 64 97 against 95 with 32 rows, but 79
      // against 83 with 16), three waves a SIMD in the registers that are free without the block
      // ahead slower too (28.7; 243).
      Page<DH> t;
      int limit = load(n_block, t);
      if (AHEAD && has_block) work_block(std::false_type{});
#pragma unroll 1
      for (int i = n_block; i < n; ++i) {
        size_t at;
        int next = 0;
        prefix_tiles<T, DH, NQ, 0, 4, false>(st, far, t, qf, limit, p.scale_log2, lg, [&] {
          next = locate(i + 1, at);
          load_keys(i + 1, at, t);
        });
        load_values(i + 1, at, t);
        limit = next;
      }
    } else {
      // Two pages in flight (with one page's registers as above fp32 calls take 78 us for 75, 32
      // rows of dh 128 179 for 170).
      Page<DH> ta, tb;
      int i = n_block;
      int la = load(i, ta);
      if (AHEAD && has_block) work_block(std::false_type{});
      int lb = load(i + 1, tb);
      auto work = [&](Page<DH> &t, int limit) {
        if constexpr (WHOLE) {
          prefix_tiles<T, DH, NQ, 0, 4, false>(st, far, t, qf, limit, p.scale_log2, lg, [] {});
        } else {
          prefix_tiles<T, DH, NQ, 0, 2, false>(st, far, t, qf, limit, p.scale_log2, lg, [] {});
          prefix_tiles<T, DH, NQ, 1, 2, false>(st, far, t, qf, limit, p.scale_log2, lg, [] {});
        }
      };
      for (; i < n; i += 2) {
        work(ta, la);
        la = load(i + 2, ta);
        if (i + 1 < n) work(tb, lb);
        lb = load(i + 3, tb);
      }
    }
  } else {
    // Each wave brings its pieces of a page into registers, a step ahead, and writes them
    // converted to LDS, from where all multiply. One barrier a step publishes page s and frees
    // the place of page s - 1, which page s + 1 takes. Pieces: values to the first dh / 32
    // waves; keys to the others, at dh 128 one to each.
    constexpr int NK = KS == 3 ? 3 : 1;
    const bool has_v = wave < KS;
    const bool has_k = KS == 4 || (KS == 3 ? wave == 3 : wave >= 2);
    const int k_first = KS == 4 ? wave : KS == 3 ? 0 : max(wave - 2, 0);
    u32x4 rawk[NK], rawv, ve;
    uint32_t ke[NK];
    int limit = 0, ahead = 0;
    // always issued, what is not the wave's and past the last page from empty buffers
    auto fetch = [&](int i) {
      size_t at;
      const int visible = locate(i, at);
      ahead = i < n ? visible : 0;
      const bool lk = i < n && has_k, lv = i < n && has_v;
      const auto rk = buffer_of(p.k_layer + at * q4_page_bytes(DH), lk ? q4_page_bytes(DH) : 0);
      const auto rv = buffer_of(p.v_layer + at * q4_page_bytes(DH), lv ? q4_page_bytes(DH) : 0);
      const auto rke = buffer_of(p.k_exp + at * q4_page_exps(DH), lk ? q4_page_exps(DH) : 0);
      const auto rve = buffer_of(p.v_exp + at * q4_page_exps(DH), lv ? q4_page_exps(DH) : 0);
      const int vp = min(wave, KS - 1);
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        ke[c] = __builtin_amdgcn_raw_buffer_load_b32(rke, ln * 4 * KS, 4 * (k_first + c), kCached);
        rawk[c] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rk, 16 * lane,
                                                                                 1024 * (k_first + c), kNonTemporal));
      }
      ve = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rve, lg * 16 * KS, 16 * vp, kCached));
      rawv = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, 16 * lane, 1024 * vp, kNonTemporal));
    };
    auto convert = [&](int step) {
      uint8_t *slot = smem + (step % 2) * L::STEP + 16 * lane;
      limit = ahead;
      if (has_k) {
#pragma unroll
        for (int c = 0; c < NK; ++c)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int at = 4 * (k_first + c) + j, te = at / KS, s = at % KS;  // te: 2 t + e
            *reinterpret_cast<u32x4 *>(slot + (te / 2 * 4 * KS + 2 * s + te % 2) * kFragBytes) =
                key_operand(rawk[c][j], scale_of(ke[c], j));
          }
      }
      if (has_v) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          uint32_t e0 = ve[2 * t], e1 = ve[2 * t + 1];
          if (limit < kTokens) clear_unseen(e0, e1, limit - kTile * t - 8 * lg);
          u32x4 even, odd;
          value_operands(rawv[2 * t], rawv[2 * t + 1], e0, e1, even, odd);
          uint8_t *to = slot + (t * 4 * KS + 2 * KS + 2 * wave) * kFragBytes;
          *reinterpret_cast<u32x4 *>(to) = even;
          *reinterpret_cast<u32x4 *>(to + kFragBytes) = odd;
        }
      }
    };
    if (has_block) work_block(std::false_type{});
    const int np = n - n_block;
    fetch(n_block);  // not ahead of the block: registers
    convert(0);
    fetch(n_block + 1);
#pragma unroll 1
    for (int step = 0; step < np; ++step) {
      __syncthreads();
      const int now = limit;
      convert(step + 1);
      fetch(n_block + step + 2);
      const uint8_t *slot = smem + (step % 2) * L::STEP;
      const int limits[2] = {now, now - kTile};
      shared_tiles4<T, DH, NQ, 2>(st, far, slot, qf, limits, p.scale_log2, lane);
    }
    __syncthreads();  // the pages have been read
  }

  // far references: the wave by itself, one tile after the other
  const bool again = far != 0;
  if (again) {
    clear(kLowest);
    work_block(std::true_type{});
    window = load_window(0);
#pragma unroll 1
    for (int i = n_block; i < n; ++i) {
      Page<DH> t;
      const int visible = load(i, t);
      prefix_tiles<T, DH, NQ, 0, 2, true>(st, far, t, qf, visible, p.scale_log2, lg, [] {});
      prefix_tiles<T, DH, NQ, 1, 2, true>(st, far, t, qf, visible, p.scale_log2, lg, [] {});
    }
  }
  float m[NQ];
#pragma unroll
  for (int qt = 0; qt < NQ; ++qt) {
    m[qt] = again ? (st.neg[qt] == kLowest ? kNegInf : st.neg[qt] * p.scale_log2)
            : st.neg[qt] == kNoRef ? kNegInf : kShift - st.neg[qt];
    st.l[qt] = group_sum(st.l[qt]);
  }
  if (late) {
    float *probs = reinterpret_cast<float *>(smem + L::PROBS + wave * L::PROB_STRIDE);
    for (int u = 0; u < u_end; ++u)
      late_values<T, DH, NQ, kLate4<T>>(st, again, m, p, b, kvh, u, qf, row_pos, probs, ln, lg);
  }
  uint8_t *rec = p.ws + (static_cast<size_t>(unit) * p.nsplit + chunk) * p.piece_stride;
  if constexpr (RW == 4) {  // a row's result is one wave's
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
      const int row = row0 + 16 * qt + ln;
      if (row >= p.rows) continue;  // a row's four lanes together
      if (nsb > 1) write_record_row<T, DH>(rec, p.rows, row, lg, st.o[qt], m[qt], st.l[qt]);
      else write_output_row<T, DH>(p, b, kvh, row, lg, st.o[qt], m[qt], st.l[qt]);
    }
  } else {
    merge_waves<T, DH, NQ, RW>(p, st, m, reinterpret_cast<float(*)[16 * L::RS]>(smem), sm, sl, sa, rec, nsb, rg, b,
                               kvh, wave, ln, lg);
  }
}

template <typename T, int DH>
__global__ __launch_bounds__(64 * kWavesQ8) void attn_q4_combine_kernel(AttnQ8Params p) {
  combine_chunks<T, DH, kTokens>(p);
}

template <typename T, int DH, int NQ, int RW>
hipError_t launch_shape(const AttnQ8Params &p, hipStream_t s) {
  constexpr int GR = 16 * NQ * RW;
  const int n_rg = (p.rows + GR - 1) / GR;
  const dim3 grid(static_cast<unsigned>(p.batch) * p.hkv * p.nsplit * n_rg);
  return launch_kernel(attn_q4_kernel<T, DH, NQ, RW>, grid, dim3(64 * kWavesQ8), s, p, n_rg);
}

template <typename T, int DH>
hipError_t launch_dh(const AttnQ8Params &p, hipStream_t s) {
  constexpr int ES = sizeof(T);
  const int nq = q4_row_tiles(p.rows, ES), rw = q4_row_waves(p.rows);
  hipError_t e = hipErrorInvalidValue;
  if (nq == 1 && rw == 1) e = launch_shape<T, DH, 1, 1>(p, s);
  if (nq == 1 && rw == 4) e = launch_shape<T, DH, 1, 4>(p, s);
  if constexpr (ES == 2) {
    if (nq == 2 && rw == 1) e = launch_shape<T, DH, 2, 1>(p, s);
    if (nq == 2 && rw == 4) e = launch_shape<T, DH, 2, 4>(p, s);
  }
  if (e != hipSuccess || p.nsplit == 1) return e;
  const dim3 merge(static_cast<unsigned>(p.batch) * p.hkv, (p.rows * (DH / 4) + 63) / 64);
  return launch_kernel(attn_q4_combine_kernel<T, DH>, merge, dim3(256), s, p);
}

}  // namespace

hipError_t launch_attn_q4(const AttnQ8Params &p, int dtype, int dh, hipStream_t s) {
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
