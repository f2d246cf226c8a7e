// What the attention kernels over caches of codes (8 and 4 bits) share: the softmax step,
// the draft block's tiles, the merge of a workgroup's waves and of a unit's chunks.
// Layouts of both products as in mfma_tile.h; a 32-token tile's S^T rows are tokens 8 g + 4 e
// + v, so that a lane's logits are those of its own 8 tokens, and O^T tiles 2 k and 2 k + 1
// hold dims 32 k + 8 g + 2 v and + 1.
#pragma once

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
constexpr float kBySlack = 0x1p-6f, kFromSlack = 0x1p6f;  // 2^-kSlack, 2^kSlack
constexpr float kNoRef = 3e38f;  // in place of shift - reference: nothing seen yet
// A reference past this (in base-2 units) is far: the rounding of reference * scale would be
// a factor of its own in every probability, past fp16's range from 2^27 on. A wave that has
// met one goes through its tiles again, in a form that takes the references off the logits
// (5 x 32 heads x 4 x 29 rows x 2005 tokens: 43.6 us without, 44.6 so, 46.7 with that form
// in the steps themselves).
constexpr float kFar = 0x1p20f;
constexpr float kLowest = -3.402823466e38f;  // as a reference of that form: nothing seen yet
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
// A word of block values (two bf16 or one fp32) with those of them replaced by 0.
template <typename T, uint32_t LATE>
__device__ __forceinline__ uint32_t without_late(uint32_t w) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t lo = (w & 0x7fffu) >= LATE ? 0u : w & 0xffffu;
    return (w >> 16 & 0x7fffu) >= LATE ? lo : lo | (w & 0xffff0000u);
  } else {
    return (w & 0x7fffffffu) >= LATE ? 0u : w;
  }
}
template <typename T, uint32_t LATE>
__device__ __forceinline__ bool is_late(float x) {
  return (__float_as_uint(x) & 0x7fffffffu) >= (sizeof(T) == 2 ? LATE << 16 : LATE);
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

// The largest magnitude of a tile's values in a lane, as their type's bits.
template <typename T, int DH>
__device__ __forceinline__ uint32_t most_value(const Block<T, DH> &t) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 most = {0, 0};
  uint32_t most32 = 0;
#pragma unroll
  for (int k = 0; k < DH / 32; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (sizeof(T) == 2)
        most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, t.v[k][j][0] & 0x7fff7fffu));
      else
        most32 = max(most32, max(t.v[k][j][0] & 0x7fffffffu, t.v[k][j][1] & 0x7fffffffu));
    }
  if constexpr (sizeof(T) == 2) most32 = max(most[0], most[1]);
  return most32;
}
template <typename T, int DH, uint32_t LATE>
__device__ __forceinline__ void drop_late(Block<T, DH> &t) {
#pragma unroll
  for (int k = 0; k < DH / 32; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int h = 0; h < Block<T, DH>::W; ++h) t.v[k][j][h] = without_late<T, LATE>(t.v[k][j][h]);
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
// The late values of tile u of the draft block, for the rows that see them (in a product
// 0 * NaN would reach the rows that do not). Of st, sums are plain here and m their
// references in base-2 units; probs: the wave's place in LDS for the tile's probabilities,
// [row tile][row][token].
template <typename T, int DH, int NQ, uint32_t LATE, typename Q>
__device__ __forceinline__ void late_values(Acc<DH, NQ> &st, bool far, const float (&m)[NQ], const AttnQ8Params &p,
                                            int b, int kvh, int u, const Q (&qf)[NQ],
                                            const int (&row_pos)[NQ], float *probs, int ln, int lg) {
  Block<T, DH> t;
  load_block<T, DH>(t, p, b, kvh, u, ln, lg);
  f32x4 s[NQ][2];
  block_logits(s, t, qf);
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
          if (is_late<T, LATE>(x) && kTile * u + i <= row_pos[qt]) st.o[qt][2 * k + j % 2][j / 2] += pt * x;
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
// Merge of the waves' results: every row's maxima and sums first, then, one
// 16-row tile at a time, the outputs scaled to the common maximum. Waves k * RW + rw, k <
// 4 / RW, hold rows 16 * NQ * (RW * rg + rw) and up; part is the merge area in LDS (rows of
// DH + 4), sm, sl and sa are the rows' maxima, sums and largest outputs, per wave. nsb > 1:
// into the record, else into the output.
template <typename T, int DH, int NQ, int RW>
__device__ __forceinline__ void merge_waves(const AttnQ8Params &p, const Acc<DH, NQ> &st, const float (&m)[NQ],
                                            float (*part)[16 * (DH + 4)], float (*sm)[16 * NQ],
                                            float (*sl)[16 * NQ], float (*sa)[16 * NQ], uint8_t *rec, int nsb,
                                            int rg, int b, int kvh, int wave, int ln, int lg) {
  constexpr int IW = kWavesQ8 / RW, RS = DH + 4, KS = DH / 32;
  const int rw = wave % RW;
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
// merged one by one past the eighth, took 11 us longer). TOKENS: of a tile.
constexpr int kEagerQ8 = 8;

template <typename T, int DH, int TOKENS>
__device__ __forceinline__ void combine_chunks(const AttnQ8Params &p) {
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
      const int ntile = (p.w + TOKENS - 1) / TOKENS + (S + TOKENS - 1) / TOKENS;
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
  const int ntile = (p.w + TOKENS - 1) / TOKENS + (S + TOKENS - 1) / TOKENS;
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

}  // namespace
}  // namespace das
