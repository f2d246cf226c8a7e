// Commit of verified block K/V into the 4-bit cache (das_kv_append_q4), and cached elements
// back in the call's type (das_kv_read_q4).
//
// 32 neighbouring dims of a token share an exponent e (stored as e + 127), the smallest for
// which the largest magnitude is at most 7 * 2^e, so that no element is further from its code
// than half the distance of the two largest codes, 4 and 6. A code is x * 2^-e rounded to the
// nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to an even code: one rounding an element, in
// v_cvt_scalef32_pk_fp4_*. Tokens do not share anything, so a commit touches no earlier one
// and its result does not depend on how tokens come together. Blocks with a NaN or an
// infinity get the exponent byte 255, which reads as NaN.
//
// A wave's unit is a quad of neighbouring tokens of one (plane, layer) and sequence, and 12
// blocks of 32 dims along the heads, four a step: lane 16 a + 4 c + q has dims 8 c .. + 7 of
// block a of token q, 16 bytes of a bf16 row, so that a step takes 256 bytes of each row and
// the wave 768. The four lanes of a token's block agree on its exponent by two rotations within
// 16 lanes. Keys: a lane's 8 codes are one word of the page. Values: the four lanes c hold words
// of four tokens; a transposition of bytes in each quad of lanes (four broadcasts and three byte
// permutations, its own inverse) makes of them the words of the page, four tokens of two dims.
// A commit to part of a quad stores its bytes one by one, which leaves the others as they were.
//
// 2005 tokens of 24 planes and layers, 55 heads, dh 96 (135 MB in, 508 MB out) come back in 206 us,
// 3.1 TB/s, where a copy of large arrays reaches 4.9 (131 us; fp32, 1.15 GB, 357 us for 235). Without
// its loads the kernel takes 105 us, without its stores 87, which is nearly the whole together:
// they do not overlap, and neither is at the memory's rate, since a load takes 4-byte words of the
// pages' 16-byte pieces, whose others other quads and heads come for. Commits of 0-32 tokens of 32
// sequences (130 MB in, 34 MB out) take 66 us, what lies in part of a 128-byte line of the page
// going out as several writes (63 MB by the counters); of 8 tokens of 64 planes x 4 layers x 55
// heads 13 us, the launch and three dependent round trips.
// Measured and not kept: a wave along the tokens of one head, 192 bytes of each row (213, 67
// and 16 us), 2, 4, 6 and 8 steps a wave (216, 211, 222, 257 us), all steps in a loop (220 us).

#include "mfma_tile.h"
#include "q4_internal.h"

namespace das {
namespace {

constexpr int kWaves = 4;
constexpr int kSteps = kQ4Steps;  // of a wave, whose loads are issued together
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// 8 elements as loaded.
template <typename T>
struct Eight {
  static constexpr int W = 8 * sizeof(T) / 4;
  uint32_t w[W];
};

// The exponent byte of a block whose largest magnitude has these fp32 bits: 7 = 1.75 * 2^2.
__device__ __forceinline__ uint32_t exponent_byte(uint32_t u) {
  if (u >= 0x7f800000u) return kQ4NanByte;
  const int e = static_cast<int>(u >> 23) - 127 - 2 + ((u & 0x7fffffu) > 0x600000u);
  return min(max(e, kQ4MinExp), kQ4MaxExp) + 127;
}
template <typename T>
__device__ __forceinline__ uint32_t largest(const Eight<T> &x) {
  if constexpr (sizeof(T) == 4) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, x.w[i] & 0x7fffffffu);
    return m;
  } else {
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x.w[i] & 0x7fff7fffu));
    return static_cast<uint32_t>(max(m[0], m[1])) << 16;
  }
}
// The maximum over lanes 4, 8 and 12 apart within 16.
__device__ __forceinline__ uint32_t block_max(uint32_t u) {
  u = max(u, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, u, 0x128, 0xf, 0xf, false)));  // row_ror:8
  return max(u, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, u, 0x124, 0xf, 0xf, false)));
}
// Byte j of lane i's word in a quad becomes byte i of lane j's; q: lane % 4.
__device__ __forceinline__ uint32_t transposed(uint32_t w, int q) {
  const uint32_t a = __builtin_amdgcn_update_dpp(0, w, 0x00, 0xf, 0xf, false);
  const uint32_t b = __builtin_amdgcn_update_dpp(0, w, 0x55, 0xf, 0xf, false);
  const uint32_t c = __builtin_amdgcn_update_dpp(0, w, 0xAA, 0xf, 0xf, false);
  const uint32_t d = __builtin_amdgcn_update_dpp(0, w, 0xFF, 0xf, 0xf, false);
  const uint32_t pick = q | (q + 4) << 8;
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, pick), __builtin_amdgcn_perm(b, a, pick), 0x05040100);
}
// Codes of 8 elements in a word.
template <typename T>
__device__ __forceinline__ uint32_t encode(const Eight<T> &x, float scale) {
  uint32_t c = 0;
  if constexpr (sizeof(T) == 4) {
    auto f = [&](int i) { return __uint_as_float(x.w[i]); };
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(0), f(1), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(2), f(3), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(4), f(5), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f(6), f(7), scale, 3);
  } else {
    auto h = [&](int i) { return __builtin_bit_cast(bf16x2, x.w[i]); };
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, h(0), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, h(1), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, h(2), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, h(3), scale, 3);
  }
  return c;
}
// The elements of a word of codes.
template <typename T>
__device__ __forceinline__ Eight<T> decode(uint32_t c, float scale) {
  Eight<T> x;
  if constexpr (sizeof(T) == 4) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
    const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2);
    const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
    const float f[8] = {a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
#pragma unroll
    for (int i = 0; i < 8; ++i) x.w[i] = __float_as_uint(f[i]);
  } else {
    x.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
    x.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
    x.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
    x.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
  }
  return x;
}

// READ: from the cache into the rows; else from the rows into the cache. grid: (plane, layer)
// and share of the heads, keys first; sequences; groups of four quads, one a wave.
template <typename T, int DH, bool READ>
__global__ __launch_bounds__(64 * kWaves) void kv_q4_kernel(TokensQ4Params p, int shares) {
  constexpr int KS = DH / 32;
  const int b = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int share = blockIdx.x % shares, unit = blockIdx.x / shares;
  const int k_units = p.n_k_planes * p.layers;
  const bool is_v = unit >= k_units;
  const int rel = is_v ? unit - k_units : unit;  // plane * layers + layer

  const int S = p.first[b];
  const int n = p.num[b];
  const long end = static_cast<long>(S) + n;
  bool bad = S < 0 || n < 0 || n > p.w_max || end > static_cast<long>(p.max_pages) * kPage;
  if (READ) bad |= end > p.limit[b];
  if (blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0) {
    if (bad) report_error(p.dev_error, READ ? DAS_DEVERR_PREFIX : DAS_DEVERR_COMMIT);
    if (!READ && p.len_out) p.len_out[b] = bad ? S : S + n;
  }
  if (bad || n == 0) return;
  const int quad_end = (S + n + 3) / 4;
  const int32_t *table = p.block_table + static_cast<size_t>(b) * p.max_pages;
  const int a = lane / 16, c = lane / 4 % 4, q = lane % 4;
  const int blocks = p.hkv * KS, first_block = share * (4 * kSteps) + a;
  const size_t row = static_cast<size_t>(blocks) * 32;
  T *rows = static_cast<T *>(is_v ? p.v_new : p.k_new) + (static_cast<size_t>(rel) * p.batch + b) * p.w_max * row;
  const size_t heads = static_cast<size_t>(rel) * p.hkv * p.num_pages;
  uint8_t *pool = (is_v ? p.v_pool : p.k_pool) + heads * q4_page_bytes(DH);
  uint8_t *exponents = (is_v ? p.v_exp : p.k_exp) + heads * q4_page_exps(DH);
  const uint64_t head_bytes = static_cast<uint64_t>(p.num_pages) * q4_page_bytes(DH);
  const uint64_t head_exps = static_cast<uint64_t>(p.num_pages) * q4_page_exps(DH);

  for (int quad = S / 4 + 4 * blockIdx.z + wave; quad < quad_end; quad += 4 * gridDim.z) {
    const int id = table[quad / 16];
    const int t = 4 * quad + q;
    const bool live = t >= S && t < S + n, whole = 4 * quad >= S && 4 * quad + 4 <= S + n;
    T *line = rows + static_cast<size_t>(live ? t - S : 0) * row + 8 * c;
    Eight<T> x[kSteps];
    if constexpr (!READ) {  // whatever the page
#pragma unroll
      for (int r = 0; r < kSteps; ++r) {
        x[r] = Eight<T>{};
        if (live && first_block + 4 * r < blocks)
          __builtin_memcpy(&x[r], __builtin_assume_aligned(line + 32 * (first_block + 4 * r), 16), sizeof(x[r]));
      }
    }
    if (id < 0 || id >= p.num_pages) {  // uniform
      if (blockIdx.x == 0 && lane == 0) report_error(p.dev_error, DAS_DEVERR_PAGE);
      continue;
    }
    const int half = quad % 16 / 8, g = quad % 8 / 2, e = quad % 2;  // token 32 half + 8 g + 4 e + q of the page
    const int at0 = (2 * half + e) * KS;
    uint8_t *page = pool + static_cast<size_t>(id) * q4_page_bytes(DH) +
                    (is_v ? (16 * g + 4 * c + q) * 16 + 8 * half + 4 * e : (16 * c + 4 * g + q) * 16);
    uint8_t *exps = exponents + static_cast<size_t>(id) * q4_page_exps(DH) +
                    (is_v ? g * 16 * KS + 8 * half + 4 * e + q : (4 * g + q) * 4 * KS + at0);
    // the lane's word of block s of head h, and the exponent
    auto word_of = [&](uint32_t block) {
      const uint32_t h = block / KS, s = block % KS, at = at0 + s;
      return reinterpret_cast<uint32_t *>(page + h * head_bytes + (is_v ? 1024 * s : at / 4 * 1024 + at % 4 * 4));
    };
    auto exp_of = [&](uint32_t block) {
      const uint32_t h = block / KS, s = block % KS;
      return exps + h * head_exps + (is_v ? 16 * s : s);
    };
    if constexpr (READ) {
      uint32_t w[kSteps], ex[kSteps];
#pragma unroll
      for (int r = 0; r < kSteps; ++r) {
        const int block = first_block + 4 * r;
        w[r] = block < blocks ? *word_of(block) : 0;
        ex[r] = block < blocks ? *exp_of(block) : 0;
      }
#pragma unroll
      for (int r = 0; r < kSteps; ++r) {
        const int block = first_block + 4 * r;
        const Eight<T> y = decode<T>(is_v ? transposed(w[r], q) : w[r], __uint_as_float(ex[r] << 23));
        if (live && block < blocks) __builtin_memcpy(__builtin_assume_aligned(line + 32 * block, 16), &y, sizeof(y));
      }
    } else {
#pragma unroll
      for (int r = 0; r < kSteps; ++r) {
        const int block = first_block + 4 * r;
        const bool in = block < blocks;
        const uint32_t byte = exponent_byte(block_max(largest<T>(x[r])));
        const uint32_t w = encode<T>(x[r], __uint_as_float(byte << 23));
        if (is_v) {
          const uint32_t wt = transposed(w, q);
          if (in && whole) {
            *word_of(block) = wt;
          } else if (in) {
            uint8_t *to = reinterpret_cast<uint8_t *>(word_of(block));
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (4 * quad + j >= S && 4 * quad + j < S + n) to[j] = static_cast<uint8_t>(wt >> (8 * j));
          }
        } else if (in && live) {
          *word_of(block) = w;
        }
        if (in && live && c == 0) *exp_of(block) = static_cast<uint8_t>(byte);
      }
    }
  }
}

template <typename T, int DH, bool READ>
hipError_t launch_typed(const TokensQ4Params &p, hipStream_t s) {
  const int64_t units = static_cast<int64_t>(p.n_k_planes + p.n_v_planes) * p.layers;
  // quads that w_max positions can touch, four to a workgroup
  const int groups = ((p.w_max + 2) / 4 + 1 + 3) / 4;
  const int shares = q4_head_shares(p.hkv, DH);
  return launch_kernel(kv_q4_kernel<T, DH, READ>,
                       dim3(static_cast<unsigned>(units * shares), p.batch, groups < 65535 ? groups : 65535),
                       dim3(64 * kWaves), s, p, shares);
}

template <bool READ>
hipError_t launch(const TokensQ4Params &p, int dtype, int dh, hipStream_t s) {
  if (dtype == DAS_F32) {
    if (dh == 64) return launch_typed<float, 64, READ>(p, s);
    if (dh == 96) return launch_typed<float, 96, READ>(p, s);
    return launch_typed<float, 128, READ>(p, s);
  }
  if (dh == 64) return launch_typed<bf16_t, 64, READ>(p, s);
  if (dh == 96) return launch_typed<bf16_t, 96, READ>(p, s);
  return launch_typed<bf16_t, 128, READ>(p, s);
}

}  // namespace

hipError_t launch_kv_append_q4(const TokensQ4Params &p, int dtype, int dh, hipStream_t s) {
  return launch<false>(p, dtype, dh, s);
}
hipError_t launch_kv_read_q4(const TokensQ4Params &p, int dtype, int dh, hipStream_t s) {
  return launch<true>(p, dtype, dh, s);
}

}  // namespace das
