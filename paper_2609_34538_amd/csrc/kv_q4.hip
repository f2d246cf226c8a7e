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
// A wave's unit is the call's positions of one page, of one (plane, layer, KV head) and
// sequence, in groups of 8 tokens. A lane's item is 8 dims of a token, 16 bytes of a bf16
// row; the four lanes of a block agree on its exponent by two DPP steps. Keys: an item is one
// word of the page. Values: an item is four bytes, 16 apart, beside those of the group's
// other tokens, so groups go through LDS for 8-byte accesses; a commit into part of a group
// stores its bytes one by one, which leaves the others as they were.

#include "mfma_tile.h"
#include "q4_internal.h"

namespace das {
namespace {

constexpr int kWaves = 4;
constexpr int kGroup = 8;  // tokens
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

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
// The maximum over the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t u) {
  u = max(u, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, u, 0xB1, 0xf, 0xf, false)));
  return max(u, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, u, 0x4E, 0xf, 0xf, false)));
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

// Where the word of keys of token t of a page, dims 8 c .. + 7, lies, and its exponent.
template <int DH>
__device__ __forceinline__ void key_place(int t, int c, int &word, int &exp) {
  constexpr int KS = DH / 32;
  const int n = t % 32 / 8 * 4 + t % 4, at = (t / 32 * 2 + t / 4 % 2) * KS + c / 4;
  word = at / 4 * 1024 + (c % 4 * 16 + n) * 16 + at % 4 * 4;
  exp = n * 4 * KS + at;
}
// Where the 8 tokens of group j of dims 2 pair, + 1 lie, and the exponent of token t, block s.
__device__ __forceinline__ int value_place(int j, int pair) {
  return pair / 16 * 1024 + (j % 4 * 16 + pair % 16) * 16 + j / 4 * 8;
}
template <int DH>
__device__ __forceinline__ int value_exp(int t, int s) {
  return t % 32 / 8 * 16 * (DH / 32) + s * 16 + t / 32 * 8 + t % 8;
}

// READ: from the cache into the rows; else from the rows into the cache.
template <typename T, int DH, bool READ>
__global__ __launch_bounds__(64 * kWaves) void kv_q4_kernel(TokensQ4Params p) {
  constexpr int CH = DH / 8, IT = (kGroup * CH + 63) / 64;  // items of a token, a lane's of a group
  // a group's value codes: [8 tokens][dh / 2] on the way back, [dh / 2][8 tokens] into the cache
  __shared__ __attribute__((aligned(8))) uint8_t codes[kWaves][kGroup * DH / 2];
  const int b = blockIdx.y;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int per_plane = p.layers * p.hkv;
  const int k_units = p.n_k_planes * per_plane, v_units = p.n_v_planes * per_plane;
  const int k_blocks = (k_units + kWaves - 1) / kWaves;
  const bool is_v = static_cast<int>(blockIdx.x) >= k_blocks;
  const int rel = (is_v ? blockIdx.x - k_blocks : blockIdx.x) * kWaves + wave;
  const bool first_wg = blockIdx.x == 0 && blockIdx.z == 0;

  const int S = p.first[b];
  const int n = p.num[b];
  const long end = static_cast<long>(S) + n;
  bool bad = S < 0 || n < 0 || n > p.w_max || end > static_cast<long>(p.max_pages) * kPage;
  if (READ) bad |= end > p.limit[b];
  if (first_wg && threadIdx.x == 0) {
    if (bad) report_error(p.dev_error, READ ? DAS_DEVERR_PREFIX : DAS_DEVERR_COMMIT);
    if (!READ && p.len_out) p.len_out[b] = bad ? S : S + n;
  }
  if (bad || n == 0) return;
  const int32_t *table = p.block_table + static_cast<size_t>(b) * p.max_pages;
  const int first_page = S / kPage, last_page = (S + n - 1) / kPage;
  // every page id once, whoever writes there
  if (blockIdx.x == 0) {
    for (int pg = first_page + blockIdx.z + gridDim.z * threadIdx.x; pg <= last_page; pg += gridDim.z * blockDim.x) {
      const int id = table[pg];
      if (id < 0 || id >= p.num_pages) report_error(p.dev_error, DAS_DEVERR_PAGE);
    }
  }
  if (rel >= (is_v ? v_units : k_units)) return;

  const int plane = rel / per_plane, layer = (rel / p.hkv) % p.layers, h = rel % p.hkv;
  const size_t plane_layer = static_cast<size_t>(plane) * p.layers + layer;
  // rows [plane][layer][B][w_max][Hkv][DH]
  T *rows = static_cast<T *>(is_v ? p.v_new : p.k_new) +
            ((plane_layer * p.batch + b) * p.w_max * p.hkv + h) * DH;
  const size_t row = static_cast<size_t>(p.hkv) * DH;
  const size_t head = (plane_layer * p.hkv + h) * p.num_pages;
  uint8_t *mine = codes[wave];

  for (int pg = first_page + blockIdx.z; pg <= last_page; pg += gridDim.z) {
    const int id = table[pg];
    if (id < 0 || id >= p.num_pages) continue;  // uniform
    uint8_t *page = (is_v ? p.v_pool : p.k_pool) + (head + id) * q4_page_bytes(DH);
    uint8_t *exps = (is_v ? p.v_exp : p.k_exp) + (head + id) * q4_page_exps(DH);
    const int lo = max(S - pg * kPage, 0), hi = static_cast<int>(min(end - static_cast<long>(pg) * kPage, 64L));
#pragma unroll 1
    for (int j = lo / kGroup; j < (hi + kGroup - 1) / kGroup; ++j) {
      if (READ && is_v) {
        __builtin_amdgcn_wave_barrier();
        if (lane < DH / 2) {
          const uint64_t c = *reinterpret_cast<const uint64_t *>(page + value_place(j, lane));
#pragma unroll
          for (int i = 0; i < kGroup; ++i) mine[i * (DH / 2) + lane] = static_cast<uint8_t>(c >> (8 * i));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int item = it * 64 + lane, i = item / CH, c = item % CH, t = j * kGroup + i;
        const bool live = t >= lo && t < hi && i < kGroup;
        Eight<T> *at = reinterpret_cast<Eight<T> *>(rows + static_cast<size_t>(pg * kPage + t - S) * row + 8 * c);
        if constexpr (READ) {
          if (!live) continue;
          int word = 0, exp;
          if (is_v) exp = value_exp<DH>(t, c / 4);
          else key_place<DH>(t, c, word, exp);
          const uint32_t w = is_v ? *reinterpret_cast<const uint32_t *>(mine + i * (DH / 2) + 4 * c)
                                  : *reinterpret_cast<const uint32_t *>(page + word);
          const Eight<T> x = decode<T>(w, __uint_as_float(static_cast<uint32_t>(exps[exp]) << 23));
          __builtin_memcpy(__builtin_assume_aligned(at, 16), &x, sizeof(x));
        } else {
          Eight<T> x = {};
          if (live) __builtin_memcpy(&x, __builtin_assume_aligned(at, 16), sizeof(x));
          const uint32_t byte = exponent_byte(quad_max(largest<T>(x)));
          const uint32_t w = encode<T>(x, __uint_as_float(byte << 23));
          if (is_v) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (i < kGroup) mine[(4 * c + k) * kGroup + i] = static_cast<uint8_t>(w >> (8 * k));
            if (live && c % 4 == 0) exps[value_exp<DH>(t, c / 4)] = static_cast<uint8_t>(byte);
          } else if (live) {
            int word, exp;
            key_place<DH>(t, c, word, exp);
            *reinterpret_cast<uint32_t *>(page + word) = w;
            if (c % 4 == 0) exps[exp] = static_cast<uint8_t>(byte);
          }
        }
      }
      if (!READ && is_v) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (lane < DH / 2) {
          uint8_t *to = page + value_place(j, lane);
          const uint64_t c = *reinterpret_cast<const uint64_t *>(mine + lane * kGroup);
          if (lo <= j * kGroup && hi >= (j + 1) * kGroup) {
            *reinterpret_cast<uint64_t *>(to) = c;
          } else {
            for (int i = max(lo - j * kGroup, 0); i < min(hi - j * kGroup, kGroup); ++i)
              to[i] = static_cast<uint8_t>(c >> (8 * i));
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    }
  }
}

template <typename T, int DH, bool READ>
hipError_t launch_typed(const TokensQ4Params &p, hipStream_t s) {
  const int per_plane = p.layers * p.hkv;
  const int blocks = (p.n_k_planes * per_plane + kWaves - 1) / kWaves +
                     (p.n_v_planes * per_plane + kWaves - 1) / kWaves;
  // pages that w_max positions can touch
  const int pages = (p.w_max + kPage - 2) / kPage + 1;
  return launch_kernel(kv_q4_kernel<T, DH, READ>, dim3(blocks, p.batch, READ ? min(pages, 65535) : 1),
                       dim3(64 * kWaves), s, p);
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
