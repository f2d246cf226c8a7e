// Commit of verified block K/V into the 8-bit cache (das_kv_append_q8): the block
// entries that das_kv_append copies are quantised on the way.
//
// A group is 8 tokens of one (plane, layer, KV head): 8 * dh e4m3 codes, one
// contiguous run of the page, and one exponent e (stored as e + 127); a code stands
// for code * 2^e. Fresh groups take the smallest e for which the largest finite
// magnitude is at most 448 * 2^e. A group that already holds tokens of the sequence
// takes the larger of its own and the new tokens' exponent, and when that is not its
// own, its codes are rounded again (exact but for codes that become subnormal). Scales
// are powers of two, so each new code is a single rounding (to nearest even) of its
// value; NaN and infinities become NaN. Places of the group past the last new token
// keep what they held.
//
// One wave per (plane, layer, KV head) of one sequence, four independent waves per
// workgroup, all keys or all values; it goes through its at most 9 groups. Keys: a lane's
// item is 8 dims of one token, items in the order of the page's bytes. Values: a lane holds
// the 8 tokens of two dims, 16 bytes of the page. Bound by the waves' dependent round trips
// and their instructions (bf16 goes into the conversions packed, the largest magnitude is
// taken on the bits): 32 + 32 planes x 4 layers x 55 heads x 8 tokens 17 us, 6 planes x 4 x
// 55 x 32 sequences x 0-32 tokens 60-63 us (3.2 TB/s); from fp32 19 and 83 us (3.9 TB/s). Measured and not kept: the loads of one
// or two groups ahead (22 and 29 us on the first, 81 and 108 on the second: more registers
// and instructions for groups that most waves do not have), a wave per group (22, 110).

#include "mfma_tile.h"
#include "q8_internal.h"

namespace das {
namespace {

constexpr int kWaves = 4;
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, false));
}
// Maximum over the wave, in every lane.
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, dpp<0xB1>(x));   // lanes 1 apart
  x = fmaxf(x, dpp<0x4E>(x));   // 2 apart
  x = fmaxf(x, dpp<0x141>(x));  // mirrored in 8
  x = fmaxf(x, dpp<0x140>(x));  // mirrored in 16
  return group_max(x);
}

// |x| where it is finite, else 0.
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < __builtin_huge_valf() ? a : 0.f;
}

// The stored exponent byte of a fresh group whose largest finite magnitude is amax:
// 448 = 1.75 * 2^8.
__device__ __forceinline__ int exponent_byte(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
  return min(max(e, kQ8MinExp), kQ8MaxExp) + 127;
}
__device__ __forceinline__ float exp2_of_byte(int byte) {
  return __uint_as_float(static_cast<uint32_t>(byte) << 23);
}

// x, or where the group has the largest exponent the largest code's value past that.
__device__ __forceinline__ float within(float x, float scale) {
  return finite_abs(x) > 448.f * scale ? copysignf(448.f * scale, x) : x;
}
// Codes of a / scale, b / scale, c / scale, d / scale in a word.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float scale) {
  s16x2 r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s16x2{0, 0}, a, b, scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
// The same of two words of two bf16.
__device__ __forceinline__ uint32_t encode4(uint32_t ab, uint32_t cd, float scale) {
  s16x2 r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(s16x2{0, 0}, __builtin_bit_cast(bf16x2, ab), scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, cd), scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
// Four codes whose group's exponent rose by log2(rise), rounded again.
__device__ __forceinline__ uint32_t requantise(uint32_t w, float rise) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, 1.f, false);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, 1.f, true);
  return encode4(a[0], a[1], b[0], b[1], rise);
}

// What a lane loads of a group: new elements, old codes, the old exponent byte. Keys: its
// items' 8 dims (item 64 i + lane: dims 8 c .. of token j, in the order of the page's
// bytes); values: two dims of 8 tokens.
template <typename T, int DH>
struct Group {
  static constexpr int IT = DH == 64 ? 1 : 2;              // key items of a lane
  static constexpr int W = 8 * sizeof(T) / 4;              // words of 8 elements
  uint32_t w[2 * W];
  uint32_t old[4];
  uint32_t had;
};
// The largest magnitude of N words' elements, as the bits of an fp32.
template <typename T, int N>
__device__ __forceinline__ uint32_t largest(const uint32_t (&w)[N]) {
  if constexpr (sizeof(T) == 4) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m = max(m, w[i] & 0x7fffffffu);
    return m;
  } else {
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    return static_cast<uint32_t>(max(m[0], m[1])) << 16;
  }
}
// The same of the finite ones.
template <typename T, int N>
__device__ __forceinline__ uint32_t largest_finite(const uint32_t (&w)[N]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (sizeof(T) == 4) m = fmaxf(m, finite_abs(__uint_as_float(w[i])));
    else m = fmaxf(m, fmaxf(finite_abs(__uint_as_float(w[i] << 16)), finite_abs(__uint_as_float(w[i] & 0xffff0000u))));
  }
  return __float_as_uint(m);
}

template <typename T, int DH>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 8 : 4)))
void kv_append_q8_kernel(AppendQ8Params p) {
  const int b = blockIdx.y;
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int per_plane = p.layers * p.hkv;
  const int k_units = p.n_k_planes * per_plane, v_units = p.n_v_planes * per_plane;
  const int k_blocks = (k_units + kWaves - 1) / kWaves;
  const bool is_v = static_cast<int>(blockIdx.x) >= k_blocks;
  const int rel = (is_v ? blockIdx.x - k_blocks : blockIdx.x) * kWaves + wave;

  const int S = p.prefix_len[b];
  const int n = p.num_new[b];
  const bool bad = S < 0 || n < 0 || n > p.w_max ||
                   static_cast<long>(S) + n > static_cast<long>(p.max_pages) * kPage;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (bad) report_error(p.dev_error, DAS_DEVERR_COMMIT);
    if (p.len_out) p.len_out[b] = bad ? S : S + n;
  }
  if (bad || n == 0 || rel >= (is_v ? v_units : k_units)) return;

  // n <= 64 new positions span at most two pages
  const int32_t *table = p.block_table + static_cast<size_t>(b) * p.max_pages;
  const int first_page = S / kPage;
  const int pg0 = table[first_page], pg1 = table[(S + n - 1) / kPage];
  const bool ok0 = pg0 >= 0 && pg0 < p.num_pages, ok1 = pg1 >= 0 && pg1 < p.num_pages;
  if (blockIdx.x == 0 && threadIdx.x == 0 && (!ok0 || !ok1))
    report_error(p.dev_error, DAS_DEVERR_PAGE);

  const int plane = rel / per_plane, layer = (rel / p.hkv) % p.layers, h = rel % p.hkv;
  const size_t plane_layer = static_cast<size_t>(plane) * p.layers + layer;
  // source [plane][layer][B][w_max][Hkv][DH]; token t's row at src + t * row_bytes
  const T *src = static_cast<const T *>(is_v ? p.v_new : p.k_new) +
                 ((plane_layer * p.batch + b) * p.w_max * p.hkv + h) * DH;
  const int row_bytes = p.hkv * DH * static_cast<int>(sizeof(T));
  uint8_t *pool = (is_v ? p.v_pool : p.k_pool) + (plane_layer * p.hkv + h) * p.num_pages * kPage * DH;
  uint8_t *exps = (is_v ? p.v_exp : p.k_exp) + (plane_layer * p.num_pages * p.hkv + h) * kQ8GroupsPerPage;
  // Offsets outside this buffer (tokens before the first and after the last new one, lanes
  // without a dim) bring zeros: no lane's load depends on a test.
  const auto rows = buffer_of(src, (n - 1) * row_bytes + DH * static_cast<int>(sizeof(T)));
  using G = Group<T, DH>;
  struct Place {
    uint8_t *codes, *exp;
    int lo, hi;  // new tokens of the group
    bool live;
  };
  auto place = [&](int gbase) {
    // 8 | 64: a group lies in one page
    const bool second = gbase / kPage != first_page;
    const int page = second ? pg1 : pg0, g = gbase % kPage / kQ8Group;
    Place at;
    at.live = gbase < S + n && (second ? ok1 : ok0);
    const size_t used = at.live ? page : 0;
    at.codes = pool + (used * kQ8GroupsPerPage + g) * (kQ8Group * DH);
    at.exp = exps + used * p.hkv * kQ8GroupsPerPage + g;
    at.lo = max(S - gbase, 0);
    at.hi = min(S + n - gbase, kQ8Group);
    return at;
  };
  constexpr uint32_t kOutside = 0x80000000u;
  auto load = [&](int gbase, G &x) {
    const Place at = place(gbase);
    const uint32_t first = static_cast<uint32_t>((gbase - S) * row_bytes);
    x.had = 0;
    x.old[0] = x.old[1] = x.old[2] = x.old[3] = 0;
    if (at.live && at.lo > 0) x.had = *at.exp;
    const bool partial = at.live && (at.lo > 0 || (is_v && at.hi < kQ8Group));  // uniform
    if (!is_v) {
#pragma unroll
      for (int i = 0; i < G::IT; ++i) {
        const int item = i * 64 + lane, c = item / 8, j = 4 * (item % 2) + item % 8 / 2;
        const uint32_t off = item < DH ? first + j * row_bytes + c * 8 * static_cast<int>(sizeof(T)) : kOutside;
#pragma unroll
        for (int q = 0; q < G::W / 4; ++q) {
          const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, off + 16 * q, 0, 0));
#pragma unroll
          for (int z = 0; z < 4; ++z) x.w[i * G::W + 4 * q + z] = v[z];
        }
        if (partial && item < DH) {
          const u32x2 o = *reinterpret_cast<const u32x2 *>(at.codes + 8 * item);
          x.old[2 * i] = o[0], x.old[2 * i + 1] = o[1];
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t off = lane < DH / 2 ? first + j * row_bytes + lane * 2 * static_cast<int>(sizeof(T)) : kOutside;
        if constexpr (sizeof(T) == 2) {
          x.w[j] = __builtin_amdgcn_raw_buffer_load_b32(rows, off, 0, 0);
        } else {
          const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rows, off, 0, 0));
          x.w[2 * j] = v[0], x.w[2 * j + 1] = v[1];
        }
      }
      if (partial && lane < DH / 2) {
        const u32x4 o = *reinterpret_cast<const u32x4 *>(at.codes + 16 * lane);
        x.old[0] = o[0], x.old[1] = o[1], x.old[2] = o[2], x.old[3] = o[3];
      }
    }
  };
  auto store = [&](int gbase, G &x) {
    const Place at = place(gbase);
    if (!at.live) return;  // uniform
    const int lo = at.lo, hi = at.hi;
    // Largest finite magnitude; that some are not finite shows in the largest, and rarely.
    auto of_wave = [&](uint32_t bits) {
      return static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(__float_as_uint(wave_max(__uint_as_float(bits)))));
    };
    if (!is_v && G::IT == 1) {
#pragma unroll
      for (int i = 0; i < G::W; ++i) x.w[G::W + i] = 0;
    }
    const uint32_t mine = largest<T>(x.w);
    uint32_t amax;
    if (__builtin_amdgcn_ballot_w64(mine >= 0x7f800000u) == 0) amax = of_wave(mine);
    else amax = of_wave(largest_finite<T>(x.w));
    const int had = __builtin_amdgcn_readfirstlane(x.had);
    const int byte = max(exponent_byte(__uint_as_float(amax)), had);
    const float scale = exp2_of_byte(byte), rise = exp2_of_byte(min(byte - had, 127) + 127);
    if (byte >= kQ8MaxExp + 127) {  // uniform; codes of the largest numbers end at 448
#pragma unroll
      for (int i = 0; i < 2 * G::W; ++i) {
        if constexpr (sizeof(T) == 4) {
          x.w[i] = __float_as_uint(within(__uint_as_float(x.w[i]), scale));
        } else {  // 448 * 2^119 is a bf16
          const uint32_t l = __float_as_uint(within(__uint_as_float(x.w[i] << 16), scale));
          const uint32_t h = __float_as_uint(within(__uint_as_float(x.w[i] & 0xffff0000u), scale));
          x.w[i] = l >> 16 | (h & 0xffff0000u);
        }
      }
    }
    if (!is_v) {
#pragma unroll
      for (int i = 0; i < G::IT; ++i) {
        const int item = i * 64 + lane, j = 4 * (item % 2) + item % 8 / 2;
        if (item >= DH) continue;
        u32x2 *to = reinterpret_cast<u32x2 *>(at.codes + 8 * item);
        const uint32_t *w = x.w + i * G::W;
        if (j >= lo && j < hi) {
          if constexpr (sizeof(T) == 2) {
            *to = u32x2{encode4(w[0], w[1], scale), encode4(w[2], w[3], scale)};
          } else {
            auto f = [&](int e) { return __uint_as_float(w[e]); };
            *to = u32x2{encode4(f(0), f(1), f(2), f(3), scale), encode4(f(4), f(5), f(6), f(7), scale)};
          }
        } else if (j < lo && byte != had) {
          *to = u32x2{requantise(x.old[2 * i], rise), requantise(x.old[2 * i + 1], rise)};
        }
      }
    } else {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int q = 0; q < 2; ++q) {  // tokens 4 q .. + 3 of dim i
          if constexpr (sizeof(T) == 2) {
            const uint32_t sel = i ? 0x07060302u : 0x05040100u;
            w[2 * i + q] = encode4(__builtin_amdgcn_perm(x.w[4 * q + 1], x.w[4 * q], sel),
                                   __builtin_amdgcn_perm(x.w[4 * q + 3], x.w[4 * q + 2], sel), scale);
          } else {
            auto f = [&](int j) { return __uint_as_float(x.w[2 * (4 * q + j) + i]); };
            w[2 * i + q] = encode4(f(0), f(1), f(2), f(3), scale);
          }
        }
      if (lo > 0 || hi < kQ8Group) {
        // bytes before lo: the old tokens; from hi on: left as they were
        const uint64_t below = lo == 0 ? 0 : ~0ull >> (64 - 8 * lo);
        const uint64_t above = hi == 8 ? 0 : ~0ull << (8 * hi);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t mb = static_cast<uint32_t>(below >> (32 * (k % 2)));
          const uint32_t ma = static_cast<uint32_t>(above >> (32 * (k % 2)));
          const uint32_t kept = byte != had ? requantise(x.old[k], rise) : x.old[k];
          w[k] = (w[k] & ~(mb | ma)) | (kept & mb) | (x.old[k] & ma);
        }
      }
      if (lane < DH / 2) *reinterpret_cast<u32x4 *>(at.codes + 16 * lane) = w;
    }
    if (lane == 0) *at.exp = static_cast<uint8_t>(byte);
  };
#pragma unroll 1
  for (int gbase = S & ~7; gbase < S + n; gbase += kQ8Group) {
    G x;
    load(gbase, x);
    store(gbase, x);
  }
}

template <typename T, int DH>
hipError_t launch_typed(const AppendQ8Params &p, hipStream_t s) {
  const int per_plane = p.layers * p.hkv;
  const int blocks = (p.n_k_planes * per_plane + kWaves - 1) / kWaves +
                     (p.n_v_planes * per_plane + kWaves - 1) / kWaves;
  return launch_kernel(kv_append_q8_kernel<T, DH>, dim3(blocks, p.batch), dim3(64 * kWaves), s, p);
}

}  // namespace

hipError_t launch_kv_append_q8(const AppendQ8Params &p, int dtype, int dh, hipStream_t s) {
  if (dtype == DAS_F32) {
    if (dh == 64) return launch_typed<float, 64>(p, s);
    if (dh == 96) return launch_typed<float, 96>(p, s);
    return launch_typed<float, 128>(p, s);
  }
  if (dh == 64) return launch_typed<bf16_t, 64>(p, s);
  if (dh == 96) return launch_typed<bf16_t, 96>(p, s);
  return launch_typed<bf16_t, 128>(p, s);
}

}  // namespace das
