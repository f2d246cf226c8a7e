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
// workgroup, all keys or all values; it goes through its at most 9 groups, with the
// reads of a group (new rows, its exponent, its old codes where it has any) in one
// round trip. Keys: a lane's item is 8 dims of one token, items in the order of the
// page's bytes. Values: a lane holds the 8 tokens of two dims, 16 bytes of the page.

#include "mfma_tile.h"
#include "q8_internal.h"

namespace das {
namespace {

constexpr int kWaves = 4;
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

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

// Codes of a / scale and b / scale in the low two bytes.
__device__ __forceinline__ uint32_t encode2(float a, float b, float scale) {
  const s16x2 r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s16x2{0, 0}, a, b, scale, false);
  return __builtin_bit_cast(uint32_t, r) & 0xffffu;
}
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float scale) {
  return encode2(a, b, scale) | (encode2(c, d, scale) << 16);
}
// Four codes whose group's exponent rose by log2(rise), rounded again.
__device__ __forceinline__ uint32_t requantise(uint32_t w, float rise) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, 1.f, false);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, 1.f, true);
  return encode4(a[0], a[1], b[0], b[1], rise);
}

// N consecutive elements as floats.
template <int N>
__device__ __forceinline__ void load_row(const float *src, float (&x)[N]) {
  static_assert(N == 2 || N == 8, "sizes in use");
  if constexpr (N == 2) {
    const float2 v = *reinterpret_cast<const float2 *>(src);
    x[0] = v.x, x[1] = v.y;
  } else {
    const float4 a = reinterpret_cast<const float4 *>(src)[0], b = reinterpret_cast<const float4 *>(src)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
}
template <int N>
__device__ __forceinline__ void load_row(const bf16_t *src, float (&x)[N]) {
  uint32_t w[N / 2];
  if constexpr (N == 2) w[0] = *reinterpret_cast<const uint32_t *>(src);
  else {
    const u32x4 v = *reinterpret_cast<const u32x4 *>(src);
    w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
  }
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

template <typename T, int DH>
__global__ __launch_bounds__(64 * kWaves) void kv_append_q8_kernel(AppendQ8Params p) {
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
  // source [plane][layer][B][w_max][Hkv][DH]; token t's row at src + t * hkv * DH
  const T *src = static_cast<const T *>(is_v ? p.v_new : p.k_new) +
                 ((plane_layer * p.batch + b) * p.w_max * p.hkv + h) * DH;
  const size_t row = static_cast<size_t>(p.hkv) * DH;
  uint8_t *pool = (is_v ? p.v_pool : p.k_pool) + (plane_layer * p.hkv + h) * p.num_pages * kPage * DH;
  uint8_t *exps = (is_v ? p.v_exp : p.k_exp) + (plane_layer * p.num_pages * p.hkv + h) * kQ8GroupsPerPage;

  for (int gbase = S & ~7; gbase < S + n; gbase += kQ8Group) {
    // 8 | 64: a group lies in one page
    const bool second = gbase / kPage != first_page;
    if (!(second ? ok1 : ok0)) continue;  // uniform
    const int page = second ? pg1 : pg0, g = gbase % kPage / kQ8Group;
    const int lo = max(S - gbase, 0), hi = min(S + n - gbase, kQ8Group);  // new: lo <= j < hi
    uint8_t *dst = pool + (static_cast<size_t>(page) * kQ8GroupsPerPage + g) * (kQ8Group * DH);
    uint8_t *exp_at = exps + static_cast<size_t>(page) * p.hkv * kQ8GroupsPerPage + g;
    const T *rows = src + static_cast<ptrdiff_t>(gbase - S) * row;  // row j of the group
    const int had = lo > 0 ? *exp_at : 0;
    if (!is_v) {
      constexpr int IT = DH / 64 + (DH % 64 != 0);  // items of a lane
      float x[IT][8];
      u32x2 old[IT];
      float amax = 0.f;
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int item = it * 64 + lane, c = item / 8, j = 4 * (item % 2) + item % 8 / 2;
        const bool live = item < DH;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[it][i] = 0.f;
        old[it] = u32x2{0, 0};
        if (live && j >= lo && j < hi) load_row<8>(rows + j * row + 8 * c, x[it]);
        if (live && j < lo) old[it] = *reinterpret_cast<const u32x2 *>(dst + 8 * item);
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, finite_abs(x[it][i]));
      }
      const int fresh = exponent_byte(__uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(wave_max(amax)))));
      const int byte = max(fresh, had);
      const float scale = exp2_of_byte(byte);
      const float rise = exp2_of_byte(min(byte - had, 127) + 127);
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        const int item = it * 64 + lane, j = 4 * (item % 2) + item % 8 / 2;
        if (item >= DH) continue;
        u32x2 *at = reinterpret_cast<u32x2 *>(dst + 8 * item);
        if (j >= lo && j < hi) {
          if (byte == kQ8MaxExp + 127) {  // the largest finite values pass 448 * 2^119
#pragma unroll
            for (int i = 0; i < 8; ++i)
              x[it][i] = finite_abs(x[it][i]) > 448.f * scale ? copysignf(448.f * scale, x[it][i]) : x[it][i];
          }
          *at = u32x2{encode4(x[it][0], x[it][1], x[it][2], x[it][3], scale),
                      encode4(x[it][4], x[it][5], x[it][6], x[it][7], scale)};
        } else if (j < lo && byte != had) {
          *at = u32x2{requantise(old[it][0], rise), requantise(old[it][1], rise)};
        }
      }
      if (lane == 0) *exp_at = static_cast<uint8_t>(byte);
    } else {
      const bool live = lane < DH / 2;
      float x[8][2];
      u32x4 old = {0, 0, 0, 0};
      float amax = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j][0] = x[j][1] = 0.f;
        if (live && j >= lo && j < hi) load_row<2>(rows + j * row + 2 * lane, x[j]);
      }
      const bool whole = lo == 0 && hi == kQ8Group;
      if (live && !whole) old = *reinterpret_cast<const u32x4 *>(dst + 16 * lane);
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fmaxf(finite_abs(x[j][0]), finite_abs(x[j][1])));
      const int fresh = exponent_byte(__uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(wave_max(amax)))));
      const int byte = max(fresh, had);
      const float scale = exp2_of_byte(byte);
      const float rise = exp2_of_byte(min(byte - had, 127) + 127);
      if (byte == kQ8MaxExp + 127) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            x[j][i] = finite_abs(x[j][i]) > 448.f * scale ? copysignf(448.f * scale, x[j][i]) : x[j][i];
      }
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        w[2 * i] = encode4(x[0][i], x[1][i], x[2][i], x[3][i], scale);
        w[2 * i + 1] = encode4(x[4][i], x[5][i], x[6][i], x[7][i], scale);
      }
      if (!whole) {
        // bytes before lo: the old tokens; from hi on: left as they were
        const uint64_t below = lo == 0 ? 0 : ~0ull >> (64 - 8 * lo);
        const uint64_t above = hi == 8 ? 0 : ~0ull << (8 * hi);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t mb = static_cast<uint32_t>(below >> (32 * (k % 2)));
          const uint32_t ma = static_cast<uint32_t>(above >> (32 * (k % 2)));
          const uint32_t kept = byte != had ? requantise(old[k], rise) : old[k];
          w[k] = (w[k] & ~(mb | ma)) | (kept & mb) | (old[k] & ma);
        }
      }
      if (live) *reinterpret_cast<u32x4 *>(dst + 16 * lane) = w;
      if (lane == 0) *exp_at = static_cast<uint8_t>(byte);
    }
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
