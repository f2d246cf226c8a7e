// Norms of a block's queries and keys for each head and their rotation by position, out of
// a fused projection or separate ones, in one pass (das_qk_rope).
//
//   y = x * weight / sqrt(mean(x^2) + eps),  (y_i, y_j) -> (y_i cos t - y_j sin t, y_j cos t + y_i sin t)
//
// with t = position * inv_freq. One workgroup takes a token's heads, or a share of them. Its
// first threads make the token's cosines and sines, one pair of dims each, in 64 bits (a far
// position's angle has no bits left of its fraction of a turn in 32): reduction to a quarter
// of a turn by two-part pi / 2, then the series. A lane holds 16 dims of a head, both dims of
// its 8 pairs; LPR lanes a head, which add their squares, in 64 bits so that no finite
// element's passes the largest number. The next head's pieces are under way while one is worked
// on.
//
// Bound by memory for batches: 32 x 32 tokens of 165 heads, dh 96, bf16 out of a fused projection
// (65 MB) 14.8-16.1 us, 4.0-4.4 TB/s, where a copy of large arrays reaches 4.9; 8 tokens 3.7-5.2 us,
// the launch and two round trips. A token's heads are shared by workgroups until there are eight a
// compute unit: 64 tokens 4.4 us, with one workgroup each 8.4, 256 tokens 8.2 and 10.6; 1024
// tokens with three each 16.2, six 18.7. Where half of a workgroup or more would be idle, it takes
// several tokens, from four a compute unit on: 17955 tokens of 15 heads, dh 64, 17.0 us, with one
// each 27.8, of 6 heads 9.7 and 27.5; 2048 tokens 4.5 and 5.8; 768 tokens 4.1 and 4.0. Measured and
// not kept: several tokens in several rounds, where a token's last round is half empty (1024
// tokens of 24 heads, dh 128, 5.1 -> 6.3 us, 2048 of 40 heads 11.4 -> 12.9).

#include <algorithm>

#include "mfma_tile.h"
#include "q4_internal.h"

namespace das {
namespace {

constexpr int kThreads = 256;

// cos and sin of t in 64 bits, |t| up to 2^31 (the largest position times a frequency of 1).
__device__ __forceinline__ void turn(double t, float &c, float &s) {
  const double n = __builtin_rint(t * 0.63661977236758134);  // quarters of a turn
  double r = __builtin_fma(-n, 1.5707963267948966, t);        // pi / 2 in two parts
  r = __builtin_fma(-n, 6.123233995736766e-17, r);
  const double z = r * r;
  // series to r^15 and r^16: the rest is below 2^-53 at pi / 4
  double a = -1.0 / 1307674368000.0;
  a = __builtin_fma(a, z, 1.0 / 6227020800.0);
  a = __builtin_fma(a, z, -1.0 / 39916800.0);
  a = __builtin_fma(a, z, 1.0 / 362880.0);
  a = __builtin_fma(a, z, -1.0 / 5040.0);
  a = __builtin_fma(a, z, 1.0 / 120.0);
  a = __builtin_fma(a, z, -1.0 / 6.0);
  const double sn = __builtin_fma(a * z, r, r);
  double b = 1.0 / 20922789888000.0;
  b = __builtin_fma(b, z, -1.0 / 87178291200.0);
  b = __builtin_fma(b, z, 1.0 / 479001600.0);
  b = __builtin_fma(b, z, -1.0 / 3628800.0);
  b = __builtin_fma(b, z, 1.0 / 40320.0);
  b = __builtin_fma(b, z, -1.0 / 720.0);
  b = __builtin_fma(b, z, 1.0 / 24.0);
  b = __builtin_fma(b, z, -0.5);
  const double cs = __builtin_fma(b, z, 1.0);
  const int64_t q = static_cast<int64_t>(n);
  const double x = q & 1 ? sn : cs, y = q & 1 ? cs : sn;
  c = static_cast<float>((q + 1) & 2 ? -x : x);
  s = static_cast<float>(q & 2 ? -y : y);
}

template <int CTRL>
__device__ __forceinline__ double plus_dpp(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<uint32_t>(u), CTRL, 0xf, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<uint32_t>(u >> 32), CTRL, 0xf, 0xf, false);
  return x + __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}

// 1 / sqrt(a) as r * unit, unit a power of two (1 but where r would leave fp32's range): one
// step of Newton's on the estimate for a * 4^-k in [1, 4).
__device__ __forceinline__ float inverse_root(double a, float &unit) {
  unit = 1.f;
  if (!(a < __builtin_huge_val())) return a == a ? 0.f : __builtin_nanf("");
  if (a <= 0.0) return __builtin_huge_valf();
  const int k = (__builtin_amdgcn_frexp_exp(a) - 1) >> 1, near = min(max(k, -60), 60);
  const float m = static_cast<float>(__builtin_amdgcn_ldexp(a, -2 * k));
  float r = __builtin_amdgcn_rsqf(m);
  r = __builtin_fmaf(0.5f * r, __builtin_fmaf(-m * r, r, 1.f), r);
  unit = __builtin_amdgcn_ldexpf(1.f, near - k);
  return __builtin_amdgcn_ldexpf(r, -near);
}

// 8 elements as loaded.
template <typename T>
struct Eight {
  static constexpr int W = 8 * sizeof(T) / 4;
  uint32_t w[W];
};
template <typename T>
__device__ __forceinline__ Eight<T> load8(const T *src) {
  Eight<T> x;
  __builtin_memcpy(&x, __builtin_assume_aligned(src, 16), sizeof(x));
  return x;
}
template <typename T>
__device__ __forceinline__ void floats(const Eight<T> &x, float *f) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (sizeof(T) == 4) f[i] = __uint_as_float(x.w[i]);
    else f[i] = __uint_as_float(i % 2 ? x.w[i / 2] & 0xffff0000u : x.w[i / 2] << 16);
  }
}
template <typename T>
__device__ __forceinline__ void store8(T *dst, const float *f) {
  Eight<T> x;
#pragma unroll
  for (int i = 0; i < Eight<T>::W; ++i) {
    if constexpr (sizeof(T) == 4) {
      x.w[i] = __float_as_uint(f[i]);
    } else {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      const bf16x2 h = {static_cast<__bf16>(f[2 * i]), static_cast<__bf16>(f[2 * i + 1])};
      x.w[i] = __builtin_bit_cast(uint32_t, h);
    }
  }
  __builtin_memcpy(__builtin_assume_aligned(dst, 16), &x, sizeof(x));
}

// PACKED: per_wg tokens a workgroup, one head a slot; else one, a share of its heads.
template <typename T, int DH, bool PACKED>
__global__ __launch_bounds__(kThreads) void qk_rope_kernel(RopeParams p, int per_wg) {
  constexpr int LPR = DH == 64 ? 4 : 8, ROWS = kThreads / LPR;  // lanes of a head, heads at once
  __shared__ float cs[kThreads], sn[kThreads];
  const int heads = p.hq + p.hkv + (p.v ? p.hkv : 0), pairs = p.rotary / 2;
  const int slot = threadIdx.x / LPR;
  const int tokens = p.batch * p.w, token0 = blockIdx.x * per_wg;
  const float per_head = 1.f / static_cast<float>(heads);
  const int lane = threadIdx.x % LPR;
  const bool in_head = lane < DH / 16;
  // the lane's 8-dim pieces; half-split pairs lie rotary / 2 apart, interleaved ones side by side
  const int turned = p.rotary / 16;  // lanes whose dims are rotated
  const bool turns = lane < turned;
  const bool halves = turns && !p.interleaved;
  const int first = halves ? 8 * lane : 16 * lane;
  const int second = halves ? first + p.rotary / 2 : first + 8;

  struct Row {
    Eight<T> a, b, wa, wb;
  };
  const int per = (heads + gridDim.y - 1) / gridDim.y;
  const int begin = PACKED ? slot : blockIdx.y * per + slot;
  const int end = PACKED ? min(per_wg, tokens - token0) * heads : min(heads, static_cast<int>(blockIdx.y + 1) * per);
  // the token of the workgroup's that row r is of
  auto local_of = [&](int r) { return PACKED ? static_cast<int>((static_cast<float>(r) + 0.5f) * per_head) : 0; };
  const int b0 = token0 / p.w, i0 = token0 - b0 * p.w;
  auto load = [&](int r, Row &row) {
    if (r >= end || !in_head) return;
    const int local = local_of(r), h = r - local * heads;
    int b = b0, i = i0 + local;
    if (PACKED && i >= p.w) {
      const int over = i / p.w;
      b += over;
      i -= over * p.w;
    }
    const bool is_q = h < p.hq, is_v = h >= p.hq + p.hkv;
    const int at = is_q ? h : is_v ? h - p.hq - p.hkv : h - p.hq;
    const T *src = static_cast<const T *>(is_q ? p.q : is_v ? p.v : p.k) +
                   b * (is_q ? p.q_batch : is_v ? p.v_batch : p.k_batch) +
                   i * (is_q ? p.q_token : is_v ? p.v_token : p.k_token) + static_cast<int64_t>(at) * DH;
    row.a = load8<T>(src + first);
    row.b = load8<T>(src + second);
    const T *w = static_cast<const T *>(is_q ? p.q_weight : p.k_weight);
    if (w && !is_v) {
      row.wa = load8<T>(w + first);
      row.wb = load8<T>(w + second);
    }
  };
  int r = begin;
  Row row;
  load(r, row);
  if (static_cast<int>(threadIdx.x) < per_wg * pairs) {
    const int local = PACKED ? threadIdx.x / pairs : 0, pair = threadIdx.x - local * pairs;
    const int token = min(token0 + local, tokens - 1), b = token / p.w;
    const double pos = p.each ? static_cast<double>(p.positions[token])
                              : static_cast<double>(p.positions[b]) + static_cast<double>(token - b * p.w);
    turn(pos * static_cast<double>(p.inv_freq[pair]), cs[threadIdx.x], sn[threadIdx.x]);
  }
  __syncthreads();
  float c[8], s[8];
  auto angles = [&](int local) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      c[j] = turns ? cs[local * pairs + 8 * lane + j] : 1.f;
      s[j] = turns ? sn[local * pairs + 8 * lane + j] : 0.f;
    }
  };
  if (!PACKED) angles(0);
  // the same number of rounds for all lanes of a head; its lanes have the same r
  for (; r < end; r += ROWS) {
    Row next;
    if (!PACKED) load(r + ROWS, next);
    const int local = local_of(r), h = r - local * heads;
    if (PACKED) angles(local);
    const bool is_q = h < p.hq, is_v = h >= p.hq + p.hkv;
    const int at = is_q ? h : is_v ? h - p.hq - p.hkv : h - p.hq;
    const int n = is_q ? p.hq : p.hkv;
    T *dst = static_cast<T *>(is_q ? p.q_out : is_v ? p.v_out : p.k_out) + (static_cast<int64_t>(token0 + local) * n + at) * DH;
    if (is_v) {
      if (in_head) {
        __builtin_memcpy(__builtin_assume_aligned(dst + first, 16), &row.a, sizeof(row.a));
        __builtin_memcpy(__builtin_assume_aligned(dst + second, 16), &row.b, sizeof(row.b));
      }
    } else {
      float x[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = 0.f;
      if (in_head) {
        floats<T>(row.a, x);
        floats<T>(row.b, x + 8);
      }
      if (is_q ? p.q_weight != nullptr : p.k_weight != nullptr) {
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const double d = x[j];
          sum = __builtin_fma(d, d, sum);
        }
        sum = plus_dpp<0xB1>(sum);
        sum = plus_dpp<0x4E>(sum);
        if (LPR == 8) sum = plus_dpp<0x141>(sum);
        float unit;
        const float r = inverse_root(__builtin_fma(sum, 1.0 / DH, static_cast<double>(p.eps)), unit);
        float w[16] = {};
        if (in_head) {
          floats<T>(row.wa, w);
          floats<T>(row.wb, w + 8);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = x[j] * unit * r * w[j];
      }
      float y[16];
      if (halves) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          y[j] = x[j] * c[j] - x[8 + j] * s[j];
          y[8 + j] = x[8 + j] * c[j] + x[j] * s[j];
        }
      } else if (turns) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          y[2 * j] = x[2 * j] * c[j] - x[2 * j + 1] * s[j];
          y[2 * j + 1] = x[2 * j + 1] * c[j] + x[2 * j] * s[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = x[j];
      }
      if (in_head) {
        store8<T>(dst + first, y);
        store8<T>(dst + second, y + 8);
      }
    }
    row = next;
  }
}

template <typename T, int DH>
hipError_t launch_dh(const RopeParams &p, hipStream_t s) {
  constexpr int ROWS = kThreads / (DH == 64 ? 4 : 8);
  const int heads = p.hq + p.hkv + (p.v ? p.hkv : 0);
  const int64_t tokens = static_cast<int64_t>(p.batch) * p.w;
  const int pack = std::min({ROWS / heads, 8, p.rotary ? kThreads / (p.rotary / 2) : 8});
  if (pack >= 2 && tokens >= 4 * kNumCUs)
    return launch_kernel(qk_rope_kernel<T, DH, true>, dim3(static_cast<unsigned>((tokens + pack - 1) / pack)),
                         dim3(kThreads), s, p, pack);
  const int rounds = (heads + ROWS - 1) / ROWS;
  // eight workgroups a compute unit, where there are heads for them
  const int64_t want = (8 * kNumCUs + tokens - 1) / tokens;
  const int split = static_cast<int>(want < rounds ? want : rounds);
  return launch_kernel(qk_rope_kernel<T, DH, false>, dim3(static_cast<unsigned>(tokens), split), dim3(kThreads), s, p, 1);
}

template <typename T>
hipError_t launch_typed(const RopeParams &p, hipStream_t s) {
  if (p.dh == 64) return launch_dh<T, 64>(p, s);
  if (p.dh == 96) return launch_dh<T, 96>(p, s);
  return launch_dh<T, 128>(p, s);
}

}  // namespace

hipError_t launch_qk_rope(const RopeParams &p, int dtype, hipStream_t s) {
  return dtype == DAS_F32 ? launch_typed<float>(p, s) : launch_typed<bf16_t>(p, s);
}

}  // namespace das
