// Verification of drafted tokens against the target's probabilities (das_sampled_accept).
//
// With p and q the target's and the draft's distributions at a position, proposal y is
// accepted if u q(y) < p(y). The first rejected position emits a token of the residual
// max(p - q, 0), one after the last tested proposal a token of p, by a second random number:
// every emitted token then is a draw from p, whatever q is.
//
// Weights are w = exp((z - max) / T) in 64 bits, right to 2^-50 and what the rounding of their
// exponent costs, 2^-52.4 an octave below the largest. Sums Z of a row are right to 2^-41.2: each
// weight by the rounding of its exponent to 2^-41.5, by its polynomial to 2^-45, as the one of the
// largest that they are divided by, and by the sums' and the temperature's roundings to 2^-45.2.
// So a token is another one only where the random number lies within 2^-40 of a border, in a draw
// from a residual 2^-40 of p's whole. Residuals are w_p Z_q - w_q Z_p: exactly 0 where both are
// equal with equal sums; below 2^-40 of p they count as 0, so that rounding leaves no token that p
// does not exceed q at (2 x 2^-41.2 + 2 x 2^-45.9 < 2^-40 for weights down to 2^-64; what is
// under that matters where nothing else is left).
//
// Three kernels: the largest logit and the sum of weights of every part of every row; per
// sequence the run of accepted proposals, and of every part of the row where it ends the sum
// of the residual; the token in the part where the running sum passes the random number's
// share.
//
// 32 sequences x 32 positions x 65536 bf16 logits, target and draft, three quarters of which are
// tested (200 MB): 69-78 us, of which the rows' sums 58 (3.4 TB/s, bound by their 64-bit
// arithmetic), the run 12 and the draw 8, 43 with a greedy draft; one sequence of 8 positions, fp32:
// 12-19 us, three launches and their round trips. Measured and not kept: the draw in the second kernel, by the
// last part to end (14.7 -> 14.4 us, but 76 -> 91: what its counter needs to be seen in order
// writes a cache back for every part); the sums of weights under 2^-12 in fp32 (no gain: nearly
// every piece of a row has a larger one).

#include "mfma_tile.h"
#include "q4_internal.h"

namespace das {
namespace {

#pragma clang fp contract(off)

constexpr int kThreads = 256;
constexpr int kWavesA = kThreads / 64;
constexpr double kNone = 0x1p-40;  // a residual below this share of p is none

// What is known of a row, or of a part of one.
struct Stat {
  float max;
  int at;      // lowest index of the largest logit (one-hot rows only)
  double sum;  // of weights relative to max
};
// What the second kernel leaves for the third.
struct Chain {
  Stat p, q;
  int accepted, y, drawn, pad;  // drawn: kLeft, kPlain or kNothing
};
constexpr int kNothing = 0, kPlain = 1, kLeft = 2;

// A sequence's temperature: the factor of z - max in units of 1 / 32 octave; 0 for one-hot rows.
__device__ __forceinline__ double temper(const float *temperature, int b, bool *bad) {
  const float T = temperature ? temperature[b] : 1.f;
  const bool ok = T >= 0.f && T < __builtin_huge_valf();
  if (!ok) *bad = true;
  return !ok || T == 0.f ? 0.0 : 32.0 * 1.4426950408889634 / static_cast<double>(T);
}

// Powers of two in 64 bits, as products a e: a from a table of N entries, 2^(j / N) with j << lg(2^20
// / N) taken from their upper halves, where the exponent is in units of 1 << 20: adding the
// numerator, shifted the same way, leaves its quotient by N, rounded down, in the exponent.
constexpr int kCoarse = 32, kFine = 256;
template <int N>
struct Powers {
  static constexpr int SHIFT = N == kCoarse ? 15 : 12;
  u32x2 at[N];
  __device__ __forceinline__ double of(uint32_t k) const {
    u32x2 t = at[k % N];
    t[1] += k << SHIFT;
    return __builtin_bit_cast(double, t);
  }
  __device__ __forceinline__ void fill() {  // by all threads, of which there are at least N
    static_assert(N << SHIFT == 1 << 20, "an octave");
    if (threadIdx.x < N) {
      // from the series of e^x - 1 for a 16th of the exponent, doubled four times
      const double x = threadIdx.x * (0.69314718055994531 / N / 16.0);
      double q = 1.0 / 40320.0;
      q = __builtin_fma(q, x, 1.0 / 5040.0);
      q = __builtin_fma(q, x, 1.0 / 720.0);
      q = __builtin_fma(q, x, 1.0 / 120.0);
      q = __builtin_fma(q, x, 1.0 / 24.0);
      q = __builtin_fma(q, x, 1.0 / 6.0);
      q = __builtin_fma(q, x, 0.5);
      q = __builtin_fma(q, x, 1.0);
      double e = q * x;
      for (int i = 0; i < 4; ++i) e = __builtin_fma(e, e, 2.0 * e);
      u32x2 t = __builtin_bit_cast(u32x2, 1.0 + e);
      t[1] -= threadIdx.x << SHIFT;
      at[threadIdx.x] = t;
    }
    __syncthreads();
  }
};

// 2^(d c32 / 32) for d <= 0, d c32 >= -32000: of k + f = d c32, |f| <= 1/2, 2^(k / 32) from the
// table (kCoarse entries lie in different banks), and 2^(f / 32) by 1 + f r(f), r the polynomial
// that agrees with (2^(f / 32) - 1) / f at the five Chebyshev points: 2^-52.6 of it. 1 exactly at
// d = 0.
// Times 2^UP, with which d c32 may go down to -32 (1022 + UP).
template <int UP = 0, int N>
__device__ __forceinline__ double exp2_near(double d, double c32, const Powers<N> &table) {
  constexpr double kRound = 0x1.8p52;  // leaves a sum with it rounded to an integer, in its lower half
  const double big = __builtin_fma(d, c32, kRound), f = __builtin_fma(d, c32, -(big - kRound));
  double r = 3.9737238568525983e-11;
  r = __builtin_fma(r, f, 9.172607532092245e-09);
  r = __builtin_fma(r, f, 1.6938509724285119e-06);
  r = __builtin_fma(r, f, 2.345961981994449e-04);
  r = __builtin_fma(r, f, 2.166084939249829e-02);
  const uint32_t k = static_cast<uint32_t>(__builtin_bit_cast(uint64_t, big)) * (N / kCoarse) + UP * N;
  return table.of(k) * __builtin_fma(r, f, 1.0);
}
// The same for any d <= 0; what is under 2^-1000 becomes that, which no sum notices.
template <int N>
__device__ __forceinline__ double exp2_of(double d, double c32, const Powers<N> &table) {
  return exp2_near(d * c32 < -32000.0 ? -32000.0 / c32 : d, c32, table);
}
// Of a sum with it: the integer part in the lower 20 bits of the upper half (modulo 2^19), the rest
// in units of 2^-32 in the lower half.
constexpr double kFixed = 0x1.8p20;
// -2^(n / 256) as a product a e, of n + kFixed, |n| < 2^18: 2^-41.5 of it is what n's rounding costs
// at most, 2^-45 the polynomial in its rest (relative error, exactly 1 at 0, the least of degree 3).
__device__ __forceinline__ void fixed_power(double n, const Powers<kFine> &table, double &a, double &e) {
  const u32x2 w = __builtin_bit_cast(u32x2, n);
  const double f = w[0];
  e = 0x1.c747fdca05451p-125;
  e = __builtin_fma(e, f, 0x1.ebfbca05b01afp-83);
  e = __builtin_fma(e, f, 0x1.62e42ff08b09bp-41);
  e = __builtin_fma(e, f, 1.0);
  a = table.of(w[1]);
}

// The weight of logit z at index j of a row, times kOne: with that, all that an exponential in 64
// bits holds are normal numbers. Under 2^-1075, half of its smallest, a weight is 0, so that no
// random number of 0 accepts or draws its token.
constexpr int kUp = 128;
constexpr double kOne = 0x1p128, kLeast = -32.0 * 1075.0;
__device__ __forceinline__ double weight(float z, int j, const Stat &r, double c32, const Powers<kCoarse> &table) {
  if (c32 == 0.0 || r.max == kNegInf) return j == r.at ? kOne : 0.0;
  if (r.max == __builtin_huge_valf()) return z == r.max ? kOne : 0.0;
  const double d = static_cast<double>(z) - static_cast<double>(r.max), w = exp2_near<kUp>(d, c32, table);
  return d * c32 >= kLeast ? w : 0.0;
}
// What a draw weighs token `at` by, from the target's and the draft's logits.
__device__ __forceinline__ double residual(const SampledAcceptParams &p, float zp, float zq, int at, const Chain &ch,
                                           double cp, double cq, const Powers<kCoarse> &table) {
  if (at >= p.vocab) return 0.0;
  const double w = weight(zp, at, ch.p, cp, table);
  if (ch.drawn != kLeft) return w;
  const double wq = p.draft ? weight(zq, at, ch.q, cq, table) : at == ch.y ? kOne : 0.0;
  const double a = w * ch.q.sum, d = a - wq * ch.p.sum;
  return d > kNone * a ? d : 0.0;
}

// 8 logits of a row of n (at least 1) from index i on, which may lie past its end; what does is
// -inf.
template <typename T>
struct Eight {
  uint32_t w[8 * sizeof(T) / 4];
};
template <typename T>
__device__ __forceinline__ Eight<T> load8(const T *row, int i, int n) {
  Eight<T> r;
  if (i + 8 <= n) {
    __builtin_memcpy(&r, row + i, sizeof(r));
    return r;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const T z = row[min(i + j, n - 1)];
    if constexpr (sizeof(T) == 2) {
      const uint32_t v = i + j < n ? z : 0xff80u;
      r.w[j / 2] = j % 2 ? r.w[j / 2] | v << 16 : v;
    } else {
      r.w[j] = i + j < n ? __float_as_uint(z) : 0xff800000u;
    }
  }
  return r;
}
// Logit j of the eight as it is, and with -inf for NaN.
template <typename T>
__device__ __forceinline__ float raw_logit(const Eight<T> &r, int j) {
  if constexpr (sizeof(T) == 2) return __uint_as_float(j % 2 ? r.w[j / 2] & 0xffff0000u : r.w[j / 2] << 16);
  else return __uint_as_float(r.w[j]);
}
__device__ __forceinline__ float no_nan(float z) { return z == z ? z : kNegInf; }
template <typename T>
__device__ __forceinline__ float logit(const Eight<T> &r, int j) { return no_nan(raw_logit<T>(r, j)); }

__device__ __forceinline__ double join64(uint32_t lo, uint32_t hi) {
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
template <int CTRL>
__device__ __forceinline__ double plus_dpp(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return x + join64(__builtin_amdgcn_update_dpp(0, static_cast<uint32_t>(u), CTRL, 0xf, 0xf, false),
                    __builtin_amdgcn_update_dpp(0, static_cast<uint32_t>(u >> 32), CTRL, 0xf, 0xf, false));
}
// Sum over the wave, in every lane: lanes 1 and 2 apart, mirrored in 8 and 16, then the swaps
// of 16 and 32 lanes.
__device__ __forceinline__ double wave_sum(double x) {
  x = plus_dpp<0xB1>(x);
  x = plus_dpp<0x4E>(x);
  x = plus_dpp<0x141>(x);
  x = plus_dpp<0x140>(x);
  uint64_t u = __builtin_bit_cast(uint64_t, x);
  uint32_t lo = static_cast<uint32_t>(u), hi = static_cast<uint32_t>(u >> 32);
  auto a = __builtin_amdgcn_permlane16_swap(lo, lo, false, false);
  auto b = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
  x = join64(a[0], b[0]) + join64(a[1], b[1]);
  u = __builtin_bit_cast(uint64_t, x);
  lo = static_cast<uint32_t>(u), hi = static_cast<uint32_t>(u >> 32);
  a = __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
  b = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
  return join64(a[0], b[0]) + join64(a[1], b[1]);
}
template <int CTRL>
__device__ __forceinline__ float max_dpp(float x) {
  return fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, false)));
}
__device__ __forceinline__ float wave_max(float x) {
  return group_max(max_dpp<0x140>(max_dpp<0x141>(max_dpp<0x4E>(max_dpp<0xB1>(x)))));
}

// Tokens of a sequence that are verified, clamped as das_greedy_accept does.
__device__ __forceinline__ int tested_of(const SampledAcceptParams &p, int b, bool *bad) {
  const int raw = p.tested ? p.tested[b] : p.w;
  const int m = min(max(raw, 0), p.w);
  if (raw != m) *bad = true;
  return m;
}

// The workspace: statistics of all parts of target and draft rows, sums of the draw's parts,
// and a Chain for every sequence.
__device__ __forceinline__ Stat *stats_of(const SampledAcceptParams &p, int side, int64_t row) {
  return reinterpret_cast<Stat *>(p.ws) + (static_cast<int64_t>(side) * p.batch * p.w + row) * p.parts;
}
__device__ __forceinline__ double *lefts_of(const SampledAcceptParams &p, int b) {
  return reinterpret_cast<double *>(stats_of(p, 2, 0)) + static_cast<int64_t>(b) * p.draw_parts;
}
__device__ __forceinline__ Chain *chain_of(const SampledAcceptParams &p, int b) {
  return reinterpret_cast<Chain *>(lefts_of(p, p.batch)) + b;
}

constexpr int kVec = kAcceptPart / (kThreads * 8);  // pieces of 8 logits of a thread
constexpr int kDraw = kThreads * 8;                 // tokens of a part of the draw, one piece each
static_assert(kDraw == kAcceptDraw && sizeof(Stat) == kAcceptStatBytes && sizeof(Chain) == kAcceptChainBytes,
              "the workspace's layout");

// The sums' arithmetic bounds it: 11 operations a logit beside the unpacking and the maximum (1530
// rows of 65536 bf16 logits, 200 MB: 58 us; with 20 operations 74 us, and 61 us with as many
// registers as the compiler takes by itself, which is 4 waves a SIMD instead of 6).
template <typename T>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(6)))
void accept_stats_kernel(SampledAcceptParams p) {
  __shared__ Powers<kFine> table;
  __shared__ double part_sum[kWavesA];
  __shared__ float part_max[kWavesA];
  __shared__ int part_at[kWavesA];
  const int part = blockIdx.x % p.parts;
  const int64_t side_row = blockIdx.x / p.parts, rows = static_cast<int64_t>(p.batch) * p.w;
  const int side = side_row >= rows;
  const int64_t row = side ? side_row - rows : side_row;
  const int b = static_cast<int>(row / p.w), i = static_cast<int>(row % p.w);
  bool bad = false;
  const int m = tested_of(p, b, &bad);
  if (i > m || (side && i == m)) return;  // nobody asks for it
  const double c32 = temper(side ? p.draft_temperature : p.temperature, b, &bad);
  const T *src = static_cast<const T *>(side ? p.draft : p.target) + row * (side ? p.draft_stride : p.target_stride);
  Eight<T> x[kVec];
  const int begin = part * kAcceptPart + static_cast<int>(threadIdx.x) * 8;
#pragma unroll
  for (int v = 0; v < kVec; ++v) x[v] = load8<T>(src, begin + v * kThreads * 8, p.vocab);
  table.fill();
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  float mx = kNegInf;
#pragma unroll
  for (int v = 0; v < kVec; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) mx = fmaxf(mx, raw_logit<T>(x[v], j));  // NaN gives way
  mx = wave_max(mx);
  if (lane == 0) part_max[wave] = mx;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWavesA; ++k) mx = fmaxf(mx, part_max[k]);
  double sum = 0.0, largest = 1.0;  // what the largest logit weighs in the sum
  int at = 0x7fffffff;
  if (c32 == 0.0 || mx == kNegInf) {
#pragma unroll
    for (int v = 0; v < kVec; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) at = logit<T>(x[v], j) == mx ? min(at, begin + v * kThreads * 8 + j) : at;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) at = min(at, __shfl_xor(at, d));
  } else if (mx == __builtin_huge_valf()) {
#pragma unroll
    for (int v = 0; v < kVec; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += logit<T>(x[v], j) == mx ? 1.0 : 0.0;
  } else if (const float low = static_cast<float>(static_cast<double>(mx) - 28000.0 / c32);
             low > -3e38f && (static_cast<double>(mx) - static_cast<double>(low)) * c32 < 32000.0 &&
             (static_cast<double>(mx) - static_cast<double>(low)) * c32 > 24000.0 &&
             fabs(static_cast<double>(mx) * c32) < 0x1p30) {
    // Logits under `low` weigh nothing (2^-875, give or take fp32's rounding of it); as that they,
    // NaN and -inf need no more tests. The weights are taken relative to the power of two under
    // the largest, which saves the difference of each logit and the largest, and their sum is
    // brought to be relative to the largest afterwards.
    const double step = 8.0 * c32, top = static_cast<double>(mx) * step, whole = 256.0 * floor(top / 256.0);
    const double base = kFixed - whole, least = low;
    double a, e;
#pragma unroll
    for (int v = 0; v < kVec; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        fixed_power(__builtin_fma(fmax(static_cast<double>(raw_logit<T>(x[v], j)), least), step, base), table, a, e);
        sum = __builtin_fma(a, e, sum);
      }
    // with what the rounding of its exponent leaves: every weight of the row is relative to it
    const double n = __builtin_fma(static_cast<double>(mx), step, base);
    const double rest = (top - whole - (n - kFixed)) + __builtin_fma(static_cast<double>(mx), step, -top);
    fixed_power(n, table, a, e);
    largest = a * e;  // both have the sign of a
    largest = __builtin_fma(largest, rest * (0.69314718055994531 / 256.0), largest);
  } else {  // so hot that every finite logit counts, or so cold that fp32 has no such `low`
    const double top = mx;
#pragma unroll 1
    for (int v = 0; v < kVec; ++v) {
      Eight<T> y = x[0];
#pragma unroll
      for (int i = 1; i < kVec; ++i)
        if (i == v) y = x[i];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float z = logit<T>(y, j);
        const double w = exp2_of(static_cast<double>(z) - top, c32, table);
        sum += z > kNegInf ? w : 0.0;
      }
    }
  }
  sum = wave_sum(sum);
  if (lane == 0) {
    part_sum[wave] = sum;
    part_at[wave] = at;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    Stat r = {mx, at, 0.0};
    for (int k = 0; k < kWavesA; ++k) {
      r.sum += part_sum[k];
      r.at = min(r.at, part_at[k]);
    }
    r.sum /= largest;
    stats_of(p, side, row)[part] = r;
  }
}

// A row's parts as one; sums of one-hot rows are 1. `x`: the first kAhead of them (the last, where
// there are fewer), as load_parts has them.
constexpr int kAhead = 8;
__device__ __forceinline__ void load_parts(Stat (&x)[kAhead], const Stat *s, int from, int parts) {
#pragma unroll
  for (int k = 0; k < kAhead; ++k) x[k] = s[min(from + k, parts - 1)];
}
__device__ __forceinline__ Stat join_parts(Stat (&x)[kAhead], const Stat *s, int parts, double c32,
                                           const Powers<kCoarse> &table) {
  Stat r = {kNegInf, 0x7fffffff, 0.0};
  for (int k0 = 0; k0 < parts; k0 += kAhead) {
    if (k0) load_parts(x, s, k0, parts);
    float mx = r.max;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) mx = fmaxf(mx, x[k].max);
    auto scaled = [&](const Stat &a) {
      if (a.max == mx) return a.sum;
      if (a.max == kNegInf || mx == __builtin_huge_valf()) return 0.0;
      return a.sum * exp2_of(static_cast<double>(a.max) - static_cast<double>(mx), c32, table);
    };
    double sum = scaled(r);
    int at = r.max == mx ? r.at : 0x7fffffff;
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (k0 + k < parts) {
        sum += scaled(x[k]);
        if (x[k].max == mx) at = min(at, x[k].at);
      }
    r = Stat{mx, at, sum};
  }
  if (c32 == 0.0 || r.max == kNegInf) r.sum = 1.0;
  return r;
}

// One piece of the row where the run of accepted proposals ends: tokens 8 t .. + 7 of part
// `part` of the draw for thread t, and what the draw weighs them by.
template <typename T>
__device__ __forceinline__ void draw_weights(const SampledAcceptParams &p, int b, int part, const Chain &ch,
                                             double cp, double cq, const Powers<kCoarse> &table, double (&w)[8]) {
  const int64_t row = static_cast<int64_t>(b) * p.w + ch.accepted;
  const bool drafted = ch.drawn == kLeft && p.draft;
  const int first = part * kDraw + static_cast<int>(threadIdx.x) * 8;
  const Eight<T> x = load8<T>(static_cast<const T *>(p.target) + row * p.target_stride, first, p.vocab);
  Eight<T> y = {};
  if (drafted) y = load8<T>(static_cast<const T *>(p.draft) + row * p.draft_stride, first, p.vocab);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    w[j] = residual(p, logit<T>(x, j), drafted ? logit<T>(y, j) : 0.f, first + j, ch, cp, cq, table);
}
// The sum over a part, for all threads.
__device__ __forceinline__ double part_total(const double (&w)[8], double *seg) {
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < 8; ++j) sum += w[j];
  sum = wave_sum(sum);
  __syncthreads();  // the call before has been read
  if (threadIdx.x % 64 == 0) seg[threadIdx.x / 64] = sum;
  __syncthreads();
  double total = 0.0;
#pragma unroll
  for (int k = 0; k < kWavesA; ++k) total += seg[k];
  return total;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void accept_chain_kernel(SampledAcceptParams p) {
  __shared__ Powers<kCoarse> table;
  __shared__ double seg[kWavesA];
  __shared__ Chain chain;
  __shared__ Stat drafts[64];
  __shared__ double draft_weight[64];
  const int b = blockIdx.x / p.draw_parts, part = blockIdx.x % p.draw_parts;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  // all that needs no other result first, in one round trip: lane i of the first two waves has
  // position i of the target and of the draft
  const int64_t at_row = static_cast<int64_t>(b) * p.w + lane;
  const bool sided = lane < p.w && (wave == 0 || (wave == 1 && p.draft));
  Stat parts[kAhead];
  int y = 0;
  float u = 0.f;
  if (sided) {
    y = p.proposals[at_row];
    u = p.uniform[at_row];
    load_parts(parts, stats_of(p, wave, at_row), 0, p.parts);  // those that nobody asked for are not used
  }
  bool bad_temp = false, bad_tested = false;
  const int m = tested_of(p, b, &bad_tested);
  const double cp = temper(p.temperature, b, &bad_temp);
  const double cq = p.draft ? temper(p.draft_temperature, b, &bad_temp) : 0.0;
  const bool mine = sided && (wave == 0 ? lane <= m : lane < m);
  float zy = kNegInf;
  if (mine && lane < m) {
    const T *rows = static_cast<const T *>(wave == 0 ? p.target : p.draft);
    if (y >= 0 && y < p.vocab) zy = to_f32<T>(rows[at_row * (wave == 0 ? p.target_stride : p.draft_stride) + y]);
  }
  table.fill();
  Stat s = {kNegInf, 0, 1.0};
  double wy = 0.0;
  if (mine) {
    s = join_parts(parts, stats_of(p, wave, at_row), p.parts, wave == 0 ? cp : cq, table);
    if (lane < m) wy = weight(no_nan(zy), y, s, wave == 0 ? cp : cq, table);
  }
  if (wave == 1) {
    drafts[lane] = s;
    draft_weight[lane] = wy;
  }
  __syncthreads();
  if (wave == 0) {
    const bool checked = lane < m;
    const bool bad_token = checked && (y < 0 || y >= p.vocab), bad_number = checked && !(u >= 0.f && u < 1.f);
    const Stat sq = p.draft ? drafts[lane] : Stat{kNegInf, 0, 1.0};
    const double wq = p.draft ? draft_weight[lane] : kOne, py = wy / s.sum;  // times kOne
    const bool ok = checked && !bad_token && !bad_number && static_cast<double>(u) * (wq / sq.sum) < py;
    const uint64_t miss = ~__ballot(ok);
    const int a = min(miss ? static_cast<int>(__builtin_ctzll(miss)) : 64, m);
    if (lane == min(a, p.w - 1)) {
      chain.p = s;
      chain.q = sq;
      chain.accepted = a;
      chain.y = bad_token ? -1 : y;
      chain.drawn = a == p.w ? kNothing : a == m ? kPlain : kLeft;
    }
    if (part == 0) {
      const float v = p.draw[b];
      const bool bad_draw = lane == 0 && a < p.w && !(v >= 0.f && v < 1.f);
      const bool reached = lane <= a;  // what lies behind the first rejected one does not count
      const uint32_t word = (bad_temp || bad_draw || (reached && bad_number) ? DAS_DEVERR_SAMPLE : 0) |
                            (bad_tested ? DAS_DEVERR_TESTED : 0) |
                            (reached && bad_token ? DAS_DEVERR_PROPOSAL : 0);
      if (word) report_error(p.dev_error, word);
      const int keep = min(a + 1, p.w);
      if (lane == 0) {
        p.accepted[b] = a;
        p.num_keep[b] = keep;
        if (p.num_emitted) p.num_emitted[b] = keep;
      }
      if (lane < a) {
        if (p.emitted) p.emitted[at_row] = y;
        if (p.probs) p.probs[at_row] = static_cast<float>(py / kOne);
      }
    }
  }
  __syncthreads();
  const Chain ch = chain;
  if (part == 0 && threadIdx.x == 0) *chain_of(p, b) = ch;
  if (ch.drawn == kNothing) return;
  double w[8];
  draw_weights<T>(p, b, part, ch, cp, cq, table, w);
  const double total = part_total(w, seg);
  if (threadIdx.x == 0) lefts_of(p, b)[part] = total;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void accept_draw_kernel(SampledAcceptParams p) {
  __shared__ Powers<kCoarse> table;
  __shared__ double seg[kWavesA], lefts[kAcceptMostDraws];
  const int b = blockIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  Chain ch = *chain_of(p, b);
  for (int k = threadIdx.x; k < p.draw_parts; k += kThreads) lefts[k] = lefts_of(p, b)[k];
  if (ch.drawn == kNothing) return;
  bool bad;  // reported before
  const double cp = temper(p.temperature, b, &bad);
  const double cq = p.draft ? temper(p.draft_temperature, b, &bad) : 0.0;
  const float number = p.draw[b];
  table.fill();
  // the running sum over the parts: a lane's parts, then the lanes before
  auto total_of = [&]() {
    double sum = 0.0;
    for (int k = lane; k < p.draw_parts; k += 64) sum += lefts[k];
    return wave_sum(sum);
  };
  double total = total_of(), w[8];
  if (total == 0.0) {  // p does not exceed q anywhere: a token of p
    ch.drawn = kPlain;
    for (int k = 0; k < p.draw_parts; ++k) {
      draw_weights<T>(p, b, k, ch, cp, cq, table, w);
      const double sum = part_total(w, seg);
      if (threadIdx.x == 0) lefts[k] = sum;
    }
    __syncthreads();
    total = total_of();
  }
  const double target = (number >= 0.f && number < 1.f ? static_cast<double>(number) : 0.0) * total;
  // Inclusive sums of 64 values, one a lane.
  auto scan = [&](double x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint64_t v = __builtin_bit_cast(uint64_t, x);
      const double o = join64(__shfl_up(static_cast<int>(v), d), __shfl_up(static_cast<int>(v >> 32), d));
      x += lane >= d ? o : 0.0;
    }
    return x;
  };
  auto lane_of = [&](double x, int l) {
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    return join64(__builtin_amdgcn_readlane(static_cast<uint32_t>(v), l),
                  __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), l));
  };
  // the part that passes the target; where rounding lets none, the last with a token
  int part = 0;
  double run = 0.0, before = 0.0;
  for (int k0 = 0; k0 < p.draw_parts; k0 += 64) {
    const double x = k0 + lane < p.draw_parts ? lefts[k0 + lane] : 0.0, incl = scan(x);
    const uint64_t pass = __ballot(x > 0.0 && target < run + incl), some = __ballot(x > 0.0);
    if (pass || some) {
      const int l = pass ? static_cast<int>(__builtin_ctzll(pass)) : 63 - static_cast<int>(__builtin_clzll(some));
      part = k0 + l;
      before = run + (lane_of(incl, l) - lane_of(x, l));
      if (pass) break;
    }
    run += lane_of(incl, 63);
  }
  draw_weights<T>(p, b, part, ch, cp, cq, table, w);
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < 8; ++j) sum += w[j];
  const double incl = scan(sum);
  __syncthreads();
  if (lane == 63) seg[wave] = incl;
  __syncthreads();
  // the wave whose 512 tokens pass the target, the same way
  int found = 0;
  run = before;
  double from = before;
#pragma unroll
  for (int k = 0; k < kWavesA; ++k) {
    const double x = seg[k];
    if (x > 0.0 && !(target < from + seg[found] && seg[found] > 0.0)) {
      found = k;
      from = run;
    }
    run += x;
  }
  if (found != wave) return;
  double at = from + (incl - sum);
  const int first = part * kDraw + static_cast<int>(threadIdx.x) * 8;
  int token = 0x7fffffff, last = -1;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    at += w[j];
    if (w[j] > 0.0) {
      last = first + j;
      if (target < at) token = min(token, first + j);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    token = min(token, __shfl_xor(token, d));
    last = max(last, __shfl_xor(last, d));
  }
  if (lane == 0) {
    token = min(max(token == 0x7fffffff ? last : token, 0), p.vocab - 1);
    const int64_t row = static_cast<int64_t>(b) * p.w + ch.accepted;
    if (p.emitted) p.emitted[row] = token;
    if (p.probs) {
      const float z = no_nan(to_f32<T>(static_cast<const T *>(p.target)[row * p.target_stride + token]));
      p.probs[row] = static_cast<float>(weight(z, token, ch.p, cp, table) / ch.p.sum / kOne);
    }
  }
}

template <typename T>
hipError_t launch_typed(const SampledAcceptParams &p, hipStream_t s) {
  const int64_t rows = static_cast<int64_t>(p.batch) * p.w * (p.draft ? 2 : 1);
  hipError_t e = launch_kernel(accept_stats_kernel<T>, dim3(static_cast<unsigned>(rows * p.parts)), dim3(kThreads), s, p);
  if (e != hipSuccess) return e;
  e = launch_kernel(accept_chain_kernel<T>, dim3(static_cast<unsigned>(p.batch) * p.draw_parts), dim3(kThreads), s, p);
  if (e != hipSuccess) return e;
  return launch_kernel(accept_draw_kernel<T>, dim3(p.batch), dim3(kThreads), s, p);
}

}  // namespace

hipError_t launch_sampled_accept(const SampledAcceptParams &p, int dtype, hipStream_t s) {
  return dtype == DAS_F32 ? launch_typed<float>(p, s) : launch_typed<bf16_t>(p, s);
}

}  // namespace das
