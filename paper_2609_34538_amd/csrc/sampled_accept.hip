// Verification of drafted tokens against the target's probabilities (das_sampled_accept).
//
// With p and q the target's and the draft's distributions at a position, proposal y is
// accepted if u q(y) < p(y). The first rejected position emits a token of the residual
// max(p - q, 0), one after the last tested proposal a token of p, by a second random number:
// every emitted token then is a draw from p, whatever q is.
//
// Weights are w = exp((z - max) / T) in 64 bits, so that a token is another one only where
// the random number lies within 2^-40 of a border, and sums of equal weights are exact in any
// order. Residuals are w_p Z_q - w_q Z_p: exactly 0 where both are equal with equal sums;
// below 2^-40 of p they count as 0, so that rounding leaves no token that p does not exceed q
// at.
//
// Three kernels: the largest logit and the sum of weights of every part of every row (bound
// by HBM and its 64-bit arithmetic); per sequence the run of accepted proposals, and of every
// part of the row where it ends the sum of the residual; the token in the part where the
// running sum passes the random number's share.

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
  int at;      // lowest index of the largest logit (greedy rows only)
  double sum;  // of weights relative to max
};
// What the second kernel leaves for the third.
struct Chain {
  Stat p, q;
  int accepted, y, drawn, pad;  // drawn: kLeft, kPlain or kNothing
};
constexpr int kNothing = 0, kPlain = 1, kLeft = 2;

// 2^x for x <= 0 in 64 bits: 2^x = 2^n 2^(j / 32) 2^f with |f| <= 1 / 64 and the series of
// e^(f ln 2) to f^5 (rest below 2^-48); table: 2^(j / 32), 32 entries that lie in different banks.
__device__ __forceinline__ double exp2_of(double x, const double *table) {
  const double t = fmax(x, -1000.0);
  const double big = __builtin_fma(t, 32.0, 0x1.8p52);
  const int k = static_cast<int>(__builtin_bit_cast(uint64_t, big));
  const double f = __builtin_fma(big - 0x1.8p52, -0.03125, t);
  double q = 0.0013333558146428443;
  q = __builtin_fma(q, f, 0.0096181291076284772);
  q = __builtin_fma(q, f, 0.055504108664821580);
  q = __builtin_fma(q, f, 0.24022650695910071);
  q = __builtin_fma(q, f, 0.69314718055994531);
  const double a = table[k & 31];
  return __builtin_amdgcn_ldexp(__builtin_fma(a * f, q, a), k >> 5);
}
__device__ __forceinline__ void fill_table(double *table) {
  if (threadIdx.x < 32) {
    // 2^(j / 32), j < 32, from the series of e^x on [0, ln 2) by halving
    const double x = threadIdx.x * (0.69314718055994531 / 32.0 / 16.0);
    double q = 1.0 / 40320.0;
    q = __builtin_fma(q, x, 1.0 / 5040.0);
    q = __builtin_fma(q, x, 1.0 / 720.0);
    q = __builtin_fma(q, x, 1.0 / 120.0);
    q = __builtin_fma(q, x, 1.0 / 24.0);
    q = __builtin_fma(q, x, 1.0 / 6.0);
    q = __builtin_fma(q, x, 0.5);
    q = __builtin_fma(q, x, 1.0);
    double e = q * x;  // e^x - 1, doubled four times
    for (int i = 0; i < 4; ++i) e = __builtin_fma(e, e, 2.0 * e);
    table[threadIdx.x] = 1.0 + e;
  }
  __syncthreads();
}

// A distribution's parameters: greedy rows are one-hot.
struct Temper {
  double c;  // log2(e) / T
  bool greedy;
};
__device__ __forceinline__ Temper temper(const float *temperature, int b, bool *bad) {
  const float T = temperature ? temperature[b] : 1.f;
  const bool ok = T >= 0.f && T < __builtin_huge_valf();
  if (!ok) *bad = true;
  Temper t;
  t.greedy = !ok || T == 0.f;
  t.c = t.greedy ? 0.0 : 1.4426950408889634 / static_cast<double>(T);
  return t;
}
// The weight of logit z at index j of a row.
__device__ __forceinline__ double weight(float z, int j, const Stat &r, const Temper &t, const double *table) {
  if (t.greedy || r.max == kNegInf) return j == r.at ? 1.0 : 0.0;
  if (z == r.max) return 1.0;
  if (z == kNegInf || r.max == __builtin_huge_valf()) return 0.0;
  return exp2_of((static_cast<double>(z) - static_cast<double>(r.max)) * t.c, table);
}
// What a draw weighs token `at` by, from the target's and the draft's logits.
__device__ __forceinline__ double residual(const SampledAcceptParams &p, float zp, float zq, int at, const Chain &ch,
                                           const Temper &tp, const Temper &tq, const double *table) {
  if (at >= p.vocab) return 0.0;
  const double w = weight(zp, at, ch.p, tp, table);
  if (ch.drawn != kLeft) return w;
  const double wq = p.draft ? weight(zq, at, ch.q, tq, table) : at == ch.y ? 1.0 : 0.0;
  const double a = w * ch.q.sum, d = a - wq * ch.p.sum;
  return d > kNone * a ? d : 0.0;
}
// Two parts of a row as one.
__device__ __forceinline__ Stat join(const Stat &a, const Stat &b, const Temper &t, const double *table) {
  const bool first = a.max > b.max || (a.max == b.max && a.at <= b.at);
  const Stat &hi = first ? a : b, &lo = first ? b : a;
  Stat r = hi;
  if (!t.greedy && lo.max > kNegInf) {
    const double w = lo.max == hi.max ? 1.0
                     : hi.max == __builtin_huge_valf()
                         ? 0.0
                         : exp2_of((static_cast<double>(lo.max) - static_cast<double>(hi.max)) * t.c, table);
    r.sum = hi.sum + lo.sum * w;
  }
  return r;
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
template <typename T>
__device__ __forceinline__ float logit(const Eight<T> &r, int j) {
  float z;
  if constexpr (sizeof(T) == 2) z = __uint_as_float(j % 2 ? r.w[j / 2] & 0xffff0000u : r.w[j / 2] << 16);
  else z = __uint_as_float(r.w[j]);
  return z == z ? z : kNegInf;
}

__device__ __forceinline__ double join64(uint32_t lo, uint32_t hi) {
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ double shuffled(double x, int mask) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return join64(__shfl_xor(static_cast<int>(u), mask), __shfl_xor(static_cast<int>(u >> 32), mask));
}
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x += shuffled(x, m);
  return x;
}

// Tokens of a sequence that are verified, clamped as das_greedy_accept does.
__device__ __forceinline__ int tested_of(const SampledAcceptParams &p, int b, bool *bad) {
  const int raw = p.tested ? p.tested[b] : p.w;
  const int m = min(max(raw, 0), p.w);
  if (raw != m) *bad = true;
  return m;
}

constexpr int kVec = 4;                       // pieces of 8 logits of a thread
constexpr int kPart = kThreads * 8 * kVec;    // tokens of a part
static_assert(kPart == kAcceptPart && sizeof(Stat) == kAcceptStatBytes && sizeof(Chain) == kAcceptChainBytes,
              "the workspace's layout");

// Part `part` of a row: its tokens kThreads * 8 * v + 8 * thread .. + 7.
template <typename T, typename Fn>
__device__ __forceinline__ void for_part(const Eight<T> (&x)[kVec], int begin, Fn &&fn) {
#pragma unroll
  for (int v = 0; v < kVec; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) fn(begin + (v * kThreads + static_cast<int>(threadIdx.x)) * 8 + j, logit<T>(x[v], j));
}
template <typename T>
__device__ __forceinline__ void load_part(Eight<T> (&x)[kVec], const T *row, int begin, int n) {
#pragma unroll
  for (int v = 0; v < kVec; ++v)
    x[v] = load8<T>(row, begin + (v * kThreads + static_cast<int>(threadIdx.x)) * 8, n);
}

__device__ __forceinline__ Stat *stats_of(const SampledAcceptParams &p, int side, int64_t row) {
  return reinterpret_cast<Stat *>(p.ws) + (static_cast<int64_t>(side) * p.batch * p.w + row) * p.parts;
}
__device__ __forceinline__ double *lefts_of(const SampledAcceptParams &p, int b) {
  return reinterpret_cast<double *>(stats_of(p, 2, 0)) + static_cast<int64_t>(b) * p.parts;
}
__device__ __forceinline__ Chain *chain_of(const SampledAcceptParams &p, int b) {
  return reinterpret_cast<Chain *>(lefts_of(p, p.batch)) + b;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void accept_stats_kernel(SampledAcceptParams p) {
  __shared__ double table[32], part_sum[kWavesA];
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
  const Temper t = temper(side ? p.draft_temperature : p.temperature, b, &bad);
  const T *src = static_cast<const T *>(side ? p.draft : p.target) + row * (side ? p.draft_stride : p.target_stride);
  Eight<T> x[kVec];
  const int begin = part * kPart;
  load_part<T>(x, src, begin, p.vocab);
  fill_table(table);
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  float mx = kNegInf;
  for_part<T>(x, begin, [&](int, float z) { mx = fmaxf(mx, z); });
#pragma unroll
  for (int d = 1; d < 64; d *= 2) mx = fmaxf(mx, __shfl_xor(mx, d));
  if (lane == 0) part_max[wave] = mx;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWavesA; ++k) mx = fmaxf(mx, part_max[k]);
  double sum = 0.0;
  int at = 0x7fffffff;
  if (t.greedy || mx == kNegInf) {
    for_part<T>(x, begin, [&](int j, float z) { at = z == mx ? min(at, j) : at; });
#pragma unroll
    for (int d = 1; d < 64; d *= 2) at = min(at, __shfl_xor(at, d));
  } else if (mx == __builtin_huge_valf()) {
    for_part<T>(x, begin, [&](int, float z) { sum += z == mx ? 1.0 : 0.0; });
  } else {
    const double top = mx;
    for_part<T>(x, begin, [&](int, float z) { sum += exp2_of((static_cast<double>(z) - top) * t.c, table); });
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
    stats_of(p, side, row)[part] = r;
  }
}

// The sum over a part of the row where the run of accepted proposals ends: of the residual or
// of p. All threads of the workgroup, which all get it.
template <typename T>
__device__ __forceinline__ double part_sum(const SampledAcceptParams &p, int b, int part, const Chain &ch, const Temper &tp,
                           const Temper &tq, const double *table, double *seg) {
  const int64_t row = static_cast<int64_t>(b) * p.w + ch.accepted;
  const T *zp = static_cast<const T *>(p.target) + row * p.target_stride;
  const bool left = ch.drawn == kLeft, drafted = left && p.draft;
  const int begin = part * kPart;
  Eight<T> x[kVec], y[kVec];
  load_part<T>(x, zp, begin, p.vocab);
  if (drafted) load_part<T>(y, static_cast<const T *>(p.draft) + row * p.draft_stride, begin, p.vocab);
  double sum = 0.0;
#pragma unroll
  for (int v = 0; v < kVec; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = begin + (v * kThreads + static_cast<int>(threadIdx.x)) * 8 + j;
      sum += residual(p, logit<T>(x[v], j), drafted ? logit<T>(y[v], j) : 0.f, at, ch, tp, tq, table);
    }
  sum = wave_sum(sum);
  __syncthreads();  // the call before has been read
  if (threadIdx.x % 64 == 0) seg[threadIdx.x / 64] = sum;
  __syncthreads();
  double total = 0.0;
#pragma unroll
  for (int k = 0; k < kWavesA; ++k) total += seg[k];
  return total;
}

// The row's token number that the draw takes, from a part: its residuals in token order.
// All threads of the workgroup; `before`: the sum of the parts before.
template <typename T>
__device__ __forceinline__ int pick(const SampledAcceptParams &p, int b, int part, double before, double target, const Chain &ch,
                    const Temper &tp, const Temper &tq, const double *table, double *seg, int *answer) {
  const int64_t row = static_cast<int64_t>(b) * p.w + ch.accepted;
  const T *zp = static_cast<const T *>(p.target) + row * p.target_stride;
  const T *zq = p.draft ? static_cast<const T *>(p.draft) + row * p.draft_stride : nullptr;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, begin = part * kPart;
  Eight<T> x[kVec], y[kVec] = {};
  load_part<T>(x, zp, begin, p.vocab);
  const bool drafted = ch.drawn == kLeft && zq;
  if (drafted) load_part<T>(y, zq, begin, p.vocab);
  // segments of 512 tokens: wave `wave` of piece v, in token order v * waves + wave
#pragma unroll
  for (int v = 0; v < kVec; ++v) {
    double mine = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int at = begin + (v * kThreads + static_cast<int>(threadIdx.x)) * 8 + j;
      mine += residual(p, logit<T>(x[v], j), drafted ? logit<T>(y[v], j) : 0.f, at, ch, tp, tq, table);
    }
    mine = wave_sum(mine);
    if (lane == 0) seg[v * kWavesA + wave] = mine;
  }
  __syncthreads();
  // the segment that passes the target; where rounding lets none, the last with a token
  int found = 0;
  double run = before, from = before;
  for (int k = 0; k < kVec * kWavesA; ++k) {
    const double s = seg[k];
    if (s > 0.0) {
      found = k;
      from = run;
      if (target < run + s) break;
    }
    run += s;
  }
  if (found % kWavesA == wave) {
    Eight<T> xs = x[0], ys = y[0];
#pragma unroll
    for (int v = 1; v < kVec; ++v)
      if (v == found / kWavesA) xs = x[v], ys = y[v];
    const int first = begin + found * 512 + lane * 8;
    double w[8], mine = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = residual(p, logit<T>(xs, j), drafted ? logit<T>(ys, j) : 0.f, first + j, ch, tp, tq, table);
      mine += w[j];
    }
    // inclusive sum of the lanes
    double incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint64_t u = __builtin_bit_cast(uint64_t, incl);
      const uint32_t lo = __shfl_up(static_cast<int>(u), d), hi = __shfl_up(static_cast<int>(u >> 32), d);
      incl += lane >= d ? join64(lo, hi) : 0.0;
    }
    double at = from + (incl - mine);
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
    if (lane == 0) *answer = token == 0x7fffffff ? last : token;
  }
  __syncthreads();
  return *answer;
}

// The drawn token into the outputs, by thread 0.
template <typename T>
__device__ __forceinline__ void emit_drawn(const SampledAcceptParams &p, int b, int token, const Chain &ch, const Temper &tp,
                           const double *table) {
  const int64_t row = static_cast<int64_t>(b) * p.w + ch.accepted;
  if (p.emitted) p.emitted[row] = token;
  if (p.probs) {
    const T *zp = static_cast<const T *>(p.target) + row * p.target_stride;
    float z = to_f32<T>(zp[token]);
    z = z == z ? z : kNegInf;
    p.probs[row] = static_cast<float>(weight(z, token, ch.p, tp, table) / ch.p.sum);
  }
}

// target: the share of the whole that the draw takes.
__device__ __forceinline__ double share_of(const SampledAcceptParams &p, int b, double total) {
  const float u = p.draw[b];
  return (u >= 0.f && u < 1.f ? static_cast<double>(u) : 0.0) * total;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void accept_chain_kernel(SampledAcceptParams p) {
  __shared__ double table[32], seg[kWavesA];
  __shared__ Chain chain;
  const int b = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  fill_table(table);
  bool bad_temp = false, bad_tested = false;
  const int m = tested_of(p, b, &bad_tested);
  const Temper tp = temper(p.temperature, b, &bad_temp);
  const Temper tq = p.draft ? temper(p.draft_temperature, b, &bad_temp) : Temper{0.0, true};
  if (wave == 0) {
    // lane i: position i
    Stat sp = {kNegInf, 0, 0.0}, sq = {kNegInf, 0, 1.0};
    int y = 0;
    double py = 0.0;
    bool ok = false, bad_number = false, bad_token = false;
    if (lane < p.w && lane <= m) {
      const int64_t row = static_cast<int64_t>(b) * p.w + lane;
      const Stat *s = stats_of(p, 0, row);
      sp = s[0];
      for (int k = 1; k < p.parts; ++k) sp = join(sp, s[k], tp, table);
      if (tp.greedy || sp.max == kNegInf) sp.sum = 1.0;
      if (lane < m) {
        if (p.draft) {
          s = stats_of(p, 1, row);
          sq = s[0];
          for (int k = 1; k < p.parts; ++k) sq = join(sq, s[k], tq, table);
          if (tq.greedy || sq.max == kNegInf) sq.sum = 1.0;
        }
        y = p.proposals[row];
        bad_token = y < 0 || y >= p.vocab;
        const float u = p.uniform[row];
        bad_number = !(u >= 0.f && u < 1.f);
        if (!bad_token) {
          auto at = [&](const void *rows, int64_t stride) {
            const float z = to_f32<T>(static_cast<const T *>(rows)[row * stride + y]);
            return z == z ? z : kNegInf;
          };
          const double wp = weight(at(p.target, p.target_stride), y, sp, tp, table);
          const double wq = p.draft ? weight(at(p.draft, p.draft_stride), y, sq, tq, table) : 1.0;
          py = wp / sp.sum;
          ok = !bad_number && static_cast<double>(u) * (wq / sq.sum) < py;
        }
      }
    }
    const uint64_t miss = ~__ballot(ok);
    const int a = min(miss ? static_cast<int>(__builtin_ctzll(miss)) : 64, m);
    if (lane == min(a, p.w - 1)) {
      chain.p = sp;
      chain.q = sq;
      chain.accepted = a;
      chain.y = bad_token ? -1 : y;
      chain.drawn = a == p.w ? kNothing : a == m ? kPlain : kLeft;
    }
    if (part == 0) {
      const float u = p.draw[b];
      const bool bad_draw = lane == 0 && a < p.w && !(u >= 0.f && u < 1.f);
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
        const int64_t row = static_cast<int64_t>(b) * p.w + lane;
        if (p.emitted) p.emitted[row] = y;
        if (p.probs) p.probs[row] = static_cast<float>(py);
      }
    }
  }
  __syncthreads();
  const Chain ch = chain;
  if (part == 0 && threadIdx.x == 0) *chain_of(p, b) = ch;
  if (ch.drawn == kNothing) return;
  const double total = part_sum<T>(p, b, part, ch, tp, tq, table, seg);
  if (threadIdx.x == 0) lefts_of(p, b)[part] = total;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void accept_draw_kernel(SampledAcceptParams p) {
  __shared__ double table[32], seg[kVec * kWavesA];
  __shared__ int answer;
  const int b = blockIdx.x;
  Chain ch = *chain_of(p, b);
  if (ch.drawn == kNothing) return;
  bool bad;  // reported before
  const Temper tp = temper(p.temperature, b, &bad);
  const Temper tq = p.draft ? temper(p.draft_temperature, b, &bad) : Temper{0.0, true};
  fill_table(table);
  const double *lefts = lefts_of(p, b);
  double total = 0.0;
  for (int k = 0; k < p.parts; ++k) total += lefts[k];
  const bool none = total == 0.0;  // p does not exceed q anywhere: a token of p
  if (none) {
    ch.drawn = kPlain;
    for (int k = 0; k < p.parts; ++k) total += part_sum<T>(p, b, k, ch, tp, tq, table, seg);
  }
  const double target = share_of(p, b, total);
  int part = 0;
  double before = 0.0, run = 0.0;
  for (int k = 0; k < p.parts; ++k) {
    const double w = none ? part_sum<T>(p, b, k, ch, tp, tq, table, seg) : lefts[k];
    if (w > 0.0) {
      part = k;
      before = run;
      if (target < run + w) break;
    }
    run += w;
  }
  __syncthreads();
  const int token = min(max(pick<T>(p, b, part, before, target, ch, tp, tq, table, seg, &answer), 0), p.vocab - 1);
  if (threadIdx.x == 0) emit_drawn<T>(p, b, token, ch, tp, table);
}

template <typename T>
hipError_t launch_typed(const SampledAcceptParams &p, hipStream_t s) {
  const int64_t rows = static_cast<int64_t>(p.batch) * p.w * (p.draft ? 2 : 1);
  hipError_t e = launch_kernel(accept_stats_kernel<T>, dim3(static_cast<unsigned>(rows * p.parts)), dim3(kThreads), s, p);
  if (e != hipSuccess) return e;
  e = launch_kernel(accept_chain_kernel<T>, dim3(static_cast<unsigned>(p.batch) * p.parts), dim3(kThreads), s, p);
  if (e != hipSuccess) return e;
  return launch_kernel(accept_draw_kernel<T>, dim3(p.batch), dim3(kThreads), s, p);
}

}  // namespace

hipError_t launch_sampled_accept(const SampledAcceptParams &p, int dtype, hipStream_t s) {
  return dtype == DAS_F32 ? launch_typed<float>(p, s) : launch_typed<bf16_t>(p, s);
}

}  // namespace das
