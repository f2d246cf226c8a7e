// A token for every row of logits, from a given random number (das_sample).
//
// With m the row's largest logit and T its temperature, token i weighs
// w_i = exp((z_i - m) / T). In the order (z descending, index ascending) top-k keeps
// the first k tokens, top-p of those the shortest run whose weights reach p of their
// sum, min-p of those the ones with w_i >= min_p. The drawn token is the first, in
// index order, whose running sum of kept weights passes u times their sum.
//
// Weights are integers, round(2^40 w_i) from a 64-bit exponential, so sums of up to
// 2^20 of them are exact in 64 bits and do not depend on their order: atomics, any
// split of a row and any sort of it give the same token.
//
// One workgroup per row (the call has no workspace to join parts of one through); the
// first pass reads memory, later ones the caches. What bounds it is a pass's vector and
// LDS work on one compute unit, not HBM: 1024 rows of 65536 bf16 logits take 70 us, 1.9
// TB/s. No row is sorted.
// - bf16 rows (sample_values) are counted by value in LDS; counts, one exponential per
//   value and a scan give every cut, a second pass adds up the looked-up weights of every
//   block of 512 tokens or more, and one wave goes once more through the block that holds
//   the drawn one (64 rows of 100003: 35 us).
// - fp32 rows, and bf16 ones whose logits that does not suit: a pass for the maximum, then
//   a cut in the order is found by counting (top-k) or weighing (top-p) the row in 2048
//   bins of equal width below it. Where few tokens lie above the end of the cut's bin, the
//   draw is made from the list of them (draw_few). Else the tokens of that bin are compared
//   with each other, or, too many for that (rows of many equal logits), searched by the
//   bytes of their keys; a pass weighs the kept tokens of every block as above.

#include "q8_internal.h"

namespace das {
namespace {

constexpr int kMaxThreads = 1024;
constexpr int kStep = 512;                      // tokens of a wave's step
constexpr int kMaxBlocks = 256;                 // blocks of a row, kStep << row_shift tokens each
constexpr int kBins = 2048;
constexpr int kList = 2048;                     // tokens that are compared with each other
constexpr int kFew = 512;                       // tokens that a draw is made from directly
constexpr float kNegInf = -__builtin_huge_valf();
constexpr double kOne = 0x1p40;                 // weight of the largest logit

// Order of the logits as unsigned integers: larger logits, larger keys. NaN was
// replaced by -inf and -0 by 0 before.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// 8 logits of a row as they lie in memory.
template <typename T>
struct Raw8 {
  uint32_t w[8 * sizeof(T) / 4];
};
// ... from index i of a row of n, -inf past its end.
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T *row, int i, int n) {
  Raw8<T> r;
  if (i + 8 <= n) {
    __builtin_memcpy(&r, row + i, sizeof(r));
    return r;
  }
  // all at once: one after the other they held a row's last wave up, and with it every pass
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
// Logit j of the eight, NaN as -inf and -0 as 0.
template <typename T>
__device__ __forceinline__ float logit(const Raw8<T> &r, int j) {
  float z;
  if constexpr (sizeof(T) == 2)
    z = __uint_as_float(j % 2 ? r.w[j / 2] & 0xffff0000u : r.w[j / 2] << 16);
  else
    z = __uint_as_float(r.w[j]);
  return z == z ? z + 0.f : kNegInf;
}

// 2^x for x <= 0 as round(2^40 2^x): 2^x = 2^n 2^f with |f| <= 1/2 and the series of
// e^(f ln 2) to f^11 (rest below 2^-47), in 64 bits; the addition of 2^52 rounds.
__device__ __forceinline__ uint64_t weight_of(double x) {
  if (!(x > -42.0)) return 0;
  const double n = __builtin_rint(x), f = x - n;
  double q = 4.4455382718708115e-10;
  q = __builtin_fma(q, f, 7.0549116208011233e-09);
  q = __builtin_fma(q, f, 1.0178086009239699e-07);
  q = __builtin_fma(q, f, 1.3215486790144309e-06);
  q = __builtin_fma(q, f, 1.5252733804059841e-05);
  q = __builtin_fma(q, f, 0.00015403530393381609);
  q = __builtin_fma(q, f, 0.0013333558146428443);
  q = __builtin_fma(q, f, 0.0096181291076284772);
  q = __builtin_fma(q, f, 0.055504108664821580);
  q = __builtin_fma(q, f, 0.24022650695910071);
  q = __builtin_fma(q, f, 0.69314718055994531);
  q = __builtin_fma(q, f, 1.0);
  const double w = __builtin_amdgcn_ldexp(q, static_cast<int>(n) + 40);
  return __builtin_bit_cast(uint64_t, w + 0x1p52) & 0xfffffffffffffull;
}

struct Row {
  float best;      // largest logit
  double c;        // log2(e) / T
  uint64_t least;  // min-p: smallest weight kept
  // cut of top-k and top-p: keys above `key` are kept, of those equal to it the first `ties`
  uint32_t key;
  uint32_t ties;
  // bins of equal width below the largest logit; weights further down than the last are 0
  float width;
  __device__ __forceinline__ int bin(float z) const {
    const float d = (best - z) * width;  // NaN where both are infinite: bin 0
    return static_cast<int>(fminf(fmaxf(d, 0.f), kBins - 1.f));
  }
  __device__ __forceinline__ uint64_t weight(float z) const {
    // infinities as 2^1000, so that they are 0 apart, and all others infinitely far
    return weight_of((fmin(static_cast<double>(z), 0x1p1000) - fmin(static_cast<double>(best), 0x1p1000)) * c);
  }
};

// The bins of a bf16 row, one for each value of 2^-9 <= |z| < 2^7, larger logits in
// lower bins: 0 for larger ones, kCentre for those around 0, kBottom for the rest.
constexpr int kSmall = 0x3b00, kLarge = 0x4300;  // bits of 2^-9 and 2^7
constexpr float kLowest = -128.f;
constexpr int kCentre = kLarge - kSmall + 1, kBottom = 2 * kCentre;
constexpr int kValues = kBottom + 1;
constexpr int kAround = 512;                     // tokens around 0 that a row may have

struct Blocks {
  unsigned long long above[kMaxBlocks];  // kept weights above the cut, per block
  uint32_t ties[kMaxBlocks];             // tokens at the cut
};
struct Few {
  uint64_t order;   // key and inverted index: larger comes first
  uint64_t weight;
};
struct Shared {
  union {
    struct {
      union {
        uint64_t weight[kBins];
        uint32_t count[kBins];
      } bin;
      union {
        struct {
          uint32_t list_key[kList];
          uint64_t list_weight[kList];
        };
        Few few[kFew];
      };
    } cut;
    struct {
      uint64_t weight[kValues];  // of a kept token of each bin
      union {
        uint32_t count[kValues];
        Blocks last;
      };
      int32_t centre[kAround];   // the tokens around 0, and their bits
      uint16_t centre_bits[kAround];
    } value;
    Blocks last;
  };
  uint64_t part[kMaxThreads / 64];
  uint32_t part32[kMaxThreads / 64];
  uint64_t answer64;
  uint32_t answer32, answer_ties, n_list;
  int at;
};

__device__ __forceinline__ uint64_t join(uint32_t lo, uint32_t hi) {
  return static_cast<uint64_t>(hi) << 32 | lo;
}
// x plus what CTRL brings from another lane, 0 where it brings nothing (and in the rows
// of 16 lanes outside ROWS).
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint64_t plus_dpp(uint64_t x) {
  const uint32_t lo = static_cast<uint32_t>(x), hi = static_cast<uint32_t>(x >> 32);
  return x + join(__builtin_amdgcn_update_dpp(0, lo, CTRL, ROWS, 0xf, false),
                  __builtin_amdgcn_update_dpp(0, hi, CTRL, ROWS, 0xf, false));
}
// Inclusive prefix sum over the wave: within rows of 16 lanes (shifts), then the row's
// last lane into the next row, and lane 31 into the upper half.
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {
  x = plus_dpp<0x111>(x);
  x = plus_dpp<0x112>(x);
  x = plus_dpp<0x114>(x);
  x = plus_dpp<0x118>(x);
  x = plus_dpp<0x142, 0xa>(x);
  return plus_dpp<0x143, 0xc>(x);
}
// Sum over the wave, in every lane: lanes 1 and 2 apart, mirrored in 8 and 16, then the
// swaps of 16 and 32 lanes.
__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
  x = plus_dpp<0xB1>(x);
  x = plus_dpp<0x4E>(x);
  x = plus_dpp<0x141>(x);
  x = plus_dpp<0x140>(x);
  uint32_t lo = static_cast<uint32_t>(x), hi = static_cast<uint32_t>(x >> 32);
  auto a = __builtin_amdgcn_permlane16_swap(lo, lo, false, false);
  auto b = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
  x = join(a[0], b[0]) + join(a[1], b[1]);
  lo = static_cast<uint32_t>(x), hi = static_cast<uint32_t>(x >> 32);
  a = __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
  b = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
  return join(a[0], b[0]) + join(a[1], b[1]);
}
// Exclusive prefix sum over the workgroup; *total is the sum.
template <int THREADS>
__device__ __forceinline__ uint64_t block_scan(uint64_t x, Shared &sh, uint64_t *total) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint64_t incl = wave_scan(x);
  __syncthreads();  // the previous call's parts have been read
  if (lane == 63) sh.part[wave] = incl;
  __syncthreads();
  // the waves' sums, scanned in a row of 16 lanes
  uint64_t v = lane < THREADS / 64 ? sh.part[lane] : 0;
  v = plus_dpp<0x111>(v);
  v = plus_dpp<0x112>(v);
  v = plus_dpp<0x114>(v);
  v = plus_dpp<0x118>(v);
  auto at = [&](int l) {
    return join(__builtin_amdgcn_readlane(static_cast<uint32_t>(v), l),
                __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), l));
  };
  *total = at(THREADS / 64 - 1);
  const int w = __builtin_amdgcn_readfirstlane(wave);
  return (w > 0 ? at(w - 1) : 0) + incl - x;
}

// fn(first index, 8 logits) over the whole row, a wave on 512 neighbouring tokens, the
// last of which may be past the end (-inf: no weight, and after every token in the order).
// The loads of a thread's next 16 or 8 tokens (bf16, fp32) are under way while it works
// on the ones before.
template <int THREADS, typename T, typename Fn>
__device__ __forceinline__ void for_row(const T *row, int n, Fn &&fn) {
  constexpr int GROUP = 4 / sizeof(T), STEP = THREADS * 8;
  const int lane8 = threadIdx.x % 64 * 8;
  Raw8<T> r[GROUP], next[GROUP];
  auto load = [&](int i0, Raw8<T> (&to)[GROUP]) {
#pragma unroll
    for (int c = 0; c < GROUP; ++c)
      if (i0 + c * STEP < n) to[c] = load8<T>(row, i0 + lane8 + c * STEP, n);
  };
  int i0 = threadIdx.x / 64 * kStep;  // uniform in the wave
  load(i0, r);
  for (; i0 < n; i0 += GROUP * STEP) {
    load(i0 + GROUP * STEP, next);
#pragma unroll
    for (int c = 0; c < GROUP; ++c)
      if (i0 + c * STEP < n) fn(i0 + lane8 + c * STEP, r[c]);
#pragma unroll
    for (int c = 0; c < GROUP; ++c) r[c] = next[c];
  }
}

// fn(index, logit) one token a lane at a time, for work that is long against a load (an
// exponential each); tokens past the end come as -inf. Two loads are ahead.
template <typename T, typename Fn>
__device__ __forceinline__ void for_each(const T *row, int n, int begin, int tokens, Fn &&fn) {
  const int i0 = begin + threadIdx.x % 64;
  auto load = [&](int i) {
    const float z = i < n ? to_f32<T>(row[i]) : kNegInf;
    return z == z ? z + 0.f : kNegInf;
  };
  float z0 = load(i0), z1 = load(i0 + 64);
#pragma unroll 1
  for (int i = i0; i < i0 + tokens; i += 64) {
    const float z2 = i + 128 < i0 + tokens ? load(i + 128) : 0.f;
    fn(i, z0);
    z0 = z1;
    z1 = z2;
  }
}

// fn(index, logit) for every token: eight at a time, or in fp32's place the compact loop
// for bf16 rows, which come here only when sample_values does not take them.
template <int THREADS, typename T, typename Fn>
__device__ __forceinline__ void for_tokens(const T *row, int n, Fn &&fn) {
  if constexpr (sizeof(T) == 2) {
    for (int i = threadIdx.x / 64 * kStep; i < n; i += THREADS / 64 * kStep)
      for_each<T>(row, n, i, kStep, fn);
  } else {
    for_row<THREADS, T>(row, n, [&](int i, const Raw8<T> &z8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) fn(i + j, logit<T>(z8, j));
    });
  }
}

// The draw from the tokens of the bins up to `last`, if there are few of them and they
// hold all that the filters keep: each is compared with every other, once for its place
// in the order (its rank and the weight before it), once for the kept weight before its
// index. `total`: what top-p takes its share of, or 0 for the sum of the first k. False
// if there are more than kFew. One pass and no exponentials but the list's, where cutting
// the row and weighing its blocks takes three and one for every token near the cut: 8 rows
// of 65536 fp32 logits with top-k 50 35 -> 24 us, and top-p 47 -> 24, top-p alone 58 -> 44,
// min-p alone 38 -> 16; 8 us lost where min-p keeps more.
template <int THREADS, typename T>
__device__ bool draw_few(const SampleParams &p, const T *row, int row_id, const Row &r, int last, uint32_t k,
                         float top_p, uint64_t total, float u, Shared &sh) {
  static_assert(kFew <= THREADS, "a token a thread");
  const int tid = threadIdx.x;
  if (tid == 0) sh.n_list = 0;
  __syncthreads();
  for_tokens<THREADS, T>(row, p.vocab, [&](int i, float z) {
    // once there are too many the count need not be right (its additions, one lane after
    // the other, would take longer than the pass)
    if (r.bin(z) > last || __hip_atomic_load(&sh.n_list, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) > kFew)
      return;
    const uint32_t at = atomicAdd(&sh.n_list, 1u);
    if (at < kFew) sh.cut.few[at].order = static_cast<uint64_t>(key_of(z)) << 32 | (0xffffffffu - i);
  });
  __syncthreads();
  const int listed = sh.n_list;
  if (listed > kFew) return false;
  uint64_t own = 0, w = 0, before = 0;
  uint32_t rank = 0;
  if (tid < listed) {
    own = sh.cut.few[tid].order;
    w = r.weight(of_key(static_cast<uint32_t>(own >> 32)));
    sh.cut.few[tid].weight = w;
  }
  __syncthreads();
  if (tid < listed) {
#pragma unroll 4
    for (int j = 0; j < listed; ++j) {
      const Few f = sh.cut.few[j];
      const bool first = f.order > own;
      rank += first;
      before += first ? f.weight : 0;
    }
  }
  const bool in_k = tid < listed && rank < k;
  if (!total) block_scan<THREADS>(in_k ? w : 0, sh, &total);
  uint64_t limit = total;
  if (top_p < 1.f) {
    const double q = __builtin_ceil(static_cast<double>(top_p) * static_cast<double>(total));
    limit = q < 1.0 ? 1 : min(static_cast<uint64_t>(q), total);
  }
  const uint64_t kept = in_k && before < limit && w >= r.least ? w : 0;
  uint64_t sum;
  block_scan<THREADS>(kept, sh, &sum);
  if (tid < listed) sh.cut.few[tid].weight = kept;
  __syncthreads();
  if (!kept) return true;
  uint64_t target = static_cast<uint64_t>(static_cast<double>(u) * static_cast<double>(sum));
  if (target >= sum) target = sum - 1;
  uint64_t run = 0;
#pragma unroll 4
  for (int j = 0; j < listed; ++j) {
    const Few f = sh.cut.few[j];
    run += static_cast<uint32_t>(f.order) > static_cast<uint32_t>(own) ? f.weight : 0;
  }
  if (run <= target && target < run + kept) {
    p.tokens[row_id] = static_cast<int>(0xffffffffu - static_cast<uint32_t>(own));
    if (p.probs) p.probs[row_id] = static_cast<float>(static_cast<double>(kept) / static_cast<double>(sum));
  }
  return true;
}

// The cut of an order statistic: with f a token's weight (WEIGH) or 1, over the tokens
// with key >= row.key (at row.key itself only row.ties of them), the largest key t such
// that the f of the keys >= t reach `target` (0 < target <= their sum; WEIGH: share of
// the sum), and how many tokens at t that takes. Moves row.key and row.ties there. True
// if the draw has been made, since there are few tokens above the end of the cut's bin.
template <int THREADS, bool WEIGH, typename T>
__device__ bool find_cut(const SampleParams &p, const T *row, int row_id, Row &r, uint32_t count, float share,
                         float u, Shared &sh) {
  const int tid = threadIdx.x, lane = tid % 64, n = p.vocab;
  auto bin_of = [&](float z) { return r.bin(z); };
  for (int i = tid; i < kBins; i += THREADS) {
    if (WEIGH) sh.cut.bin.weight[i] = 0;
    else sh.cut.bin.count[i] = 0;
  }
  __syncthreads();
  const int wave = tid / 64;
  // in the order of the keys, as no logit is NaN or -0; NaN where there is no cut yet
  const float cut = of_key(r.key);
  if constexpr (WEIGH) {
    for_tokens<THREADS, T>(row, n, [&](int, float z) {
      if (z <= cut) return;  // those equal are added below, as many as count
      const uint64_t w = r.weight(z);
      if (w) atomicAdd(reinterpret_cast<unsigned long long *>(&sh.cut.bin.weight[bin_of(z)]),
                       static_cast<unsigned long long>(w));
    });
  } else {
    for_tokens<THREADS, T>(row, n, [&](int, float z) {
      if (!(z < cut)) atomicAdd(&sh.cut.bin.count[bin_of(z)], 1u);
    });
  }
  __syncthreads();
  const uint64_t tie_weight = WEIGH && r.ties ? r.weight(of_key(r.key)) : 0;
  if (WEIGH && tid == 0 && r.ties) sh.cut.bin.weight[bin_of(of_key(r.key))] += tie_weight * r.ties;
  __syncthreads();
  // the bin that reaches the target
  uint64_t a[kBins / THREADS], mine = 0, total;
#pragma unroll
  for (int k = 0; k < kBins / THREADS; ++k) {
    const int i = tid * (kBins / THREADS) + k;
    a[k] = WEIGH ? sh.cut.bin.weight[i] : sh.cut.bin.count[i];
    mine += a[k];
  }
  uint64_t before = block_scan<THREADS>(mine, sh, &total);
  uint64_t target = WEIGH ? 0 : count;
  if (WEIGH) {
    const double q = __builtin_ceil(static_cast<double>(share) * static_cast<double>(total));
    target = q < 1.0 ? 1 : static_cast<uint64_t>(q);
  }
  if (target > total) target = total;
#pragma unroll
  for (int k = 0; k < kBins / THREADS; ++k) {
    if (before < target && before + a[k] >= target) {
      sh.at = tid * (kBins / THREADS) + k;
      sh.answer64 = target - before;
      sh.answer32 = static_cast<uint32_t>(min(before + a[k], static_cast<uint64_t>(kFew + 1)));
    }
    before += a[k];
  }
  __syncthreads();
  const int bin = sh.at;
  uint64_t rest = sh.answer64;  // to be reached within the bin, >= 1
  // a token weighs kOne at most: more weight up to the cut than kFew of them have, more tokens
  if (WEIGH ? target <= kFew * static_cast<uint64_t>(kOne) : sh.answer32 <= kFew) {
    if (draw_few<THREADS, T>(p, row, row_id, r, bin, count, share, WEIGH ? total : 0, u, sh)) return true;
  }
  __syncthreads();
  if (tid == 0) sh.n_list = 0;
  __syncthreads();
  // the bin's tokens
  for_tokens<THREADS, T>(row, n, [&](int, float z) {
    const uint32_t key = key_of(z);
    if (key < r.key || bin_of(z) != bin || (WEIGH && key == r.key)) return;
    const uint32_t at = atomicAdd(&sh.n_list, 1u);
    if (at < kList) sh.cut.list_key[at] = key;
  });
  __syncthreads();
  const uint32_t listed = sh.n_list;
  if (listed <= kList) {
    for (uint32_t i = tid; i < listed; i += THREADS)
      sh.cut.list_weight[i] = WEIGH ? r.weight(of_key(sh.cut.list_key[i])) : 1;
    if (tid == 0) {
      // reached by none of the list: by the ties of the cut that was there
      sh.answer32 = r.key;
      sh.answer64 = rest;
      sh.answer_ties = 0;
    }
    __syncthreads();
    uint64_t all = 0;
    for (uint32_t i = tid; i < listed; i += THREADS) {
      const uint32_t key = sh.cut.list_key[i];
      uint64_t above = 0, equal = 0;
      all = 0;
      for (uint32_t j = 0; j < listed; ++j) {
        const uint64_t w = sh.cut.list_weight[j];
        const uint32_t kj = sh.cut.list_key[j];
        above += kj > key ? w : 0;
        equal += kj == key ? w : 0;
        all += w;
      }
      if (above < rest && above + equal >= rest) {  // equal keys write the same values
        const uint64_t w = sh.cut.list_weight[i];
        sh.answer32 = key;
        sh.answer_ties = static_cast<uint32_t>((rest - above + w - 1) / w);
      }
      if (i == 0) sh.answer64 = all;
    }
    __syncthreads();
    if (WEIGH && sh.answer_ties == 0) {
      const uint64_t left = rest - (listed ? sh.answer64 : 0);
      r.ties = min(r.ties, static_cast<uint32_t>((left + tie_weight - 1) / tie_weight));
    } else {
      r.key = sh.answer32;
      r.ties = sh.answer_ties;
    }
    __syncthreads();
    return false;
  }
  // too many: byte by byte of the key, from the top
  uint32_t prefix = 0;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += THREADS) sh.cut.bin.weight[i] = 0;
    __syncthreads();
    for (int i0 = wave * kStep; i0 < n; i0 += THREADS / 64 * kStep) {
      for_each<T>(row, n, i0, kStep, [&](int, float z) {
        const uint32_t key = key_of(z);
        bool in = key >= r.key && bin_of(z) == bin;
        if (WEIGH) in = in && key != r.key;
        if (shift < 24) in = in && (key >> (shift + 8)) == prefix;
        const uint32_t digit = key >> shift & 255;
        const uint64_t voters = __builtin_amdgcn_ballot_w64(in);
        if (!voters) return;
        // equal logits are what leads here: one addition for lanes with the same key
        const uint32_t lead = __builtin_amdgcn_readlane(key, __builtin_ctzll(voters));
        const uint64_t same = __builtin_amdgcn_ballot_w64(in && key == lead);
        if (in) {
          const uint64_t w = WEIGH ? r.weight(z) : 1;
          const bool first = lane == __builtin_ctzll(same);
          if (key != lead || first)
            atomicAdd(reinterpret_cast<unsigned long long *>(&sh.cut.bin.weight[digit]),
                      static_cast<unsigned long long>(key != lead ? w : w * __builtin_popcountll(same)));
        }
      });
    }
    __syncthreads();
    if (WEIGH && tid == 0 && r.ties && bin_of(of_key(r.key)) == bin &&
        (shift == 24 || (r.key >> (shift + 8)) == prefix))
      sh.cut.bin.weight[r.key >> shift & 255] += tie_weight * r.ties;
    __syncthreads();
    const uint64_t w = tid < 256 ? sh.cut.bin.weight[255 - tid] : 0;  // from the top
    uint64_t all;
    const uint64_t over = block_scan<THREADS>(w, sh, &all);
    if (over < rest && over + w >= rest) {
      sh.at = 255 - tid;
      sh.answer64 = rest - over;
    }
    __syncthreads();
    prefix = prefix << 8 | static_cast<uint32_t>(sh.at);
    rest = sh.answer64;
    __syncthreads();
  }
  const uint64_t w = WEIGH ? r.weight(of_key(prefix)) : 1;
  r.key = prefix;
  r.ties = static_cast<uint32_t>((rest + w - 1) / w);
  return false;
}

// Tokens of a block: the fewest doublings of a step that leave kMaxBlocks of them.
__device__ __forceinline__ int row_shift(int n) {
  int s = 9;
  static_assert(kStep == 1 << 9 && (DAS_MAX_VOCAB >> 9) / kMaxBlocks <= 32, "few doublings");
  while ((n - 1) >> s >= kMaxBlocks) ++s;
  return s;
}
template <int THREADS>
__device__ __forceinline__ void clear(Blocks &blk) {
  for (int i = threadIdx.x; i < kMaxBlocks; i += THREADS) blk.above[i] = 0, blk.ties[i] = 0;
  __syncthreads();
}
// A wave's step of block b: its weights (below 2^50) and ties, in one sum over the wave.
__device__ __forceinline__ void add_step(Blocks &blk, int b, uint64_t sum, uint32_t ties) {
  sum += static_cast<uint64_t>(ties) << 52;
  if (__builtin_amdgcn_ballot_w64(sum != 0) == 0) return;
  sum = wave_sum(sum);
  if (threadIdx.x % 64 != 0) return;
  atomicAdd(&blk.above[b], static_cast<unsigned long long>(sum & 0xfffffffffffffull));
  if (sum >> 52) atomicAdd(&blk.ties[b], static_cast<uint32_t>(sum >> 52));
}

// The drawn token from the sums of the blocks: `above(z)` is the weight of a token that is
// kept whatever its index (else 0), the tokens with `tie(z)` weigh tie_weight each, the
// first `limit` of them are kept. The block that passes the target is gone through once
// more by one wave.
template <int THREADS, typename T, typename Above, typename Tie>
__device__ __forceinline__ void pick(const SampleParams &p, const T *row, int row_id, float u, bool greedy,
                                     uint64_t tie_weight, uint32_t limit, const Blocks &blk, Shared &sh,
                                     Above &&above, Tie &&tie) {
  const int tid = threadIdx.x, lane = tid % 64, n = p.vocab, shift = row_shift(n);
  static_assert(kMaxBlocks <= THREADS, "a block a thread");
  __syncthreads();
  const uint64_t ab = tid < kMaxBlocks ? blk.above[tid] : 0, ti = tid < kMaxBlocks ? blk.ties[tid] : 0;
  uint64_t all_above, all_ties = 0, ti_before = 0;
  const uint64_t ab_before = block_scan<THREADS>(ab, sh, &all_above);
  if (limit) ti_before = block_scan<THREADS>(ti, sh, &all_ties);
  const uint64_t most = limit;
  const uint64_t total = all_above + min(all_ties, most) * tie_weight;
  uint64_t target = static_cast<uint64_t>(static_cast<double>(u) * static_cast<double>(total));
  if (target >= total) target = total - 1;
  const uint64_t lo = ab_before + min(ti_before, most) * tie_weight;
  const uint64_t hi = ab_before + ab + min(ti_before + ti, most) * tie_weight;
  if (lo <= target && target < hi) {
    sh.at = tid;
    sh.answer64 = lo;
    sh.answer32 = static_cast<uint32_t>(ti_before);
  }
  __syncthreads();
  if (tid >= 64) return;
  uint64_t run = sh.answer64;
  uint32_t rank = sh.answer32;
  // 8 tokens a lane: their sums, and in the step that passes the target each of them
#pragma unroll 1
  for (int i0 = sh.at << shift; i0 < n; i0 += kStep) {
    const int i = i0 + 8 * lane;
    const Raw8<T> z8 = load8<T>(row, i, n);
    uint64_t sum = 0, w[8];
    uint32_t ties = 0;
    bool at_cut[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = logit<T>(z8, j);
      at_cut[j] = limit && tie(x);
      w[j] = !at_cut[j] && i + j < n ? above(x) : 0;
      ties += at_cut[j];
      sum += w[j];
    }
    const uint32_t ties_before = rank + static_cast<uint32_t>(wave_scan(ties)) - ties;
    const uint32_t ties_kept = min(ties_before + ties, limit) - min(ties_before, limit);
    sum += ties_kept * tie_weight;
    uint64_t w_run = run + wave_scan(sum) - sum;
    const uint64_t end = run + wave_sum(sum);
    if (target < end) {
      uint32_t own = ties_before;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (at_cut[j]) w[j] = own++ < limit ? tie_weight : 0;
        if (w_run <= target && target < w_run + w[j]) {
          p.tokens[row_id] = i + j;
          if (p.probs)
            p.probs[row_id] = greedy ? 1.f : static_cast<float>(static_cast<double>(w[j]) / static_cast<double>(total));
        }
        w_run += w[j];
      }
      return;
    }
    run = end;
    rank += static_cast<uint32_t>(wave_sum(ties));
  }
}

// The bin of a bf16 logit; a positive NaN counts as a large logit, a negative one as a
// small one (rows with large logits are left to the other way).
__device__ __forceinline__ int value_bin(uint32_t h) {
  const int t = min(max(static_cast<int>(h & 0x7fffu), kSmall - 1), kLarge) - (kSmall - 1);
  return h & 0x8000u ? kCentre + t : kCentre - t;
}
// The same for two logits in a word, times 2^SHIFT (offsets into a table), and |z| - 2^-9 in
// steps, 0 for the tokens around 0. Seven packed instructions for the two, no selections
// (ten: 64 rows of 100003 38 us, not 35).
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <int SHIFT>
__device__ __forceinline__ u16x2 value_offsets(uint32_t w, u16x2 &steps) {
  static_assert((kValues - 1) << SHIFT <= 0xffff, "offsets fit");
  const u16x2 a = __builtin_bit_cast(u16x2, w & 0x7fff7fffu);
  steps = __builtin_elementwise_min(__builtin_elementwise_sub_sat(a, u16x2{kSmall - 1, kSmall - 1}),
                                    u16x2{kCentre, kCentre});
  // -2^SHIFT for positive ones, 2^SHIFT for negative ones
  const u16x2 by = (__builtin_bit_cast(u16x2, __builtin_bit_cast(i16x2, w) >> 15) & static_cast<uint16_t>(2 << SHIFT)) -
                   static_cast<uint16_t>(1 << SHIFT);
  return steps * by + static_cast<uint16_t>(kCentre << SHIFT);
}
template <typename E>
__device__ __forceinline__ E *at_offset(E *table, uint32_t bytes) {
  return reinterpret_cast<E *>(reinterpret_cast<char *>(table) + bytes);
}
// Two bf16 as signed integers in their order.
__device__ __forceinline__ i16x2 ordered(uint32_t w) {
  const i16x2 z = __builtin_bit_cast(i16x2, w);
  return z ^ ((z >> 15) & static_cast<int16_t>(0x7fff));
}
__device__ __forceinline__ float bin_value(int bin) {
  const uint32_t h = kSmall - 1 + (bin < kCentre ? kCentre - bin : (bin - kCentre) | 0x8000);
  return __uint_as_float(h << 16);
}

// A bf16 row by the counts of its values: there are few thousand of them in the range
// that logits have, so one pass of counting holds the order, every cut and, with one
// exponential per value, every sum; the last pass looks its weights up. Returns false
// (having done nothing) for rows out of that range: a largest logit of 2^7 or more, or
// within 2^-9 of 0, weights that matter below -2^7, many tokens within 2^-9 of 0, or a
// cut there. Those take the other way a token a lane at a time: 64 rows of 65536 logits
// without a filter 23 us here, 61 at temperature 30, 65 with 5536 tokens at 0, 102 with all
// logits around 130; with top-p 0.9 26, 133 and 356; 1024 rows 70, 296 and 397 us.
template <int THREADS>
__device__ bool sample_values(const SampleParams &p, const bf16_t *row, int row_id, float temperature, int k,
                              float top_p, float min_p, float u, bool greedy, Shared &sh) {
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, n = p.vocab;
  constexpr int PER = (kValues + THREADS - 1) / THREADS;
  for (int i = tid; i < kValues; i += THREADS) sh.value.count[i] = 0;
  if (tid == 0) sh.n_list = 0;
  __syncthreads();
  for_row<THREADS, bf16_t>(row, n, [&](int i, const Raw8<bf16_t> &z8) {
    u16x2 steps[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const u16x2 at = value_offsets<2>(z8.w[k], steps[k]);
      atomicAdd(at_offset<uint32_t>(sh.value.count, at[0]), 1u);
      atomicAdd(at_offset<uint32_t>(sh.value.count, at[1]), 1u);
    }
    const u16x2 least = __builtin_elementwise_min(__builtin_elementwise_min(steps[0], steps[1]),
                                                  __builtin_elementwise_min(steps[2], steps[3]));
    if (least[0] == 0 || least[1] == 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (steps[j / 2][j % 2] != 0) continue;
        const uint32_t at = atomicAdd(&sh.n_list, 1u);
        if (at < kAround) {
          sh.value.centre[at] = i + j;
          sh.value.centre_bits[at] = static_cast<uint16_t>(z8.w[j / 2] >> (16 * (j % 2)));
        }
      }
    }
  });
  __syncthreads();
  // a thread's bins, from the largest logits down
  const int bin0 = tid * PER, bin1 = min(bin0 + PER, kValues);
  int first = kBottom;
  for (int i = bin1 - 1; i >= bin0; --i)
    if (sh.value.count[i]) first = i;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) first = min(first, __shfl_xor(first, d, 64));
  if (lane == 0) sh.part32[wave] = first;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < (THREADS / 64); ++i) first = min(first, static_cast<int>(sh.part32[i]));
  const uint32_t centre = sh.n_list;
  if (first == 0 || first == kCentre || first == kBottom || centre > kAround) return false;
  Row r;
  r.best = bin_value(first);
  r.c = 1.4426950408889634074 / static_cast<double>(greedy ? 1.f : temperature);
  r.least = 1;
  if (min_p > 0.f && !greedy) r.least = static_cast<uint64_t>(__builtin_ceil(fmin(min_p, 1.f) * kOne));
  if (!greedy && r.weight(kLowest) != 0) return false;

  int cut = kBottom;       // bins above it are kept, of the cut the first `ties` tokens
  uint32_t ties = 0;
  uint64_t tie_weight = 1;
  if (greedy) {
    cut = first;
    ties = 1;
  } else {
    uint64_t mine = 0;     // the tokens around 0, whatever their filter
    for (uint32_t i = tid; i < centre; i += THREADS)
      mine += r.weight(bf16_to_f32(sh.value.centre_bits[i]));
    uint64_t centre_sum;
    block_scan<THREADS>(mine, sh, &centre_sum);
    uint64_t counts = 0, sums = 0, all, unused;
    uint64_t weights[PER], own[PER];  // of a token, and of all tokens of the thread's bins
    uint32_t held[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = bin0 + j;
      held[j] = i < bin1 ? sh.value.count[i] : 0;
      weights[j] = held[j] && i != kCentre && i < kBottom ? r.weight(bin_value(i)) : 0;
      own[j] = i < bin1 && i == kCentre ? centre_sum : weights[j] * held[j];
      if (i < bin1) sh.value.weight[i] = weights[j];
      counts += held[j];
      sums += own[j];
    }
    const uint64_t sums_before = block_scan<THREADS>(sums, sh, &all);
    uint64_t limit = all;  // weight that top-k leaves
    if (k > 0 && k < n) {
      uint64_t before = block_scan<THREADS>(counts, sh, &unused), sum = sums_before;
      const uint64_t want = static_cast<uint32_t>(k);
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        if (before < want && before + held[j] >= want) {
          sh.at = bin0 + j;
          sh.answer_ties = static_cast<uint32_t>(want - before);
          sh.answer64 = sum + weights[j] * (want - before);
          sh.answer32 = held[j];
        }
        before += held[j];
        sum += own[j];
      }
      __syncthreads();
      cut = sh.at;
      ties = sh.answer_ties;
      limit = sh.answer64;
      if (cut == kCentre) {
        if (ties != sh.answer32) return false;
        ++cut;             // all of it
        ties = 0;
        limit += centre_sum;
      }
      __syncthreads();
    }
    if (top_p < 1.f) {
      const double share = __builtin_ceil(static_cast<double>(top_p) * static_cast<double>(limit));
      uint64_t target = share < 1.0 ? 1 : static_cast<uint64_t>(share);
      if (target > limit) target = limit;
      uint64_t sum = sums_before;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        if (sum < target && sum + own[j] >= target) {
          sh.at = bin0 + j;
          sh.answer64 = target - sum;
        }
        sum += own[j];
      }
      __syncthreads();
      if (sh.at == kCentre) return false;
      cut = sh.at;
      const uint64_t w = sh.value.weight[cut];
      ties = static_cast<uint32_t>((sh.answer64 + w - 1) / w);
    }
    tie_weight = cut < kBottom && cut != kCentre ? sh.value.weight[cut] : 0;
    if (tie_weight < r.least) ties = 0;
  }
  __syncthreads();  // counts and weights have been read
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = bin0 + j;
    if (i >= bin1) break;
    const uint64_t w = i < cut && !greedy ? sh.value.weight[i] : 0;
    sh.value.weight[i] = w >= r.least ? w : 0;
  }
  __syncthreads();
  // kept weights and ties of the blocks; a step whose largest logit lies below the cut
  // (all but a few, where a filter is on) has none
  clear<THREADS>(sh.value.last);
  const int shift = row_shift(n);
  const int lowest = cut == kBottom ? -32768 : ordered(__float_as_uint(bin_value(cut)) >> 16)[0];
  for_row<THREADS, bf16_t>(row, n, [&](int i, const Raw8<bf16_t> &z8) {
    const i16x2 most = __builtin_elementwise_max(__builtin_elementwise_max(ordered(z8.w[0]), ordered(z8.w[1])),
                                                 __builtin_elementwise_max(ordered(z8.w[2]), ordered(z8.w[3])));
    if (__builtin_amdgcn_ballot_w64(max(most[0], most[1]) >= lowest) == 0) return;
    u16x2 at[4], steps;
#pragma unroll
    for (int k = 0; k < 4; ++k) at[k] = value_offsets<3>(z8.w[k], steps);
    uint64_t sum = 0;
    uint32_t at_cut = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += *at_offset<uint64_t>(sh.value.weight, at[j / 2][j % 2]);
    if (ties) {
#pragma unroll
      for (int j = 0; j < 8; ++j) at_cut += at[j / 2][j % 2] == cut << 3;
    }
    add_step(sh.value.last, i >> shift, sum, at_cut);
  });
  if (!greedy && kCentre < cut) {
    for (uint32_t i = tid; i < centre; i += THREADS) {
      const uint64_t w = r.weight(bf16_to_f32(sh.value.centre_bits[i]));
      if (w >= r.least)
        atomicAdd(&sh.value.last.above[sh.value.centre[i] >> shift], static_cast<unsigned long long>(w));
    }
  }
  pick<THREADS, bf16_t>(p, row, row_id, greedy ? 0.f : u, greedy, tie_weight, ties, sh.value.last, sh,
                        [&](float z) -> uint64_t {
                          const int bin = value_bin(__float_as_uint(z) >> 16);
                          if (bin != kCentre) return sh.value.weight[bin];
                          if (greedy || kCentre >= cut) return 0;
                          const uint64_t w = r.weight(z);
                          return w >= r.least ? w : 0;
                        },
                        [&](float z) { return value_bin(__float_as_uint(z) >> 16) == cut; });
  return true;
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(4))) void sample_kernel(SampleParams p) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int row_id = blockIdx.x, b = row_id / p.w, n = p.vocab;
  const T *row = static_cast<const T *>(p.logits) + static_cast<int64_t>(row_id) * p.row_stride;
  const float T_raw = p.temperature ? p.temperature[b] : 1.f;
  const int k = p.top_k ? p.top_k[b] : 0;
  const float top_p = p.top_p ? p.top_p[b] : 1.f, min_p = p.min_p ? p.min_p[b] : 0.f;
  const float u = p.uniform[row_id];
  const bool fine = T_raw >= 0.f && T_raw < __builtin_huge_valf() && top_p == top_p &&
                    min_p == min_p && u >= 0.f && u < 1.f;
  if (!fine && tid == 0) report_error(p.dev_error, DAS_DEVERR_SAMPLE);

  const bool greedy = T_raw == 0.f || !fine;
  if constexpr (sizeof(T) == 2) {
    if (sample_values<THREADS>(p, row, row_id, T_raw, k, top_p, min_p, u, greedy, sh)) return;
    __syncthreads();  // its last reads of the shared memory
  }

  // the largest logit and its lowest index
  float best = kNegInf;
  int best_at = 0;
  for_tokens<THREADS, T>(row, n, [&](int i, float z) {
    if (z > best) best = z, best_at = i;
  });
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const float o = __shfl_xor(best, d, 64);
    const int at = __shfl_xor(best_at, d, 64);
    if (o > best || (o == best && at < best_at)) best = o, best_at = at;
  }
  if (lane == 0) sh.part[wave] = static_cast<uint64_t>(key_of(best)) << 32 | (0xffffffffu - best_at);
  __syncthreads();
  uint64_t top = 0;
#pragma unroll
  for (int i = 0; i < (THREADS / 64); ++i) top = sh.part[i] > top ? sh.part[i] : top;
  best = of_key(static_cast<uint32_t>(top >> 32));
  best_at = static_cast<int>(0xffffffffu - static_cast<uint32_t>(top));
  if (best == kNegInf) best_at = 0;  // nothing to choose from
  // greedy; numbers out of range, and rows without a finite or infinite logit, too
  if (greedy || best == kNegInf) {
    if (tid == 0) {
      p.tokens[row_id] = best_at;
      if (p.probs) p.probs[row_id] = 1.f;
    }
    return;
  }

  Row r;
  r.best = best;
  r.c = 1.4426950408889634074 / static_cast<double>(T_raw);
  r.least = 1;
  if (min_p > 0.f) r.least = static_cast<uint64_t>(__builtin_ceil(fmin(min_p, 1.f) * kOne));
  r.key = 0;
  r.ties = 0;
  r.width = static_cast<float>(r.c) * (kBins / 44.f);
  const bool by_k = k > 0 && k < n;
  const uint32_t first = by_k ? k : 0xffffffffu;
  if (by_k && find_cut<THREADS, false, T>(p, row, row_id, r, first, top_p, u, sh)) return;
  if (top_p < 1.f && find_cut<THREADS, true, T>(p, row, row_id, r, first, top_p, u, sh)) return;
  if (min_p > 0.f && !by_k && !(top_p < 1.f)) {
    // the bins of what min-p keeps, and one for the rounding of a token's bin
    const float bins = -log2f(fminf(min_p, 1.f)) * (kBins / 44.f);
    const int last = bins < kBins - 2 ? static_cast<int>(bins) + 1 : kBins - 1;
    if (draw_few<THREADS, T>(p, row, row_id, r, last, first, 1.f, 0, u, sh)) return;
    __syncthreads();
  }
  const uint64_t cut_weight = r.weight(of_key(r.key));
  if (cut_weight < r.least) r.ties = 0;
  __syncthreads();
  clear<THREADS>(sh.last);
  const int shift = row_shift(n);
  const float cut = of_key(r.key);  // NaN: none
  auto above = [&](float z) -> uint64_t {
    if (z <= cut) return 0;
    const uint64_t w = r.weight(z);
    return w >= r.least ? w : 0;
  };
  auto tie = [&](float z) { return z == cut; };
  if constexpr (sizeof(T) == 4) {
    for_row<THREADS, T>(row, n, [&](int i, const Raw8<T> &z8) {
      uint64_t sum = 0;
      uint32_t ties = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float z = logit<T>(z8, j);
        sum += above(z);
        ties += tie(z);
      }
      add_step(sh.last, i >> shift, sum, r.ties ? ties : 0);
    });
  } else {
    for (int i0 = wave * kStep; i0 < n; i0 += THREADS / 64 * kStep) {
      uint64_t sum = 0;
      uint32_t ties = 0;
      for_each<T>(row, n, i0, kStep, [&](int, float z) {
        sum += above(z);
        ties += tie(z);
      });
      add_step(sh.last, i0 >> shift, sum, r.ties ? ties : 0);
    }
  }
  pick<THREADS, T>(p, row, row_id, u, false, cut_weight, r.ties, sh.last, sh, above, tie);
}

}  // namespace

// Up to a row for every compute unit: 1024 threads, a CU's waves; more rows: 512, two
// rows to a CU, one of which works while the other waits at a barrier. Rows of 65536 without
// a filter, 1024 against 512 threads: bf16 64 rows 24.2, 27.5 us, 256 25.2, 28.1, 257 44.0,
// 35.9, 1024 90, 71; fp32 256 45.7, 48.4, 257 76.6, 67.7, 1024 159, 137.
hipError_t launch_sample(const SampleParams &p, int dtype, hipStream_t s) {
  const int rows = p.batch * p.w;
  const dim3 grid(static_cast<unsigned>(rows));
  if (rows <= kNumCUs) {
    if (dtype == DAS_F32) return launch_kernel(sample_kernel<float, 1024>, grid, dim3(1024), s, p);
    return launch_kernel(sample_kernel<bf16_t, 1024>, grid, dim3(1024), s, p);
  }
  if (dtype == DAS_F32) return launch_kernel(sample_kernel<float, 512>, grid, dim3(512), s, p);
  return launch_kernel(sample_kernel<bf16_t, 512>, grid, dim3(512), s, p);
}

}  // namespace das
