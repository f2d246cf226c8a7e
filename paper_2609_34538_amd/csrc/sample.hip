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
// One workgroup per row, several passes over it; the first reads memory, the others
// the caches. No row is sorted: a cut in the order is found by counting (top-k) or
// weighing (top-p) the row in 2048 bins of equal width below m, and then among the
// tokens of the one bin that holds the cut, by comparing them with each other; a bin
// with too many tokens for that (rows of many equal logits) is searched by the bytes
// of its keys. The last pass weighs the kept tokens of every block of 512; the block
// that holds the drawn one is gone through once more by one wave.

#include "q8_internal.h"

namespace das {
namespace {

constexpr int kThreads = 1024;
constexpr int kWavesS = kThreads / 64;
constexpr int kBlock = 512;                     // tokens of a wave's step
constexpr int kMaxBlocks = DAS_MAX_VOCAB / kBlock;
constexpr int kBins = 2048;
constexpr int kList = 2048;                     // tokens that are compared with each other
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

// 8 logits from index i of a row of n (-inf past its end).
template <typename T>
__device__ __forceinline__ void load8(const T *row, int i, int n, float (&z)[8]) {
  T raw[8];
  if (i + 8 <= n) {
    __builtin_memcpy(raw, row + i, sizeof(raw));
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = to_f32<T>(raw[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = i + j < n ? to_f32<T>(row[i + j]) : kNegInf;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) z[j] = z[j] == z[j] ? z[j] + 0.f : kNegInf;
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
  __device__ __forceinline__ uint64_t weight(float z) const {
    return z == best ? static_cast<uint64_t>(kOne)
                     : weight_of((static_cast<double>(z) - static_cast<double>(best)) * c);
  }
};

struct Shared {
  union {
    struct {
      union {
        uint64_t weight[kBins];
        uint32_t count[kBins];
      } bin;
      uint32_t list_key[kList];
      uint64_t list_weight[kList];
    } cut;
    struct {
      uint64_t above[kMaxBlocks];  // kept weights above the cut key, per block
      uint32_t ties[kMaxBlocks];   // tokens at the cut key
    } last;
  };
  uint64_t part[kWavesS];
  uint32_t part32[kWavesS];
  uint64_t answer64;
  uint32_t answer32, answer_ties, n_list;
  int at;
};

__device__ __forceinline__ uint64_t shfl_up64(uint64_t x, int d) {
  return static_cast<uint64_t>(__shfl_up(static_cast<unsigned long long>(x), d, 64));
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t y = shfl_up64(x, d);
    if (lane >= d) x += y;
  }
  return x;
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1)
    x += static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(x), d, 64));
  return x;
}
// Exclusive prefix sum over the workgroup; *total is the sum.
__device__ __forceinline__ uint64_t block_scan(uint64_t x, Shared &sh, uint64_t *total) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint64_t incl = wave_scan(x, lane);
  __syncthreads();  // the previous call's parts have been read
  if (lane == 63) sh.part[wave] = incl;
  __syncthreads();
  uint64_t before = 0, all = 0;
#pragma unroll
  for (int k = 0; k < kWavesS; ++k) {
    const uint64_t v = sh.part[k];
    if (k < wave) before += v;
    all += v;
  }
  *total = all;
  return before + incl - x;
}

// fn(first index, 8 logits) over the whole row, a wave on 512 neighbouring tokens.
template <typename T, typename Fn>
__device__ __forceinline__ void for_row(const T *row, int n, Fn &&fn) {
  for (int i = threadIdx.x * 8; i < (n + kBlock - 1) / kBlock * kBlock; i += kThreads * 8) {
    float z[8];
    load8<T>(row, i, n, z);
    fn(i, z);
  }
}

// The cut of an order statistic: with f a token's weight (WEIGH) or 1, over the tokens
// with key >= row.key (at row.key itself only row.ties of them), the largest key t such
// that the f of the keys >= t reach `target` (0 < target <= their sum; WEIGH: share of
// the sum), and how many tokens at t that takes. Moves row.key and row.ties there.
template <bool WEIGH, typename T>
__device__ void find_cut(const T *row, int n, Row &r, uint32_t count, float share, Shared &sh) {
  const int tid = threadIdx.x, lane = tid % 64;
  // bins of equal width below the maximum; weights further down than the last are 0
  const float width = static_cast<float>(r.c) * (kBins / 44.f);
  auto bin_of = [&](float z) {
    const float d = (r.best - z) * width;  // NaN where both are infinite: bin 0
    return d < kBins - 1 ? static_cast<int>(d) : d >= kBins - 1 ? kBins - 1 : 0;
  };
  for (int i = tid; i < kBins; i += kThreads) {
    if (WEIGH) sh.cut.bin.weight[i] = 0;
    else sh.cut.bin.count[i] = 0;
  }
  if (tid == 0) sh.n_list = 0;
  __syncthreads();
  for_row<T>(row, n, [&](int i, const float (&z)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (i + j >= n || key_of(z[j]) < r.key) continue;
      if (WEIGH) {
        if (key_of(z[j]) == r.key) continue;  // added below, as many as count
        const uint64_t w = r.weight(z[j]);
        if (w) atomicAdd(reinterpret_cast<unsigned long long *>(&sh.cut.bin.weight[bin_of(z[j])]),
                         static_cast<unsigned long long>(w));
      } else {
        atomicAdd(&sh.cut.bin.count[bin_of(z[j])], 1u);
      }
    }
  });
  __syncthreads();
  const uint64_t tie_weight = WEIGH && r.ties ? r.weight(of_key(r.key)) : 0;
  if (WEIGH && tid == 0 && r.ties) sh.cut.bin.weight[bin_of(of_key(r.key))] += tie_weight * r.ties;
  __syncthreads();
  // the bin that reaches the target
  uint64_t a[kBins / kThreads], mine = 0, total;
#pragma unroll
  for (int k = 0; k < kBins / kThreads; ++k) {
    const int i = tid * (kBins / kThreads) + k;
    a[k] = WEIGH ? sh.cut.bin.weight[i] : sh.cut.bin.count[i];
    mine += a[k];
  }
  uint64_t before = block_scan(mine, sh, &total);
  uint64_t target = count;
  if (WEIGH) {
    const double q = __builtin_ceil(static_cast<double>(share) * static_cast<double>(total));
    target = q < 1.0 ? 1 : static_cast<uint64_t>(q);
  }
  if (target > total) target = total;
#pragma unroll
  for (int k = 0; k < kBins / kThreads; ++k) {
    if (before < target && before + a[k] >= target) {
      sh.at = tid * (kBins / kThreads) + k;
      sh.answer64 = target - before;
    }
    before += a[k];
  }
  __syncthreads();
  const int bin = sh.at;
  uint64_t rest = sh.answer64;  // to be reached within the bin, >= 1
  // its tokens
  for_row<T>(row, n, [&](int i, const float (&z)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t key = key_of(z[j]);
      if (i + j >= n || key < r.key || bin_of(z[j]) != bin) continue;
      if (WEIGH && key == r.key) continue;
      const uint32_t at = atomicAdd(&sh.n_list, 1u);
      if (at < kList) {
        sh.cut.list_key[at] = key;
        sh.cut.list_weight[at] = WEIGH ? r.weight(z[j]) : 1;
      }
    }
  });
  __syncthreads();
  const uint32_t listed = sh.n_list;
  __syncthreads();
  if (listed <= kList) {
    if (tid == 0) {
      // reached by none of the list: by the ties of the cut that was there
      sh.answer32 = r.key;
      sh.answer64 = rest;
      sh.answer_ties = 0;
    }
    __syncthreads();
    uint64_t all = 0;
    for (uint32_t i = tid; i < listed; i += kThreads) {
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
    return;
  }
  // too many: byte by byte of the key, from the top
  uint32_t prefix = 0;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kThreads) sh.cut.bin.weight[i] = 0;
    __syncthreads();
    for_row<T>(row, n, [&](int i, const float (&z)[8]) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t key = key_of(z[j]);
        bool in = i + j < n && key >= r.key && bin_of(z[j]) == bin;
        if (WEIGH) in = in && key != r.key;
        if (shift < 24) in = in && (key >> (shift + 8)) == prefix;
        const uint32_t digit = key >> shift & 255;
        const uint64_t voters = __builtin_amdgcn_ballot_w64(in);
        if (!voters) continue;
        // equal logits are what leads here: one addition for lanes with the same key
        const uint32_t lead = __builtin_amdgcn_readlane(key, __builtin_ctzll(voters));
        const uint64_t same = __builtin_amdgcn_ballot_w64(in && key == lead);
        if (in) {
          const uint64_t w = WEIGH ? r.weight(z[j]) : 1;
          const bool first = lane == __builtin_ctzll(same);
          if (key != lead || first)
            atomicAdd(reinterpret_cast<unsigned long long *>(&sh.cut.bin.weight[digit]),
                      static_cast<unsigned long long>(key != lead ? w : w * __builtin_popcountll(same)));
        }
      }
    });
    __syncthreads();
    if (WEIGH && tid == 0 && r.ties && bin_of(of_key(r.key)) == bin &&
        (shift == 24 || (r.key >> (shift + 8)) == prefix))
      sh.cut.bin.weight[r.key >> shift & 255] += tie_weight * r.ties;
    __syncthreads();
    const uint64_t w = tid < 256 ? sh.cut.bin.weight[255 - tid] : 0;  // from the top
    uint64_t all;
    const uint64_t over = block_scan(w, sh, &all);
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
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleParams p) {
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

  // the largest logit and its lowest index
  float best = kNegInf;
  int best_at = 0;
  for_row<T>(row, n, [&](int i, const float (&z)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (z[j] > best) best = z[j], best_at = i + j;
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
  for (int i = 0; i < kWavesS; ++i) top = sh.part[i] > top ? sh.part[i] : top;
  best = of_key(static_cast<uint32_t>(top >> 32));
  best_at = static_cast<int>(0xffffffffu - static_cast<uint32_t>(top));
  if (best == kNegInf) best_at = 0;  // nothing to choose from
  // greedy; numbers out of range, and rows without a finite or infinite logit, too
  if (T_raw == 0.f || !fine || best == kNegInf) {
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
  if (k > 0 && k < n) find_cut<false, T>(row, n, r, k, 0.f, sh);
  if (top_p < 1.f) find_cut<true, T>(row, n, r, 0, top_p, sh);
  const uint64_t cut_weight = r.weight(of_key(r.key));
  if (cut_weight < r.least) r.ties = 0;
  __syncthreads();

  // kept weights of every block of 512
  for_row<T>(row, n, [&](int i, const float (&z)[8]) {
    uint64_t sum = 0;
    uint32_t ties = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t key = key_of(z[j]);
      if (i + j < n && key > r.key) {
        const uint64_t w = r.weight(z[j]);
        sum += w >= r.least ? w : 0;
      }
      ties += i + j < n && key == r.key;
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) ties += __shfl_xor(ties, d, 64);
    if (lane == 0) {
      sh.last.above[i / kBlock] = sum;
      sh.last.ties[i / kBlock] = ties;
    }
  });
  __syncthreads();
  // their prefix sums: two blocks a thread
  const int blocks = (n + kBlock - 1) / kBlock;
  constexpr int PER = kMaxBlocks / kThreads;
  uint64_t ab[PER], ab_mine = 0;
  uint64_t ti[PER], ti_mine = 0;
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    const int i = tid * PER + q;
    ab[q] = i < blocks ? sh.last.above[i] : 0;
    ti[q] = i < blocks ? sh.last.ties[i] : 0;
    ab_mine += ab[q];
    ti_mine += ti[q];
  }
  uint64_t all_above, all_ties;
  uint64_t ab_before = block_scan(ab_mine, sh, &all_above);
  uint64_t ti_before = block_scan(ti_mine, sh, &all_ties);
  const uint64_t limit = r.ties;  // ties that are kept, at most all there are
  const uint64_t total = all_above + min(all_ties, limit) * cut_weight;
  uint64_t target = static_cast<uint64_t>(static_cast<double>(u) * static_cast<double>(total));
  if (target >= total) target = total - 1;
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    const uint64_t lo = ab_before + min(ti_before, limit) * cut_weight;
    const uint64_t hi = ab_before + ab[q] + min(ti_before + ti[q], limit) * cut_weight;
    if (lo <= target && target < hi) {
      sh.at = tid * PER + q;
      sh.answer64 = lo;
      sh.answer32 = static_cast<uint32_t>(ti_before);
    }
    ab_before += ab[q];
    ti_before += ti[q];
  }
  __syncthreads();
  if (wave != 0) return;
  // the block that passes the target, by one wave
  const int i = sh.at * kBlock + lane * 8;
  float z[8];
  load8<T>(row, i, n, z);
  uint64_t w[8], mine = 0;
  uint32_t ties = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) ties += i + j < n && key_of(z[j]) == r.key;
  uint32_t rank = static_cast<uint32_t>(wave_scan(ties, lane)) - ties + sh.answer32;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t key = key_of(z[j]);
    w[j] = 0;
    if (i + j < n && key > r.key) w[j] = r.weight(z[j]);
    if (i + j < n && key == r.key) w[j] = rank++ < limit ? cut_weight : 0;
    if (w[j] < r.least) w[j] = 0;
    mine += w[j];
  }
  uint64_t run = sh.answer64 + wave_scan(mine, lane) - mine;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (run <= target && target < run + w[j]) {
      p.tokens[row_id] = i + j;
      if (p.probs) p.probs[row_id] = static_cast<float>(static_cast<double>(w[j]) / static_cast<double>(total));
    }
    run += w[j];
  }
}

}  // namespace

hipError_t launch_sample(const SampleParams &p, int dtype, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(p.batch) * p.w), block(kThreads);
  if (dtype == DAS_F32) return launch_kernel(sample_kernel<float>, grid, block, s, p);
  return launch_kernel(sample_kernel<bf16_t>, grid, block, s, p);
}

}  // namespace das
