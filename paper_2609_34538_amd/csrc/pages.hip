// Page bookkeeping of a batch on the device (das_pages_update): block tables, held
// counts, the stack of free pages and the slots of new positions, from the lengths
// that the sequences shall have.
//
// A sequence of length n holds ceil(n / 64) pages. Pages that a sequence holds past
// that go back first, then sequences that lack pages get them, in sequence order,
// each all it lacks or nothing: with inclusive prefix sums over the batch of what is
// given back (R in all) and of what is lacking, released page r goes to place
// F + R - 1 - r of the free stack and granted page j comes from place F + R - 1 - j, so
// that giving back undoes a grant exactly. A sequence is served when its inclusive
// sum is at most F + R.
//
// One workgroup: the prefix sums run over the batch 1024 sequences at a time, and the
// entries that change are few (a step of w tokens moves about w / 64 pages a sequence; a
// sequence with many is moved by its wave). Slots of few positions are written by the same
// workgroup, others by a grid of their own. Bound by the launch and its dependent round
// trips.

#include "q8_internal.h"

namespace das {
namespace {

constexpr int kThreads = 1024;

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int plus_dpp(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
// Inclusive prefix sums: in rows of 16 lanes, then from row to row.
__device__ __forceinline__ int row_scan(int x) {
  x = plus_dpp<0x111>(x);
  x = plus_dpp<0x112>(x);
  x = plus_dpp<0x114>(x);
  return plus_dpp<0x118>(x);
}
__device__ __forceinline__ int wave_scan(int x) {
  return plus_dpp<0x143, 0xc>(plus_dpp<0x142, 0xa>(row_scan(x)));
}
// Inclusive prefix sum over the workgroup; *total is the sum. `part`: 16 words.
__device__ __forceinline__ int block_scan(int x, int *part, int *total) {
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  x = wave_scan(x);
  __syncthreads();  // the previous call's parts have been read
  if (lane == 63) part[wave] = x;
  __syncthreads();
  const int v = row_scan(lane < kThreads / 64 ? part[lane] : 0);
  *total = __builtin_amdgcn_readlane(v, kThreads / 64 - 1);
  return x + (wave > 0 ? __builtin_amdgcn_readlane(v, wave - 1) : 0);
}

// fn(table entry, item) for `count` entries from `column` and `item` of
// every lane's sequence b: a lane by itself up to kOwn, else the whole wave.
constexpr int kOwn = 4;
// Slots that the bookkeeping's workgroup writes itself, rather than a grid in a launch of its
// own; a step's two calls: 32 x 32 slots 7.4 against 9.0 us, 4096 9.3 against 9.4, 128 x 64
// 12.2 against 10.4, 2000 x 64 79 against 19.5.
constexpr int kOwnSlots = 4096;
template <typename Fn>
__device__ __forceinline__ void for_entries(const PagesParams &p, int b, int count, int column, int item, Fn &&fn) {
  const int lane = threadIdx.x % 64;
  auto row = [&](int seq) { return p.block_table + static_cast<size_t>(seq) * p.max_pages; };
  for (int k = 0; k < (count <= kOwn ? count : 0); ++k) fn(row(b)[column + k], item + k);
  uint64_t many = __builtin_amdgcn_ballot_w64(count > kOwn);
  while (many) {
    const int l = __builtin_ctzll(many);
    many &= many - 1;
    const int n = __builtin_amdgcn_readlane(count, l), c = __builtin_amdgcn_readlane(column, l);
    const int first = __builtin_amdgcn_readlane(item, l), seq = __builtin_amdgcn_readlane(b, l);
    for (int k = lane; k < n; k += 64) fn(row(seq)[c + k], first + k);
  }
}

struct Seq {
  int held, need;
  bool ok;  // its numbers are in range
};
__device__ __forceinline__ Seq read_seq(const PagesParams &p, int b) {
  Seq s = {0, 0, false};
  if (b >= p.batch) return s;
  const int len = p.lengths[b];
  s.held = p.pages_held[b];
  s.need = len / kPage + (len % kPage != 0);
  s.ok = len >= 0 && s.need <= p.max_pages && s.held >= 0 && s.held <= p.max_pages;
  return s;
}

__device__ __forceinline__ int slot_of(const PagesParams &p, int b, int i) {
  const long pos = static_cast<long>(p.first[b]) + i;
  const int held = p.pages_held[b];
  if (pos < 0 || pos >= p.lengths[b] || held > p.max_pages || pos / kPage >= held) return -1;
  const int page = p.block_table[static_cast<size_t>(b) * p.max_pages + pos / kPage];
  return page >= 0 && page < p.num_pages ? page * kPage + static_cast<int>(pos % kPage) : -1;
}

__global__ __launch_bounds__(256) void page_slots_kernel(PagesParams p) {
  const int it = blockIdx.x * 256 + threadIdx.x;
  if (it < p.batch * p.w) p.slots[it] = slot_of(p, it / p.w, it % p.w);
}

__global__ __launch_bounds__(kThreads) void pages_update_kernel(PagesParams p) {
  __shared__ int part[kThreads / 64];
  __shared__ int s_back, s_taken;
  const int tid = threadIdx.x;
  if (tid == 0) s_back = s_taken = 0;
  const int F = *p.num_free;
  // what is given back, in all (at most batch * max_pages, which fits)
  int mine = 0;
  for (int b = tid; b < p.batch; b += kThreads) {
    const Seq s = read_seq(p, b);
    if (!s.ok) report_error(p.dev_error, DAS_DEVERR_PREFIX);
    else mine += max(s.held - s.need, 0);
  }
  __syncthreads();
  mine = wave_scan(mine);
  if (tid % 64 == 63 && mine) atomicAdd(&s_back, mine);
  __syncthreads();
  const int R = s_back;
  // a stack that cannot hold them all: nothing is moved
  if (F < 0 || F > p.num_pages || R > p.num_pages - F) {
    if (tid == 0) report_error(p.dev_error, DAS_DEVERR_POOL);
  } else {
    const int top = F + R;
    for (int b0 = 0, r0 = 0; R > 0 && b0 < p.batch; b0 += kThreads) {
      const Seq s = read_seq(p, b0 + tid);
      const int back = s.ok ? max(s.held - s.need, 0) : 0;
      int total;
      const int r = r0 + block_scan(back, part, &total) - back;
      r0 += total;
      for_entries(p, b0 + tid, back, s.need, r, [&](int32_t &entry, int item) {
        p.free_pages[top - 1 - item] = entry;
        entry = -1;
      });
    }
    __syncthreads();  // released pages are on the stack
    for (int b0 = 0, j0 = 0; b0 < p.batch; b0 += kThreads) {
      const int b = b0 + tid;
      const Seq s = read_seq(p, b);
      const int more = s.ok ? max(s.need - s.held, 0) : 0;
      int total;
      const int incl = j0 + block_scan(more, part, &total);
      j0 += total;
      const bool served = incl <= top;
      if (more > 0 && !served) report_error(p.dev_error, DAS_DEVERR_POOL);
      for_entries(p, b, served ? more : 0, s.held, incl - more,
                  [&](int32_t &entry, int item) { entry = p.free_pages[top - 1 - item]; });
      // sums grow along the batch, so the last served one's is what was taken
      if (served && more > 0) atomicMax(&s_taken, incl);
      if (b < p.batch && s.ok && (more == 0 || served)) p.pages_held[b] = s.need;
    }
    __syncthreads();
    if (tid == 0) *p.num_free = top - s_taken;
  }
  if (!p.slots || p.batch * p.w > kOwnSlots) return;
  __syncthreads();  // tables and counts are written
  for (int it = tid; it < p.batch * p.w; it += kThreads) p.slots[it] = slot_of(p, it / p.w, it % p.w);
}

}  // namespace

hipError_t launch_pages_update(const PagesParams &p, hipStream_t s) {
  const hipError_t e = launch_kernel(pages_update_kernel, dim3(1), dim3(kThreads), s, p);
  if (e != hipSuccess || !p.slots || p.batch * p.w <= kOwnSlots) return e;
  return launch_kernel(page_slots_kernel, dim3((p.batch * p.w + 255) / 256), dim3(256), s, p);
}

}  // namespace das
