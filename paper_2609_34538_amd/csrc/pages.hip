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
// entries that change are few (a step of w tokens moves about w / 64 pages a sequence).
// Bound by the launch and its dependent round trips.

#include "q8_internal.h"

namespace das {
namespace {

constexpr int kThreads = 1024;

// Inclusive prefix sum over the workgroup; *total is the sum. `part`: 16 words.
__device__ __forceinline__ int block_scan(int x, int *part, int *total) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  __syncthreads();  // the previous call's parts have been read
  if (lane == 63) part[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int k = 0; k < kThreads / 64; ++k) {
    if (k < wave) before += part[k];
    all += part[k];
  }
  *total = all;
  return x + before;
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

__global__ __launch_bounds__(kThreads) void pages_update_kernel(PagesParams p) {
  __shared__ int part[kThreads / 64];
  const int tid = threadIdx.x;
  const int F = *p.num_free;
  // what is given back, in all
  int R = 0;
  for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
    const Seq s = read_seq(p, b0 + tid);
    if (b0 + tid < p.batch && !s.ok) report_error(p.dev_error, DAS_DEVERR_PREFIX);
    int total;
    block_scan(s.ok ? max(s.held - s.need, 0) : 0, part, &total);
    R += total;
  }
  // a stack that cannot hold them all: nothing is moved
  const bool broken = F < 0 || F > p.num_pages || R > p.num_pages - F;
  if (broken) {
    if (tid == 0) report_error(p.dev_error, DAS_DEVERR_POOL);
  } else {
    const int top = F + R;
    int r0 = 0;
    if (R > 0) {
      for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
        const int b = b0 + tid;
        const Seq s = read_seq(p, b);
        const int back = s.ok ? max(s.held - s.need, 0) : 0;
        int total;
        int r = r0 + block_scan(back, part, &total) - back;
        r0 += total;
        int32_t *row = p.block_table + static_cast<size_t>(b) * p.max_pages;
        for (int c = s.need; back > 0 && c < s.held; ++c, ++r) {
          p.free_pages[top - 1 - r] = row[c];
          row[c] = -1;
        }
      }
    }
    __syncthreads();  // released pages are on the stack
    int j0 = 0, taken = 0;
    for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
      const int b = b0 + tid;
      const Seq s = read_seq(p, b);
      const int more = s.ok ? max(s.need - s.held, 0) : 0;
      int total;
      const int upto = block_scan(more, part, &total);
      const int incl = j0 + upto;  // at most batch * max_pages, which fits
      const bool served = incl <= top;
      int32_t *row = p.block_table + static_cast<size_t>(b) * p.max_pages;
      if (more > 0 && served)
        for (int c = s.held, j = incl - more; c < s.need; ++c, ++j) row[c] = p.free_pages[top - 1 - j];
      if (more > 0 && !served) report_error(p.dev_error, DAS_DEVERR_POOL);
      if (b < p.batch && s.ok && (more == 0 || served)) p.pages_held[b] = s.need;
      int given;
      block_scan(served ? more : 0, part, &given);
      taken += given;
      j0 += total;
    }
    if (tid == 0) *p.num_free = top - taken;
  }
  if (!p.slots) return;
  __syncthreads();  // tables and counts are written
  const int items = p.batch * p.w;
  for (int it = tid; it < items; it += kThreads) {
    const int b = it / p.w;
    const long pos = static_cast<long>(p.first[b]) + it % p.w;
    const int held = p.pages_held[b];
    int slot = -1;
    if (pos >= 0 && pos < p.lengths[b] && held <= p.max_pages && pos / kPage < held) {
      const int page = p.block_table[static_cast<size_t>(b) * p.max_pages + pos / kPage];
      if (page >= 0 && page < p.num_pages) slot = page * kPage + static_cast<int>(pos % kPage);
    }
    p.slots[it] = slot;
  }
}

}  // namespace

hipError_t launch_pages_update(const PagesParams &p, hipStream_t s) {
  return launch_kernel(pages_update_kernel, dim3(1), dim3(kThreads), s, p);
}

}  // namespace das
