// Host side of the 8-bit cache, the sampler and the page tables: argument validation,
// the attention's cut into chunks, and dispatch behind the C ABI of das.h. As in
// das_api.hip every check runs before the first HIP call.

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "q8_internal.h"

namespace das {
namespace {

bool aligned(const void *ptr, size_t a) { return reinterpret_cast<uintptr_t>(ptr) % a == 0; }

// Whether two arrays of `bytes` bytes share any.
bool overlap(const void *a, const void *b, size_t bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y ? y - x < bytes : x - y < bytes;
}

das_status check_cache(const das_cache_q8 *cache) {
  if (!cache) return DAS_ERR_NULL;
  const das_cache *c = &cache->base;
  if (!c->k_pool || !c->v_pool || !cache->k_exp || !cache->v_exp) return DAS_ERR_NULL;
  if (!aligned(c->k_pool, 16) || !aligned(c->v_pool, 16) || !aligned(cache->k_exp, 4) ||
      !aligned(cache->v_exp, 4))
    return DAS_ERR_ALIGN;
  if (c->dtype != DAS_F32 && c->dtype != DAS_BF16) return DAS_ERR_DTYPE;
  if (c->num_depths < 1 || c->num_depths > DAS_MAX_DEPTH) return DAS_ERR_SHAPE;
  if (c->num_layers < 1 || c->num_kv_heads < 1 || c->num_pages < 1) return DAS_ERR_SHAPE;
  if (c->num_kv_heads > 65535) return DAS_ERR_SHAPE;
  if (c->num_k_planes < 1 || c->num_v_planes < 1) return DAS_ERR_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128) return DAS_ERR_SHAPE;
  for (int r = 1; r <= c->num_depths; ++r) {
    if (c->k_plane[r] < -1 || c->k_plane[r] >= c->num_k_planes) return DAS_ERR_SHAPE;
    if (c->v_plane[r] < -1 || c->v_plane[r] >= c->num_v_planes) return DAS_ERR_SHAPE;
  }
  return DAS_OK;
}

das_status check_table(int batch, int max_pages) {
  if (batch < 1 || batch > 65535 || max_pages < 1) return DAS_ERR_SHAPE;
  if (max_pages > (1 << 24) || static_cast<long long>(batch) * max_pages > 0x7fffffffLL)
    return DAS_ERR_SHAPE;
  return DAS_OK;
}

das_status check_batch(const das_batch *b) {
  if (!b) return DAS_ERR_NULL;
  if (!b->prefix_len || !b->block_table) return DAS_ERR_NULL;
  if (!aligned(b->prefix_len, 4) || !aligned(b->block_table, 4) || !aligned(b->dev_error, 4))
    return DAS_ERR_ALIGN;
  return check_table(b->batch, b->max_pages_per_seq);
}

struct PlanQ8 {
  int rows, chunk_tiles, nsplit, piece_stride;
  size_t total;
};

// Cuts the units (sequence, KV head) of a call into chunks of equal length, one workgroup
// each, by the table's width. A chunk costs its start (three dependent round trips) and a
// record, and a second chunk of any unit the merge's launch, about 4 us in all, so
// - few tiles are one chunk (55 heads x 700 tokens, 22 tiles: 7.8 us against 9.5 in three;
//   fp32 tiles take several times the matrix-core time, and half as many of them),
// - and so are units that fill three quarters of the compute units (4 x 55 heads x
//   512-2048 tokens 15.6 against 19.7 us in two; 16 x 55 x 512-4096 77 against 84; 24 x 8
//   x 1-4099, dh 128, 26.6 against 25.3-27.8);
// - others are cut for a workgroup per CU, two for batches, whose lengths fill part of the
//   table (16 x 8 x 512-8192, 258 tiles: 2 chunks 89, 4 to 8 66, 16 74 us; 30011 tokens x
//   8: 20 to 30 chunks 17.5, 59 18.9), but for 16 tiles at least, 8 where there are few
//   (8 x 4000 tokens, 126 tiles: 8 tiles 9.7 us, 4 10.5, 16 11.1).
// - Waves with different rows share a chunk's tiles instead of taking them in turn: two
//   workgroups per CU, which is what is resident (4 x 8 x 16384 x 128 rows: 33 tiles 58
//   us, 24 69, 43 67), of 8 tiles at least, 4 with two such waves (96 rows, 81 tiles: 8
//   23 us, 4 29; 64 rows, 127 tiles: 4 17, 8 19).
// The width stands for the lengths, which only the device knows: sequences far shorter than
// their table get fewer chunks than would suit them (2 x 8 heads x 4000 tokens, one query:
// 9.6 us in a table of 63 pages, 14.2 of 512, 28.3 of 2048), and a long one among many units
// is one workgroup's work (24 x 8 heads, one sequence of 32768 tokens among 2048: 173 us,
// all of 2048 19).
das_status plan_attn(const das_cache_q8 *cache, const das_batch *b, int hq, int w, PlanQ8 *plan) {
  const das_cache *c = &cache->base;
  if (hq < 1 || hq % c->num_kv_heads != 0) return DAS_ERR_SHAPE;
  const int group = hq / c->num_kv_heads;
  if (group > 8) return DAS_ERR_UNSUPPORTED;
  if (w < 1 || w > DAS_MAX_BLOCK) return DAS_ERR_SHAPE;
  plan->rows = w * group;
  const int es = c->dtype == DAS_F32 ? 4 : 2;
  const int gr = q8_group_rows(plan->rows, c->head_dim, es);
  const long long n_rg = (plan->rows + gr - 1) / gr;
  const long long units = static_cast<long long>(b->batch) * c->num_kv_heads;
  const long long tiles = 2LL * b->max_pages_per_seq + (w + 31) / 32;
  const int rw = q8_row_waves(plan->rows, c->head_dim, es);
  const long long wgs = units * n_rg;  // of one chunk per unit
  const bool one = rw == 1 && (tiles <= (es == 2 ? 32 : 16) || 4 * wgs >= 3 * kNumCUs);
  const long long target = rw == 1 && b->batch == 1 ? kNumCUs : 2 * kNumCUs;
  const long long least = rw == 1 ? (wgs * ((tiles + 7) / 8) <= kNumCUs ? 8 : 16) : rw == 2 ? 4 : 8;
  long long ns = one ? 1 : std::max<long long>(1, target / wgs);
  const long long ct = std::max<long long>((tiles + ns - 1) / ns, least);
  ns = (tiles + ct - 1) / ct;
  if (units * n_rg * ns * 256 > 0xffffffffLL) return DAS_ERR_SHAPE;
  plan->chunk_tiles = static_cast<int>(ct);
  plan->nsplit = static_cast<int>(ns);
  plan->piece_stride = static_cast<int>(piece_record_bytes(plan->rows, c->head_dim, es));
  plan->total = std::max<size_t>(256, ns > 1 ? static_cast<size_t>(units) * ns * plan->piece_stride : 0);
  return DAS_OK;
}

}  // namespace
}  // namespace das

using namespace das;

extern "C" {

size_t das_attn_q8_workspace_bytes(const das_cache_q8 *cache, const das_batch *batch,
                                   int32_t num_q_heads, int32_t block_len) {
  if (check_cache(cache) != DAS_OK || check_batch(batch) != DAS_OK) return 0;
  PlanQ8 plan;
  if (plan_attn(cache, batch, num_q_heads, block_len, &plan) != DAS_OK) return 0;
  return plan.total;
}

das_status das_attn_q8(const das_cache_q8 *cache, const das_batch *batch, int32_t layer,
                       int32_t kappa, int32_t nu, int32_t num_q_heads, int32_t block_len,
                       const void *q, const void *k_blk, const void *v_blk, void *out, float *lse,
                       void *workspace, size_t workspace_bytes, hipStream_t stream) {
  das_status st = check_cache(cache);
  if (st != DAS_OK) return st;
  st = check_batch(batch);
  if (st != DAS_OK) return st;
  if (!q || !k_blk || !v_blk || !out) return DAS_ERR_NULL;
  if (!aligned(q, 16) || !aligned(k_blk, 16) || !aligned(v_blk, 16) || !aligned(out, 16) ||
      !aligned(lse, 4))
    return DAS_ERR_ALIGN;
  const das_cache *c = &cache->base;
  if (layer < 0 || layer >= c->num_layers) return DAS_ERR_SHAPE;
  if (kappa < 1 || kappa > c->num_depths || nu < 1 || nu > c->num_depths) return DAS_ERR_DEPTH;
  const int kplane = c->k_plane[kappa], vplane = c->v_plane[nu];
  if (kplane < 0 || vplane < 0) return DAS_ERR_DEPTH;
  PlanQ8 plan;
  st = plan_attn(cache, batch, num_q_heads, block_len, &plan);
  if (st != DAS_OK) return st;
  if (!workspace || workspace_bytes < plan.total || !aligned(workspace, 256)) return DAS_ERR_WORKSPACE;
  const int dh = c->head_dim;
  const size_t page_heads = static_cast<size_t>(c->num_kv_heads) * c->num_pages;
  const size_t k_at = static_cast<size_t>(kplane) * c->num_layers + layer;
  const size_t v_at = static_cast<size_t>(vplane) * c->num_layers + layer;
  AttnQ8Params p;
  p.k_layer = static_cast<const uint8_t *>(c->k_pool) + k_at * page_heads * kPage * dh;
  p.v_layer = static_cast<const uint8_t *>(c->v_pool) + v_at * page_heads * kPage * dh;
  p.k_exp = cache->k_exp + k_at * page_heads * kQ8GroupsPerPage;
  p.v_exp = cache->v_exp + v_at * page_heads * kQ8GroupsPerPage;
  p.q = q;
  p.kb = k_blk;
  p.vb = v_blk;
  p.out = out;
  p.lse = lse;
  p.prefix_len = batch->prefix_len;
  p.block_table = batch->block_table;
  p.dev_error = batch->dev_error;
  p.ws = static_cast<uint8_t *>(workspace);
  p.batch = batch->batch;
  p.hq = num_q_heads;
  p.hkv = c->num_kv_heads;
  p.group = num_q_heads / c->num_kv_heads;
  p.w = block_len;
  p.rows = plan.rows;
  p.num_pages = c->num_pages;
  p.max_pages = batch->max_pages_per_seq;
  p.chunk_tiles = plan.chunk_tiles;
  p.nsplit = plan.nsplit;
  p.piece_stride = plan.piece_stride;
  p.scale_log2 = static_cast<float>(1.4426950408889634074 / __builtin_sqrt(static_cast<double>(dh)));
  return launch_attn_q8(p, c->dtype, dh, stream) == hipSuccess ? DAS_OK : DAS_ERR_HIP;
}

das_status das_kv_append_q8(const das_cache_q8 *cache, const das_batch *batch, const void *k_new,
                            const void *v_new, int32_t w_max, const int32_t *num_new,
                            int32_t *len_out, hipStream_t stream) {
  das_status st = check_cache(cache);
  if (st != DAS_OK) return st;
  st = check_batch(batch);
  if (st != DAS_OK) return st;
  if (!k_new || !v_new || !num_new) return DAS_ERR_NULL;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(num_new, 4) || !aligned(len_out, 4))
    return DAS_ERR_ALIGN;
  if (w_max < 1 || w_max > DAS_MAX_BLOCK) return DAS_ERR_SHAPE;
  const das_cache *c = &cache->base;
  // the grid: one wave per (plane, layer, KV head), four per workgroup, keys and
  // values in separate workgroups; at most 2^32 - 1 work-items along x
  const long long per_plane = static_cast<long long>(c->num_layers) * c->num_kv_heads;
  constexpr long long kMost = 1 << 26;  // units that such a grid holds; the products fit 64 bits
  if (per_plane > kMost || c->num_k_planes > kMost || c->num_v_planes > kMost) return DAS_ERR_SHAPE;
  const long long blocks =
      (c->num_k_planes * per_plane + 3) / 4 + (c->num_v_planes * per_plane + 3) / 4;
  if (blocks * 256 > 0xffffffffLL) return DAS_ERR_SHAPE;
  // every workgroup of a sequence reads its length and count, one of them writes len_out
  const size_t per_seq = sizeof(int32_t) * static_cast<size_t>(batch->batch);
  if (len_out && (overlap(len_out, batch->prefix_len, per_seq) || overlap(len_out, num_new, per_seq)))
    return DAS_ERR_SHAPE;
  AppendQ8Params p;
  p.k_new = k_new;
  p.v_new = v_new;
  p.k_pool = static_cast<uint8_t *>(c->k_pool);
  p.v_pool = static_cast<uint8_t *>(c->v_pool);
  p.k_exp = cache->k_exp;
  p.v_exp = cache->v_exp;
  p.prefix_len = batch->prefix_len;
  p.block_table = batch->block_table;
  p.num_new = num_new;
  p.len_out = len_out;
  p.dev_error = batch->dev_error;
  p.batch = batch->batch;
  p.n_k_planes = c->num_k_planes;
  p.n_v_planes = c->num_v_planes;
  p.layers = c->num_layers;
  p.hkv = c->num_kv_heads;
  p.num_pages = c->num_pages;
  p.max_pages = batch->max_pages_per_seq;
  p.w_max = w_max;
  return launch_kv_append_q8(p, c->dtype, c->head_dim, stream) == hipSuccess ? DAS_OK : DAS_ERR_HIP;
}

das_status das_sample(int32_t batch, int32_t block_len, int32_t vocab, int32_t dtype,
                      const void *logits, int64_t row_stride, const float *temperature,
                      const int32_t *top_k, const float *top_p, const float *min_p,
                      const float *uniform, int32_t *tokens, float *probs, uint32_t *dev_error,
                      hipStream_t stream) {
  if (!logits || !uniform || !tokens) return DAS_ERR_NULL;
  if (dtype != DAS_F32 && dtype != DAS_BF16) return DAS_ERR_DTYPE;
  if (batch < 1 || batch > 65535 || block_len < 1 || block_len > DAS_MAX_BLOCK || vocab < 1 ||
      vocab > DAS_MAX_VOCAB || row_stride < vocab)
    return DAS_ERR_SHAPE;
  // every byte offset fits 64 bits
  if (row_stride > (INT64_MAX >> 3) / (static_cast<int64_t>(batch) * block_len)) return DAS_ERR_SHAPE;
  if (!aligned(logits, dtype == DAS_F32 ? 4 : 2) || !aligned(temperature, 4) || !aligned(top_k, 4) ||
      !aligned(top_p, 4) || !aligned(min_p, 4) || !aligned(uniform, 4) || !aligned(tokens, 4) ||
      !aligned(probs, 4) || !aligned(dev_error, 4))
    return DAS_ERR_ALIGN;
  // one workgroup of 1024 threads per row; at most 2^32 - 1 work-items
  if (static_cast<long long>(batch) * block_len * 1024 > 0xffffffffLL) return DAS_ERR_SHAPE;
  SampleParams p;
  p.logits = logits;
  p.temperature = temperature;
  p.top_k = top_k;
  p.top_p = top_p;
  p.min_p = min_p;
  p.uniform = uniform;
  p.tokens = tokens;
  p.probs = probs;
  p.dev_error = dev_error;
  p.row_stride = row_stride;
  p.batch = batch;
  p.w = block_len;
  p.vocab = vocab;
  return launch_sample(p, dtype, stream) == hipSuccess ? DAS_OK : DAS_ERR_HIP;
}

das_status das_pages_update(int32_t batch, int32_t max_pages_per_seq, int32_t num_pages,
                            const int32_t *lengths, int32_t *block_table, int32_t *pages_held,
                            int32_t *free_pages, int32_t *num_free, const int32_t *first,
                            int32_t block_len, int32_t *slots, uint32_t *dev_error,
                            hipStream_t stream) {
  if (!lengths || !block_table || !pages_held || !free_pages || !num_free) return DAS_ERR_NULL;
  if (!slots != !first) return DAS_ERR_NULL;
  const das_status st = check_table(batch, max_pages_per_seq);
  if (st != DAS_OK) return st;
  if (num_pages < 1 || num_pages >= (1 << 25)) return DAS_ERR_SHAPE;
  if (slots ? block_len < 1 || block_len > DAS_MAX_BLOCK : block_len != 0) return DAS_ERR_SHAPE;
  if (!aligned(lengths, 4) || !aligned(block_table, 4) || !aligned(pages_held, 4) ||
      !aligned(free_pages, 4) || !aligned(num_free, 4) || !aligned(first, 4) ||
      !aligned(slots, 4) || !aligned(dev_error, 4))
    return DAS_ERR_ALIGN;
  PagesParams p;
  p.lengths = lengths;
  p.first = first;
  p.block_table = block_table;
  p.pages_held = pages_held;
  p.free_pages = free_pages;
  p.num_free = num_free;
  p.slots = slots;
  p.dev_error = dev_error;
  p.batch = batch;
  p.max_pages = max_pages_per_seq;
  p.num_pages = num_pages;
  p.w = block_len;
  return launch_pages_update(p, stream) == hipSuccess ? DAS_OK : DAS_ERR_HIP;
}

}  // extern "C"
