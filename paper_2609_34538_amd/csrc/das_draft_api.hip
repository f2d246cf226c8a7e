// Host side of the 4-bit cache, the queries' and keys' norm and rotation and the sampled
// verification: argument validation, the attention's cut into chunks, and dispatch behind
// the C ABI of das.h. As in das_api.hip every check runs before the first HIP call.

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "q4_internal.h"

namespace das {
namespace {

bool aligned(const void *ptr, size_t a) { return reinterpret_cast<uintptr_t>(ptr) % a == 0; }

// Whether arrays of `na` and `nb` bytes share any.
bool overlap(const void *a, uint64_t na, const void *b, uint64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && (x < y ? y - x < na : x - y < nb);
}

das_status check_cache(const das_cache_q4 *cache) {
  if (!cache) return DAS_ERR_NULL;
  const das_cache *c = &cache->base;
  if (!c->k_pool || !c->v_pool || !cache->k_exp || !cache->v_exp) return DAS_ERR_NULL;
  if (!aligned(c->k_pool, 16) || !aligned(c->v_pool, 16) || !aligned(cache->k_exp, 16) ||
      !aligned(cache->v_exp, 16))
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

das_status check_batch(const das_batch *b) {
  if (!b) return DAS_ERR_NULL;
  if (!b->prefix_len || !b->block_table) return DAS_ERR_NULL;
  if (!aligned(b->prefix_len, 4) || !aligned(b->block_table, 4) || !aligned(b->dev_error, 4))
    return DAS_ERR_ALIGN;
  if (b->batch < 1 || b->batch > 65535 || b->max_pages_per_seq < 1) return DAS_ERR_SHAPE;
  if (b->max_pages_per_seq > (1 << 24) ||
      static_cast<long long>(b->batch) * b->max_pages_per_seq > 0x7fffffffLL)
    return DAS_ERR_SHAPE;
  return DAS_OK;
}

struct PlanQ4 {
  int rows, chunk_tiles, nsplit, piece_stride;
  size_t total;
};

// Cuts the units (sequence, KV head) of a call into chunks of equal length, one workgroup
// each, by the table's width, in tiles of 64 tokens. A chunk costs about 5 us beside its tiles
// (1 us for four of them), and more than one a unit a second launch; without enough of them the
// longest unit is what the call takes.
//
// RW == 1: three a compute unit of a batch, whose lengths differ, one a compute unit of a single
// sequence; in chunks of at least 32 tiles where that leaves 384 of them, 16 where 256, 8
// where 128 (us, 4 query heads a KV head, one token each, dh 128, up to 8191 tokens; in
// parentheses with chunks of 8, 16, 32 and all tiles):
//   32 units 11.1 (11.5 11.0 14.5 32), 64 units 15.0 (17 15.0 15.2 32), 128 units 22.3 (27 23 22
//   34), 192 units 27.2 (35 30 27 35), 384 units 51 (63 54 51 56), 512 units 65 (80 69 65 67);
//   55 units of one sequence, 8192 tokens, 32 rows, dh 96: 21.0-22.5 (27 22 21 43).
// A unit is not cut at all below 16 tiles, and up to 65 where there are 192 of them (192 units of
// 4096 tokens: 23.7; 26.2 with 16 tiles a chunk, 28.1 with 24, 25.7 with 32).
//
// RW == 4, where a page is a step for all waves: three a compute unit of a batch, two of a single
// sequence, from four tiles on, from 32 on beyond 4096 tokens where that leaves 384 of them (us;
// in parentheses with 4, 8, 16, 32 and 64 tiles a chunk): 32 heads of 128 rows, dh 128, 32768
// tokens 93 (156 116 103 93 114); 192 of 48 rows, up to 8191 tokens 68 (100 77 70 68 93); 55 of one
// sequence, 64 rows, dh 96, 2048 tokens 18.7 (18.7 20.9 28 44 40), 8192 tokens 34 (44 38 35 46 78).
das_status plan_attn(const das_cache_q4 *cache, const das_batch *b, int hq, int w, PlanQ4 *plan) {
  const das_cache *c = &cache->base;
  if (hq < 1 || hq % c->num_kv_heads != 0) return DAS_ERR_SHAPE;
  const int group = hq / c->num_kv_heads;
  if (group > 8) return DAS_ERR_UNSUPPORTED;
  if (w < 1 || w > DAS_MAX_BLOCK) return DAS_ERR_SHAPE;
  plan->rows = w * group;
  const int es = c->dtype == DAS_F32 ? 4 : 2;
  const int gr = q4_group_rows(plan->rows, es);
  const long long n_rg = (plan->rows + gr - 1) / gr;
  const long long units = static_cast<long long>(b->batch) * c->num_kv_heads;
  const long long tiles = 1LL + b->max_pages_per_seq;
  const int rw = q4_row_waves(plan->rows);
  const long long wgs = units * n_rg;  // of one chunk per unit
  const auto enough = [&](long long ct, long long n) { return wgs * ((tiles + ct - 1) / ct) >= n; };
  long long ns, least;
  if (rw == 1) {
    const bool one = tiles <= 16 || (tiles <= 65 && 4 * wgs >= 3 * kNumCUs);
    ns = one ? 1 : std::min<long long>((b->batch == 1 ? 1 : 3) * kNumCUs / wgs, 64);
    least = enough(32, 384) ? 32 : enough(16, 256) ? 16 : enough(8, 128) ? 8 : 4;
  } else {
    ns = (b->batch == 1 ? 2 : 3) * kNumCUs / wgs;
    least = tiles > 65 && enough(32, 384) ? 32 : 4;
  }
  ns = std::max<long long>(ns, 1);
  const long long ct = std::max((tiles + ns - 1) / ns, least);
  ns = (tiles + ct - 1) / ct;
  if (units * n_rg * ns * 256 > 0xffffffffLL) return DAS_ERR_SHAPE;
  plan->chunk_tiles = static_cast<int>(ct);
  plan->nsplit = static_cast<int>(ns);
  plan->piece_stride = static_cast<int>(piece_record_bytes(plan->rows, c->head_dim, es));
  plan->total = std::max<size_t>(256, ns > 1 ? static_cast<size_t>(units) * ns * plan->piece_stride : 0);
  return DAS_OK;
}

// What commit and read-back share; `rows` are their inputs or outputs.
das_status tokens_params(const das_cache_q4 *cache, const das_batch *batch, const void *k_rows,
                         const void *v_rows, int w_max, TokensQ4Params *p) {
  const das_cache *c = &cache->base;
  if (!k_rows || !v_rows) return DAS_ERR_NULL;
  if (!aligned(k_rows, 16) || !aligned(v_rows, 16)) return DAS_ERR_ALIGN;
  // the grid: workgroups of 256 per (plane, layer) and share of its heads, at most 2^32 - 1
  // work-items along x
  const int64_t units = (static_cast<int64_t>(c->num_k_planes) + c->num_v_planes) * c->num_layers;
  if (units > 0xffffffffLL / 256 / q4_head_shares(c->num_kv_heads, c->head_dim)) return DAS_ERR_SHAPE;
  p->k_new = const_cast<void *>(k_rows);
  p->v_new = const_cast<void *>(v_rows);
  p->k_pool = static_cast<uint8_t *>(c->k_pool);
  p->v_pool = static_cast<uint8_t *>(c->v_pool);
  p->k_exp = cache->k_exp;
  p->v_exp = cache->v_exp;
  p->block_table = batch->block_table;
  p->dev_error = batch->dev_error;
  p->batch = batch->batch;
  p->n_k_planes = c->num_k_planes;
  p->n_v_planes = c->num_v_planes;
  p->layers = c->num_layers;
  p->hkv = c->num_kv_heads;
  p->num_pages = c->num_pages;
  p->max_pages = batch->max_pages_per_seq;
  p->w_max = w_max;
  return DAS_OK;
}

// An array, its bytes from the first to the last element, and whether there are none between
// its rows.
struct Span {
  const void *at;
  uint64_t bytes;
  bool dense = true;
};
// That of [B][w][heads][dh] at these distances; false where they are none.
bool span_of(const void *at, int batch, int w, int heads, int dh, int64_t sb, int64_t st, int es, Span *out) {
  const int64_t row = static_cast<int64_t>(heads) * dh;
  constexpr int64_t kMost = INT64_MAX >> 4;
  if (w > 1 && (st < row || st > kMost / w)) return false;
  const int64_t seq = (w > 1 ? (w - 1) * st : 0) + row;
  if (batch > 1 && (sb < seq || sb > kMost / batch)) return false;
  const int64_t total = (batch > 1 ? (batch - 1) * sb : 0) + seq;
  if (total > kMost) return false;
  out->at = at;
  out->bytes = static_cast<uint64_t>(total) * es;
  out->dense = total == row * w * batch;
  return true;
}

// Parts of a row of the sampled verification, and the workspace: statistics of target's and
// draft's parts, the residual's sums, and what is known of a sequence.
size_t accept_workspace(int64_t batch, int64_t w, int64_t vocab) {
  const int64_t parts = (vocab + kAcceptPart - 1) / kAcceptPart, draws = (vocab + kAcceptDraw - 1) / kAcceptDraw;
  const int64_t bytes = 2 * batch * w * parts * kAcceptStatBytes + batch * draws * 8 + batch * kAcceptChainBytes;
  return static_cast<size_t>(bytes + 255) / 256 * 256;
}

}  // namespace
}  // namespace das

using namespace das;

extern "C" {

size_t das_attn_q4_workspace_bytes(const das_cache_q4 *cache, const das_batch *batch,
                                   int32_t num_q_heads, int32_t block_len) {
  if (check_cache(cache) != DAS_OK || check_batch(batch) != DAS_OK) return 0;
  PlanQ4 plan;
  if (plan_attn(cache, batch, num_q_heads, block_len, &plan) != DAS_OK) return 0;
  return plan.total;
}

das_status das_attn_q4(const das_cache_q4 *cache, const das_batch *batch, int32_t layer,
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
  PlanQ4 plan;
  st = plan_attn(cache, batch, num_q_heads, block_len, &plan);
  if (st != DAS_OK) return st;
  if (!workspace || workspace_bytes < plan.total || !aligned(workspace, 256)) return DAS_ERR_WORKSPACE;
  const int dh = c->head_dim;
  const size_t page_heads = static_cast<size_t>(c->num_kv_heads) * c->num_pages;
  const size_t k_at = (static_cast<size_t>(kplane) * c->num_layers + layer) * page_heads;
  const size_t v_at = (static_cast<size_t>(vplane) * c->num_layers + layer) * page_heads;
  AttnQ8Params p;
  p.k_layer = static_cast<const uint8_t *>(c->k_pool) + k_at * q4_page_bytes(dh);
  p.v_layer = static_cast<const uint8_t *>(c->v_pool) + v_at * q4_page_bytes(dh);
  p.k_exp = cache->k_exp + k_at * q4_page_exps(dh);
  p.v_exp = cache->v_exp + v_at * q4_page_exps(dh);
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
  return launch_attn_q4(p, c->dtype, dh, stream) == hipSuccess ? DAS_OK : DAS_ERR_HIP;
}

das_status das_kv_append_q4(const das_cache_q4 *cache, const das_batch *batch, const void *k_new,
                            const void *v_new, int32_t w_max, const int32_t *num_new,
                            int32_t *len_out, hipStream_t stream) {
  das_status st = check_cache(cache);
  if (st != DAS_OK) return st;
  st = check_batch(batch);
  if (st != DAS_OK) return st;
  if (!num_new) return DAS_ERR_NULL;
  if (!aligned(num_new, 4) || !aligned(len_out, 4)) return DAS_ERR_ALIGN;
  if (w_max < 1 || w_max > DAS_MAX_BLOCK) return DAS_ERR_SHAPE;
  TokensQ4Params p;
  st = tokens_params(cache, batch, k_new, v_new, w_max, &p);
  if (st != DAS_OK) return st;
  // every workgroup of a sequence reads its length and count, one of them writes len_out
  const uint64_t per_seq = sizeof(int32_t) * static_cast<uint64_t>(batch->batch);
  if (overlap(len_out, per_seq, batch->prefix_len, per_seq) || overlap(len_out, per_seq, num_new, per_seq))
    return DAS_ERR_SHAPE;
  p.first = batch->prefix_len;
  p.limit = nullptr;
  p.num = num_new;
  p.len_out = len_out;
  return launch_kv_append_q4(p, cache->base.dtype, cache->base.head_dim, stream) == hipSuccess ? DAS_OK
                                                                                              : DAS_ERR_HIP;
}

das_status das_kv_read_q4(const das_cache_q4 *cache, const das_batch *batch, const int32_t *first,
                          const int32_t *num, int32_t w_max, void *k_out, void *v_out,
                          hipStream_t stream) {
  das_status st = check_cache(cache);
  if (st != DAS_OK) return st;
  st = check_batch(batch);
  if (st != DAS_OK) return st;
  if (!first || !num) return DAS_ERR_NULL;
  if (!aligned(first, 4) || !aligned(num, 4)) return DAS_ERR_ALIGN;
  if (w_max < 1 || w_max > DAS_MAX_READ) return DAS_ERR_SHAPE;
  TokensQ4Params p;
  st = tokens_params(cache, batch, k_out, v_out, w_max, &p);
  if (st != DAS_OK) return st;
  // the arrays' sizes fit 64 bits: 2^46 elements a (plane, layer), at most 2^32 of these
  const das_cache *c = &cache->base;
  if (static_cast<int64_t>(batch->batch) * w_max > (1LL << 46) / (static_cast<int64_t>(c->num_kv_heads) * c->head_dim))
    return DAS_ERR_SHAPE;
  const double per = static_cast<double>(c->num_layers) * batch->batch * w_max * c->num_kv_heads * c->head_dim *
                     (c->dtype == DAS_F32 ? 4 : 2);
  if (per * std::max(c->num_k_planes, c->num_v_planes) >= 0x1p62) return DAS_ERR_SHAPE;
  const uint64_t k_bytes = static_cast<uint64_t>(per) * c->num_k_planes, v_bytes = static_cast<uint64_t>(per) * c->num_v_planes;
  if (overlap(k_out, k_bytes, v_out, v_bytes)) return DAS_ERR_SHAPE;
  const double heads = static_cast<double>(c->num_layers) * c->num_kv_heads * c->num_pages;
  const auto bytes_of = [&](int planes, int of_page) {
    return static_cast<uint64_t>(std::min(heads * planes * of_page, 0x1p62));
  };
  const Span held[] = {{c->k_pool, bytes_of(c->num_k_planes, q4_page_bytes(c->head_dim))},
                       {c->v_pool, bytes_of(c->num_v_planes, q4_page_bytes(c->head_dim))},
                       {cache->k_exp, bytes_of(c->num_k_planes, q4_page_exps(c->head_dim))},
                       {cache->v_exp, bytes_of(c->num_v_planes, q4_page_exps(c->head_dim))}};
  for (const Span &h : held)
    if (overlap(k_out, k_bytes, h.at, h.bytes) || overlap(v_out, v_bytes, h.at, h.bytes)) return DAS_ERR_SHAPE;
  p.first = first;
  p.limit = batch->prefix_len;
  p.num = num;
  p.len_out = nullptr;
  return launch_kv_read_q4(p, c->dtype, c->head_dim, stream) == hipSuccess ? DAS_OK : DAS_ERR_HIP;
}

das_status das_qk_rope(const das_rope *rope, int32_t batch, int32_t block_len, const void *q,
                       int64_t q_batch_stride, int64_t q_token_stride, const void *k,
                       int64_t k_batch_stride, int64_t k_token_stride, const void *v,
                       int64_t v_batch_stride, int64_t v_token_stride, const int32_t *positions,
                       void *q_out, void *k_out, void *v_out, hipStream_t stream) {
  if (!rope || !q || !k || !q_out || !k_out) return DAS_ERR_NULL;
  if (!v != !v_out) return DAS_ERR_NULL;
  if (rope->dtype != DAS_F32 && rope->dtype != DAS_BF16) return DAS_ERR_DTYPE;
  const int dh = rope->head_dim, hq = rope->num_q_heads, hkv = rope->num_kv_heads;
  if (dh != 64 && dh != 96 && dh != 128) return DAS_ERR_SHAPE;
  if (rope->rotary_dim < 0 || rope->rotary_dim > dh || rope->rotary_dim % 16 != 0) return DAS_ERR_SHAPE;
  if (rope->rotary_dim > 0 && (!rope->inv_freq || !positions)) return DAS_ERR_NULL;
  if (hq < 1 || hq > 65535 || hkv < 1 || hkv > 65535) return DAS_ERR_SHAPE;
  if (batch < 1 || batch > 65535 || block_len < 1 || block_len > DAS_MAX_READ ||
      static_cast<int64_t>(batch) * block_len >= 1 << 24)
    return DAS_ERR_SHAPE;
  if (!(rope->eps >= 0.f && rope->eps < __builtin_huge_valf())) return DAS_ERR_SHAPE;
  const int es = rope->dtype == DAS_F32 ? 4 : 2;
  const void *rows[] = {q, k, v, q_out, k_out, v_out, rope->q_weight, rope->k_weight};
  for (const void *r : rows)
    if (!aligned(r, 16)) return DAS_ERR_ALIGN;
  if (!aligned(rope->inv_freq, 4) || !aligned(positions, 4)) return DAS_ERR_ALIGN;
  const int64_t row_q = static_cast<int64_t>(hq) * dh, row_k = static_cast<int64_t>(hkv) * dh;
  Span in[3], out[3];
  const int n = v ? 3 : 2;
  if (!span_of(q, batch, block_len, hq, dh, q_batch_stride, q_token_stride, es, &in[0]) ||
      !span_of(k, batch, block_len, hkv, dh, k_batch_stride, k_token_stride, es, &in[1]) ||
      (v && !span_of(v, batch, block_len, hkv, dh, v_batch_stride, v_token_stride, es, &in[2])))
    return DAS_ERR_SHAPE;
  const int64_t strides[] = {q_batch_stride, k_batch_stride, v ? v_batch_stride : 0};
  const int64_t tokens[] = {q_token_stride, k_token_stride, v ? v_token_stride : 0};
  for (int i = 0; i < n; ++i)
    if ((batch > 1 && strides[i] * es % 16 != 0) || (block_len > 1 && tokens[i] * es % 16 != 0)) return DAS_ERR_ALIGN;
  void *outs[] = {q_out, k_out, v_out};
  for (int i = 0; i < n; ++i) {
    const int64_t row = i == 0 ? row_q : row_k;
    span_of(outs[i], batch, block_len, i == 0 ? hq : hkv, dh, row * block_len, row, es, &out[i]);
  }
  const uint64_t weight_bytes = static_cast<uint64_t>(dh) * es;
  for (int i = 0; i < n; ++i) {
    for (int j = 0; j < n; ++j) {
      const bool own = i == j && out[i].at == in[j].at && in[j].dense;
      if (!own && overlap(out[i].at, out[i].bytes, in[j].at, in[j].bytes)) return DAS_ERR_SHAPE;
      if (i < j && overlap(out[i].at, out[i].bytes, out[j].at, out[j].bytes)) return DAS_ERR_SHAPE;
    }
    if (overlap(out[i].at, out[i].bytes, rope->q_weight, weight_bytes) ||
        overlap(out[i].at, out[i].bytes, rope->k_weight, weight_bytes) ||
        overlap(out[i].at, out[i].bytes, rope->inv_freq, rope->rotary_dim * 2) ||
        overlap(out[i].at, out[i].bytes, positions, 4ull * batch * (rope->each_position ? block_len : 1)))
      return DAS_ERR_SHAPE;
  }
  RopeParams p;
  p.q = q;
  p.k = k;
  p.v = v;
  p.q_out = q_out;
  p.k_out = k_out;
  p.v_out = v_out;
  p.q_weight = rope->q_weight;
  p.k_weight = rope->k_weight;
  p.inv_freq = rope->inv_freq;
  p.positions = positions;
  p.q_batch = q_batch_stride;
  p.q_token = q_token_stride;
  p.k_batch = k_batch_stride;
  p.k_token = k_token_stride;
  p.v_batch = v_batch_stride;
  p.v_token = v_token_stride;
  p.eps = rope->eps;
  p.batch = batch;
  p.w = block_len;
  p.hq = hq;
  p.hkv = hkv;
  p.dh = dh;
  p.rotary = rope->rotary_dim;
  p.interleaved = rope->interleaved != 0;
  p.each = rope->each_position != 0;
  return launch_qk_rope(p, rope->dtype, stream) == hipSuccess ? DAS_OK : DAS_ERR_HIP;
}

size_t das_sampled_accept_workspace_bytes(int32_t batch, int32_t block_len, int32_t vocab) {
  if (batch < 1 || batch > 65535 || block_len < 1 || block_len > DAS_MAX_BLOCK || vocab < 1 ||
      vocab > DAS_MAX_VOCAB)
    return 0;
  return accept_workspace(batch, block_len, vocab);
}

das_status das_sampled_accept(int32_t batch, int32_t block_len, int32_t vocab, int32_t dtype,
                              const int32_t *proposals, const void *target_logits,
                              int64_t target_stride, const void *draft_logits,
                              int64_t draft_stride, const float *temperature,
                              const float *draft_temperature, const int32_t *tested,
                              const float *uniform, const float *draw, int32_t *accepted,
                              int32_t *num_keep, int32_t *emitted, int32_t *num_emitted,
                              float *probs, void *workspace, size_t workspace_bytes,
                              uint32_t *dev_error, hipStream_t stream) {
  if (!proposals || !target_logits || !uniform || !draw || !accepted || !num_keep) return DAS_ERR_NULL;
  if (dtype != DAS_F32 && dtype != DAS_BF16) return DAS_ERR_DTYPE;
  if (batch < 1 || batch > 65535 || block_len < 1 || block_len > DAS_MAX_BLOCK || vocab < 1 ||
      vocab > DAS_MAX_VOCAB || target_stride < vocab || (draft_logits && draft_stride < vocab))
    return DAS_ERR_SHAPE;
  // every byte offset fits 64 bits
  const int64_t most = (INT64_MAX >> 3) / (static_cast<int64_t>(batch) * block_len);
  if (target_stride > most || (draft_logits && draft_stride > most)) return DAS_ERR_SHAPE;
  const size_t es = dtype == DAS_F32 ? 4 : 2;
  if (!aligned(target_logits, es) || !aligned(draft_logits, es)) return DAS_ERR_ALIGN;
  const void *words[] = {proposals, temperature, draft_temperature, tested, uniform,   draw,
                         accepted,  num_keep,    emitted,           num_emitted, probs, dev_error};
  for (const void *w : words)
    if (!aligned(w, 4)) return DAS_ERR_ALIGN;
  const int parts = (vocab + kAcceptPart - 1) / kAcceptPart;
  const int64_t rows = static_cast<int64_t>(batch) * block_len;
  // one workgroup of 256 threads per part of a target's and a draft's row; at most 2^32 - 1 work-items
  // (and per part of a sequence's draw)
  const int draws = (vocab + kAcceptDraw - 1) / kAcceptDraw;
  if (rows * (draft_logits ? 2 : 1) * parts * 256 > 0xffffffffLL ||
      static_cast<int64_t>(batch) * draws * 256 > 0xffffffffLL)
    return DAS_ERR_SHAPE;
  if (!workspace || workspace_bytes < accept_workspace(batch, block_len, vocab) || !aligned(workspace, 256))
    return DAS_ERR_WORKSPACE;
  // every workgroup of a sequence reads its inputs, one of them writes its results
  const uint64_t seqs = 4ull * batch, all = 4ull * rows;
  const Span in[] = {{proposals, all},         {uniform, all}, {draw, seqs}, {temperature, seqs},
                     {draft_temperature, seqs}, {tested, seqs},
                     {target_logits, ((rows - 1) * target_stride + vocab) * es},
                     {draft_logits, ((rows - 1) * draft_stride + vocab) * es}};
  const Span out[] = {{accepted, seqs}, {num_keep, seqs}, {num_emitted, seqs}, {emitted, all}, {probs, all}};
  for (const Span &o : out) {
    for (const Span &i : in)
      if (overlap(o.at, o.bytes, i.at, i.bytes)) return DAS_ERR_SHAPE;
    for (const Span *other = out; other != &o; ++other)
      if (overlap(o.at, o.bytes, other->at, other->bytes)) return DAS_ERR_SHAPE;
  }
  SampledAcceptParams p;
  p.proposals = proposals;
  p.target = target_logits;
  p.draft = draft_logits;
  p.temperature = temperature;
  p.draft_temperature = draft_temperature;
  p.tested = tested;
  p.uniform = uniform;
  p.draw = draw;
  p.accepted = accepted;
  p.num_keep = num_keep;
  p.emitted = emitted;
  p.num_emitted = num_emitted;
  p.probs = probs;
  p.dev_error = dev_error;
  p.ws = static_cast<uint8_t *>(workspace);
  p.target_stride = target_stride;
  p.draft_stride = draft_stride;
  p.batch = batch;
  p.w = block_len;
  p.vocab = vocab;
  p.parts = parts;
  p.draw_parts = draws;
  return launch_sampled_accept(p, dtype, stream) == hipSuccess ? DAS_OK : DAS_ERR_HIP;
}

}  // extern "C"
