// Internal declarations of the 8-bit cache's kernels, the sampler and the page
// tables, shared by their host side (das_serve_api.hip). Not part of the public C ABI.
#pragma once

#include "das_internal.h"

namespace das {

// Tokens that share one exponent: the value page's group.
constexpr int kQ8Group = 8;
constexpr int kQ8GroupsPerPage = kPage / kQ8Group;
// Exponents that the commit gives (the stored byte is 127 more). Below -64 the
// values are under 2^-55, above 119 a code would pass the largest fp32.
constexpr int kQ8MinExp = -64, kQ8MaxExp = 119;

// One attention call over the 8-bit cache. Pool pointers include the plane and
// core-layer offsets.
struct AttnQ8Params {
  const uint8_t *k_layer;  // [Hkv][P][8][8 * dh]
  const uint8_t *v_layer;  // [Hkv][P][8][dh][8]
  const uint8_t *k_exp;    // [P][Hkv][8]
  const uint8_t *v_exp;    // [P][Hkv][8]
  const void *q;           // [B][w][Hq][dh]
  const void *kb, *vb;     // [B][w][Hkv][dh]
  void *out;               // [B][w][Hq][dh]
  float *lse;              // [B][Hq][w] or nullptr
  const int32_t *prefix_len;
  const int32_t *block_table;
  uint32_t *dev_error;
  uint8_t *ws;             // piece records [unit][nsplit] of piece_stride bytes
  int32_t batch, hq, hkv, group, w, rows;  // rows = w * group
  int32_t num_pages, max_pages;
  int32_t chunk_tiles;     // 32-token tiles of one workgroup
  int32_t nsplit;          // chunks of the longest unit
  int32_t piece_stride;
  float scale_log2;        // log2(e) / sqrt(dh)
};
hipError_t launch_attn_q8(const AttnQ8Params &p, int dtype, int dh, hipStream_t s);

// Launch shape of the attention kernel: 16-row tiles of a wave (two fp32 ones do not
// fit its registers at head dim 128, nor at 96 where waves share tiles) and waves with
// different rows, and with them the rows of a workgroup.
__host__ __device__ constexpr int q8_row_tiles(int rows, int dh, int es) {
  return rows <= 16 || (es == 4 && (dh == 128 || (dh == 96 && rows > 32))) ? 1 : 2;
}
__host__ __device__ constexpr int q8_row_waves(int rows, int dh, int es) {
  return rows <= 16 * q8_row_tiles(rows, dh, es) ? 1 : rows <= 32 * q8_row_tiles(rows, dh, es) ? 2 : 4;
}
__host__ __device__ constexpr int q8_group_rows(int rows, int dh, int es) {
  return 16 * q8_row_tiles(rows, dh, es) * q8_row_waves(rows, dh, es);
}

struct AppendQ8Params {
  const void *k_new;       // [nK][L][B][w_max][Hkv][dh]
  const void *v_new;       // [nV][L][B][w_max][Hkv][dh]
  uint8_t *k_pool;         // [nK][L][Hkv][P][8][8 * dh]
  uint8_t *v_pool;         // [nV][L][Hkv][P][8][dh][8]
  uint8_t *k_exp, *v_exp;  // [planes][L][P][Hkv][8]
  const int32_t *prefix_len;
  const int32_t *block_table;
  const int32_t *num_new;
  int32_t *len_out;
  uint32_t *dev_error;
  int32_t batch, n_k_planes, n_v_planes, layers, hkv, num_pages, max_pages, w_max;
};
hipError_t launch_kv_append_q8(const AppendQ8Params &p, int dtype, int dh, hipStream_t s);

struct SampleParams {
  const void *logits;         // [rows] rows of `vocab`, row_stride elements apart
  const float *temperature;   // [B] or null (1)
  const int32_t *top_k;       // [B] or null (off)
  const float *top_p, *min_p; // [B] or null (off)
  const float *uniform;       // [B][w]
  int32_t *tokens;            // [B][w]
  float *probs;               // [B][w] or null
  uint32_t *dev_error;
  int64_t row_stride;
  int32_t batch, w, vocab;
};
hipError_t launch_sample(const SampleParams &p, int dtype, hipStream_t s);

struct PagesParams {
  const int32_t *lengths;     // [B]
  const int32_t *first;       // [B] or null
  int32_t *block_table;       // [B][max_pages]
  int32_t *pages_held;        // [B]
  int32_t *free_pages;        // [num_pages]
  int32_t *num_free;          // [1]
  int32_t *slots;             // [B][w] or null
  uint32_t *dev_error;
  int32_t batch, max_pages, num_pages, w;
};
hipError_t launch_pages_update(const PagesParams &p, hipStream_t s);

}  // namespace das
