// Internal declarations of the 4-bit cache's kernels, the queries' and keys' norm and
// rotation, and the sampled verification, shared by their host side (das_draft_api.hip).
// Not part of the public C ABI.
#pragma once

#include "q8_internal.h"

namespace das {

// Elements of a token that share one exponent, and the exponents that the commit gives (the
// stored byte is 127 more): the smallest code of the smallest is 2^-121, a normal bf16, and
// 6 * 2^125 is the largest multiple of 6 that fits one.
constexpr int kQ4Block = 32;
constexpr int kQ4MinExp = -120, kQ4MaxExp = 125;
constexpr int kQ4NanByte = 255;
// Bytes of a page of one head: two codes each, and the exponents.
__host__ __device__ constexpr int q4_page_bytes(int dh) { return kPage * dh / 2; }
__host__ __device__ constexpr int q4_page_exps(int dh) { return kPage * dh / kQ4Block; }

// One attention call over the 4-bit cache: AttnQ8Params with k_layer, v_layer
// [Hkv][P][dh / 32][64][16], k_exp, v_exp [Hkv][P][2 * dh], and chunk_tiles in tiles of 64
// tokens (the draft block's, then a page each).
hipError_t launch_attn_q4(const AttnQ8Params &p, int dtype, int dh, hipStream_t s);

// Launch shape of the attention kernel: 16-row tiles of a wave, and whether all waves have the
// same rows and pages of their own (1) or rows of their own and the same pages, whose conversion
// they share (4). An fp32 call's queries are three operands each: one row tile. us of (tiles,
// waves), bf16 calls, 32 sequences x 55 heads, dh 96, 4096-8192 tokens unless said:
//   16 rows (1, 1) 197, (2, 1) 227; 32 rows (2, 1) 232, (1, 1) twice 368, (1, 4) 428;
//   32 rows of 32 x 32 heads, dh 128: (2, 1) 190, (1, 1) twice 275, (1, 4) 330;
//   64 rows, 2048-4096 tokens: (1, 4) 239, (2, 1) twice 253, (2, 4) 357; 128 rows of 4 x 8 heads,
//   dh 128, 32768 tokens: (2, 4) 96, (1, 4) twice 122, (2, 1) four times 165;
//   fp32, 16 x 55 heads, dh 96, 32 rows: (1, 1) twice 144, (1, 4) 220; 64 rows, 8 x 55 heads:
//   (1, 4) 143, (1, 1) four times 154.
// Two waves with the same rows and two with others, in between, were no faster than the better
// of these anywhere (64 rows 267, fp32 32 rows 154).
__host__ __device__ constexpr int q4_row_tiles(int rows, int es) {
  return es == 2 && ((rows > 16 && rows <= 32) || rows > 64) ? 2 : 1;
}
__host__ __device__ constexpr int q4_row_waves(int rows) { return rows <= 32 ? 1 : 4; }
__host__ __device__ constexpr int q4_group_rows(int rows, int es) {
  return 16 * q4_row_tiles(rows, es) * q4_row_waves(rows);
}

// Workgroups of the commit and of the way back that share a (plane, layer)'s heads: a wave takes
// kQ4Steps times four neighbouring blocks of each of its tokens. Units (plane, layer) times
// shares are a grid's width.
constexpr int kQ4Steps = 3;
__host__ __device__ constexpr int q4_head_shares(int hkv, int dh) {
  return (hkv * (dh / kQ4Block) + 4 * kQ4Steps - 1) / (4 * kQ4Steps);
}
// The commit into the 4-bit cache, and the way back (k_new, v_new written).
struct TokensQ4Params {
  void *k_new;             // [nK][L][B][w_max][Hkv][dh]
  void *v_new;             // [nV][L][B][w_max][Hkv][dh]
  uint8_t *k_pool;         // [nK][L][Hkv][P][dh / 32][64][16]
  uint8_t *v_pool;         // [nV][L][Hkv][P][dh / 32][64][16]
  uint8_t *k_exp, *v_exp;  // [planes][L][Hkv][P][2 * dh]
  const int32_t *first;    // [B] first position: the prefix lengths of a commit
  const int32_t *limit;    // [B] or null: positions that there are (reading)
  const int32_t *block_table;
  const int32_t *num;      // [B]
  int32_t *len_out;        // [B] or null (commit)
  uint32_t *dev_error;
  int32_t batch, n_k_planes, n_v_planes, layers, hkv, num_pages, max_pages, w_max;
};
hipError_t launch_kv_append_q4(const TokensQ4Params &p, int dtype, int dh, hipStream_t s);
hipError_t launch_kv_read_q4(const TokensQ4Params &p, int dtype, int dh, hipStream_t s);

struct RopeParams {
  const void *q, *k, *v;             // rows of heads; v may be null
  void *q_out, *k_out, *v_out;
  const void *q_weight, *k_weight;   // [dh] or null: no norm
  const float *inv_freq;             // [rotary / 2]
  const int32_t *positions;          // [B] first positions, or [B][w] (each)
  int64_t q_batch, q_token, k_batch, k_token, v_batch, v_token;  // strides in elements
  float eps;
  int32_t batch, w, hq, hkv, dh, rotary, interleaved, each;
};
hipError_t launch_qk_rope(const RopeParams &p, int dtype, hipStream_t s);

// Tokens of a row that one workgroup of the verification takes, for the rows' sums and for the
// draw, and what it keeps of a part and of a sequence in the workspace.
constexpr int kAcceptPart = 8192, kAcceptDraw = 2048;
constexpr int kAcceptMostDraws = DAS_MAX_VOCAB / kAcceptDraw;
constexpr int kAcceptStatBytes = 16, kAcceptChainBytes = 48;
struct SampledAcceptParams {
  const int32_t *proposals;         // [B][w]
  const void *target, *draft;       // rows of `vocab` logits; draft may be null
  const float *temperature, *draft_temperature;  // [B] or null (1)
  const int32_t *tested;            // [B] or null (w)
  const float *uniform, *draw;      // [B][w], [B]
  int32_t *accepted, *num_keep, *emitted, *num_emitted;  // the last may be null
  float *probs;                     // [B][w] or null
  uint32_t *dev_error;
  uint8_t *ws;
  int64_t target_stride, draft_stride;
  int32_t batch, w, vocab, parts, draw_parts;
};
hipError_t launch_sampled_accept(const SampledAcceptParams &p, int dtype, hipStream_t s);

}  // namespace das
