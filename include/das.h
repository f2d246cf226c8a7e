/*
 * das.h -- C ABI of the depth-asynchronous self-speculation (DAS) attention
 * library for AMD Instinct MI355X (gfx950).
 *
 * The library computes the policy attention of Eq. (2)-(3) of
 * "Shallow Queries, Mature Values: Depth-Asynchronous Self-Speculation for
 * Looped Transformers" over a depth-indexed, paged key/value cache, and the
 * commit of verified tokens into that cache (Sec. 3.4 and App. B.1).
 *
 *   [Pi_C, Pi_U] = softmax( Q [K_C^kappa ; K_U]^T / sqrt(d_h) + M )     Eq. (2)
 *   O            = Pi_C V_C^nu + Pi_U V_U                               Eq. (3)
 *
 * C is the verified, materialised prefix of a sequence, U the active block
 * (draft-side positions). kappa and nu are the recurrence depths at which the
 * prefix keys and values are read (Eq. (4)); block K/V always come from the
 * caller's current computation and are never read from the cache. M is the
 * causal mask: every prefix position is visible, block query i sees block
 * keys j <= i. Prefix and block positions share one softmax normaliser.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Ownership: every pointer is owned by the caller. The library allocates
 *   no device or host memory and frees nothing; its only device memory is
 *   the fixed scratch array of das_attn_policy_noalloc (one per GPU, part of
 *   the loaded code). Device pointers must stay valid until the enqueued
 *   work has completed on `stream`.
 * - Asynchrony: calls only validate arguments and enqueue kernels on
 *   `stream`; they return before the GPU work runs. Device faults surface at
 *   the caller's next synchronisation of that stream.
 * - Errors: every argument check runs on the host before any HIP call. A
 *   failed check returns a negative das_status and enqueues nothing. A
 *   failed kernel launch returns DAS_ERR_HIP; the status is that of the
 *   library's own launches, so an error left pending by the caller's earlier
 *   HIP work is neither reported as the library's nor cleared. Requests whose
 *   launch grid would exceed what HIP accepts (2^32 - 1 work-items along a
 *   grid dimension) are rejected with DAS_ERR_SHAPE. No exception and no
 *   exit() crosses this boundary.
 * - Device-side range checks: when `dev_error` in das_batch is non-NULL the
 *   kernels OR bits into it (DAS_DEVERR_*) for out-of-range page ids,
 *   prefix lengths or commit counts, and skip the offending data instead of
 *   reading or writing out of bounds.
 * - Reentrancy: apart from the per-device scratch address of
 *   das_attn_policy_noalloc (set once, under a lock) the library keeps no
 *   global state; calls from several host threads are safe. Concurrent calls that share a workspace or write the
 *   same cache rows race on the device, as any two kernels writing the same
 *   memory would.
 * - Alignment: the kernels move K/V/Q/O rows with 16-byte accesses, so
 *   k_pool, v_pool, q, k_blk, v_blk, out, k_new and v_new must be 16-byte
 *   aligned (any allocation, or a view starting on a row, is); int32 and
 *   fp32 arrays must be 4-byte aligned. Otherwise DAS_ERR_ALIGN.
 * - Numerics: scale is 1/sqrt(head_dim). Query head h reads KV head
 *   h / (Hq / Hkv). Accumulation is fp32; outputs are rounded to the input
 *   dtype (round to nearest even).
 */
#ifndef DAS_H
#define DAS_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Largest supported recurrence depth R; depths are 1-based (1..R). */
#define DAS_MAX_DEPTH 64
/* Tokens per cache page. */
#define DAS_PAGE_TOKENS 64
/* Largest block (draft or verifier input) width w. */
#define DAS_MAX_BLOCK 64

typedef enum das_status {
  DAS_OK = 0,
  DAS_ERR_NULL = -1,        /* a required pointer is NULL                     */
  DAS_ERR_SHAPE = -2,       /* a size is out of range or inconsistent         */
  DAS_ERR_DEPTH = -3,       /* depth outside 1..R or not stored in the cache  */
  DAS_ERR_DTYPE = -4,       /* unknown element type                           */
  DAS_ERR_WORKSPACE = -5,   /* workspace missing or smaller than required     */
  DAS_ERR_HIP = -6,         /* a HIP launch failed                            */
  DAS_ERR_UNSUPPORTED = -7, /* valid request that this build does not handle  */
  DAS_ERR_ALIGN = -8        /* a device array is not aligned as required      */
} das_status;

typedef enum das_dtype { DAS_F32 = 0, DAS_BF16 = 1 } das_dtype;

/* Bits OR-ed into das_batch.dev_error by the kernels. */
#define DAS_DEVERR_PAGE 1u       /* block_table entry outside [0, num_pages)      */
#define DAS_DEVERR_PREFIX 2u     /* prefix_len[b] < 0 or beyond the table's pages */
#define DAS_DEVERR_COMMIT 4u     /* num_new[b] outside [0, w_max], or the commit
                                    would run past the sequence's table pages     */
#define DAS_DEVERR_TESTED 8u     /* tested[b] outside [0, block_len]; clamped      */
#define DAS_DEVERR_SAMPLE 16u    /* a sampling parameter or random number out of
                                    range; the row was taken greedily               */
#define DAS_DEVERR_POOL 32u      /* too few free pages for a sequence, or a free
                                    list that cannot be right                       */
#define DAS_DEVERR_PROPOSAL 64u  /* a drafted token outside the vocabulary; rejected */

/*
 * Depth-indexed, paged KV cache (caller-owned device memory).
 *
 * The cache stores, for each stored recurrence depth r ("plane"), each core
 * layer l and each KV head h, the verified prefix's K^{r,l} and V^{r,l}
 * (Sec. 2: depth-indexed cached representations; the core-layer index is
 * never remapped). Tokens live in pages of DAS_PAGE_TOKENS positions; a
 * sequence's logical page p is the physical page block_table[b][p], the same
 * physical page in every plane, layer and head.
 *
 *   k_pool: [num_k_planes][L][Hkv][num_pages][64][head_dim]     token-major
 *   v_pool: [num_v_planes][L][Hkv][num_pages][8][head_dim][8]   token-grouped
 *
 * Keys are stored token-major: position t of a page is row t. Values are
 * stored in groups of 8 positions: position t of a page is element
 * [t / 8][d][t % 8], so for every head dimension d the 8 positions of a
 * group are 16 contiguous bytes (bf16). Both products then read their
 * reduction dimension contiguously (Q K^T reduces over head_dim, P V over
 * positions), any 8-aligned run of positions of the value page is one
 * contiguous block, and a commit of 8 aligned positions writes one
 * contiguous head_dim x 16-byte block per (plane, layer, head).
 *
 * k_plane[r] / v_plane[r] (r = 1..R) give the plane holding depth r, or -1
 * when that depth is not stored; entry 0 is unused. Only the depths that a
 * workload reads need be stored.
 */
typedef struct das_cache {
  int32_t dtype;         /* das_dtype of every K/V/Q/O element               */
  int32_t num_depths;    /* R, 1..DAS_MAX_DEPTH                              */
  int32_t num_layers;    /* L core layers, >= 1                              */
  int32_t num_kv_heads;  /* Hkv, 1..65535                                    */
  int32_t head_dim;      /* 64, 96 or 128                                    */
  int32_t num_pages;     /* physical pages per (plane, layer, head), >= 1    */
  int32_t num_k_planes;  /* >= 1                                             */
  int32_t num_v_planes;  /* >= 1                                             */
  int32_t k_plane[DAS_MAX_DEPTH + 1];
  int32_t v_plane[DAS_MAX_DEPTH + 1];
  void *k_pool;
  void *v_pool;
} das_cache;

/*
 * A batch of sequences reading (or committing to) the cache.
 * prefix_len[b] is S_b, the number of verified, materialised positions of
 * sequence b (0 is legal). The anchor and the draft block are never prefix
 * positions. block_table has max_pages_per_seq columns; prefix_len[b] may
 * not exceed 64 * max_pages_per_seq. All three arrays are device memory.
 */
typedef struct das_batch {
  int32_t batch;               /* B, 1..65535                                 */
  int32_t max_pages_per_seq;   /* columns of block_table, 1..2^24, and
                                  batch * max_pages_per_seq < 2^31             */
  const int32_t *prefix_len;   /* device [B]                                  */
  const int32_t *block_table;  /* device [B][max_pages_per_seq], int32 pages  */
  uint32_t *dev_error;         /* optional device word (see DAS_DEVERR_*)     */
} das_batch;

/* Kernel family and schedule selection (measurement and tests). */
typedef enum das_attn_path {
  DAS_PATH_AUTO = 0,     /* library choice                                   */
  DAS_PATH_VALU = 1,     /* vector-ALU kernel (on fp32 caches the only path that
                            can be asked for; DAS_PATH_AUTO runs most fp32
                            requests on the matrix cores, in full fp32)      */
  DAS_PATH_MFMA = 2,     /* matrix-core kernel over prefix splits (bf16)     */
  DAS_PATH_BALANCED = 3  /* matrix-core kernel, persistent balanced schedule:
                            every resident wave streams an equal share of
                            all sequences' tiles (bf16, 1..64 sequences,
                            blocks of at most 32 query rows, i.e.
                            w * Hq / Hkv <= 32, or 16 at head_dim 128;
                            DAS_ERR_UNSUPPORTED otherwise). DAS_PATH_AUTO takes it for batches
                            of 2..64 sequences when pages_per_split is 0
                            and the batch has more than W / 8 (sequence,
                            KV head) units, W = 256 x (7, 5, 4) workers
                            at head_dim (64, 96, 128), unless the units are
                            short enough for one workgroup each.  */
} das_attn_path;

typedef struct das_attn_options {
  int32_t path;             /* das_attn_path                                 */
  int32_t pages_per_split;  /* prefix pages per split (the first split of a
                               sequence, which also takes the draft block,
                               holds one page less); 0 = library choice;
                               clamped to the block table width + 1 (one
                               split then holds any sequence, and no merge
                               kernel runs), and to 64 on the matrix-core
                               path; not used by the balanced schedule      */
} das_attn_options;

/*
 * Bytes of device workspace an attention call with these shapes needs (the
 * partial results of the prefix splits or pieces: records of fp16 (bf16
 * caches) or fp32 outputs with fp32 maxima and sums on the matrix-core paths,
 * fp32 arrays on the vector-ALU path).
 * Returns 0 for arguments that the attention entry points would reject.
 * `opts` may be NULL.
 */
size_t das_attn_workspace_bytes(const das_cache *cache, const das_batch *batch,
                                int32_t num_q_heads, int32_t block_len);
size_t das_attn_workspace_bytes_ex(const das_cache *cache, const das_batch *batch,
                                   int32_t num_q_heads, int32_t block_len,
                                   const das_attn_options *opts);

/*
 * Mature-V draft attention (Eq. (2)-(3) with the Mature-V / Deep V policy of
 * Eq. (4): kappa = draft_depth, nu = R). Prefix keys are read at the draft
 * depth d, prefix values at the full depth R, at core layer `layer`.
 *
 *   q      [B][w][Hq][head_dim]   queries of the current draft computation
 *   k_blk  [B][w][Hkv][head_dim]  draft-side keys at the current depth
 *   v_blk  [B][w][Hkv][head_dim]  draft-side values at the current depth
 *                                 (Mature-V changes prefix V only)
 *   out    [B][w][Hq][head_dim]   written, same dtype as the inputs
 *   lse    [B][Hq][w] fp32        optional natural-log softmax normaliser
 *   workspace                     >= das_attn_workspace_bytes(...) bytes,
 *                                 256-byte aligned, contents need no init;
 *                                 calls that run concurrently need separate
 *                                 workspaces
 *
 * w = block_len in 1..DAS_MAX_BLOCK; Hq a multiple of Hkv with Hq/Hkv <= 8;
 * layer in 0..L-1; draft_depth in 1..R; K at draft_depth and V at R stored.
 */
das_status das_attn_draft_maturev(const das_cache *cache, const das_batch *batch,
                                  int32_t layer, int32_t draft_depth,
                                  int32_t num_q_heads, int32_t block_len,
                                  const void *q, const void *k_blk, const void *v_blk,
                                  void *out, float *lse,
                                  void *workspace, size_t workspace_bytes,
                                  hipStream_t stream);

/*
 * The target's ordinary attention at depth r (Aligned policy of Eq. (4),
 * kappa = nu = depth). With depth = R this is one core-layer attention of the
 * full-depth verifier of Sec. 3.4, over the verifier input block
 * [x_t, y_1 .. y_{w-1}]. Arguments as for das_attn_draft_maturev, with the
 * block tensors at depth `depth`.
 */
das_status das_attn_verify(const das_cache *cache, const das_batch *batch,
                           int32_t layer, int32_t depth,
                           int32_t num_q_heads, int32_t block_len,
                           const void *q, const void *k_blk, const void *v_blk,
                           void *out, float *lse,
                           void *workspace, size_t workspace_bytes,
                           hipStream_t stream);

/*
 * Any read policy of Eq. (4): prefix keys at depth kappa, prefix values at
 * depth nu (Aligned (r,r), Mature-V (r,R), Deep K (R,r), Deep K/V (R,R)).
 * The two entry points above are this call with fixed (kappa, nu).
 * `opts` may be NULL (library choices); a workspace sized with the same
 * `opts` must be passed.
 */
das_status das_attn_policy(const das_cache *cache, const das_batch *batch,
                           int32_t layer, int32_t kappa, int32_t nu,
                           int32_t num_q_heads, int32_t block_len,
                           const void *q, const void *k_blk, const void *v_blk,
                           void *out, float *lse,
                           void *workspace, size_t workspace_bytes,
                           const das_attn_options *opts, hipStream_t stream);

/* Bytes of the library-owned scratch of das_attn_policy_noalloc (per GPU). */
#define DAS_NOALLOC_SCRATCH_BYTES (64u << 20)

/*
 * das_attn_policy without a caller workspace, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid allocation). The split partials go to a
 * library-owned scratch array of DAS_NOALLOC_SCRATCH_BYTES bytes per GPU,
 * placed when the library's code is loaded on that GPU and held until the
 * process ends; this call allocates nothing. Results are those of
 * das_attn_policy with the same arguments and `opts`, bit for bit.
 *
 * - The first call on a device (with that device current) looks up the
 *   device address of that device's scratch copy; `stream` must belong to
 *   the current device (DAS_ERR_UNSUPPORTED otherwise; NULL = the current
 *   device's null stream).
 * - DAS_ERR_WORKSPACE when the request's workspace
 *   (das_attn_workspace_bytes_ex with the same arguments) exceeds
 *   DAS_NOALLOC_SCRATCH_BYTES.
 * - Every call on a GPU shares that GPU's scratch, and the scratch keeps
 *   whatever the last call left there (nothing in it needs clearing: each
 *   call writes every partial it reads). Calls that can overlap on one GPU
 *   (on different streams, or from different threads without ordering)
 *   race on it: serialise them on one stream, or use das_attn_policy with
 *   separate workspaces.
 */
das_status das_attn_policy_noalloc(const das_cache *cache, const das_batch *batch,
                                   int32_t layer, int32_t kappa, int32_t nu,
                                   int32_t num_q_heads, int32_t block_len,
                                   const void *q, const void *k_blk, const void *v_blk,
                                   void *out, float *lse, const das_attn_options *opts,
                                   hipStream_t stream);

/*
 * Commit (Sec. 3.4; App. B.1): for each sequence b, write the full-depth K/V
 * of the first num_new[b] block inputs to prefix positions
 * prefix_len[b] .. prefix_len[b] + num_new[b] - 1, in every stored plane and
 * every core layer. Entries past num_new[b] (rejected candidates) are not
 * written. Draft-side K/V are never committed.
 *
 *   k_new   [num_k_planes][L][B][w_max][Hkv][head_dim]  plane order = k_pool
 *   v_new   [num_v_planes][L][B][w_max][Hkv][head_dim]  plane order = v_pool
 *   num_new device [B] int32, each in 0..w_max
 *   len_out device [B] int32 or NULL: receives prefix_len[b] + num_new[b];
 *           must not alias batch->prefix_len
 *
 * The target pages must already be present in block_table. The verifier's
 * block K/V at plane p and layer l, k_new[p][l], is the same buffer the
 * attention calls take as k_blk. DAS_ERR_SHAPE when w_max is outside
 * 1..DAS_MAX_BLOCK or the commit's grid (one 64-lane wave per (plane, layer,
 * KV head), four per workgroup) exceeds 2^32 - 1 work-items.
 */
das_status das_kv_append(const das_cache *cache, const das_batch *batch,
                         const void *k_new, const void *v_new, int32_t w_max,
                         const int32_t *num_new, int32_t *len_out,
                         hipStream_t stream);

/*
 * Greedy verification of a block on the device (Sec. 3.4), so that the
 * commit count reaches das_kv_append without a host round trip.
 *
 * For each sequence b, the first m_b = tested[b] proposals are checked in
 * order against the verifier's predictions; proposals are accepted while
 * y_i equals yhat_i (i = 1..m_b). With a_b accepted:
 *   - emitted tokens: y_1..y_{a_b}, then yhat_{a_b+1} when a_b < w (the
 *     target prediction at the first mismatch, or the bonus token from an
 *     unused conditional when all m_b < w tested proposals agree); w tokens
 *     when every proposal of a full block is accepted;
 *   - retained verifier inputs: num_keep[b] = min(a_b + 1, w) (the anchor and
 *     the accepted inputs among [x_t, y_1 .. y_{w-1}]).
 *
 *   proposals   device [B][w] int32: y_1..y_w (index i-1 holds y_i)
 *   target_pred device [B][w] int32: yhat_i = argmax of the verifier's
 *               conditional p_i (computed by the model's readout)
 *   tested      device [B] int32 m_b in 0..w, or NULL for m_b = w; values
 *               outside 0..w are clamped and reported with DAS_DEVERR_TESTED
 *   accepted    device [B] int32, written: a_b
 *   num_keep    device [B] int32, written: min(a_b + 1, w); pass it as the
 *               num_new argument of das_kv_append (w_max = w)
 *   emitted     device [B][w] int32 or NULL, written: the emitted tokens;
 *               entries past num_emitted[b] are left untouched
 *   num_emitted device [B] int32 or NULL, written: min(a_b + 1, w)
 *   dev_error   optional device word (DAS_DEVERR_TESTED)
 *
 * batch >= 1; block_len w in 1..DAS_MAX_BLOCK. Integer work only: results
 * are exact. The output arrays must not overlap the inputs.
 */
das_status das_greedy_accept(int32_t batch, int32_t block_len, const int32_t *proposals,
                             const int32_t *target_pred, const int32_t *tested,
                             int32_t *accepted, int32_t *num_keep, int32_t *emitted,
                             int32_t *num_emitted, uint32_t *dev_error, hipStream_t stream);

/* -------------------------------------------------------------------------
 * A cache held in 8 bits
 * -------------------------------------------------------------------------
 * The same planes, layers, heads, pages and block tables with every element one
 * e4m3 code (OCP 8-bit float: 4 exponent bits, 3 mantissa bits, largest 448) and
 * one power-of-two scale per 8 tokens and KV head ("group": positions 8 G .. 8 G + 7
 * of a page). Element = code * 2^(byte - 127), byte in 1..254.
 *
 *   base.k_pool  [num_k_planes][L][Hkv][num_pages][8][8 * head_dim] codes: in a
 *                group, token 4 e + n (e < 2, n < 4), dim 32 s + 8 g + i (g < 4,
 *                i < 8) is byte 256 s + 64 g + 16 n + 8 e + i
 *   base.v_pool  [num_v_planes][L][Hkv][num_pages][8][head_dim][8] codes
 *   k_exp        [num_k_planes][L][num_pages][Hkv][8] bytes, one per group
 *   v_exp        [num_v_planes][L][num_pages][Hkv][8] bytes
 *
 * base.dtype is the type of queries, block K/V, outputs and committed K/V; the
 * other fields of `base` are as in das_cache. Pools are 16-byte aligned, exponent
 * arrays 4-byte aligned. Half the bytes of a bf16 cache, and one exponent to 8 *
 * head_dim codes, so half the time of a call that is bound by them. Places that hold no
 * token of a sequence (behind its length) may hold anything.
 */
typedef struct das_cache_q8 {
  das_cache base;
  uint8_t *k_exp;
  uint8_t *v_exp;
} das_cache_q8;

/*
 * das_attn_policy over an 8-bit cache: prefix keys at depth kappa and values at
 * depth nu are the elements above, block keys and values are the caller's in
 * base.dtype. Arguments, masks, bounds and error words as for das_attn_policy, and
 * the same limits (w in 1..DAS_MAX_BLOCK, Hq / Hkv <= 8), for any batch size.
 *
 * Numerics: elements are exact in the products' types. bf16 calls multiply values
 * in fp16 with probabilities of 11 bits; a group's values below 2^-24 of the largest
 * scale's unit met so far round there (beside a block with values of 2^-40 and more,
 * below 2^-88 at least). Block values keep bf16's range. fp32 calls multiply in fp32.
 * Accumulation and softmax statistics are fp32, for logits of any finite size; sums are
 * divided last, so that values whose sum over the positions passes the largest fp32
 * give infinities. Sequences that are cut into parts are joined from the parts' results,
 * in bf16 calls from fp16 relative to each row's largest: what is under 2^-39 of it in
 * its part is lost. lse as for das_attn_policy.
 *
 * das_attn_q8_workspace_bytes returns 0 for arguments that das_attn_q8 rejects; the
 * workspace is 256-byte aligned, needs no init, and calls that run concurrently need
 * separate ones.
 */
size_t das_attn_q8_workspace_bytes(const das_cache_q8 *cache, const das_batch *batch,
                                   int32_t num_q_heads, int32_t block_len);
das_status das_attn_q8(const das_cache_q8 *cache, const das_batch *batch, int32_t layer,
                       int32_t kappa, int32_t nu, int32_t num_q_heads, int32_t block_len,
                       const void *q, const void *k_blk, const void *v_blk, void *out, float *lse,
                       void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * das_kv_append into an 8-bit cache. Arguments as for das_kv_append, with k_new and
 * v_new in base.dtype; len_out must share no element with batch->prefix_len or num_new
 * (DAS_ERR_SHAPE).
 *
 * A group without earlier tokens of the sequence gets the smallest exponent e in
 * -64..119 with |x| <= 448 * 2^e for its new finite elements. A group with earlier
 * tokens gets the larger of that and its own; when its own grows, the earlier codes
 * are rounded again (which changes only those that become subnormal). Codes are
 * x * 2^-e rounded to nearest even; NaN and infinities become the code NaN, finite
 * values past 448 * 2^119 become that. Places of the group from the sequence's new
 * length on are left as they were.
 */
das_status das_kv_append_q8(const das_cache_q8 *cache, const das_batch *batch, const void *k_new,
                            const void *v_new, int32_t w_max, const int32_t *num_new,
                            int32_t *len_out, hipStream_t stream);

/* Largest vocabulary that das_sample takes. */
#define DAS_MAX_VOCAB (1 << 20)

/*
 * A token for every position of a batch of blocks, from its logits and a given random
 * number: the target's predictions for das_greedy_accept. A proposal that equals the
 * token drawn from the verifier's conditional is accepted, so the emitted tokens are
 * draws from the verifier's (filtered) distribution whatever the draft proposes, and
 * with temperature 0 they are its greedy continuation.
 *
 * Row (b, i) uses the parameters of sequence b. With z its logits (NaN counts as
 * -inf), m = max z and weights w_j = exp((z_j - m) / temperature[b]), tokens in the
 * order (z descending, index ascending):
 *   top-k  keeps the first top_k[b] tokens (0 or less, or vocab or more: all);
 *   top-p  keeps, of those, the shortest run from the first whose weights sum to
 *          top_p[b] of their total or more (1 or more: all; the first is always kept);
 *   min-p  keeps, of those, the tokens with w_j >= min_p[b] (0 or less: all; over 1
 *          counts as 1).
 * The token is the first in index order at which the running sum of kept weights
 * passes uniform[b][i] times their sum. Weights are rounded to 2^-40, for every filter
 * and the draw, and their sums are exact; a token below 2^-41 of the largest is never
 * drawn. A temperature of 0 takes
 * the largest logit, lowest index first; so do rows with a NaN, negative or infinite
 * temperature, a NaN filter or a random number outside [0, 1), which set
 * DAS_DEVERR_SAMPLE, and a row without any logit above -inf gives token 0.
 *
 *   logits       device rows of `vocab` elements of `dtype`, row_stride elements from
 *                one to the next (>= vocab), in the order [B][w]
 *   temperature  device [B] fp32, or NULL: 1
 *   top_k        device [B] int32, or NULL: all
 *   top_p, min_p device [B] fp32, or NULL: all
 *   uniform      device [B][w] fp32 in [0, 1)
 *   tokens       device [B][w] int32, written
 *   probs        device [B][w] fp32 or NULL, written: the token's share of the kept
 *                weights (1 where it was taken greedily)
 *   dev_error    optional device word
 *
 * batch in 1..65535, block_len in 1..DAS_MAX_BLOCK, vocab in 1..DAS_MAX_VOCAB. Logits
 * are aligned to their type, the other arrays to 4 bytes; tokens and probs must not
 * overlap the inputs or each other. Results do not depend on the order of the work:
 * equal calls give equal bits.
 */
das_status das_sample(int32_t batch, int32_t block_len, int32_t vocab, int32_t dtype,
                      const void *logits, int64_t row_stride, const float *temperature,
                      const int32_t *top_k, const float *top_p, const float *min_p,
                      const float *uniform, int32_t *tokens, float *probs, uint32_t *dev_error,
                      hipStream_t stream);

/*
 * Block tables from the lengths that sequences shall have, on the device: pages for a
 * step before its commit, their release after a rollback, and a finished sequence's
 * (length 0).
 *
 * Sequence b shall hold ceil(lengths[b] / 64) pages, the first pages_held[b] entries of
 * its table row. Sequences that hold more give the rest back, their entries become -1;
 * then sequences that hold less get what they lack, in sequence order: each all of it,
 * or nothing once the running sum of what was asked for passes the free pages
 * (DAS_DEVERR_POOL; its row and count stay as they were). Free pages are a stack: a
 * release undoes the grant before it exactly, so tables do not depend on timing.
 *
 *   lengths      device [B], each in 0 .. 64 * max_pages_per_seq; a sequence with
 *                another length, or a held count out of range, is left alone
 *                (DAS_DEVERR_PREFIX)
 *   block_table  device [B][max_pages_per_seq], updated
 *   pages_held   device [B], updated
 *   free_pages   device [num_pages], updated: the free page ids are its first *num_free
 *   num_free     device [1], updated. Where it is out of range or the list could not
 *                hold what comes back, nothing is moved (DAS_DEVERR_POOL)
 *   first, slots, block_len
 *                device [B], device [B][block_len] and the width, or NULL, NULL, 0:
 *                slots[b][i] receives the slot page * 64 + position % 64 of position
 *                first[b] + i in the updated table, or -1 where it is not below
 *                lengths[b] or has no page
 *   dev_error    optional device word
 *
 * batch in 1..65535, max_pages_per_seq in 1..2^24, batch * max_pages_per_seq < 2^31,
 * num_pages in 1..2^25 - 1, block_len in 1..DAS_MAX_BLOCK where slots are asked for.
 * The arrays must not overlap. One sequence's entry may be any page id: ids are moved,
 * not read through.
 */
das_status das_pages_update(int32_t batch, int32_t max_pages_per_seq, int32_t num_pages,
                            const int32_t *lengths, int32_t *block_table, int32_t *pages_held,
                            int32_t *free_pages, int32_t *num_free, const int32_t *first,
                            int32_t block_len, int32_t *slots, uint32_t *dev_error,
                            hipStream_t stream);

/* -------------------------------------------------------------------------
 * A cache held in 4 bits
 * -------------------------------------------------------------------------
 * The same planes, layers, heads, pages and block tables with every element one e2m1 code
 * (a sign bit and 0, 0.5, 1, 1.5, 2, 3, 4 or 6) and one power-of-two scale per token, KV head
 * and 32 neighbouring dims ("block"), as OCP's MX formats have them. Element = code *
 * 2^(byte - 127); byte 255 makes the block's 32 elements NaN. 4.25 bits an element: a cache
 * holds 3.8 times the tokens of a bf16 one, and its attention reads a quarter of the bytes.
 *
 * A page of one head is 32 * head_dim bytes of two codes each, the even dim in the low four
 * bits, and 2 * head_dim exponent bytes. With S = head_dim / 32, 64 "lanes" 16 g + n (g < 4,
 * n < 16) and 16 bytes of each in every piece:
 *
 *   base.k_pool  [num_k_planes][L][Hkv][num_pages][S][64][16]: token 32 T + 8 (n / 4) + 4 e +
 *                n % 4 (T, e < 2), dims 32 s + 8 g + 2 j and + 1 (j < 4): byte
 *                4 ((2 T + e) S + s) + j of lane 16 g + n, 16 bytes to a piece
 *   base.v_pool  [num_v_planes][L][Hkv][num_pages][S][64][16]: token 32 T + 8 g + i (i < 8),
 *                dims 32 s + 2 n and + 1: byte 8 T + i of lane 16 g + n of piece s
 *   k_exp        [num_k_planes][L][Hkv][num_pages][16][4 S]: the token and block above are
 *                byte (2 T + e) S + s of n
 *   v_exp        [num_v_planes][L][Hkv][num_pages][4][S][16]: byte 8 T + i of (g, s)
 *
 * base.dtype is the type of queries, block K/V, outputs, committed K/V and what is read back;
 * the other fields of `base` are as in das_cache. All four arrays are 16-byte aligned. Bytes
 * 0..252 keep every element within the range of both types. Places that hold no token of a
 * sequence (behind its length) may hold anything.
 */
typedef struct das_cache_q4 {
  das_cache base;
  uint8_t *k_exp;
  uint8_t *v_exp;
} das_cache_q4;

/*
 * das_attn_policy over a 4-bit cache: prefix keys at depth kappa and values at depth nu are
 * the elements above, block keys and values are the caller's in base.dtype. Arguments, masks,
 * bounds and error words as for das_attn_policy, and the same limits (w in
 * 1..DAS_MAX_BLOCK, Hq / Hkv <= 8), for any batch size.
 *
 * Numerics: cached elements are exact in the products' types. bf16 calls round probabilities
 * to bf16 for cached values, and to twice its bits for block values; fp32 calls take every
 * factor with its 24 bits, as far as they are 2^-133 or more. Accumulation and softmax
 * statistics are fp32, for logits of any finite size; sums are divided last, so that values
 * whose sum over the positions passes the largest fp32 give infinities. Block values that are
 * infinite or NaN reach only the rows that see them; a position whose logit is -infinity has
 * no weight (in fp32 calls an infinite key times a query of less than 2^-93 is NaN). Sequences
 * that are cut into parts are joined from the parts' results, in bf16 calls from fp16 relative
 * to each row's largest: what is under 2^-39 of it in its part is lost. lse as for
 * das_attn_policy.
 *
 * das_attn_q4_workspace_bytes returns 0 for arguments that das_attn_q4 rejects; the
 * workspace is 256-byte aligned, needs no init, and calls that run concurrently need
 * separate ones.
 */
size_t das_attn_q4_workspace_bytes(const das_cache_q4 *cache, const das_batch *batch,
                                   int32_t num_q_heads, int32_t block_len);
das_status das_attn_q4(const das_cache_q4 *cache, const das_batch *batch, int32_t layer,
                       int32_t kappa, int32_t nu, int32_t num_q_heads, int32_t block_len,
                       const void *q, const void *k_blk, const void *v_blk, void *out, float *lse,
                       void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * das_kv_append into a 4-bit cache. Arguments as for das_kv_append, with k_new and v_new in
 * base.dtype; len_out must share no element with batch->prefix_len or num_new
 * (DAS_ERR_SHAPE). The grid is one workgroup of 256 per (plane, layer) and 12 blocks of a
 * token's heads: these must be fewer than 2^24 (DAS_ERR_SHAPE), in das_kv_read_q4 too.
 *
 * A block gets the smallest exponent e in -120..125 with |x| <= 7 * 2^e for its 32 elements,
 * so that none is further from its code than half the distance of the largest two (4 and 6).
 * Codes are x * 2^-e rounded to the nearest, ties to an even code, past 6 to 6. A block with
 * a NaN or an infinity gets byte 255. Tokens share nothing: the result does not depend on
 * which tokens are committed together, and places of other tokens are left as they were.
 */
das_status das_kv_append_q4(const das_cache_q4 *cache, const das_batch *batch, const void *k_new,
                            const void *v_new, int32_t w_max, const int32_t *num_new,
                            int32_t *len_out, hipStream_t stream);

/* Largest row count per sequence of das_kv_read_q4. */
#define DAS_MAX_READ (1 << 20)

/*
 * Cached elements back in base.dtype, in the layout of a commit's inputs: positions first[b]
 * .. first[b] + num[b] - 1 of sequence b, of every stored plane and core layer. For moving a
 * sequence to a cache of another kind (with das_kv_append), or a block's K/V out of it.
 *
 *   k_out  [num_k_planes][L][B][w_max][Hkv][head_dim]  written, rows past num[b] left alone
 *   v_out  [num_v_planes][L][B][w_max][Hkv][head_dim]  the same
 *   first  device [B], num device [B] in 0..w_max: the positions must lie in the prefix
 *          (first[b] + num[b] <= prefix_len[b]); else nothing of the sequence is written
 *          (DAS_DEVERR_PREFIX). Positions on a page out of range are not written
 *          (DAS_DEVERR_PAGE).
 *
 * w_max in 1..DAS_MAX_READ, batch * w_max * Hkv * head_dim < 2^46. k_out and v_out are
 * 16-byte aligned and overlap neither the cache nor each other (DAS_ERR_SHAPE).
 */
das_status das_kv_read_q4(const das_cache_q4 *cache, const das_batch *batch, const int32_t *first,
                          const int32_t *num, int32_t w_max, void *k_out, void *v_out,
                          hipStream_t stream);

/*
 * Norms of queries and keys for each head and their rotation by position, in one pass: what
 * comes between a projection and das_attn_policy.
 *
 *   y = x * weight / sqrt(mean(x^2) + eps)                     over a head's head_dim elements
 *   (y_i, y_j) -> (y_i cos t - y_j sin t, y_j cos t + y_i sin t),  t = position * inv_freq[pair]
 *
 * The first rotary_dim dims are rotated, in pairs (i, i + rotary_dim / 2), or (2 i, 2 i + 1)
 * where `interleaved` is not 0; the others are only normalised. Values, if given, are copied:
 * the block K/V of an attention or a commit are rows without gaps, a projection's need not be.
 *
 *   q  [B][w][Hq][head_dim], k, v [B][w][Hkv][head_dim] with the distances of sequences and
 *      of tokens in elements (heads lie side by side), so that the three may be parts of one
 *      projection's output. v may be NULL, and then v_out is.
 *   q_out, k_out, v_out   without gaps. An output may be its own input where that has no gaps;
 *      else outputs overlap no input and no other output (DAS_ERR_SHAPE).
 *   q_weight, k_weight    device [head_dim] in `dtype`, or NULL: no norm of these
 *   inv_freq   device [rotary_dim / 2] fp32
 *   positions  device [B] int32: the position of a sequence's first token (prefix_len); or,
 *      with each_position not 0, [B][w]
 *
 * head_dim 64, 96 or 128; rotary_dim a multiple of 16 in 0..head_dim (0: norm only, inv_freq
 * may be NULL); Hq, Hkv in 1..65535; w in 1..DAS_MAX_READ, batch * w < 2^24; eps >= 0 and
 * finite. Distances are multiples of 16 bytes, rows are 16-byte aligned. Angles are taken in
 * 64 bits, the mean in 64, the rest in fp32, and results are rounded once. A head of zeros
 * with eps 0 gives NaN.
 */
typedef struct das_rope {
  int32_t dtype;          /* das_dtype of q, k, v, weights and outputs */
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t rotary_dim;
  int32_t interleaved;
  int32_t each_position;
  float eps;
  const float *inv_freq;
  const void *q_weight;
  const void *k_weight;
} das_rope;
das_status das_qk_rope(const das_rope *rope, int32_t batch, int32_t block_len, const void *q,
                       int64_t q_batch_stride, int64_t q_token_stride, const void *k,
                       int64_t k_batch_stride, int64_t k_token_stride, const void *v,
                       int64_t v_batch_stride, int64_t v_token_stride, const int32_t *positions,
                       void *q_out, void *k_out, void *v_out, hipStream_t stream);

/*
 * Verification of a block whose proposals were drawn from the draft's distributions, on the
 * device: das_greedy_accept for sampling. Every emitted token is a draw from the target's
 * distribution, whatever the draft's is; the nearer the two are, the more is accepted.
 *
 * Row (b, i) has the target's distribution p_i = softmax(target / temperature[b]) and the
 * draft's q_i = softmax(draft / draft_temperature[b]), where the proposals must have been
 * drawn (das_sample without filters; a caller's filter puts -inf in the logits of both). NaN
 * logits count as -inf; a temperature of 0 makes the distribution one-hot at the largest
 * logit, lowest index first, and a row without any logit above -inf is one-hot at token 0.
 * Without draft logits q_i is one-hot at the proposal (a greedy draft).
 *
 * The first m_b = tested[b] proposals are checked in order; y_i is accepted while
 * uniform[b][i] * q_i(y_i) < p_i(y_i). With a_b accepted, the next token is drawn with draw[b]
 * - from max(p - q, 0) of position a_b where that was rejected (a difference below 2^-40 of
 *   p counts as 0; where none is left, from p),
 * - from p of position a_b where a_b = m_b < w,
 * and with a_b = w none is. The token drawn is the first in index order at which the running
 * sum passes draw[b] times the whole. Weights are 64-bit exponentials relative to the row's
 * largest: a logit more than 745.1 temperatures below it weighs nothing, and its token is neither
 * accepted nor drawn, with numbers of 0 either.
 *
 *   proposals    device [B][w] int32. One that is checked and lies outside the vocabulary is
 *                rejected, with the whole of p as the residual but for q
 *                (DAS_DEVERR_PROPOSAL)
 *   target_logits, draft_logits   device rows of `vocab` elements of `dtype`, in the order
 *                [B][w], their distances in elements (>= vocab); draft_logits may be NULL
 *   temperature, draft_temperature   device [B] fp32, or NULL: 1. One that is NaN, negative
 *                or infinite counts as 0 (DAS_DEVERR_SAMPLE)
 *   tested       device [B] int32 or NULL (w), clamped to 0..w (DAS_DEVERR_TESTED)
 *   uniform      device [B][w] fp32, draw device [B] fp32, in [0, 1). A uniform outside
 *                rejects its proposal, a draw outside counts as 0 (DAS_DEVERR_SAMPLE)
 *   accepted, num_keep, num_emitted, emitted   written as by das_greedy_accept: a_b,
 *                min(a_b + 1, w) (das_kv_append's num_new), the same, and the tokens;
 *                emitted and num_emitted may be NULL
 *   probs        device [B][w] fp32 or NULL, written: p of the emitted tokens
 *   workspace    >= das_sampled_accept_workspace_bytes(...), 256-byte aligned, needs no init;
 *                calls that run concurrently need separate ones
 *   dev_error    optional device word
 *
 * Rows past what is checked (and the row after it) are not read. batch in 1..65535, block_len
 * in 1..DAS_MAX_BLOCK, vocab in 1..DAS_MAX_VOCAB. Logits are aligned to their type, the other
 * arrays to 4 bytes; outputs overlap neither the inputs nor each other (DAS_ERR_SHAPE). Entries
 * of emitted and probs past num_emitted[b] are left alone. Equal calls give equal bits.
 */
size_t das_sampled_accept_workspace_bytes(int32_t batch, int32_t block_len, int32_t vocab);
das_status das_sampled_accept(int32_t batch, int32_t block_len, int32_t vocab, int32_t dtype,
                              const int32_t *proposals, const void *target_logits,
                              int64_t target_stride, const void *draft_logits,
                              int64_t draft_stride, const float *temperature,
                              const float *draft_temperature, const int32_t *tested,
                              const float *uniform, const float *draw, int32_t *accepted,
                              int32_t *num_keep, int32_t *emitted, int32_t *num_emitted,
                              float *probs, void *workspace, size_t workspace_bytes,
                              uint32_t *dev_error, hipStream_t stream);

/* Static description of a status code; never NULL. */
const char *das_status_string(das_status status);

/* Library version as major * 10000 + minor * 100 + patch. */
int32_t das_version(void);

#ifdef __cplusplus
}
#endif

#endif /* DAS_H */
