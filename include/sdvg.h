/*
 * sdvg.h -- C ABI of libsdvg: block-causal attention over a KV cache, KV-cache commit and
 * rollback, and worst-frame routing, for speculative decoding of autoregressive video
 * generation (SDVG) on AMD MI355X (gfx950).
 *
 * Conventions shared by every call
 *   - Pointers named "device" are HIP device pointers owned by the caller; the library never
 *     frees or reallocates them. Pointers named "host" are ordinary host memory.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *   - Every call returns an int: >= 0 on success, a negative sdvg_status on error. Arguments
 *     are validated on the host before anything is launched; on error nothing is launched
 *     and no state (device memory, descriptor fields) is changed. No call throws or aborts.
 *   - Strides are in elements of the tensor's type; the innermost (dim) stride is always 1.
 *   - Logical index order is (layer, token, head, dim). head_dim must be 128.
 *   - bf16 tensors are raw bfloat16 bit patterns (2 bytes per element).
 */
#ifndef SDVG_H
#define SDVG_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SDVG_OK = 0,
  SDVG_ERR_NULL = -1,        /* a required pointer is NULL */
  SDVG_ERR_SHAPE = -2,       /* a size is non-positive or inconsistent */
  SDVG_ERR_RANGE = -3,       /* slot / length / threshold outside its valid range */
  SDVG_ERR_ALIGN = -4,       /* pointer not 16-byte aligned, or stride not a multiple of 8 */
  SDVG_ERR_UNSUPPORTED = -5, /* head_dim != 128, unknown dtype, stride >= 2^30 elements */
  SDVG_ERR_DEVICE = -6       /* a HIP runtime call failed (see sdvg_last_device_error) */
} sdvg_status;

enum { SDVG_BF16 = 0, SDVG_F32 = 1, SDVG_F16 = 2, SDVG_E4M3 = 3 }; /* the last two: paged cache only */

/* Key-split policy of sdvg_block_attn_batch (see there). */
enum { SDVG_SPLIT_NEVER = 0, SDVG_SPLIT_AUTO = 1, SDVG_SPLIT_ALWAYS = 2 };

/*
 * Describes the caller-owned KV cache of one model: two device arrays k and v of bf16,
 * logical [n_layers][capacity_tokens][n_heads][head_dim]. cache_len is a HOST field: the
 * number of valid tokens (the same in every layer); commit and rollback update it at enqueue
 * time, so later calls on the same stream see a consistent length.
 */
typedef struct {
  void *k, *v;              /* device */
  int32_t n_layers, n_heads, head_dim;
  int32_t block_tokens;     /* T: tokens per video block (3 latent frames) */
  int64_t capacity_tokens;  /* tokens allocated per layer */
  int64_t cache_len;        /* valid tokens, 0 <= cache_len <= capacity_tokens */
  int64_t layer_stride, token_stride, head_stride; /* elements */
} sdvg_kv_cache;

/* Shapes and strides of one attention call (one layer, one denoising step). */
typedef struct {
  int32_t n_q;      /* query tokens of the current block */
  int32_t n_blk;    /* key/value tokens of the current block (normally == n_q) */
  int32_t n_heads;
  int32_t head_dim; /* must be 128 */
  int64_t q_token_stride, q_head_stride;     /* q */
  int64_t o_token_stride, o_head_stride;     /* out */
  int64_t kv_token_stride, kv_head_stride;   /* k_cache, v_cache (one layer) */
  int64_t blk_token_stride, blk_head_stride; /* k_blk, v_blk */
  float scale;      /* softmax scale; 0 selects 1/sqrt(head_dim), the paper's models' value */
  int32_t dtype;    /* SDVG_BF16: all tensors bf16. SDVG_F32: all tensors fp32 (check path) */
} sdvg_attn_desc;

/*
 * Block-causal attention of one video block over the KV cache (paper Sec. 1: blocks are
 * generated against a shared KV cache; Sec. 4.1 "Models": causal attention backbone with KV
 * caching). For every head h and query row i:
 *     out[i,h,:] = sum_j p_ij V[j,h,:],   p_i = softmax_j(scale * q[i,h,:] . K[j,h,:]),
 * where K, V are the cache's first cache_len tokens followed by the block's n_blk tokens.
 * No mask: a block's queries see the whole cache and the whole block.
 *   desc      host. Shapes, strides, scale, dtype.
 *   q         device [n_q][n_heads][128]; k_blk, v_blk device [n_blk][n_heads][128].
 *   k_cache, v_cache  device, ONE layer's base pointers, at least cache_len tokens; may be
 *             NULL when cache_len == 0. Tokens at or past cache_len are never read.
 *   out       device [n_q][n_heads][128], same dtype as the inputs; every element is written. It may be q
 *             itself (same address and strides: in place); any other overlap with an input is the caller's error.
 *   Arithmetic (bf16): products on the matrix cores with fp32 accumulation, fp32 softmax
 *   statistics, probabilities rounded to bf16 before the PV product (the row sum is taken over
 *   the rounded values), bf16 output (RNE). SDVG_F32 is a slow all-fp32 check path: a separate,
 *   simple kernel that validates the mathematics (softmax over the concatenation) to 1e-4; it
 *   shares no tiling or copy logic with the bf16 kernel and says nothing about that kernel's
 *   indexing.
 *   scale must be finite and >= 0 (0 = 1/sqrt(head_dim)), else SDVG_ERR_RANGE. Inputs are
 *   assumed finite.
 * Asynchronous: enqueued on `stream`; returns SDVG_OK or a negative status. The call only
 * launches kernels (one, or two over different heads or rows), so it may be recorded into a HIP graph -- but the first SDVG_BF16 call on
 * a device also raises that kernel's dynamic-LDS limit (once per device, thread-safe), which
 * is not a capturable operation: make one eager call on the device before capturing.
 */
int sdvg_block_attn(const sdvg_attn_desc *desc, const void *q, const void *k_cache,
                    const void *v_cache, const void *k_blk, const void *v_blk,
                    int64_t cache_len, void *out, void *stream);

/*
 * Attention with the commit fused in (paper Sec. 3 "Inference flow": the block the target keeps
 * -- an accepted draft, or the target's own regeneration -- updates its KV cache): sdvg_block_attn
 * for one layer (bf16 only), and in the same launch (or two) the block's K and V rows are copied into
 * tokens [cache_len, cache_len + n_blk) of k_cache / v_cache (this layer's base pointers, which
 * must have room for them), addressed with the descriptor's kv strides. Meant for the LAST
 * denoising step of a block: the copy runs on compute units the attention leaves idle (behind the
 * attention where they would not be done in time), so the block's commit costs no extra launch and little or no time. The attention result is bit-identical to
 * sdvg_block_attn's; the copied rows are bit-exact. k_blk / v_blk must not overlap the
 * destination rows (SDVG_ERR_RANGE). The cache length is the caller's to advance: after the
 * call has been made for every layer, sdvg_kv_commit_mark(cache, slot) moves the descriptor's
 * cache_len to (slot + 1) * T under the same append-only rule as sdvg_kv_commit, without
 * touching device memory. Asynchronous on `stream`.
 */
int sdvg_block_attn_commit(const sdvg_attn_desc *desc, const void *q, void *k_cache, void *v_cache,
                           const void *k_blk, const void *v_blk, int64_t cache_len, void *out,
                           void *stream);
int sdvg_kv_commit_mark(sdvg_kv_cache *cache, int32_t slot);

/*
 * The same attention for up to 8 independent (q, cache, block, out) sets in ONE call -- e.g. the
 * conditional and the unconditional pass of classifier-free guidance (paper Sec. 4.1 "Models":
 * guidance scale 3.0), which share shapes and cache length but have their own tensors. Result
 * item by item as n_items calls of sdvg_block_attn (same softmax, same error bounds; also the same
 * bits where both take workgroups of the same shape, see below); one launch for all fills the chip better
 * and halves the launch count.
 *   n_items   1 .. 8. q, k_cache, v_cache, k_blk, v_blk, out: HOST arrays of n_items device
 *             pointers (k_cache / v_cache and their entries may be NULL when cache_len == 0).
 *             All items share desc (shapes, strides, scale, dtype) and cache_len. out[i] may be q[i], but
 *             not overlap another item's tensors.
 *   workspace device, nullable, 16-byte aligned, workspace_bytes long; split_mode one of
 *             SDVG_SPLIT_*. Without a workspace (or with SDVG_SPLIT_NEVER) every query tile is
 *             one workgroup: 256 rows, or, when the launch has few of those, 128, 64 or 32 rows whose
 *             keys are dealt out over 2, 4 or 8 parts of the workgroup's waves; where these fill some rounds and a small
 *             part of another, the heads or rows of the whole rounds and the others are launched one after the other. With a workspace of at least
 *             sdvg_block_attn_workspace_bytes(desc, n_items, cache_len, split_mode) bytes the
 *             library may cut the keys of every query tile and deal them out about evenly over whole
 *             rounds of workgroups instead, so that a launch with few query tiles still fills the
 *             chip, and merge the partial results in a second small kernel on the same stream. SDVG_SPLIT_AUTO does so when at least a quarter of the
 *             workgroup slots of the launch's rounds would idle (few heads or short blocks) and the keys are many
 *             enough for it to be the faster way (otherwise the workspace stays unused); SDVG_SPLIT_ALWAYS
 *             whenever the query tiles do not fill whole rounds. For the paper's own shapes the
 *             split does not pay (a 12-head drafter layer has 228 query tiles for 256 compute
 *             units; the split costs more than the 11 % it could win) and AUTO leaves them alone.
 *             Same softmax and same error bounds; not bit-identical to the unsplit result (P is
 *             rounded to bf16 against each piece's own running maximum). A workspace that is
 *             too small is ignored (plain launch). The workspace is scratch: contents are
 *             undefined afterwards; concurrent calls need their own.
 * Errors as sdvg_block_attn, plus SDVG_ERR_SHAPE for n_items outside 1 .. 8 or a negative
 * workspace_bytes and SDVG_ERR_UNSUPPORTED for an unknown split_mode. Asynchronous on `stream`.
 */
int sdvg_block_attn_batch(const sdvg_attn_desc *desc, int32_t n_items, const void *const *q,
                          const void *const *k_cache, const void *const *v_cache,
                          const void *const *k_blk, const void *const *v_blk, int64_t cache_len,
                          void *const *out, void *workspace, int64_t workspace_bytes,
                          int32_t split_mode, void *stream);

/*
 * sdvg_block_attn_batch for callers that cannot allocate device memory or provide a workspace:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc. Same
 * arguments, results and errors, but the partial results of a key split go to a fixed 64 MiB
 * array inside the library's device image (sdvg_block_attn_static_workspace_limit() bytes,
 * held by every GPU the library runs on until the process ends) instead of caller memory.
 * The call allocates nothing and frees nothing. A shape whose split needs more than the array
 * holds returns SDVG_ERR_RANGE (nothing is launched). Only SDVG_SPLIT_ALWAYS can need that much:
 * sdvg_block_attn_workspace_bytes with SDVG_SPLIT_ALWAYS tells the need beforehand. SDVG_SPLIT_NEVER
 * needs none. SDVG_SPLIT_AUTO splits from 60 % idle slots on here, not from a quarter on, and always
 * fits the array on a GPU with 256 compute units; what sdvg_block_attn_workspace_bytes returns for
 * SDVG_SPLIT_AUTO holds for sdvg_block_attn_batch alone and may be more than the limit where this call
 * does not split. Every call on a GPU uses that GPU's one
 * array: calls that overlap in time on one GPU (different streams or threads) race -- serialise
 * them, or use sdvg_block_attn_batch with workspaces of their own. Nothing in the array has to
 * be cleared between calls: each call writes every partial result it later reads.
 */
int sdvg_block_attn_batch_static(const sdvg_attn_desc *desc, int32_t n_items, const void *const *q,
                                 const void *const *k_cache, const void *const *v_cache,
                                 const void *const *k_blk, const void *const *v_blk, int64_t cache_len,
                                 void *const *out, int32_t split_mode, void *stream);
int64_t sdvg_block_attn_static_workspace_limit(void);

/*
 * Bytes of workspace with which sdvg_block_attn_batch may split keys for this shape and
 * split_mode on the current device; 0 if it would not split (then no workspace is needed). From 60 %
 * idle workgroup slots on, the size under SDVG_SPLIT_AUTO is that of the split, taken or not. On 256
 * compute units at most 277 MB, under SDVG_SPLIT_AUTO 182 MB. Negative sdvg_status on a bad
 * descriptor.
 */
int64_t sdvg_block_attn_workspace_bytes(const sdvg_attn_desc *desc, int32_t n_items, int64_t cache_len,
                                        int32_t split_mode);

/*
 * KV commit (paper Sec. 3 "Inference flow": an accepted draft block is committed to the
 * target's KV cache; a regenerated block updates it; the drafter's own cache is updated
 * unconditionally). Copies k_blk, v_blk -- device, dense [n_layers][T][n_heads][128] bf16 --
 * into tokens [slot*T, (slot+1)*T) of every layer, then sets cache->cache_len = (slot+1)*T.
 * Append-only: requires slot*T == cache->cache_len and (slot+1)*T <= capacity_tokens, else
 * SDVG_ERR_RANGE. k_blk / v_blk must not overlap the destination slot of any layer
 * (SDVG_ERR_RANGE). The descriptor's strides must keep rows and layers apart: the larger of
 * token_stride and head_stride steps over everything the smaller one spans, and layer_stride
 * over a whole layer (SDVG_ERR_SHAPE otherwise; the same check guards sdvg_kv_rollback).
 * One launch covers all layers. Asynchronous on `stream`.
 */
int sdvg_kv_commit(sdvg_kv_cache *cache, const void *k_blk, const void *v_blk, int32_t slot,
                   void *stream);

/*
 * Rotary position embedding of q / k rows (paper Sec. 4.1 "Models": KV caching "via RoPE positional
 * embeddings"; no formula is printed). Reading taken: elements 2i and 2i+1 of every head's vector
 * are the real and imaginary part of a complex number that is multiplied by exp(i * angle); the
 * angle of (token, pair i) is given by the caller as tables, so the position scheme is the
 * caller's. fp32 arithmetic in a fixed order, bf16 result (RNE):
 *     re' = fma(re, cos, -(im * sin)),   im' = fma(re, sin, im * cos).
 *   x, out     device bf16 [n_tokens][n_heads][128] with the given token / head strides
 *              (elements; multiples of 8, >= 128); out may be x itself (in place), otherwise the
 *              two must not overlap.
 *   cos_table, sin_table  device fp32, dense [n_tokens][64], 16-byte aligned.
 * head_dim must be 128. n_tokens == 0 is a no-op. Asynchronous on `stream`.
 */
int sdvg_rope(const void *x, const float *cos_table, const float *sin_table, void *out,
              int64_t n_tokens, int32_t n_heads, int32_t head_dim, int64_t x_token_stride,
              int64_t x_head_stride, int64_t out_token_stride, int64_t out_head_stride, void *stream);

/*
 * sdvg_kv_commit with the rotation of K fused into the copy: k_blk holds the block's keys BEFORE
 * the rotary embedding; they are rotated (as sdvg_rope, tables [T][64] shared by all layers) on
 * their way into the cache, v_blk is copied as it is. One pass over the block instead of two,
 * and the cache holds rotated keys, which is what sdvg_block_attn expects to find there. (Keys
 * are not rotated "on load" inside the attention kernel: its K tiles go from HBM to LDS without
 * passing registers, and each of a head's workgroups would rotate every tile again.)
 * Arguments, rules and errors otherwise as sdvg_kv_commit.
 */
int sdvg_kv_commit_rope(sdvg_kv_cache *cache, const void *k_blk, const void *v_blk, int32_t slot,
                        const float *cos_table, const float *sin_table, void *stream);

/*
 * KV rollback (paper Sec. 3 "Inference flow", reject branch: the target regenerates the block
 * as if the draft had never been in its cache). Sets cache->cache_len = new_len and zero-fills
 * tokens [new_len, old cache_len) of k and v in every layer, so no rejected data survives.
 * Requires 0 <= new_len <= cache->cache_len, else SDVG_ERR_RANGE; equal lengths is a no-op.
 * Asynchronous on `stream`.
 */
int sdvg_kv_rollback(sdvg_kv_cache *cache, int64_t new_len, void *stream);

/*
 * Snapshot / restore of an opaque device buffer (paper Sec. 3 "Inference flow" and Sec. 4.1
 * "Hardware and implementation": the VAE decode cache is cloned before a draft is scored and
 * restored when the draft is rejected). One call copies n_bytes from src to dst; cloning is
 * (snapshot <- live), restoring is (live <- snapshot). The library knows nothing of the contents.
 *   dst, src  device, 16-byte aligned, caller-owned, must not overlap (SDVG_ERR_RANGE).
 *   n_bytes   >= 0; 0 is a no-op that touches nothing (pointers may then be NULL).
 * Bit-exact; bytes outside [dst, dst + n_bytes) are not written. Asynchronous on `stream`.
 */
int sdvg_buffer_snapshot(void *dst, const void *src, int64_t n_bytes, void *stream);

/*
 * Worst-frame routing (paper Sec. 3 Eq. (1): q_b = min over the block's F decoded frames of
 * the per-frame reward; "Inference flow": accept iff q_b >= tau; "Force-reject the first
 * block": block 0 is always rejected, whatever its score).
 *   frame_scores  device, n_frames fp32 rewards (n_frames >= 1).
 *   tau           threshold; NaN -> SDVG_ERR_RANGE.
 *   block_idx     >= 0.
 *   q_b_out       host, nullable: receives q_b (also for block 0).
 * Any NaN score -> reject with q_b = quiet NaN (bits 0x7FC00000). Of +0.0 and -0.0 the
 * negative zero is the smaller, so q_b is bit-exact under any reduction order.
 * Synchronises `stream` (the caller branches on the result, as the paper's loop does).
 * Returns 1 (accept), 0 (reject) or a negative status.
 */
int sdvg_worst_frame_route(const float *frame_scores, int32_t n_frames, float tau,
                           int32_t block_idx, float *q_b_out, void *stream);

/*
 * Batched, asynchronous form of the same rule for n_blocks blocks at once.
 *   frame_scores  device [n_blocks][n_frames] fp32, dense.
 *   block_idx     device, n_blocks int32 (the block's position in its video), or NULL
 *                 meaning block i has index first_block_idx + i.
 *   decisions_out device, n_blocks int32 (1 accept / 0 reject); q_b_out device, n_blocks
 *                 fp32, nullable.
 * Does not synchronise. Returns SDVG_OK or a negative status.
 */
int sdvg_worst_frame_route_batch(const float *frame_scores, int32_t n_blocks, int32_t n_frames,
                                 float tau, const int32_t *block_idx, int32_t first_block_idx,
                                 int32_t *decisions_out, float *q_b_out, void *stream);

/*
 * Average-frame routing, the variant the paper's ablation compares with (Sec. 4.3 "Min-frame
 * vs. average-frame scoring", Table 2): q_b = mean of the block's F per-frame rewards instead
 * of their minimum; everything else (accept iff q_b >= tau, block 0 always rejected, NaN ->
 * reject with q_b = quiet NaN, arguments, return values, synchronisation) as in
 * sdvg_worst_frame_route / _batch. The mean is the fp64 sum of the rewards taken in frame order,
 * divided by F in fp64 and rounded once to fp32, so it is bit-exact against a sequential loop;
 * a mean that comes out NaN (+inf and -inf among the rewards) is reported as the same quiet NaN.
 */
int sdvg_avg_frame_route(const float *frame_scores, int32_t n_frames, float tau, int32_t block_idx,
                         float *q_b_out, void *stream);
int sdvg_avg_frame_route_batch(const float *frame_scores, int32_t n_blocks, int32_t n_frames,
                               float tau, const int32_t *block_idx, int32_t first_block_idx,
                               int32_t *decisions_out, float *q_b_out, void *stream);

/*
 * ---- Paged cache -----------------------------------------------------------------------------
 * Where many requests of different lengths are generated at once, token by token (a draft of a few tokens, then
 * their verification), a cache per request sized for the longest one does not pay. The paged cache is one pool
 * of pages of page_tokens tokens; a row of the block table lists a request's pages in order. One step of a model:
 *   sdvg_page_plan     once per step: pages for the new tokens, their slots and positions, from the requests' lengths
 *   sdvg_paged_commit  per layer: the new tokens' K (rotated) and V into their slots, q rotated in the same launch
 *   sdvg_paged_attn    per layer: every new token's attention over its request's cached tokens and itself
 * Undoing rejected tokens needs no call: the next plan is given the shorter lengths, the pages stay held. All
 * lengths, tables and slots are read on the device, so a captured graph of the step may be replayed with other values in
 * the same arrays. Device values out of range are never followed out of the arrays they index (each call says what
 * they mean).
 */

/* One layer's pools k and v: device, logical [n_pages][page_tokens][n_kv_heads][128], strides alike. */
typedef struct {
  void *k, *v;                    /* device, 16-byte aligned */
  const float *k_scale, *v_scale; /* device [n_kv_heads], nullable (1): a stored number x stands for x * scale */
  int32_t n_pages, page_tokens;   /* page_tokens: a multiple of 8; n_pages * page_tokens < 2^31 */
  int32_t n_kv_heads, head_dim;   /* head_dim must be 128 */
  int64_t page_stride, token_stride, head_stride; /* elements, multiples of 16 bytes; rows must not overlap */
  int32_t dtype;                  /* SDVG_BF16, SDVG_F16 or SDVG_E4M3 (largest 448, no infinities); scales with SDVG_E4M3 only */
} sdvg_paged_kv;

/*
 * Plan of one step: from c = cached[r] tokens in the cache and n = new_tokens[r] new ones of each of n_requests requests
 *   q_start[0] = 0, q_start[r + 1] = q_start[r] + n        rows of request r among all new tokens
 *   kv_lens[r] = c + n
 *   block_table[r][j], held[r] <= j < ceil((c + n) / page_tokens): the next pages of free_pages, request by request
 *                      in order, from place *next_free on; other entries stay as they are
 *   positions[t] = c + i, slots[t] = page * page_tokens + position % page_tokens    of the new token t = q_start[r] + i
 * A token without a page (free_pages ran out, the table is too narrow, the entry is negative) has slot -1; rows t
 * behind the last token have slot -1 and position 0. held_out[r] is the number of pages the request holds now and
 * *next_free_out = *next_free + all pages asked for: more than n_free says by how many they ran out.
 * Negative lengths, held pages and cursors count as 0. New tokens past max_tokens have pages, but no row: q_start, kv_lens,
 * positions and slots count them as not there.
 *   held     device [n_requests], or NULL: every page a request needs is in its row of the table already, none is taken
 *            (free_pages, next_free, held_out and next_free_out are then not used and may be NULL).
 *   next_free device, one int32, or NULL (0). free_pages may be NULL with n_free == 0.
 * Outputs must not overlap inputs or each other (SDVG_ERR_RANGE): the same call again gives the same answer. n_requests and
 * max_tokens may be 0. One launch, asynchronous on `stream`.
 */
typedef struct {
  int32_t n_requests, page_tokens; /* page_tokens: a multiple of 8 */
  int32_t table_width;             /* entries per row of the table, >= 1 */
  int32_t n_free;                  /* entries of free_pages */
  int64_t table_stride;            /* elements between rows of the table, >= table_width */
  int64_t max_tokens;              /* length of positions and slots, < 2^31 */
  const int32_t *cached, *new_tokens, *free_pages, *held, *next_free;               /* device */
  int32_t *block_table, *q_start, *kv_lens, *positions, *held_out, *next_free_out;  /* device */
  int64_t *slots;                                                                   /* device */
} sdvg_page_plan_args;
int sdvg_page_plan(const sdvg_page_plan_args *args, void *stream);

/*
 * Rotary embedding by positions. For pair p < rotary_dim / 2 of every row's vector, at angle = position * freqs[p],
 *     (a, b) -> (a c - b s, a s + b c),   c = gain * cos(angle), s = gain * sin(angle),
 * where (a, b) are elements (p, p + rotary_dim / 2) in SDVG_ROPE_HALF and (2p, 2p + 1) in SDVG_ROPE_INTERLEAVED; elements from
 * rotary_dim on are copied. The angle is taken modulo one turn in 64 bits and what their roundings leave, before
 * anything is rounded to 32, so all positions keep full accuracy; the rest is fp32, the result rounded once. Scaling for contexts
 * longer than the original one is in freqs and gain (the Python package's rope_frequencies makes them).
 *   positions device int32 [n_tokens], 4-byte aligned, of either sign; freqs device double [rotary_dim / 2], 8-byte aligned,
 *   in radians per position. rotary_dim: a multiple of 16, at most 128.
 */
enum { SDVG_ROPE_INTERLEAVED = 0, SDVG_ROPE_HALF = 1 };
typedef struct {
  const int32_t *positions; /* device */
  const double *freqs;      /* device */
  int32_t rotary_dim, layout;
  float gain;               /* finite */
} sdvg_rope_desc;

/* Rows [n_tokens][n_heads][128] that are read at in and written at out (which may be in itself, with the same strides;
 * otherwise they must not overlap, nor other rows of the call; an equal start is refused, SDVG_ERR_RANGE). 16-byte aligned;
 * strides in elements, multiples of 16 bytes below 2^30, those of dimensions of size 1 are not looked at. */
typedef struct {
  const void *in; /* device */
  void *out;      /* device */
  int32_t n_heads;
  int64_t in_token_stride, in_head_stride, out_token_stride, out_head_stride;
} sdvg_rows;

/*
 * Rotates x and, in the same launch, y (nullable: e.g. q and k of a layer), both of n_tokens tokens and of type `dtype`
 * (SDVG_BF16, SDVG_F16, SDVG_F32). n_tokens < 2^26 - 3; 0 is a no-op. Asynchronous on `stream`.
 */
int sdvg_rope_positions(const sdvg_rope_desc *rope, const sdvg_rows *x, const sdvg_rows *y, int64_t n_tokens,
                        int32_t head_dim, int32_t dtype, void *stream);

/*
 * Commit into the paged cache: k->in and v->in, rows [n_tokens][n_kv_heads][128] of type `dtype` (SDVG_BF16 or SDVG_F16; the
 * cache's own type unless that is SDVG_E4M3), go to slots[t] = page * page_tokens + place in the page. Rows whose slot is
 * negative or past the pools are not written. Slots that are written must differ (two rows of one slot: either may win, in parts).
 *   rope      nullable. K is rotated on its way (v is not); a 16-bit cache then holds what sdvg_rope_positions would give.
 *   q         nullable, needs rope: rows that are rotated to q->out in the same launch.
 *   SDVG_E4M3: stored = round(x * (1 / scale)) in fp32, clamped to +-448 first (NaN stays NaN); x is not rounded to `dtype` after
 *             the rotation.
 * k->out and v->out are not looked at. The sources and q->out must not overlap the pools (SDVG_ERR_RANGE). n_tokens < 2^26 - 3; 0 is a no-op.
 * Asynchronous on `stream`.
 */
int sdvg_paged_commit(const sdvg_paged_kv *cache, const sdvg_rows *k, const sdvg_rows *v, const int64_t *slots,
                      int64_t n_tokens, int32_t dtype, const sdvg_rope_desc *rope, const sdvg_rows *q, void *stream);

/*
 * Attention of the new tokens of every request over its pages. New token i of the n = q_start[r + 1] - q_start[r] tokens of
 * request r has position kv_lens[r] - n + i and sees the keys of its request at positions up to its own, with
 * window > 0 only the last `window` of them; its own K and V are in the cache already (sdvg_paged_commit). Query head h
 * belongs to key head h / (n_heads / n_kv_heads):
 *     out[t,h,:] = sum_j p_j V[j,:],  p = softmax_j(scale * q[t,h,:] . K[j,:]),  lse[t,h] = log sum_j exp(scale * q . K[j]).
 *   desc      host. dtype SDVG_BF16 or SDVG_F16 of q and out; the cache's own type unless that is SDVG_E4M3.
 *   q, out    device [n_tokens][n_heads][128]; out may be q itself (same strides). lse device float, dense
 *             [n_tokens][n_heads], nullable. Rows from q_start[n_requests] on, and below q_start[0], are left as they are.
 *   block_table  device int32 [n_requests][table_width]; q_start device int32 [n_requests + 1], not decreasing;
 *             kv_lens device int32 [n_requests], kv_lens[r] >= n: all as sdvg_page_plan leaves them.
 *             Keys on a page whose number is negative or not below n_pages, or past the table, count as not there. A row without any key gets
 *             out = 0 and lse = -infinity. A row whose scores are NaN gets NaN in both, and no other row sees it. Numbers
 *             out of range in q_start and kv_lens are clamped.
 *   workspace device, nullable, 16-byte aligned: with at least sdvg_paged_attn_workspace_bytes(desc, cache) bytes the keys of long
 *             requests are split over workgroups and the pieces joined by a second small launch; without, every
 *             request's keys are one workgroup's per key head and tile of rows. A workspace that is too small is ignored. The
 *             need may grow or shrink with n_requests, n_tokens and table_width: one that serves several shapes has the largest of
 *             their sizes. It is 0 where a row of the table names too few keys to be split (256). Scratch: overlapping calls need their own.
 *   Arithmetic: products on the matrix cores with fp32 accumulation, fp32 softmax statistics and sums; a probability goes into
 *   the product with V as two numbers of `dtype` that together have 16 (bf16) or 22 bits (fp16 down to 2^-16 of the largest one
 *   of the keys that a wave takes, below that in steps of 2^-37 of it), and whole into the sum; e4m3 numbers are exact in it. What
 *   lies in the cache outside of the keys that a row of the request sees (behind the last one, ahead of the first one's
 *   window) may be anything, and pages that hold nothing else need not be there; keys that any row of a request sees must be finite.
 *   Made for few new tokens per request (1 .. some 16); longer ones are right, but every 32 rows (tokens x query heads of a group)
 *   read all keys that any row of the request sees: a prompt of 4680 tokens, 40 / 8 heads, takes 1.15 ms. Made for some hundred
 *   requests: every workgroup looks through all their lengths, 64 at a time.
 * scale as in sdvg_attn_desc. n_requests and n_tokens may be 0 (no-op); n_tokens * n_heads < 2^31 - 64, and the
 * tiles of 16 or 32 rows times the key heads below some 2^23 (SDVG_ERR_UNSUPPORTED). Asynchronous on `stream`; launches kernels only.
 */
typedef struct {
  int32_t n_requests, n_tokens, n_heads, head_dim; /* n_heads: a multiple of the cache's; head_dim must be 128 */
  int32_t table_width, window;                     /* window: 0 = none */
  int64_t table_stride;                            /* elements */
  int64_t q_token_stride, q_head_stride, o_token_stride, o_head_stride;
  float scale;
  int32_t dtype;
} sdvg_paged_attn_desc;
int sdvg_paged_attn(const sdvg_paged_attn_desc *desc, const sdvg_paged_kv *cache, const void *q, const int32_t *block_table,
                    const int32_t *q_start, const int32_t *kv_lens, void *out, float *lse, void *workspace,
                    int64_t workspace_bytes, void *stream);
int64_t sdvg_paged_attn_workspace_bytes(const sdvg_paged_attn_desc *desc, const sdvg_paged_kv *cache);

/*
 * Measurement aid (no passage of the paper: it exists so that a benchmark can report what the
 * matrix cores of the chip it runs on deliver, next to the attention kernel's rate). Launches
 * 256 workgroups of 4 waves (one wave per SIMD of the chip); every wave issues iters x 16 v_mfma_f32_32x32x16_bf16 from
 * registers and nothing else. Asynchronous on `stream`; the caller times it.
 *   out        device, at least 65536 floats (n_out = its length): checksums, never read back.
 *   cycles     device, one uint64: shader clocks wave 0 took (clock = cycles / measured time).
 *   iters      1 .. 2^24.
 *   flops_out  host, nullable: the FLOPs the launch performs (256 x 4 x iters x 16 x 32768).
 * Returns SDVG_OK or a negative status.
 */
int sdvg_probe_mfma(float *out, int64_t n_out, uint64_t *cycles, int32_t iters, double *flops_out,
                    void *stream);

/*
 * The same measurement with operands that change: the A operand of every MFMA differs from the
 * previous one's and the B operand changes every second MFMA (register sets filled with random
 * signs and mantissas, magnitudes 1/8 .. 4), as the operands of an attention kernel do. The
 * chip holds a lower clock under this load than under sdvg_probe_mfma's, whose two operand
 * registers never change; this is the rate to compare a real kernel with.
 * Arguments, return values and FLOP count as for sdvg_probe_mfma.
 */
int sdvg_probe_mfma_changing(float *out, int64_t n_out, uint64_t *cycles, int32_t iters,
                             double *flops_out, void *stream);

/* Human-readable name of a status code (static storage; never NULL). */
const char *sdvg_status_string(int status);

/* hipError_t of the most recent SDVG_ERR_DEVICE on this thread, as an int (0 if none). */
int sdvg_last_device_error(void);

/* Library version, major*10000 + minor*100 + patch. */
int sdvg_version(void);

/* Releases the small pinned host buffer the router keeps. Safe to call more than once. */
void sdvg_shutdown(void);

#ifdef __cplusplus
}
#endif
#endif /* SDVG_H */
