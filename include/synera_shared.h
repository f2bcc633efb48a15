/*
 * synera_shared.h - C ABI of the decoder operators around a paged cache whose pages requests may share:
 * rotary positions, norms of query and key heads with the rotation, appends with the rotation on the way, and
 * attention whose shared prefixes are read once for all requests.  General rules, status codes and the layout of
 * the pools are those of synera.h; the decoders may be others than the one synera_verify runs.
 *
 * Element types: 0 = f32, 1 = bf16, 2 = f16.  The cache is bf16, gains are bf16.
 * Arithmetic is 32-bit throughout, angles are 64-bit; each output is rounded once, to nearest even.
 * The handles belong to the HIP device that was current when they were made: a call with another device current is
 * refused (EINVAL).  They must outlive the graphs that captured calls with them.  Nothing here waits for the GPU except
 * the creates and destroys, and synera_batch_plan if it runs more than four plans ahead of its uploads.  Destroys leave a capture of
 * any stream alone; creates, like other allocations, end one that is under way.
 */
#ifndef SYNERA_SHARED_H
#define SYNERA_SHARED_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------- rotary positions
 * Pair i of a head turns by the angle pos * f_i: (a, b) -> (a c - b s, b c + a s), c and s the angle's cosine and sine
 * times `magnitude`.  The pairs are the first rot_dim values of a head: (2 i, 2 i + 1) where interleaved,
 * (i, i + rot_dim / 2) where half; values from rot_dim on pass unchanged.  f_i = base^(-2 i / rot_dim), and
 *   SYNERA_ROPE_LINEAR  f_i / factor
 *   SYNERA_ROPE_BANDS   with r = original * f_i / (2 pi) turns over the original context: f_i / factor for r <= low,
 *                       f_i for r >= high, and (1 - t) f_i / factor + t f_i, t = (r - low) / (high - low), between
 * or the caller's own table.  pos * f_i / (2 pi) is formed in 64 bits and only what is left of whole turns is rounded to
 * 32: with |f_i| <= 1 any int32 position is good to 5e-7 rad.
 */
#define SYNERA_ROPE_INTERLEAVED 0
#define SYNERA_ROPE_HALF 1
#define SYNERA_ROPE_PLAIN 0
#define SYNERA_ROPE_LINEAR 1
#define SYNERA_ROPE_BANDS 2

typedef struct synera_rope_desc {
  int32_t head_dim;          /* even, 2 .. 256                                              */
  int32_t rot_dim;           /* even, 2 .. head_dim                                         */
  int32_t layout;            /* SYNERA_ROPE_INTERLEAVED or SYNERA_ROPE_HALF                 */
  int32_t scaling;           /* SYNERA_ROPE_PLAIN, _LINEAR or _BANDS                        */
  double base;               /* > 1                                                         */
  double factor;             /* LINEAR, BANDS: > 0                                          */
  double low, high;          /* BANDS: 0 <= low < high                                      */
  double original;           /* BANDS: > 0                                                  */
  double magnitude;          /* of cos and sin, finite in f32; 1 for a rotation proper      */
  const double* h_inv_freq;  /* HOST [rot_dim / 2] f_i in place of base and scaling, or NULL */
} synera_rope_desc;

typedef struct synera_rope synera_rope;

/* Errors: EINVAL (null, a value outside the ranges above or not finite, an f_i whose 2^31 f_i / (2 pi) is not finite in 64 bits), EUNSUP (head_dim > 256), EHIP, ENOMEM. */
int32_t synera_rope_create(synera_rope** out, const synera_rope_desc* desc);
/* Waits for the device.  NULL is allowed. */
int32_t synera_rope_destroy(synera_rope* rope);

/* The heads of one tensor, [tokens][n_heads][head_dim] with the values of a head side by side and any strides between
 * heads and tokens (in elements, >= 0).  Outputs must not lie on one another; d_out == d_in with the same strides
 * works in place, any other overlap of an output with an input of the call is refused where it shows (EINVAL). */
typedef struct synera_heads {
  const void* d_in;
  void* d_out;
  const void* d_gain;        /* bf16 [head_dim]: the norm's gains, or NULL where the heads are not normed */
  int32_t n_heads;
  int32_t n_rows;            /* tokens that d_in and d_out have room for, 0: not said.  Calls with a batch look at it */
  int64_t in_token, in_head;
  int64_t out_token, out_head;
} synera_heads;

/*
 * Turns the heads of q and of k (NULL: none) of n_tokens tokens by their positions d_pos (device i32 [n_tokens], any
 * values).  In and out have the type `dtype`; gains must be NULL.  n_tokens == 0 is a no-op.
 * Errors: EINVAL (null, sizes, strides, a pointer off its type's alignment, gains), EUNSUP (tokens x heads >= 2^31), EHIP.
 */
int32_t synera_rope_apply(const synera_rope* rope, int32_t dtype, int64_t n_tokens, const int32_t* d_pos,
                          const synera_heads* q, const synera_heads* k, void* stream);

/*
 * The same behind an RMS norm of each head, x g / sqrt(mean(x^2) + eps) over all its head_dim values, in one pass: the
 * normed values are never rounded.  q and k need their gains.  Errors: as synera_rope_apply, EINVAL for eps < 0.
 */
int32_t synera_qk_norm_rope(const synera_rope* rope, int32_t dtype, int64_t n_tokens, const int32_t* d_pos,
                            const synera_heads* q, const synera_heads* k, float eps, void* stream);

/* ------------------------------------------------------------------------------------------- batches that share pages
 * A batch is what one step of a serving loop runs: request i has L_i cached tokens and appends n_i new ones, at positions
 * L_i .. L_i + n_i - 1, through its row of the block table.  Requests may share pages: the same page ids in the same
 * first columns of their rows, whole pages of cached tokens (column < L_i / 16 in every request that names the page).
 * n_i == 0 keeps a place in the batch without rows.  A batch is planned once a step and then used for each layer.
 */
typedef struct synera_batch synera_batch;

/* head_dim 64 or 128, n_q_heads a multiple of n_kv_heads, at most 1024; room for max_batch requests, max_tokens new tokens
 * a plan, max_pages block-table columns.  Keeps 0.3 to 0.6 GB of device memory (head_dim 128; half of it at 64) for partial
 * results, and the plan on the device and four times in pinned host memory.  Errors: EINVAL, EUNSUP, EHIP, ENOMEM. */
int32_t synera_batch_create(synera_batch** out, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_batch,
                            int32_t max_tokens, int32_t max_pages);
/* Waits for the device.  NULL is allowed. */
int32_t synera_batch_destroy(synera_batch* batch);

/*
 * Host-only validation of a batch (callable without a GPU), what synera_batch_plan applies.
 *   EINVAL: null pointer, B < 1, n_new[i] < 0, max_pages < 1, n_pages_in_pool < 1
 *   ERANGE: ctx_len[i] < 0; a needed page id outside the pool; a page used twice other than as a shared prefix
 *   ENOSPC: B > max_batch; sum of n_new > max_tokens; ceil((ctx_len[i] + n_new[i]) / 16) > max_pages
 *   EUNSUP: n_pages_in_pool >= 2^27
 * Block-table entries beyond the pages a request needs are ignored.
 */
int32_t synera_validate_shared(int32_t B, const int32_t* h_ctx_len, const int32_t* h_n_new, const int32_t* h_block_table,
                               int32_t max_pages, int32_t n_pages_in_pool, int32_t max_batch, int64_t max_tokens);

/*
 * Plans a batch: finds the shared prefixes, cuts the attention's work, and uploads both on `stream`.  The calls below
 * must be on the same stream, or ordered behind it by the caller; so must a plan behind calls that use the one before.
 * Not while the stream is being captured (EINVAL).  Calls that were captured into a graph work for any later plan of
 * this batch: what is planned is read on the device; their tensors and pools need room for the tokens and pages of those
 * plans, which nothing checks.  That no output lies on an input or on itself is checked, when they are captured, for as many tokens as
 * the smallest n_rows of the call (for two, or those of the plan at hand, where none is said).  max_pages: columns of h_block_table (<= the batch's).  A refused
 * plan leaves the one before as it was.  Errors: as synera_validate_shared, EHIP, ENOMEM.
 */
int32_t synera_batch_plan(synera_batch* batch, int32_t B, const int32_t* h_ctx_len, const int32_t* h_n_new,
                          const int32_t* h_block_table, int32_t max_pages, int32_t n_pages_in_pool, void* stream);

/*
 * One layer's new tokens: queries turned into q->d_out (bf16; q NULL: no queries), keys turned into their pages, values into
 * theirs.  Inputs of type `dtype`, T = sum n_new tokens, request after request; heads are normed first where they come
 * with gains (not v).  k->d_out, v->d_out and their strides are not looked at.  d_k_layer, d_v_layer: one layer of the pools,
 * 16-byte aligned, of at least the planned n_pages_in_pool pages.  Slots that are not appended to stay as they were.
 * Outputs must not lie on inputs (but for q in place, bf16) nor on the pools.
 * Errors: EINVAL (also: no plan, head counts or head_dim other than the batch's, n_rows below the plan's tokens), EHIP.
 */
int32_t synera_append_rope(synera_batch* batch, const synera_rope* rope, int32_t dtype, const synera_heads* q,
                           const synera_heads* k, const synera_heads* v, float eps, void* d_k_layer, void* d_v_layer,
                           void* stream);

/*
 * o = softmax(scale q K^T) V of one layer: new token j of request i sees the keys at positions 0 .. L_i + j, its own
 * included (append first).  Query head h reads KV head h / (n_q_heads / n_kv_heads).  A prefix that requests share is
 * read once for all of them where that is the shorter way.
 *   q->d_in, q->d_out   bf16 [T][n_q_heads][head_dim], rotated queries in, o out; gains unused.  Not in place.  d_in and its
 *                       strides on 16 bytes, d_out and its strides on 8
 *   scale               > 0, finite in 32 bits times log2 e: below 2.35e38 (0 takes 1 / sqrt(head_dim)).  Scores scale q k beyond that do
 *                       not fit 32 bits either: their rows may be NaN
 *   d_lse               f32 [T][n_q_heads], ln sum exp(scale q k), or NULL
 * Softmax statistics and sums are 32-bit; the probabilities meet the bf16 values as bf16.  Keys and values that a
 * row does not see may hold anything, infinities and NaN too.  Outputs must not lie on inputs.  Calls with one batch
 * must be ordered (they share its scratch), in graphs as well.  Errors: EINVAL, EHIP.
 */
int32_t synera_shared_attention(synera_batch* batch, const synera_heads* q, const void* d_k_layer, const void* d_v_layer,
                                float scale, float* d_lse, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SYNERA_SHARED_H */
