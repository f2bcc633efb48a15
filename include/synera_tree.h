/*
 * synera_tree.h - C ABI of the operators that verify trees of drafted tokens with all lengths on the GPU: page tables and slot
 * maps, appends and attention of the trees over the paged cache, the path that is accepted with the move of its keys and values, and
 * penalties, biases and masks on the logits in between.  A step of a serving loop that uses them has no need to read anything back,
 * and all calls but creates and destroys may be captured into a graph.
 *
 * General rules, status codes and the layout of the pools are those of synera.h, element types, heads and the ownership of handles those
 * of synera_shared.h.  What the host says (sizes, pointers) is checked on the host: a refused call has launched nothing.  What only the
 * device knows is checked there: each request has a status of its own (0, or one of the codes of synera.h), and a refused request
 * changes nothing and has no outputs but those that say so: what a call would have written for its rows stays as it was, in a tensor that nothing else
 * filled as the memory was found.  Arrays named [rows] are flattened, request after request, and have as many
 * places as n_rows says; those behind the last request's stay as they were, but for the places of synera_pages_update.  Nothing here waits for the GPU but creates and destroys.
 */
#ifndef SYNERA_TREE_H
#define SYNERA_TREE_H

#include <stdint.h>

#include "synera_shared.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------- pages
 * The pages of a pool are in the rows of a block table or on a stack of free ones.  Row i holds the pages of its first d_held[i]
 * columns.  A call makes every row hold what its lengths need, ceil((L_i + n_i) / 16) pages:
 *   - rows that hold fewer take pages from the top of the stack, in the order of requests and columns.  Where the stack as it was
 *     before the call does not cover a request's and all those before it, the request and all later ones that need pages
 *     are refused (ENOSPC): their rows stay as they were, with fewer pages than their lengths need (synera_tree_plan_held refuses such requests);
 *   - rows that hold more return those behind, all but their first d_shared[i] columns; the first one returned ends on top.
 * So a step that is taken back leaves the stack as it was.  Entries behind a row's held columns and behind the stack's top stay.
 * Then each token's place, for token j of request i in row cu[i] + j:
 *   d_cu      i32 [B + 1]   prefix sums of n_i (of 0 where n_i is below 0 or above 16 x columns)
 *   d_pos     i32 [rows]    L_i + j, or -1 where the request is refused and behind the last request's tokens
 *   d_slot    i32 [rows]    page x 16 + slot in the page, or -1
 *   d_status  i32 [B]       0; ERANGE: L_i or n_i below 0, or L_i + n_i beyond int32; ENOSPC: more pages than columns, or than there are;
 *                           EINVAL: d_held[i] outside 0 .. columns
 * The lengths and d_shared are device i32 [B], d_shared may be NULL (none).  d_table is i32 [B][columns], d_free i32 [n_pages], d_n_free
 * i32 [1] (taken as 0 below 0, as n_pages above).  A page must be held once or be free once; nothing checks that.  n_rows may be 0 (d_pos and
 * d_slot are not looked at).  Rows of tokens beyond n_rows are left out.
 * What is written lies on no other array of the call.  Errors: EINVAL (null, sizes, pointers off 4 bytes, overlaps), EUNSUP (n_pages >= 2^27,
 * B x columns >= 2^27), EHIP.
 */
int32_t synera_pages_update(int32_t B, const int32_t* d_ctx_len, const int32_t* d_n_new, const int32_t* d_shared, int32_t* d_table,
                            int32_t columns, int32_t* d_held, int32_t* d_free, int32_t* d_n_free, int32_t n_pages, int64_t n_rows,
                            int32_t* d_cu, int32_t* d_pos, int32_t* d_slot, int32_t* d_status, void* stream);

/* ------------------------------------------------------------------------------------------- trees
 * Request i has L_i cached tokens and n_i nodes (0 .. SYNERA_TREE_NODES).  Node j has a parent among the nodes before it, or -1:
 * a child of the cached context.  It lies at position L_i + j of the cache, through the request's row of the block table, and is turned
 * by the position L_i + (nodes on its path) - 1 that it has in its text.  It sees the cached tokens, its path's nodes and itself.  A chunk is a
 * tree whose parents are j - 1.  Requests may share whole pages of cached tokens (they are read for each of them).
 */
#define SYNERA_TREE_NODES 256
typedef struct synera_tree synera_tree;

/* head_dim, n_q_heads, n_kv_heads as synera_batch_create; room for max_batch requests, max_tokens rows, max_pages block-table columns.
 * Keeps 35 (head_dim 64) or 68 MB of device memory for partial results, beside the plan.  Errors: EINVAL, EUNSUP (also: max_batch > 2^14, max_batch x n_q_heads >= 2^26,
 * max_tokens x n_q_heads or max_batch x (max_pages + 16) >= 2^30), EHIP, ENOMEM. */
int32_t synera_tree_create(synera_tree** out, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_batch,
                           int32_t max_tokens, int32_t max_pages);
/* Waits for the device.  NULL is allowed. */
int32_t synera_tree_destroy(synera_tree* tree);

/*
 * Rows are numbered as by synera_pages_update: cu_i sums up the n of the requests before, of 0 where n is below 0 or above 16 x columns, also
 * where n is more than a tree may have or the request is refused.  So with tables of the same columns both have the same rows for all requests.
 * Plans a step, once for all layers: d_ctx_len, d_n_nodes i32 [B], d_parent i32 [rows], d_table i32 [B][columns] (columns <= max_pages), all
 * read by this call alone.  The calls below must be on the same stream, or ordered behind it by the caller; so must a plan behind calls
 * that use the one before.  Captured calls work for any later plan of this handle (captured or not).  Calls look at what the last plan that was
 * called, or captured, says of rows and pages; once a plan was captured, those whose tensors say n_rows work on as many of the rows that the plan on the device has as there is room for, also where the last one that was called had none. Where a replayed plan on the device has more rows than a call's tensors (those that say n_rows),
 * the requests that do not lie in them whole are left out, as an accept or a commit leaves out requests beyond the B of the plan that it was called behind; before a captured plan's
 * first replay the handle has the requests of the plan before, or none.  That pools have room for a replayed plan's pages nothing checks.
 *   d_status  i32 [B], or NULL: 0; EINVAL: n_i outside 0 .. SYNERA_TREE_NODES, a parent outside -1 .. j - 1; ERANGE: L_i below 0, a page
 *             id outside the pool; ENOSPC: more pages than columns, more rows than n_rows
 * Errors: EINVAL (null, sizes, alignment), ENOSPC (B > max_batch, n_rows > max_tokens, columns > max_pages), EUNSUP (n_pages_in_pool >= 2^27), EHIP.
 */
int32_t synera_tree_plan(synera_tree* tree, int32_t B, const int32_t* d_ctx_len, const int32_t* d_n_nodes, const int32_t* d_parent,
                         int64_t n_rows, const int32_t* d_table, int32_t columns, int32_t n_pages_in_pool, int32_t* d_status, void* stream);

/*
 * The same behind synera_pages_update: of each row of the table only the first d_held[i] columns are the request's own (i32 [B], NULL: all).  A request that
 * synera_pages_update refused, whose row ends in entries that are no pages or by now another request's, is refused here too:
 * ENOSPC where its tokens and nodes need more than d_held[i] pages, EINVAL where that is outside 0 .. columns.  A plan without d_held takes
 * all entries that a request's lengths reach for its own.
 */
int32_t synera_tree_plan_held(synera_tree* tree, int32_t B, const int32_t* d_ctx_len, const int32_t* d_n_nodes, const int32_t* d_parent,
                              int64_t n_rows, const int32_t* d_table, int32_t columns, const int32_t* d_held, int32_t n_pages_in_pool,
                              int32_t* d_status, void* stream);

/* As synera_append_rope, each node at its places in text and cache.  Tensors have room for the plan's n_rows tokens. */
int32_t synera_tree_append_rope(synera_tree* tree, const synera_rope* rope, int32_t dtype, const synera_heads* q,
                                const synera_heads* k, const synera_heads* v, float eps, void* d_k_layer, void* d_v_layer, void* stream);

/* As synera_shared_attention, over the keys that each node sees.  Calls with one handle must be ordered (they share its scratch). */
int32_t synera_tree_attention(synera_tree* tree, const synera_heads* q, const void* d_k_layer, const void* d_v_layer, float scale,
                              float* d_lse, void* stream);

/*
 * The path of each planned tree that the targets follow.  d_target i32 [rows]: the token that the model puts after each node (its
 * argmax, or a sample).  The first d_n_given[i] nodes (clamped to 0 .. n_i; NULL: none) are accepted as they are and taken for a chain; what
 * follows them, or the context where there are none, is the target of the last one, or d_anchor[i].  From there the path goes to the
 * first child whose token (d_tokens i32 [rows]) is the target, and on with that child's target.
 *   d_accept_len i32 [B]     nodes on the path behind the given ones
 *   d_token      i32 [B]     the target at the path's end, which no child has; -1: none (no nodes, no given ones and no anchor, or refused)
 *   d_path       i32 [rows]  row cu_i + k: the k-th node of the path, the given ones first; -1 behind its end
 *   d_n_path     i32 [B]     nodes on the path, the given ones included
 * Outputs must not lie on inputs.  Errors: EINVAL (null, no plan, n_rows below the plan's, neither d_anchor nor d_n_given), EHIP.
 */
int32_t synera_tree_accept(synera_tree* tree, int64_t n_rows, const int32_t* d_tokens, const int32_t* d_target, const int32_t* d_anchor,
                           const int32_t* d_n_given, int32_t* d_accept_len, int32_t* d_token, int32_t* d_path, int32_t* d_n_path, void* stream);

/*
 * Moves the keys and values of each path together, position L_i + k <- L_i + path[k], in n_layers layers that lie layer_stride elements
 * apart in both pools.  d_path [rows] and d_n_path [B] as synera_tree_accept leaves them; nodes that are not k .. n_i - 1 stay where they are, and
 * so do all positions behind the path.  L_i += n_path[i] makes the path part of the context.
 * Errors: EINVAL (null, no plan, n_rows below the plan's, n_layers < 1, a stride below a layer's pages, pools off 16 bytes), EHIP.
 */
int32_t synera_tree_commit(synera_tree* tree, int64_t n_rows, const int32_t* d_path, const int32_t* d_n_path, int32_t n_layers,
                           int64_t layer_stride, void* d_k_pool, void* d_v_pool, void* stream);

/* ------------------------------------------------------------------------------------------- logits
 * For row r of request i and token t with logit x, in this order and in 32 bits:
 *   seen: t is among the first history_len[i] tokens of d_history[i] or on the row's path; g: how often it is there from n_prompt[i] on
 *   x = x / repetition (x > 0; times its reciprocal, rounded) or x * repetition     where t was seen
 *   x -= frequency x g + presence                    where g > 0
 *   x += bias                                        of the last entry of d_bias_id[i] that names t
 *   x = -infinity                                    where bit t % 32 of word t / 32 of d_mask[r] is not set, whatever x was
 * and rounded once to the type of the output.  A mask may leave nothing.
 */
typedef struct synera_logits_desc {
  int32_t B;                   /* requests, at most 65535                                                               */
  int32_t dtype;               /* of logits, in and out: 0, 1 or 2                                                      */
  int64_t rows, vocab;         /* vocab <= 2^30                                                                         */
  int64_t in_stride, out_stride;   /* elements from row to row, >= vocab where there are several                        */
  const int32_t* d_cu;         /* [B + 1] row cu[i] is the first of request i (clamped to 0 .. rows; a row of two requests, where it falls, may come out as either's); NULL: row i is request i's, rows == B */
  const int32_t* d_history;    /* [B][history_columns], or NULL: none.  Tokens outside the vocabulary do not count        */
  const int32_t* d_history_len;    /* [B] clamped to 0 .. history_columns; NULL with d_history                            */
  const int32_t* d_n_prompt;   /* [B] or NULL: 0                                                                        */
  int32_t history_columns;     /* below 2^19                                                                            */
  int32_t bias_columns;        /* <= 1022                                                                               */
  const float* d_repetition;   /* [B], above 0, or NULL: 1                                                              */
  const float* d_presence;     /* [B] or NULL: 0                                                                        */
  const float* d_frequency;    /* [B] or NULL: 0                                                                        */
  const int32_t* d_bias_id;    /* [B][bias_columns] or NULL: none.  Ids outside the vocabulary name nothing               */
  const float* d_bias;         /* [B][bias_columns]                                                                     */
  const int32_t* d_mask;       /* [rows][(vocab + 31) / 32] bits of tokens that are allowed, or NULL: all                 */
  const int32_t* d_tokens;     /* [rows], at most 2^19, or NULL: no paths.  With d_cu: row j of a request stands behind node j of its tree, */
  const int32_t* d_parent;     /* [rows]  whose path, itself included, was seen and counts for g, beside the history, which has to end before the first node.  A parent outside 0 .. j - 1 ends the path */
} synera_logits_desc;

/*
 * d_out == d_in with the same stride works in place (then only what changes is written); any other overlap is refused, also with
 * the desc's arrays.  rows == 0 is a no-op.  Errors: EINVAL (null, sizes, strides, alignment, overlaps, d_tokens without d_cu), EUNSUP (beyond the limits above), EHIP.
 */
int32_t synera_logits_adjust(const synera_logits_desc* desc, const void* d_in, void* d_out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SYNERA_TREE_H */
