/*
 * cp_tree.h — C ABI of speculative decoding and forked requests over the
 * paged K/V cache of cp_attn.h, for AMD Instinct MI355X (gfx950).
 *
 * A decode row of cp_attn.h yields one token per iteration.  With a draft, a
 * request instead submits a tree of guessed tokens in one iteration and keeps
 * the branch that the model agrees with:
 *
 *   cp_tree_layout   parents -> masks and rotary positions of the nodes
 *   cp_kv_append     (cp_attn.h) node j's K/V into slot chunk_start + j
 *   cp_tree_attn     every node attends to the committed keys and its ancestors
 *   cp_tree_verify   the logits' argmax of every node, and the accepted path
 *   cp_kv_compact    the accepted nodes' K/V to slots chunk_start + 0, 1, ...
 *   cp_kv_fork       a request continued by several: shared full pages and a
 *                    copy of the partly filled one
 *
 * A drafted row is a cp_row_meta: chunk_start keys are committed, and
 * chunk_len nodes, at most CP_TREE_MAX_NODES, follow in slots chunk_start ..
 * ctx_len - 1, packed in row order like the tokens of cp_attn.h.  Node 0 is
 * the root (the last token known, whose K/V is not cached yet), and a node's
 * parent comes before it.  A decode row is a tree of one node.
 *
 * Layouts, ownership, asynchrony and error codes are those of cp_attn.h: dense
 * row-major bf16 tensors, caller-owned device memory, everything enqueued on
 * `stream` of the current device, all validation before anything is enqueued,
 * nothing enqueued by a call that fails.  These calls only launch kernels (no
 * copy, allocation or wait, unless CP_DEBUG is 1), so they can be captured in
 * a HIP graph; the rows and forks, read during the call, are captured with
 * them.  A workspace must not be used by two calls in flight at once, those
 * of graph replays among them.  With CP_DEBUG=1 the entries of the block table
 * that a call reads are checked first, as in cp_attn.h.
 */
#ifndef CP_TREE_H
#define CP_TREE_H

#include <stddef.h>
#include <stdint.h>

#include "cp_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CP_TREE_MAX_NODES 256

/* Keys (chunk_start + chunk_len) that a row of cp_tree_attn may have: more do
 * not fit the memory with pages of their own, and the bound keeps key indexes
 * in 32 bits when they are rounded up to pieces. */
#define CP_TREE_MAX_KEYS (1 << 30)

/* Masks and positions of drafted trees.  parents[t] is the index inside its
 * row of node t's parent; anything but an index before the node's own (-1, by
 * convention, for the root) ends the chain of ancestors.  With W = mask_words
 * (1 to 4) 64-bit words per node, bit j % 64 of mask[t * W + j / 64] is set
 * where node j of t's row is t or an ancestor of t, and
 * positions[t] = chunk_start + number of t's ancestors.
 * A row has at most min(64 * W, CP_TREE_MAX_NODES) nodes; req_id is not used.
 * mask is 8-byte aligned. */
int cp_tree_layout(const int32_t *parents, const cp_row_meta *rows, int32_t n_rows,
                   uint64_t *mask, int32_t mask_words, int32_t *positions, void *stream);

/* Workspace bytes cp_tree_attn needs for this batch, or 0 if desc/rows are
 * invalid or a row has more than CP_TREE_MAX_NODES nodes or CP_TREE_MAX_KEYS
 * keys. */
size_t cp_tree_attn_workspace_bytes(const cp_attn_desc *desc, const cp_row_meta *rows,
                                    int32_t n_rows);

/* Attention of every drafted node: with c = chunk_start and n = chunk_len of
 * node t's row,
 *     out[t][h] = sum_{i in S} softmax_{i in S}(sm_scale * q[t][h] . K_i) V_i,
 *     S = {0 .. c - 1} and those c + j, j < n, whose bit j of mask[t] is set.
 * Any mask goes (bits from n on are ignored); a node that sees no key gets
 * zeros.  What a node does not see does not touch its output, infinities and
 * NaN there included.  fp32 softmax and accumulation, the softmax weights
 * rounded to bf16 for the product with V and summed as rounded.  q, out
 * [T][Hq][D], mask [T][mask_words] (8-byte aligned), ws 256-byte aligned; out
 * must not overlap q.  Checks as for cp_attn_mixed; more nodes than
 * min(64 * mask_words, CP_TREE_MAX_NODES) in a row is CP_ERR_BAD_META, more
 * keys than CP_TREE_MAX_KEYS CP_ERR_UNSUPPORTED.
 * Long key ranges are split and merged by a log-sum-exp pass; the result of a
 * batch does not depend on anything but its inputs. */
int cp_tree_attn(const cp_attn_desc *desc, const void *q, const void *k_cache,
                 const void *v_cache, const int32_t *block_tables, const uint64_t *mask,
                 int32_t mask_words, const cp_row_meta *rows, int32_t n_rows, void *out, void *ws,
                 size_t ws_bytes, void *stream);

/* Workspace bytes cp_tree_verify needs for up to n_tokens nodes in all (one
 * that serves a batch serves every smaller one), or 0 if a size is out of range
 * (n_tokens < 0, vocab < 1). */
size_t cp_tree_verify_workspace_bytes(int64_t n_tokens, int32_t vocab);

/* Greedy verification.  logits: bf16 [T], rows of vocab values at a stride of
 * ld >= vocab elements.  target[t] = the index of the largest logit of node t,
 * the lowest one where several are; -0 and +0 are equal, and NaN counts as
 * larger than any number (as in torch.argmax).  Then, in every row, from the
 * current node k = 0: the next node is the lowest child j of k (parents as in
 * cp_tree_layout) whose tokens[j] is target[k], until there is none or the
 * path has max_path nodes.  Written per row r: path[r * max_path + i], the
 * path's nodes (0 first) and -1 behind them; n_accepted[r], their number;
 * next_token[r], the last one's target.  A row without nodes gets 0 accepted
 * and the next token -1.  req_id and chunk_start are not used; tokens and
 * parents are packed [T]; max_path is 1 to CP_TREE_MAX_NODES; ws is 256-byte
 * aligned. */
int cp_tree_verify(const void *logits, int64_t ld, int32_t vocab, const int32_t *tokens,
                   const int32_t *parents, const cp_row_meta *rows, int32_t n_rows,
                   int32_t max_path, int32_t *target, int32_t *path, int32_t *n_accepted,
                   int32_t *next_token, void *ws, size_t ws_bytes, void *stream);

/* Keeps the accepted nodes: for every row r and i < n_accepted[r], the K and V
 * of slot chunk_start + path[r * max_path + i] move to slot chunk_start + i of
 * the same request, for every kv head of every layer's pools, as if all were
 * read before the first is written.  k_caches and v_caches: host arrays of
 * n_layers device pointers.  path and n_accepted live on the device: entries
 * count while they rise strictly and name nodes of the row (0 <= entry <
 * chunk_len), the first one that does not ends the row's path; an
 * n_accepted[r] outside [0, max_path] is taken as the nearer bound.  Every
 * other slot is left as it was; a move whose table entry lies outside
 * [0, num_blocks) is left out.  No two rows may share a page that is written
 * to, nor two layers a pool, and no other call in flight writes to such a page:
 * those of V are read and written whole. */
int cp_kv_compact(const cp_attn_desc *desc, void *const *k_caches, void *const *v_caches,
                  int32_t n_layers, const int32_t *block_tables, const cp_row_meta *rows,
                  int32_t n_rows, const int32_t *path, int32_t max_path,
                  const int32_t *n_accepted, void *stream);

/* A request that continues another's first ctx_len tokens. */
typedef struct {
    int32_t src_req; /* block-table row of the request that goes on          */
    int32_t dst_req; /* block-table row that is filled in                    */
    int32_t ctx_len; /* tokens the two have in common                        */
    int32_t block;   /* a free physical block for the partly filled page (not
                      * used when ctx_len is a multiple of block_size)       */
} cp_fork;

/* Forks requests: with f = ctx_len / block_size, entries [0, f) of table row
 * dst_req become those of src_req (the pages are shared from then on: none of
 * the two writes to a full page again), and where ctx_len is no multiple of
 * block_size entry f becomes `block`, to which page f of src_req is copied
 * whole, K and V, in every layer's pools.  Other entries and pages are left as
 * they were.  0 <= ctx_len <= max_blocks_per_req * block_size; rows in
 * [0, num_reqs_in_table); every dst_req is named once, and by no fork as its
 * src_req; every used block is in [0, num_blocks) and named once; else
 * CP_ERR_BAD_META.  A page whose source entry lies outside [0, num_blocks) is
 * not copied.  Which blocks are free is the caller's to know; a pool is named
 * once. */
int cp_kv_fork(const cp_attn_desc *desc, void *const *k_caches, void *const *v_caches,
               int32_t n_layers, int32_t *block_tables, const cp_fork *forks, int32_t n_forks,
               void *stream);

#ifdef __cplusplus
}
#endif

#endif /* CP_TREE_H */
