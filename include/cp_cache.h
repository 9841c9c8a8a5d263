/*
 * cp_cache.h — C ABI of the operators for long and shared contexts over the
 * paged K/V cache of cp_attn.h, for AMD Instinct MI355X (gfx950).
 *
 *   cp_qkv_append    the fused projection's q and k heads normalised and
 *                    rotated, K and V written straight into their pages
 *   cp_page_bounds   the smallest and largest value of every feature over the
 *                    keys of the pages that a batch wrote
 *   cp_page_select   the pages that each token reads, by these bounds
 *   cp_page_attn     attention over the selected pages
 *   cp_prefix_attn   attention of requests with a common prefix, which is read
 *                    once for all of them
 *
 * A decode iteration over long contexts runs append, bounds, select and
 * page_attn in place of cpl_qkv_rope, cp_kv_append and cp_attn_mixed; one over
 * requests that cp_kv_fork continued from one prompt runs append and
 * prefix_attn.
 *
 * Rows, layouts, ownership, asynchrony and error codes are those of cp_attn.h:
 * dense row-major bf16 tensors, 16-byte aligned, caller-owned device memory,
 * everything enqueued on `stream` of the current device, all validation before
 * anything is enqueued, nothing enqueued by a call that fails.  Token t of row r
 * is at position p = chunk_start + j.  These calls only launch kernels (no
 * copy, allocation or wait, unless CP_DEBUG is 1), so they can be captured in
 * a HIP graph; rows and groups, read during the call, are captured with them.
 * A workspace must not be used by two calls in flight at once, those of graph
 * replays among them.  With CP_DEBUG=1 the entries of the block table that a
 * call reads are checked first, as in cp_attn.h.
 *
 * Besides the limits of cp_attn.h: num_kv_heads <= 1024, at most 2^23 tokens and
 * 2^27 (token, q head) pairs in a batch, rows of at most CP_CACHE_MAX_KEYS keys;
 * else CP_ERR_UNSUPPORTED.
 */
#ifndef CP_CACHE_H
#define CP_CACHE_H

#include <stddef.h>
#include <stdint.h>

#include "cp_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CP_CACHE_MAX_KEYS (1 << 30) /* ctx_len of a row */
#define CP_CACHE_MAX_PAGES 4096     /* pages that a token selects */

/* cpl_qkv_rope and cp_kv_append in one: qkv[T][(Hq + 2 Hkv) * D] holds a
 * token's q heads, then its k heads, then its v heads.  Every q and k head is
 * RMS-normalised over D with q_norm_w[D] or k_norm_w[D] and rotated: elements
 * d and d + D/2 form a pair turned by the angle positions[t] * theta^(-2d/D),
 * d < D/2 (positions: int32, device, >= 0; NULL: every token's own position p).
 * The q heads go to q[T][Hq][D], the k and v heads to slot p of the request's
 * pages, whatever `positions` holds.  The same bits as the two calls; every
 * other slot is left untouched, and a slot whose table entry lies outside
 * [0, num_blocks) is not written.  q overlaps none of the inputs.  theta > 1,
 * eps > 0; sm_scale is not used. */
int cp_qkv_append(const cp_attn_desc *desc, const void *qkv, const void *q_norm_w,
                  const void *k_norm_w, const int32_t *positions, double theta, float eps,
                  void *q, void *k_cache, void *v_cache, const int32_t *block_tables,
                  const cp_row_meta *rows, int32_t n_rows, void *stream);

/* bounds[num_blocks][Hkv][2][D] (bf16): for every row, the pages that hold a
 * slot of chunk_start .. ctx_len - 1, and each of their kv heads,
 *     bounds[page][h][0][d] = min K[i][h][d],  bounds[page][h][1][d] = max K[i][h][d]
 * over the page's keys i < ctx_len, those before chunk_start among them.  Where
 * one of them is an infinity or NaN, the lowest and the largest finite value.
 * Other pages' entries are left as they were.  A page whose table entry lies
 * outside [0, num_blocks) is left out.  Behind cp_kv_compact the rows that the
 * trees had bring the moved keys into their new pages' bounds; behind
 * cp_kv_fork the copied page gets its bounds with the next append. */
int cp_page_bounds(const cp_attn_desc *desc, const void *k_cache, const int32_t *block_tables,
                   const cp_row_meta *rows, int32_t n_rows, void *bounds, void *stream);

/* Workspace bytes cp_page_select needs for this batch, or 0 if the arguments
 * are invalid.  They serve every batch that leaves out some of its rows or
 * tokens, too. */
size_t cp_page_select_workspace_bytes(const cp_attn_desc *desc, const cp_row_meta *rows,
                                      int32_t n_rows, int32_t n_pages);

/* The n_pages logical pages that every token reads, per kv head.  Of the pages
 * 0 .. p / B that hold keys of token t: the first `n_first` and the last
 * `n_last` ones, and of the others those with the largest score
 *     s(i) = max over the q heads e of kv head h of
 *            sum_d max(q[t][e][d] lo[i][d], q[t][e][d] hi[i][d]),
 * lo and hi the page's bounds: no key of the page has a larger product with q.
 * Scores are summed in fp64; equal ones go to the lower page.  (Where q or bounds
 * hold infinities or NaN, the list is one of that many pages all the same, the
 * fixed ones among them.)  pages[T][Hkv][n_pages] (int32) gets them in rising
 * order, and -1 behind them where there are fewer.
 * 1 <= n_pages <= CP_CACHE_MAX_PAGES, n_first, n_last >= 0, n_first + n_last <=
 * n_pages.  Bounds of a page whose table entry lies outside [0, num_blocks) are
 * taken as the lowest score.  bounds 16-byte, pages 4-byte, ws 256-byte
 * aligned; sm_scale is not used. */
int cp_page_select(const cp_attn_desc *desc, const void *q, const void *bounds,
                   const int32_t *block_tables, const cp_row_meta *rows, int32_t n_rows,
                   int32_t n_pages, int32_t n_first, int32_t n_last, int32_t *pages, void *ws,
                   size_t ws_bytes, void *stream);

/* Workspace bytes cp_page_attn needs for this batch, or 0 if the arguments are
 * invalid.  Few lists are cut into pieces and merged, many are not: a smaller
 * batch can need more.  max(256, (4 D + 4) Hq T ceil(n_pages B / 256)) bytes serve
 * every batch of up to T tokens. */
size_t cp_page_attn_workspace_bytes(const cp_attn_desc *desc, const cp_row_meta *rows,
                                    int32_t n_rows, int32_t n_pages);

/* Attention of every token over the keys i <= p of the logical pages that
 * pages[t][h][0 .. n_pages - 1] (int32, device) names for each kv head h:
 *     out[t][e] = sum_i softmax_i(sm_scale * q[t][e] . K_i) V_i.
 * A list's entries count while they rise strictly and lie in 0 .. p / B; the
 * first one that does not ends it.  A token without a page gets zeros.  Slots
 * behind p may hold anything.  fp32 softmax and accumulation, the weights
 * rounded to bf16 for the product with V and summed as rounded; long lists are
 * split and merged by a log-sum-exp pass.  out must not overlap q. */
int cp_page_attn(const cp_attn_desc *desc, const void *q, const void *k_cache,
                 const void *v_cache, const int32_t *block_tables, const int32_t *pages,
                 int32_t n_pages, const cp_row_meta *rows, int32_t n_rows, void *out, void *ws,
                 size_t ws_bytes, void *stream);

/* Rows that have their first tokens in common. */
typedef struct {
    int32_t first_row; /* rows first_row .. first_row + n_rows - 1 of the batch */
    int32_t n_rows;
    int32_t common;    /* tokens they have in common                          */
} cp_prefix_group;

/* Workspace bytes cp_prefix_attn needs for this batch, or 0 if the arguments
 * are invalid.  As for cp_page_attn, a smaller batch can need more.
 * max(256, (4 D + 4) Hq T (floor(N / 256) + 2)) bytes serve every batch of up to T
 * tokens whose contexts have up to N keys, if no row has more than one token;
 * 16 Hkv / Hq times as many every other one. */
size_t cp_prefix_attn_workspace_bytes(const cp_attn_desc *desc, const cp_row_meta *rows,
                                      int32_t n_rows, const cp_prefix_group *groups,
                                      int32_t n_groups);

/* Causal attention as in cp_attn_mixed, for decode rows and short chunks of
 * requests with a common prefix.  The first common / B entries of the table
 * rows of a group's requests are the same (as cp_kv_fork leaves them): those
 * pages are read once for the whole group, through its first row's table (where
 * few tokens have few keys, by each of them), and every row's other keys one by
 * one.  Groups come in rising order and do not
 * overlap; 0 <= common <= chunk_start of each of the group's rows that has
 * tokens; else CP_ERR_BAD_META.  A row in no group shares nothing.  Behind the
 * prefix a row's tokens are taken some at a time, 16 (token, q head) pairs of a
 * kv head at most, so long chunks belong to cp_attn_mixed.  Precision, ws and out as in cp_page_attn.  With CP_DEBUG=1
 * table rows of a group that differ where they should not are
 * CP_ERR_BAD_META. */
int cp_prefix_attn(const cp_attn_desc *desc, const void *q, const void *k_cache,
                   const void *v_cache, const int32_t *block_tables, const cp_row_meta *rows,
                   int32_t n_rows, const cp_prefix_group *groups, int32_t n_groups, void *out,
                   void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* CP_CACHE_H */
