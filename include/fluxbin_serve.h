/*
 * fluxbin_serve.h - operators around the paged 8-bit key/value cache of fluxbin_quant.h, on AMD Instinct MI355X (gfx950):
 * norms and rotation of queries and keys, trees of drafted tokens, and the pages that sequences hold. Same conventions: fp16
 * values are binary16 bit patterns passed as uint16_t, device pointers are memory of the current device, the caller owns
 * every buffer, arguments are checked on the host before any launch, work is enqueued on the given stream, and the same
 * inputs give bitwise identical outputs. No call here synchronizes, allocates or keeps state on the host, and lengths,
 * tables and trees are read on the device, so all of them can be captured into a graph that serves changing sequences.
 * Memory that a call writes may not overlap memory that it reads or another output, from first to last element, unless
 * stated otherwise.
 */
#ifndef FLUXBIN_SERVE_H_
#define FLUXBIN_SERVE_H_

#include "fluxbin_quant.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Norm of each head and rotation by position, of queries and keys in one pass over them.
 *   y = x * (sum(x^2) / head_dim + eps)^(-1/2) * weight   (only where a weight is given)
 *   then the pair (a, b) of elements i, i < rotary_dim / 2, becomes (a c - b s, a s + b c) with c and s the cosine and sine of
 *   position * frequency[i], both times magnitude; elements from rotary_dim on are not rotated.
 * Held in fp32 and rounded to fp16 once; the angle is formed and reduced in fp64, so that far positions lose nothing.
 *
 *   head_dim       64, 128 or 256.   rotary_dim  a multiple of 16, 0 (norms only) to head_dim.
 *   interleaved    0: a pair is (i, i + rotary_dim / 2), 1: (2 i, 2 i + 1).
 *   eps            >= 0.   magnitude  a finite number.
 *   d_frequencies  fp32 [rotary_dim / 2], radians per position (NULL if rotary_dim is 0).
 *   d_q_weight, d_k_weight  fp32 [head_dim], or NULL: that side is not normalized.
 */
typedef struct {
  int32_t head_dim, rotary_dim, interleaved, reserved0;
  float eps, magnitude;
  const float* d_frequencies;
  const float* d_q_weight;
  const float* d_k_weight;
} fluxbin_rotary;

/*
 *   rows         0..2^22, rows * (q_heads + k_heads) * head_dim <= 2^35.   d_positions  int32 [rows].
 *   q_heads      1..1024.   k_heads  0..1024 (0: queries only, the keys' arguments are not used).
 *   d_q, d_q_out, d_k, d_k_out  fp16, element (row, head, d) at row * token_stride + head * head_stride + d (strides in
 *                elements, any element alignment). An output may be its own input, at the same strides, and rows may be
 *                slices of the rows of one buffer (a fused projection's), queries and keys side by side.
 */
fluxbin_status fluxbin_qk_rotate(const fluxbin_rotary* rotary, int64_t rows, const int32_t* d_positions, int32_t q_heads,
                                 const uint16_t* d_q, int64_t q_token_stride, int64_t q_head_stride, uint16_t* d_q_out,
                                 int64_t q_out_token_stride, int64_t q_out_head_stride, int32_t k_heads,
                                 const uint16_t* d_k, int64_t k_token_stride, int64_t k_head_stride, uint16_t* d_k_out,
                                 int64_t k_out_token_stride, int64_t k_out_head_stride, hipStream_t stream);

/*
 * Trees of drafted tokens. The rows of a sequence (rows, sequences, d_offsets and d_context as in fluxbin_kv8_batch) are the
 * nodes of its tree, each behind its parent; their keys and values are stored as any rows are. What a row attends is a mask of
 * its sequence's rows: bit j % 64 of word j / 64 of uint64 [rows][words] stands for row j. words: 1..16 (trees of up to 1024
 * nodes); a sequence of more than 64 * words rows is left out, as one whose range is not inside [0, rows).
 */

/*
 * Masks and positions from parents: d_parents int32 [rows], the index among its sequence's rows of a node's parent, or negative:
 * the node follows the last cached token (so do nodes whose parent is not before them). A node's mask has its own bit and its
 * ancestors'; its position (d_positions int32 [rows], or NULL) is d_context - n + its number of ancestors. Once a step: the
 * masks serve the attention of every layer, the positions its rotation.
 */
fluxbin_status fluxbin_tree_masks(int64_t rows, int32_t sequences, const int32_t* d_offsets, const int32_t* d_context,
                                  const int32_t* d_parents, int32_t words, uint64_t* d_masks, int32_t* d_positions,
                                  hipStream_t stream);

/*
 * fluxbin_kv8_attention with a mask for the newest tokens: a row of a sequence of n rows attends the positions before the
 * sequence's first row (j < d_context - n) and, of its n rows, those whose bit is set in the row's mask, at any place in the
 * order. With window > 0 it attends only the last `window` of these (bits at negative positions do not count, positions
 * without a page do). Masks that fluxbin_tree_masks makes of a chain are the causal mask. A row that attends nothing is 0.
 * Precision, strides and argument checks as fluxbin_kv8_attention's; the workspace is this call's own size, whose bytes go by
 * the cache's head_dim and the device alone. How work is split goes by max_blocks, since lengths are read on the device: for contexts
 * of up to 900 tokens or so, a table no wider than they need (a view of its first columns) takes down to half of the time.
 */
fluxbin_status fluxbin_kv8_tree_workspace_query(const fluxbin_kv8_cache* cache, int64_t rows, int32_t sequences,
                                                int32_t q_heads, size_t* bytes);
fluxbin_status fluxbin_kv8_tree_attention(const fluxbin_kv8_cache* cache, const fluxbin_kv8_batch* batch, int32_t q_heads,
                                          const uint16_t* d_q, int64_t q_token_stride, int64_t q_head_stride,
                                          uint16_t* d_out, int64_t out_token_stride, int64_t out_head_stride,
                                          float softmax_scale, const uint64_t* d_masks, int32_t words, int32_t window,
                                          void* d_workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Moves accepted rows together. batch is that of the append that stored the rows; of sequence b's n rows the first
 * m = d_kept[b] (int32 [sequences], taken into 0..n) entries of d_keep (int32 [rows], from the sequence's offset on) name, in
 * rising order, the rows to keep: afterwards the k-th of them is at position d_context[b] - n + k, and d_context[b] - n + m is
 * the sequence's new length, for the caller to store (once, after every layer's call). Positions behind it are not defined.
 * Where a sequence's entries do not rise or are not in 0..n-1, what its positions from d_context - n on hold is not defined.
 * For each page and head that gets moved rows, keys and values each:
 *   s = the largest scale of the pages that they were in and, if the page holds earlier tokens, its own
 *   code = rne(code * (s_old / s)) of every row that stays or comes whose page had s_old < s
 * in fp32: rows moved inside a page, or between pages of one scale, keep their codes. A row that is already in its place,
 * behind none that moves, is not touched. Sources without a page count as zero, targets without one are not stored.
 */
fluxbin_status fluxbin_kv8_keep(const fluxbin_kv8_cache* cache, const fluxbin_kv8_batch* batch, const int32_t* d_keep,
                                const int32_t* d_kept, hipStream_t stream);

/*
 * Pages: who holds which. A pool counts the references of its pages; a page without any is free. The pages of a block table's
 * row are its first entries: behind the first entry that is no page there is none (a new table is filled with -1); a row for
 * which that does not hold gets or gives back some of its pages only. The pool serves the tables of all layers' caches (whose
 * pages are numbered alike).
 *   pages, page_size  as the caches'.
 *   d_state   int32 [pages + 4], 16-byte aligned, zero-filled at first: [0] a page below which none is free (0 is always
 *             valid), [1] pages that the last call wanted and did not find (2^31 - 1 if there were more), [2], [3] the
 *             library's, [4 + p] the references of page p. A caller may raise references of its own, and lower them (a page
 *             that gets 0 by that needs [0] = 0).
 * Calls that share a pool must not overlap in time. Free pages are taken lowest number first, in the order of the sequences.
 *
 * fluxbin_kv8_append and fluxbin_kv8_keep write the pages of the positions that they store, all of their tokens where the
 * scale grows, and look at no counts: a page with more than one reference that a row writes changes for every row that holds
 * it. Rows that are forked at their length and grow from there write no such page. A row that is resized into a page with other
 * references (or a batch whose rows to keep begin in one) would: fork it at the shorter length instead, and release the old row.
 */
typedef struct {
  int64_t pages;
  int32_t page_size, reserved0;
  int32_t* d_state;
} fluxbin_page_pool;

/*
 * Gives every row of a block table the pages of its first d_tokens[b] tokens (int32 [sequences]; a row with a negative number
 * stays as it is): entries past the last are released (-1), then missing ones taken, as far as the table has columns and the
 * pool has free pages. A last page that the tokens fill partly stays the row's, also where other rows hold it (see above for
 * what then may not be stored there). d_block_table is read and written, int32 [sequences][max_blocks], row stride
 * block_table_stride.
 */
fluxbin_status fluxbin_pages_resize(const fluxbin_page_pool* pool, int32_t sequences, int32_t max_blocks,
                                    int32_t* d_block_table, int64_t block_table_stride, const int32_t* d_tokens,
                                    hipStream_t stream);

/*
 * Forks sequences: row c of d_child_table (int32 [children][child_blocks]) becomes that of a sequence with the same tokens as
 * sequence d_source[c] (int32 [children]) of the table (lengths in d_context, int32 [sequences]). Pages that the tokens fill
 * are shared and get a reference; a last page that they fill partly is taken from the pool, and d_copies[c] (int32
 * [children][2]) is (old page, new page) for fluxbin_kv8_copy_pages, of every layer's cache, otherwise (-1, -1). The rest of
 * the row becomes -1, with the partly filled page where the pool had none: such a row lacks its last tokens. The child
 * table's old entries are overwritten, not released (resize them to 0 first). A source outside [0, sequences) gives an empty
 * row; tokens past child_blocks are cut off.
 */
fluxbin_status fluxbin_pages_fork(const fluxbin_page_pool* pool, int32_t sequences, int32_t max_blocks,
                                  const int32_t* d_block_table, int64_t block_table_stride, const int32_t* d_context,
                                  int32_t children, int32_t child_blocks, int32_t* d_child_table,
                                  int64_t child_table_stride, const int32_t* d_source, int32_t* d_copies,
                                  hipStream_t stream);

/*
 * Copies pages with their scales, from d_copies[i][0] of `from` to d_copies[i][1] of `to` (int32 [copies][2], copies
 * 0..2^22). The caches have the same page_size, kv_heads and head_dim; they may be one. Pairs with a number that is not a
 * page of its cache are left out. What a page holds that is written twice, or written and read, by one call is not defined.
 */
fluxbin_status fluxbin_kv8_copy_pages(const fluxbin_kv8_cache* to, const fluxbin_kv8_cache* from, int64_t copies,
                                      const int32_t* d_copies, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FLUXBIN_SERVE_H_ */
