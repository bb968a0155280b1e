/*
 * fluxbin_quant.h - operators of quantized LLM decoding next to the binary linears of fluxbin.h, on AMD Instinct MI355X
 * (gfx950). Same conventions: fp16 values are binary16 bit patterns passed as uint16_t, device pointers are memory of the
 * current device, the caller owns every buffer, arguments are checked on the host before any launch, work is enqueued on
 * the given stream, and the same inputs on the same device give bitwise identical outputs (no float atomics). No call
 * here synchronizes, allocates or keeps state, so all of them can be captured into a graph.
 */
#ifndef FLUXBIN_QUANT_H_
#define FLUXBIN_QUANT_H_

#include "fluxbin.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Linears in 4 bits with group scales, for the layers of a model that are not stored in binary bases (an output head,
 * the first and last blocks, a router).
 *
 *   W-hat[i, n] = (q[i, n] - z[i, n / g]) * s[i, n / g],   q in 0..15, s fp16, z in 0..15 (8 everywhere without zeros)
 *
 *   M  rows, 1..2^24.   N  columns, 1..2^20, M * N <= 2^34.
 *   g  group of columns with one scale (and zero point) per row: 32, 64, a multiple of 128, or g >= N (one per row). The
 *      last group may be shorter. G = ceil(N/g) groups per row.
 *   has_zeros  1: zero points per row and group; 0: symmetric, z = 8.
 */
typedef struct {
  int64_t M, N, g;
  int32_t has_zeros;
  int32_t reserved0;
} fluxbin_w4_shape;

/* A packed layer: a POD descriptor of a caller-owned device buffer written by fluxbin_w4_pack. */
typedef struct {
  fluxbin_w4_shape shape;
  void* d_base;
  uint64_t bytes;
  uint32_t format_version;
  uint32_t reserved1;
} fluxbin_w4_layer;
#define FLUXBIN_W4_FORMAT_VERSION 1u

/*
 * Round-to-nearest quantization of W (fp16, or fp32 with w_is_fp32) into the canonical form that fluxbin_w4_pack takes.
 * Over each group, with lo = min(0, W), hi = max(0, W):
 *   zeros:     s = fp16((hi - lo) * (1/15)), z = clamp(rne(-lo * (1/s)), 0, 15), q = clamp(rne(w * (1/s)) + z, 0, 15);
 *   symmetric: s = fp16(max(hi, -lo) * (1/7)), q = clamp(rne(w * (1/s)), -8, 7) + 8;
 * in fp32, rne to nearest even, 1/s = 0 where s is 0. NaN counts as 0, values past fp16's range as its largest.
 *   d_W       device [M] rows of N elements, row stride ldw >= N elements.
 *   d_codes   uint32 [M][ceil(N/8)]: column 8 w + t in bits 4t..4t+3 of word w (bits past column N-1 zero).
 *   d_scales  fp16 [M][G].   d_zeros  uint8 [M][G] with has_zeros, else NULL.
 *   d_values  NULL, or fp16 [M] rows of stride ldv >= N: (q - z) s, rounded to nearest even (largest fp16 past its range).
 * No output may overlap W or another output. Asynchronous on `stream`.
 */
fluxbin_status fluxbin_w4_quantize(const fluxbin_w4_shape* shape, const void* d_W, int32_t w_is_fp32, int64_t ldw,
                                   uint32_t* d_codes, uint16_t* d_scales, uint8_t* d_zeros, uint16_t* d_values,
                                   int64_t ldv, hipStream_t stream);

/*
 * Packed form: codes [ceil(M/16)][ceil(N/128)][64][16] bytes, then scale quads and zero-point quads (each section at a
 * multiple of 256 bytes; the layout is private to the library's version). d_codes, d_scales and d_zeros: device, as
 * fluxbin_w4_quantize writes them (zero points above 15 keep their low 4 bits). Asynchronous on `stream`.
 */
fluxbin_status fluxbin_w4_pack_query(const fluxbin_w4_shape* shape, size_t* packed_bytes);
fluxbin_status fluxbin_w4_pack(const fluxbin_w4_shape* shape, const uint32_t* d_codes, const uint16_t* d_scales,
                               const uint8_t* d_zeros, void* d_packed, size_t packed_bytes, fluxbin_w4_layer* out,
                               hipStream_t stream);

/*
 * Y[b, :] = W-hat X[b, :] for b < B (1..8192). d_x fp16 with row stride ldx >= N, any alignment of an element; d_y fp16 or
 * fp32 with row stride ldy >= M; strides in elements, for B = 1 not used. (q - z) x is summed in fp32 from exact products
 * and multiplied by the scale once per group of at most 128 columns.
 * Workspace: partial sums where the columns are split over workgroups; every call writes what it reads, nothing needs
 * clearing, and the workspace queried for B serves every smaller batch and any layer whose query is no larger. It may be
 * NULL where the query says 0. Calls that share it must not overlap in time. Memory that a call writes may not overlap
 * memory that it reads, from first to last element.
 */
fluxbin_status fluxbin_w4_workspace_query(const fluxbin_w4_layer* layer, int32_t B, size_t* bytes);
fluxbin_status fluxbin_w4_gemm(const fluxbin_w4_layer* layer, int32_t B, const uint16_t* d_x, int64_t ldx, void* d_y,
                               int64_t ldy, int32_t y_is_fp32, void* d_workspace, size_t workspace_bytes,
                               hipStream_t stream);

/*
 * Paged key/value cache in 8 bits, with one scale for each page (block of tokens) and head, and the attention that reads
 * it. The value of a cached element is code * scale, code in -127..127, scale fp32.
 *
 *   pages      pages of the pool, 1..2^24 (pages * page_size * kv_heads * head_dim <= 2^40).
 *   page_size  tokens of a page: 16, 32, 64, 128 or 256.
 *   kv_heads   1..1024.   head_dim  64, 128 or 256.
 *   d_base     device buffer of fluxbin_kv8_cache_query bytes, 256-byte aligned. It needs no initialization: a page's
 *              contents are defined by what is appended to it. The layout is private to the library's version.
 */
typedef struct {
  int64_t pages;
  int32_t page_size, kv_heads, head_dim;
  uint32_t format_version;
  void* d_base;
  uint64_t bytes;
} fluxbin_kv8_cache;
#define FLUXBIN_KV8_FORMAT_VERSION 1u
fluxbin_status fluxbin_kv8_cache_query(int64_t pages, int32_t page_size, int32_t kv_heads, int32_t head_dim,
                                       size_t* bytes);

/*
 * The sequences of a call. All arrays are device memory, read by the kernels (so that a captured call serves changing
 * lengths). Ranges of memory that a call writes may not overlap those it reads, from first to last element.
 *   rows         rows (tokens) of the call's packed tensors, 0..2^22.    sequences  1..65535.
 *   d_offsets    int32 [sequences + 1]: sequence b has rows d_offsets[b] .. d_offsets[b+1] - 1, n_b of them. Rows that
 *                belong to no sequence are neither read nor written; a sequence whose range is not inside [0, rows) is
 *                left out. Offsets do not fall from one sequence to the next: where they do, what the rows and pages of
 *                the call get is not defined (nothing else is affected).
 *   d_context    int32 [sequences]: tokens of each sequence with the call's own among them (taken into 0..2^30): row i of
 *                a sequence is at position d_context[b] - n_b + i. What is read at a position that was never stored is not
 *                defined.
 *   d_block_table  int32 [sequences][max_blocks], row stride block_table_stride >= max_blocks: the page of positions
 *                p * page_size .. (p + 1) * page_size - 1 is entry p. A position with no entry (negative, or past the table),
 *                or whose entry is not a page of the pool, is not stored, reads as zero, and is not attended.
 * Arrays need their elements' alignment.
 */
typedef struct {
  int64_t rows;
  int32_t sequences, max_blocks;
  int64_t block_table_stride;
  const int32_t* d_offsets;
  const int32_t* d_context;
  const int32_t* d_block_table;
} fluxbin_kv8_batch;

/*
 * Stores the keys and values of the batch's rows. d_k, d_v: fp16, element (row, head, d) at row * token_stride +
 * head * head_stride + d (strides in elements, >= 0; head_stride at least head_dim if there are several heads; rows may
 * be slices of a fused projection's rows). For each page and head that gets tokens, keys and values each:
 *   s = max(s_old if the page holds earlier tokens (its first new position is not its first position), max|new| * (1/127))
 *   code = rne(v * (1/s)) of a new value, rne(code * (s_old / s)) of an earlier token's where s > s_old
 * in fp32, 1/s = 0 where s is 0. NaN is stored as 0, infinities as the largest fp16. Positions behind the new ones in
 * their page lose what they held. A page belongs to one entry of one sequence's table: what a page holds after a call
 * that stores to it through two entries is not defined (nothing else is affected).
 */
fluxbin_status fluxbin_kv8_append(const fluxbin_kv8_cache* cache, const fluxbin_kv8_batch* batch, const uint16_t* d_k,
                                  int64_t k_token_stride, int64_t k_head_stride, const uint16_t* d_v,
                                  int64_t v_token_stride, int64_t v_head_stride, hipStream_t stream);

/* The values of the batch's rows from the cache, fp16 [rows][kv_heads][head_dim] each, rounded to nearest even. */
fluxbin_status fluxbin_kv8_read(const fluxbin_kv8_cache* cache, const fluxbin_kv8_batch* batch, uint16_t* d_k,
                                uint16_t* d_v, hipStream_t stream);

/*
 * Attention of the batch's rows over their sequences' cached tokens:
 *   out[row, h] = sum_j softmax_j(softmax_scale * q[row, h] . k[j, h / (q_heads / kv_heads)]) v[j, ...]
 * over positions j < d_context[b]; with causal (1) only those up to the row's own position; with window > 0 only those
 * after the row's position - window. A row without any position is 0.
 *   d_q, d_out  fp16, element (row, head, d) at row * token_stride + head * head_stride + d, any element alignment.
 *   q_heads     a multiple of kv_heads, up to 1024.
 * Scores, softmax sums and results are held in fp32; products are of fp16 operands: codes, which are exact in fp16 (their
 * scales stay apart), and softmax weights times their page's value scale, as the sum of two fp16 numbers: such a product is
 * off by at most 2^-21 of itself and 2^-33 of the row's largest one (an element in which the tokens of the largest products
 * have code 0 is as far off as that leaves it). A row's result may differ in its last bits between a call that has it among
 * many rows and one that does not.
 * Workspace: partial results of sequences that are split over workgroups; nothing needs clearing; of the size queried
 * with the largest rows and sequences it serves all smaller calls. Calls that share it must not overlap in time.
 */
fluxbin_status fluxbin_kv8_workspace_query(const fluxbin_kv8_cache* cache, int64_t rows, int32_t sequences,
                                           int32_t q_heads, size_t* bytes);
fluxbin_status fluxbin_kv8_attention(const fluxbin_kv8_cache* cache, const fluxbin_kv8_batch* batch, int32_t q_heads,
                                     const uint16_t* d_q, int64_t q_token_stride, int64_t q_head_stride, uint16_t* d_out,
                                     int64_t out_token_stride, int64_t out_head_stride, float softmax_scale,
                                     int32_t causal, int32_t window, void* d_workspace, size_t workspace_bytes,
                                     hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FLUXBIN_QUANT_H_ */
