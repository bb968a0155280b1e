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
 * Workspace: partial sums where the columns are split over workgroups, or the call's activations in operand order; every
 * call rewrites what it reads, nothing needs clearing, and the workspace queried for B serves every smaller batch and any
 * layer whose query is no larger. It may be NULL where the query says 0. Calls that share it must not overlap in time.
 */
fluxbin_status fluxbin_w4_workspace_query(const fluxbin_w4_layer* layer, int32_t B, size_t* bytes);
fluxbin_status fluxbin_w4_gemm(const fluxbin_w4_layer* layer, int32_t B, const uint16_t* d_x, int64_t ldx, void* d_y,
                               int64_t ldy, int32_t y_is_fp32, void* d_workspace, size_t workspace_bytes,
                               hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* FLUXBIN_QUANT_H_ */
