// Internal declarations of the operators next to the binary linears: 4-bit linears
// (fluxbin_w4_*) and the paged 8-bit key/value cache (fluxbin_kv8_*).
#pragma once

#include "fluxbin_internal.h"
#include "fluxbin_quant.h"

namespace fluxbin {

// ---- 4-bit linears ----
constexpr int kW4MaxBatch = kMaxBatchCall;   // batch rows of one call
// Row tiles of 16 rows, column chunks of kChunk columns, steps of 4 chunks. Scales (and zero points) come in quads per
// row: 4 chunks' at one per chunk (group >= 128), 2 chunks' at two, one chunk's at four.
struct W4Derived {
  int64_t g, G;        // columns of a group, at most N; groups per row, canonical
  int64_t Mt, Nc;      // row tiles, chunks
  int gc;              // scales per chunk and row: 1, 2 or 4
  int64_t Nq;          // quads per row
  uint64_t off_scales, off_zeros, total;
};

inline W4Derived w4_derive(const fluxbin_w4_shape& s) {
  W4Derived d{};
  d.g = s.g < s.N ? s.g : s.N;
  d.G = ceil_div(s.N, d.g);
  d.Mt = ceil_div(s.M, 16);
  d.Nc = ceil_div(s.N, kChunk);
  d.gc = s.g < kChunk && s.g < s.N ? int(kChunk / s.g) : 1;
  d.Nq = ceil_div(d.Nc * d.gc, 4);
  d.off_scales = round_up256(uint64_t(d.Mt) * uint64_t(d.Nc) * 1024u);
  d.off_zeros = d.off_scales + round_up256(uint64_t(d.Mt) * uint64_t(d.Nq) * 128u);
  d.total = d.off_zeros + (s.has_zeros ? round_up256(uint64_t(d.Mt) * uint64_t(d.Nq) * 64u) : 0u);
  return d;
}

struct W4Args {
  const uint8_t* codes;
  const uint8_t* scales;
  const uint8_t* zeros;   // NULL: every zero point is 8
  const uint16_t* x;
  void* y;
  float* partials;        // [parts][B][M]
  int64_t ldx, ldy;
  int32_t M, N, B, Mt, Nc, Nq, y_fp32, parts;
};

struct W4Plan {
  bool many;    // the kernel for many batch rows
  int nw;       // wavefronts of a workgroup
  int bt;       // 16-row batch tiles of a workgroup
  int rt;       // row tiles of a workgroup
  int parts;    // workgroups per row tile, each with a part of the columns
  uint64_t ws_bytes;
};

W4Plan w4_plan(const fluxbin_w4_shape& s, int B, int cus);
uint64_t w4_workspace(const fluxbin_w4_shape& s, int B, int cus);   // of calls of up to B rows
fluxbin_status launch_w4_gemm(const W4Args& a, const W4Plan& p, int gc, hipStream_t stream);
fluxbin_status launch_w4_pack(const fluxbin_w4_shape& s, const uint32_t* d_codes, const uint16_t* d_scales,
                              const uint8_t* d_zeros, void* d_packed, hipStream_t stream);
fluxbin_status launch_w4_quantize(const void* d_W, int w_is_fp32, int64_t ldw, const fluxbin_w4_shape& s,
                                  uint32_t* d_codes, uint16_t* d_scales, uint8_t* d_zeros, uint16_t* d_values,
                                  int64_t ldv, hipStream_t stream);

// ---- paged 8-bit key/value cache ----
// Sections: key codes, value codes (each pages x kv_heads x page_size x head_dim bytes), key scales, value scales.
struct Kv8Derived {
  uint64_t off_v, off_ks, off_vs, total;
};

inline Kv8Derived kv8_derive(int64_t pages, int32_t page_size, int32_t kv_heads, int32_t head_dim) {
  Kv8Derived d{};
  const uint64_t heads = uint64_t(pages) * uint64_t(kv_heads);
  const uint64_t codes = heads * uint64_t(page_size) * uint64_t(head_dim);   // a multiple of 1024
  d.off_v = codes;
  d.off_ks = 2 * codes;
  d.off_vs = d.off_ks + round_up256(heads * 4);
  d.total = d.off_vs + round_up256(heads * 4);
  return d;
}

struct Kv8Args {
  uint8_t* k;
  uint8_t* v;
  float* ks;
  float* vs;
  const int32_t* offsets;
  const int32_t* context;
  const int32_t* table;
  int64_t table_stride;
  int32_t pages, pshift, Hkv, T, B, max_blocks;   // page_size = 1 << pshift
};

struct Kv8AppendArgs {
  Kv8Args c;
  const uint16_t* src[2];      // keys, values
  int64_t ts[2], hs[2];        // token and head strides
};

struct Kv8ReadArgs {
  Kv8Args c;
  uint16_t* dst[2];
};

struct Kv8AttnArgs {
  Kv8Args c;
  const uint16_t* q;
  uint16_t* out;
  float* part;
  int64_t qts, qhs, ots, ohs;
  int32_t G, causal, window, wgs;   // query heads per cached head; workgroups that share the work
  int32_t chunk_from;               // columns (rows times G) of a sequence from which the prompt chunks' kernel takes it
  int32_t whole;                    // 1: a sequence's column tile and head is not split over workgroups
  float scale2;                     // softmax_scale * log2(e)
  const uint64_t* masks;            // of trees: [rows][words]
  int32_t words, col_shift;         // log2 of the columns of a column tile
};

uint64_t kv8_workspace(int32_t D, int cus);
fluxbin_status launch_kv8_append(const Kv8AppendArgs& a, int D, hipStream_t stream);
fluxbin_status launch_kv8_read(const Kv8ReadArgs& a, int D, hipStream_t stream);
fluxbin_status launch_kv8_attention(Kv8AttnArgs a, int D, int cus, hipStream_t stream);

}  // namespace fluxbin
