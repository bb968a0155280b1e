// Internal declarations of the operators next to the binary linears: 4-bit linears (fluxbin_w4_*).
#pragma once

#include "fluxbin_internal.h"
#include "fluxbin_quant.h"

namespace fluxbin {

// ---- 4-bit linears ----
constexpr int kW4MaxBatch = kMaxBatchCall;   // batch rows of one call
// Row tiles of 16 rows, column chunks of kChunk columns, steps of 4 chunks. Scales (and zero points) come in quads per
// row: 4 chunks' at one per chunk (group >= 128), 2 chunks' at two, one chunk's at four.
struct W4Derived {
  int64_t G;           // groups per row, canonical
  int64_t Mt, Nc;      // row tiles, chunks
  int gc;              // scales per chunk and row: 1, 2 or 4
  int64_t Nq;          // quads per row
  uint64_t off_scales, off_zeros, total;
};

inline W4Derived w4_derive(const fluxbin_w4_shape& s) {
  W4Derived d{};
  d.G = ceil_div(s.N, s.g);
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

}  // namespace fluxbin
