// Device-side pieces of the paged 8-bit key/value cache: its layout, and which sequence and page a row belongs to.
//
// A page and head holds page_size x D codes, as blocks of 16 tokens x 64 elements (1 KB), [page][head][token / 16][D / 64]
// [64 lanes][16 bytes], in the order in which the attention's matrix instructions take them, so that a wavefront reads a
// block with one 16-byte load per lane and no exchange between lanes:
//   keys    lane (token m = lane & 15, q = lane >> 4): elements 32 f + 8 q + e, f = 0, 1, e = 0..7, at byte 8 f + e;
//   values  lane (element m, q): elements 16 t + m of tokens 4 q + i, t = 0..3, i = 0..3, at byte 4 t + i.
// A byte is the code + 128.
#pragma once

#include "fluxbin_device.h"
#include "fluxbin_quant_internal.h"

namespace fluxbin {

typedef _Float16 kv_h2 __attribute__((ext_vector_type(2)));
typedef _Float16 kv_h4 __attribute__((ext_vector_type(4)));
typedef _Float16 kv_h8 __attribute__((ext_vector_type(8)));
typedef float kv_f4 __attribute__((ext_vector_type(4)));
typedef unsigned int kv_u2 __attribute__((ext_vector_type(2)));
typedef unsigned int kv_u4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kKvZero = 0x80808080u;   // four codes of 0

// Byte offset of a page and head in a section of codes, and of a token block in it.
template <int D>
__device__ __forceinline__ int64_t kv_page_offset(const Kv8Args& a, int page, int head) {
  return ((int64_t(page) * a.Hkv + head) << a.pshift) * D;
}

// The sequence of row t (the same for all lanes of a wavefront), or -1: the last whose offset is not above t, 64 candidates
// at a time.
__device__ __forceinline__ int kv_sequence(const Kv8Args& a, int t, int& start, int& end) {
  const int lane = int(threadIdx.x) & 63;
  int lo = 0, n = a.B;   // it is one of lo .. lo + n - 1, where the offsets do not fall
  while (n > 1) {
    const int step = (n + 63) >> 6, at = lo + lane * step;
    const uint64_t below = __ballot(lane * step < n && a.offsets[lane * step < n ? at : lo] <= t);
    const int l = below ? 63 - __clzll((long long)below) : 0;
    lo += l * step;
    n = n - l * step < step ? n - l * step : step;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  start = a.offsets[lo];
  end = a.offsets[lo + 1];
  return start >= 0 && end <= a.T && start <= t && t < end ? lo : -1;
}

// Tokens of sequence b, within the 2^30 positions that a block table can have.
__device__ __forceinline__ int kv_context(const Kv8Args& a, int b) {
  const int c = a.context[b];
  return c < 0 ? 0 : c > (1 << 30) ? 1 << 30 : c;
}

// The page of a position of sequence b, or -1.
__device__ __forceinline__ int kv_page(const Kv8Args& a, int b, int pos) {
  const int p = pos >> a.pshift;
  if (pos < 0 || p >= a.max_blocks) return -1;
  const int page = a.table[b * a.table_stride + p];
  return page >= 0 && page < a.pages ? page : -1;
}

}  // namespace fluxbin
