// Checks of arguments that the host sides of the operators share: overlaps, alignment, the paged 8-bit cache and its batches.
// All of them run before any HIP call.
#pragma once

#include <initializer_list>

#include "fluxbin_quant_internal.h"

namespace fluxbin {

struct Range {
  const void* p;
  uint64_t bytes;
};

// Whether any two of the buffers overlap (NULL and empty ones do not).
inline bool any_overlap(std::initializer_list<Range> written, std::initializer_list<Range> read) {
  auto hit = [](const Range& a, const Range& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return x && y && a.bytes && b.bytes && (x < y ? y - x < a.bytes : x - y < b.bytes);
  };
  for (const Range* w = written.begin(); w != written.end(); ++w) {
    for (const Range* v = w + 1; v != written.end(); ++v)
      if (hit(*w, *v)) return true;
    for (const Range& r : read)
      if (hit(*w, r)) return true;
  }
  return false;
}

inline bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

inline fluxbin_status check_kv8_sizes(int64_t pages, int32_t P, int32_t H, int32_t D) {
  if (pages < 1 || pages > (int64_t(1) << 24))
    return fail(FLUXBIN_ERR_INVALID_ARG, "pages = %lld out of range [1, 2^24]", (long long)pages);
  if (P < 1) return fail(FLUXBIN_ERR_INVALID_ARG, "page_size = %d must be >= 1", P);
  if (P != 16 && P != 32 && P != 64 && P != 128 && P != 256)
    return fail(FLUXBIN_ERR_UNSUPPORTED, "page_size = %d: supported are 16, 32, 64, 128, 256", P);
  if (H < 1 || H > 1024) return fail(FLUXBIN_ERR_INVALID_ARG, "kv_heads = %d out of range [1, 1024]", H);
  if (D < 1) return fail(FLUXBIN_ERR_INVALID_ARG, "head_dim = %d must be >= 1", D);
  if (D != 64 && D != 128 && D != 256)
    return fail(FLUXBIN_ERR_UNSUPPORTED, "head_dim = %d: supported are 64, 128, 256", D);
  if (pages * H > (int64_t(1) << 40) / (int64_t(P) * D))
    return fail(FLUXBIN_ERR_UNSUPPORTED, "the cache has more than 2^40 elements");
  return FLUXBIN_OK;
}

inline fluxbin_status check_kv8_cache(const fluxbin_kv8_cache* c) {
  if (!c) return fail(FLUXBIN_ERR_INVALID_ARG, "cache is NULL");
  if (c->format_version != FLUXBIN_KV8_FORMAT_VERSION)
    return fail(FLUXBIN_ERR_INVALID_ARG, "cache format version %u (expected %u)", c->format_version,
                FLUXBIN_KV8_FORMAT_VERSION);
  const fluxbin_status st = check_kv8_sizes(c->pages, c->page_size, c->kv_heads, c->head_dim);
  if (st != FLUXBIN_OK) return st;
  if (!c->d_base || misaligned(c->d_base, 256))
    return fail(FLUXBIN_ERR_INVALID_ARG, "cache buffer is NULL or not 256-byte aligned");
  if (c->bytes < kv8_derive(c->pages, c->page_size, c->kv_heads, c->head_dim).total)
    return fail(FLUXBIN_ERR_BUFFER_TOO_SMALL, "cache buffer is smaller than its format needs");
  return FLUXBIN_OK;
}

inline fluxbin_status check_kv8_rows(int64_t rows, int32_t sequences) {
  if (rows < 0 || rows > (int64_t(1) << 22))   // the kernels' grids have fewer than 2^32 threads
    return fail(FLUXBIN_ERR_INVALID_ARG, "rows = %lld out of range [0, 2^22]", (long long)rows);
  if (sequences < 1 || sequences > 65535)
    return fail(FLUXBIN_ERR_INVALID_ARG, "sequences = %d out of range [1, 65535]", sequences);
  return FLUXBIN_OK;
}

inline fluxbin_status check_kv8_call(const fluxbin_kv8_cache* c, const fluxbin_kv8_batch* b, Kv8Args* a) {
  fluxbin_status st = check_kv8_cache(c);
  if (st != FLUXBIN_OK) return st;
  if (!b) return fail(FLUXBIN_ERR_INVALID_ARG, "batch is NULL");
  st = check_kv8_rows(b->rows, b->sequences);
  if (st != FLUXBIN_OK) return st;
  if (!b->d_offsets || !b->d_context || !b->d_block_table)
    return fail(FLUXBIN_ERR_INVALID_ARG, "offsets, context or block table is NULL");
  if (misaligned(b->d_offsets, 4) || misaligned(b->d_context, 4) || misaligned(b->d_block_table, 4))
    return fail(FLUXBIN_ERR_INVALID_ARG, "offsets, context or block table is not aligned to its elements");
  if (b->max_blocks < 1 || b->max_blocks > (1 << 24))
    return fail(FLUXBIN_ERR_INVALID_ARG, "max_blocks = %d out of range [1, 2^24]", b->max_blocks);
  if (int64_t(b->max_blocks) * c->page_size > (int64_t(1) << 30))   // positions are 32-bit numbers
    return fail(FLUXBIN_ERR_UNSUPPORTED, "max_blocks * page_size exceeds 2^30 tokens");
  if (b->block_table_stride < b->max_blocks || b->block_table_stride > (int64_t(1) << 40))
    return fail(FLUXBIN_ERR_INVALID_ARG, "block_table_stride = %lld < max_blocks", (long long)b->block_table_stride);
  const Kv8Derived d = kv8_derive(c->pages, c->page_size, c->kv_heads, c->head_dim);
  uint8_t* base = static_cast<uint8_t*>(c->d_base);
  a->k = base;
  a->v = base + d.off_v;
  a->ks = reinterpret_cast<float*>(base + d.off_ks);
  a->vs = reinterpret_cast<float*>(base + d.off_vs);
  a->offsets = b->d_offsets;
  a->context = b->d_context;
  a->table = b->d_block_table;
  a->table_stride = b->block_table_stride;
  a->pages = int32_t(c->pages);
  a->pshift = 0;
  while ((1 << a->pshift) < c->page_size) ++a->pshift;
  a->Hkv = c->kv_heads;
  a->T = int32_t(b->rows);
  a->B = b->sequences;
  a->max_blocks = b->max_blocks;
  return FLUXBIN_OK;
}

inline Range table_range(const fluxbin_kv8_batch& b) {
  return {b.d_block_table, (uint64_t(b.sequences - 1) * uint64_t(b.block_table_stride) + uint64_t(b.max_blocks)) * 4};
}
inline Range offsets_range(const fluxbin_kv8_batch& b) { return {b.d_offsets, (uint64_t(b.sequences) + 1) * 4}; }
inline Range context_range(const fluxbin_kv8_batch& b) { return {b.d_context, uint64_t(b.sequences) * 4}; }

// A packed tensor of rows x heads x D with element strides: its bounds, and whether no two of its elements are the same.
inline fluxbin_status check_strided(const char* name, const void* p, int64_t rows, int32_t heads, int32_t D, int64_t ts, int64_t hs,
                             bool written, Range* r) {
  if (rows > 0 && !p) return fail(FLUXBIN_ERR_INVALID_ARG, "%s is NULL", name);
  if (misaligned(p, 2)) return fail(FLUXBIN_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
  if (ts < 0 || hs < 0 || ts > (int64_t(1) << 36) || hs > (int64_t(1) << 36))
    return fail(FLUXBIN_ERR_INVALID_ARG, "%s: strides must be in [0, 2^36]", name);
  if (heads > 1 && hs < D) return fail(FLUXBIN_ERR_INVALID_ARG, "%s: head stride %lld < head_dim", name, (long long)hs);
  const int64_t row = int64_t(heads - 1) * hs + D;   // extent of a token
  if (written && rows > 1 && ts < row && !(ts >= D && hs >= int64_t(rows - 1) * ts + D))
    return fail(FLUXBIN_ERR_INVALID_ARG, "%s: rows overlap (token stride %lld)", name, (long long)ts);
  *r = {p, rows > 0 ? uint64_t((rows - 1) * ts + row) * 2 : 0};
  return FLUXBIN_OK;
}

}  // namespace fluxbin
