// Host side of the operators next to the binary linears: argument validation and the C ABI entry points.
// Every check runs before any HIP call so that invalid input never reaches a kernel.
#include <hip/hip_runtime.h>

#include <cstring>
#include <initializer_list>

#include "fluxbin_quant_internal.h"

namespace fluxbin {

namespace {

struct Range {
  const void* p;
  uint64_t bytes;
};

// Whether any two of the buffers overlap (NULL and empty ones do not).
bool any_overlap(std::initializer_list<Range> written, std::initializer_list<Range> read) {
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

bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// ---------------------------------------------------------------------------------------------- 4-bit linears

fluxbin_status check_w4_shape(const fluxbin_w4_shape* s) {
  if (!s) return fail(FLUXBIN_ERR_INVALID_ARG, "shape is NULL");
  if (s->M < 1 || s->M > (int64_t(1) << 24))
    return fail(FLUXBIN_ERR_INVALID_ARG, "M = %lld out of range [1, 2^24]", (long long)s->M);
  if (s->N < 1 || s->N > (int64_t(1) << 20))
    return fail(FLUXBIN_ERR_INVALID_ARG, "N = %lld out of range [1, 2^20]", (long long)s->N);
  if (s->M * s->N > (int64_t(1) << 34))   // the quantizer's grid has 2^32 threads at most
    return fail(FLUXBIN_ERR_UNSUPPORTED, "M * N = %lld exceeds 2^34", (long long)(s->M * s->N));
  if (s->g < 1) return fail(FLUXBIN_ERR_INVALID_ARG, "g = %lld must be >= 1", (long long)s->g);
  if (s->g < s->N && s->g != 32 && s->g != 64 && s->g % kChunk != 0)
    return fail(FLUXBIN_ERR_UNSUPPORTED, "g = %lld: supported are 32, 64, multiples of 128, or g >= N", (long long)s->g);
  if (s->has_zeros != 0 && s->has_zeros != 1) return fail(FLUXBIN_ERR_INVALID_ARG, "has_zeros must be 0 or 1");
  return FLUXBIN_OK;
}

fluxbin_status check_w4_layer(const fluxbin_w4_layer* L) {
  if (!L) return fail(FLUXBIN_ERR_INVALID_ARG, "layer is NULL");
  if (L->format_version != FLUXBIN_W4_FORMAT_VERSION)
    return fail(FLUXBIN_ERR_INVALID_ARG, "4-bit layer format version %u (expected %u)", L->format_version,
                FLUXBIN_W4_FORMAT_VERSION);
  if (!L->d_base) return fail(FLUXBIN_ERR_INVALID_ARG, "layer has no device buffer");
  if (misaligned(L->d_base, 16)) return fail(FLUXBIN_ERR_INVALID_ARG, "layer buffer is not 16-byte aligned");
  const fluxbin_status st = check_w4_shape(&L->shape);
  if (st != FLUXBIN_OK) return st;
  if (L->bytes < w4_derive(L->shape).total)
    return fail(FLUXBIN_ERR_BUFFER_TOO_SMALL, "layer buffer is smaller than its format needs");
  return FLUXBIN_OK;
}

// ---------------------------------------------------------------------------------------------- 8-bit cache

fluxbin_status check_kv8_sizes(int64_t pages, int32_t P, int32_t H, int32_t D) {
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

fluxbin_status check_kv8_cache(const fluxbin_kv8_cache* c) {
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

fluxbin_status check_kv8_rows(int64_t rows, int32_t sequences) {
  if (rows < 0 || rows > (int64_t(1) << 22))   // the kernels' grids have fewer than 2^32 threads
    return fail(FLUXBIN_ERR_INVALID_ARG, "rows = %lld out of range [0, 2^22]", (long long)rows);
  if (sequences < 1 || sequences > 65535)
    return fail(FLUXBIN_ERR_INVALID_ARG, "sequences = %d out of range [1, 65535]", sequences);
  return FLUXBIN_OK;
}

fluxbin_status check_kv8_call(const fluxbin_kv8_cache* c, const fluxbin_kv8_batch* b, Kv8Args* a) {
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

Range table_range(const fluxbin_kv8_batch& b) {
  return {b.d_block_table, (uint64_t(b.sequences - 1) * uint64_t(b.block_table_stride) + uint64_t(b.max_blocks)) * 4};
}
Range offsets_range(const fluxbin_kv8_batch& b) { return {b.d_offsets, (uint64_t(b.sequences) + 1) * 4}; }
Range context_range(const fluxbin_kv8_batch& b) { return {b.d_context, uint64_t(b.sequences) * 4}; }

// A packed tensor of rows x heads x D with element strides: its bounds, and whether no two of its elements are the same.
fluxbin_status check_strided(const char* name, const void* p, int64_t rows, int32_t heads, int32_t D, int64_t ts, int64_t hs,
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

}  // namespace

extern "C" {

fluxbin_status fluxbin_w4_quantize(const fluxbin_w4_shape* shape, const void* d_W, int32_t w_is_fp32, int64_t ldw,
                                   uint32_t* d_codes, uint16_t* d_scales, uint8_t* d_zeros, uint16_t* d_values,
                                   int64_t ldv, hipStream_t stream) {
  clear_error();
  const fluxbin_status st = check_w4_shape(shape);
  if (st != FLUXBIN_OK) return st;
  const fluxbin_w4_shape& s = *shape;
  if (!d_W || !d_codes || !d_scales) return fail(FLUXBIN_ERR_INVALID_ARG, "W, codes or scales is NULL");
  if (w_is_fp32 != 0 && w_is_fp32 != 1) return fail(FLUXBIN_ERR_INVALID_ARG, "w_is_fp32 must be 0 or 1");
  if ((d_zeros != nullptr) != (s.has_zeros != 0))
    return fail(FLUXBIN_ERR_INVALID_ARG, "zeros must be given with has_zeros, and only then");
  if (ldw < s.N || ldw > (int64_t(1) << 40)) return fail(FLUXBIN_ERR_INVALID_ARG, "ldw = %lld < N", (long long)ldw);
  if (d_values && (ldv < s.N || ldv > (int64_t(1) << 40)))
    return fail(FLUXBIN_ERR_INVALID_ARG, "ldv = %lld < N", (long long)ldv);
  const uint64_t elt = w_is_fp32 ? 4 : 2;
  if (misaligned(d_W, elt) || misaligned(d_codes, 4) || misaligned(d_scales, 2) || misaligned(d_values, 2))
    return fail(FLUXBIN_ERR_INVALID_ARG, "W, codes, scales or values is not aligned to its elements");
  const uint64_t M = uint64_t(s.M), G = uint64_t(w4_derive(s).G);
  if (any_overlap({{d_codes, M * uint64_t(ceil_div(s.N, 8)) * 4}, {d_scales, M * G * 2}, {d_zeros, M * G},
                   {d_values, ((M - 1) * uint64_t(d_values ? ldv : 0) + uint64_t(s.N)) * 2}},
                  {{d_W, ((M - 1) * uint64_t(ldw) + uint64_t(s.N)) * elt}}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "W and the outputs overlap");
  return launch_w4_quantize(d_W, w_is_fp32, ldw, s, d_codes, d_scales, d_zeros, d_values, ldv, stream);
}

fluxbin_status fluxbin_w4_pack_query(const fluxbin_w4_shape* shape, size_t* packed_bytes) {
  clear_error();
  const fluxbin_status st = check_w4_shape(shape);
  if (st != FLUXBIN_OK) return st;
  if (!packed_bytes) return fail(FLUXBIN_ERR_INVALID_ARG, "packed_bytes is NULL");
  *packed_bytes = size_t(w4_derive(*shape).total);
  return FLUXBIN_OK;
}

fluxbin_status fluxbin_w4_pack(const fluxbin_w4_shape* shape, const uint32_t* d_codes, const uint16_t* d_scales,
                               const uint8_t* d_zeros, void* d_packed, size_t packed_bytes, fluxbin_w4_layer* out,
                               hipStream_t stream) {
  clear_error();
  fluxbin_status st = check_w4_shape(shape);
  if (st != FLUXBIN_OK) return st;
  if (!out) return fail(FLUXBIN_ERR_INVALID_ARG, "out is NULL");
  if (!d_codes || !d_scales || !d_packed) return fail(FLUXBIN_ERR_INVALID_ARG, "codes, scales or d_packed is NULL");
  if ((d_zeros != nullptr) != (shape->has_zeros != 0))
    return fail(FLUXBIN_ERR_INVALID_ARG, "zeros must be given with has_zeros, and only then");
  const W4Derived d = w4_derive(*shape);
  if (packed_bytes < d.total)
    return fail(FLUXBIN_ERR_BUFFER_TOO_SMALL, "packed buffer has %zu bytes, needs %llu", packed_bytes,
                (unsigned long long)d.total);
  if (misaligned(d_packed, 16) || misaligned(d_codes, 4) || misaligned(d_scales, 2))
    return fail(FLUXBIN_ERR_INVALID_ARG, "d_packed is not 16-byte aligned, or codes or scales not to their elements");
  const uint64_t M = uint64_t(shape->M);
  if (any_overlap({{d_packed, d.total}}, {{d_codes, M * uint64_t(ceil_div(shape->N, 8)) * 4},
                                          {d_scales, M * uint64_t(d.G) * 2}, {d_zeros, M * uint64_t(d.G)}}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "the packed buffer overlaps an input");
  st = launch_w4_pack(*shape, d_codes, d_scales, d_zeros, d_packed, stream);
  if (st != FLUXBIN_OK) return st;
  std::memset(out, 0, sizeof(*out));
  out->shape = *shape;
  out->d_base = d_packed;
  out->bytes = packed_bytes;
  out->format_version = FLUXBIN_W4_FORMAT_VERSION;
  return FLUXBIN_OK;
}

fluxbin_status fluxbin_w4_workspace_query(const fluxbin_w4_layer* layer, int32_t B, size_t* bytes) {
  clear_error();
  fluxbin_status st = check_w4_layer(layer);
  if (st != FLUXBIN_OK) return st;
  if (!bytes) return fail(FLUXBIN_ERR_INVALID_ARG, "bytes is NULL");
  if (B < 1 || B > kW4MaxBatch) return fail(FLUXBIN_ERR_INVALID_ARG, "B = %d out of range [1, %d]", B, kW4MaxBatch);
  const int cus = device_cu_count();
  if (cus < 1) return fail(FLUXBIN_ERR_HIP, "reading the device's CU count failed");
  *bytes = size_t(w4_workspace(layer->shape, B, cus));
  return FLUXBIN_OK;
}

fluxbin_status fluxbin_w4_gemm(const fluxbin_w4_layer* layer, int32_t B, const uint16_t* d_x, int64_t ldx, void* d_y,
                               int64_t ldy, int32_t y_is_fp32, void* d_workspace, size_t workspace_bytes,
                               hipStream_t stream) {
  clear_error();
  fluxbin_status st = check_w4_layer(layer);
  if (st != FLUXBIN_OK) return st;
  const fluxbin_w4_shape& s = layer->shape;
  if (B < 1 || B > kW4MaxBatch) return fail(FLUXBIN_ERR_INVALID_ARG, "B = %d out of range [1, %d]", B, kW4MaxBatch);
  if (!d_x || !d_y) return fail(FLUXBIN_ERR_INVALID_ARG, "x or y is NULL");
  if (y_is_fp32 != 0 && y_is_fp32 != 1) return fail(FLUXBIN_ERR_INVALID_ARG, "y_is_fp32 must be 0 or 1");
  if (B == 1) {
    ldx = s.N;
    ldy = s.M;
  }
  if (ldx < s.N || ldx > (int64_t(1) << 40)) return fail(FLUXBIN_ERR_INVALID_ARG, "ldx = %lld < N", (long long)ldx);
  if (ldy < s.M || ldy > (int64_t(1) << 40)) return fail(FLUXBIN_ERR_INVALID_ARG, "ldy = %lld < M", (long long)ldy);
  if (misaligned(d_x, 2) || misaligned(d_y, y_is_fp32 ? 4 : 2))
    return fail(FLUXBIN_ERR_INVALID_ARG, "x or y is not aligned to its elements");
  const int cus = device_cu_count();
  if (cus < 1) return fail(FLUXBIN_ERR_HIP, "reading the device's CU count failed");
  const W4Plan p = w4_plan(s, B, cus);
  if (p.ws_bytes > workspace_bytes)
    return fail(FLUXBIN_ERR_BUFFER_TOO_SMALL, "workspace has %zu bytes, needs %llu", workspace_bytes,
                (unsigned long long)w4_workspace(s, B, cus));
  if (p.ws_bytes > 0 && (!d_workspace || misaligned(d_workspace, 16)))
    return fail(FLUXBIN_ERR_INVALID_ARG, "workspace is NULL or not 16-byte aligned");
  if (any_overlap({{d_y, (uint64_t(B - 1) * uint64_t(ldy) + uint64_t(s.M)) * (y_is_fp32 ? 4 : 2)},
                   {d_workspace, p.ws_bytes}},
                  {{d_x, (uint64_t(B - 1) * uint64_t(ldx) + uint64_t(s.N)) * 2}, {layer->d_base, layer->bytes}}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "x, y, the workspace and the layer overlap");
  const W4Derived d = w4_derive(s);
  const uint8_t* base = static_cast<const uint8_t*>(layer->d_base);
  W4Args a{};
  a.codes = base;
  a.scales = base + d.off_scales;
  a.zeros = s.has_zeros ? base + d.off_zeros : nullptr;
  a.x = d_x;
  a.y = d_y;
  a.partials = static_cast<float*>(d_workspace);
  a.ldx = ldx;
  a.ldy = ldy;
  a.M = int32_t(s.M);
  a.N = int32_t(s.N);
  a.B = B;
  a.Mt = int32_t(d.Mt);
  a.Nc = int32_t(d.Nc);
  a.Nq = int32_t(d.Nq);
  a.y_fp32 = y_is_fp32;
  a.parts = p.parts;
  return launch_w4_gemm(a, p, d.gc, stream);
}

fluxbin_status fluxbin_kv8_cache_query(int64_t pages, int32_t page_size, int32_t kv_heads, int32_t head_dim,
                                       size_t* bytes) {
  clear_error();
  const fluxbin_status st = check_kv8_sizes(pages, page_size, kv_heads, head_dim);
  if (st != FLUXBIN_OK) return st;
  if (!bytes) return fail(FLUXBIN_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = size_t(kv8_derive(pages, page_size, kv_heads, head_dim).total);
  return FLUXBIN_OK;
}

fluxbin_status fluxbin_kv8_append(const fluxbin_kv8_cache* cache, const fluxbin_kv8_batch* batch, const uint16_t* d_k,
                                  int64_t k_token_stride, int64_t k_head_stride, const uint16_t* d_v,
                                  int64_t v_token_stride, int64_t v_head_stride, hipStream_t stream) {
  clear_error();
  Kv8AppendArgs a{};
  fluxbin_status st = check_kv8_call(cache, batch, &a.c);
  if (st != FLUXBIN_OK) return st;
  Range k, v;
  const int32_t H = cache->kv_heads, D = cache->head_dim;
  st = check_strided("k", d_k, batch->rows, H, D, k_token_stride, k_head_stride, false, &k);
  if (st != FLUXBIN_OK) return st;
  st = check_strided("v", d_v, batch->rows, H, D, v_token_stride, v_head_stride, false, &v);
  if (st != FLUXBIN_OK) return st;
  if (any_overlap({{cache->d_base, cache->bytes}},
                  {k, v, table_range(*batch), offsets_range(*batch), context_range(*batch)}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "the cache overlaps an input");
  if (batch->rows == 0) return FLUXBIN_OK;
  a.src[0] = d_k;
  a.src[1] = d_v;
  a.ts[0] = k_token_stride;
  a.ts[1] = v_token_stride;
  a.hs[0] = k_head_stride;
  a.hs[1] = v_head_stride;
  return launch_kv8_append(a, D, stream);
}

fluxbin_status fluxbin_kv8_read(const fluxbin_kv8_cache* cache, const fluxbin_kv8_batch* batch, uint16_t* d_k,
                                uint16_t* d_v, hipStream_t stream) {
  clear_error();
  Kv8ReadArgs a{};
  const fluxbin_status st = check_kv8_call(cache, batch, &a.c);
  if (st != FLUXBIN_OK) return st;
  if (batch->rows == 0) return FLUXBIN_OK;
  if (!d_k || !d_v) return fail(FLUXBIN_ERR_INVALID_ARG, "k or v is NULL");
  if (misaligned(d_k, 16) || misaligned(d_v, 16)) return fail(FLUXBIN_ERR_INVALID_ARG, "k or v is not 16-byte aligned");
  const uint64_t n = uint64_t(batch->rows) * uint64_t(cache->kv_heads) * uint64_t(cache->head_dim) * 2;
  if (any_overlap({{d_k, n}, {d_v, n}}, {{cache->d_base, cache->bytes}, table_range(*batch), offsets_range(*batch),
                                         context_range(*batch)}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "k, v, the cache and the batch's arrays overlap");
  a.dst[0] = d_k;
  a.dst[1] = d_v;
  return launch_kv8_read(a, cache->head_dim, stream);
}

fluxbin_status fluxbin_kv8_workspace_query(const fluxbin_kv8_cache* cache, int64_t rows, int32_t sequences,
                                           int32_t q_heads, size_t* bytes) {
  clear_error();
  fluxbin_status st = check_kv8_cache(cache);
  if (st != FLUXBIN_OK) return st;
  st = check_kv8_rows(rows, sequences);
  if (st != FLUXBIN_OK) return st;
  if (q_heads < 1 || q_heads > 1024 || q_heads % cache->kv_heads != 0)
    return fail(FLUXBIN_ERR_INVALID_ARG, "q_heads = %d must be a multiple of kv_heads, up to 1024", q_heads);
  if (!bytes) return fail(FLUXBIN_ERR_INVALID_ARG, "bytes is NULL");
  const int cus = device_cu_count();
  if (cus < 1) return fail(FLUXBIN_ERR_HIP, "reading the device's CU count failed");
  *bytes = size_t(kv8_workspace(cache->head_dim, cus));
  return FLUXBIN_OK;
}

fluxbin_status fluxbin_kv8_attention(const fluxbin_kv8_cache* cache, const fluxbin_kv8_batch* batch, int32_t q_heads,
                                     const uint16_t* d_q, int64_t q_token_stride, int64_t q_head_stride, uint16_t* d_out,
                                     int64_t out_token_stride, int64_t out_head_stride, float softmax_scale,
                                     int32_t causal, int32_t window, void* d_workspace, size_t workspace_bytes,
                                     hipStream_t stream) {
  clear_error();
  Kv8AttnArgs a{};
  fluxbin_status st = check_kv8_call(cache, batch, &a.c);
  if (st != FLUXBIN_OK) return st;
  const int32_t H = cache->kv_heads, D = cache->head_dim;
  if (q_heads < 1 || q_heads > 1024 || q_heads % H != 0)
    return fail(FLUXBIN_ERR_INVALID_ARG, "q_heads = %d must be a multiple of kv_heads, up to 1024", q_heads);
  if (batch->rows * (q_heads / H) > (int64_t(1) << 30))   // rows times heads of a group are 32-bit numbers
    return fail(FLUXBIN_ERR_UNSUPPORTED, "rows * (q_heads / kv_heads) exceeds 2^30");
  if (!(softmax_scale > -1e30f && softmax_scale < 1e30f))
    return fail(FLUXBIN_ERR_INVALID_ARG, "softmax_scale must be a finite number");
  if (causal != 0 && causal != 1) return fail(FLUXBIN_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (window < 0) return fail(FLUXBIN_ERR_INVALID_ARG, "window = %d must be >= 0", window);
  Range q, out;
  st = check_strided("q", d_q, batch->rows, q_heads, D, q_token_stride, q_head_stride, false, &q);
  if (st != FLUXBIN_OK) return st;
  st = check_strided("out", d_out, batch->rows, q_heads, D, out_token_stride, out_head_stride, true, &out);
  if (st != FLUXBIN_OK) return st;
  const int cus = device_cu_count();
  if (cus < 1) return fail(FLUXBIN_ERR_HIP, "reading the device's CU count failed");
  const uint64_t need = kv8_workspace(D, cus);
  if (workspace_bytes < need)
    return fail(FLUXBIN_ERR_BUFFER_TOO_SMALL, "workspace has %zu bytes, needs %llu", workspace_bytes,
                (unsigned long long)need);
  if (!d_workspace || misaligned(d_workspace, 16))
    return fail(FLUXBIN_ERR_INVALID_ARG, "workspace is NULL or not 16-byte aligned");
  if (any_overlap({out, {d_workspace, need}}, {q, {cache->d_base, cache->bytes}, table_range(*batch),
                                               offsets_range(*batch), context_range(*batch)}))
    return fail(FLUXBIN_ERR_INVALID_ARG, "out, the workspace and the inputs overlap");
  if (batch->rows == 0) return FLUXBIN_OK;
  a.q = d_q;
  a.out = d_out;
  a.part = static_cast<float*>(d_workspace);
  a.qts = q_token_stride;
  a.qhs = q_head_stride;
  a.ots = out_token_stride;
  a.ohs = out_head_stride;
  a.G = q_heads / H;
  a.causal = causal;
  a.window = window;
  a.scale2 = softmax_scale * 1.4426950408889634f;
  return launch_kv8_attention(a, D, cus, stream);
}

}  // extern "C"

}  // namespace fluxbin
