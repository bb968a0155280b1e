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

}  // extern "C"

}  // namespace fluxbin
