// Paged key/value cache in 8 bits: storing new tokens and reading them back.
//
// Both are bound by memory where there is much to do: storing four prompts of 301 to 2000 tokens, 40 heads of 128, from rows of
// a fused projection 50 us (126 MB; 42 us from dense rows), reading them back 25.5 us (145 MB, 5.7 TB/s). A single token of 32
// sequences is 4.2 to 5.3 us under the profiler: five requests one after another (sequence, lengths, page, values, scale).
#include "fluxbin_kv8_device.h"

namespace fluxbin {

namespace {

// Eight new elements as they are stored: NaN as 0, an infinity as the largest fp16. Returns the bits of the largest magnitude
// (the order of fp16 magnitudes is that of their bits).
__device__ __forceinline__ uint32_t kv_clean8(uint16_t (&h)[8]) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  uint32_t w[4];
  __builtin_memcpy(w, h, 16);
  u16x2 pair = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) pair = __builtin_elementwise_max(pair, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
  uint32_t most = pair.x > pair.y ? pair.x : pair.y;
  if (most < 0x7C00u) return most;   // nearly always: all finite
  most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t m = h[i] & 0x7FFFu;
    h[i] = m > 0x7C00u ? uint16_t(0) : m == 0x7C00u ? uint16_t(h[i] - 1) : h[i];
    const uint32_t k = h[i] & 0x7FFFu;
    most = k > most ? k : most;
  }
  return most;
}

// rne(v * inv) + 128 in the low byte of the result (v * inv is in -127.5 .. 127.5, past 127 by roundings only): the sum with
// 1.5 * 2^23 + 128 has no bits below one.
__device__ __forceinline__ uint32_t kv_code(uint16_t h, float inv) {
#pragma clang fp contract(off)
  const float p = h2f(h) * inv;   // rounded to fp32 before it is rounded to a number
  return __builtin_bit_cast(uint32_t, p + 12583040.f);
}

__device__ __forceinline__ uint32_t kv_code4(uint16_t a, uint16_t b, uint16_t c, uint16_t d, float inv) {
  const uint32_t lo = __builtin_amdgcn_perm(kv_code(b, inv), kv_code(a, inv), 0x0C0C0400u);
  const uint32_t hi = __builtin_amdgcn_perm(kv_code(d, inv), kv_code(c, inv), 0x04000C0Cu);
  return lo | hi;
}

// An earlier token's code after its page's scale has grown.
__device__ __forceinline__ uint32_t kv_recode(uint32_t byte, float ratio) {
  return uint32_t(int(__builtin_rintf(float(int(byte) - 128) * ratio)) + 128);
}

constexpr int kSlab = 64;   // tokens that are staged in LDS at a time (units straight from memory, two bytes of sixteen
                            // places each, took four times as long)

// One page and head's new tokens, keys (SIDE 0) or values (SIDE 1), by a whole workgroup: the largest new magnitude, the
// scale, then every 16-byte unit of the page that holds a new token or, where the scale grows, an earlier one. The new
// values go through LDS, where a unit of values picks its sixteen elements from four tokens.
template <int D, int SIDE>
__device__ void kv_store_page(const Kv8AppendArgs& a, int page, int head, int row, int first, int count, float* red,
                              uint16_t (*slab)[D]) {
  const Kv8Args& c = a.c;
  const uint16_t* src = a.src[SIDE] + int64_t(row) * a.ts[SIDE] + int64_t(head) * a.hs[SIDE];
  // tokens 0 .. staged - 1 of the new ones are in the slab afterwards
  const int staged = count < kSlab ? count : kSlab;
  uint32_t most = 0;
#pragma unroll 4
  for (int e = int(threadIdx.x); e < count * (D / 8); e += 256) {
    uint16_t h[8];
    const int t = e / (D / 8), d = e % (D / 8) * 8;
    __builtin_memcpy(h, src + int64_t(t) * a.ts[SIDE] + d, 16);
    const uint32_t m = kv_clean8(h);
    most = m > most ? m : most;
    if (t < staged) __builtin_memcpy(&slab[t][d], h, 16);
  }
  float amax = h2f(uint16_t(most));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  float* scale = (SIDE ? c.vs : c.ks) + int64_t(page) * c.Hkv + head;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = amax;
  if (threadIdx.x == 0) red[4] = first > 0 ? *scale : 0.f;   // read and written by one thread only
  __syncthreads();
  const float old = red[4];
  amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float s = fmaxf(old, amax * (1.f / 127.f));
  const float inv = s > 0.f ? 1.f / s : 0.f, ratio = s > old ? old / s : 1.f;
  if (threadIdx.x == 0) *scale = s;
  const int last = first + count;
  uint8_t* base = (SIDE ? c.v : c.k) + kv_page_offset<D>(c, page, head);
  int from = 0;   // the new token that slab[0] holds
  // blocks of 16 tokens up to the last new one, those that the slab covers at a time
  for (int b0 = s > old ? 0 : first >> 4; b0 < (last + 15) >> 4;) {
    int b1 = (first + from + kSlab) >> 4;   // whole blocks only, or all that are left
    if (first + from + kSlab >= last) b1 = (last + 15) >> 4;
    for (int u = b0 * D + int(threadIdx.x); u < b1 * D; u += 256) {   // 16-byte units: D per block
      const int lane = u & 63, blk = (u >> 6) % (D / 64), tb = (u >> 6) / (D / 64), m = lane & 15, q = lane >> 4;
      const int t0 = 16 * tb + (SIDE ? 4 * q : m), t1 = t0 + (SIDE ? 4 : 1);   // the unit's tokens
      const bool fresh = t1 > first && t0 < last;
      if (!fresh && (t0 >= last || ratio == 1.f)) continue;
      kv_u4 w = {kKvZero, kKvZero, kKvZero, kKvZero};
      if (t0 < first) {
        w = *reinterpret_cast<const kv_u4*>(base + int64_t(u) * 16);
        if (ratio != 1.f) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t r = kv_recode((w[i >> 2] >> (8 * (i & 3))) & 255u, ratio);
            w[i >> 2] = (w[i >> 2] & ~(255u << (8 * (i & 3)))) | (r << (8 * (i & 3)));
          }
        }
      }
      if (fresh) {
        if (SIDE == 0) {
          const uint16_t* p = &slab[t0 - first - from][64 * blk + 8 * q];
#pragma unroll
          for (int f = 0; f < 2; ++f) {
            uint16_t h[8];
            __builtin_memcpy(h, p + 32 * f, 16);
#pragma unroll
            for (int e = 0; e < 8; e += 4)
              w[2 * f + e / 4] = kv_code4(h[e], h[e + 1], h[e + 2], h[e + 3], inv);
          }
        } else if (t0 >= first && t1 <= last) {   // all four tokens are new
          const uint16_t* p = &slab[t0 - first - from][64 * blk + m];
#pragma unroll
          for (int dt = 0; dt < 4; ++dt)
            w[dt] = kv_code4(p[16 * dt], p[D + 16 * dt], p[2 * D + 16 * dt], p[3 * D + 16 * dt], inv);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int t = t0 + i;
            if (t < first) continue;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
              const uint32_t r = t < last ? kv_code(slab[t - first - from][64 * blk + 16 * dt + m], inv) & 255u : 128u;
              w[dt] = (w[dt] & ~(255u << (8 * i))) | (r << (8 * i));
            }
          }
        }
      }
      *reinterpret_cast<kv_u4*>(base + int64_t(u) * 16) = w;
    }
    b0 = b1;
    if (b0 < (last + 15) >> 4) {   // the next tokens into the slab, from block b0's first on
      from = 16 * b0 - first;
      __syncthreads();
      for (int e = int(threadIdx.x); e < kSlab * (D / 8); e += 256) {
        const int t = e / (D / 8), d = e % (D / 8) * 8;
        if (from + t >= count) continue;
        uint16_t h[8];
        __builtin_memcpy(h, src + int64_t(from + t) * a.ts[SIDE] + d, 16);
        kv_clean8(h);
        __builtin_memcpy(&slab[t][d], h, 16);
      }
      __syncthreads();
    }
  }
}

// Workgroup (window of `span` rows, `heads` heads, side): the rows of its window that are the first of their sequence or of
// their page start a page's new tokens.
template <int D>
__global__ void __launch_bounds__(256) k_kv8_append(Kv8AppendArgs a, int span, int heads) {
  __shared__ float red[5];
  __shared__ __attribute__((aligned(16))) uint16_t slab[kSlab][D];
  const Kv8Args& c = a.c;
  const int P = 1 << c.pshift;
  const int stop = int(blockIdx.x) * span + span < c.T ? int(blockIdx.x) * span + span : c.T;
  for (int t = int(blockIdx.x) * span, next; t < stop; t = next) {
    int start, end;
    const int b = kv_sequence(c, t, start, end);
    next = t + 1;
    if (b < 0) continue;
    const int pos = kv_context(c, b) - (end - t);   // may be negative
    next = t + (P - (pos & (P - 1))) < end ? t + (P - (pos & (P - 1))) : end;   // the next page's or sequence's first row
    if (pos < 0 || (t != start && (pos & (P - 1)) != 0)) continue;
    const int page = kv_page(c, b, pos);
    if (page < 0) continue;
    const int first = pos & (P - 1), left = end - t, count = left < P - first ? left : P - first;
    const int h1 = int(blockIdx.y) * heads + heads < c.Hkv ? int(blockIdx.y) * heads + heads : c.Hkv;
    for (int h = int(blockIdx.y) * heads; h < h1; ++h) {
      __syncthreads();   // red and slab of the page or head before
      if (blockIdx.z == 0)
        kv_store_page<D, 0>(a, page, h, t, first, count, red, slab);
      else
        kv_store_page<D, 1>(a, page, h, t, first, count, red, slab);
    }
  }
}

// Wavefront (window of `span` rows, head; workgroup: four heads): the rows of its window that are the first of their sequence
// or of 16 positions start a block of 16 tokens, which it reads as it is stored. Values go through LDS: a unit holds one
// element of 16, four tokens deep.
template <int D>
__global__ void __launch_bounds__(256) k_kv8_read(Kv8ReadArgs a, int span) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[4][16][64 + 8];
  const Kv8Args& c = a.c;
  const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6, m = lane & 15, q = lane >> 4, side = int(blockIdx.z);
  const int head = int(blockIdx.y) * 4 + wave;
  if (head >= c.Hkv) return;
  const int stop = int(blockIdx.x) * span + span < c.T ? int(blockIdx.x) * span + span : c.T;
  for (int t = int(blockIdx.x) * span, next; t < stop; t = next) {
    int start, end;
    const int b = kv_sequence(c, t, start, end);
    next = t + 1;
    if (b < 0) continue;
    const int pos = kv_context(c, b) - (end - t);   // may be negative
    next = t + (16 - (pos & 15)) < end ? t + (16 - (pos & 15)) : end;   // the next block's or sequence's first row
    if (t != start && (pos & 15) != 0) continue;
    const int left = end - t, first = pos & 15, count = left < 16 - first ? left : 16 - first;
    const int page = kv_page(c, b, pos);   // also of the others: a block does not cross pages (nor position 0)
    const float s = page < 0 ? 0.f : (side ? c.vs : c.ks)[int64_t(page) * c.Hkv + head];
    const uint8_t* base = (side ? c.v : c.k) + kv_page_offset<D>(c, page < 0 ? 0 : page, head) +
                          ((pos & ((1 << c.pshift) - 1)) >> 4) * 16 * D + lane * 16;
    uint16_t* out = a.dst[side] + (int64_t(t) * c.Hkv + head) * D;   // of the block's first row
    const int64_t stride = int64_t(c.Hkv) * D;
#pragma unroll
    for (int k = 0; k < D / 64; ++k) {
      kv_u4 w = *reinterpret_cast<const kv_u4*>(base + k * 1024);
      uint16_t h[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) h[e] = page < 0 ? 0 : f2h(float(int((w[e >> 2] >> (8 * (e & 3))) & 255u) - 128) * s);
      if (side == 0) {
        if (m >= first && m < first + count) {
          __builtin_memcpy(out + (m - first) * stride + 64 * k + 8 * q, h, 16);
          __builtin_memcpy(out + (m - first) * stride + 64 * k + 32 + 8 * q, h + 8, 16);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) tile[wave][4 * q + (e & 3)][16 * (e >> 2) + m] = h[e];
        // the same wavefront's LDS operations happen in order
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int tok = 8 * r + (lane >> 3), d = (lane & 7) * 8;
          uint16_t v[8];
          __builtin_memcpy(v, &tile[wave][tok][d], 16);
          if (tok >= first && tok < first + count) __builtin_memcpy(out + (tok - first) * stride + 64 * k + d, v, 16);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
      }
    }
  }
}

// Rows per window. A window does its sequences and pages one after another, `each` us a sequence; one that holds no first row
// of either still has to find that out, `idle` us of the call for each row and windows of one. Batches of nearly only single
// tokens: one row (append of 32 x 1, 8 heads: 7.8 us, 34 with 8 rows). Many rows: a page's or block's (8192 rows, 8 heads:
// 14 us, 61 with 8, 298 with 1). In between, the size that is best if every row is a sequence of its own: append of 2048 rows,
// 8 heads, as one sequence 8.6 us with a page's 64, 33 with 4, 79 with 1; as 32 sequences 8.6, 34 and 85; as one of 2000 and
// 31 single tokens 129, 29 and 38; reading them back with 16, 4 and 1 rows 9.0, 10.1 and 22; 8.9, 10.4 and 23; 32, 15 and 13
// (2 rows 16: sizes go up by `by`).
static int rows_per_window(const Kv8Args& c, int most, int by, double each, double idle) {
  if (c.T <= 4 * c.B) return 1;
  if (int64_t(c.T) * c.Hkv > 16384) return most;
  int best = 1;
  double least = 0;
  for (int span = 1; span <= most; span *= by) {
    const double us = each * (span < c.B ? span : c.B) + idle * c.T / span;
    if (span == 1 || us < least) {
      best = span;
      least = us;
    }
  }
  return best;
}

// Two heads a workgroup where windows are long: four prompts of 301 to 2000 tokens, 40 heads, 44 us; 49 with one, 47.5 with four.
template <int D>
void append_launch(const Kv8AppendArgs& a, hipStream_t stream) {
  const int span = rows_per_window(a.c, 1 << a.c.pshift, 2, 4.0, a.c.Hkv / 225.0), heads = span > 1 ? 2 : 1;
  const dim3 grid(unsigned(ceil_div(a.c.T, span)), unsigned(ceil_div(a.c.Hkv, heads)), 2);
  hipLaunchKernelGGL(k_kv8_append<D>, grid, dim3(256), 0, stream, a, span, heads);
}

template <int D>
void read_launch(const Kv8ReadArgs& a, hipStream_t stream) {
  const int quads = int(ceil_div(a.c.Hkv, 4)), span = rows_per_window(a.c, 16, 4, 1.8, quads / 500.0);
  const dim3 grid(unsigned(ceil_div(a.c.T, span)), unsigned(quads), 2);
  hipLaunchKernelGGL(k_kv8_read<D>, grid, dim3(256), 0, stream, a, span);
}

}  // namespace

fluxbin_status launch_kv8_append(const Kv8AppendArgs& a, int D, hipStream_t stream) {
  if (D == 64)
    append_launch<64>(a, stream);
  else if (D == 128)
    append_launch<128>(a, stream);
  else
    append_launch<256>(a, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the cache append");
}

fluxbin_status launch_kv8_read(const Kv8ReadArgs& a, int D, hipStream_t stream) {
  if (D == 64)
    read_launch<64>(a, stream);
  else if (D == 128)
    read_launch<128>(a, stream);
  else
    read_launch<256>(a, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the cache read");
}

}  // namespace fluxbin
