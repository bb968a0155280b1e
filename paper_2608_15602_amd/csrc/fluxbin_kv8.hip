// Paged key/value cache in 8 bits: storing new tokens and reading them back.
#include "fluxbin_kv8_device.h"

namespace fluxbin {

namespace {

// A new element: NaN is stored as 0, an infinity as the largest fp16.
__device__ __forceinline__ float kv_value(uint16_t h) {
  const float v = h2f(h);
  return v == v ? fminf(fmaxf(v, -65504.f), 65504.f) : 0.f;
}

__device__ __forceinline__ uint32_t kv_code(float v, float inv) {
  return uint32_t(int(fminf(fmaxf(__builtin_rintf(v * inv), -127.f), 127.f)) + 128);
}

// An earlier token's code after its page's scale has grown.
__device__ __forceinline__ uint32_t kv_recode(uint32_t byte, float ratio) {
  return uint32_t(int(__builtin_rintf(float(int(byte) - 128) * ratio)) + 128);
}

// One page and head's new tokens, keys (SIDE 0) or values (SIDE 1), by a whole workgroup: the largest new magnitude, the
// scale, then every 16-byte unit of the page that holds a new token or, where the scale grows, an earlier one.
template <int D, int SIDE>
__device__ void kv_store_page(const Kv8AppendArgs& a, int page, int head, int row, int first, int count, float* red) {
  const Kv8Args& c = a.c;
  const uint16_t* src = a.src[SIDE] + int64_t(row) * a.ts[SIDE] + int64_t(head) * a.hs[SIDE];
  float amax = 0.f;
  for (int e = int(threadIdx.x); e < count * (D / 8); e += 256) {
    uint16_t h[8];
    __builtin_memcpy(h, src + int64_t(e / (D / 8)) * a.ts[SIDE] + (e % (D / 8)) * 8, 16);
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(kv_value(h[i])));
  }
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
  const int b0 = s > old ? 0 : first >> 4, b1 = (last + 15) >> 4;   // blocks of 16 tokens
  for (int u = b0 * D + int(threadIdx.x); u < b1 * (D / 64) * 64; u += 256) {
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
        const uint16_t* p = src + int64_t(t0 - first) * a.ts[0] + 64 * blk + 8 * q;
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          uint16_t h[8];
          __builtin_memcpy(h, p + 32 * f, 16);
#pragma unroll
          for (int e = 0; e < 8; e += 4)
            w[2 * f + e / 4] = kv_code(kv_value(h[e]), inv) | kv_code(kv_value(h[e + 1]), inv) << 8 |
                               kv_code(kv_value(h[e + 2]), inv) << 16 | kv_code(kv_value(h[e + 3]), inv) << 24;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = t0 + i;
          if (t < first) continue;
#pragma unroll
          for (int dt = 0; dt < 4; ++dt) {
            const uint32_t r =
                t < last ? kv_code(kv_value(src[int64_t(t - first) * a.ts[1] + 64 * blk + 16 * dt + m]), inv) : 128u;
            w[dt] = (w[dt] & ~(255u << (8 * i))) | (r << (8 * i));
          }
        }
      }
    }
    *reinterpret_cast<kv_u4*>(base + int64_t(u) * 16) = w;
  }
}

// Workgroup (window of `span` rows, head, side): the rows of its window that are the first of their sequence or of their
// page start a page's new tokens.
template <int D>
__global__ void __launch_bounds__(256) k_kv8_append(Kv8AppendArgs a, int span) {
  __shared__ float red[5];
  const Kv8Args& c = a.c;
  const int P = 1 << c.pshift;
  for (int i = 0; i < span; ++i) {
    const int t = int(blockIdx.x) * span + i;
    if (t >= c.T) return;
    int start, end;
    const int b = kv_sequence(c, t, start, end);
    if (b < 0) continue;
    const int pos = kv_context(c, b) - (end - t);   // may be negative
    if (pos < 0 || (t != start && (pos & (P - 1)) != 0)) continue;
    const int page = kv_page(c, b, pos);
    if (page < 0) continue;
    const int first = pos & (P - 1), left = end - t, count = left < P - first ? left : P - first;
    __syncthreads();   // red of the page before
    if (blockIdx.z == 0)
      kv_store_page<D, 0>(a, page, int(blockIdx.y), t, first, count, red);
    else
      kv_store_page<D, 1>(a, page, int(blockIdx.y), t, first, count, red);
  }
}

// Workgroup (row, side): four wavefronts take the heads in turn, a lane 8 elements at a time.
template <int D>
__global__ void __launch_bounds__(256) k_kv8_read(Kv8ReadArgs a) {
  const Kv8Args& c = a.c;
  const int t = int(blockIdx.x), side = int(blockIdx.y);
  int start, end;
  const int b = kv_sequence(c, t, start, end);
  if (b < 0) return;
  const int pos = kv_context(c, b) - (end - t), page = kv_page(c, b, pos), slot = pos & ((1 << c.pshift) - 1);
  for (int e = int(threadIdx.x); e < c.Hkv * (D / 8); e += 256) {
    const int head = e / (D / 8), d = e % (D / 8) * 8;
    uint16_t h[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (page >= 0) {
      const float s = (side ? c.vs : c.ks)[int64_t(page) * c.Hkv + head];
      const uint8_t* p = (side ? c.v : c.k) + kv_page_offset<D>(c, page, head) + ((slot >> 4) * (D / 64) + (d >> 6)) * 1024;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int x = (d & 63) + i;
        const int at = side ? ((slot & 15) / 4 * 16 + (x & 15)) * 16 + (x >> 4) * 4 + (slot & 3)
                            : (((x & 31) >> 3) * 16 + (slot & 15)) * 16 + (x >> 5) * 8 + (x & 7);
        h[i] = f2h(float(int(p[at]) - 128) * s);
      }
    }
    __builtin_memcpy(a.dst[side] + (int64_t(t) * c.Hkv + head) * D + d, h, 16);
  }
}

template <int D>
void append_launch(const Kv8AppendArgs& a, hipStream_t stream) {
  const int P = 1 << a.c.pshift;
  const int span = a.c.T <= 4 * a.c.B ? 1 : P;   // mostly single tokens: a workgroup for each
  const dim3 grid(unsigned(ceil_div(a.c.T, span)), unsigned(a.c.Hkv), 2);
  hipLaunchKernelGGL(k_kv8_append<D>, grid, dim3(256), 0, stream, a, span);
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
  const dim3 grid(unsigned(a.c.T), 2), block(256);
  if (D == 64)
    hipLaunchKernelGGL(k_kv8_read<64>, grid, block, 0, stream, a);
  else if (D == 128)
    hipLaunchKernelGGL(k_kv8_read<128>, grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL(k_kv8_read<256>, grid, block, 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the cache read");
}

}  // namespace fluxbin
