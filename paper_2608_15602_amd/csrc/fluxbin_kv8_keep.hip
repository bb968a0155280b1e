// Accepted rows of the paged 8-bit cache moved together.
//
// Row indices rise, so that the k-th kept row, which goes to place k, comes from place k or behind it. Pages are filled in order,
// and a page's rows come from it or from pages behind it, of which none has been written yet: reading all of a page's rows
// before the first is written is enough. Bound by the chain of requests (the sequence, its list, pages, scales, codes): one path of
// a tree of 16 nodes, 32 heads, 4.4 us; 64 paths of trees of 10 to 200 nodes, 8 heads, 7 us.
#include "fluxbin_kv8_device.h"
#include "fluxbin_serve_internal.h"

namespace fluxbin {

namespace {

// Four codes brought to another scale.
__device__ __forceinline__ uint32_t kv_recode4(uint32_t w, float ratio) {
  if (ratio == 1.f) return w;
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) r |= kv_recode((w >> (8 * i)) & 255u, ratio) << (8 * i);
  return r;
}

// Workgroup (sequence, head, side): its pages one after another. A page's moved rows go through LDS as rows of codes, brought
// to the page's new scale, and from there into its 16-byte units; those of earlier tokens are rewritten where the scale grows.
template <int D, int W>
__global__ void __launch_bounds__(W) k_kv8_keep(Kv8KeepArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t slab[];   // [rows of a page][D]
  __shared__ int64_t unit[W];      // of a row: the offset of its block of 16 tokens in the codes, plus its place there
  __shared__ float ratios[W];
  __shared__ float red[W / 64];
  __shared__ int moved;
  const Kv8Args& c = a.c;
  const int tid = int(threadIdx.x), b = int(blockIdx.x), head = int(blockIdx.y), side = int(blockIdx.z), P = 1 << c.pshift;
  const int o0 = c.offsets[b], o1 = c.offsets[b + 1];
  if (o0 < 0 || o1 > c.T || o1 <= o0) return;
  const int n = o1 - o0, base = kv_context(c, b) - n;
  int m = a.kept[b];
  m = m < 0 ? 0 : m > n ? n : m;
  // the first row that is not in its place
  if (tid == 0) moved = m;
  __syncthreads();
  for (int k0 = 0; k0 < m; k0 += W) {
    const int k = k0 + tid;
    if (k < m && a.keep[o0 + k] != k) atomicMin(&moved, k);
    __syncthreads();
    const bool found = moved < m;
    __syncthreads();   // before the next rows change it
    if (found) break;
  }
  uint8_t* codes = side ? c.v : c.k;
  float* scales = side ? c.vs : c.ks;
  for (int k = moved; k < m;) {
    const int pos = base + k;
    if (pos < 0) {
      k = -base;
      continue;
    }
    const int first = pos & (P - 1), count = m - k < P - first ? m - k : P - first, last = first + count;
    const int page = kv_page(c, b, pos);
    if (page < 0) {
      k += count;
      continue;
    }
    float* at = scales + int64_t(page) * c.Hkv + head;
    const float old = first > 0 ? *at : 0.f;
    float s_row = 0.f;
    int64_t u = -1;
    if (tid < count) {
      const int i = a.keep[o0 + k + tid];
      const int of = i >= k + tid && i < n ? base + i : -1, src = kv_page(c, b, of);
      if (src >= 0) {
        s_row = scales[int64_t(src) * c.Hkv + head];
        u = kv_page_offset<D>(c, src, head) + int64_t(of & (P - 1)) * D;   // 16 D a block, D a place
      }
    }
    float s = s_row;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) s = fmaxf(s, __shfl_xor(s, o));
    __syncthreads();   // what the page before left in LDS has been used
    if ((tid & 63) == 0) red[tid >> 6] = s;
    __syncthreads();
    s = old;
#pragma unroll
    for (int w = 0; w < W / 64; ++w) s = fmaxf(s, red[w]);
    if (tid < count) {
      unit[tid] = u;
      ratios[tid] = s_row < s ? s_row / s : 1.f;
    }
    const float grow = old < s ? old / s : 1.f;
    if (tid == 0) *at = s;   // everyone has read the old one: two barriers ago
    __syncthreads();
    if (side == 0) {
      for (int e = tid; e < count * (D / 16); e += W) {   // a row's unit: 8 elements from 8 q on, 8 from 32 + 8 q on
        const int t = e / (D / 16), blk = e % (D / 16) / 4, q = e % 4;
        const int64_t o = unit[t];
        kv_u4 w = {kKvZero, kKvZero, kKvZero, kKvZero};
        if (o >= 0) {
          const int m16 = int(o / D) & 15;   // blocks are 16 D bytes
          w = *reinterpret_cast<const kv_u4*>(codes + (o - int64_t(m16) * D) + blk * 1024 + (q * 16 + m16) * 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<uint32_t*>(&slab[t * D + 64 * blk + 32 * (i >> 1) + 8 * q + 4 * (i & 1)]) = kv_recode4(w[i], ratios[t]);
      }
    } else {
      for (int e = tid; e < count * (D / 4); e += W) {   // a unit: elements 16 t + m of four rows
        const int t = e / (D / 4), blk = e % (D / 4) / 16, m16 = e % 16;
        const int64_t o = unit[t];
        kv_u4 w = {kKvZero, kKvZero, kKvZero, kKvZero};
        int shift = 0;
        if (o >= 0) {
          const int place = int(o / D) & 15;
          shift = 8 * (place & 3);
          w = *reinterpret_cast<const kv_u4*>(codes + (o - int64_t(place) * D) + blk * 1024 + ((place >> 2) * 16 + m16) * 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t byte = (w[i] >> shift) & 255u;
          slab[t * D + 64 * blk + 16 * i + m16] = uint8_t(ratios[t] == 1.f ? byte : kv_recode(byte, ratios[t]));
        }
      }
    }
    __syncthreads();
    uint8_t* to = codes + kv_page_offset<D>(c, page, head);
    for (int e = (grow != 1.f ? 0 : first >> 4) * D + tid; e < ((last + 15) >> 4) * D; e += W) {   // D units a block
      const int lane = e & 63, blk = (e >> 6) % (D / 64), tb = (e >> 6) / (D / 64), m16 = lane & 15, q = lane >> 4;
      const int t0 = 16 * tb + (side ? 4 * q : m16), t1 = t0 + (side ? 4 : 1);   // the unit's tokens
      const bool fresh = t1 > first && t0 < last;
      if (!fresh && (t0 >= first || grow == 1.f)) continue;
      kv_u4 w = {kKvZero, kKvZero, kKvZero, kKvZero};
      if (t0 < first) {
        w = *reinterpret_cast<const kv_u4*>(to + int64_t(e) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = kv_recode4(w[i], grow);
      }
      if (fresh && side == 0) {
        const uint8_t* p = &slab[(t0 - first) * D + 64 * blk + 8 * q];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const uint32_t*>(p + 32 * (i >> 1) + 4 * (i & 1));
      } else if (fresh) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = t0 + i;
          if (t < first || t >= last) continue;
#pragma unroll
          for (int dt = 0; dt < 4; ++dt)
            w[dt] = (w[dt] & ~(255u << (8 * i))) | (uint32_t(slab[(t - first) * D + 64 * blk + 16 * dt + m16]) << (8 * i));
        }
      }
      *reinterpret_cast<kv_u4*>(to + int64_t(e) * 16) = w;
    }
    k += count;
  }
}

// Threads: at least a page's rows. 128 where there are more workgroups than 256 threads leave room for at a time (8 a CU): 256
// sequences that keep 8 rows of 64, 8 and 32 heads, 7.9 and 25.2 us, 10.8 and 36.2 with 256; 64 that keep 40, 8 and 32 heads, 9.6 and
// 18.3, and 8.6 and 20.8 with 256 (64 threads 13.1 and 21.0).
template <int D>
void keep_launch(const Kv8KeepArgs& a, int cus, hipStream_t stream) {
  const int P = 1 << a.c.pshift, rows = a.c.T < P ? a.c.T : P;
  const dim3 grid(unsigned(a.c.B), unsigned(a.c.Hkv), 2);
  if (P <= 128 && int64_t(a.c.B) * a.c.Hkv * 2 > 8 * cus)
    hipLaunchKernelGGL((k_kv8_keep<D, 128>), grid, dim3(128), unsigned(rows * D), stream, a);
  else
    hipLaunchKernelGGL((k_kv8_keep<D, 256>), grid, dim3(256), unsigned(rows * D), stream, a);
}

}  // namespace

fluxbin_status launch_kv8_keep(const Kv8KeepArgs& a, int D, int cus, hipStream_t stream) {
  if (D == 64)
    keep_launch<64>(a, cus, stream);
  else if (D == 128)
    keep_launch<128>(a, cus, stream);
  else
    keep_launch<256>(a, cus, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the cache's moves");
}

}  // namespace fluxbin
