// Norm of each head and rotation by position, queries and keys in one pass.
//
//   y = x * rsqrt(mean(x^2) + eps) * w,   (a, b) -> (a c - b s, a s + b c),   c, s of the angle position * frequency[i].
//
// A lane holds 16 elements of a head in two pieces of 8: elements 8 j .. and R / 2 + 8 j .. of the rotated ones (2 x 8 in a row
// where pairs are neighbours), so that both elements of a pair are in one lane, requests are 16 bytes and the D / 16 lanes of a
// head cover it without gaps. Elements from R on go to the lanes behind in pieces of 8 as well. The mean is a sum over the
// lanes of a head. Cosines and sines are those of a row for all of its heads: a workgroup makes them once, in LDS, while its
// elements are on their way. An angle is far past 2 pi at far positions (2^20 radians leave an fp32 angle 2^-4): the product is
// formed in fp64, where it is exact, and brought to half a turn there.
#include "fluxbin_device.h"
#include "fluxbin_serve_internal.h"

namespace fluxbin {

namespace {

typedef float rot_f4 __attribute__((ext_vector_type(4)));

// Workgroup: U * 256 lanes' pieces in a row, of the heads of rows in order. LDS: D floats for each row (16 for each of a head's
// lanes: four of cosines, sines, as [4][lanes][4], without bank conflicts), then both weights in the same order.
template <int D, int U, bool INTER>
__global__ void __launch_bounds__(256) k_qk_rotate(RotateArgs a) {
  constexpr int L = D / 16;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int tid = int(threadIdx.x), j = tid & (L - 1), hl = a.H * L, half = a.R / 2;
  const int64_t u0 = int64_t(blockIdx.x) * (256 * U), total = a.rows * hl;
  const int64_t r0 = u0 / hl;
  const int off = int(u0 - r0 * hl);
  const int last = int((total - u0 < 256 * U ? total - u0 : 256 * U) + off - 1) / hl;   // row of the last lane, from r0
  float* weights = lds + (last + 1) * D;
  const bool rot = j < a.R / 16;
  const int c0 = rot ? (INTER ? 16 * j : 8 * j) : 16 * j, c1 = rot && !INTER ? half + 8 * j : c0 + 8;

  uint16_t x[U][16];
  int row[U], head[U];
  bool has[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int at = off + 256 * i + tid;
    has[i] = u0 + 256 * i + tid < total;
    row[i] = has[i] ? at / hl : 0;
    head[i] = has[i] ? (at - row[i] * hl) / L : 0;
    if (has[i]) {
      const bool k = head[i] >= a.Hq;
      const RotateSide& s = a.side[k];
      const uint16_t* p = s.src + (r0 + row[i]) * s.ts + (head[i] - (k ? a.Hq : 0)) * s.hs;
      __builtin_memcpy(&x[i][0], p + c0, 16);
      __builtin_memcpy(&x[i][8], p + c1, 16);
    }
  }
  for (int t = tid; t < (last + 1) * half; t += 256) {
    const int r = t / half, f = t - r * half;
    const double angle = double(a.positions[r0 + r]) * double(a.freq[f]);
    const double turns = angle * 0.15915494309189533577;   // 1 / (2 pi)
    float sn, cs;
    sincospif(2.f * float(turns - __builtin_rint(turns)), &sn, &cs);
    float* to = lds + r * D + (f >> 3) * 4 + (f & 3) + ((f >> 2) & 1) * 4 * L;
    to[0] = cs * a.magnitude;
    to[8 * L] = sn * a.magnitude;
  }
  for (int t = tid; t < 2 * D; t += 256) {
    const float* w = a.side[t / D].weight;
    const int e = t % D, piece = e / (4 * L), lane = (e / 4) % L, in = (piece & 1) * 4 + (e & 3);
    const bool lr = lane < a.R / 16;
    const int d = (piece < 2 ? (lr && !INTER ? 8 * lane : 16 * lane) : (lr && !INTER ? half + 8 * lane : 16 * lane + 8)) + in;
    if (w) weights[t] = w[d];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < U; ++i) {
    float y[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = has[i] ? h2f(x[i][e]) : 0.f;
    const bool k = head[i] >= a.Hq;
    const RotateSide& s = a.side[k];
    if (s.weight) {   // the same for all lanes of a head
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) sum = __builtin_fmaf(y[e], y[e], sum);
#pragma unroll
      for (int o = 1; o < L; o <<= 1) sum += __shfl_xor(sum, o);
      const float inv = rsqrtf(__builtin_fmaf(sum, 1.f / D, a.eps));
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const rot_f4 w = *reinterpret_cast<const rot_f4*>(weights + (k ? D : 0) + (p * L + j) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[4 * p + e] = y[4 * p + e] * inv * w[e];
      }
    }
    if (rot) {
      const float* t = lds + row[i] * D + j * 4;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const rot_f4 c = *reinterpret_cast<const rot_f4*>(t + p * 4 * L), sn = *reinterpret_cast<const rot_f4*>(t + (2 + p) * 4 * L);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int f = 4 * p + e;   // pair of this lane
          float& u = y[INTER ? 2 * f : f];
          float& v = y[INTER ? 2 * f + 1 : 8 + f];
          const float u0f = u;
          u = u0f * c[e] - v * sn[e];
          v = u0f * sn[e] + v * c[e];
        }
      }
    }
    if (has[i]) {
      uint16_t h[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) h[e] = f2h(y[e]);
      uint16_t* p = s.dst + (r0 + row[i]) * s.ots + (head[i] - (k ? a.Hq : 0)) * s.ohs;
      __builtin_memcpy(p + c0, &h[0], 16);
      __builtin_memcpy(p + c1, &h[8], 16);
    }
  }
}

template <int D, int U>
void rotate_launch(const RotateArgs& a, int interleaved, hipStream_t stream) {
  constexpr int L = D / 16;
  const int64_t hl = int64_t(a.H) * L, blocks = ceil_div(a.rows * hl, 256 * U);
  int64_t most = (256 * U - 2) / hl + 2;   // rows that a workgroup's lanes can touch
  if (most > a.rows) most = a.rows;
  const unsigned bytes = unsigned((most + 2) * D * 4);
  if (interleaved)
    hipLaunchKernelGGL((k_qk_rotate<D, U, true>), dim3(unsigned(blocks)), dim3(256), bytes, stream, a);
  else
    hipLaunchKernelGGL((k_qk_rotate<D, U, false>), dim3(unsigned(blocks)), dim3(256), bytes, stream, a);
}

template <int D>
void rotate_any(const RotateArgs& a, int interleaved, int cus, hipStream_t stream) {
  // Two pieces a lane where a workgroup's rows then still fit 64 KB of LDS and there is work for all CUs.
  const int64_t lanes = a.rows * a.H * (D / 16);
  if (lanes >= int64_t(cus) * 256 * 8 && a.H >= 4)
    rotate_launch<D, 4>(a, interleaved, stream);
  else
    rotate_launch<D, 1>(a, interleaved, stream);
}

}  // namespace

fluxbin_status launch_qk_rotate(const RotateArgs& a, int D, int interleaved, int cus, hipStream_t stream) {
  if (D == 64)
    rotate_any<64>(a, interleaved, cus, stream);
  else if (D == 128)
    rotate_any<128>(a, interleaved, cus, stream);
  else
    rotate_any<256>(a, interleaved, cus, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the rotation");
}

}  // namespace fluxbin
