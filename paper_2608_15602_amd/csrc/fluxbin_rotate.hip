// Norm of each head and rotation by position, queries and keys in one pass.
//
//   y = x * rsqrt(mean(x^2) + eps) * w,   (a, b) -> (a c - b s, a s + b c),   c, s of the angle position * frequency[i].
//
// A lane holds 16 elements of a head in two pieces of 8: elements 8 j .. and R / 2 + 8 j .. of the rotated ones, so that both
// elements of a pair are in one lane, whichever they are, and neighbouring lanes' requests of 16 bytes lie side by side. Elements
// from R on go to the lanes behind in the same way. (A lane's pieces in a row, for neighbouring pairs and elements from R on: 16384
// rows of 40 heads of 128 and 256, half of each rotated, 65 and 129 us instead of 62 and 115.) The mean is a sum over the lanes of
// a head. Cosines and sines are those of a row for all of its heads: a workgroup makes them once, in LDS, while its
// elements are on their way. An angle is far past 2 pi at far positions (2^20 radians leave an fp32 angle 2^-4): the product is
// formed in fp64, exact up to position 2^29, and brought to half a turn there.
//
// Bound by memory: 8192 rows of 64 + 8 heads of 128 from fused rows 54 us, 5.55 TB/s (a 1 GiB copy: 5.13 TB/s). Two, four and
// eight pieces a lane took 61.8, 63.1 and 65.8 us where one took 60.7 (all with ordinary requests); one kernel for both sides that picks
// strides and weights by lane 75.6. A single row takes 2.9 us under the profiler, of which most is the chain of requests.
#include "fluxbin_device.h"
#include "fluxbin_serve_internal.h"

namespace fluxbin {

namespace {

typedef float rot_f4 __attribute__((ext_vector_type(4)));
typedef unsigned int rot_u4 __attribute__((ext_vector_type(4), aligned(2)));   // eight elements, at any element's address

// Workgroup: 256 lanes' pieces of the heads of rows in order, of the queries or (blocks from q_blocks on) of the keys. LDS: D
// floats for each row (16 for each of a head's lanes: four of cosines, sines, as [4][lanes][4], without bank conflicts), then the
// weight in the same order. STREAM: past the caches' ordinary order.
template <int D, bool INTER, bool STREAM>
__global__ void __launch_bounds__(256) k_qk_rotate(RotateArgs a, uint32_t q_blocks) {
  constexpr int L = D / 16;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const bool keys = blockIdx.x >= q_blocks;
  const RotateSide s = keys ? a.side[1] : a.side[0];
  const int tid = int(threadIdx.x), j = tid & (L - 1), H = keys ? a.H - a.Hq : a.Hq, half = a.R / 2;
  const uint32_t hl = uint32_t(H) * L;
  const int64_t u0 = int64_t(blockIdx.x - (keys ? q_blocks : 0)) * 256, total = a.rows * hl;
  const int64_t r0 = u0 / hl;
  const uint32_t off = uint32_t(u0 - r0 * hl), units = total - u0 < 256 ? uint32_t(total - u0) : 256;
  const int rows = int((off + units - 1) / hl) + 1;   // from r0 on
  float* weight = lds + rows * D;
  const bool rot = j < a.R / 16;
  const auto piece = [&](int lane, int second) __attribute__((always_inline)) {   // the first element of a lane's pieces
    const int rl = a.R / 16;
    return lane < rl ? 8 * lane + second * half : a.R + 8 * (lane - rl) + second * ((D - a.R) / 2);
  };
  const int c0 = piece(j, 0), c1 = piece(j, 1);

  const uint32_t at = off + (tid < int(units) ? tid : 0);   // past the end: the first again, not stored
  const uint32_t row = at / hl, head = (at - row * hl) / L;
  const uint16_t* src = s.src + (r0 + row) * s.ts + int64_t(head) * s.hs;
  const rot_u4* from[2] = {reinterpret_cast<const rot_u4*>(src + c0), reinterpret_cast<const rot_u4*>(src + c1)};
  rot_u4 x[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) x[p] = STREAM ? __builtin_nontemporal_load(from[p]) : *from[p];
  for (int t = tid; t < rows * half; t += 256) {
    const int r = t / half, f = t - r * half;
    const double angle = double(a.positions[r0 + r]) * double(a.freq[f]);
    const double turns = angle * 0.15915494309189533577;   // 1 / (2 pi)
    float sn, cs;
    sincospif(2.f * float(turns - __builtin_rint(turns)), &sn, &cs);
    // the lane's four pairs of its first piece and of its second, or of the first half of its pieces and of the second
    const int second = INTER ? 2 * f >= half : (f >> 2) & 1, lane = INTER ? (f - second * (half / 2)) >> 2 : f >> 3;
    float* to = lds + r * D + lane * 4 + (f & 3) + second * 4 * L;
    to[0] = cs * a.magnitude;
    to[8 * L] = sn * a.magnitude;
  }
  if (s.weight && tid < D) {
    const int part = tid / (4 * L), lane = (tid / 4) % L;   // four elements of a lane
    weight[tid] = s.weight[piece(lane, part >> 1) + (part & 1) * 4 + (tid & 3)];
  }
  __syncthreads();
  float y[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) y[e] = h2f(uint16_t(x[e >> 3][(e & 7) >> 1] >> (16 * (e & 1))));
  if (s.weight) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) sum = __builtin_fmaf(y[e], y[e], sum);
#pragma unroll
    for (int o = 1; o < L; o <<= 1) sum += __shfl_xor(sum, o);
    const float inv = rsqrtf(__builtin_fmaf(sum, 1.f / D, a.eps));
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const rot_f4 w = *reinterpret_cast<const rot_f4*>(weight + (p * L + j) * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[4 * p + e] = y[4 * p + e] * inv * w[e];
    }
  }
  if (rot) {
    const float* t = lds + row * D + j * 4;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const rot_f4 c = *reinterpret_cast<const rot_f4*>(t + p * 4 * L), sn = *reinterpret_cast<const rot_f4*>(t + (2 + p) * 4 * L);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int f = 4 * p + e;   // pair of this lane
        float& u = y[INTER ? 2 * f : f];
        float& v = y[INTER ? 2 * f + 1 : 8 + f];
        const float was = u;
        u = was * c[e] - v * sn[e];
        v = was * sn[e] + v * c[e];
      }
    }
  }
  if (tid >= int(units)) return;
  uint16_t h[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) h[e] = f2h(y[e]);
  __builtin_memcpy(x, h, 32);
  uint16_t* dst = s.dst + (r0 + row) * s.ots + int64_t(head) * s.ohs;
  rot_u4* to[2] = {reinterpret_cast<rot_u4*>(dst + c0), reinterpret_cast<rot_u4*>(dst + c1)};
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    if (STREAM)
      __builtin_nontemporal_store(x[p], to[p]);
    else
      *to[p] = x[p];
  }
}

template <int D, bool INTER>
void rotate_launch(const RotateArgs& a, hipStream_t stream) {
  constexpr int L = D / 16;
  const int64_t heads[2] = {a.Hq, a.H - a.Hq};
  int64_t blocks[2], most = 1;
  for (int i = 0; i < 2; ++i) {
    blocks[i] = ceil_div(a.rows * heads[i] * L, 256);
    const int64_t rows = heads[i] > 0 ? 254 / (heads[i] * L) + 2 : 0;   // that a workgroup's lanes can touch
    most = rows > most ? rows : most;
  }
  if (most > a.rows) most = a.rows;
  const unsigned bytes = unsigned((most + 1) * D * 4);
  const dim3 grid(unsigned(blocks[0] + blocks[1]));
  // Outputs that the L2 caches (32 MB) do not hold until they are read: 8192 rows as above 60.7 us without streaming.
  if (a.rows * a.H * D * 2 > (int64_t(32) << 20))
    hipLaunchKernelGGL((k_qk_rotate<D, INTER, true>), grid, dim3(256), bytes, stream, a, uint32_t(blocks[0]));
  else
    hipLaunchKernelGGL((k_qk_rotate<D, INTER, false>), grid, dim3(256), bytes, stream, a, uint32_t(blocks[0]));
}

template <int D>
void rotate_any(const RotateArgs& a, int interleaved, hipStream_t stream) {
  if (interleaved)
    rotate_launch<D, true>(a, stream);
  else
    rotate_launch<D, false>(a, stream);
}

}  // namespace

fluxbin_status launch_qk_rotate(const RotateArgs& a, int D, int interleaved, hipStream_t stream) {
  if (D == 64)
    rotate_any<64>(a, interleaved, stream);
  else if (D == 128)
    rotate_any<128>(a, interleaved, stream);
  else
    rotate_any<256>(a, interleaved, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the rotation");
}

}  // namespace fluxbin
