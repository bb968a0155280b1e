// Masks and positions of the nodes of drafted trees, from their parents.
//
// A node's mask is its own bit and its parent's mask. Whatever the tree's shape, after k rounds in which every node adds the mask
// of the node that it points to and then points to where that one points, it has its 2^k - 1 nearest ancestors: a chain of 1024
// nodes takes ten rounds (one ancestor after another, a request to LDS each, 50 us by count). Bound by the call: 24 nodes take
// 1.7 us under the profiler.
#include "fluxbin_device.h"
#include "fluxbin_serve_internal.h"

namespace fluxbin {

namespace {

// Workgroup: a sequence; thread: a node, whose mask is W words or fewer.
template <int W>
__global__ void __launch_bounds__(64 * W) k_tree_masks(MasksArgs a) {
  __shared__ uint64_t mask[W][64 * W];
  __shared__ int up[64 * W];
  const int b = int(blockIdx.x), o0 = a.offsets[b], o1 = a.offsets[b + 1], i = int(threadIdx.x);
  if (o0 < 0 || o1 > a.T || o1 <= o0 || o1 - o0 > 64 * a.words) return;
  const int n = o1 - o0, ctx = a.context[b];
  int p = i < n ? a.parents[o0 + i] : -1;
  if (p >= i) p = -1;   // a node follows its parent
  uint64_t m[W];
#pragma unroll
  for (int w = 0; w < W; ++w) m[w] = i >> 6 == w ? uint64_t(1) << (i & 63) : 0;
  while (__syncthreads_or(p >= 0)) {
#pragma unroll
    for (int w = 0; w < W; ++w) mask[w][i] = m[w];
    up[i] = p;
    __syncthreads();
    if (p >= 0) {
#pragma unroll
      for (int w = 0; w < W; ++w) m[w] |= mask[w][p];
      p = up[p];
    }
  }
  if (i >= n) return;
  int count = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w < a.words) a.masks[int64_t(o0 + i) * a.words + w] = m[w];
    count += __popcll((unsigned long long)m[w]);
  }
  if (a.positions) a.positions[o0 + i] = (ctx < 0 ? 0 : ctx > (1 << 30) ? 1 << 30 : ctx) - n + count - 1;
}

template <int W>
void masks_launch(const MasksArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(k_tree_masks<W>, dim3(unsigned(a.B)), dim3(64 * W), 0, stream, a);
}

}  // namespace

fluxbin_status launch_tree_masks(const MasksArgs& a, hipStream_t stream) {
  static_assert(kTreeMaxWords == 16, "a thread for each node");
  if (a.words == 1)
    masks_launch<1>(a, stream);
  else if (a.words == 2)
    masks_launch<2>(a, stream);
  else if (a.words <= 4)
    masks_launch<4>(a, stream);
  else if (a.words <= 8)
    masks_launch<8>(a, stream);
  else
    masks_launch<16>(a, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the tree's masks");
}

}  // namespace fluxbin
