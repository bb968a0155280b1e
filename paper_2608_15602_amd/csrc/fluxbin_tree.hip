// Masks and positions of the nodes of drafted trees, from their parents.
#include "fluxbin_device.h"
#include "fluxbin_serve_internal.h"

namespace fluxbin {

namespace {

// Workgroup: a sequence. A thread goes up from a node, for one word of its mask (the node's index falls at every step, so a
// word ends with the first ancestor below it); word 0's threads go all the way and count.
__global__ void __launch_bounds__(256) k_tree_masks(MasksArgs a) {
  __shared__ int16_t up[64 * kTreeMaxWords];
  const int b = int(blockIdx.x), o0 = a.offsets[b], o1 = a.offsets[b + 1];
  if (o0 < 0 || o1 > a.T || o1 <= o0 || o1 - o0 > 64 * a.words) return;
  const int n = o1 - o0;
  for (int i = int(threadIdx.x); i < n; i += 256) {
    const int p = a.parents[o0 + i];
    up[i] = int16_t(p >= 0 && p < i ? p : -1);
  }
  const int ctx = a.context[b], first = (ctx < 0 ? 0 : ctx > (1 << 30) ? 1 << 30 : ctx) - n;
  __syncthreads();
  for (int t = int(threadIdx.x); t < n * a.words; t += 256) {
    const int i = t / a.words, w = t - i * a.words;
    uint64_t bits = 0;
    int depth = -1;
    for (int at = i; at >= 64 * w; at = up[at]) {   // word 0: to the root's -1
      if (at < 64 * w + 64) bits |= uint64_t(1) << (at & 63);
      ++depth;
    }
    a.masks[int64_t(o0) * a.words + t] = bits;
    if (w == 0 && a.positions) a.positions[o0 + i] = first + depth;
  }
}

}  // namespace

fluxbin_status launch_tree_masks(const MasksArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(k_tree_masks, dim3(unsigned(a.B)), dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FLUXBIN_OK : hip_fail(e, "launching the tree's masks");
}

}  // namespace fluxbin
