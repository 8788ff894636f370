// How the kernels around the attention find a token's segment, and how a cluster of blocks is launched.
#pragma once
#include "pp_internal.h"
#include "pp_ptx.cuh"

namespace pp {

// Largest i in [0, n) with start[i] <= t, for ascending `start` with start[0] <= t < start[n].  By a whole
// warp, 32 probes a step: two dependent loads for a thousand entries, which hit L1 after a block's first.
__device__ __forceinline__ int warp_upper(const int32_t* start, int n, int t) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) >> 5;
    const int at = lo + step * (lane + 1);
    const bool below = at < hi && start[at] <= t;
    lo += step * __popc(__ballot_sync(0xffffffffu, below));
    hi = min(hi, lo + step);
  }
  return lo;
}

// The same by one thread.
__device__ __forceinline__ int thread_upper(const int32_t* start, int n, int t) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// launch_kernel with overlap, for blocks in clusters of `cluster`.
template <typename... P, typename... A>
cudaError_t launch_clusters(int cluster, void (*kern)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream,
                            A&&... args) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(cluster);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}

}  // namespace pp
