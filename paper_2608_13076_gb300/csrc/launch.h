// launch.h -- kernel launches with programmatic dependent launch.
#pragma once
#include <cuda_runtime.h>

namespace spade {

// `grid` CTAs of `kern` in clusters of `cluster` (1: none).  The kernel may be scheduled
// while the one before it in the stream still runs: it waits (griddep_wait) before it
// reads or writes anything of the caller's, and reads it by plain loads (a read-only one
// promises that nothing writes its data while the kernel lives).
template <class... A>
static cudaError_t launch(void (*kern)(A...), dim3 grid, unsigned cluster, unsigned threads, size_t smem, cudaStream_t s,
                          A... a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, a...);
}

}  // namespace spade
