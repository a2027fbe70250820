// Kernel launches with attributes.
#pragma once
#include <cuda_runtime.h>

namespace slim {

// Launches k on stream s; `cluster` > 1: in clusters of that many blocks;
// `after`: as a programmatic dependent of the stream's previous kernel, which k
// waits for itself (griddepcontrol.wait) before it touches what that one writes.
template <typename... Args>
bool launch_on(void (*k)(Args...), dim3 blocks, int threads, size_t smem, int cluster,
               bool after, cudaStream_t s, const Args&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = blocks;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  unsigned n = 0;
  if (cluster > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = cluster;
    at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
    ++n;
  }
  if (after) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = at;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, k, args...) == cudaSuccess;
}

}  // namespace slim
