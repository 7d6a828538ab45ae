// Programmatic dependent launch: a kernel's start (its CTAs' arrival on the SMs, barriers, tensor memory, descriptors) overlaps
// the end of the kernel before it in the stream.
#pragma once
#include <cuda_runtime.h>

namespace hdet {

// In a kernel: lets the next kernel of the stream start its prologue now, and waits until the kernels before this one are done
// and their writes visible.  Every kernel that is launched below waits before it touches global memory.  Neither does
// anything in a launch without the attribute.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Launches a kernel with that attribute, in clusters of `cluster` CTAs.
template <typename... Params, typename... Args>
cudaError_t launch(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

}  // namespace hdet
