// Launches of one call that follow each other closely.
#pragma once

#include <cuda_runtime.h>

namespace mixlora {

// Lets a kernel use `bytes` of dynamic shared memory: asked of the runtime once per kernel and device.
template <typename K>
cudaError_t allow_smem(K kernel, int bytes, bool (&done)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev >= 0 && dev < 64 && done[dev])) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;      // a race only repeats the call
  return e;
}

// A kernel launched with launch_behind() may start, and set itself up, as soon as every block of the kernel before it has
// begun (let_next_start), and waits for that kernel's end and results with wait_for_last before it touches anything that
// the call's kernels share.  Saves 2 to 3 us a launch.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename... Params, typename... Args>
cudaError_t launch_behind_in_clusters(int cluster, void (*kernel)(Params...), unsigned grid, unsigned block, size_t smem,
                                      cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}
template <typename... Params, typename... Args>
cudaError_t launch_behind(void (*kernel)(Params...), unsigned grid, unsigned block, size_t smem, cudaStream_t st,
                          const Args&... args) {
  return launch_behind_in_clusters(1, kernel, grid, block, smem, st, args...);
}

}  // namespace mixlora
