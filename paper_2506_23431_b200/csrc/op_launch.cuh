// Launch of the operators around the 8-bit cache: one after the other on a step's rows, a few microseconds each.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "pd.h"

namespace pd {

// Whether every address (null ones among them) is a multiple of n.
template <typename... P>
bool aligned_to(uintptr_t n, P... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) % n) == 0; }

// Everything enqueued before is complete and visible behind this; the kernel's first instruction.  What follows it in the stream may then be brought
// onto the SMs while the kernel runs, up to its own wait: 1.3 to 2.2 us per launch between two of these operators in a stream (a step's three 13.4 us, without 18.5); in a
// graph, whose launches are as close by themselves, nothing (12.9 and 12.8).
__device__ __forceinline__ void op_begin() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// A launch that may be brought onto the SMs ahead of the end of the one before it, whatever that is; `cluster` CTAs along x.
template <typename... P, typename... A>
cudaError_t op_launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t s, A... args) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// What an entry point returns.  A refused launch is the caller's to handle by that alone: CUDA's own note of it would come up in the next check anyone makes.
inline pd_status op_status(cudaError_t st) {
  if (st == cudaSuccess) return PD_OK;
  cudaGetLastError();
  return PD_ERR_CUDA;
}

}  // namespace pd
