// Launching a kernel before the one in front of it in the stream has ended (programmatic dependent launch): the steps of
// a decode loop are a few microseconds each, and the time from one kernel's end to the next one's start is a good part of
// it (decode attention on short caches, one call behind the other: 10.3 -> 8.9 us a call).
#pragma once
#include <cuda_runtime.h>

namespace ckv {

// Every kernel that is launched early calls this first: nothing but its own shared memory is touched before it, so
// that nothing is read before it is written and nothing overwritten before it is read.  Loads for data that is constant
// while a kernel runs (__ldg, ld.global.nc, what const __restrict__ pointers become) are not for these kernels: the one in
// front may still write while they are resident, and such a load is held behind the wait by nothing.
__device__ __forceinline__ void wait_for_previous_kernel() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// cluster: CTAs of a thread-block cluster (0, 1: none).
template <typename... P>
cudaError_t launch_early_in_clusters(void (*kernel)(P...), dim3 grid, int threads, int smem, int cluster, cudaStream_t st,
                                     P... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <typename... P>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, int threads, int smem, cudaStream_t st, P... args) {
  return launch_early_in_clusters<P...>(kernel, grid, threads, smem, 0, st, args...);
}

}  // namespace ckv
