// bf_launches.cuh -- launches of the learning kernels.  Where a call has several
// kernels, each but the first may start before the one ahead of it ends: it
// waits for that one (and so for all before) where it first reads what they
// wrote, or writes what they read.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace bfk {

// What the call's kernels ahead wrote is visible from here on.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The call's next kernel may start.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename K, typename... Args>
cudaError_t launch_shared(K kernel, uint64_t blocks, uint32_t threads, uint32_t cluster, bool follows, uint64_t shared,
                          cudaStream_t st, const Args&... args) {
  if (blocks > 0x7FFFFFFFu) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((uint32_t)blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = shared;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  cfg.attrs = attr;
  if (follows) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = cluster;
    attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename K, typename... Args>
cudaError_t launch_shaped(K kernel, uint64_t blocks, uint32_t threads, uint32_t cluster, bool follows, cudaStream_t st,
                          const Args&... args) {
  return launch_shared(kernel, blocks, threads, cluster, follows, 0, st, args...);
}

template <typename K, typename... Args>
cudaError_t launch_plain(K kernel, uint64_t blocks, uint32_t threads, cudaStream_t st, const Args&... args) {
  return launch_shaped(kernel, blocks, threads, 1, false, st, args...);
}
// A kernel behind another one of the same call.
template <typename K, typename... Args>
cudaError_t launch_after(K kernel, uint64_t blocks, uint32_t threads, cudaStream_t st, const Args&... args) {
  return launch_shaped(kernel, blocks, threads, 1, true, st, args...);
}

}  // namespace bfk
