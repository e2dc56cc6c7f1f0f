// Launches of the layer operators' kernels: the small ones may come up under the tail of the kernel in front of it (programmatic dependent launch) and
// wait on the device before they touch memory, which takes a launch's latency off every step of a chain of small kernels.
#pragma once
#include <cuda_runtime.h>

namespace aet {
namespace layer {

// cluster: CTAs of a cluster along x (1: none)
template <bool kEarly, class... P, class... A>
inline cudaError_t launch_as(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, unsigned cluster, cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = kEarly;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}
template <class... P, class... A>
inline cudaError_t launch(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, unsigned cluster, cudaStream_t s, const A&... args) {
  return launch_as<true>(kernel, grid, threads, smem, cluster, s, args...);
}
// A kernel that has the SMs to itself: behind the one in front, and nobody comes up beside it (with early launches on either side the fp32
// evaluation of 60,000 rows took 114 us instead of 106, a product of 1,003 x 785 x 1,017 17.9 instead of 15.9).
template <class... P, class... A>
inline cudaError_t launch_alone(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, unsigned cluster, cudaStream_t s, const A&... args) {
  return launch_as<false>(kernel, grid, threads, smem, cluster, s, args...);
}

#if defined(__CUDACC__)
// First thing of a kernel launched so, by every thread: the next kernel may come up; nothing of memory is touched before the one in front
// is done.
__device__ __forceinline__ void in_line() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
#endif

}  // namespace layer
}  // namespace aet
