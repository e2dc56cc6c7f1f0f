// How the elementwise layer kernels walk over an array: a thread keeps its columns, so that a row costs it one addition of pointers.
#pragma once
#include "layer_common.cuh"

namespace aet {
namespace layer {

// A CTA of 256 threads: `lanes` of them (a power of two) side by side over groups of N columns, 256 / lanes rows at a time.
template <int N> __host__ __device__ inline uint32_t log_lanes(uint32_t cols) {
  uint32_t l = 0;
  while (l < 8 && ((uint64_t)N << l) < cols) ++l;
  return l;
}

}  // namespace layer
}  // namespace aet
