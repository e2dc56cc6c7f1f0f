// Dropout whose mask is never stored: y = residual + drop(x), each element's sixteen random bits a function of where it stands.
//
// The counter-based generator costs some 22 integer instructions a draw of 64 bits; with four elements to a draw a bf16 array stays
// bound by memory (about 5.8 elements a cycle and SM at the copy rate, 22 issue slots each).  The gradient is the same call on dy.
#include <cuda_runtime.h>

#include "layer_common.cuh"

namespace aet {
namespace layer {
namespace {

template <class T, bool kVec>
__global__ void __launch_bounds__(256) dropout_kernel(size_t rows, uint32_t cols, Drop d, const T* x, size_t ld_x, const T* res, size_t ld_res,
                                                      T* y, size_t ld_y, uint64_t groups) {
  const uint32_t per = (cols + 3) / 4;
  for (uint64_t g = (uint64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += (uint64_t)gridDim.x * 256) {
    const uint64_t row = g / per;
    const uint32_t col = (uint32_t)(g - row * per) * 4;
    const int n = (int)min(4u, cols - col);
    float v[4];
    load4(x + row * ld_x + col, kVec, n, v);
    if (d.q) drop4(d, draw(d.key, d.counter + g), v);
    if (res) {
      float r[4];
      load4(res + row * ld_res + col, kVec, n, r);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += r[i];
    }
    store4(y + row * ld_y + col, kVec, n, v);
  }
}

template <class T>
cudaError_t run(size_t rows, uint32_t cols, const Drop& d, const void* x, size_t ld_x, const void* res, size_t ld_res, void* y, size_t ld_y,
                cudaStream_t s) {
  const uint64_t groups = (uint64_t)rows * ((cols + 3) / 4);
  const uint64_t want = (groups + 255) / 256;
  const unsigned grid = (unsigned)(want < 148 * 64 ? want : 148 * 64);
  const size_t q = 4 * sizeof(T);
  const bool vec = (((uintptr_t)x | (uintptr_t)y | (uintptr_t)res) % q) == 0 && ((ld_x | ld_y | (res ? ld_res : 0)) % 4) == 0;
  if (vec) dropout_kernel<T, true><<<grid, 256, 0, s>>>(rows, cols, d, (const T*)x, ld_x, (const T*)res, ld_res, (T*)y, ld_y, groups);
  else dropout_kernel<T, false><<<grid, 256, 0, s>>>(rows, cols, d, (const T*)x, ld_x, (const T*)res, ld_res, (T*)y, ld_y, groups);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_dropout(uint32_t type, size_t rows, uint32_t cols, const Drop& d, const void* x, size_t ld_x, const void* residual,
                           size_t ld_res, void* y, size_t ld_y, cudaStream_t s) {
  if (type == kF32) return run<float>(rows, cols, d, x, ld_x, residual, ld_res, y, ld_y, s);
  if (type == kBf16) return run<__nv_bfloat16>(rows, cols, d, x, ld_x, residual, ld_res, y, ld_y, s);
  return run<__half>(rows, cols, d, x, ld_x, residual, ld_res, y, ld_y, s);
}

}  // namespace layer
}  // namespace aet
