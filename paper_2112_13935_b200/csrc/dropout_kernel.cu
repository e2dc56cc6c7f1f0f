// Dropout whose mask is never stored: y = residual + drop(x), each element's sixteen random bits a function of where it stands.
//
// The counter-based generator costs some 22 integer instructions a draw of 64 bits; with four elements to a draw a bf16 array stays
// bound by memory (about 5.8 elements a cycle and SM at the copy rate, 22 issue slots each).  A thread keeps its 16 bytes of columns and
// goes down the rows, three at a time with all their loads under way.  The gradient is the same call on dy.
#include <cuda_runtime.h>

#include "layer_rows.cuh"

namespace aet {
namespace layer {
namespace {

constexpr int kThreads = 256, kRows = 3;

template <class T, int N, bool kVec>
__global__ void __launch_bounds__(kThreads, 3) dropout_kernel(const size_t rows, const uint32_t cols, const Drop d, const T* x, const size_t ld_x, const T* res,
                                                           const size_t ld_res, T* y, const size_t ld_y, const uint32_t log) {
  in_line();
  const uint32_t col = ((blockIdx.x << log) + (threadIdx.x & ((1u << log) - 1))) * N;
  if (col >= cols) return;
  const int n = (int)min((uint32_t)N, cols - col);
  const bool whole = kVec && n == N;
  const size_t step = (size_t)gridDim.y * (kThreads >> log);     // rows between two of a thread's
  for (size_t r0 = (size_t)blockIdx.y * (kThreads >> log) + (threadIdx.x >> log); r0 < rows; r0 += kRows * step) {
    Words<T, N> q[kRows], e[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const size_t r = r0 + i * step;
      if (r >= rows) break;
      q[i] = load_words<T, N>(x + r * ld_x + col, whole, n);
      if (res) e[i] = load_words<T, N>(res + r * ld_res + col, whole, n);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const size_t r = r0 + i * step;
      if (r >= rows) break;
      keep_words(q[i]);
      float v[N];
      unpack<T, N>(q[i], v);
      if (d.q) drop_n<N>(d, drop_at(d, r, cols, col), v);
      if (res) {
        keep_words(e[i]);
        float a[N];
        unpack<T, N>(e[i], a);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += a[k];
      }
      store_n<T, N>(y + r * ld_y + col, whole, n, v);
    }
  }
}

template <class T, int N, bool kVec>
cudaError_t go(size_t rows, uint32_t cols, const Drop& d, const void* x, size_t ld_x, const void* res, size_t ld_res, void* y, size_t ld_y, cudaStream_t s) {
  const uint32_t log = log_lanes<N>(cols);
  const uint64_t across = (((uint64_t)cols + N - 1) / N + (1u << log) - 1) >> log;     // CTAs across the columns
  // eight CTAs for each of 148 SMs, which go round the rows
  const uint64_t at_once = (uint64_t)(kThreads >> log) * kRows, most = (rows + at_once - 1) / at_once, want = (148 * 8 + across - 1) / across;
  return launch(dropout_kernel<T, N, kVec>, dim3((unsigned)across, (unsigned)(most < want ? most : want)), kThreads, 0, 1, s, rows, cols, d, (const T*)x,
                ld_x, (const T*)res, ld_res, (T*)y, ld_y, log);
}
template <class T>
cudaError_t run(size_t rows, uint32_t cols, const Drop& d, const void* x, size_t ld_x, const void* res, size_t ld_res, void* y, size_t ld_y,
                cudaStream_t s) {
  constexpr int N = 16 / (int)sizeof(T);
  const bool vec = (((uintptr_t)x | (uintptr_t)y | (uintptr_t)res) % 16) == 0 && ((ld_x | ld_y | (res ? ld_res : 0)) % N) == 0;
  return vec ? go<T, N, true>(rows, cols, d, x, ld_x, res, ld_res, y, ld_y, s) : go<T, 4, false>(rows, cols, d, x, ld_x, res, ld_res, y, ld_y, s);
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
