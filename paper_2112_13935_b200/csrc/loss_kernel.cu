// Softmax cross-entropy of rows of logits z with class y: loss = log sum_j exp(z_j) - z_y, its gradient
// scale * weight * (softmax(z) - 1_y), and the lowest index of the row's maximum.
//
// One CTA per row, two passes: the running maximum m and the sum of exp(z - m) of each thread, joined over the CTA, then the gradient.
#include <cuda_runtime.h>
#include <math_constants.h>

#include "layer_common.cuh"

namespace aet {
namespace layer {
namespace {

// What a part of a row says: its maximum, where it stands first, and the sum of exp(z - base(maximum)).  The sum is NaN where a logit
// is and only there (a maximum that is infinite counts as zero in it); a row whose maximum is infinite has no loss: NaN.
struct Part { float top, sum; int32_t at; };
__device__ __forceinline__ float base(float top) { return isinf(top) ? 0.f : top; }
__device__ __forceinline__ Part part_of(float v, int32_t j) {
  return Part{v == v ? v : -CUDART_INF_F, v == v ? (v == -CUDART_INF_F ? 0.f : 1.f) : v, v == v ? j : 0x7fffffff};
}
__device__ __forceinline__ Part join(const Part& a, const Part& b) {
  Part r;
  const bool first = a.top > b.top || (a.top == b.top && a.at <= b.at);
  r.top = first ? a.top : b.top;
  r.at = first ? a.at : b.at;
  r.sum = (a.top == r.top ? a.sum : a.sum * expf(a.top - base(r.top))) + (b.top == r.top ? b.sum : b.sum * expf(b.top - base(r.top)));
  return r;
}

template <class T>
__global__ void __launch_bounds__(256) loss_rows_kernel(const LossLaunch p) {
  __shared__ Part parts[8];
  for (size_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const int32_t y = p.labels[row];
    const T* z = static_cast<const T*>(p.logits) + row * p.ld;
    T* g = p.grad ? static_cast<T*>(p.grad) + row * p.ld_grad : nullptr;
    if (y < 0) {   // a row without an answer is not read
      if (g)
        for (uint32_t j = threadIdx.x; j < p.classes; j += 256) g[j] = from_f32<T>(0.f);
      if (threadIdx.x == 0) {
        if (p.loss) p.loss[row] = 0.f;
        if (p.top) p.top[row] = -1;
      }
      continue;
    }
    Part a{-CUDART_INF_F, 0.f, 0x7fffffff};
    for (uint32_t j = threadIdx.x; j < p.classes; j += 256) {
      a = join(a, part_of(to_f32(z[j]), (int32_t)j));
    }
    for (int o = 16; o; o >>= 1) {
      Part b;
      b.top = __shfl_xor_sync(~0u, a.top, o);
      b.sum = __shfl_xor_sync(~0u, a.sum, o);
      b.at = __shfl_xor_sync(~0u, a.at, o);
      a = join(a, b);
    }
    __syncthreads();
    if (threadIdx.x % 32 == 0) parts[threadIdx.x / 32] = a;
    __syncthreads();
    a = parts[0];
    for (int q = 1; q < 8; ++q) a = join(a, parts[q]);
    const bool known = (uint32_t)y < p.classes;
    const float zy = known ? to_f32(z[y]) : CUDART_NAN_F;
    __syncthreads();   // the label's logit has been read before the gradient may take its place
    if (threadIdx.x == 0) {
      if (p.loss) p.loss[row] = isinf(a.top) ? CUDART_NAN_F : logf(a.sum) + (a.top - zy);
      if (p.top) p.top[row] = a.sum == a.sum ? a.at : -1;
    }
    if (g) {
      const float f = known ? p.scale * (p.weight ? p.weight[row] : 1.f) : CUDART_NAN_F;
      const float inv = isinf(a.top) ? CUDART_NAN_F : 1.f / a.sum;
      for (uint32_t j = threadIdx.x; j < p.classes; j += 256)
        g[j] = from_f32<T>(f * (expf(to_f32(z[j]) - a.top) * inv - (j == (uint32_t)y ? 1.f : 0.f)));
    }
  }
}

template <class T>
cudaError_t run(const LossLaunch& p, cudaStream_t s) {
  const unsigned grid = (unsigned)(p.rows < 148 * 64 ? p.rows : 148 * 64);
  loss_rows_kernel<T><<<grid, 256, 0, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_loss(const LossLaunch& p, cudaStream_t s) {
  if (p.type == kF32) return run<float>(p, s);
  if (p.type == kBf16) return run<__nv_bfloat16>(p, s);
  return run<__half>(p, s);
}

}  // namespace layer
}  // namespace aet
