// What the gradient of a dense layer starts with: dz = drop(dy) act'(pre), and the sums of dz over the rows (the bias's gradient).
//
// One pass over dy and pre, bound by memory.  A thread keeps 16 bytes of columns and goes down a slab of rows, two at a time with all
// their loads under way; the sums of a slab go to the workspace and a second small kernel adds the slabs up in their order, so that
// they are the same from call to call.
#include <cuda_runtime.h>

#include "layer_rows.cuh"

namespace aet {
namespace layer {
namespace {

constexpr int kThreads = 256, kRows = 2;

template <int N>
__device__ __forceinline__ void store_wide(float* p, bool whole, int n, const float (&v)[N]) {
#pragma unroll
  for (int g = 0; g < N; g += 4) {
    const float q[4] = {v[g], v[g + 1], v[g + 2], v[g + 3]};
    store_n<float, 4>(p + g, whole, n - g, q);
  }
}

template <class T, int N, bool kVec>
__global__ void __launch_bounds__(kThreads, 4) slope_kernel(const SlopeLaunch p, const uint32_t slabs, const uint32_t log) {
  __shared__ __align__(16) float sums[kThreads * N];
  in_line();
  const uint32_t lane = threadIdx.x & ((1u << log) - 1), down = threadIdx.x >> log, at_once = kThreads >> log;
  const uint32_t col = ((blockIdx.x << log) + lane) * N;
  const size_t r_from = (size_t)p.rows * blockIdx.y / slabs, r_to = (size_t)p.rows * (blockIdx.y + 1) / slabs;
  const int n = col < p.cols ? (int)min((uint32_t)N, p.cols - col) : 0;
  const bool whole = kVec && n == N;
  const T* dy = static_cast<const T*>(p.dy);
  const T* pre = static_cast<const T*>(p.pre);
  float acc[N] = {};
  if (n) {
    for (size_t r0 = r_from + down; r0 < r_to; r0 += (size_t)kRows * at_once) {
      Words<T, N> q[kRows], w[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const size_t r = r0 + (size_t)i * at_once;
        if (r >= r_to) break;
        q[i] = load_words<T, N>(dy + r * p.ld_dy + col, whole, n);
        if (pre) w[i] = load_words<T, N>(pre + r * p.ld_pre + col, whole, n);
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const size_t r = r0 + (size_t)i * at_once;
        if (r >= r_to) break;
        keep_words(q[i]);
        float v[N];
        unpack<T, N>(q[i], v);
        if (p.drop.q) drop_n<N>(p.drop, drop_at(p.drop, r, p.cols, col), v);
        if (pre) {
          keep_words(w[i]);
          float z[N];
          unpack<T, N>(w[i], z);
          if (p.act == kRelu) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = z[k] > 0.f ? v[k] : 0.f;
          } else if (p.act == kGelu) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] *= act_slope<T>(kGelu, z[k]);
          } else {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] *= act_slope<T>(kSilu, z[k]);
          }
        }
        if (p.parts) store_parts<N>(p.parts + r * p.ld_parts + col, p.plane, v);   // (0 past the last column)
        if (p.dz && p.dz_type == kF32) store_wide<N>(static_cast<float*>(p.dz) + r * p.ld_dz + col, whole, n, v);
        else if (p.dz && sizeof(T) == 4) store_n<__nv_bfloat16, N>(static_cast<__nv_bfloat16*>(p.dz) + r * p.ld_dz + col, whole, n, v);
        else if (p.dz) store_n<T, N>(static_cast<T*>(p.dz) + r * p.ld_dz + col, whole, n, v);
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] += v[k];
      }
    }
  }
  if (!p.db) return;
#pragma unroll
  for (int k = 0; k < N; ++k) sums[(down << log) * N + k * (1u << log) + lane] = acc[k];
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < (uint32_t)N << log; e += kThreads) {
    const uint32_t c = ((blockIdx.x << log) + (e & ((1u << log) - 1))) * N + (e >> log);
    if (c >= p.cols) continue;
    float v = 0.f;
    for (uint32_t q = 0; q < at_once; ++q) v += sums[(q << log) * N + e];
    p.partial[(size_t)blockIdx.y * p.cols + c] = v;
  }
}

// db = (db +) the sums of the slabs; 32 columns a CTA, eight threads to a column
template <class T>
__global__ void __launch_bounds__(256) slab_sums_kernel(const float* partial, uint32_t slabs, uint32_t cols, T* db, uint32_t accumulate) {
  __shared__ float sums[8][32];
  in_line();
  const int lane = threadIdx.x % 32, part = threadIdx.x / 32;
  const uint32_t c = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (uint32_t q = part; q < slabs; q += 8) v += partial[(size_t)q * cols + c];
  }
  sums[part][lane] = v;
  __syncthreads();
  if (part || c >= cols) return;
  v = accumulate ? to_f32(db[c]) : 0.f;
  for (int q = 0; q < 8; ++q) v += sums[q][lane];
  db[c] = from_f32<T>(v);
}

// Slabs for about eight CTAs on each of 148 SMs, each with two rows and more to a thread.  (By the narrowest columns a thread may keep,
// so that the workspace does not hang on where the arrays start.)
uint32_t slabs_of(uint32_t rows, uint32_t cols) {
  const uint32_t log = log_lanes<4>(cols);
  const uint64_t across = (((uint64_t)cols + 3) / 4 + (1u << log) - 1) >> log, at_once = (uint64_t)(kThreads >> log) * kRows;
  const uint64_t want = (148 * 8 + across - 1) / across, most = (rows + at_once - 1) / at_once;
  const uint64_t n = want < most ? want : most;
  return n ? (uint32_t)n : 1;
}

bool aligned(const void* p, size_t ld, size_t n, size_t bytes) { return !p || ((uintptr_t)p % (n * bytes) == 0 && ld % n == 0); }

template <class T, int N, bool kVec>
cudaError_t go(const SlopeLaunch& p, uint32_t slabs, cudaStream_t s) {
  const uint32_t log = log_lanes<N>(p.cols);
  const uint64_t across = (((uint64_t)p.cols + N - 1) / N + (1u << log) - 1) >> log;
  return launch(slope_kernel<T, N, kVec>, dim3((unsigned)across, slabs), kThreads, 0, 1, s, p, slabs, log);
}
template <class T>
cudaError_t run(const SlopeLaunch& p, cudaStream_t s) {
  constexpr int N = 16 / (int)sizeof(T);
  const uint32_t slabs = slabs_of(p.rows, p.cols);
  const bool vec = aligned(p.dy, p.ld_dy, N, sizeof(T)) && aligned(p.pre, p.ld_pre, N, sizeof(T)) && aligned(p.dz, p.ld_dz, N, type_bytes(p.dz_type));
  const cudaError_t e = vec ? go<T, N, true>(p, slabs, s) : go<T, 4, false>(p, slabs, s);
  if (e != cudaSuccess || !p.db) return e;
  const dim3 grid((p.cols + 31) / 32);
  if (p.db_type == kF32) return launch(slab_sums_kernel<float>, grid, 256, 0, 1, s, p.partial, slabs, p.cols, static_cast<float*>(p.db), p.accumulate);
  if (p.db_type == kBf16)
    return launch(slab_sums_kernel<__nv_bfloat16>, grid, 256, 0, 1, s, p.partial, slabs, p.cols, static_cast<__nv_bfloat16*>(p.db), p.accumulate);
  return launch(slab_sums_kernel<__half>, grid, 256, 0, 1, s, p.partial, slabs, p.cols, static_cast<__half*>(p.db), p.accumulate);
}

}  // namespace

size_t slope_partial_floats(uint32_t rows, uint32_t cols) { return (size_t)slabs_of(rows, cols) * cols; }

cudaError_t launch_slope(const SlopeLaunch& p, cudaStream_t s) {
  if (p.type == kF32) return run<float>(p, s);
  if (p.type == kBf16) return run<__nv_bfloat16>(p, s);
  return run<__half>(p, s);
}

}  // namespace layer
}  // namespace aet
