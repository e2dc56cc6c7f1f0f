// A few rows through a dense layer (a server that answers single requests): C = A B with up to eight rows of A.
//
// Bound by reading B once.  A thread keeps 16 bytes of columns and goes down B eight rows at a time with all their loads under way; a warp
// covers 512 bytes of a row, so that whole lines are read, the eight warps of a CTA and the up to eight CTAs of a cluster share k.  A's values
// lie in shared memory as fp32 and are read as broadcasts, four of k at once.  The warps' sums are added up in shared memory and the CTAs'
// through the cluster, both always in the same order, and every CTA takes a share of the columns through the epilogue: one launch, no
// workspace.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "layer_common.cuh"

namespace cg = cooperative_groups;

namespace aet {
namespace layer {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps, kAhead = 8;

template <class T> constexpr int kV = 16 / (int)sizeof(T);

template <class T, class Out, int R, bool kVec>
__global__ void __launch_bounds__(kThreads) product_rows_kernel(const Product p, const uint32_t kc) {   // kc: of k a CTA, a multiple of 64
  constexpr int V = kV<T>, kCols = 32 * V;
  extern __shared__ __align__(16) float smem[];
  float* xs = smem;                      // [R][kc]
  float* sums = smem + R * kc;           // [kWarps][R][kCols]
  in_line();
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t split = cluster.num_blocks(), rank = cluster.block_rank();
  const uint32_t n0 = blockIdx.x / split * kCols, k0 = rank * kc;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const T* a = static_cast<const T*>(p.a);
  const T* b = static_cast<const T*>(p.b);
  for (uint32_t e = tid; e < R * kc; e += kThreads) {
    const uint32_t r = e / kc, k = k0 + e % kc;
    xs[e] = r < p.m && k < p.k ? to_f32(a[(size_t)r * p.a_row + k]) : 0.f;
  }
  __syncthreads();

  float acc[R][V] = {};
  const uint32_t kw = kc / kWarps, from = warp * kw, to = k0 + from >= p.k ? from : min(from + kw, p.k - k0);
  const T* col = b + (size_t)k0 * p.b_row + n0;       // a lane's columns: V neighbours, or every 32nd where rows start anywhere
  const auto fma_row = [&](const float (&w)[V], uint32_t k) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float x = xs[r * kc + k];
#pragma unroll
      for (int i = 0; i < V; ++i) acc[r][i] = fmaf(x, w[i], acc[r][i]);
    }
  };
  if (kVec) {
    if (n0 + lane * V < p.n) {      // (rows are whole 16 bytes and more apart: what is read past the last column is of the same row's gap)
      const bool whole = n0 + lane * V + V <= p.n;
      uint32_t k = from;
      if (whole) {
        for (; k + kAhead <= to; k += kAhead) {
          Words<T, V> q[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j) q[j] = *reinterpret_cast<const Words<T, V>*>(col + (size_t)(k + j) * p.b_row + lane * V);
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            float w[V];
            unpack<T, V>(q[j], w);
            fma_row(w, k + j);
          }
        }
      }
      for (; k < to; ++k) {
        float w[V];
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = n0 + lane * V + i < p.n ? to_f32(col[(size_t)k * p.b_row + lane * V + i]) : 0.f;
        fma_row(w, k);
      }
    }
  } else {
#pragma unroll 4
    for (uint32_t k = from; k < to; ++k) {
      float w[V];
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = n0 + lane + 32 * i < p.n ? to_f32(col[(size_t)k * p.b_row + lane + 32 * i]) : 0.f;
      fma_row(w, k);
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) sums[(warp * R + r) * kCols + (kVec ? lane * V + i : lane + 32 * i)] = acc[r][i];
  __syncthreads();
  for (uint32_t e = tid; e < R * kCols / 4; e += kThreads) {       // the CTA's sums, in the first warp's place
    float4 s = reinterpret_cast<float4*>(sums)[e];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
      const float4 v = reinterpret_cast<float4*>(sums)[w * (R * kCols / 4) + e];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    reinterpret_cast<float4*>(sums)[e] = s;
  }
  cluster.sync();
  const uint32_t all = R * kCols / 4, share = (all + split - 1) / split;
  for (uint32_t e = rank * share + tid; e < min(all, (rank + 1) * share); e += kThreads) {
    const uint32_t r = e / (kCols / 4), c = n0 + e % (kCols / 4) * 4;
    if (r >= p.m || c >= p.n) continue;
    float v[4] = {};
    for (uint32_t q = 0; q < split; ++q) {
      const float4 s = *cluster.map_shared_rank(reinterpret_cast<float4*>(sums) + e, q);
      v[0] += s.x; v[1] += s.y; v[2] += s.z; v[3] += s.w;
    }
    with_bias<Out>(p, r, c, v);
  }
  cluster.sync();   // a CTA's sums stay until the others have read them
}

template <class T, class Out, int R, bool kVec>
cudaError_t go(const Product& p, cudaStream_t s) {
  constexpr int kCols = 32 * kV<T>;
  const uint64_t across = ((uint64_t)p.n + kCols - 1) / kCols;
  // CTAs along k: four and more for each of 148 SMs, each with 64 of k and more; at most 2,048 of k, so that A's values fit
  uint32_t split = 1;
  while (split < 8 && (p.k > 2048 * split || (across * split < 148 * 4 && p.k > 64 * split))) split *= 2;
  const uint32_t kc = (uint32_t)((((uint64_t)p.k + split - 1) / split + 63) / 64 * 64);
  const size_t smem = ((size_t)R * kc + (size_t)kWarps * R * kCols) * 4;
  const auto kernel = product_rows_kernel<T, Out, R, kVec>;
  if (const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024)) return e;
  return launch(kernel, dim3((unsigned)(across * split)), kThreads, smem, split, s, p, kc);
}
template <class T, class Out>
cudaError_t run(const Product& p, cudaStream_t s) {
  const bool vec = (uintptr_t)p.b % 16 == 0 && p.b_row % kV<T> == 0;
#define AET_ROWS(R) (vec ? go<T, Out, R, true>(p, s) : go<T, Out, R, false>(p, s))
  return p.m == 1 ? AET_ROWS(1) : p.m <= 2 ? AET_ROWS(2) : p.m <= 4 ? AET_ROWS(4) : AET_ROWS(8);
#undef AET_ROWS
}

}  // namespace

// k that eight CTAs hold (eight rows of 2,048 values and their sums are 128 KB and less)
bool rows_kernel_takes(uint32_t m, uint32_t k) { return m <= 8 && k <= 8 * 2048; }

cudaError_t launch_product_rows(const Product& p, cudaStream_t s) {
  if (p.type == kF32) return run<float, float>(p, s);
  if (p.type == kBf16 && p.e.out_type == kF32) return run<__nv_bfloat16, float>(p, s);
  if (p.type == kBf16) return run<__nv_bfloat16, __nv_bfloat16>(p, s);
  return run<__half, __half>(p, s);
}

}  // namespace layer
}  // namespace aet
