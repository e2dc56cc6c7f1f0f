// Small products of the dense layer: C = A B on FMAs, with any strides, through the layer's epilogue.
//
// 64 x 64 tiles, 256 threads with 4 x 4 sums each, operands as fp32 in shared memory in steps of 16 along k.  A product this
// small is bound by latency, so k is split over the CTAs of a cluster: each leaves its sums in its own shared memory, and every
// CTA adds up a share of the tile's rows over all of them, always in the order of the ranks (the same sums from call to call),
// and takes those rows through the epilogue.  One launch, no workspace.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "layer_common.cuh"

namespace cg = cooperative_groups;

namespace aet {
namespace layer {
namespace {

constexpr int kTile = 64, kStep = 16, kThreads = 256, kLd = kTile + 4;

template <class T, class Out>
__global__ void __launch_bounds__(kThreads) product_fma_kernel(const Product p, const uint32_t tiles_n) {
  __shared__ __align__(16) float as[2][kStep][kLd], bs[2][kStep][kLd];
  __shared__ __align__(16) float sum[kTile][kLd];
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t split = cluster.num_blocks(), rank = cluster.block_rank();
  const uint32_t tile = blockIdx.x / split;
  const uint32_t m0 = tile / tiles_n * kTile, n0 = tile % tiles_n * kTile;
  const uint32_t k0 = (uint32_t)((uint64_t)p.k * rank / split), k1 = (uint32_t)((uint64_t)p.k * (rank + 1) / split);
  const int tid = threadIdx.x, tr = tid / 16 * 4, tc = tid % 16 * 4;
  const T* a = static_cast<const T*>(p.a);
  const T* b = static_cast<const T*>(p.b);
  // neighbouring threads read neighbouring elements of whichever index runs along memory
  const bool a_k = p.a_col == 1, b_n = p.b_col == 1;

  float ra[4], rb[4];
  auto fetch = [&](uint32_t k) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e = tid + u * kThreads;
      const uint32_t ai = a_k ? e / kStep : e % kTile, ak = k + (a_k ? e % kStep : e / kTile);
      ra[u] = m0 + ai < p.m && ak < k1 ? to_f32(a[(size_t)(m0 + ai) * p.a_row + (size_t)ak * p.a_col]) : 0.f;
      const uint32_t bj = b_n ? e % kTile : e / kStep, bk = k + (b_n ? e / kTile : e % kStep);
      rb[u] = n0 + bj < p.n && bk < k1 ? to_f32(b[(size_t)bk * p.b_row + (size_t)(n0 + bj) * p.b_col]) : 0.f;
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e = tid + u * kThreads;
      if (a_k) as[buf][e % kStep][e / kStep] = ra[u]; else as[buf][e / kTile][e % kTile] = ra[u];
      if (b_n) bs[buf][e / kTile][e % kTile] = rb[u]; else bs[buf][e % kStep][e / kStep] = rb[u];
    }
  };

  float acc[4][4] = {};
  if (k0 < k1) fetch(k0);
  int buf = 0;
  for (uint32_t k = k0; k < k1; k += kStep, buf ^= 1) {
    put(buf);
    __syncthreads();     // (one barrier a step: a buffer is written again two steps on, behind the next step's barrier)
    if (k + kStep < k1) fetch(k + kStep);
#pragma unroll
    for (int q = 0; q < kStep; ++q) {
      const float4 x = *reinterpret_cast<const float4*>(&as[buf][q][tr]);
      const float4 y = *reinterpret_cast<const float4*>(&bs[buf][q][tc]);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[i], ys[j], acc[i][j]);
    }
  }
  if (split == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (m0 + tr + i < p.m && n0 + tc < p.n) with_bias<Out>(p, m0 + tr + i, n0 + tc, acc[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<float4*>(&sum[tr + i][tc]) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
  cluster.sync();
  const uint32_t share = kTile / split;    // rows of the tile that this CTA finishes
  for (uint32_t e = tid; e < share * (kTile / 4); e += kThreads) {
    const uint32_t r = rank * share + e / (kTile / 4), c = e % (kTile / 4) * 4;
    if (m0 + r >= p.m || n0 + c >= p.n) continue;
    float v[4] = {};
    for (uint32_t q = 0; q < split; ++q) {
      const float4 s = *reinterpret_cast<const float4*>(cluster.map_shared_rank(&sum[r][c], q));
      v[0] += s.x; v[1] += s.y; v[2] += s.z; v[3] += s.w;
    }
    with_bias<Out>(p, m0 + r, n0 + c, v);
  }
  cluster.sync();   // a CTA's sums stay until the others have read them
}

}  // namespace

// as many CTAs along k as there are SMs for them, each with 32 and more of it
uint32_t fma_split(uint32_t m, uint32_t n, uint32_t k) {
  const uint64_t tiles = ((uint64_t)n + kTile - 1) / kTile * (((uint64_t)m + kTile - 1) / kTile);
  uint32_t split = 1;
  while (split < 8 && tiles * split * 2 <= 148 && k >= 32 * 2 * split) split *= 2;
  return split;
}

cudaError_t launch_product_fma(const Product& p, cudaStream_t s) {
  const uint64_t tiles_n = (p.n + kTile - 1) / kTile, tiles = tiles_n * ((p.m + kTile - 1) / kTile);
  const uint32_t split = fma_split(p.m, p.n, p.k);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(tiles * split));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = split;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const uint32_t tn = (uint32_t)tiles_n;
  if (p.type == kF32) return cudaLaunchKernelEx(&cfg, product_fma_kernel<float, float>, p, tn);
  if (p.type == kBf16 && p.e.out_type == kF32) return cudaLaunchKernelEx(&cfg, product_fma_kernel<__nv_bfloat16, float>, p, tn);
  if (p.type == kBf16) return cudaLaunchKernelEx(&cfg, product_fma_kernel<__nv_bfloat16, __nv_bfloat16>, p, tn);
  return cudaLaunchKernelEx(&cfg, product_fma_kernel<__half, __half>, p, tn);
}

}  // namespace layer
}  // namespace aet
