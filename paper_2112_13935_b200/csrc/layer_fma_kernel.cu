// Small products of the dense layer: C = A B on FMAs, with any strides, through the layer's epilogue.
//
// A product this small is bound by latency, so it is spread: tiles of 64 x 64 sums, or of 32 x 32 where those would leave SMs idle; k in up
// to eight parts over the CTAs of a cluster and, in the small tiles, in four over groups of two warps.  A thread has 4 x 4 sums and reads
// eight values from shared memory for sixteen FMAs; 32 of k are multiplied while the next 64 are on their way to registers.  Each CTA leaves
// its sums in its own shared memory, and every CTA adds up a share of the tile's rows over all of them, always in the order of the ranks (the
// same sums from call to call), and takes those rows through the epilogue.  One launch, no workspace.
//
// A gradient's dz comes in fp32 here (the tensor cores take it rounded to the element type).
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "layer_common.cuh"

namespace cg = cooperative_groups;

namespace aet {
namespace layer {
namespace {

constexpr int kStep = 32, kThreads = 256;

template <int TILE> struct Shape {
  static constexpr int groups = 64 * 64 / (TILE * TILE), group_threads = kThreads / groups, ld = TILE + 4;
  static constexpr int loads = TILE * kStep / kThreads;      // values of an operand a thread brings a step
  static constexpr int across = TILE / 4;                    // threads along a row of the tile
};

template <class TA, class TB, class Out, int TILE>
__global__ void __launch_bounds__(kThreads, 2) product_fma_kernel(const Product p, const uint32_t tiles_n) {
  using S = Shape<TILE>;
  __shared__ __align__(16) float smem[4 * kStep * S::ld];
  float(*as)[kStep][S::ld] = reinterpret_cast<float(*)[kStep][S::ld]>(smem);
  float(*bs)[kStep][S::ld] = reinterpret_cast<float(*)[kStep][S::ld]>(smem + 2 * kStep * S::ld);
  float(*sums)[TILE][S::ld] = reinterpret_cast<float(*)[TILE][S::ld]>(smem);      // in the operands' place when they are done with
  static_assert(S::groups * TILE <= 4 * kStep, "the sums do not fit");
  in_line();
  cg::cluster_group cluster = cg::this_cluster();
  const uint32_t split = cluster.num_blocks(), rank = cluster.block_rank();
  const uint32_t tile = blockIdx.x / split;
  const uint32_t m0 = tile / tiles_n * TILE, n0 = tile % tiles_n * TILE;
  const uint32_t k0 = (uint32_t)((uint64_t)p.k * rank / split), k1 = (uint32_t)((uint64_t)p.k * (rank + 1) / split);
  const int tid = threadIdx.x, group = tid / S::group_threads, in = tid % S::group_threads, tr = in / S::across * 4, tc = in % S::across * 4;
  const TA* a = static_cast<const TA*>(p.a);
  const TB* b = static_cast<const TB*>(p.b);
  const bool a_k = p.a_col == 1, b_n = p.b_col == 1;

  // Where a thread's u-th value of an operand stands.  Neighbouring lanes read neighbouring elements: of an operand laid out across k a row
  // of the tile, of one laid out along k eight of k in four rows, which then go to 32 different banks.
  const auto along = [&](int u, int& i, int& k) { k = tid % 8 + u % 4 * 8; i = tid / 8 + u / 4 * 32; };
  const auto across = [&](int u, int& i, int& k) { const int e = tid + u * kThreads; i = e % TILE; k = e / TILE; };
  float ra[2][S::loads], rb[2][S::loads];
  const auto fetch = [&](uint32_t k, float (&xa)[S::loads], float (&xb)[S::loads]) {
#pragma unroll
    for (int u = 0; u < S::loads; ++u) {
      int i, kk;
      if (a_k) along(u, i, kk); else across(u, i, kk);
      xa[u] = m0 + i < p.m && k + kk < k1 ? to_f32(a[(size_t)(m0 + i) * p.a_row + (size_t)(k + kk) * p.a_col]) : 0.f;
      if (b_n) across(u, i, kk); else along(u, i, kk);
      xb[u] = n0 + i < p.n && k + kk < k1 ? to_f32(b[(size_t)(k + kk) * p.b_row + (size_t)(n0 + i) * p.b_col]) : 0.f;
    }
  };
  float acc[4][4] = {};
  const auto step = [&](uint32_t k, int buf, float (&xa)[S::loads], float (&xb)[S::loads]) {
#pragma unroll
    for (int u = 0; u < S::loads; ++u) {
      int i, kk;
      if (a_k) along(u, i, kk); else across(u, i, kk);
      as[buf][kk][i] = xa[u];
      if (b_n) across(u, i, kk); else along(u, i, kk);
      bs[buf][kk][i] = xb[u];
    }
    __syncthreads();     // (one barrier a step: a buffer is written again two steps on, behind the next step's barrier)
    if (k + 2 * kStep < k1) fetch(k + 2 * kStep, xa, xb);
#pragma unroll
    for (int q = 0; q < kStep / S::groups; ++q) {
      const int kk = group * (kStep / S::groups) + q;
      const float4 x = *reinterpret_cast<const float4*>(&as[buf][kk][tr]);
      const float4 y = *reinterpret_cast<const float4*>(&bs[buf][kk][tc]);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[i], ys[j], acc[i][j]);
    }
  };
  if (k0 < k1) fetch(k0, ra[0], rb[0]);
  if (k0 + kStep < k1) fetch(k0 + kStep, ra[1], rb[1]);
  for (uint32_t k = k0; k < k1; k += 2 * kStep) {
    step(k, 0, ra[0], rb[0]);
    if (k + kStep < k1) step(k + kStep, 1, ra[1], rb[1]);
  }
  if (S::groups == 1 && split == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (m0 + tr + i < p.m && n0 + tc < p.n) with_bias<Out>(p, m0 + tr + i, n0 + tc, acc[i]);
    return;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<float4*>(&sums[group][tr + i][tc]) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
  if (S::groups > 1) {        // the groups' sums, in the first one's place
    __syncthreads();
    for (int e = tid; e < TILE * S::across; e += kThreads) {
      float4* to = reinterpret_cast<float4*>(&sums[0][e / S::across][e % S::across * 4]);
      float4 s = *to;
#pragma unroll
      for (int g = 1; g < S::groups; ++g) {
        const float4 v = *reinterpret_cast<const float4*>(&sums[g][e / S::across][e % S::across * 4]);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      *to = s;
    }
  }
  cluster.sync();
  const uint32_t share = TILE / split;    // rows of the tile that this CTA finishes
  for (uint32_t e = tid; e < share * S::across; e += kThreads) {
    const uint32_t r = rank * share + e / S::across, c = e % S::across * 4;
    if (m0 + r >= p.m || n0 + c >= p.n) continue;
    float v[4] = {};
    for (uint32_t q = 0; q < split; ++q) {
      const float4 s = *reinterpret_cast<const float4*>(cluster.map_shared_rank(&sums[0][r][c], q));
      v[0] += s.x; v[1] += s.y; v[2] += s.z; v[3] += s.w;
    }
    with_bias<Out>(p, m0 + r, n0 + c, v);
  }
  cluster.sync();   // a CTA's sums stay until the others have read them
}

uint64_t tiles_of(uint32_t m, uint32_t n, uint32_t tile) { return ((uint64_t)m + tile - 1) / tile * (((uint64_t)n + tile - 1) / tile); }
// 64 x 64 tiles where they fill the 148 SMs
bool wide_tiles(uint32_t m, uint32_t n) { return tiles_of(m, n, 64) >= 148; }

template <class TA, class TB, class Out>
cudaError_t run(const Product& p, cudaStream_t s) {
  const bool wide = wide_tiles(p.m, p.n);
  const uint32_t tile = wide ? 64 : 32, split = fma_split(p.m, p.n, p.k), tiles_n = (uint32_t)(((uint64_t)p.n + tile - 1) / tile);
  return launch(wide ? product_fma_kernel<TA, TB, Out, 64> : product_fma_kernel<TA, TB, Out, 32>, dim3((unsigned)(tiles_of(p.m, p.n, tile) * split)), kThreads, 0,
                split, s, p, tiles_n);
}
template <class T>
cudaError_t of_type(const Product& p, cudaStream_t s) {     // a gradient's dz may be fp32 beside operands of T
  if (p.a_f32) return run<float, T, T>(p, s);
  if (p.b_f32) return run<T, float, T>(p, s);
  return run<T, T, T>(p, s);
}

}  // namespace

// as many CTAs along k as there are SMs for them, each with 64 and more of it
uint32_t fma_split(uint32_t m, uint32_t n, uint32_t k) {
  const uint64_t tiles = tiles_of(m, n, wide_tiles(m, n) ? 64 : 32);
  uint32_t split = 1;
  while (split < 8 && tiles * split * 2 <= 2 * 148 && k >= 64 * 2 * split) split *= 2;
  return split;
}

uint64_t fma_volume(uint32_t m, uint32_t n, uint32_t k) {
  const uint64_t tile = wide_tiles(m, n) ? 64 : 32;
  return tiles_of(m, n, (uint32_t)tile) * tile * tile * k;
}

cudaError_t launch_product_fma(const Product& p, cudaStream_t s) {
  if (p.type == kF32) return run<float, float, float>(p, s);
  if (p.type == kBf16 && p.e.out_type == kF32) return run<__nv_bfloat16, __nv_bfloat16, float>(p, s);
  return p.type == kBf16 ? of_type<__nv_bfloat16>(p, s) : of_type<__half>(p, s);
}

}  // namespace layer
}  // namespace aet
