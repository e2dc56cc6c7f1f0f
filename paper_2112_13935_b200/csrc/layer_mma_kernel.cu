// Large products of the dense layer on the 5th-generation tensor cores: C = A B, sums in tensor memory, through the layer's epilogue.
//
// One persistent CTA per SM (or a pair of CTAs on two) walks over output tiles of 128 rows a CTA and BN columns.  One thread feeds a
// ring of stages by TMA (64 of k each, 128-byte swizzle), one issues tcgen05.mma, the others take finished sums out of tensor memory
// through a transposing buffer, so that rows are stored in whole sectors, while the next tile's products run into the other half of
// tensor memory.  Either operand may be laid out along k or across it: TMA brings 64 x 64 blocks either way and the matrix
// descriptors say which, so that the gradients' transposed products read the tensors as they are.
//
// PLANES 3: fp32 operands as three bf16 parts of 8 bits and more each (launch_planes), six products of parts per k; what is left out is
// below 2^-24 of a product.  Tensor cores cut the sums they form, so sums of 256 of k leave tensor memory and are added up in fp32
// registers.  A stage then holds the three parts of both operands: each part is loaded once for the products it takes part in.
//
// Few tiles and a long k: k is split, the parts' sums go to the workspace and a second kernel adds them up in their order.
//
// Every wait is bounded; a role whose wait has given up stops issuing, and tiles that were not summed are stored as NaN.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math_constants.h>

#include <atomic>

#include "aet_kernels.h"
#include "layer_common.cuh"

namespace aet {
namespace layer {
namespace {

constexpr int kBlock = 16;         // columns that go through a warp's buffer at once

constexpr uint32_t kWaitLimit = 1u << 22;
constexpr int kChunk = 256;         // PLANES 3: of k per sum in tensor memory
constexpr uint32_t kGroup = 16;     // tile rows that are walked together, so that their operands meet in L2

template <int PLANES, int BN, int CG>
struct Ring {
  static constexpr int bk = PLANES == 1 ? 64 : 32;     // of k in a stage
  static constexpr int b_rows = BN / CG;
  static constexpr int a_part = 128 * bk * 2, b_part = b_rows * bk * 2, mn_block = 64 * bk * 2;
  static constexpr int a_bytes = PLANES * a_part, stage = a_bytes + PLANES * b_part;
  // warps that store: four to a quarter of tensor memory, since they wait for memory most of the time; fp32 sums in registers leave room
  // for two (sixteen registers a thread and column block)
  static constexpr int epi_warps = PLANES == 1 ? 16 : 8, threads = 64 + 32 * epi_warps;
  static constexpr int cols = BN / (epi_warps / 4);     // columns a warp takes
  static constexpr int trans = epi_warps * 32 * kBlock * 4, rest = 512;
  static constexpr int fit = (232448 - 1024 - trans - rest) / stage;
  static constexpr int stages = fit < 6 ? fit : 6;
  static constexpr int total = 1024 + stages * stage + trans + rest;
  static_assert(stages >= 2, "no ring");
};

struct Launch {
  Product p;            // a, b and their strides are in the tensor maps
  float* partial;       // [splits, m, ld_partial] where k is split
  size_t ld_partial;
  uint32_t a_mn, b_mn;  // laid out across k
  uint32_t splits, tiles_m, tiles_n, idesc;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count)); }
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  for (uint32_t i = 0; i < kWaitLimit; ++i) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred q;\n\tmbarrier.try_wait.parity.shared::cta.b64 q, [%1], %2;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok) return true;
  }
  return false;
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Arrives on a barrier of the cluster (an address of mapa, or the CTA's own).
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  if (CG == 1)
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
  else   // the barrier may be the other CTA's of the pair
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (CG == 1)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// The barrier (of both CTAs of a pair) gets an arrival when the products issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
  if (CG == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t cols) {
  if (CG == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t cols) {
  if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols));
  else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols));
}
// 16 columns of the warp's rows; they are there after tmem_wait.
__device__ __forceinline__ void tmem_ld(uint32_t at, uint32_t (&r)[kBlock]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at));
}
template <int N>
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[N][kBlock]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int c = 0; c < N; ++c)
#pragma unroll
    for (int i = 0; i < kBlock; ++i) asm volatile("" : "+r"(r[c][i]));     // (no use of a value moves in front of the wait)
}
// Matrix descriptor of a swizzled tile.  Along k: rows of bk elements (128 or 64 bytes, swizzled as wide), 8-row groups one after another.
// Across k: 128-byte rows of 64 of M or N, bk of them to a block, blocks one after another, in them 8 of k every 1,024 bytes.
template <int bk>
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, bool mn) {
  const uint32_t lead = mn ? 64 * bk * 2 : 16, stride = mn || bk == 64 ? 1024 : 512;
  const uint64_t swizzle = mn || bk == 64 ? 2 : 4;
  return (uint64_t)((addr & 0x3FFFF) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | (uint64_t)1 << 46 | swizzle << 61;
}

struct Tile { uint32_t m, n, kb0, kb1, split; };
__device__ __forceinline__ Tile tile_of(const Launch& L, uint32_t item, uint32_t kbs) {
  const uint32_t tiles = L.tiles_m * L.tiles_n;
  Tile t;
  t.split = item / tiles;
  const uint32_t i = item % tiles, in_group = kGroup * L.tiles_n, g = i / in_group, r = i % in_group;
  const uint32_t rows = min(kGroup, L.tiles_m - g * kGroup);
  t.m = g * kGroup + r % rows;
  t.n = r / rows;
  t.kb0 = (uint32_t)((uint64_t)kbs * t.split / L.splits);
  t.kb1 = (uint32_t)((uint64_t)kbs * (t.split + 1) / L.splits);
  return t;
}

// What a lane needs of a block of 32 rows and 16 columns besides the sums: four columns (lane mod 4) of the bias, and of the residual in
// four rows (lane / 4 + 8 i).  Asked for before the sums are there.
template <class Out> struct Ahead {
  float res[4][4];
  float bias[4];
  __device__ __forceinline__ void ask(const Launch& L, int lane, uint32_t m0, uint32_t n0) {
    const Epilogue& e = L.p.e;
    const uint32_t col = n0 + 4 * (lane & 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) bias[i] = 0.f;
    if (L.splits > 1 || col >= L.p.n) return;
    const int n = (int)min(4u, L.p.n - col);
    if (e.bias) load4(e.bias_type, e.bias, col, false, n, bias);
    if (!e.residual) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t row = m0 + 8 * i + lane / 4;
      if (row >= L.p.m) continue;
      const Out* r = static_cast<const Out*>(e.residual) + row * e.ld_res + col;
      load_n<Out, 4>(r, e.vec && n == 4, n, res[i]);
    }
  }
};
// A block of sums, a row per lane, through the warp's buffer to four lanes a row; then the epilogue (or the workspace).
template <class Out>
__device__ __forceinline__ void store_block(const Launch& L, uint32_t split, float4* buf, int lane, const float (&v)[kBlock], const Ahead<Out>& ahead,
                                            uint32_t m0, uint32_t n0) {
#pragma unroll
  for (int j = 0; j < 4; ++j) buf[lane * 4 + (j ^ (lane >> 1 & 3))] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
  __syncwarp();
  const Product& p = L.p;
  const int j = lane & 3;
  const uint32_t col = n0 + 4 * j;
  if (col < p.n) {
    const int n = (int)min(4u, p.n - col);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 8 * i + lane / 4;
      if (m0 + r >= p.m) continue;
      const float4 q = buf[r * 4 + (j ^ (r >> 1 & 3))];
      if (L.splits > 1) {
        *reinterpret_cast<float4*>(L.partial + ((size_t)split * p.m + m0 + r) * L.ld_partial + col) = q;
      } else {
        float z[4] = {q.x + ahead.bias[0], q.y + ahead.bias[1], q.z + ahead.bias[2], q.w + ahead.bias[3]}, res[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) res[k] = p.e.residual ? ahead.res[i][k] : 0.f;
        finish4<Out>(p.e, m0 + r, col, p.n, n, z, res);
      }
    }
  }
  __syncwarp();
}

template <class Out, int PLANES, int BN, int CG>
__global__ void __launch_bounds__((Ring<PLANES, BN, CG>::threads), 1) product_mma_kernel(const __grid_constant__ Launch L, const __grid_constant__ CUtensorMap map_a,
                                                                  const __grid_constant__ CUtensorMap map_b) {
  using R = Ring<PLANES, BN, CG>;
  extern __shared__ unsigned char raw[];
  const uint32_t base = (smem_u32(raw) + 1023) & ~1023u;
  unsigned char* sm = raw + (base - smem_u32(raw));
  float4* trans = reinterpret_cast<float4*>(sm + R::stages * R::stage);
  const uint32_t bars = base + R::stages * R::stage + R::trans;
  const uint32_t full = bars, empty = bars + 8 * R::stages, acc_full = bars + 16 * R::stages, acc_empty = acc_full + 16, slot = acc_empty + 16;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = CG == 1 ? 0 : blockIdx.x % CG;   // of the pair; the even CTA issues for both
  const uint32_t first = blockIdx.x / CG, step = gridDim.x / CG;
  const uint32_t kbs = (L.p.k + R::bk - 1) / R::bk, items = L.tiles_m * L.tiles_n * L.splits;
  constexpr uint32_t kCols = 2 * BN;

  if (threadIdx.x == 0) {
    for (int s = 0; s < R::stages; ++s) {
      bar_init(full + 8 * s, 1);
      bar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      bar_init(acc_full + 8 * b, 1);
      bar_init(acc_empty + 8 * b, R::epi_warps * CG);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<CG>(slot, kCols);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *reinterpret_cast<uint32_t*>(sm + (slot - base));

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (uint32_t item = first; item < items && ok; item += step) {
        const Tile t = tile_of(L, item, kbs);
        const int m0 = (int)(t.m * (128 * CG) + rank * 128), n0 = (int)(t.n * BN + rank * R::b_rows);
        for (uint32_t kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const uint32_t s = it % R::stages;
          ok = bar_wait(empty + 8 * s, (it / R::stages & 1) ^ 1);
          if (!ok) break;
          const uint32_t bar = CG == 1 ? full + 8 * s : in_cta(full + 8 * s, 0);
          if (rank == 0) bar_expect(full + 8 * s, R::stage * CG);
          const uint32_t at = base + s * R::stage;
          const int k0 = (int)(kb * R::bk);
#pragma unroll
          for (int q = 0; q < PLANES; ++q) {
            const uint32_t a = at + q * R::a_part, b = at + R::a_bytes + q * R::b_part;
            if (L.a_mn) {
              tma_load<CG>(a, &map_a, bar, m0, k0, q);
              tma_load<CG>(a + R::mn_block, &map_a, bar, m0 + 64, k0, q);
            } else {
              tma_load<CG>(a, &map_a, bar, k0, m0, q);
            }
            if (L.b_mn) {
#pragma unroll
              for (int c = 0; c < R::b_rows / 64; ++c) tma_load<CG>(b + c * R::mn_block, &map_b, bar, n0 + c * 64, k0, q);
            } else {
              tma_load<CG>(b, &map_b, bar, k0, n0, q);
            }
          }
        }
      }
      if (!ok && rank == 0) {   // given up: what is under way lands before the CTA leaves
        for (uint32_t i = it > R::stages ? it - R::stages : 0; i < it; ++i) bar_wait(full + 8 * (i % R::stages), i / R::stages & 1);
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, ac = 0;
      bool ok = true;
      const uint32_t a_step = L.a_mn ? 2048 >> 4 : 32 >> 4, b_step = L.b_mn ? 2048 >> 4 : 32 >> 4;
      for (uint32_t item = first; item < items && ok; item += step) {
        const Tile t = tile_of(L, item, kbs);
        for (uint32_t kb = t.kb0; kb < t.kb1 && ok; ++ac) {
          const uint32_t end = PLANES == 1 ? t.kb1 : min(kb + kChunk / R::bk, t.kb1);
          const uint32_t d = tmem + (ac & 1) * BN;
          ok = bar_wait(acc_empty + 8 * (ac & 1), (ac >> 1 & 1) ^ 1);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          uint32_t accumulate = 0;
          for (; kb < end; ++kb, ++it) {
            const uint32_t s = it % R::stages;
            ok = bar_wait(full + 8 * s, it / R::stages & 1);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t at = base + s * R::stage;
            const uint64_t da = tile_desc<R::bk>(at, L.a_mn), db = tile_desc<R::bk>(at + R::a_bytes, L.b_mn);
            if (PLANES == 1) {
#pragma unroll
              for (int k = 0; k < R::bk / 16; ++k) {
                mma<CG>(d, da + k * a_step, db + k * b_step, L.idesc, accumulate);
                accumulate = 1;
              }
            } else {
              // small products first: low x high and middle x middle, then middle x high, then high x high
              constexpr int pa[6] = {2, 1, 0, 1, 0, 0}, pb[6] = {0, 1, 2, 0, 1, 0};
#pragma unroll
              for (int q = 0; q < 6; ++q)
#pragma unroll
                for (int k = 0; k < R::bk / 16; ++k) {
                  mma<CG>(d, da + pa[q] * (R::a_part >> 4) + k * a_step, db + pb[q] * (R::b_part >> 4) + k * b_step, L.idesc, accumulate);
                  accumulate = 1;
                }
            }
            commit<CG>(empty + 8 * s);
          }
          if (ok) commit<CG>(acc_full + 8 * (ac & 1));
        }
      }
    }
  } else {
    const int ew = warp - 2, part = ew / 4;
    const uint32_t lanes = (uint32_t)(warp % 4) * 32;      // the quarter of tensor memory this warp may read
    float4* buf = trans + ew * (32 * kBlock / 4);
    constexpr int kBlocks = R::cols / kBlock;
    uint32_t ac = 0;
    bool ok = true;
    for (uint32_t item = first; item < items; item += step) {
      const Tile t = tile_of(L, item, kbs);
      const uint32_t m0 = t.m * (128 * CG) + rank * 128 + lanes, n0 = t.n * BN + part * R::cols;
      const uint32_t at = tmem + (lanes << 16) + part * R::cols;
      Ahead<Out> ahead;
      if (PLANES == 1) {
        ahead.ask(L, lane, m0, n0);
        if (ok) ok = bar_wait(acc_full + 8 * (ac & 1), ac >> 1 & 1);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
        for (int c = 0; c < kBlocks; ++c) {
          uint32_t w[1][kBlock];
          tmem_ld(at + (ac & 1) * BN + c * kBlock, w[0]);
          tmem_wait(w);
          float v[kBlock];
#pragma unroll
          for (int i = 0; i < kBlock; ++i) v[i] = __uint_as_float(w[0][i]);
          if (c == kBlocks - 1) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(CG == 1 ? acc_empty + 8 * (ac & 1) : in_cta(acc_empty + 8 * (ac & 1), 0));
          }
          if (!ok) {
#pragma unroll
            for (int i = 0; i < kBlock; ++i) v[i] = CUDART_NAN_F;
          }
          store_block<Out>(L, t.split, buf, lane, v, ahead, m0, n0 + c * kBlock);
          if (c + 1 < kBlocks) ahead.ask(L, lane, m0, n0 + (c + 1) * kBlock);
        }
        ++ac;
      } else {
        float sum[kBlocks][kBlock];
#pragma unroll
        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
          for (int i = 0; i < kBlock; ++i) sum[c][i] = 0.f;
        for (uint32_t kb = t.kb0; kb < t.kb1; kb += kChunk / R::bk, ++ac) {
          if (ok) ok = bar_wait(acc_full + 8 * (ac & 1), ac >> 1 & 1);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
          for (int c = 0; c < kBlocks; c += 2) {
            uint32_t w[2][kBlock];
            tmem_ld(at + (ac & 1) * BN + c * kBlock, w[0]);
            tmem_ld(at + (ac & 1) * BN + (c + 1) * kBlock, w[1]);
            tmem_wait(w);
#pragma unroll
            for (int i = 0; i < kBlock; ++i) sum[c][i] += __uint_as_float(w[0][i]), sum[c + 1][i] += __uint_as_float(w[1][i]);
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) bar_arrive(CG == 1 ? acc_empty + 8 * (ac & 1) : in_cta(acc_empty + 8 * (ac & 1), 0));
        }
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) {
          if (!ok) {
#pragma unroll
            for (int i = 0; i < kBlock; ++i) sum[c][i] = CUDART_NAN_F;
          }
          ahead.ask(L, lane, m0, n0 + c * kBlock);
          store_block<Out>(L, t.split, buf, lane, sum[c], ahead, m0, n0 + c * kBlock);
        }
      }
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG > 1) {   // neither CTA of a pair leaves while the other's products or barriers reach into it
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1) tmem_free<CG>(tmem, kCols);
}

// The parts' sums of a split k, in their order, through the epilogue: four columns a thread.
template <class Out>
__global__ void __launch_bounds__(256) split_sums_kernel(const Product p, const float* partial, size_t ld, uint32_t splits) {
  const uint32_t per = (p.n + 3) / 4;
  const uint64_t g = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (g >= (uint64_t)per * p.m) return;
  const uint32_t row = (uint32_t)(g / per), col = (uint32_t)(g % per) * 4;
  const int n = (int)min(4u, p.n - col);
  float v[4] = {};
  if (p.e.bias) load4(p.e.bias_type, p.e.bias, col, false, n, v);
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (uint32_t q = 0; q < splits; ++q) {
    const float4 x = *reinterpret_cast<const float4*>(partial + ((size_t)q * p.m + row) * ld + col);
    s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
  }
  v[0] += s.x; v[1] += s.y; v[2] += s.z; v[3] += s.w;
  finish4<Out>(p.e, row, col, p.n, n, v);
}

// Rows of 16-bit elements onto a stride of whole 16 bytes, as they are (kPlanes 1), or fp32 rows as three bf16 planes.
// x = h + m + l: h holds the upper 8 bits of x (cut, so that it cannot overflow), m and l the rest to nearest; an x that is no
// number or infinite is all in h.
template <class T, int kPlanes>
__global__ void __launch_bounds__(256) planes_kernel(const T* src, size_t ld, uint16_t* dst, size_t ld_dst, size_t plane, uint32_t rows, uint32_t cols) {
  const uint32_t per = (uint32_t)(ld_dst / 8);
  const uint64_t g = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (g >= (uint64_t)per * rows) return;
  const size_t row = g / per;
  const uint32_t col = (uint32_t)(g % per) * 8;
  const T* s = src + row * ld + col;
  uint16_t* d = dst + row * ld_dst + col;
  const bool whole = col + 8 <= cols && (uintptr_t)s % 16 == 0;
  if (kPlanes == 1) {
    uint4 v;
    if (whole) {
      v = *reinterpret_cast<const uint4*>(s);
    } else {
      const uint16_t* q = reinterpret_cast<const uint16_t*>(s);
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (col + 2 * i < cols ? q[2 * i] : 0u) | (col + 2 * i + 1 < cols ? (uint32_t)q[2 * i + 1] : 0u) << 16;
      v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    *reinterpret_cast<uint4*>(d) = v;
  } else {
    float x[2][4];
    const float* f = reinterpret_cast<const float*>(s);
    load_n<float, 4>(f, whole, col < cols ? (int)min(4u, cols - col) : 0, x[0]);
    load_n<float, 4>(f + 4, whole, col + 4 < cols ? (int)min(4u, cols - col - 4) : 0, x[1]);
    store_parts<4>(d, plane, x[0]);
    store_parts<4>(d + 4, plane, x[1]);
  }
}

// The driver's encoder of tensor maps, asked for once (the library links the runtime alone).
using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                            const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder() {
  static std::atomic<void*> known{nullptr};
  void* f = known.load(std::memory_order_acquire);
  if (!f) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
    known.store(f, std::memory_order_release);
  }
  return reinterpret_cast<Encode>(f);
}

// [planes][outer][inner] elements, boxes of box_cols x box_rows.
cudaError_t encode(CUtensorMap* map, const MmaOperand& o, uint32_t type, uint32_t planes, uint64_t inner, uint64_t outer, uint32_t box_cols, uint32_t box_rows) {
  const Encode f = encoder();
  if (!f) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {inner, outer, planes}, strides[2] = {o.ld * 2, (planes > 1 ? o.plane : (outer * o.ld + 7) / 8 * 8) * 2};
  const cuuint32_t box[3] = {box_cols, box_rows, 1}, steps[3] = {1, 1, 1};
  const CUresult r = f(map, type == kF16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.p), dims, strides, box, steps,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <class Out, int PLANES, int BN, int CG>
cudaError_t run(const MmaProduct& m, cudaStream_t s) {
  using R = Ring<PLANES, BN, CG>;
  Launch L{};
  L.p = m.p;
  L.a_mn = m.a.mn; L.b_mn = m.b.mn;
  L.splits = m.shape.splits;
  L.partial = m.partial; L.ld_partial = ((size_t)m.p.n + 3) / 4 * 4;
  L.tiles_m = (m.p.m + 128 * CG - 1) / (128 * CG);
  L.tiles_n = (m.p.n + BN - 1) / BN;
  const uint32_t format = m.type == kF16 ? 0 : 1;
  L.idesc = (1u << 4) | (format << 7) | (format << 10) | (L.a_mn << 15) | (L.b_mn << 16) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(128 * CG >> 4) << 24);
  CUtensorMap ma, mb;
  cudaError_t e = L.a_mn ? encode(&ma, m.a, m.type, PLANES, m.p.m, m.p.k, 64, R::bk) : encode(&ma, m.a, m.type, PLANES, m.p.k, m.p.m, R::bk, 128);
  if (e == cudaSuccess)
    e = L.b_mn ? encode(&mb, m.b, m.type, PLANES, m.p.n, m.p.k, 64, R::bk) : encode(&mb, m.b, m.type, PLANES, m.p.k, m.p.n, R::bk, R::b_rows);
  if (e != cudaSuccess) return e;
  const auto kernel = product_mma_kernel<Out, PLANES, BN, CG>;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, R::total);
  if (e != cudaSuccess) return e;
  uint32_t slots = 0;
  e = clusters_at_once(CG, &slots);
  if (e != cudaSuccess) return e;
  const uint32_t items = L.tiles_m * L.tiles_n * L.splits;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((items < slots ? items : slots) * CG);
  cfg.blockDim = dim3(R::threads);
  cfg.dynamicSmemBytes = R::total;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CG;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kernel, L, ma, mb);
  if (e != cudaSuccess || L.splits == 1) return e;
  const uint64_t groups = (uint64_t)m.p.m * ((m.p.n + 3) / 4);
  split_sums_kernel<Out><<<(unsigned)((groups + 255) / 256), 256, 0, s>>>(L.p, L.partial, L.ld_partial, L.splits);
  return cudaGetLastError();
}

template <class Out, int PLANES>
cudaError_t run(const MmaProduct& m, cudaStream_t s) {
  if (m.shape.pair) return run<Out, PLANES, 256, 2>(m, s);
  return run<Out, PLANES, 128, 1>(m, s);
}

}  // namespace

MmaShape mma_shape(uint32_t planes, uint32_t m, uint32_t n, uint32_t k) {
  MmaShape r{};
  r.use = (uint64_t)m * n * k >= (uint64_t)1 << 26;
  if (!r.use) return r;
  const uint64_t pairs = (uint64_t)((m + 255) / 256) * ((n + 255) / 256);
  r.pair = pairs >= 74;
  const uint64_t tiles = r.pair ? pairs : (uint64_t)((m + 127) / 128) * ((n + 127) / 128), slots = r.pair ? 74 : 148;
  const uint64_t kbs = (k + 63) / 64;
  uint64_t splits = slots / tiles;                       // as many parts as there are SMs left, each with 256 of k and more
  if (splits > kbs / 4) splits = kbs / 4;
  if (splits > 32) splits = 32;
  r.splits = splits < 2 ? 1 : (uint32_t)splits;
  (void)planes;
  return r;
}
size_t mma_partial_floats(const MmaShape& s, uint32_t m, uint32_t n) { return s.splits > 1 ? (size_t)s.splits * m * (((size_t)n + 3) / 4 * 4) : 0; }

cudaError_t launch_product_mma(const MmaProduct& m, cudaStream_t s) {
  if (m.planes == 3) return run<float, 3>(m, s);
  if (m.p.e.out_type == kF32) return run<float, 1>(m, s);
  if (m.p.e.out_type == kBf16) return run<__nv_bfloat16, 1>(m, s);
  return run<__half, 1>(m, s);
}

cudaError_t launch_planes(uint32_t type, const void* src, size_t ld, void* dst, size_t ld_dst, size_t plane, uint32_t rows, uint32_t cols, cudaStream_t s) {
  const uint64_t groups = (uint64_t)rows * (ld_dst / 8);
  const unsigned grid = (unsigned)((groups + 255) / 256);
  if (type == kF32) planes_kernel<float, 3><<<grid, 256, 0, s>>>((const float*)src, ld, (uint16_t*)dst, ld_dst, plane, rows, cols);
  else planes_kernel<__nv_bfloat16, 1><<<grid, 256, 0, s>>>((const __nv_bfloat16*)src, ld, (uint16_t*)dst, ld_dst, plane, rows, cols);
  return cudaGetLastError();
}

}  // namespace layer
}  // namespace aet
