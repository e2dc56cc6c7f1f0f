// What the kernels on the tensor cores share: barriers, TMA, tcgen05, the order of tiles, and the way out of tensor memory.
#pragma once
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

constexpr uint32_t kGroup = 16;     // tile rows that are walked together, so that their operands meet in L2

struct Launch {
  Product p;            // a, b and their strides are in the tensor maps
  float* partial;       // [splits, m, ld_partial] where k is split
  size_t ld_partial;
  uint32_t a_mn, b_mn;  // laid out across k
  uint32_t splits, tiles_m, tiles_n, idesc;
  Waits waits;
};

// One lane of the warp, as the compiler knows: what only it does is kept in uniform registers, where tcgen05.mma takes its operands from.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count)); }
// Waits, but not for ever (Waits says how long: the longest wait there is, for the sums of 2^17 of k, takes some 3 ms).
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, unsigned long long most_ns) {
  unsigned long long from = 0;
  for (uint32_t i = 1;; ++i) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred q;\n\tmbarrier.try_wait.parity.shared::cta.b64 q, [%1], %2;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok) return true;
    if (i % 1024 == 0) {
      unsigned long long now;
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
      if (!from) from = now;
      if (now - from > most_ns) return false;
    }
  }
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Arrives on a barrier of the CTA, or of the pair (an address of in_cta).  What is handed over is tensor memory that has been read, behind a
// wait and a tcgen05 fence, and nothing in ordinary memory: the pair's arrival is relaxed, since a release at cluster scope waits for the
// thread's stores to global memory (half of the stalls in the fp32 kernel when it was one).
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_arrive_pair(uint32_t bar) { asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
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
// In front of the end of a CTA, by the warp that frees tensor memory, when all its roles are done: the products that were issued read shared
// memory and write tensor memory until `drained` says that they are through, also where the roles that wait for sums have given up.  Then
// copies whose barrier nobody waits for any more may be under way too; they land within some microseconds.
__device__ __forceinline__ void drain(uint32_t drained, bool gave_up, unsigned long long most_ns) {
  bar_wait(drained, 0, most_ns);
  if (gave_up) {
    unsigned long long from, now;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(from));
    for (int i = 0; i < 1 << 20; ++i) {
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
      if (now - from > 100000) break;
    }
  }
  __syncwarp();
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
// Across k: 128-byte rows of 64 of M or N, bk of them to a block, blocks one after another (of as many planes), in them 8 of k every 1,024 bytes.
template <int bk, int planes = 1>
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, bool mn) {
  const uint32_t lead = mn ? planes * 64 * bk * 2 : 16, stride = mn || bk == 64 ? 1024 : 512;
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

// The parts' sums of a split k, in their order, through the epilogue: four columns a thread.
template <class Out>
__global__ void __launch_bounds__(256) split_sums_kernel(const Product p, const float* partial, size_t ld, uint32_t splits) {
  in_line();
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

// The driver's encoder of tensor maps, asked for once (the library links the runtime alone).
using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                            const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline Encode encoder() {
  static std::atomic<void*> known{nullptr};
  void* f = known.load(std::memory_order_acquire);
  if (!f) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
    known.store(f, std::memory_order_release);
  }
  return reinterpret_cast<Encode>(f);
}

// [planes][outer][inner] elements, boxes of box_cols x box_rows of all planes, swizzled as wide as a box's rows (128 or 64 bytes).
inline cudaError_t encode(CUtensorMap* map, const MmaOperand& o, uint32_t type, uint32_t planes, uint64_t inner, uint64_t outer, uint32_t box_cols,
                          uint32_t box_rows) {
  const Encode f = encoder();
  if (!f) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {inner, outer, planes}, size = type == kF32 ? 4 : 2;
  const cuuint64_t strides[2] = {o.ld * size, (planes > 1 ? o.plane * size : (outer * o.ld * size + 15) / 16 * 16)};
  const cuuint32_t box[3] = {box_cols, box_rows, planes}, steps[3] = {1, 1, 1};
  const CUresult r = f(map, type == kF32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type == kF16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.p), dims, strides, box, steps,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, box_cols * size == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace
}  // namespace layer
}  // namespace aet
