// Large fp32 products on the 5th-generation tensor cores: C = A B, through the layer's epilogue.
//
// An fp32 value is three bf16 values of 8 bits and more each; six products of parts give the product of the values to 2^-24 (the three
// left out are below that).  B's parts come from a pass of their own (launch_rows_copies; the weights, mostly, which are the smaller
// operand); A is taken as it is: TMA brings 32 of k by 128 rows of fp32, four warps take them apart in registers, a row a thread, and
// store the parts in tensor memory, from where tcgen05.mma reads its A operand.  So A's parts cost neither memory traffic nor shared-memory
// bandwidth: reading A (16 KB every 768 cycles of six products) and multiplying take about the same time where B has 128 columns.
//
// Swapped, C^T = B^T A^T: where A has fewer rows than B columns (few rows through a wide layer) the parts are A's and the weights are read
// once, as they are (64 x 4,096 x 4,096 25 us; 66 with a pass for the weights' parts).  A lane then has a column of C.
//
// One persistent CTA per SM: a thread for TMA, a thread that issues, four warps that take apart (some 230
// instructions a stage: more warps would leave fewer registers for the sums, which then spill), eight that take sums out.  Tensor cores
// cut the sums they form: sums of 64 of k (24 additions) leave tensor memory and are added up in registers in fp32.  Against 64 bits the
// rms error of 784 and 4,096 terms is 3.1e-7 and 3.4e-7 of the rms, with sums of 128 of k 7.3e-7, of 256 1.5e-6; fp32 FMAs have 3.5e-7 and 8.1e-7.
//
// A split k, the bounded waits and the order of tiles are those of layer_mma_kernel.cu.
#include "layer_mma.cuh"

namespace aet {
namespace layer {
namespace {

template <int BN>
struct Ring {
  static constexpr int bk = 32;     // of k in a stage
  static constexpr int chunk = 2;   // stages to a sum in tensor memory
  static constexpr int a_bytes = 128 * bk * 4, b_part = BN * bk * 2, stage = a_bytes + 3 * b_part;
  static constexpr int a_block = 32 * bk * 4, b_block = 64 * bk * 2;       // 32 rows of A, 64 of B's columns, laid out across k
  static constexpr int epi_warps = 8, conv_warps = 4, threads = 64 + 32 * (epi_warps + conv_warps);
  static constexpr int cols = BN / 2;                                      // columns a warp takes out
  static constexpr int trans = epi_warps * 32 * kBlock * 4, rest = 512;
  static constexpr int fit = (232448 - 1024 - trans - rest) / stage;
  static constexpr int stages = fit < 5 ? fit : 5;
  static constexpr int total = 1024 + stages * stage + trans + rest;
  static constexpr int a_cols = 3 * bk / 2;                                // tensor memory columns of a stage's A
  static_assert(stages >= 3 && 2 * BN + stages * a_cols <= 512, "no ring");
};

// Sixteen words a lane into the warp's rows.
__device__ __forceinline__ void tmem_st(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
               "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// (the descriptor's halves apart: only the lower one, with the address, changes)
__device__ __forceinline__ void mma_a_tmem(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 b, {%2, %3};\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}

template <int BN, bool kSwapped>
__global__ void __launch_bounds__((Ring<BN>::threads), 1) product_f32_kernel(const __grid_constant__ Launch L, const __grid_constant__ CUtensorMap map_a,
                                                                             const __grid_constant__ CUtensorMap map_b) {
  using R = Ring<BN>;
  extern __shared__ unsigned char raw[];
  const uint32_t base = (smem_u32(raw) + 1023) & ~1023u;
  unsigned char* sm = raw + (base - smem_u32(raw));
  float4* trans = reinterpret_cast<float4*>(sm + R::stages * R::stage);
  const uint32_t bars = base + R::stages * R::stage + R::trans;
  const uint32_t full = bars, empty = bars + 8 * R::stages, apart = bars + 16 * R::stages, acc_full = bars + 24 * R::stages, acc_empty = acc_full + 16,
                 slot = acc_empty + 16, drained = slot + 8;
  volatile uint32_t* gave_up = reinterpret_cast<uint32_t*>(sm + (drained + 8 - base));
  const unsigned long long ns = L.waits.ns;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t kbs = (L.p.k + R::bk - 1) / R::bk, items = L.tiles_m * L.tiles_n * L.splits;

  if (threadIdx.x == 0) {
    for (int s = 0; s < R::stages; ++s) {
      bar_init(full + 8 * s, 1);
      bar_init(empty + 8 * s, 1);
      bar_init(apart + 8 * s, 4);
    }
    for (int b = 0; b < 2; ++b) {
      bar_init(acc_full + 8 * b, 1);
      bar_init(acc_empty + 8 * b, R::epi_warps);
    }
    bar_init(drained, 1);
    *gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<1>(slot, 512);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *reinterpret_cast<uint32_t*>(sm + (slot - base)), tmem_a = tmem + 2 * BN;

  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0;
      bool ok = true;
      for (uint32_t item = blockIdx.x; item < items && ok; item += gridDim.x) {
        const Tile t = tile_of(L, item, kbs);
        const int m0 = (int)(t.m * 128), n0 = (int)(t.n * BN);
        for (uint32_t kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const uint32_t s = it % R::stages, bar = full + 8 * s, a = base + s * R::stage, b = a + R::a_bytes;
          ok = bar_wait(empty + 8 * s, (it / R::stages & 1) ^ 1, ns) && (blockIdx.x || it < L.waits.stages);
          if (!ok) break;
          bar_expect(bar, R::stage);
          const int k0 = (int)(kb * R::bk);
          if (L.a_mn) {
#pragma unroll
            for (int c = 0; c < 4; ++c) tma_load<1>(a + c * R::a_block, &map_a, bar, m0 + 32 * c, k0, 0);
          } else {
            tma_load<1>(a, &map_a, bar, k0, m0, 0);
          }
          if (L.b_mn) {
#pragma unroll
            for (int c = 0; c < BN / 64; ++c) tma_load<1>(b + 3 * c * R::b_block, &map_b, bar, n0 + c * 64, k0, 0);
          } else {
            tma_load<1>(b, &map_b, bar, k0, n0, 0);
          }
        }
      }
      if (!ok) {   // what is under way lands before the CTA leaves
        *gave_up = 1;
        for (uint32_t i = it > R::stages ? it - R::stages : 0; i < it; ++i)
          if (!bar_wait(full + 8 * (i % R::stages), i / R::stages & 1, ns)) break;
      }
    }
  } else if (warp == 1) {
    if (elect_one()) {
      uint32_t it = 0, ac = 0;
      bool ok = true;
      const uint32_t b_step = L.b_mn ? 2048 >> 4 : 32 >> 4, b_plane = (L.b_mn ? R::b_block : R::b_part) >> 4;     // of k, of the parts
      for (uint32_t item = blockIdx.x; item < items && ok; item += gridDim.x) {
        const Tile t = tile_of(L, item, kbs);
        for (uint32_t kb = t.kb0; kb < t.kb1 && ok; ++ac) {
          const uint32_t end = min(kb + R::chunk, t.kb1), d = tmem + (ac & 1) * BN;
          ok = bar_wait(acc_empty + 8 * (ac & 1), (ac >> 1 & 1) ^ 1, ns);
          if (!ok) break;
          uint32_t accumulate = 0;
          for (; kb < end; ++kb, ++it) {
            const uint32_t s = it % R::stages;
            ok = bar_wait(full + 8 * s, it / R::stages & 1, ns) && bar_wait(apart + 8 * s, it / R::stages & 1, ns);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t a = tmem_a + s * R::a_cols;
            const uint64_t b = tile_desc<R::bk, 3>(base + s * R::stage + R::a_bytes, L.b_mn);
            // small products first: low x high and middle x middle, then middle x high, then high x high
            constexpr int pa[6] = {2, 1, 0, 1, 0, 0}, pb[6] = {0, 1, 2, 0, 1, 0};
#pragma unroll
            for (int q = 0; q < 6; ++q)
#pragma unroll
              for (int k = 0; k < R::bk / 16; ++k) {
                mma_a_tmem(d, a + pa[q] * (R::bk / 2) + k * 8, (uint32_t)b + pb[q] * b_plane + k * b_step, (uint32_t)(b >> 32), L.idesc, accumulate);
                accumulate = 1;
              }
            commit<1>(empty + 8 * s);
          }
          if (ok) commit<1>(acc_full + 8 * (ac & 1));
        }
      }
      if (!ok) *gave_up = 1;
      commit<1>(drained);
    }
  } else if (warp < 2 + R::epi_warps) {
    const int ew = warp - 2;
    const uint32_t lanes = (uint32_t)(warp % 4) * 32;      // the quarter of tensor memory this warp may read
    float4* buf = trans + ew * (32 * kBlock / 4);
    constexpr int kBlocks = R::cols / kBlock;
    uint32_t ac = 0;
    bool ok = true;
    for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
      const Tile t = tile_of(L, item, kbs);
      const uint32_t m0 = t.m * 128 + lanes, n0 = t.n * BN + ew / 4 * R::cols, at = tmem + (lanes << 16) + ew / 4 * R::cols;
      float sum[kBlocks][kBlock];
#pragma unroll
      for (int c = 0; c < kBlocks; ++c)
#pragma unroll
        for (int i = 0; i < kBlock; ++i) sum[c][i] = 0.f;
      for (uint32_t kb = t.kb0; kb < t.kb1; kb += R::chunk, ++ac) {
        if (ok) {
          ok = __all_sync(~0u, bar_wait(acc_full + 8 * (ac & 1), ac >> 1 & 1, ns));
          if (!ok) *gave_up = 1;      // (from here on nothing is handed back either: the others may still take sums out)
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) {
          uint32_t w[1][kBlock];
          tmem_ld(at + (ac & 1) * BN + c * kBlock, w[0]);
          tmem_wait(w);
#pragma unroll
          for (int i = 0; i < kBlock; ++i) sum[c][i] += __uint_as_float(w[0][i]);
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0 && ok) bar_arrive(acc_empty + 8 * (ac & 1));
      }
#pragma unroll
      for (int c = 0; c < kBlocks; ++c) {
        if (!ok) {
#pragma unroll
          for (int i = 0; i < kBlock; ++i) sum[c][i] = CUDART_NAN_F;
        }
        if (kSwapped) {       // a lane has a column of C, and its registers the rows: lanes store neighbours as they are
          const uint32_t col = m0 + lane;
          if (col < L.p.n) {
#pragma unroll
            for (int i = 0; i < kBlock; ++i) {
              const uint32_t row = n0 + c * kBlock + i;
              if (row >= L.p.m) break;
              if (L.splits > 1) L.partial[((size_t)t.split * L.p.m + row) * L.ld_partial + col] = sum[c][i];
              else finish1<float>(L.p.e, row, col, L.p.n, sum[c][i]);
            }
          }
        } else {
          Ahead<float> ahead;
          ahead.ask(L, lane, m0, n0 + c * kBlock);
          store_block<float>(L, t.split, buf, lane, sum[c], ahead, m0, n0 + c * kBlock);
        }
      }
    }
  } else {
    // takes A apart
    const uint32_t row = (uint32_t)(warp % 4) * 32 + lane;
    bool ok = true;
    uint32_t it = 0;
    for (uint32_t item = blockIdx.x; item < items && ok; item += gridDim.x) {
      const Tile t = tile_of(L, item, kbs);
      for (uint32_t kb = t.kb0; kb < t.kb1; ++kb, ++it) {
        const uint32_t s = it % R::stages;
        ok = bar_wait(full + 8 * s, it / R::stages & 1, ns);
        if (!__all_sync(~0u, ok)) { ok = false, *gave_up = 1; break; }
        const unsigned char* a = sm + s * R::stage;
        uint32_t h[16], m[16], l[16];
        if (L.a_mn) {
          const unsigned char* col = a + row / 32 * R::a_block + row % 4 * 4;
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            const float x0 = *reinterpret_cast<const float*>(col + k * 128 + ((row % 32 / 4) ^ (k & 7)) * 16);
            const float x1 = *reinterpret_cast<const float*>(col + (k + 1) * 128 + ((row % 32 / 4) ^ ((k + 1) & 7)) * 16);
            three_parts(x0, x1, h[k / 2], m[k / 2], l[k / 2]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float4 x = *reinterpret_cast<const float4*>(a + row * 128 + (j ^ (row & 7)) * 16);
            three_parts(x.x, x.y, h[2 * j], m[2 * j], l[2 * j]);
            three_parts(x.z, x.w, h[2 * j + 1], m[2 * j + 1], l[2 * j + 1]);
          }
        }
        const uint32_t to = tmem_a + ((row & ~31u) << 16) + s * R::a_cols;
        tmem_st(to, h);
        tmem_st(to + 16, m);
        tmem_st(to + 32, l);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive(apart + 8 * s);
      }
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 1) drain(drained, *gave_up != 0, ns);
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1) tmem_free<1>(tmem, 512);
}

template <int BN, bool kSwapped>
cudaError_t run(const MmaProduct& m, cudaStream_t s) {
  using R = Ring<BN>;
  const uint32_t rows = kSwapped ? m.p.n : m.p.m, cols = kSwapped ? m.p.m : m.p.n;     // of the product as the tensor cores see it
  Launch L{};
  L.p = m.p;
  L.a_mn = m.a.mn; L.b_mn = m.b.mn;
  L.waits = m.waits;
  L.splits = m.shape.splits;
  L.partial = m.partial; L.ld_partial = ((size_t)m.p.n + 3) / 4 * 4;
  L.tiles_m = (rows + 127) / 128;
  L.tiles_n = (cols + BN - 1) / BN;
  L.idesc = (1u << 4) | (1u << 7) | (1u << 10) | (L.b_mn << 16) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
  CUtensorMap ma, mb;
  cudaError_t e = L.a_mn ? encode(&ma, m.a, kF32, 1, rows, m.p.k, 32, R::bk) : encode(&ma, m.a, kF32, 1, m.p.k, rows, R::bk, 128);
  if (e == cudaSuccess) e = L.b_mn ? encode(&mb, m.b, kBf16, 3, cols, m.p.k, 64, R::bk) : encode(&mb, m.b, kBf16, 3, m.p.k, cols, R::bk, BN);
  if (e != cudaSuccess) return e;
  const auto kernel = product_f32_kernel<BN, kSwapped>;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, R::total);
  if (e != cudaSuccess) return e;
  uint32_t slots = 0;
  e = clusters_at_once(1, &slots);
  if (e != cudaSuccess) return e;
  const uint32_t items = L.tiles_m * L.tiles_n * L.splits;
  e = launch_alone(kernel, dim3(items < slots ? items : slots), R::threads, R::total, 1, s, L, ma, mb);
  if (e != cudaSuccess || L.splits == 1) return e;
  const uint64_t groups = (uint64_t)m.p.m * ((m.p.n + 3) / 4);
  return launch(split_sums_kernel<float>, dim3((unsigned)((groups + 255) / 256)), 256, 0, 1, s, L.p, L.partial, L.ld_partial, L.splits);
}

}  // namespace

// 64 columns at a time where there are no more (a tile of 128 would multiply zeros half of the time)
cudaError_t launch_product_f32(const MmaProduct& m, cudaStream_t s) {
  if (m.swapped) return m.p.m <= 64 ? run<64, true>(m, s) : run<128, true>(m, s);
  return m.p.n <= 64 ? run<64, false>(m, s) : run<128, false>(m, s);
}

}  // namespace layer
}  // namespace aet
