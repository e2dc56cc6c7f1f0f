// Large products of 16-bit operands on the 5th-generation tensor cores: C = A B, sums in tensor memory, through the layer's epilogue.
//
// One persistent CTA per SM (or a pair of CTAs on two) walks over output tiles of 128 rows a CTA and BN columns.  One thread feeds a
// ring of stages by TMA (64 of k each, 128-byte swizzle), one issues tcgen05.mma, the others take finished sums out of tensor memory
// through a transposing buffer, so that rows are stored in whole sectors, while the next tile's products run into the other half of
// tensor memory.  Either operand may be laid out along k or across it: TMA brings 64 x 64 blocks either way and the matrix
// descriptors say which, so that the gradients' transposed products read the tensors as they are.
//
// Few tiles, or a very long k: k is split, the parts' sums go to the workspace and a second kernel adds them up in their order.
//
// Every wait is bounded; a role whose wait has given up stops issuing, and tiles that were not summed are stored as NaN.
#include "layer_mma.cuh"

namespace aet {
namespace layer {
namespace {

template <int BN, int CG>
struct Ring {
  static constexpr int bk = 64;     // of k in a stage
  static constexpr int b_rows = BN / CG;
  static constexpr int a_bytes = 128 * bk * 2, stage = a_bytes + b_rows * bk * 2, mn_block = 64 * bk * 2;
  static constexpr int epi_warps = 16, threads = 64 + 32 * epi_warps;    // four to a quarter of tensor memory: they wait for memory most of the time
  static constexpr int cols = BN / (epi_warps / 4);                      // columns a warp takes
  static constexpr int trans = epi_warps * 32 * kBlock * 4, rest = 512;
  static constexpr int fit = (232448 - 1024 - trans - rest) / stage;
  static constexpr int stages = fit < 6 ? fit : 6;
  static constexpr int total = 1024 + stages * stage + trans + rest;
  static_assert(stages >= 2, "no ring");
};

template <class Out, int BN, int CG>
__global__ void __launch_bounds__((Ring<BN, CG>::threads), 1) product_mma_kernel(const __grid_constant__ Launch L, const __grid_constant__ CUtensorMap map_a,
                                                                  const __grid_constant__ CUtensorMap map_b) {
  using R = Ring<BN, CG>;
  extern __shared__ unsigned char raw[];
  const uint32_t base = (smem_u32(raw) + 1023) & ~1023u;
  unsigned char* sm = raw + (base - smem_u32(raw));
  float4* trans = reinterpret_cast<float4*>(sm + R::stages * R::stage);
  const uint32_t bars = base + R::stages * R::stage + R::trans;
  const uint32_t full = bars, empty = bars + 8 * R::stages, acc_full = bars + 16 * R::stages, acc_empty = acc_full + 16, slot = acc_empty + 16,
                 drained = slot + 8;
  volatile uint32_t* gave_up = reinterpret_cast<uint32_t*>(sm + (drained + 8 - base));
  const unsigned long long ns = L.waits.ns;
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
    bar_init(drained, 1);
    *gave_up = 0;
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
    if (elect_one()) {
      uint32_t it = 0;
      bool ok = true;
      for (uint32_t item = first; item < items && ok; item += step) {
        const Tile t = tile_of(L, item, kbs);
        const int m0 = (int)(t.m * (128 * CG) + rank * 128), n0 = (int)(t.n * BN + rank * R::b_rows);
        for (uint32_t kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const uint32_t s = it % R::stages;
          ok = bar_wait(empty + 8 * s, (it / R::stages & 1) ^ 1, ns) && (first || it < L.waits.stages);
          if (!ok) break;
          const uint32_t bar = CG == 1 ? full + 8 * s : in_cta(full + 8 * s, 0);
          if (rank == 0) bar_expect(full + 8 * s, R::stage * CG);
          const uint32_t at = base + s * R::stage;
          const int k0 = (int)(kb * R::bk);
          const uint32_t b = at + R::a_bytes;
          if (L.a_mn) {
            tma_load<CG>(at, &map_a, bar, m0, k0, 0);
            tma_load<CG>(at + R::mn_block, &map_a, bar, m0 + 64, k0, 0);
          } else {
            tma_load<CG>(at, &map_a, bar, k0, m0, 0);
          }
          if (L.b_mn) {
#pragma unroll
            for (int c = 0; c < R::b_rows / 64; ++c) tma_load<CG>(b + c * R::mn_block, &map_b, bar, n0 + c * 64, k0, 0);
          } else {
            tma_load<CG>(b, &map_b, bar, k0, n0, 0);
          }
        }
      }
      if (!ok) *gave_up = 1;
      if (!ok && rank == 0) {   // what is under way lands before the CTA leaves
        for (uint32_t i = it > R::stages ? it - R::stages : 0; i < it; ++i)
          if (!bar_wait(full + 8 * (i % R::stages), i / R::stages & 1, ns)) break;
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) {
      uint32_t it = 0, ac = 0;
      bool ok = true;
      const uint32_t a_step = L.a_mn ? 2048 >> 4 : 32 >> 4, b_step = L.b_mn ? 2048 >> 4 : 32 >> 4;
      for (uint32_t item = first; item < items && ok; item += step) {
        const Tile t = tile_of(L, item, kbs);
        const uint32_t d = tmem + (ac & 1) * BN;
        ok = bar_wait(acc_empty + 8 * (ac & 1), (ac >> 1 & 1) ^ 1, ns);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        uint32_t accumulate = 0;
        for (uint32_t kb = t.kb0; kb < t.kb1; ++kb, ++it) {
          const uint32_t s = it % R::stages;
          ok = bar_wait(full + 8 * s, it / R::stages & 1, ns);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t at = base + s * R::stage;
          const uint64_t da = tile_desc<R::bk>(at, L.a_mn), db = tile_desc<R::bk>(at + R::a_bytes, L.b_mn);
#pragma unroll
          for (int k = 0; k < R::bk / 16; ++k) {
            mma<CG>(d, da + k * a_step, db + k * b_step, L.idesc, accumulate);
            accumulate = 1;
          }
          commit<CG>(empty + 8 * s);
        }
        if (ok) commit<CG>(acc_full + 8 * (ac & 1));
        ++ac;
      }
      if (!ok) *gave_up = 1;
      commit<CG>(drained);
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
      ahead.ask(L, lane, m0, n0);
      if (ok) {
        ok = __all_sync(~0u, bar_wait(acc_full + 8 * (ac & 1), ac >> 1 & 1, ns));
        if (!ok) *gave_up = 1;      // (from here on nothing is handed back either: the others may still take sums out)
      }
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
          if (lane == 0 && ok) {
            if (CG == 1) bar_arrive(acc_empty + 8 * (ac & 1));
            else bar_arrive_pair(in_cta(acc_empty + 8 * (ac & 1), 0));
          }
        }
        if (!ok) {
#pragma unroll
          for (int i = 0; i < kBlock; ++i) v[i] = CUDART_NAN_F;
        }
        store_block<Out>(L, t.split, buf, lane, v, ahead, m0, n0 + c * kBlock);
        if (c + 1 < kBlocks) ahead.ask(L, lane, m0, n0 + (c + 1) * kBlock);
      }
      ++ac;
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 1) drain(drained, *gave_up != 0, ns);
  if (CG > 1) {   // neither CTA of a pair leaves while the other's products or barriers reach into it
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1) tmem_free<CG>(tmem, kCols);
}

template <class Out, int BN, int CG>
cudaError_t run(const MmaProduct& m, cudaStream_t s) {
  using R = Ring<BN, CG>;
  Launch L{};
  L.p = m.p;
  L.a_mn = m.a.mn; L.b_mn = m.b.mn;
  L.waits = m.waits;
  L.splits = m.shape.splits;
  L.partial = m.partial; L.ld_partial = ((size_t)m.p.n + 3) / 4 * 4;
  L.tiles_m = (m.p.m + 128 * CG - 1) / (128 * CG);
  L.tiles_n = (m.p.n + BN - 1) / BN;
  const uint32_t format = m.type == kF16 ? 0 : 1;
  L.idesc = (1u << 4) | (format << 7) | (format << 10) | (L.a_mn << 15) | (L.b_mn << 16) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(128 * CG >> 4) << 24);
  CUtensorMap ma, mb;
  cudaError_t e = L.a_mn ? encode(&ma, m.a, m.type, 1, m.p.m, m.p.k, 64, R::bk) : encode(&ma, m.a, m.type, 1, m.p.k, m.p.m, R::bk, 128);
  if (e == cudaSuccess)
    e = L.b_mn ? encode(&mb, m.b, m.type, 1, m.p.n, m.p.k, 64, R::bk) : encode(&mb, m.b, m.type, 1, m.p.k, m.p.n, R::bk, R::b_rows);
  if (e != cudaSuccess) return e;
  const auto kernel = product_mma_kernel<Out, BN, CG>;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, R::total);
  if (e != cudaSuccess) return e;
  uint32_t slots = 0;
  e = clusters_at_once(CG, &slots);
  if (e != cudaSuccess) return e;
  const uint32_t items = L.tiles_m * L.tiles_n * L.splits;
  e = launch_alone(kernel, dim3((items < slots ? items : slots) * CG), R::threads, R::total, CG, s, L, ma, mb);
  if (e != cudaSuccess || L.splits == 1) return e;
  const uint64_t groups = (uint64_t)m.p.m * ((m.p.n + 3) / 4);
  return launch(split_sums_kernel<Out>, dim3((unsigned)((groups + 255) / 256)), 256, 0, 1, s, L.p, L.partial, L.ld_partial, L.splits);
}

template <class Out>
cudaError_t run(const MmaProduct& m, cudaStream_t s) {
  return m.shape.pair ? run<Out, 256, 2>(m, s) : run<Out, 128, 1>(m, s);
}

}  // namespace

// The tensor cores take a product from so many multiplications on (in whole tiles of the FMA kernel), and one whose tiles are so few that
// that kernel's clusters would go down more than 512 of k each.  Both kernels in us on either side: bf16 256^3 (2^24) 7.7 here, 6.9 there,
// 512 x 512 x 256 (2^26) 9.2 and 12.8; fp32, which needs a pass for the parts and six products, 512 x 512 x 256 18.4 and 12.0, 512^3 (2^27)
// 19.0 and 19.5; fp32 60,000 x 128 x 10, in whole tiles 2^28.9, 19.5 and 47.
bool mma_takes(uint32_t type, uint32_t m, uint32_t n, uint32_t k) {
  return fma_volume(m, n, k) >= (type == kF32 ? 1ull << 27 : 1ull << 25) || k / fma_split(m, n, k) > 512;
}
constexpr uint64_t kMostBlocks = (1u << 17) / 64;
MmaShape mma_shape(uint32_t type, uint32_t m, uint32_t n, uint32_t k) {
  MmaShape r{};
  const uint64_t pairs = (uint64_t)((m + 255) / 256) * ((n + 255) / 256);
  r.pair = type != kF32 && pairs >= 74;
  const uint64_t cols = type == kF32 && n <= 64 ? 64 : 128;
  const uint64_t tiles = r.pair ? pairs : ((uint64_t)m + 127) / 128 * ((n + cols - 1) / cols), slots = r.pair ? 74 : 148;
  const uint64_t kbs = ((uint64_t)k + 63) / 64;
  uint64_t splits = slots / tiles;                       // as many parts as there are SMs left, each with 256 of k (fp32: 128) and more
  const uint64_t least = type == kF32 ? 2 : 4;
  if (splits > kbs / least) splits = kbs / least;
  if (splits > 32) splits = 32;
  // At most 2^17 of k in a sum: the tensor cores cut what they add, 16 of k at a time, so that a long sum of one sign falls behind (0.6 of 2^-24
  // of it every time: 2.4 % over 2^22 rows, 19 % over 2^31 in 32 parts); over 2^17 it is 3e-4, well below a rounding to 16 bits.
  const uint64_t need = (kbs + kMostBlocks - 1) / kMostBlocks;
  if (splits < need) splits = need;
  r.splits = splits < 2 ? 1 : (uint32_t)splits;
  return r;
}
size_t mma_partial_floats(const MmaShape& s, uint32_t m, uint32_t n) { return s.splits > 1 ? (size_t)s.splits * m * (((size_t)n + 3) / 4 * 4) : 0; }

cudaError_t launch_product_mma(const MmaProduct& m, cudaStream_t s) {
  if (m.type == kF32) return launch_product_f32(m, s);
  if (m.p.e.out_type == kF32) return run<float>(m, s);
  if (m.p.e.out_type == kBf16) return run<__nv_bfloat16>(m, s);
  return run<__half>(m, s);
}

}  // namespace layer
}  // namespace aet
