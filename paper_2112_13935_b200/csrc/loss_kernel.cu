// Softmax cross-entropy of rows of logits z with class y: loss = log sum_j exp(z_j) - z_y, its gradient
// scale * weight * (softmax(z) - 1_y), and the lowest index of the row's maximum.
//
// Bound by memory: each logit is read once and each gradient written once.  A row stays with those who read it: 4 to 32 lanes of a warp
// (short rows, several to a warp), a CTA, or a cluster of up to eight CTAs, in 16-byte pieces as they lie in memory (those of CTAs wait in
// shared memory).  The maximum m comes first, over lanes and warps, then the sum of exp(z - m); the CTAs of a cluster join both by one
// push into the others' shared memory; then the gradient is formed.  Several CTAs share an SM, so that one's loads run under another's
// stores.  A thread takes up to sixteen pieces, counted as if its row started anywhere, so that aligned rows of a power of two of logits
// get one step more CTAs than they would need, which is about even: 8,192 rows of 65,536 bf16 logits, eight pieces a thread, 395 us in a graph
// (5.4 TB/s), with sixteen 406; 16,384 rows of 32,768 381 and 375.  Rows too long for a cluster (1.6 MB) are read again, from L2 as far as
// they fit there.
// Rows may start at any element: the pieces are those of the 16-byte grid, and what they hold besides the row counts as -inf.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <math_constants.h>

#include "layer_common.cuh"

namespace cg = cooperative_groups;

namespace aet {
namespace layer {
namespace {

constexpr int kThreads = 256, kNone = 0x7fffffff;

// Exponentials are powers of two: e^(z - m) as 2^(c z - t), one fused multiply-add and one instruction of the special function unit each,
// with c = log2 e and t = c m rounded.  The maximum's own exponent is then t's rounding, which all the row's sum shares and which is put right
// where a sum becomes a loss, so that only z - m enters the error, with 2^-24.  That holds while the rounding is small: up to |m| = 2^20 it
// is 2^-4 at most.  At 1e10 it would be 440, and a row masked with -1e10 had the sum inf.  A maximum further out is subtracted first,
// 2^((z - m) c), with no rounding of its own and one instruction more; the difference of two fp32 values that matters is exact there.
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float exp2_of(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
struct Base { float t; bool far; };
__device__ __forceinline__ bool far_out(float top) { return fabsf(top) > 0x1p20f && !isinf(top); }
__device__ __forceinline__ Base base_of(float top) {
  const bool far = far_out(top);
  return Base{isinf(top) ? 0.f : far ? top : __fmul_rn(top, kLog2e), far};
}
template <bool kFar> __device__ __forceinline__ float power(float z, float t) { return exp2_of(kFar ? (z - t) * kLog2e : fmaf(z, kLog2e, -t)); }
// What is done with a row's powers, one way or the other: asked once a row, since a branch in the loops over pieces cost 2 % of long rows.
template <class F> __device__ __forceinline__ void by_base(const Base& b, const F& f) {
  if (b.far) f(std::true_type{});
  else f(std::false_type{});
}
// The maximum's own exponent by its base.
__device__ __forceinline__ float excess(float top) { return far_out(top) || isinf(top) ? 0.f : fmaf(top, kLog2e, -__fmul_rn(top, kLog2e)); }
// What a sum by the base of maximum `top` is multiplied by to be one by that of a maximum `to` that is not below it.
__device__ __forceinline__ float rebase(float top, float to) {
  return exp2_of(far_out(top) || far_out(to) || isinf(to) ? (top - to) * kLog2e + (excess(to) - excess(top)) : __fmul_rn(top, kLog2e) - __fmul_rn(to, kLog2e));
}
// What a part of a row says: its maximum, the first piece it stands in, and the sum of powers by the maximum's base.  The sum is NaN
// where a logit is and only there (a maximum that is infinite counts as zero); a row whose maximum is infinite has no loss: NaN.
struct Part { float top, sum; int32_t at; };
// Maximum, sum and minimum over N neighbouring lanes, the same in all of them.
template <int N> __device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int o = N / 2; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
  return v;
}
template <int N> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = N / 2; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}
template <int N> __device__ __forceinline__ int32_t lanes_min(int32_t v) {
#pragma unroll
  for (int o = N / 2; o; o >>= 1) v = min(v, __shfl_xor_sync(~0u, v, o));
  return v;
}

template <class T> constexpr int kV = 16 / (int)sizeof(T);     // elements of a piece

// The row as the 16-byte grid sees it: element j is number j + shift of its `count` pieces.
template <class T> struct Row {
  const uint4* pieces;
  int32_t shift, n, count;
  __device__ __forceinline__ Row(const T* z, uint32_t classes)
      : pieces(reinterpret_cast<const uint4*>((uintptr_t)z & ~(uintptr_t)15)), shift((int32_t)((uintptr_t)z % 16 / sizeof(T))), n((int32_t)classes),
        count((n + shift + kV<T> - 1) / kV<T>) {}
  __device__ __forceinline__ bool ragged(int32_t q) const { return (q == 0 && shift) || (q == count - 1 && (n + shift) % kV<T>); }
  __device__ __forceinline__ bool mine(int32_t j) const { return j >= 0 && j < n; }
};
// Piece q of the row, where there is one (below `end`); what is not of the row is -inf.
template <class T> __device__ __forceinline__ uint4 fetch(const Row<T>& r, int32_t q, int32_t end) {
  const uint32_t none = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u;
  uint4 v = make_uint4(none, none, none, none);
  if (q < end) v = __ldcs(r.pieces + q);
  return v;
}
template <class T> __device__ __forceinline__ void trim(const Row<T>& r, uint4& v, int32_t q) {
  if (!r.ragged(q)) return;
  float f[kV<T>];
  unpack<T, kV<T>>(v, f);
#pragma unroll
  for (int i = 0; i < kV<T>; ++i)
    if (!r.mine(q * kV<T> - r.shift + i)) f[i] = -CUDART_INF_F;
  v = pack<T, kV<T>>(f);
}
template <class T> __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {   // of the halves of a word; a NaN loses
  uint32_t r;
  if constexpr (std::is_same<T, __half>::value) asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <class T> __device__ __forceinline__ float largest(const uint4& v) {
  float f[kV<T>];
  if constexpr (sizeof(T) == 4) {
    unpack<T, kV<T>>(v, f);
    return fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3]));
  } else {
    const uint32_t m = max2<T>(max2<T>(v.x, v.y), max2<T>(v.z, v.w));
    unpack<T, kV<T>>(make_uint4(m, m, m, m), f);
    return fmaxf(f[0], f[1]);
  }
}
template <class T, bool kFar> __device__ __forceinline__ float powers(const uint4& v, float t) {
  float f[kV<T>], sum = 0.f;
  unpack<T, kV<T>>(v, f);
#pragma unroll
  for (int k = 0; k < kV<T>; ++k) sum += power<kFar>(f[k], t);
  return sum;
}

// What the gradient of a row is formed with; `whole`: its pieces lie on the 16-byte grid as the logits' do.
template <class T> struct Slope {
  T* g;
  Base b;
  float w, f, inv;
  int32_t y;
  bool whole;
  __device__ __forceinline__ Slope(const LossLaunch& p, size_t row, int32_t label, const Part& a, int32_t shift)
      : g(static_cast<T*>(p.grad) + row * p.ld_grad), b(base_of(a.top)), y(label) {
    inv = isinf(a.top) ? CUDART_NAN_F : 1.f / a.sum;
    f = (uint32_t)y < p.classes ? p.scale * (p.weight ? p.weight[row] : 1.f) : CUDART_NAN_F;
    w = f * inv;
    whole = ((uintptr_t)g / sizeof(T) + kV<T> - shift) % kV<T> == 0;
  }
};
template <bool kFar, class T> __device__ __forceinline__ void write_grad(const Row<T>& r, const uint4& q, int32_t at, const Slope<T>& s, bool whole) {
  const int32_t j = at * kV<T> - r.shift;
  float v[kV<T>];
  unpack<T, kV<T>>(q, v);
#pragma unroll
  for (int i = 0; i < kV<T>; ++i) v[i] = power<kFar>(v[i], s.b.t) * s.w;
  if (whole) {
    __stcs(reinterpret_cast<uint4*>(s.g + j), pack<T, kV<T>>(v));
  } else {
#pragma unroll
    for (int i = 0; i < kV<T>; ++i)
      if (r.mine(j + i)) s.g[j + i] = from_f32<T>(v[i]);
  }
}
// ... at the label, by the thread that has written its piece.
template <class T> __device__ __forceinline__ int32_t label_piece(const Row<T>& r, int32_t y) { return (uint32_t)y < (uint32_t)r.n ? (y + r.shift) / kV<T> : -1; }
template <class T> __device__ __forceinline__ void write_label(const Slope<T>& s, float zy) {
  s.g[s.y] = from_f32<T>(s.f * ((s.b.far ? power<true>(zy, s.b.t) : power<false>(zy, s.b.t)) * s.inv - 1.f));
}
// The loss, and -1 or 0 for a row without a first maximum (a NaN; -inf only); otherwise who holds its piece writes `top`.
__device__ __forceinline__ void write_loss(const LossLaunch& p, size_t row, const Part& a, float zy) {
  if (p.loss) p.loss[row] = isinf(a.top) ? CUDART_NAN_F : logf(a.sum) - kLn2 * excess(a.top) + (a.top - zy);
  if (p.top && (a.sum != a.sum || a.at == kNone)) p.top[row] = a.sum != a.sum ? -1 : 0;
}
template <class T> __device__ __forceinline__ void write_top(const LossLaunch& p, const Row<T>& r, size_t row, const Part& a, const uint4& q, int32_t at) {
  if (a.at != at || a.sum != a.sum) return;
  float v[kV<T>];
  unpack<T, kV<T>>(q, v);
  int32_t first = kNone;
#pragma unroll
  for (int i = kV<T> - 1; i >= 0; --i)
    if (v[i] == a.top) first = at * kV<T> - r.shift + i;
  p.top[row] = first;
}
template <class T> __device__ __forceinline__ float logit(const LossLaunch& p, const T* z, int32_t y) {
  return (uint32_t)y < p.classes ? to_f32(z[y]) : CUDART_NAN_F;
}
// A row without an answer is not read.
template <class T> __device__ __forceinline__ void no_answer(const LossLaunch& p, size_t row, uint32_t first, uint32_t step) {
  if (p.grad) {
    T* g = static_cast<T*>(p.grad) + row * p.ld_grad;
    const Row<T> r(g, p.classes);
    for (int32_t c = first; c < r.count; c += step) {
      if (!r.ragged(c)) {
        __stcs(reinterpret_cast<uint4*>(g + (c * kV<T> - r.shift)), make_uint4(0, 0, 0, 0));
      } else {
        for (int32_t j = c * kV<T> - r.shift, end = j + kV<T>; j < end; ++j)
          if (r.mine(j)) g[j] = from_f32<T>(0.f);
      }
    }
  }
  if (first == 0) {
    if (p.loss) p.loss[row] = 0.f;
    if (p.top) p.top[row] = -1;
  }
}

// Short rows: G lanes a row, NV pieces a lane.
template <class T, int G, int NV>
__global__ void __launch_bounds__(kThreads) loss_lanes_kernel(const LossLaunch p) {
  in_line();
  const size_t row = ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * (kThreads / G) + threadIdx.x / G;
  const int lane = threadIdx.x % G;
  const bool here = row < p.rows;
  const int32_t y = here ? p.labels[row] : -1;
  const T* z = static_cast<const T*>(p.logits) + (here ? row * p.ld : 0);
  const Row<T> r(z, p.classes);
  uint4 q[NV];
  float zy = 0.f, top = -CUDART_INF_F;
#pragma unroll
  for (int i = 0; i < NV; ++i) q[i] = fetch(r, lane + i * G, y < 0 ? 0 : r.count);
  if (y >= 0) zy = logit(p, z, y);
  int32_t at = kNone;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    trim(r, q[i], lane + i * G);
    const float m = largest<T>(q[i]);
    if (m > top) top = m, at = lane + i * G;
  }
  Part a;
  a.top = lanes_max<G>(top);
  a.at = p.top ? lanes_min<G>(top == a.top ? at : kNone) : 0;
  a.sum = 0.f;
  const Base b = base_of(a.top);
  by_base(b, [&](auto far) {
#pragma unroll
    for (int i = 0; i < NV; ++i) a.sum += powers<T, decltype(far)::value>(q[i], b.t);
  });
  a.sum = lanes_sum<G>(a.sum);
  __syncwarp();      // (the row has been read before its gradient may take its place)
  if (!here) return;
  if (y < 0) {
    no_answer<T>(p, row, lane, G);
    return;
  }
  if (lane == 0) write_loss(p, row, a, zy);
  if (p.top) {
#pragma unroll
    for (int i = 0; i < NV; ++i) write_top(p, r, row, a, q[i], lane + i * G);
  }
  if (p.grad) {
    const Slope<T> s(p, row, y, a, r.shift);
    by_base(s.b, [&](auto far) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (lane + i * G < r.count) write_grad<decltype(far)::value>(r, q[i], lane + i * G, s, s.whole && !r.ragged(lane + i * G));
    });
    const int32_t at = label_piece(r, y);
    if (at >= 0 && at % G == lane) write_label(s, zy);
  }
}

// Long rows: a cluster of CTAs (or one) a row.  The pieces wait in shared memory (kOnce; a thread reads back what it copied itself, so that
// nobody waits for anyone), where three short loops pass over them; in registers, eight pieces a thread were spilled (1.75 ms for the rows above).
template <class T, bool kOnce, int THREADS>
__global__ void __launch_bounds__(THREADS) loss_cluster_kernel(const LossLaunch p, const uint32_t log_width) {
  extern __shared__ uint4 mine[];
  __shared__ Part ctas[8];
  __shared__ float tops[THREADS / 32], sums[THREADS / 32];
  __shared__ int32_t firsts[THREADS / 32];
  in_line();
  // (width is a power of two; no division)
  const uint32_t width = 1u << log_width, rank = blockIdx.x & (width - 1);
  const size_t row = (size_t)blockIdx.y * (gridDim.x >> log_width) + (blockIdx.x >> log_width);
  if (row >= p.rows) return;      // (all CTAs of a cluster)
  const int tid = threadIdx.x;
  const int32_t y = p.labels[row];
  if (y < 0) {
    no_answer<T>(p, row, rank * THREADS + tid, width * THREADS);
    return;
  }
  if (width > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");    // I run: the others may push
  const T* z = static_cast<const T*>(p.logits) + row * p.ld;
  const Row<T> r(z, p.classes);
  const int32_t per = (r.count + (int32_t)width - 1) >> log_width, q0 = (int32_t)rank * per, q1 = min(r.count, q0 + per);
  if (kOnce) {
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine);
    for (int32_t c = q0 + tid; c < q1; c += THREADS)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 16 * (uint32_t)(c - q0)), "l"(r.pieces + c) : "memory");
    asm volatile("cp.async.wait_all;" ::: "memory");
    for (int32_t e = 0; e < 2; ++e) {     // the row's first and last pieces, by who copied them
      const int32_t c = e ? r.count - 1 : 0;
      if (c >= q0 && c < q1 && (c - q0) % THREADS == tid) trim(r, mine[c - q0], c);
    }
  }
  const float zy = logit(p, z, y);
  const auto piece = [&](int32_t c) {
    if (kOnce) return mine[c - q0];
    uint4 v = r.pieces[c];      // (not through the read-only cache: the gradient may take its place)
    trim(r, v, c);
    return v;
  };
  float top = -CUDART_INF_F, sum = 0.f;
  int32_t first = kNone;
#pragma unroll 4
  for (int32_t c = q0 + tid; c < q1; c += THREADS) {
    const float m = largest<T>(piece(c));
    if (m > top) top = m, first = c;
  }
  Part a;
  a.top = lanes_max<32>(top);
  if (tid % 32 == 0) tops[tid / 32] = a.top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < THREADS / 32; ++i) a.top = fmaxf(a.top, tops[i]);
  const Base b = base_of(a.top);
  by_base(b, [&](auto far) {
#pragma unroll 2
    for (int32_t c = q0 + tid; c < q1; c += THREADS) sum += powers<T, decltype(far)::value>(piece(c), b.t);
  });
  sum = lanes_sum<32>(sum);
  first = p.top ? lanes_min<32>(top == a.top ? first : kNone) : 0;
  if (tid % 32 == 0) sums[tid / 32] = sum, firsts[tid / 32] = first;
  __syncthreads();
  a.sum = 0.f;
  a.at = kNone;
#pragma unroll
  for (int i = 0; i < THREADS / 32; ++i) a.sum += sums[i], a.at = min(a.at, firsts[i]);
  if (width > 1) {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (tid < (int)width) *cg::this_cluster().map_shared_rank(&ctas[rank], tid) = a;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    Part b{-CUDART_INF_F, 0.f, kNone};
    if (tid % 8 < (int)width) b = ctas[tid % 8];
    a.top = lanes_max<8>(b.top);
    // (a part that holds nothing but -inf keeps its sum, 0 or NaN: there is no power of two for it)
    a.sum = lanes_sum<8>(b.top == a.top || b.top == -CUDART_INF_F ? b.sum : b.sum * rebase(b.top, a.top));
    a.at = lanes_min<8>(b.top == a.top ? b.at : kNone);
  }
  if (rank == 0 && tid == 0) write_loss(p, row, a, zy);
  if (p.top && a.at >= q0 && a.at < q1 && (a.at - q0) % THREADS == tid) write_top(p, r, row, a, piece(a.at), a.at);
  if (!p.grad) return;
  const Slope<T> s(p, row, y, a, r.shift);
  by_base(s.b, [&](auto far) {
    constexpr bool kFar = decltype(far)::value;
    if (s.whole) {
      const int32_t i0 = r.ragged(0), i1 = r.count - r.ragged(r.count - 1);     // pieces within [i0, i1) are the row's alone
#pragma unroll 2
      for (int32_t c = q0 + tid; c < q1; c += THREADS)
        if (c >= i0 && c < i1) write_grad<kFar>(r, piece(c), c, s, true);
      for (int32_t e = 0; e < 2; ++e) {
        const int32_t c = e ? r.count - 1 : 0;
        if (r.ragged(c) && c >= q0 && c < q1 && (c - q0) % THREADS == tid) write_grad<kFar>(r, piece(c), c, s, false);
      }
    } else {
      for (int32_t c = q0 + tid; c < q1; c += THREADS) write_grad<kFar>(r, piece(c), c, s, false);
    }
  });
  const int32_t at = label_piece(r, y);
  if (at >= q0 && at < q1 && (at - q0) % THREADS == tid) write_label(s, zy);
}

constexpr uint64_t kMostX = 1u << 20;     // CTAs along x; the rest along y

template <class T, int G, int NV>
cudaError_t lanes(const LossLaunch& p, cudaStream_t s) {
  const uint64_t ctas = (p.rows + kThreads / G - 1) / (kThreads / G), x = ctas < kMostX ? ctas : kMostX;
  return launch(loss_lanes_kernel<T, G, NV>, dim3((unsigned)x, (unsigned)((ctas + x - 1) / x)), kThreads, 0, 1, s, p);
}
constexpr uint64_t kPieces = 4096, kMostPieces = 13 * 1024;     // of a CTA: 64 KB, so that three and more share an SM; 208 KB

template <class T, bool kOnce, int THREADS>
cudaError_t ctas(const LossLaunch& p, uint32_t width, uint64_t pieces, cudaStream_t s) {
  const auto kernel = loss_cluster_kernel<T, kOnce, THREADS>;
  const uint64_t most = kMostX / width, x = p.rows < most ? p.rows : most;
  if (kOnce)
    if (const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kMostPieces * 16))) return e;
  return launch(kernel, dim3((unsigned)(x * width), (unsigned)((p.rows + x - 1) / x)), THREADS, kOnce ? (pieces + width - 1) / width * 16 : 0, width, s, p,
                width == 8 ? 3u : width / 2);
}

template <class T>
cudaError_t run(const LossLaunch& p, cudaStream_t s) {
  const uint64_t pieces = ((uint64_t)p.classes + 2 * kV<T> - 2) / kV<T>;     // of a row that starts anywhere
  if (pieces <= 4) return lanes<T, 4, 1>(p, s);
  if (pieces <= 8) return lanes<T, 8, 1>(p, s);
  if (pieces <= 16) return lanes<T, 16, 1>(p, s);
  if (pieces <= 32) return lanes<T, 32, 1>(p, s);
  if (pieces <= 64) return lanes<T, 32, 2>(p, s);
  if (pieces <= 128) return lanes<T, 32, 4>(p, s);
  if (pieces <= 256) return lanes<T, 32, 8>(p, s);
  // eight pieces and more a thread, as far as there are rows enough to fill the SMs with small CTAs
  if (p.rows >= 148 * 16 && pieces <= 512) return ctas<T, true, 64>(p, 1, pieces, s);
  if (p.rows >= 148 * 8 && pieces <= 1024) return ctas<T, true, 128>(p, 1, pieces, s);
  // up to sixteen pieces a thread and the CTAs that takes; few rows: more CTAs, with as few as two pieces a thread
  uint32_t width = 1;
  while (width < 8 && (pieces > kPieces * width || (p.rows * width * 2 <= 148 && pieces > 2ull * kThreads * width))) width *= 2;
  if (pieces <= kMostPieces * width) return ctas<T, true, kThreads>(p, width, pieces, s);
  return ctas<T, false, kThreads>(p, width, pieces, s);
}

}  // namespace

cudaError_t launch_loss(const LossLaunch& p, cudaStream_t s) {
  if (p.type == kF32) return run<float>(p, s);
  if (p.type == kBf16) return run<__nv_bfloat16>(p, s);
  return run<__half>(p, s);
}

}  // namespace layer
}  // namespace aet
