// What the gradient of a dense layer starts with: dz = drop(dy) act'(pre), and the sums of dz over the rows (the bias's gradient).
//
// One pass over dy and pre, bound by memory.  A CTA takes a slab of rows and 128 columns, a thread four neighbouring columns (one
// draw of the dropout generator, one 8- or 16-byte access); the sums of a slab go to the workspace and a second small kernel adds
// the slabs up in their order, so that they are the same from call to call.
#include <cuda_runtime.h>

#include "layer_common.cuh"

namespace aet {
namespace layer {
namespace {

constexpr int kLanes = 32, kRowLanes = 8, kCols = 4 * kLanes;

template <class T>
__global__ void __launch_bounds__(kLanes* kRowLanes) slope_kernel(const SlopeLaunch p, const uint32_t slabs, const bool vec) {
  __shared__ __align__(16) float sums[kRowLanes][kCols];
  const int lane = threadIdx.x % kLanes, rl = threadIdx.x / kLanes;
  const uint32_t blocks = (p.cols + kCols - 1) / kCols;
  const uint32_t slab = blockIdx.x / blocks, col = blockIdx.x % blocks * kCols + lane * 4;
  const uint64_t r0 = (uint64_t)p.rows * slab / slabs, r1 = (uint64_t)p.rows * (slab + 1) / slabs;
  const int n = col < p.cols ? (int)min(4u, p.cols - col) : 0;
  const T* dy = static_cast<const T*>(p.dy);
  const T* pre = static_cast<const T*>(p.pre);
  float acc[4] = {};
  if (n) {
#pragma unroll 4
    for (uint64_t r = r0 + rl; r < r1; r += kRowLanes) {
      float v[4];
      load4(dy + r * p.ld_dy + col, vec, n, v);
      if (p.drop.q) drop4(p.drop, drop_bits(p.drop, r, p.cols, col), v);
      if (pre) {
        float z[4];
        load4(pre + r * p.ld_pre + col, vec, n, z);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = act_slope(p.act, z[i]);
          v[i] = p.act == kRelu ? (f != 0.f ? v[i] : 0.f) : v[i] * f;
        }
      }
      if (p.dz && p.plane) {
        Pack<uint16_t, 4> q[3] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) three_parts(v[i], q[0].v[i], q[1].v[i], q[2].v[i]);   // (0 past the last column)
        uint16_t* d = static_cast<uint16_t*>(p.dz) + r * p.ld_dz + col;
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<Pack<uint16_t, 4>*>(d + i * p.plane) = q[i];
      } else if (p.dz) {
        store4(static_cast<T*>(p.dz) + r * p.ld_dz + col, vec, n, v);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] += v[i];
    }
  }
  if (!p.db) return;
  *reinterpret_cast<float4*>(&sums[rl][lane * 4]) = make_float4(acc[0], acc[1], acc[2], acc[3]);
  __syncthreads();
  const uint32_t c = blockIdx.x % blocks * kCols + threadIdx.x;
  if (threadIdx.x < kCols && c < p.cols) {
    float v = 0.f;
    for (int q = 0; q < kRowLanes; ++q) v += sums[q][threadIdx.x];
    p.partial[(size_t)slab * p.cols + c] = v;
  }
}

// db = (db +) the sums of the slabs; 32 columns a CTA, eight threads to a column
template <class T>
__global__ void __launch_bounds__(256) slab_sums_kernel(const float* partial, uint32_t slabs, uint32_t cols, T* db, uint32_t accumulate) {
  __shared__ float sums[8][32];
  const int lane = threadIdx.x % 32, part = threadIdx.x / 32;
  const uint32_t c = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (c < cols)
    for (uint32_t q = part; q < slabs; q += 8) v += partial[(size_t)q * cols + c];
  sums[part][lane] = v;
  __syncthreads();
  if (part || c >= cols) return;
  v = accumulate ? to_f32(db[c]) : 0.f;
  for (int q = 0; q < 8; ++q) v += sums[q][lane];
  db[c] = from_f32<T>(v);
}

uint32_t slabs_of(uint32_t rows, uint32_t cols) {
  const uint32_t blocks = (cols + kCols - 1) / kCols;
  // about eight CTAs for each of 148 SMs, each with eight rows and more to a thread
  const uint32_t want = (148 * 8 + blocks - 1) / blocks, most = (rows + 8 * kRowLanes - 1) / (8 * kRowLanes);
  return want < most ? want : most ? most : 1;
}

bool aligned4(const void* p, size_t ld, size_t bytes) { return !p || ((uintptr_t)p % (4 * bytes) == 0 && ld % 4 == 0); }

template <class T>
cudaError_t run(const SlopeLaunch& p, cudaStream_t s) {
  const uint32_t slabs = slabs_of(p.rows, p.cols), blocks = (p.cols + kCols - 1) / kCols;
  const bool vec = aligned4(p.dy, p.ld_dy, sizeof(T)) && aligned4(p.pre, p.ld_pre, sizeof(T)) && aligned4(p.dz, p.ld_dz, sizeof(T));
  slope_kernel<T><<<slabs * blocks, kLanes * kRowLanes, 0, s>>>(p, slabs, vec);
  if (p.db) {
    const uint32_t grid = (p.cols + 31) / 32;
    if (p.db_type == kF32) slab_sums_kernel<<<grid, 256, 0, s>>>(p.partial, slabs, p.cols, static_cast<float*>(p.db), p.accumulate);
    else if (p.db_type == kBf16) slab_sums_kernel<<<grid, 256, 0, s>>>(p.partial, slabs, p.cols, static_cast<__nv_bfloat16*>(p.db), p.accumulate);
    else slab_sums_kernel<<<grid, 256, 0, s>>>(p.partial, slabs, p.cols, static_cast<__half*>(p.db), p.accumulate);
  }
  return cudaGetLastError();
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
