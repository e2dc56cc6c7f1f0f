// Operands of tensor-core products that cannot be used where they are: rows onto a stride of whole 16 bytes, as they are, or fp32 rows as
// three bf16 parts (x = h + m + l: h the upper 8 bits of x, cut off, m and l the rest to nearest).  Both operands of a product in one launch.
#include <cuda_runtime.h>

#include "layer_rows.cuh"

namespace aet {
namespace layer {
namespace {

constexpr int kThreads = 256, kRows = 4;
struct Jobs { RowsCopy job[2]; uint32_t log[2], across[2], first; };     // first: CTAs of the first

// Eight elements of a row from column col on, zeros past the last.
template <class T>
__device__ __forceinline__ void take8(const T* s, int n, uint32_t (&w)[8 * sizeof(T) / 4]) {
  if (n >= 8 && (uintptr_t)s % 16 == 0) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      const uint4 q = reinterpret_cast<const uint4*>(s)[i];
      w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
    }
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = i < n ? s[i] : 0u;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (2 * i < n ? (uint32_t)s[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)s[2 * i + 1] << 16 : 0u);
  }
}

__global__ void __launch_bounds__(kThreads) rows_copy_kernel(const Jobs jobs) {
  in_line();
  const int which = blockIdx.x >= jobs.first;
  const RowsCopy& j = jobs.job[which];
  const uint32_t log = jobs.log[which], cta = blockIdx.x - (which ? jobs.first : 0);
  const uint32_t col = (((cta % jobs.across[which]) << log) + (threadIdx.x & ((1u << log) - 1))) * 8;
  if (col >= j.ld_dst) return;      // (a multiple of four, and of eight for 16-bit elements and parts)
  const int n = (int)(j.cols > col ? j.cols - col : 0);
  const size_t r0 = (size_t)(cta / jobs.across[which]) * (kThreads >> log) * kRows + (threadIdx.x >> log);
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const size_t r = r0 + (size_t)i * (kThreads >> log);
    if (r >= j.rows) break;
    if (j.type != kF32) {
      uint32_t w[4];
      take8<uint16_t>(static_cast<const uint16_t*>(j.src) + r * j.ld + col, n, w);
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(j.dst) + r * j.ld_dst + col) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      uint32_t w[8];
      take8<uint32_t>(static_cast<const uint32_t*>(j.src) + r * j.ld + col, n, w);
      if (j.plane) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(w[k]);
        store_parts<8>(static_cast<uint16_t*>(j.dst) + r * j.ld_dst + col, j.plane, v);
      } else {
        uint32_t* d = static_cast<uint32_t*>(j.dst) + r * j.ld_dst + col;
        *reinterpret_cast<uint4*>(d) = make_uint4(w[0], w[1], w[2], w[3]);
        if (col + 4 < j.ld_dst) *reinterpret_cast<uint4*>(d + 4) = make_uint4(w[4], w[5], w[6], w[7]);
      }
    }
  }
}

}  // namespace

cudaError_t launch_rows_copies(const RowsCopy* copies, int n, cudaStream_t s) {
  if (!n) return cudaSuccess;
  Jobs jobs{};
  uint64_t ctas = 0;
  for (int i = 0; i < n; ++i) {
    jobs.job[i] = copies[i];
    jobs.log[i] = log_lanes<8>((uint32_t)copies[i].ld_dst);
    jobs.across[i] = (uint32_t)(((copies[i].ld_dst + 7) / 8 + (1u << jobs.log[i]) - 1) >> jobs.log[i]);
    const uint64_t at_once = (uint64_t)(kThreads >> jobs.log[i]) * kRows;
    ctas += (copies[i].rows + at_once - 1) / at_once * jobs.across[i];
    if (i == 0) jobs.first = (uint32_t)ctas;
  }
  return launch(rows_copy_kernel, dim3((unsigned)ctas), kThreads, 0, 1, s, jobs);
}

}  // namespace layer
}  // namespace aet
