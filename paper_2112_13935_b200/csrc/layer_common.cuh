// Element types, activations, the dropout generator and the epilogue that the layer operators share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "aet_rng.h"
#include "layer_ops.h"

namespace aet {
namespace layer {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// N neighbouring elements as one access (N elements from an address that is a multiple of their size)
template <class T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

template <class T>
__device__ __forceinline__ void load4(const T* p, bool vec, int n, float (&v)[4]) {   // n: how many of the four there are
  if (vec && n == 4) {
    const Pack<T, 4> q = *reinterpret_cast<const Pack<T, 4>*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_f32(q.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}
template <class T>
__device__ __forceinline__ void store4(T* p, bool vec, int n, const float (&v)[4]) {
  if (vec && n == 4) {
    Pack<T, 4> q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q.v[i] = from_f32<T>(v[i]);
    *reinterpret_cast<Pack<T, 4>*>(p) = q;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}
__device__ __forceinline__ void load4(uint32_t type, const void* p, size_t at, bool vec, int n, float (&v)[4]) {
  if (type == kF32) load4(reinterpret_cast<const float*>(p) + at, vec, n, v);
  else if (type == kBf16) load4(reinterpret_cast<const __nv_bfloat16*>(p) + at, vec, n, v);
  else load4(reinterpret_cast<const __half*>(p) + at, vec, n, v);
}

__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }
// relu'(0) = 0; gelu is z Phi(z) by the error function; silu is z sigmoid(z)
__device__ __forceinline__ float activate(uint32_t act, float z) {
  if (act == kRelu) return z > 0.f || z != z ? z : 0.f;
  if (act == kGelu) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
  if (act == kSilu) return z * sigmoid(z);
  return z;
}
__device__ __forceinline__ float act_slope(uint32_t act, float z) {
  if (act == kRelu) return z > 0.f ? 1.f : 0.f;
  if (act == kGelu) return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
  if (act == kSilu) {
    const float s = sigmoid(z);
    return s * (1.f + z * (1.f - s));
  }
  return 1.f;
}

__device__ __forceinline__ uint64_t drop_bits(const Drop& d, uint64_t row, uint32_t cols, uint32_t col) {
  return draw(d.key, d.counter + row * ((cols + 3) / 4) + col / 4);
}
// A dropped element is zero whatever it was.
__device__ __forceinline__ void drop4(const Drop& d, uint64_t bits, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = ((uint32_t)(bits >> (16 * i)) & 0xFFFFu) >= d.q ? v[i] * d.scale : 0.f;
}

// x as three bf16 values whose sum is x to 24 bits: the upper 8 bits cut off, so that they cannot overflow, the rest to nearest.
// An x that is infinite or no number is all in the first.
__device__ __forceinline__ void three_parts(float x, uint16_t& h, uint16_t& m, uint16_t& l) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7F800000u) == 0x7F800000u) {
    h = (uint16_t)((u & 0x007FFFFFu) ? 0x7FFFu : u >> 16);
    m = l = 0;
    return;
  }
  h = (uint16_t)(u >> 16);
  const float r = x - __uint_as_float(u & 0xFFFF0000u);
  const __nv_bfloat16 rm = __float2bfloat16_rn(r);
  m = __bfloat16_as_ushort(rm);
  l = __bfloat16_as_ushort(__float2bfloat16_rn(r - __bfloat162float(rm)));
}

// Four pre-activations (the bias is in them) of row `row`, columns col .. col + n - 1 of an array with `cols` columns.
template <class Out>
__device__ __forceinline__ void finish4(const Epilogue& e, size_t row, uint32_t col, uint32_t cols, int n, float (&v)[4]) {
  if (e.pre) store4(static_cast<Out*>(e.pre) + row * e.ld_pre + col, e.vec, n, v);
  if (e.act) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = activate(e.act, v[i]);
  }
  if (e.drop.q) drop4(e.drop, drop_bits(e.drop, row, cols, col), v);
  if (e.residual) {
    float r[4];
    load4(static_cast<const Out*>(e.residual) + row * e.ld_res + col, e.vec, n, r);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += r[i];
  }
  store4(static_cast<Out*>(e.out) + row * e.ld_out + col, e.vec, n, v);
}

}  // namespace layer
}  // namespace aet
