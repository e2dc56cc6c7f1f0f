// Element types, activations, the dropout generator and the epilogue that the layer operators share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "aet_rng.h"
#include "layer_launch.h"
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

// N neighbouring elements as one access of words (from an address that is a multiple of their size).  The words are taken apart and put
// together by hand: structs of 16-bit elements are copied one by one, and arrays of them go to local memory.
template <int kWords> struct WordsOf;
template <> struct WordsOf<2> { using type = uint2; };
template <> struct WordsOf<4> { using type = uint4; };
template <class T, int N> using Words = typename WordsOf<N * (int)sizeof(T) / 4>::type;
__device__ __forceinline__ void split_words(const uint2& q, uint32_t (&w)[2]) { w[0] = q.x; w[1] = q.y; }
__device__ __forceinline__ void split_words(const uint4& q, uint32_t (&w)[4]) { w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w; }
__device__ __forceinline__ uint2 join_words(const uint32_t (&w)[2]) { return make_uint2(w[0], w[1]); }
__device__ __forceinline__ uint4 join_words(const uint32_t (&w)[4]) { return make_uint4(w[0], w[1], w[2], w[3]); }
template <class T, int N>
__device__ __forceinline__ void unpack(const Words<T, N>& q, float (&v)[N]) {
  uint32_t w[N * sizeof(T) / 4];
  split_words(q, w);
#pragma unroll
  for (int i = 0; i < N * (int)sizeof(T) / 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      v[i] = __uint_as_float(w[i]);
    } else if constexpr (std::is_same<T, __half>::value) {
      v[2 * i] = __half2float(__ushort_as_half((unsigned short)w[i]));
      v[2 * i + 1] = __half2float(__ushort_as_half((unsigned short)(w[i] >> 16)));
    } else {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}
// Two values rounded to nearest in a word, the first in the lower half.
template <class T> __device__ __forceinline__ uint32_t round2(float lo, float hi) {
  uint32_t r;
  if constexpr (std::is_same<T, __half>::value) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <class T, int N>
__device__ __forceinline__ Words<T, N> pack(const float (&v)[N]) {
  uint32_t w[N * sizeof(T) / 4];
#pragma unroll
  for (int i = 0; i < N * (int)sizeof(T) / 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      w[i] = __float_as_uint(v[i]);
    } else {
      w[i] = round2<T>(v[2 * i], v[2 * i + 1]);
    }
  }
  return join_words(w);
}
// The words of N neighbouring elements, as they are (kept so until they are used, rows that are under way cost half the registers).
template <class T, int N>
__device__ __forceinline__ Words<T, N> load_words(const T* p, bool whole, int n) {
  if (whole) return *reinterpret_cast<const Words<T, N>*>(p);
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
  return pack<T, N>(v);
}
__device__ __forceinline__ void keep_words(uint2& q) { asm volatile("" : "+r"(q.x), "+r"(q.y)); }
__device__ __forceinline__ void keep_words(uint4& q) { asm volatile("" : "+r"(q.x), "+r"(q.y), "+r"(q.z), "+r"(q.w)); }
// N neighbouring elements in registers; `whole`: all N are there and may be touched at once (n: how many there are otherwise).
template <class T, int N>
__device__ __forceinline__ void load_n(const T* p, bool whole, int n, float (&v)[N]) {
  if (whole) {
    unpack<T, N>(*reinterpret_cast<const Words<T, N>*>(p), v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}
template <class T, int N>
__device__ __forceinline__ void store_n(T* p, bool whole, int n, const float (&v)[N]) {
  if (whole) {
    *reinterpret_cast<Words<T, N>*>(p) = pack<T, N>(v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}
__device__ __forceinline__ void load4(uint32_t type, const void* p, size_t at, bool whole, int n, float (&v)[4]) {
  if (type == kF32) load_n<float, 4>(reinterpret_cast<const float*>(p) + at, whole, n, v);
  else if (type == kBf16) load_n<__nv_bfloat16, 4>(reinterpret_cast<const __nv_bfloat16*>(p) + at, whole, n, v);
  else load_n<__half, 4>(reinterpret_cast<const __half*>(p) + at, whole, n, v);
}

// Activations for values that are stored as T.  relu'(0) = 0; gelu is z Phi(z) by the error function; silu is z sigmoid(z).
// 16-bit results take a shorter way: exponentials by ex2.approx, and Phi(z) = 1 - P(t) e^(-z^2/2) / 2 for z >= 0 with t = 1 / (1 + p |z| / sqrt 2)
// and Hastings' polynomial P (Abramowitz and Stegun 7.1.26), which is within 1.5e-7 / 2 of Phi everywhere and shares its exponential with
// the density that the slope needs.  (The quotient in sigmoid is 0 for a divisor over 2^126: silu is exactly 0 below -87.3, where it is 1e-36.)
template <class T> __device__ __forceinline__ float sigmoid(float z) {
  return sizeof(T) == 4 ? __fdividef(1.f, 1.f + expf(-z)) : __fdividef(1.f, 1.f + __expf(-z));
}
__device__ __forceinline__ float hastings(float z, float& gauss) {   // Phi(z), and e^(-z^2/2)
  const float x = fabsf(z) * 0.70710678118654752f, t = __fdividef(1.f, fmaf(0.3275911f, x, 1.f));
  gauss = __expf(-0.5f * z * z);
  const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
  const float tail = 0.5f * p * gauss;
  return z >= 0.f ? 1.f - tail : tail;
}
template <class T> __device__ __forceinline__ float activate(uint32_t act, float z) {
  if (act == kRelu) return z > 0.f || z != z ? z : 0.f;
  if (act == kGelu) {
    float g;
    return sizeof(T) == 4 ? 0.5f * z * (1.f + erff(z * 0.70710678118654752f)) : z * hastings(z, g);
  }
  if (act == kSilu) return z * sigmoid<T>(z);
  return z;
}
template <class T> __device__ __forceinline__ float act_slope(uint32_t act, float z) {
  if (act == kRelu) return z > 0.f ? 1.f : 0.f;
  if (act == kGelu) {
    if (sizeof(T) == 4) return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    float g;
    const float phi = hastings(z, g);
    return fmaf(z * 0.39894228040143268f, g, phi);
  }
  if (act == kSilu) {
    const float s = sigmoid<T>(z);
    return s * (1.f + z * (1.f - s));
  }
  return 1.f;
}

// N / 4 draws' bits on N elements; draw_at: the first draw's number plus 1, times the generator's step, plus the key.  A dropped element is
// zero whatever it was.
template <int N>
__device__ __forceinline__ void drop_n(const Drop& d, uint64_t draw_at, float (&v)[N]) {
#pragma unroll
  for (int g = 0; g < N / 4; ++g) {
    const uint64_t bits = mix64(draw_at + kGamma * (uint64_t)g);
    const uint32_t lo = (uint32_t)bits, hi = (uint32_t)(bits >> 32);
    const uint32_t w[4] = {lo & 0xFFFFu, lo >> 16, hi & 0xFFFFu, hi >> 16};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[4 * g + i] = w[i] >= d.q ? v[4 * g + i] * d.scale : 0.f;
  }
}
__device__ __forceinline__ uint64_t drop_at(const Drop& d, uint64_t row, uint32_t cols, uint32_t col) {
  return d.key + kGamma * (d.counter + row * ((cols + 3) / 4) + col / 4 + 1);
}

// Two values as three bf16 values each whose sum is the value to 24 bits: the upper 8 bits cut off, so that they cannot overflow, the rest to
// nearest.  Words of two, the first in the lower half.  An infinity or a NaN gives parts that are NaN.
__device__ __forceinline__ void three_parts(float x0, float x1, uint32_t& h, uint32_t& m, uint32_t& l) {
  const uint32_t u0 = __float_as_uint(x0), u1 = __float_as_uint(x1);
  h = __byte_perm(u0, u1, 0x7632);
  const float r0 = x0 - __uint_as_float(u0 & 0xFFFF0000u), r1 = x1 - __uint_as_float(u1 & 0xFFFF0000u);
  m = round2<__nv_bfloat16>(r0, r1);
  l = round2<__nv_bfloat16>(r0 - __uint_as_float(m << 16), r1 - __uint_as_float(m & 0xFFFF0000u));
}

// N neighbouring values (a multiple of four) in three parts to planes `plane` elements apart.
template <int N>
__device__ __forceinline__ void store_parts(uint16_t* to, size_t plane, const float (&v)[N]) {
#pragma unroll
  for (int g = 0; g < N; g += 4) {
    uint2 h, m, l;
    three_parts(v[g], v[g + 1], h.x, m.x, l.x);
    three_parts(v[g + 2], v[g + 3], h.y, m.y, l.y);
    *reinterpret_cast<uint2*>(to + g) = h;
    *reinterpret_cast<uint2*>(to + plane + g) = m;
    *reinterpret_cast<uint2*>(to + 2 * plane + g) = l;
  }
}

// Four pre-activations (the bias is in them) of row `row`, columns col .. col + n - 1 of an array with `cols` columns, and the residual there.
template <class Out>
__device__ __forceinline__ void finish4(const Epilogue& e, size_t row, uint32_t col, uint32_t cols, int n, float (&v)[4], const float (&residual)[4]) {
  if (e.pre) store_n<Out, 4>(static_cast<Out*>(e.pre) + row * e.ld_pre + col, e.vec && n == 4, n, v);
  if (e.act) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = activate<Out>(e.act, v[i]);
  }
  if (e.drop.q) drop_n<4>(e.drop, drop_at(e.drop, row, cols, col), v);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] += residual[i];
  store_n<Out, 4>(static_cast<Out*>(e.out) + row * e.ld_out + col, e.vec && n == 4, n, v);
}
template <class Out>
__device__ __forceinline__ void finish4(const Epilogue& e, size_t row, uint32_t col, uint32_t cols, int n, float (&v)[4]) {
  float r[4] = {};
  if (e.residual) load_n<Out, 4>(static_cast<const Out*>(e.residual) + row * e.ld_res + col, e.vec && n == 4, n, r);
  finish4<Out>(e, row, col, cols, n, v, r);
}

// One sum of a product, the bias not in it yet, where neighbouring lanes have neighbouring columns.
template <class Out>
__device__ __forceinline__ void finish1(const Epilogue& e, size_t row, uint32_t col, uint32_t cols, float v) {
  if (e.bias) {
    float b[4];
    load4(e.bias_type, e.bias, col, false, 1, b);
    v += b[0];
  }
  if (e.pre) static_cast<Out*>(e.pre)[row * e.ld_pre + col] = from_f32<Out>(v);
  v = activate<Out>(e.act, v);
  if (e.drop.q) v = ((uint32_t)(mix64(drop_at(e.drop, row, cols, col)) >> (col % 4 * 16)) & 0xFFFFu) >= e.drop.q ? v * e.drop.scale : 0.f;
  if (e.residual) v += to_f32(static_cast<const Out*>(e.residual)[row * e.ld_res + col]);
  static_cast<Out*>(e.out)[row * e.ld_out + col] = from_f32<Out>(v);
}
// Four sums of a product, the bias not in them yet.
template <class Out>
__device__ __forceinline__ void with_bias(const Product& p, uint32_t row, uint32_t col, float (&v)[4]) {
  const int n = (int)min(4u, p.n - col);
  if (p.e.bias) {
    float b[4];
    load4(p.e.bias_type, p.e.bias, col, false, n, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += b[i];
  }
  finish4<Out>(p.e, row, col, p.n, n, v);
}

}  // namespace layer
}  // namespace aet
