// Evaluation of a model over rows (the paper's experiments report a node's accuracy; Eq. 1's F(w) and its gradient): the dense layers,
// the dropout and the classification loss of this library one after another, in chunks of rows.
#include <cuda_runtime.h>

#include "aet_kernels.h"
#include "evaluate.h"
#include "layer_launch.h"

namespace aet {
using namespace layer;
namespace {

size_t up(size_t v) { return (v + 255) / 256 * 256; }
size_t most_wide(const EvalModel& m) {
  size_t w = 0;
  for (uint32_t l = 1; l <= m.n_layers; ++l) w = m.dims[l] > w ? m.dims[l] : w;
  return w;
}

// Layer l of the model, its weights at `w` (of the products' type).
Dense layer_of(const EvalModel& m, uint32_t l, size_t row0, size_t n, bool accumulate) {
  Dense L{};
  L.d.struct_size = sizeof(aet_dense_desc);
  L.d.dtype = m.bf16 ? AET_BF16 : AET_F32;
  L.d.act = l + 1 < m.n_layers ? AET_ACT_RELU : AET_ACT_NONE;
  L.d.n_in = m.dims[l];
  L.d.n_out = m.dims[l + 1];
  // rows and weights of a parameter vector start anywhere
  L.d.flags = AET_DENSE_ANY_ADDRESS | (accumulate ? AET_DENSE_ACCUMULATE : 0);
  if (l + 1 < m.n_layers) {   // hidden layer l takes its draws behind those of the layers in front of it
    L.d.drop = m.drop;
    for (uint32_t k = 0; k < l; ++k) L.d.drop.counter += (uint64_t)n * ((m.dims[k + 1] + 3) / 4);
    L.d.drop.counter += (uint64_t)row0 * ((m.dims[l + 1] + 3) / 4);
  }
  Dense out{};
  read_dense(&L.d, out);      // (sound by construction: the rate was checked)
  out.wide = m.bf16;
  return out;
}

// Where a chunk keeps what it computes.
struct Space {
  size_t w, x[8], a[8], z[8], logits, dlogits, loss, top, d[2], layer, total;
};
Space space_of(const EvalModel& m, size_t rows, bool answers, bool gradient) {
  Space s{};
  size_t at = 0;
  const auto take = [&](size_t bytes) { const size_t p = at; at += up(bytes); return p; };
  size_t P = 0;
  for (uint32_t l = 0; l < m.n_layers; ++l) P += (size_t)m.dims[l] * m.dims[l + 1] + m.dims[l + 1];
  s.w = m.bf16 ? take(P * 2) : 0;
  for (uint32_t l = 0; l < m.n_layers; ++l) {
    s.x[l] = m.bf16 ? take(rows * m.dims[l] * 2) : 0;                          // the layer's input in bf16
    if (l + 1 < m.n_layers) s.a[l] = take(rows * m.dims[l + 1] * 4);           // its activations
    if (l + 1 < m.n_layers && gradient) s.z[l] = take(rows * m.dims[l + 1] * 4);
  }
  s.logits = take(rows * m.dims[m.n_layers] * 4);
  if (answers) {
    s.loss = take(rows * 4);
    s.top = take(rows * 4);
  }
  if (gradient) {
    s.dlogits = take(rows * m.dims[m.n_layers] * 4);
    s.d[0] = take(rows * most_wide(m) * 4);
    s.d[1] = take(rows * most_wide(m) * 4);
  }
  size_t layer = 0;
  for (uint32_t l = 0; l < m.n_layers; ++l) {
    const Dense L = layer_of(m, l, 0, rows, false);
    const size_t f = dense_space(L, rows, false), b = gradient ? dense_space(L, rows, true) : 0;
    layer = f > layer ? f : layer;
    layer = b > layer ? b : layer;
  }
  s.layer = take(layer);
  s.total = at;
  return s;
}

constexpr int kThreads = 1024;
__device__ __forceinline__ double cta_sum(double v, double* part) {   // over the CTA, always in the same order; for thread 0
  for (int o = 16; o; o >>= 1) v += __shfl_down_sync(~0u, v, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = v;
  __syncthreads();
  if (threadIdx.x) return 0.;
  v = 0.;
  for (int i = 0; i < kThreads / 32; ++i) v += part[i];
  return v;
}
__global__ void __launch_bounds__(kThreads) tally_kernel(const float* loss, const int32_t* top, const int32_t* y, uint32_t rows, uint32_t classes, Tally* t) {
  __shared__ double part[kThreads / 32];
  in_line();
  double sum = 0., right = 0., bad = 0.;     // (counts below 2^53)
  for (uint32_t i = threadIdx.x; i < rows; i += kThreads) {
    const bool known = (uint32_t)y[i] < classes;
    sum += known ? (double)loss[i] : 0.;
    right += known && top[i] == y[i];
    bad += !known;
  }
  sum = cta_sum(sum, part);
  right = cta_sum(right, part);
  bad = cta_sum(bad, part);
  if (threadIdx.x == 0) {
    t->loss += sum;
    t->correct += (unsigned long long)right;
    t->bad_labels |= bad > 0.;
  }
}
__global__ void __launch_bounds__(kThreads) l2_kernel(const float* w, float* g, size_t count, float lambda, double n, Tally* t) {
  __shared__ double part[kThreads / 32];
  in_line();
  double sum = 0.;
#pragma unroll 8
  for (size_t i = threadIdx.x; i < count; i += kThreads) {
    const float v = w[i];
    sum += (double)v * v;
    if (g) g[i] = fmaf(lambda, v, g[i]);
  }
  sum = cta_sum(sum, part);
  if (threadIdx.x == 0) t->loss += 0.5 * (double)lambda * sum * n;
}

}  // namespace

size_t eval_chunk(const EvalModel& m, size_t n) {
  size_t width = 0;
  for (uint32_t l = 0; l <= m.n_layers; ++l) width += m.dims[l];
  size_t c = ((size_t)1 << 26) / width;      // some 64 M values, and a few times that in workspace
  if (c < 1024) c = 1024;
  if (c > 65536) c = 65536;
  return n < c ? n : c;
}
size_t eval_space(const EvalModel& m, size_t chunk, bool answers, bool gradient) { return space_of(m, chunk, answers, gradient).total; }

cudaError_t eval_rows(const EvalModel& m, const float* w, const float* x, const int32_t* y, size_t row0, size_t rows, size_t n, float* logits,
                      Tally* tally, float* gradient, void* workspace, cudaStream_t s) {
  const bool answers = y != nullptr, back = answers && gradient;
  const Space sp = space_of(m, rows, answers, back);      // (a last chunk that is shorter takes less)
  char* ws = static_cast<char*>(workspace);
  const auto f32 = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
  const uint32_t L = m.n_layers, classes = m.dims[L];
  cudaError_t e = cudaSuccess;
#define AET_STEP(call) if ((e = (call)) != cudaSuccess) return e
  size_t P = 0, off[8];
  for (uint32_t l = 0; l < L; ++l) {
    off[l] = P;
    P += (size_t)m.dims[l] * m.dims[l + 1] + m.dims[l + 1];
  }
  if (m.bf16) AET_STEP(launch_to_bf16(w, ws + sp.w, P, s));
  const auto weights = [&](uint32_t l) { return m.bf16 ? (const void*)(ws + sp.w + off[l] * 2) : (const void*)(w + off[l]); };
  const auto bias_at = [&](uint32_t l) { return off[l] + (size_t)m.dims[l] * m.dims[l + 1]; };
  const void* input[8];
  const float* a = x;
  for (uint32_t l = 0; l < L; ++l) {
    if (m.bf16) AET_STEP(launch_to_bf16(a, ws + sp.x[l], rows * m.dims[l], s));
    input[l] = m.bf16 ? (const void*)(ws + sp.x[l]) : a;
    float* out = l + 1 < L ? f32(sp.a[l]) : logits ? logits : f32(sp.logits);
    AET_STEP(dense_forward(layer_of(m, l, row0, n, false), rows, input[l], weights(l), w + bias_at(l), nullptr, out, back && l + 1 < L ? f32(sp.z[l]) : nullptr,
                           ws + sp.layer, s));
    a = out;
  }
  if (!answers) return cudaSuccess;
  LossLaunch p{};
  p.logits = a; p.labels = y;
  p.loss = f32(sp.loss);
  p.top = reinterpret_cast<int32_t*>(ws + sp.top);
  p.grad = back ? f32(sp.dlogits) : nullptr;
  p.ld = p.ld_grad = classes;
  p.rows = rows;
  p.type = kF32; p.classes = classes;
  p.scale = (float)(1.0 / (double)n);
  AET_STEP(launch_loss(p, s));
  AET_STEP(launch(tally_kernel, dim3(1), kThreads, 0, 1, s, p.loss, p.top, y, (uint32_t)rows, classes, tally));
  if (!back) return cudaSuccess;
  const float* dy = f32(sp.dlogits);
  for (uint32_t l = L; l-- > 0;) {
    float* dx = l ? f32(sp.d[l & 1]) : nullptr;
    AET_STEP(dense_backward(layer_of(m, l, row0, n, row0 > 0), rows, input[l], weights(l), l + 1 < L ? f32(sp.z[l]) : nullptr, dy, dx, gradient + off[l],
                            gradient + bias_at(l), ws + sp.layer, s));
    dy = dx;
  }
#undef AET_STEP
  return cudaSuccess;
}

cudaError_t eval_l2(const EvalModel& m, const float* w, size_t n, Tally* tally, float* gradient, cudaStream_t s) {
  size_t off = 0;
  for (uint32_t l = 0; l < m.n_layers; ++l) {
    const size_t count = (size_t)m.dims[l] * m.dims[l + 1];
    if (const cudaError_t e = launch(l2_kernel, dim3(1), kThreads, 0, 1, s, w + off, gradient ? gradient + off : nullptr, count, m.l2, (double)n, tally)) return e;
    off += count + m.dims[l + 1];
  }
  return cudaSuccess;
}

}  // namespace aet
