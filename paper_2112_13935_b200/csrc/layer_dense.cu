// The dense layer: which kernels a call takes, and where things lie in its workspace.
#include <cuda_runtime.h>
#include <math.h>

#include "aet_rng.h"
#include "layer_dense.h"

namespace aet {
namespace layer {
namespace {

constexpr size_t kMostCols = 0x7fffffff, kMostLd = (size_t)1 << 31;

}  // namespace

const char* read_drop(const aet_dropout_spec& s, Drop& d) {
  d = Drop{0, 0, 0, 1.f};
  if (!(s.rate >= 0.f && s.rate < 1.f)) return "dropout rate is not in [0, 1)";
  const uint32_t q = (uint32_t)floor((double)s.rate * 65536.0 + 0.5);
  if (q >= 65536) return "dropout rate rounds to 1";
  if (!q) return nullptr;
  d.key = stream_key(s.seed, kStreamDropout, s.client);
  d.counter = s.counter;
  d.q = q;
  d.scale = (float)(65536.0 / (65536 - q));
  return nullptr;
}

const char* read_dense(const aet_dense_desc* in, Dense& out) {
  if (!in) return "null descriptor";
  if (in->struct_size != sizeof(aet_dense_desc)) return "struct_size does not match sizeof(aet_dense_desc)";
  out.d = *in;
  out.wide = false;
  aet_dense_desc& d = out.d;
  if (d.dtype > AET_F16) return "unknown dtype";
  if (d.act > AET_ACT_SILU) return "unknown activation";
  if (d.flags & ~(AET_DENSE_ANY_ADDRESS | AET_DENSE_ACCUMULATE)) return "unknown flag";
  if (!d.n_in || !d.n_out || d.n_in > kMostCols || d.n_out > kMostCols) return "n_in and n_out are 1 to 2^31 - 1";
  uint64_t* lds[] = {&d.ld_x, &d.ld_dx, &d.ld_w, &d.ld_dw, &d.ld_y, &d.ld_residual, &d.ld_pre, &d.ld_dy};
  for (int i = 0; i < 8; ++i) {
    const uint64_t cols = i < 2 ? d.n_in : d.n_out;
    if (!*lds[i]) *lds[i] = cols;
    if (*lds[i] < cols || *lds[i] > kMostLd) return "an ld is shorter than its rows or over 2^31";
  }
  return read_drop(d.drop, out.drop);
}

namespace {

bool four_wide(const void* p, size_t ld, uint32_t dtype) { return !p || ((uintptr_t)p % (4 * type_bytes(dtype)) == 0 && ld % 4 == 0); }

size_t round_up(size_t v, size_t to) { return (v + to - 1) / to * to; }

// An operand of a tensor-core product: the caller's rows where TMA takes them as they are (whole 16 bytes between rows and in front), otherwise
// a copy in the workspace; `parts`: always one, of fp32 in its three parts.
struct Copy { bool needed; size_t at, ld, plane; };
Copy plan_copy(const aet_dense_desc& d, size_t rows, size_t cols, size_t ld, bool parts, size_t& at) {
  const size_t b = type_bytes(d.dtype), whole = 16 / b;
  Copy c{};
  c.needed = parts || ld % whole || (d.flags & AET_DENSE_ANY_ADDRESS);
  c.ld = !c.needed ? ld : parts ? round_up(cols, 8) : round_up(cols, whole);
  c.plane = parts ? rows * c.ld : 0;
  c.at = at;
  if (c.needed) at += round_up(rows * c.ld * (parts ? 6 : b), 256);
  return c;
}
bool by_parts(const aet_dense_desc& d) { return d.dtype == AET_F32; }
MmaOperand operand(const Copy& c, const void* src, char* ws, bool mn) { return MmaOperand{c.needed ? ws + c.at : src, c.ld, c.plane, mn}; }
// What there is to copy, collected so that one launch does it.
struct Copies {
  RowsCopy list[2];
  int n = 0;
  void add(const Copy& c, const aet_dense_desc& d, const void* src, size_t ld, size_t rows, size_t cols, char* ws) {
    if (c.needed) list[n++] = RowsCopy{src, ws + c.at, ld, c.ld, c.plane, (uint32_t)rows, (uint32_t)cols, d.dtype};
  }
};

// What a forward call does and where it keeps what it needs.
struct Forward { bool few, mma, swapped; MmaShape shape; Copy x, w; size_t partial, total; };
Forward plan_forward(const Dense& L, size_t rows) {
  const aet_dense_desc& d = L.d;
  Forward f{};
  f.few = rows_kernel_takes((uint32_t)rows, d.n_in);
  if (f.few) return f;
  f.mma = mma_takes(d.dtype, (uint32_t)rows, d.n_out, d.n_in);
  if (!f.mma) return f;
  f.swapped = by_parts(d) && rows < d.n_out;        // the smaller operand is the one in parts
  f.shape = f.swapped ? mma_shape(d.dtype, d.n_out, (uint32_t)rows, d.n_in) : mma_shape(d.dtype, (uint32_t)rows, d.n_out, d.n_in);
  f.x = plan_copy(d, rows, d.n_in, d.ld_x, f.swapped, f.total);
  f.w = plan_copy(d, d.n_in, d.n_out, d.ld_w, by_parts(d) && !f.swapped, f.total);
  f.partial = f.total;
  f.total += round_up(mma_partial_floats(f.shape, (uint32_t)rows, d.n_out) * sizeof(float), 256);
  return f;
}

// ... a backward call.  dz: what the products take in dy's place, of the operands' type, as the tensor cores take it, or in fp32 (dy itself
// where it is that); parts: the same in parts, as the fp32 product for dW takes it.
struct Backward { bool mma; MmaShape dx, dw; Copy dz, parts, x, w; uint32_t dz_type; size_t slabs, partial, total; };
Backward plan_backward(const Dense& L, size_t rows) {
  const aet_dense_desc& d = L.d;
  Backward f{};
  f.mma = mma_takes(d.dtype, (uint32_t)rows, d.n_in, d.n_out) || mma_takes(d.dtype, d.n_in, d.n_out, (uint32_t)rows);   // (dz is laid out for one or the other)
  if (f.mma) {
    f.dx = mma_shape(d.dtype, (uint32_t)rows, d.n_in, d.n_out);
    f.dw = mma_shape(d.dtype, d.n_in, d.n_out, (uint32_t)rows);
    f.x = plan_copy(d, rows, d.n_in, d.ld_x, false, f.total);
    f.w = plan_copy(d, d.n_in, d.n_out, d.ld_w, by_parts(d), f.total);
    if (by_parts(d)) f.parts = plan_copy(d, rows, d.n_out, d.ld_dy, true, f.total);
  }
  f.dz = Copy{false, 0, d.ld_dy, 0};
  if (d.act != AET_ACT_NONE || L.drop.q || L.wide || (f.mma && (d.ld_dy % (16 / type_bytes(d.dtype)) || (d.flags & AET_DENSE_ANY_ADDRESS)))) {
    f.dz = Copy{true, f.total, round_up(d.n_out, 8), 0};
    f.dz_type = f.mma || L.wide ? d.dtype : kF32;
    f.total += round_up(rows * f.dz.ld * type_bytes(f.dz_type), 256);
  }
  f.slabs = f.total;
  f.total += round_up(slope_partial_floats((uint32_t)rows, d.n_out) * sizeof(float), 256);
  f.partial = f.total;
  const size_t px = mma_partial_floats(f.dx, (uint32_t)rows, d.n_in), pw = mma_partial_floats(f.dw, d.n_in, d.n_out);
  f.total += round_up((px > pw ? px : pw) * sizeof(float), 256);
  return f;
}

Epilogue plain_epilogue(void* out, size_t ld, uint32_t dtype, bool accumulate) {
  Epilogue e{};
  e.out = out;
  e.ld_out = e.ld_res = ld;
  e.out_type = dtype;
  e.residual = accumulate ? out : nullptr;
  e.vec = four_wide(out, ld, dtype);
  return e;
}

}  // namespace

size_t dense_space(const Dense& L, size_t rows, bool backward) {
  return !rows ? 0 : backward ? plan_backward(L, rows).total : plan_forward(L, rows).total;
}

cudaError_t dense_forward(const Dense& L, size_t rows, const void* x, const void* w, const void* bias, const void* residual, void* y, void* pre,
                          void* workspace, cudaStream_t s, const Waits& waits) {
  const aet_dense_desc& d = L.d;
  const uint32_t out = L.wide ? kF32 : d.dtype;
  const Forward f = plan_forward(L, rows);
  Product p{};
  p.a = x; p.a_row = d.ld_x; p.a_col = 1;
  p.b = w; p.b_row = d.ld_w; p.b_col = 1;
  p.type = d.dtype;
  p.m = (uint32_t)rows; p.n = d.n_out; p.k = d.n_in;
  p.e.bias = bias; p.e.bias_type = out;
  p.e.residual = residual; p.e.ld_res = d.ld_residual;
  p.e.out = y; p.e.ld_out = d.ld_y; p.e.out_type = out;
  p.e.pre = pre; p.e.ld_pre = d.ld_pre;
  p.e.act = d.act;
  p.e.vec = four_wide(y, d.ld_y, out) && four_wide(pre, d.ld_pre, out) && four_wide(residual, d.ld_residual, out);
  p.e.drop = L.drop;
  if (f.few) return launch_product_rows(p, s);
  if (!f.mma) return launch_product_fma(p, s);
  char* ws = static_cast<char*>(workspace);
  Copies copies;
  copies.add(f.x, d, x, d.ld_x, rows, d.n_in, ws);
  copies.add(f.w, d, w, d.ld_w, d.n_in, d.n_out, ws);
  if (const cudaError_t e = launch_rows_copies(copies.list, copies.n, s)) return e;
  const MmaOperand ox = operand(f.x, x, ws, false), ow = operand(f.w, w, ws, true);
  return launch_product_mma(MmaProduct{p, f.swapped ? ow : ox, f.swapped ? ox : ow, d.dtype, f.shape, reinterpret_cast<float*>(ws + f.partial), f.swapped, waits}, s);
}
bool dense_forward_waits(const Dense& L, size_t rows) { return rows && plan_forward(L, rows).mma; }

cudaError_t dense_backward(const Dense& L, size_t rows, const void* x, const void* w, const void* pre, const void* dy, void* dx, void* dw, void* db,
                           void* workspace, cudaStream_t s) {
  const aet_dense_desc& d = L.d;
  const uint32_t out = L.wide ? kF32 : d.dtype;
  const Backward f = plan_backward(L, rows);
  char* ws = static_cast<char*>(workspace);
  const bool accumulate = d.flags & AET_DENSE_ACCUMULATE;

  const bool want_dz = f.dz.needed && (dx || (dw && !f.parts.needed)), want_parts = f.parts.needed && dw;
  if (db || want_dz || want_parts) {
    SlopeLaunch p{};
    p.dy = dy; p.ld_dy = d.ld_dy;
    p.pre = d.act == AET_ACT_NONE ? nullptr : pre; p.ld_pre = d.ld_pre;
    p.dz = want_dz ? ws + f.dz.at : nullptr; p.ld_dz = f.dz.ld;
    if (want_parts) p.parts = reinterpret_cast<uint16_t*>(ws + f.parts.at), p.ld_parts = f.parts.ld, p.plane = f.parts.plane;
    p.db = db; p.db_type = out; p.accumulate = accumulate;
    p.type = out; p.act = d.act; p.dz_type = f.dz_type;
    p.rows = (uint32_t)rows; p.cols = d.n_out;
    p.drop = L.drop;
    p.partial = reinterpret_cast<float*>(ws + f.slabs);
    if (const cudaError_t e = launch_slope(p, s)) return e;
  }
  const void* dz = f.dz.needed ? ws + f.dz.at : dy;
  const bool dz_f32 = f.dz.needed && f.dz_type == kF32 && d.dtype != AET_F32;
  float* partial = reinterpret_cast<float*>(ws + f.partial);
  if (f.mma) {
    Copies copies;
    if (dx) copies.add(f.w, d, w, d.ld_w, d.n_in, d.n_out, ws);
    if (dw) copies.add(f.x, d, x, d.ld_x, rows, d.n_in, ws);
    if (const cudaError_t e = launch_rows_copies(copies.list, copies.n, s)) return e;
  }
  if (dx) {
    Product p{};
    p.a = dz; p.a_row = f.dz.ld; p.a_col = 1;
    p.b = w; p.b_row = 1; p.b_col = d.ld_w;
    p.type = d.dtype; p.a_f32 = dz_f32;
    p.m = (uint32_t)rows; p.n = d.n_in; p.k = d.n_out;
    p.e = plain_epilogue(dx, d.ld_dx, out, false);
    const cudaError_t e = f.mma ? launch_product_mma(MmaProduct{p, operand(f.dz, dy, ws, false), operand(f.w, w, ws, false), d.dtype, f.dx, partial}, s)
                                : launch_product_fma(p, s);
    if (e != cudaSuccess) return e;
  }
  if (dw) {
    Product p{};
    p.a = x; p.a_row = 1; p.a_col = d.ld_x;
    p.b = dz; p.b_row = f.dz.ld; p.b_col = 1;
    p.type = d.dtype; p.b_f32 = dz_f32;
    p.m = d.n_in; p.n = d.n_out; p.k = (uint32_t)rows;
    p.e = plain_epilogue(dw, d.ld_dw, out, accumulate);
    const MmaOperand b = f.parts.needed ? operand(f.parts, nullptr, ws, true) : operand(f.dz, dy, ws, true);
    const cudaError_t e = f.mma ? launch_product_mma(MmaProduct{p, operand(f.x, x, ws, true), b, d.dtype, f.dw, partial}, s) : launch_product_fma(p, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace layer
}  // namespace aet
