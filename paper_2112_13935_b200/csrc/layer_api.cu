// C entries of the layer operators: checks of arguments, the choice of kernels, and where things lie in the workspace.
#include <cuda_runtime.h>
#include <math.h>

#include <string>

#include "../../include/aet.h"
#include "aet_rng.h"
#include "layer_ops.h"

namespace aet {
void set_thread_error(const std::string& msg);  // text returned by aet_last_error(NULL)
}
using namespace aet;
using namespace aet::layer;

namespace {

aet_status fail(aet_status s, const char* msg) noexcept {
  try {
    set_thread_error(msg);
  } catch (...) {   // no memory for the text: the status stands for itself
  }
  return s;
}
aet_status arg(const char* msg) noexcept { return fail(AET_ERR_ARG, msg); }
aet_status done(cudaError_t e) noexcept {
  if (e == cudaSuccess) return AET_OK;
  cudaGetLastError();
  return fail(AET_ERR_CUDA, cudaGetErrorString(e));
}

bool off_type(const void* p, uint32_t dtype) { return (uintptr_t)p % type_bytes(dtype) != 0; }
bool off_16(const void* p) { return (uintptr_t)p % 16 != 0; }

constexpr size_t kMostRows = 0x7fffffff;          // rows, columns: 31 bits; elements of a matrix: 2^62
constexpr size_t kMostLd = (size_t)1 << 31;

// Null if the rate can be; d keeps what the kernels need of it.
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

// A descriptor with its gaps filled in.
struct Dense {
  aet_dense_desc d;
  Drop drop;
};
const char* read_dense(const aet_dense_desc* in, Dense& out) {
  if (!in) return "null descriptor";
  if (in->struct_size != sizeof(aet_dense_desc)) return "struct_size does not match sizeof(aet_dense_desc)";
  out.d = *in;
  aet_dense_desc& d = out.d;
  if (d.dtype > AET_F16) return "unknown dtype";
  if (d.act > AET_ACT_SILU) return "unknown activation";
  if (d.flags & ~(AET_DENSE_ANY_ADDRESS | AET_DENSE_ACCUMULATE)) return "unknown flag";
  if (!d.n_in || !d.n_out || d.n_in > kMostRows || d.n_out > kMostRows) return "n_in and n_out are 1 to 2^31 - 1";
  uint64_t* lds[] = {&d.ld_x, &d.ld_dx, &d.ld_w, &d.ld_dw, &d.ld_y, &d.ld_residual, &d.ld_pre, &d.ld_dy};
  for (int i = 0; i < 8; ++i) {
    const uint64_t cols = i < 2 ? d.n_in : d.n_out;
    if (!*lds[i]) *lds[i] = cols;
    if (*lds[i] < cols || *lds[i] > kMostLd) return "an ld is shorter than its rows or over 2^31";
  }
  return read_drop(d.drop, out.drop);
}

bool four_wide(const void* p, size_t ld, uint32_t dtype) { return !p || ((uintptr_t)p % (4 * type_bytes(dtype)) == 0 && ld % 4 == 0); }

size_t round_up(size_t v, size_t to) { return (v + to - 1) / to * to; }

// An operand of a tensor-core product: the caller's rows where TMA takes them as they are (16-bit elements, whole 16 bytes between
// rows and in front), otherwise a copy in the workspace.
struct Copy { bool needed; size_t at, ld, plane, bytes; };
Copy plan_copy(const aet_dense_desc& d, size_t rows, size_t cols, size_t ld, size_t& at) {
  Copy c{};
  c.needed = d.dtype == AET_F32 || ld % 8 || (d.flags & AET_DENSE_ANY_ADDRESS);
  c.ld = c.needed ? round_up(cols, 8) : ld;
  c.plane = rows * c.ld;
  c.bytes = c.needed ? round_up(c.plane * 2 * (d.dtype == AET_F32 ? 3 : 1), 256) : 0;
  c.at = at;
  at += c.bytes;
  return c;
}
uint32_t planes_of(const aet_dense_desc& d) { return d.dtype == AET_F32 ? 3 : 1; }
MmaOperand operand(const Copy& c, const void* src, char* ws, bool mn) { return MmaOperand{c.needed ? ws + c.at : src, c.ld, c.plane, mn}; }
cudaError_t make_copy(const Copy& c, const aet_dense_desc& d, const void* src, size_t ld, size_t rows, size_t cols, char* ws, cudaStream_t s) {
  if (!c.needed) return cudaSuccess;
  return launch_planes(d.dtype, src, ld, ws + c.at, c.ld, c.plane, (uint32_t)rows, (uint32_t)cols, s);
}

// What a forward call does and where it keeps what it needs.
struct Forward { MmaShape shape; Copy x, w; size_t partial, total; };
Forward plan_forward(const Dense& L, size_t rows) {
  const aet_dense_desc& d = L.d;
  Forward f{};
  f.shape = mma_shape(planes_of(d), (uint32_t)rows, d.n_out, d.n_in);
  if (!f.shape.use) return f;
  f.x = plan_copy(d, rows, d.n_in, d.ld_x, f.total);
  f.w = plan_copy(d, d.n_in, d.n_out, d.ld_w, f.total);
  f.partial = f.total;
  f.total += round_up(mma_partial_floats(f.shape, (uint32_t)rows, d.n_out) * sizeof(float), 256);
  return f;
}

// ... a backward call.  dz: what the products take in dy's place, of the element type or, for the tensor cores' fp32 products, in parts.
struct Backward { MmaShape dx, dw; Copy dz, x, w; size_t slabs, partial, total; bool as_is; };
Backward plan_backward(const Dense& L, size_t rows) {
  const aet_dense_desc& d = L.d;
  Backward f{};
  f.as_is = d.act == AET_ACT_NONE && !L.drop.q;
  f.dx = mma_shape(planes_of(d), (uint32_t)rows, d.n_in, d.n_out);
  f.dw = mma_shape(planes_of(d), d.n_in, d.n_out, (uint32_t)rows);
  if (f.dx.use) {
    f.x = plan_copy(d, rows, d.n_in, d.ld_x, f.total);
    f.w = plan_copy(d, d.n_in, d.n_out, d.ld_w, f.total);
  }
  f.dz = Copy{true, f.total, round_up(d.n_out, 8), 0, 0};
  if (f.as_is && (!f.dx.use || (d.dtype != AET_F32 && d.ld_dy % 8 == 0 && !(d.flags & AET_DENSE_ANY_ADDRESS)))) f.dz = Copy{false, 0, d.ld_dy, 0, 0};
  f.dz.plane = rows * f.dz.ld;
  if (f.dz.needed) f.total += round_up(f.dz.plane * (d.dtype != AET_F32 ? 2 : f.dx.use ? 6 : 4), 256);
  f.slabs = f.total;
  f.total += round_up(slope_partial_floats((uint32_t)rows, d.n_out) * sizeof(float), 256);
  f.partial = f.total;
  const size_t px = mma_partial_floats(f.dx, (uint32_t)rows, d.n_in), pw = mma_partial_floats(f.dw, d.n_in, d.n_out);
  f.total += round_up((px > pw ? px : pw) * sizeof(float), 256);
  return f;
}

bool no_space(const void* workspace, size_t bytes, size_t need) { return need && (!workspace || (uintptr_t)workspace % 256 || bytes < need); }
const char* const kNoSpace = "the workspace is missing, off a 256-byte boundary or smaller than aet_dense_workspace says";

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

extern "C" aet_status aet_dropout(uint32_t dtype, size_t rows, uint32_t cols, const aet_dropout_spec* drop, const void* x, size_t ld_x,
                                  const void* residual, size_t ld_residual, void* y, size_t ld_y, void* cuda_stream) {
  if (dtype > AET_F16) return arg("unknown dtype");
  if (!drop) return arg("null dropout spec");
  Drop d;
  if (const char* why = read_drop(*drop, d)) return arg(why);
  if (!cols || cols > kMostRows || rows > kMostRows) return arg("columns are 1 to 2^31 - 1, rows up to 2^31 - 1");
  if (!rows) return AET_OK;
  if (!x || !y) return arg("null argument");
  if (!ld_x) ld_x = cols;
  if (!ld_y) ld_y = cols;
  if (!ld_residual) ld_residual = cols;
  if (ld_x < cols || ld_y < cols || ld_residual < cols || ld_x > kMostLd || ld_y > kMostLd || ld_residual > kMostLd)
    return arg("an ld is shorter than its rows or over 2^31");
  if (off_type(x, dtype) || off_type(y, dtype) || off_type(residual, dtype)) return arg("a pointer is not a multiple of the element size");
  return done(launch_dropout(dtype, rows, cols, d, x, ld_x, residual, ld_residual, y, ld_y, (cudaStream_t)cuda_stream));
}

extern "C" aet_status aet_cross_entropy(uint32_t dtype, size_t rows, uint32_t classes, const void* logits, size_t ld, const int32_t* labels,
                                        const float* weight, float scale, float* loss, void* dlogits, size_t ld_dlogits, int32_t* top,
                                        void* cuda_stream) {
  if (dtype > AET_F16) return arg("unknown dtype");
  if (!classes || classes > 1u << 30 || rows > kMostRows) return arg("classes are 1 to 2^30, rows up to 2^31 - 1");
  if (!rows) return AET_OK;
  if (!logits || !labels) return arg("null argument");
  if (!ld) ld = classes;
  if (!ld_dlogits) ld_dlogits = classes;
  if (ld < classes || ld_dlogits < classes || ld > kMostLd || ld_dlogits > kMostLd) return arg("an ld is shorter than its rows or over 2^31");
  if (off_type(logits, dtype) || off_type(dlogits, dtype) || off_type(labels, AET_F32) || off_type(weight, AET_F32) ||
      off_type(loss, AET_F32) || off_type(top, AET_F32))
    return arg("a pointer is not a multiple of the element size");
  LossLaunch p{};
  p.logits = logits; p.labels = labels; p.weight = weight; p.loss = loss; p.grad = dlogits; p.top = top;
  p.ld = ld; p.ld_grad = ld_dlogits; p.rows = rows;
  p.type = dtype; p.classes = classes; p.scale = scale;
  return done(launch_loss(p, (cudaStream_t)cuda_stream));
}

extern "C" aet_status aet_dense_workspace(const aet_dense_desc* desc, size_t rows, int backward, size_t* bytes) {
  Dense L;
  if (const char* why = read_dense(desc, L)) return arg(why);
  if (!bytes) return arg("null argument");
  if (rows > kMostRows) return arg("rows are up to 2^31 - 1");
  *bytes = !rows ? 0 : backward ? plan_backward(L, rows).total : plan_forward(L, rows).total;
  return AET_OK;
}

extern "C" aet_status aet_dense_forward(const aet_dense_desc* desc, size_t rows, const void* x, const void* w, const void* bias,
                                        const void* residual, void* y, void* pre, void* workspace, size_t workspace_bytes,
                                        void* cuda_stream) {
  Dense L;
  if (const char* why = read_dense(desc, L)) return arg(why);
  const aet_dense_desc& d = L.d;
  if (rows > kMostRows) return arg("rows are up to 2^31 - 1");
  if (!rows) return AET_OK;
  if (!x || !w || !y) return arg("null argument");
  for (const void* p : {x, w, bias, residual, (const void*)y, (const void*)pre})
    if (off_type(p, d.dtype)) return arg("a pointer is not a multiple of the element size");
  if (!(d.flags & AET_DENSE_ANY_ADDRESS) && (off_16(x) || off_16(w)))
    return arg("x and w have to start on a 16-byte boundary without AET_DENSE_ANY_ADDRESS");
  const Forward f = plan_forward(L, rows);
  if (no_space(workspace, workspace_bytes, f.total)) return arg(kNoSpace);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  Product p{};
  p.a = x; p.a_row = d.ld_x; p.a_col = 1;
  p.b = w; p.b_row = d.ld_w; p.b_col = 1;
  p.type = d.dtype;
  p.m = (uint32_t)rows; p.n = d.n_out; p.k = d.n_in;
  p.e.bias = bias; p.e.bias_type = d.dtype;
  p.e.residual = residual; p.e.ld_res = d.ld_residual;
  p.e.out = y; p.e.ld_out = d.ld_y; p.e.out_type = d.dtype;
  p.e.pre = pre; p.e.ld_pre = d.ld_pre;
  p.e.act = d.act;
  p.e.vec = four_wide(y, d.ld_y, d.dtype) && four_wide(pre, d.ld_pre, d.dtype) && four_wide(residual, d.ld_residual, d.dtype);
  p.e.drop = L.drop;
  if (!f.shape.use) return done(launch_product_fma(p, s));
  char* ws = static_cast<char*>(workspace);
  cudaError_t e = make_copy(f.x, d, x, d.ld_x, rows, d.n_in, ws, s);
  if (e == cudaSuccess) e = make_copy(f.w, d, w, d.ld_w, d.n_in, d.n_out, ws, s);
  if (e != cudaSuccess) return done(e);
  return done(launch_product_mma(MmaProduct{p, operand(f.x, x, ws, false), operand(f.w, w, ws, true), d.dtype == AET_F16 ? kF16 : kBf16, planes_of(d),
                                            f.shape, reinterpret_cast<float*>(ws + f.partial)}, s));
}

extern "C" aet_status aet_dense_backward(const aet_dense_desc* desc, size_t rows, const void* x, const void* w, const void* pre, const void* dy,
                                         void* dx, void* dw, void* db, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  Dense L;
  if (const char* why = read_dense(desc, L)) return arg(why);
  const aet_dense_desc& d = L.d;
  const size_t b = type_bytes(d.dtype);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  if (rows > kMostRows) return arg("rows are up to 2^31 - 1");
  for (const void* p : {x, w, pre, dy, (const void*)dx, (const void*)dw, (const void*)db})
    if (off_type(p, d.dtype)) return arg("a pointer is not a multiple of the element size");
  if (!rows) {   // sums over no rows
    if (d.flags & AET_DENSE_ACCUMULATE) return AET_OK;
    if (dw)
      if (const cudaError_t e = cudaMemset2DAsync(dw, d.ld_dw * b, 0, (size_t)d.n_out * b, d.n_in, s)) return done(e);
    return db ? done(cudaMemsetAsync(db, 0, (size_t)d.n_out * b, s)) : AET_OK;
  }
  if (!dy || (dw && !x) || (dx && !w) || (d.act != AET_ACT_NONE && !pre)) return arg("null argument");
  if (!(d.flags & AET_DENSE_ANY_ADDRESS) && ((dw && off_16(x)) || (dx && off_16(w)) || off_16(dy)))
    return arg("x, w and dy have to start on a 16-byte boundary without AET_DENSE_ANY_ADDRESS");
  if (!dx && !dw && !db) return AET_OK;
  const Backward f = plan_backward(L, rows);
  if (no_space(workspace, workspace_bytes, f.total)) return arg(kNoSpace);
  char* ws = static_cast<char*>(workspace);
  const bool accumulate = d.flags & AET_DENSE_ACCUMULATE, products = dx || dw;

  if (db || (products && f.dz.needed)) {
    SlopeLaunch p{};
    p.dy = dy; p.ld_dy = d.ld_dy;
    p.pre = d.act == AET_ACT_NONE ? nullptr : pre; p.ld_pre = d.ld_pre;
    p.dz = products && f.dz.needed ? ws + f.dz.at : nullptr; p.ld_dz = f.dz.ld;
    p.plane = d.dtype == AET_F32 && f.dx.use ? f.dz.plane : 0;
    p.db = db; p.db_type = d.dtype; p.accumulate = accumulate;
    p.type = d.dtype; p.act = d.act;
    p.rows = (uint32_t)rows; p.cols = d.n_out;
    p.drop = L.drop;
    p.partial = reinterpret_cast<float*>(ws + f.slabs);
    if (const cudaError_t e = launch_slope(p, s)) return done(e);
  }
  const void* dz = f.dz.needed ? ws + f.dz.at : dy;
  const uint32_t type16 = d.dtype == AET_F16 ? kF16 : kBf16;
  float* partial = reinterpret_cast<float*>(ws + f.partial);
  if (dx) {
    Product p{};
    p.a = dz; p.a_row = f.dz.ld; p.a_col = 1;
    p.b = w; p.b_row = 1; p.b_col = d.ld_w;
    p.type = d.dtype;
    p.m = (uint32_t)rows; p.n = d.n_in; p.k = d.n_out;
    p.e = plain_epilogue(dx, d.ld_dx, d.dtype, false);
    cudaError_t e;
    if (!f.dx.use) {
      e = launch_product_fma(p, s);
    } else {
      e = make_copy(f.w, d, w, d.ld_w, d.n_in, d.n_out, ws, s);
      if (e == cudaSuccess)
        e = launch_product_mma(MmaProduct{p, operand(f.dz, dy, ws, false), operand(f.w, w, ws, false), type16, planes_of(d), f.dx, partial}, s);
    }
    if (e != cudaSuccess) return done(e);
  }
  if (dw) {
    Product p{};
    p.a = x; p.a_row = 1; p.a_col = d.ld_x;
    p.b = dz; p.b_row = f.dz.ld; p.b_col = 1;
    p.type = d.dtype;
    p.m = d.n_in; p.n = d.n_out; p.k = (uint32_t)rows;
    p.e = plain_epilogue(dw, d.ld_dw, d.dtype, accumulate);
    cudaError_t e;
    if (!f.dw.use) {
      e = launch_product_fma(p, s);
    } else {
      e = make_copy(f.x, d, x, d.ld_x, rows, d.n_in, ws, s);
      if (e == cudaSuccess)
        e = launch_product_mma(MmaProduct{p, operand(f.x, x, ws, true), operand(f.dz, dy, ws, true), type16, planes_of(d), f.dw, partial}, s);
    }
    if (e != cudaSuccess) return done(e);
  }
  return AET_OK;
}
