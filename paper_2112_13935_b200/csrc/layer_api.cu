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

Epilogue plain_epilogue(void* out, size_t ld, uint32_t dtype, bool accumulate) {
  Epilogue e{};
  e.out = out;
  e.ld_out = e.ld_res = ld;
  e.out_type = dtype;
  e.residual = accumulate ? out : nullptr;
  e.vec = four_wide(out, ld, dtype);
  return e;
}

size_t round_up(size_t v, size_t to) { return (v + to - 1) / to * to; }

// Where a backward call keeps what it needs: dz and the partial sums of db.
struct BackSpace { size_t dz, dz_ld, partial, total; };
BackSpace back_space(const Dense& L, size_t rows) {
  BackSpace s{};
  s.dz = 0;
  s.dz_ld = round_up(L.d.n_out, 8);
  s.partial = round_up(rows * s.dz_ld * type_bytes(L.d.dtype), 256);
  s.total = s.partial + round_up(slope_partial_floats((uint32_t)rows, L.d.n_out) * sizeof(float), 256);
  return s;
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
  if (!classes || classes > kMostRows || rows > kMostRows) return arg("classes are 1 to 2^31 - 1, rows up to 2^31 - 1");
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
  *bytes = backward && rows ? back_space(L, rows).total : 0;
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
  (void)workspace; (void)workspace_bytes;
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
  return done(launch_product_fma(p, (cudaStream_t)cuda_stream));
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
  const BackSpace space = back_space(L, rows);
  if (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < space.total)
    return arg("the workspace is missing, off a 256-byte boundary or smaller than aet_dense_workspace says");
  char* ws = static_cast<char*>(workspace);

  const bool accumulate = d.flags & AET_DENSE_ACCUMULATE;
  const bool as_is = d.act == AET_ACT_NONE && !L.drop.q;   // dz is dy
  if (!as_is || db) {
    SlopeLaunch p{};
    p.dy = dy; p.ld_dy = d.ld_dy;
    p.pre = d.act == AET_ACT_NONE ? nullptr : pre; p.ld_pre = d.ld_pre;
    p.dz = as_is || (!dx && !dw) ? nullptr : ws + space.dz; p.ld_dz = space.dz_ld;
    p.db = db; p.db_type = d.dtype; p.accumulate = accumulate;
    p.type = d.dtype; p.act = d.act;
    p.rows = (uint32_t)rows; p.cols = d.n_out;
    p.drop = L.drop;
    p.partial = reinterpret_cast<float*>(ws + space.partial);
    if (const cudaError_t e = launch_slope(p, s)) return done(e);
  }
  const void* dz = as_is ? dy : ws + space.dz;
  const size_t ld_dz = as_is ? d.ld_dy : space.dz_ld;
  if (dx) {
    Product p{};
    p.a = dz; p.a_row = ld_dz; p.a_col = 1;
    p.b = w; p.b_row = 1; p.b_col = d.ld_w;
    p.type = d.dtype;
    p.m = (uint32_t)rows; p.n = d.n_in; p.k = d.n_out;
    p.e = plain_epilogue(dx, d.ld_dx, d.dtype, false);
    if (const cudaError_t e = launch_product_fma(p, s)) return done(e);
  }
  if (dw) {
    Product p{};
    p.a = x; p.a_row = 1; p.a_col = d.ld_x;
    p.b = dz; p.b_row = ld_dz; p.b_col = 1;
    p.type = d.dtype;
    p.m = d.n_in; p.n = d.n_out; p.k = (uint32_t)rows;
    p.e = plain_epilogue(dw, d.ld_dw, d.dtype, accumulate);
    if (const cudaError_t e = launch_product_fma(p, s)) return done(e);
  }
  return AET_OK;
}
