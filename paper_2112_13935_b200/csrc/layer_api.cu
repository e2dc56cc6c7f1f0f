// C entries of the layer operators: checks of arguments.
#include <cuda_runtime.h>

#include <string>

#include "../../include/aet.h"
#include "layer_dense.h"

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

constexpr size_t kMostRows = 0x7fffffff, kMostLd = (size_t)1 << 31;
bool no_space(const void* workspace, size_t bytes, size_t need) { return need && (!workspace || (uintptr_t)workspace % 256 || bytes < need); }
const char* const kNoSpace = "the workspace is missing, off a 256-byte boundary or smaller than aet_dense_workspace says";

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
  *bytes = dense_space(L, rows, backward != 0);
  return AET_OK;
}

namespace {

aet_status forward(const aet_dense_desc* desc, size_t rows, const void* x, const void* w, const void* bias, const void* residual, void* y, void* pre,
                   void* workspace, size_t workspace_bytes, void* cuda_stream, const Waits* played) {
  Dense L;
  if (const char* why = read_dense(desc, L)) return arg(why);
  const aet_dense_desc& d = L.d;
  if (rows > kMostRows) return arg("rows are up to 2^31 - 1");
  if (played && !dense_forward_waits(L, rows)) return fail(AET_ERR_CONFIG, "lost copies can be played for products on the tensor cores only");
  if (!rows) return AET_OK;
  if (!x || !w || !y) return arg("null argument");
  for (const void* p : {x, w, bias, residual, (const void*)y, (const void*)pre})
    if (off_type(p, d.dtype)) return arg("a pointer is not a multiple of the element size");
  if (!(d.flags & AET_DENSE_ANY_ADDRESS) && (off_16(x) || off_16(w)))
    return arg("x and w have to start on a 16-byte boundary without AET_DENSE_ANY_ADDRESS");
  if (no_space(workspace, workspace_bytes, dense_space(L, rows, false))) return arg(kNoSpace);
  return done(dense_forward(L, rows, x, w, bias, residual, y, pre, workspace, (cudaStream_t)cuda_stream, played ? *played : Waits()));
}

}  // namespace

extern "C" aet_status aet_dense_forward(const aet_dense_desc* desc, size_t rows, const void* x, const void* w, const void* bias,
                                        const void* residual, void* y, void* pre, void* workspace, size_t workspace_bytes,
                                        void* cuda_stream) {
  return forward(desc, rows, x, w, bias, residual, y, pre, workspace, workspace_bytes, cuda_stream, nullptr);
}

extern "C" aet_status aet_debug_dense_lost_copies(const aet_dense_desc* desc, size_t rows, const void* x, const void* w, void* y, void* workspace,
                                                  size_t workspace_bytes, uint32_t stages, uint32_t wait_us, void* cuda_stream) {
  if (!wait_us || wait_us > 1000000) return arg("wait_us is 1 to 10^6");
  Waits played;
  played.ns = wait_us * 1000ull;
  played.stages = stages;
  return forward(desc, rows, x, w, nullptr, nullptr, y, nullptr, workspace, workspace_bytes, cuda_stream, &played);
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
  if (no_space(workspace, workspace_bytes, dense_space(L, rows, true))) return arg(kNoSpace);
  return done(dense_backward(L, rows, x, w, pre, dy, dx, dw, db, workspace, s));
}
