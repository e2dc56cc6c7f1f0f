// The dense layer behind its C entries, for those and for the evaluation of a handle's model.
#pragma once
#include "../../include/aet.h"
#include "layer_ops.h"

namespace aet {
namespace layer {

// A descriptor with its gaps filled in.  wide: operands of the products (x, W, dz) are of d.dtype, bf16, and everything else - bias, y, pre,
// dy, dx, dW, db - is fp32, as in the rounds of bf16 models.
struct Dense {
  aet_dense_desc d;
  Drop drop;
  bool wide;
};
const char* read_drop(const aet_dropout_spec& s, Drop& d);           // null if the rate can be
const char* read_dense(const aet_dense_desc* in, Dense& out);        // null if the descriptor is sound
// Workspace, and the calls on checked arguments with that much of it (from a 256-byte boundary on).
size_t dense_space(const Dense& L, size_t rows, bool backward);
cudaError_t dense_forward(const Dense& L, size_t rows, const void* x, const void* w, const void* bias, const void* residual, void* y, void* pre,
                          void* workspace, cudaStream_t s, const Waits& waits = Waits());
bool dense_forward_waits(const Dense& L, size_t rows);               // on barriers, which may give up: on the tensor cores
cudaError_t dense_backward(const Dense& L, size_t rows, const void* x, const void* w, const void* pre, const void* dy, void* dx, void* dw, void* db,
                           void* workspace, cudaStream_t s);

}  // namespace layer
}  // namespace aet
