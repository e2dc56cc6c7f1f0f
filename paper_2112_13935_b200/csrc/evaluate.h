// Evaluation of a model over rows: what aet_predict and aet_evaluate run.
#pragma once
#include "layer_dense.h"

namespace aet {

// What an evaluation adds up on the device, over the chunks of its rows in their order.
struct Tally { double loss; unsigned long long correct; uint32_t bad_labels, pad; };

struct EvalModel {
  uint32_t n_layers, dims[8];
  bool bf16;                 // operands rounded to bf16, as in the rounds of precision 1
  float l2;
  aet_dropout_spec drop;     // behind every hidden layer's activation; rate 0: none
};
// Rows taken at a time, and the workspace that takes (the same for every chunk of a call).
size_t eval_chunk(const EvalModel& m, size_t n);
size_t eval_space(const EvalModel& m, size_t chunk, bool answers, bool gradient);

// Rows [row0, row0 + rows) of n: logits to `logits` (null: not kept); with labels, loss and right answers into *tally and, if `gradient`, the
// gradient of the mean loss over n rows into it (written by the first chunk, added to by the others).  All pointers are the device's.
cudaError_t eval_rows(const EvalModel& m, const float* w, const float* x, const int32_t* y, size_t row0, size_t rows, size_t n, float* logits,
                      Tally* tally, float* gradient, void* workspace, cudaStream_t s);
// The l2 term: its value into the tally (times n, since that becomes a mean), lambda W into the gradient (may be null).
cudaError_t eval_l2(const EvalModel& m, const float* w, size_t n, Tally* tally, float* gradient, cudaStream_t s);

}  // namespace aet
