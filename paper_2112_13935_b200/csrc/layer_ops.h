// Launch interfaces of the layer operators (dense layer, classification loss, dropout): plain structs, no library types.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace aet {
namespace layer {

enum DType : uint32_t { kF32 = 0, kBf16 = 1, kF16 = 2 };
enum Act : uint32_t { kNone = 0, kRelu = 1, kGelu = 2, kSilu = 3 };
inline size_t type_bytes(uint32_t t) { return t == kF32 ? 4 : 2; }

// Dropout of an array of rows: draw counter + row * ceil(cols / 4) + col / 4 of the key's stream holds sixteen bits for each of
// four neighbouring elements; one whose bits are below q of 65,536 is dropped, the others are multiplied by `scale`.
struct Drop {
  uint64_t key, counter;
  uint32_t q;        // 0: nothing is dropped
  float scale;       // 65536 / (65536 - q)
};

// What becomes of four neighbouring sums z = (A B)[row, col .. col + 3] of a product: pre = z + bias,
// out = residual + drop(act(pre)).
struct Epilogue {
  const void* bias;      // [cols] or null
  const void* residual;  // [rows, ld_res] of the outputs' type, or null; may be `out` itself
  void* out;             // [rows, ld_out]
  void* pre;             // [rows, ld_pre] of the outputs' type, or null
  size_t ld_res, ld_out, ld_pre;
  uint32_t bias_type, out_type, act;
  uint32_t vec;          // out, pre and residual can be touched four columns at a time
  Drop drop;
};

// C [m, n] = A B through the epilogue: A(i, k) = a[i a_row + k a_col], B(k, j) = b[k b_row + j b_col], elements of `type`.
struct Product {
  const void *a, *b;
  size_t a_row, a_col, b_row, b_col;
  uint32_t type;
  uint32_t m, n, k;
  Epilogue e;
  uint32_t a_f32, b_f32;     // that operand is fp32 beside a 16-bit `type` (launch_product_fma only)
};

// Small products, on FMAs (see layer_fma_kernel.cu).
cudaError_t launch_product_fma(const Product& p, cudaStream_t s);
uint32_t fma_split(uint32_t m, uint32_t n, uint32_t k);    // CTAs along k
uint64_t fma_volume(uint32_t m, uint32_t n, uint32_t k);   // multiplications, in whole tiles

// Up to eight rows of A along k against a B across it (see layer_rows_kernel.cu).
bool rows_kernel_takes(uint32_t m, uint32_t k);
cudaError_t launch_product_rows(const Product& p, cudaStream_t s);

// Large products (see layer_mma_kernel.cu and, for fp32, layer_f32_kernel.cu).  An operand of a tensor-core product: rows `ld` elements
// apart and from 16-byte boundaries on; mn: its rows run along k, not across.  fp32: A as it is, B as its three bf16 parts, `plane`
// elements apart.
struct MmaOperand {
  const void* p;
  size_t ld, plane;
  uint32_t mn;
};
struct MmaShape {
  uint32_t pair;     // two CTAs share a tile
  uint32_t splits;   // parts k is split into
};
// How the tensor-core kernels wait for their barriers, and a failure that can be played: the copies of the first CTA (or pair) from its
// `stages`-th stage on never come.
struct Waits {
  unsigned long long ns = 4000000000ull;
  uint32_t stages = 0xffffffffu;
};
struct MmaProduct {
  Product p;         // m, n, k and the epilogue; a and b stand here:
  MmaOperand a, b;
  uint32_t type;
  MmaShape shape;
  float* partial;    // mma_partial_floats() of workspace
  uint32_t swapped;  // fp32: a is B^T and b A^T, in parts; `shape` is that of n x m
  Waits waits = {};
};
bool mma_takes(uint32_t type, uint32_t m, uint32_t n, uint32_t k);   // rather than the FMA kernel
MmaShape mma_shape(uint32_t type, uint32_t m, uint32_t n, uint32_t k);
size_t mma_partial_floats(const MmaShape& s, uint32_t m, uint32_t n);
cudaError_t launch_product_mma(const MmaProduct& m, cudaStream_t s);
cudaError_t launch_product_f32(const MmaProduct& m, cudaStream_t s);
// Rows onto a stride that TMA takes, whole 16 bytes and from a 16-byte boundary: as they are, or (plane non-zero) fp32 as three bf16 parts
// `plane` elements apart.  Up to two arrays in one launch.
struct RowsCopy {
  const void* src;
  void* dst;
  size_t ld, ld_dst, plane;
  uint32_t rows, cols, type;
};
cudaError_t launch_rows_copies(const RowsCopy* copies, int n, cudaStream_t s);

// dz = drop(dy) act'(pre), to `dz` (null: not kept), to `parts` (null: not wanted) as three bf16 parts `plane` elements apart, and its sums
// over the rows to db.
struct SlopeLaunch {
  const void *dy, *pre;   // pre null: act is none
  void *dz, *db;          // db null: no sums
  uint16_t* parts;        // rows ld_parts apart
  size_t ld_dy, ld_pre, ld_dz, ld_parts, plane;
  uint32_t type, db_type, act, accumulate;   // of dy and pre; accumulate: db += sums
  uint32_t dz_type;       // dy's, bf16 where dy is fp32, or fp32
  uint32_t rows, cols;
  Drop drop;
  float* partial;         // slope_partial_floats() of workspace
};
size_t slope_partial_floats(uint32_t rows, uint32_t cols);
cudaError_t launch_slope(const SlopeLaunch& p, cudaStream_t s);

cudaError_t launch_dropout(uint32_t type, size_t rows, uint32_t cols, const Drop& d, const void* x, size_t ld_x, const void* residual,
                           size_t ld_res, void* y, size_t ld_y, cudaStream_t s);

struct LossLaunch {
  const void* logits;
  const int32_t* labels;
  const float* weight;    // [rows] or null
  float* loss;            // [rows] or null
  void* grad;             // [rows, ld_grad] of the logits' type, or null; may be the logits
  int32_t* top;           // [rows] or null
  size_t ld, ld_grad, rows;
  uint32_t type, classes;
  float scale;
};
cudaError_t launch_loss(const LossLaunch& p, cudaStream_t s);

}  // namespace layer
}  // namespace aet
