// Launchers of the 8-bit layers and of the optimizer's step (host-callable, all asynchronous on the given stream).
#pragma once

#include "train.h"

namespace lq {

constexpr int64_t FP8_BLOCK = 128;       // values along a row that share a scale
constexpr int64_t STATE_BLOCK = 256;     // values of an optimizer state that do
inline int64_t fp8_blocks(int64_t n) { return (n + FP8_BLOCK - 1) / FP8_BLOCK; }

// ---- quantizer (fp8_quantize_kernels.hip) -----------------------------------------------------------------
struct Fp8Quantize {
  const void* x; int64_t m, d, ldx; int dtype;
  uint8_t* codes; int64_t ld; float* scale;
  uint8_t* codes_t; int64_t ld_t; float* scale_t;
};
// One or two matrices, in one launch where their types are the same.
int launch_fp8_quantize(const Fp8Quantize* q, int count, bool tiles, hipStream_t st);

// ---- products (fp8_rows_kernels.hip) -----------------------------------------------------------------------
// Out[column][row] = sum_k rows[row][k] columns[column][k], bf16, `ld` elements from column to column: the operand whose index runs
// along a line of the output is `rows`.
struct Fp8Operand {
  const uint8_t* codes; int64_t ld;
  const float* scale; int64_t scale_row, scale_block;
  int shift;                             // rows per scale: 1 << shift (0 or 7)
  int64_t count;                         // rows
};
struct Fp8Product {
  Fp8Operand rows, columns;
  int64_t k;
  void* out; int64_t ld;
};
int launch_fp8_product(const Fp8Product& p, float* part, size_t part_floats, hipStream_t st);
// For few columns (fp8_quantizes_columns) with the columns' operand as it is before its quantization: row i of x is column i;
// p.columns holds their count.  fp8_needs_codes: whether there are operands of so many columns that this does not serve.
bool fp8_needs_codes(int64_t columns);
bool fp8_quantizes_columns(const Fp8Product& p);
int launch_fp8_product_raw(const Fp8Product& p, const void* x, int64_t ldx, int dtype, float* part, size_t part_floats, hipStream_t st);
// For many columns (fp8_product_kernels.hip).
int launch_fp8_tiles(const Fp8Product& p, float* part, size_t part_floats, hipStream_t st);
size_t fp8_tiles_part_floats(int64_t rows, int64_t columns, int64_t k);
size_t fp8_product_part_floats(int64_t rows, int64_t columns, int64_t k);

// ---- optimizer (adamw_kernels.hip) -------------------------------------------------------------------------
size_t grad_norm_parts(const lq_gradient* grads, int64_t count);
int launch_grad_norm(const lq_gradient* grads, int64_t count, float max_norm, float* norm, double* part, hipStream_t st);
int launch_adamw(const lq_adamw_tensor* tensors, int64_t count, int state_bits, const lq_adamw_params& h, const float* coef, hipStream_t st);

}  // namespace lq
