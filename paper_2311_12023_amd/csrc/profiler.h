// Optional per-kernel timing with HIP events on the launch stream (off by default; see lq_profile_enable).
#pragma once

#include <hip/hip_runtime.h>

namespace lq {
namespace prof {

enum Cls {
  GEMM_BASE = 0,            // + mode * 8 + (l/32 - 1): 16 classes of wide_gemm_kernel
  GEMM_FIXUP = 16,
  GRAM = 17,
  CHOLESKY = 18,
  TRSM = 19,
  JACOBI = 20,
  LOWRANK_BLOCKQUANT = 21,
  SCALEQUANT_ERROR = 22,
  RESIDUAL = 23,
  QUANTIZE = 24,
  DEQUANTIZE = 25,
  MISC = 26,
  GEMM_SPLIT_BASE = 27,     // + mode * 8 + (l/32 - 1): the bf16 hi/lo split variants of wide_gemm_kernel
  QMATMUL = 43,             // qmatmul_kernel (work = flops of the product)
  QMATVEC = 44,             // qmatvec_kernel (work = bytes)
  SPLIT_PROJECT = 45,       // split_project_kernel (work = bytes)
  GEMM_F16_BASE = 46,       // + planes * 8 + mode * 4 + (l/32 - 1): wide_gemm_f16_kernel (work = flops of the product)
  ABSMAX = 62,
  ROTATE = 63,              // rotate_kernel (work = bytes)
  QROWS = 64,               // qrows_kernel (work = flops of the product)
  SYM_EIG = 65,             // sym_eig_kernel (work = bytes)
  PLANE_GEMM = 66,          // plane_gemm_kernel (work = flops of the product)
  WEIGHT_PLANE = 67,        // weight_plane_kernel (work = bytes)
  COLUMN_GEMM_BASE = 68,    // + mode * 4 + (l/32 - 1): column_gemm_kernel (work = flops of the product)
  COLUMN_SUM = 76,          // column_sum_kernel (work = bytes)
  DROPOUT = 77,             // dropout_kernel (work = bytes)
  TRAIN_PLANES = 78,        // passes that bring operands into planes (work = bytes)
  ADAPTER_PRODUCT = 79,     // adapter_product_kernel (work = flops of the product)
  LOSS_LOGITS = 80,         // loss_logits_kernel, loss_gradient_kernel (work = flops of the product)
  LOSS_ACCUMULATE = 81,     // loss_accumulate_kernel, loss_dw_kernel (work = flops of the product)
  LOSS_ROWS = 82,           // the loss's passes over rows and sums (work = bytes)
  THIN_PROJECT = 83,        // thin_project_kernel (work = bytes)
  THIN_GRAM = 84,           // thin_gram_kernel (work = bytes)
  THIN_FINISH = 85,         // sums of partial results of the training operators (work = bytes)
  FP8_QUANTIZE = 86,        // fp8_quantize_kernel (work = bytes)
  FP8_ROWS = 87,            // fp8_rows_kernel (work = bytes)
  FP8_PRODUCT = 88,         // fp8_product_kernel (work = flops of the product)
  FP8_JOIN = 89,            // fp8_join_kernel (work = bytes)
  GRAD_NORM = 90,           // grad_squares_kernel, grad_norm_kernel (work = bytes)
  ADAMW = 91,               // adamw_kernel (work = bytes)
  NUM_CLASSES = 92
};

bool enabled();
// Brackets the launches issued while it is alive.  `work`: algorithmic flops (GEMM classes) or bytes.
class Scope {
 public:
  Scope(int cls, hipStream_t st, double work);
  ~Scope();
 private:
  int slot_;
  hipStream_t st_;
};

}  // namespace prof
}  // namespace lq
