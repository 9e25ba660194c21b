// C ABI of the layers in 8 bits: quantizer, product, a layer's forward pass and its gradients.
#include "fp8.h"

namespace lq {

static bool bad_type(int dtype) { return dtype != LQ_T_FP32 && dtype != LQ_T_BF16; }
static bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// A launch has fewer than 2^32 threads, 16 for a row of few rows' products.
constexpr int64_t MOST_ROWS = (int64_t)1 << 27, MOST_SIDE = (int64_t)1 << 30, MOST_DEPTH = (int64_t)1 << 22, MOST_LD = (int64_t)1 << 40;
static bool bad_rows(int64_t n) { return n <= 0 || n > MOST_ROWS; }
static bool bad_depth(int64_t n) { return n <= 0 || n > MOST_DEPTH; }
// A gradient's sizes: dX sums over n, dW over m.
static bool bad_gradients(int64_t m, int64_t n, int64_t k, bool want_dx, bool want_dw) {
  return (want_dw ? bad_depth(m) : bad_rows(m)) || (want_dx ? bad_depth(n) : bad_rows(n)) || bad_rows(k);
}

static int check_matrix(const lq_fp8_matrix* w, int64_t k) {
  if (!w || !w->codes || !w->scale) return LQ_ERR_NULL;
  if (w->ld < k || w->ld > MOST_DEPTH || w->scale_row < 0 || w->scale_block < 0 || w->scale_row > MOST_DEPTH / 2 || w->scale_block > MOST_LD)
    return LQ_ERR_SHAPE;
  if (misaligned(w->codes, 16) || w->ld % 16 || misaligned(w->scale, 4) || (w->tiles != 0 && w->tiles != 1)) return LQ_ERR_ARG;
  return LQ_OK;
}
static Fp8Operand operand(const lq_fp8_matrix& w, int64_t rows) {
  return {w.codes, w.ld, w.scale, w.scale_row, w.scale_block, w.tiles ? 7 : 0, rows};
}

// Regions of a workspace one after the other; without a base address it only counts.
struct Space {
  char* base;
  size_t used;
  template <typename T>
  T* take(size_t count) {
    T* p = base && count ? reinterpret_cast<T*>(base + used) : nullptr;
    used += up256(count * sizeof(T));
    return p;
  }
};
// A matrix quantized inside a call.
struct Codes {
  uint8_t* codes; int64_t ld; float* scale;
  Fp8Operand rows(int64_t count) const { return {codes, ld, scale, 1, count, 0, count}; }
};
static Codes take_codes(Space& s, int64_t rows, int64_t k) {
  const int64_t ld = up_to(k, 128);          // a block is a line
  uint8_t* c = s.take<uint8_t>(rows * ld);
  return {c, ld, s.take<float>(rows * fp8_blocks(k))};
}

struct ForwardPlan { Codes x; float* part; size_t part_floats, bytes; };
static ForwardPlan plan_forward(void* ws, int64_t m, int64_t n, int64_t k) {
  ForwardPlan p{};
  Space s{static_cast<char*>(ws), 0};
  if (fp8_needs_codes(m)) p.x = take_codes(s, m, k);
  p.part_floats = fp8_product_part_floats(n, m, k);
  p.part = s.take<float>(p.part_floats);
  p.bytes = s.used;
  return p;
}
struct BackwardPlan { Codes dy, dyt, xt; float* part; size_t part_floats, bytes; };
static BackwardPlan plan_backward(void* ws, int64_t m, int64_t n, int64_t k, bool want_dx, bool want_dw) {
  BackwardPlan p{};
  Space s{static_cast<char*>(ws), 0};
  if (want_dx && (want_dw || fp8_needs_codes(m))) p.dy = take_codes(s, m, n);
  if (want_dw) { p.dyt = take_codes(s, n, m); p.xt = take_codes(s, k, m); }
  p.part_floats = std::max(want_dx ? fp8_product_part_floats(k, m, n) : 0, want_dw ? fp8_product_part_floats(k, n, m) : 0);
  p.part = s.take<float>(p.part_floats);
  p.bytes = s.used;
  return p;
}
static bool no_space(const void* ws, size_t have, size_t need) { return need && (!ws || misaligned(ws, 256) || have < need); }

}  // namespace lq

using namespace lq;

extern "C" {

int lq_fp8_quantize(const void* X, int64_t m, int64_t d, int64_t ldx, int dtype, int tiles, uint8_t* codes, int64_t ld_codes, float* scale,
                    uint8_t* codes_t, int64_t ld_codes_t, float* scale_t, void* stream) {
  if (!X || (!codes && !codes_t)) return LQ_ERR_NULL;
  if ((codes || tiles == 1) && !scale) return LQ_ERR_NULL;
  if (codes_t && tiles == 0 && !scale_t) return LQ_ERR_NULL;
  if (m <= 0 || d <= 0 || m > MOST_SIDE || d > MOST_SIDE || ldx < d || ldx > MOST_LD) return LQ_ERR_SHAPE;
  if ((codes && (ld_codes < d || ld_codes > MOST_LD)) || (codes_t && (ld_codes_t < m || ld_codes_t > MOST_LD))) return LQ_ERR_SHAPE;
  if (bad_type(dtype) || (tiles != 0 && tiles != 1) || misaligned(X, type_bytes(dtype))) return LQ_ERR_ARG;
  if ((codes && (misaligned(codes, 16) || ld_codes % 16)) || (codes_t && (misaligned(codes_t, 16) || ld_codes_t % 16))) return LQ_ERR_ARG;
  if (misaligned(scale, 4) || misaligned(scale_t, 4)) return LQ_ERR_ARG;
  const Fp8Quantize q{X, m, d, ldx, dtype, codes, ld_codes, scale, codes_t, ld_codes_t, scale_t};
  return launch_fp8_quantize(&q, 1, tiles == 1, (hipStream_t)stream);
}

size_t lq_fp8_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k) {
  if (bad_rows(m) || bad_rows(n) || bad_depth(k)) return 0;
  return up256(fp8_product_part_floats(n, m, k) * 4);
}

int lq_fp8_matmul(const lq_fp8_matrix* A, const lq_fp8_matrix* B, int64_t m, int64_t n, int64_t k, void* Y, int64_t ldy, void* workspace,
                  size_t workspace_bytes, void* stream) {
  if (!Y) return LQ_ERR_NULL;
  if (bad_rows(m) || bad_rows(n) || bad_depth(k) || ldy < n || ldy > MOST_LD) return LQ_ERR_SHAPE;
  LQ_TRY(check_matrix(A, k));
  LQ_TRY(check_matrix(B, k));
  if (misaligned(Y, 2)) return LQ_ERR_ARG;
  const size_t floats = fp8_product_part_floats(n, m, k);
  if (no_space(workspace, workspace_bytes, floats * 4)) return LQ_ERR_WORKSPACE;
  return launch_fp8_product({operand(*B, n), operand(*A, m), k, Y, ldy}, static_cast<float*>(workspace), floats, (hipStream_t)stream);
}

size_t lq_fp8_forward_workspace_bytes(int64_t m, int64_t n, int64_t k) {
  if (bad_rows(m) || bad_rows(n) || bad_depth(k)) return 0;
  return plan_forward(nullptr, m, n, k).bytes;
}

int lq_fp8_forward(const void* X, int64_t ldx, int x_dtype, const lq_fp8_matrix* W, int64_t m, int64_t n, int64_t k, void* Y, void* workspace,
                   size_t workspace_bytes, void* stream) {
  if (!X || !Y) return LQ_ERR_NULL;
  if (bad_rows(m) || bad_rows(n) || bad_depth(k) || ldx < k || ldx > MOST_LD) return LQ_ERR_SHAPE;
  LQ_TRY(check_matrix(W, k));
  if (bad_type(x_dtype) || misaligned(X, type_bytes(x_dtype)) || misaligned(Y, 2)) return LQ_ERR_ARG;
  const ForwardPlan p = plan_forward(workspace, m, n, k);
  if (no_space(workspace, workspace_bytes, p.bytes)) return LQ_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  Fp8Product raw{operand(*W, n), {}, k, Y, n};
  raw.columns.count = m;
  if (fp8_quantizes_columns(raw)) return launch_fp8_product_raw(raw, X, ldx, x_dtype, p.part, p.part_floats, st);
  const Fp8Quantize q{X, m, k, ldx, x_dtype, p.x.codes, p.x.ld, p.x.scale, nullptr, 0, nullptr};
  LQ_TRY(launch_fp8_quantize(&q, 1, false, st));
  return launch_fp8_product({operand(*W, n), p.x.rows(m), k, Y, n}, p.part, p.part_floats, st);
}

size_t lq_fp8_backward_workspace_bytes(int64_t m, int64_t n, int64_t k, int want_dx, int want_dw) {
  if (bad_gradients(m, n, k, want_dx != 0, want_dw != 0)) return 0;
  return plan_backward(nullptr, m, n, k, want_dx != 0, want_dw != 0).bytes;
}

int lq_fp8_backward(const void* dY, int64_t ldy, int dy_dtype, const void* X, int64_t ldx, int x_dtype, const lq_fp8_matrix* Wt, int64_t m,
                    int64_t n, int64_t k, void* dX, void* dW, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dY || (!dX && !dW) || (dW && !X)) return LQ_ERR_NULL;
  if (bad_gradients(m, n, k, dX != nullptr, dW != nullptr) || ldy < n || ldy > MOST_LD) return LQ_ERR_SHAPE;
  if (bad_type(dy_dtype) || misaligned(dY, type_bytes(dy_dtype)) || misaligned(dX, 2) || misaligned(dW, 2)) return LQ_ERR_ARG;
  if (dW) {
    if (ldx < k || ldx > MOST_LD) return LQ_ERR_SHAPE;
    if (bad_type(x_dtype) || misaligned(X, type_bytes(x_dtype))) return LQ_ERR_ARG;
  }
  if (dX) LQ_TRY(check_matrix(Wt, n));
  const BackwardPlan p = plan_backward(workspace, m, n, k, dX != nullptr, dW != nullptr);
  if (no_space(workspace, workspace_bytes, p.bytes)) return LQ_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  if (dX && !dW) {
    Fp8Product raw{operand(*Wt, k), {}, n, dX, k};
    raw.columns.count = m;
    if (fp8_quantizes_columns(raw)) return launch_fp8_product_raw(raw, dY, ldy, dy_dtype, p.part, p.part_floats, st);
  }
  const Fp8Quantize q[2] = {{dY, m, n, ldy, dy_dtype, p.dy.codes, p.dy.ld, p.dy.scale, p.dyt.codes, p.dyt.ld, p.dyt.scale},
                            {X, m, k, ldx, x_dtype, nullptr, 0, nullptr, p.xt.codes, p.xt.ld, p.xt.scale}};
  LQ_TRY(launch_fp8_quantize(q, dW ? 2 : 1, false, st));
  if (dX) LQ_TRY(launch_fp8_product({operand(*Wt, k), p.dy.rows(m), n, dX, k}, p.part, p.part_floats, st));
  if (!dW) return LQ_OK;
  return launch_fp8_product({p.xt.rows(k), p.dyt.rows(n), m, dW, k}, p.part, p.part_floats, st);
}

}  // extern "C"
