// C ABI of the optimizer's step.
#include <cmath>
#include <vector>

#include "fp8.h"

namespace lq {

constexpr int64_t MOST_TENSORS = (int64_t)1 << 24, MOST_VALUES = (int64_t)1 << 34;

static bool bad_type(int dtype) { return dtype != LQ_T_FP32 && dtype != LQ_T_BF16; }
static bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

static int check_gradients(const lq_gradient* grads, int64_t count) {
  if (count < 1 || count > MOST_TENSORS) return LQ_ERR_ARG;
  if (!grads) return LQ_ERR_NULL;
  for (int64_t i = 0; i < count; ++i) {
    if (grads[i].n < 0 || grads[i].n > MOST_VALUES) return LQ_ERR_SHAPE;
    if (bad_type(grads[i].dtype)) return LQ_ERR_ARG;
    if (!grads[i].n) continue;
    if (!grads[i].g) return LQ_ERR_NULL;
    if (misaligned(grads[i].g, type_bytes(grads[i].dtype))) return LQ_ERR_ARG;
  }
  return LQ_OK;
}

struct Piece { uintptr_t from, to; };
static bool before(const Piece& a, const Piece& b) { return a.from < b.from; }

// Whether two pieces of memory that the step writes overlap, or one of them and one that it only reads.  written: by what they are for;
// one kind's pieces mostly come in order, so that hundreds of tensors take a few passes over them.
constexpr int KINDS = 6;
static bool overlapping(std::vector<Piece> (&written)[KINDS], const std::vector<Piece>& read) {
  std::vector<Piece> all, next;
  for (std::vector<Piece>& kind : written) {
    if (!std::is_sorted(kind.begin(), kind.end(), before)) std::sort(kind.begin(), kind.end(), before);
    next.resize(all.size() + kind.size());
    std::merge(all.begin(), all.end(), kind.begin(), kind.end(), next.begin(), before);
    all.swap(next);
  }
  for (size_t i = 1; i < all.size(); ++i)
    if (all[i].from < all[i - 1].to) return true;
  for (const Piece& r : read) {
    auto it = std::lower_bound(all.begin(), all.end(), Piece{r.to, 0}, before);
    if (it != all.begin() && (it - 1)->to > r.from) return true;
  }
  return false;
}

static int check_tensors(const lq_adamw_tensor* t, int64_t count, bool codes, const lq_adamw_params& h, const float* coef) {
  std::vector<Piece> written[KINDS], read;
  for (std::vector<Piece>& kind : written) kind.reserve((size_t)count);
  read.reserve((size_t)count + 3);
  auto reads = [&](const void* p, int64_t bytes) { if (p) read.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes}); };
  reads(coef, 4);
  reads(h.lr_device, 4);
  reads(h.step_device, 8);
  auto writes = [&](int kind, const void* p, int64_t bytes) { if (p) written[kind].push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes}); };
  for (int64_t i = 0; i < count; ++i) {
    const lq_adamw_tensor& x = t[i];
    if (x.n < 0 || x.n > MOST_VALUES) return LQ_ERR_SHAPE;
    if (bad_type(x.p_dtype) || bad_type(x.g_dtype)) return LQ_ERR_ARG;
    if (!x.n) continue;
    if (!x.p || !x.g || !x.m || !x.v || (codes && (!x.m_scale || !x.v_scale))) return LQ_ERR_NULL;
    if (misaligned(x.p, type_bytes(x.p_dtype)) || misaligned(x.g, type_bytes(x.g_dtype)) || misaligned(x.copy, 2)) return LQ_ERR_ARG;
    if (codes ? misaligned(x.m_scale, 4) || misaligned(x.v_scale, 4) : misaligned(x.m, 4) || misaligned(x.v, 4)) return LQ_ERR_ARG;
    if (x.copy && x.p_dtype != LQ_T_FP32) return LQ_ERR_ARG;
    const int64_t blocks = (x.n + STATE_BLOCK - 1) / STATE_BLOCK;
    writes(0, x.p, x.n * (int64_t)type_bytes(x.p_dtype));
    writes(1, x.m, x.n * (codes ? 1 : 4));
    writes(2, x.v, x.n * (codes ? 1 : 4));
    writes(3, x.copy, x.n * 2);
    reads(x.g, x.n * (int64_t)type_bytes(x.g_dtype));
    if (codes) { writes(4, x.m_scale, blocks * 4); writes(5, x.v_scale, blocks * 4); }
  }
  return overlapping(written, read) ? LQ_ERR_ARG : LQ_OK;
}

}  // namespace lq

using namespace lq;

extern "C" {

size_t lq_grad_norm_workspace_bytes(const lq_gradient* grads, int64_t count) {
  return check_gradients(grads, count) == LQ_OK ? up256(std::max<size_t>(1, grad_norm_parts(grads, count)) * sizeof(double)) : 0;
}

int lq_grad_norm(const lq_gradient* grads, int64_t count, double max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  if (!norm) return LQ_ERR_NULL;
  LQ_TRY(check_gradients(grads, count));
  if (!(max_norm > 0.0) || misaligned(norm, 4)) return LQ_ERR_ARG;
  if (!workspace || misaligned(workspace, 256) || workspace_bytes < up256(std::max<size_t>(1, grad_norm_parts(grads, count)) * sizeof(double)))
    return LQ_ERR_WORKSPACE;
  return launch_grad_norm(grads, count, (float)max_norm, norm, static_cast<double*>(workspace), (hipStream_t)stream);
}

int lq_adamw(const lq_adamw_tensor* tensors, int64_t count, int state_bits, const lq_adamw_params* params, const float* coef, void* stream) {
  if (!tensors || !params) return LQ_ERR_NULL;
  if (count < 1 || count > MOST_TENSORS || (state_bits != 8 && state_bits != 32)) return LQ_ERR_ARG;
  const lq_adamw_params& h = *params;
  auto fraction = [](double b) { return b >= 0.0 && b < 1.0; };
  if (!fraction(h.beta1) || !fraction(h.beta2) || !(h.eps >= 0.0) || !std::isfinite(h.eps) || !std::isfinite(h.weight_decay)) return LQ_ERR_ARG;
  if ((!h.lr_device && !std::isfinite(h.lr)) || (!h.step_device && h.step < 1)) return LQ_ERR_ARG;
  if (misaligned(h.lr_device, 4) || misaligned(h.step_device, 8) || misaligned(coef, 4)) return LQ_ERR_ARG;
  try {
    LQ_TRY(check_tensors(tensors, count, state_bits == 8, h, coef));
  } catch (...) {                          // no memory for the list of what is written
    return LQ_ERR_ARG;
  }
  return launch_adamw(tensors, count, state_bits, h, coef, (hipStream_t)stream);
}

}  // extern "C"
