// C ABI of the training operators: dropout, softmax cross entropy with its gradients, the adapter product with dropout and its
// gradients.
#include <cmath>

#include "train.h"

namespace lq {
int check_quant_args(int64_t n, lq_config& c);

int dropout_mask(double p, uint64_t seed, uint64_t offset, DropoutMask* d) {
  if (!(p >= 0.0 && p <= 1.0)) return LQ_ERR_ARG;             // NaN too
  d->seed = seed;
  d->offset = offset;
  d->cut = (uint32_t)std::floor(65536.0 * p + 0.5);
  d->scale = d->cut < 65536 ? (float)(65536.0 / (65536 - d->cut)) : 0.0f;
  return LQ_OK;
}

// Regions of a workspace one after the other; without a base address it only counts.
class Arena {
  char* base_;
  size_t used_ = 0;

 public:
  explicit Arena(void* base) : base_(static_cast<char*>(base)) {}
  template <typename T>
  T* take(size_t count) {
    T* p = base_ ? reinterpret_cast<T*>(base_ + used_) : nullptr;
    used_ += up256(count * sizeof(T));
    return count && base_ ? p : nullptr;
  }
  size_t used() const { return used_; }
};

static bool bad_type(int dtype) { return dtype != LQ_T_FP32 && dtype != LQ_T_BF16; }
static bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// ---- cross entropy ------------------------------------------------------------------------------------
// Classes per piece: E of a piece stays within 64 MiB per plane, so that it is still in the memory-side cache when the next
// product reads it; pieces of equal size, whole tiles.
static int64_t piece_classes(int64_t n, int64_t vocab) {
  const int64_t most = std::max<int64_t>(SEG_T, ((int64_t)1 << 25) / n / SEG_T * SEG_T);
  const int64_t pieces = (vocab + most - 1) / most;
  return up_to((vocab + pieces - 1) / pieces, SEG_T);
}

struct LossPlan {
  LossRows rows;
  float *factor, *part_ref, *part_sum, *acc, *part;
  uint16_t *x[2], *xt[2], *w[2], *wt[2], *e[2];      // hi, lo
  int64_t classes, d32, n64;
  size_t part_floats, bytes;
};
static LossPlan plan_loss(void* ws, int64_t n, int64_t d, int64_t vocab, int dtype, bool want_dx, bool want_dw) {
  LossPlan p{};
  Arena a(ws);
  const int planes = type_planes(dtype);
  p.classes = piece_classes(n, vocab);
  p.d32 = up_to(d, 32);
  p.n64 = up_to(n, 64);
  for (float** row : {&p.rows.ref, &p.rows.sum, &p.rows.shift, &p.rows.target, &p.rows.wrong, &p.rows.lse2}) *row = a.take<float>(n);
  p.factor = a.take<float>(1);
  const int64_t tiles = p.classes / SEG_T;
  p.part_ref = a.take<float>(tiles * n);
  p.part_sum = a.take<float>(tiles * n);
  for (int h = 0; h < planes; ++h) {
    p.x[h] = a.take<uint16_t>(n * p.d32);
    p.w[h] = a.take<uint16_t>(p.classes * p.d32);
    p.xt[h] = a.take<uint16_t>(want_dw ? d * p.n64 : 0);
    p.wt[h] = a.take<uint16_t>(want_dx ? d * p.classes : 0);
    // E of a piece, and in the second pass its gradient
    p.e[h] = a.take<uint16_t>(std::max(want_dx ? n * p.classes : 0, want_dw ? p.classes * p.n64 : 0));
  }
  p.acc = a.take<float>(want_dx ? n * d : 0);
  // The last piece may be shorter and be cut into other numbers of ranges: tiles times ranges stay within 256 in any case.
  const size_t most = (size_t)256 * SEG_T * SEG_T;
  const int s1 = want_dx ? loss_accumulate_splits(n, d, p.classes, planes) : 1;
  p.part_floats = s1 > 1 ? std::min((size_t)s1 * n * d, most) : 0;
  if (want_dw && plain_product_splits(1, 1, p.n64, planes) > 1)
    p.part_floats = std::max(p.part_floats, std::min((size_t)16 * std::min(p.classes, vocab) * d, most));
  p.part = a.take<float>(p.part_floats);
  p.bytes = a.used();
  return p;
}

static bool loss_sizes_ok(int64_t n, int64_t d, int64_t vocab) {
  const int64_t lim = (int64_t)1 << 31;
  return n > 0 && d > 0 && vocab > 0 && n <= lim - 65536 && d <= (1 << 20) && vocab <= lim - 65536;
}

// ---- adapter products ---------------------------------------------------------------------------------
struct AdapterPlan {
  int64_t r32, r64, d64, k32, m64, rows_pad, pitch;
  uint16_t *x[2], *t[2], *tt[2], *u[2], *ut[2], *q[2], *dy[2], *b[2], *l1[2], *l2t;
  float *thin, *part, *bscale;
  size_t part_floats, bytes;
};
static AdapterPlan plan_forward(void* ws, int64_t m, int64_t d, int64_t k, int rank, int dtype) {
  AdapterPlan p{};
  Arena a(ws);
  p.r32 = up_to(rank, 32); p.r64 = up_to(rank, 64); p.d64 = up_to(d, 64); p.rows_pad = up_to(m, 256); p.pitch = plane_pitch(d);
  const bool split = dtype == LQ_T_FP32;
  for (int h = 0; h < 2; ++h) {
    p.b[h] = a.take<uint16_t>(p.r32 * p.d64);                             // L1^T
    p.t[h] = a.take<uint16_t>(p.rows_pad * p.r32);
    p.x[h] = a.take<uint16_t>(split ? p.rows_pad * d : 0);
  }
  p.thin = a.take<float>((size_t)thin_project_splits(m, d) * m * p.r32);
  if (split) {
    p.bscale = a.take<float>(d * k / 16);
    p.part_floats = qmatmul_part_floats(m, k, (int)(d / 32 + p.r32 / 32));
  } else {
    p.q[0] = a.take<uint16_t>(weight_plane_elems(p.pitch, k));
    p.l2t = a.take<uint16_t>(k * p.r64);
    const int s = plain_product_splits(m, k, d, 1);
    p.part_floats = s > 1 ? (size_t)s * m * k : 0;
  }
  p.part = a.take<float>(p.part_floats);
  p.bytes = a.used();
  return p;
}
static AdapterPlan plan_backward(void* ws, int64_t m, int64_t d, int64_t k, int rank, int dtype) {
  AdapterPlan p{};
  Arena a(ws);
  p.r32 = up_to(rank, 32); p.k32 = up_to(k, 32); p.m64 = up_to(m, 64);
  const int planes = type_planes(dtype);
  for (int h = 0; h < 2; ++h) {
    p.b[h] = a.take<uint16_t>(p.r32 * p.k32);                             // L2
    p.u[h] = a.take<uint16_t>(m * p.r32);
    p.ut[h] = a.take<uint16_t>(p.r32 * p.m64);
    p.tt[h] = a.take<uint16_t>(p.r32 * p.m64);
    p.l1[h] = a.take<uint16_t>(d * p.r32);
    p.q[h] = a.take<uint16_t>(h < planes ? d * p.k32 : 0);
    p.dy[h] = a.take<uint16_t>(h < planes && (dtype == LQ_T_FP32 || k % 32) ? m * p.k32 : 0);
  }
  const size_t thin = std::max({(size_t)thin_project_splits(m, k) * m, (size_t)2 * thin_gram_splits(m, k) * k,
                                (size_t)2 * thin_gram_splits(m, d) * d});
  p.thin = a.take<float>(thin * p.r32);
  const int s = adapter_dx_splits(m, d, k, planes);
  p.part_floats = s > 1 ? (size_t)s * m * d : 0;
  p.part = a.take<float>(p.part_floats);
  p.bytes = a.used();
  return p;
}

static int check_adapter(int64_t m, int64_t d, int64_t k, int rank, int dtype, lq_config& c) {
  if (rank < 1 || rank > ADAPTER_MAX_RANK) return LQ_ERR_RANK;
  const int64_t lim = (int64_t)1 << 31;
  if (m <= 0 || d <= 0 || k <= 0 || m >= lim || d >= lim || k >= lim || d % 32) return LQ_ERR_SHAPE;
  LQ_TRY(check_quant_args(d * k, c));
  if (k % c.block) return LQ_ERR_SHAPE;
  if (bad_type(dtype)) return LQ_ERR_ARG;
  if (up_to(m, 256) * d >= lim || up_to(m, 256) * k >= lim || d * k >= lim) return LQ_ERR_SHAPE;
  return LQ_OK;
}
static bool adapter_sizes_ok(int64_t m, int64_t d, int64_t k, int rank, int dtype) {
  lq_config c{4, 16, 16, 8, LQ_V_FP32};
  return check_adapter(m, d, k, rank, dtype, c) == LQ_OK;
}
}  // namespace lq

using namespace lq;

extern "C" {

int lq_dropout(const void* x, int64_t n, int dtype, double p, uint64_t seed, uint64_t offset, void* y, void* stream) {
  if (!x || !y) return LQ_ERR_NULL;
  if (n <= 0 || n >= ((int64_t)1 << 60)) return LQ_ERR_SHAPE;
  if (bad_type(dtype) || misaligned(x, type_bytes(dtype)) || misaligned(y, type_bytes(dtype))) return LQ_ERR_ARG;
  DropoutMask d;
  LQ_TRY(dropout_mask(p, seed, offset, &d));
  return launch_dropout(x, n, dtype, d, y, (hipStream_t)stream);
}

size_t lq_cross_entropy_workspace_bytes(int64_t n, int64_t d, int64_t vocab, int dtype, int want_dx, int want_dw) {
  if (!loss_sizes_ok(n, d, vocab) || bad_type(dtype)) return 0;
  return plan_loss(nullptr, n, d, vocab, dtype, want_dx != 0, want_dw != 0).bytes;
}

int lq_cross_entropy(const void* X, int64_t ldx, const void* W, int64_t ldw, const int64_t* targets, int64_t n, int64_t d,
                     int64_t vocab, int dtype, int mean, float* loss, float* row_loss, float* lse, void* dX, void* dW,
                     void* workspace, size_t workspace_bytes, void* stream) {
  if (!X || !W || !targets || !loss || !row_loss) return LQ_ERR_NULL;
  if (!loss_sizes_ok(n, d, vocab) || ldx < d || ldw < d) return LQ_ERR_SHAPE;
  if (bad_type(dtype) || (mean != 0 && mean != 1)) return LQ_ERR_ARG;
  const size_t size = type_bytes(dtype);
  if (misaligned(X, size) || misaligned(W, size) || misaligned(dX, size) || misaligned(dW, size) || misaligned(targets, 8))
    return LQ_ERR_ARG;
  const LossPlan p = plan_loss(workspace, n, d, vocab, dtype, dX != nullptr, dW != nullptr);
  if (!workspace || misaligned(workspace, 256) || workspace_bytes < p.bytes) return LQ_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  const bool split = dtype == LQ_T_FP32;
  // bf16 operands whose rows are whole steps on 16-byte addresses are read where they are
  auto in_place = [&](const void* a, int64_t ld) { return !split && d % 32 == 0 && ld % 8 == 0 && !misaligned(a, 16); };
  Planes x{p.x[0], p.x[1], p.d32};
  if (in_place(X, ldx)) x = {static_cast<const uint16_t*>(X), nullptr, ldx};
  else LQ_TRY(launch_row_planes(X, dtype, ldx, n, d, n, p.x[0], p.x[1], p.d32, st));
  const bool w_in_place = in_place(W, ldw);
  LQ_TRY(launch_loss_begin(p.rows, n, st));
  const char* w0 = static_cast<const char*>(W);
  auto piece_planes = [&](int64_t v0, int64_t classes, Planes* w) -> int {
    const void* from = w0 + (size_t)v0 * (size_t)ldw * size;
    *w = {p.w[0], p.w[1], p.d32};
    if (w_in_place) { *w = {static_cast<const uint16_t*>(from), nullptr, ldw}; return LQ_OK; }
    return launch_row_planes(from, dtype, ldw, classes, d, classes, p.w[0], p.w[1], p.d32, st);
  };
  for (int64_t v0 = 0; v0 < vocab; v0 += p.classes) {
    const LossPiece piece{n, v0, std::min(p.classes, vocab - v0), vocab, targets};
    Planes w;
    LQ_TRY(piece_planes(v0, piece.classes, &w));
    uint16_t *e0 = dX ? p.e[0] : nullptr, *e1 = dX ? p.e[1] : nullptr;
    LQ_TRY(launch_loss_logits(w, x, p.d32, piece, p.rows, p.part_ref, p.part_sum, e0, e1, p.classes, st));
    LQ_TRY(launch_loss_join(piece, p.rows, p.part_ref, p.part_sum, e0, e1, p.classes, st));
    if (!dX) continue;
    LQ_TRY(launch_column_planes(w0 + (size_t)v0 * (size_t)ldw * size, dtype, ldw, piece.classes, d, d, nullptr, 0, p.wt[0], p.wt[1],
                                p.classes, st));
    LQ_TRY(launch_loss_accumulate({e0, e1, p.classes}, {p.wt[0], p.wt[1], p.classes}, up_to(piece.classes, 32), n, d, p.rows.shift,
                                  v0 == 0, p.acc, p.part, p.part_floats, st));
  }
  LQ_TRY(launch_loss_rows(p.rows, targets, n, vocab, mean == 1, loss, row_loss, lse, p.factor, st));
  if (dX) LQ_TRY(launch_loss_dx(p.rows, targets, n, d, vocab, p.acc, W, ldw, dtype, p.factor, dX, st));
  if (!dW) return LQ_OK;
  LQ_TRY(launch_column_planes(X, dtype, ldx, n, d, d, targets, vocab, p.xt[0], p.xt[1], p.n64, st));
  for (int64_t v0 = 0; v0 < vocab; v0 += p.classes) {
    const LossPiece piece{n, v0, std::min(p.classes, vocab - v0), vocab, targets};
    Planes w;
    LQ_TRY(piece_planes(v0, piece.classes, &w));
    LQ_TRY(launch_loss_gradient(w, x, p.d32, piece, p.rows, p.factor, p.e[0], p.e[1], p.n64, st));
    LQ_TRY(launch_plain_product({p.e[0], p.e[1], p.n64}, {p.xt[0], p.xt[1], p.n64}, p.n64, Planes{}, Planes{}, 0, piece.classes, d,
                                dtype, static_cast<char*>(dW) + (size_t)v0 * (size_t)d * size, p.part, p.part_floats, st));
  }
  return LQ_OK;
}

size_t lq_adapter_workspace_bytes(int64_t m, int64_t d, int64_t k, int rank, int dtype, int backward) {
  if (!adapter_sizes_ok(m, d, k, rank, dtype)) return 0;
  return (backward ? plan_backward(nullptr, m, d, k, rank, dtype) : plan_forward(nullptr, m, d, k, rank, dtype)).bytes;
}

int lq_adapter_forward(const void* X, int64_t m, int64_t d, int64_t k, const uint8_t* codes_packed, const uint8_t* scale_idx,
                       const float* v, lq_config c, const float* L1, const float* L2, int rank, int dtype, double p, uint64_t seed,
                       uint64_t offset, void* Y, float* T, void* workspace, size_t workspace_bytes, void* stream) {
  if (!X || !codes_packed || !scale_idx || !v || !L1 || !L2 || !Y || !T) return LQ_ERR_NULL;
  LQ_TRY(check_adapter(m, d, k, rank, dtype, c));
  if (misaligned(X, 16) || misaligned(Y, 16) || misaligned(L1, 4) || misaligned(L2, 16) || misaligned(T, 4)) return LQ_ERR_ARG;
  DropoutMask mask;
  LQ_TRY(dropout_mask(p, seed, offset, &mask));
  const AdapterPlan w = plan_forward(workspace, m, d, k, rank, dtype);
  if (!workspace || misaligned(workspace, 256) || workspace_bytes < w.bytes) return LQ_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  const MvWeights q{codes_packed, scale_idx, v, c.bits, c.block, c.scale_block, scale_levels(c)};
  const int r32 = (int)w.r32;
  LQ_TRY(launch_column_planes(L1, LQ_T_FP32, rank, d, rank, r32, nullptr, 0, w.b[0], w.b[1], w.d64, st));
  LQ_TRY(launch_thin_project(X, dtype, m, d, {w.b[0], w.b[1], w.d64}, r32, mask.cut ? &mask : nullptr, w.thin, st));
  LQ_TRY(launch_thin_finish(w.thin, thin_project_splits(m, d), m, rank, r32, mask.scale, T, w.t[0], w.t[1], nullptr, nullptr, 0, st));
  if (dtype == LQ_T_FP32) {
    LQ_TRY(launch_block_scales(scale_idx, v, d * k / c.block, c.scale_block, scale_levels(c), w.bscale, st));
    LQ_TRY(launch_split_planes(static_cast<const float*>(X), m, d, d, w.rows_pad, d, w.x[0], w.x[1], st));
    const QmmPart qp{w.x[0], w.x[1], d, codes_packed, w.bscale, c.bits, c.block};
    const DensePart tp{w.t[0], w.t[1], w.r32, L2, k, rank, k};
    return launch_qmatmul(qp, tp, m, w.rows_pad, k, static_cast<float*>(Y), k, w.part, w.part_floats, 0, st);
  }
  LQ_TRY(launch_weight_columns(q, d, k, nullptr, 0, 0, w.q[0], nullptr, ProjectSum{}, st));
  LQ_TRY(launch_column_planes(L2, LQ_T_FP32, k, rank, k, k, nullptr, 0, w.l2t, nullptr, w.r64, st));
  return launch_plain_product({static_cast<const uint16_t*>(X), nullptr, d}, {w.q[0], nullptr, w.pitch}, d,
                              {w.t[0], nullptr, w.r32}, {w.l2t, nullptr, w.r64}, w.r32, m, k, dtype, Y, w.part, w.part_floats, st);
}

int lq_adapter_backward(const void* dY, const void* X, int64_t m, int64_t d, int64_t k, const uint8_t* codes_packed,
                        const uint8_t* scale_idx, const float* v, lq_config c, const float* L1, const float* L2, int rank, int dtype,
                        const float* T, double p, uint64_t seed, uint64_t offset, void* dX, float* dL1, float* dL2, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (!dY || !X || !codes_packed || !scale_idx || !v || !L1 || !L2 || !T || !dL1 || !dL2) return LQ_ERR_NULL;
  LQ_TRY(check_adapter(m, d, k, rank, dtype, c));
  if (misaligned(dY, 16) || misaligned(X, 16) || misaligned(dX, 16) || misaligned(L1, 4) || misaligned(L2, 4) || misaligned(T, 4) ||
      misaligned(dL1, 4) || misaligned(dL2, 4))
    return LQ_ERR_ARG;
  DropoutMask mask;
  LQ_TRY(dropout_mask(p, seed, offset, &mask));
  const AdapterPlan w = plan_backward(workspace, m, d, k, rank, dtype);
  if (!workspace || misaligned(workspace, 256) || workspace_bytes < w.bytes) return LQ_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  const int r32 = (int)w.r32;
  const bool split = dtype == LQ_T_FP32;
  // U = dY L2^T, its transpose, and that of T
  LQ_TRY(launch_row_planes(L2, LQ_T_FP32, k, rank, k, r32, w.b[0], w.b[1], w.k32, st));
  LQ_TRY(launch_thin_project(dY, dtype, m, k, {w.b[0], w.b[1], w.k32}, r32, nullptr, w.thin, st));
  LQ_TRY(launch_thin_finish(w.thin, thin_project_splits(m, k), m, rank, r32, 1.0f, nullptr, w.u[0], w.u[1], w.ut[0], w.ut[1], w.m64, st));
  LQ_TRY(launch_thin_finish(T, 0, m, rank, r32, 1.0f, nullptr, nullptr, nullptr, w.tt[0], w.tt[1], w.m64, st));
  LQ_TRY(launch_thin_gram(dY, dtype, m, k, {w.tt[0], w.tt[1], w.m64}, rank, r32, nullptr, 1.0f, true, w.thin, dL2, st));
  LQ_TRY(launch_thin_gram(X, dtype, m, d, {w.ut[0], w.ut[1], w.m64}, rank, r32, mask.cut ? &mask : nullptr, mask.scale, false, w.thin,
                          dL1, st));
  if (!dX) return LQ_OK;
  const MvWeights q{codes_packed, scale_idx, v, c.bits, c.block, c.scale_block, scale_levels(c)};
  LQ_TRY(launch_weight_rows(q, d, k, w.q[0], w.q[1], w.k32, st));
  LQ_TRY(launch_row_planes(L1, LQ_T_FP32, rank, d, rank, d, w.l1[0], split ? w.l1[1] : nullptr, r32, st));
  Planes dy{w.dy[0], w.dy[1], w.k32};
  if (!split && k % 32 == 0) dy = {static_cast<const uint16_t*>(dY), nullptr, k};
  else LQ_TRY(launch_row_planes(dY, dtype, k, m, k, m, w.dy[0], w.dy[1], w.k32, st));
  return launch_adapter_dx({w.q[0], w.q[1], w.k32}, dy, w.k32, {w.l1[0], split ? w.l1[1] : nullptr, w.r32},
                           {w.u[0], split ? w.u[1] : nullptr, w.r32}, r32, m, d, mask, dtype, dX, w.part, w.part_floats, st);
}

}  // extern "C"
