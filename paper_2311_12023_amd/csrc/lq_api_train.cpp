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
// Byte offsets inside a tile of 256 rows are 32 bits wide: rows of a plane are at most this far apart.
constexpr int64_t MOST_PITCH = (int64_t)1 << 23;

// Classes per piece, whole tiles.  Up to 2^28 logits the whole vocabulary is one piece, since dW then comes from E and not from a second
// product (E and dW's operand take 3 GiB at most): 4096 x 4096 by 32000, bf16 2.83 ms for 3.46 in pieces of 2^26, 2048 x 1024 by 50265
// fp32 2.33 for 3.06; without dW 1.76 for 1.73 and 1.49 for 1.57.  Above, pieces of 2^26, whose E stays within the memory-side cache
// (4096 x 4096 by 128000 without dW 6.73 ms; pieces of 2^24 7.27, of 2^28 6.88).
static int64_t piece_classes(int64_t n, int64_t vocab) {
  const int64_t whole = up_to(vocab, SEG_T);
  if (n <= ((int64_t)1 << 28) / whole && whole <= MOST_PITCH / 2) return whole;
  const int64_t most = std::min(std::max<int64_t>(SEG_T, ((int64_t)1 << 26) / n / SEG_T * SEG_T), MOST_PITCH / 2);
  const int64_t pieces = (vocab + most - 1) / most;
  return up_to((vocab + pieces - 1) / pieces, SEG_T);
}

// Few rows by their own kernels or by the products of many rows; us of the former and the latter, without dX / with it where both are
// given.  Where rows are long and classes few, the former have few workgroups, each with a long way.
// fp32, 64 rows: d = 1024, 700 classes 42 / 62 and 40 / 69; d = 2048, 1500 classes 67 / 86 and 49 / 78, 4500 68 / 95 and 66 / 104; d = 4096,
// 3000 classes 118 / 147 and 81 / 119, 6000 117 / 154 and 118 / 171; d = 8192, 6000 classes 217 / 273 and 208 / 292.
// bf16, up to 64 rows: d = 2048, 6000 classes 29 / 46 and 32 / 58; d = 4096, 6000 classes 45 / 64 and 35 / 63, 12000 46 / 72 and 42 / 80.
// bf16, more rows, which take the former twice as long: up to 64 tiles of classes the logits of rows of 2048 and more go in ranges
// (tail_classes), the tiles of up to 65536 classes are one round of the chip.  128 rows: d = 2048, 6000 classes 38 / 64 and 33 / 62, 18000
// 45 / 84 and 55 / 97, 32000 48 / 103 and 55 / 109, 40000 59 / 123 and 57 / 116, 128000 191 / 376 and 148 / 297; d = 1024, 6000 classes
// 27 / 46 and 35 / 65; d = 512, 40000 classes 32 / 60 and 29 / 74.
static bool few_by_size(int64_t n, int64_t d, int64_t vocab, bool half, bool want_dw) {
  if (n > LOSS_FEW || vocab > MOST_PITCH / 2 || want_dw) return false;
  if (half) return d * (6500 - vocab) <= 8000000;
  if (n <= 64) return d < 2560 || vocab > 10000;
  return vocab <= 64 * SEG_T ? d < 2048 : vocab <= 36000 || d <= 512;
}

struct LossPlan {
  LossRows rows;
  float *factors, *part_ref, *part_sum, *acc, *part, *x_inv;
  uint32_t* tops;                                    // of W, of the rows of X that count
  uint16_t *x[2], *xt[2], *w[2], *e[2], *g[2];
  bool whole;                                        // one piece is the whole vocabulary
  uint16_t *few_x[3], *few_e[3];                     // the few rows' planes
  float* few_part;
  float *class_tops, *class_inv, *g32, *e32;         // fp32: for dW's operand
  int64_t classes, d64, n64, v64;
  size_t part_floats, bytes;
};
static LossPlan plan_loss(void* ws, int64_t n, int64_t d, int64_t vocab, int dtype, bool want_dx, bool want_dw) {
  LossPlan p{};
  Arena a(ws);
  const bool half = dtype == LQ_T_FP32;
  p.classes = piece_classes(n, vocab);
  p.whole = p.classes >= vocab;
  p.d64 = up_to(d, 64);
  p.n64 = up_to(n, 64);
  for (float** row : {&p.rows.ref, &p.rows.sum, &p.rows.shift, &p.rows.target, &p.rows.wrong, &p.rows.lse2}) *row = a.take<float>(n);
  p.factors = a.take<float>(2);
  p.tops = a.take<uint32_t>(2);
  p.x_inv = a.take<float>(half ? n : 0);
  const bool few = few_by_size(n, d, vocab, half, want_dw);
  p.v64 = up_to(vocab, 64);
  const int64_t tiles = std::max(p.classes / SEG_T, few ? p.v64 / LOSS_FEW_TILE : 0);
  for (int h = 0; h < (half ? 3 : 1); ++h) {
    p.few_x[h] = a.take<uint16_t>(few ? few_rows(n) * p.d64 : 0);
    p.few_e[h] = a.take<uint16_t>(few && want_dx ? few_rows(n) * p.v64 : 0);
  }
  p.few_part = a.take<float>(few && want_dx ? (size_t)few_dx_splits(vocab, d) * d * few_rows(n) : 0);
  p.part_ref = a.take<float>(tiles * n);
  p.part_sum = a.take<float>(tiles * n);
  p.e[1] = a.take<uint16_t>(!half && want_dw && p.whole ? n * p.classes : 0);      // dW comes from E then
  for (int h = 0; h < (half ? 2 : 1); ++h) {
    p.x[h] = a.take<uint16_t>(n * p.d64);
    p.w[h] = a.take<uint16_t>(p.classes * p.d64);
    p.xt[h] = a.take<uint16_t>(want_dw ? d * p.n64 : 0);
    p.e[h] = a.take<uint16_t>(want_dx || (want_dw && p.whole && !half) ? n * p.classes : 0);
    p.g[h] = a.take<uint16_t>(want_dw ? p.classes * p.n64 : 0);
  }
  p.class_tops = a.take<float>(half && want_dw && p.whole ? loss_class_ranges(n) * vocab : 0);
  p.class_inv = a.take<float>(half && want_dw ? p.classes : 0);
  p.e32 = a.take<float>(half && want_dw && p.whole ? n * p.classes : 0);
  p.g32 = a.take<float>(half && want_dw && !p.whole ? p.classes * p.n64 : 0);
  p.acc = a.take<float>(want_dx ? n * d : 0);
  // The last piece may be shorter and be cut into other numbers of ranges: tiles times ranges stay within 256 in any case.
  const size_t most = (size_t)256 * SEG_T * SEG_T;
  const int s1 = want_dx ? loss_accumulate_splits(n, d, p.classes, half) : 1;
  p.part_floats = s1 > 1 ? std::min((size_t)s1 * n * d, most) : 0;
  if (want_dw && loss_dw_splits(1, 1, p.n64, half) > 1)
    p.part_floats = std::max(p.part_floats, std::min((size_t)16 * std::min(p.classes, vocab) * d, most));
  const int64_t first = std::min(p.classes, vocab), last = vocab - (vocab - 1) / p.classes * p.classes;
  if (!few) p.part_floats = std::max({p.part_floats, loss_tail_floats(n, first, p.d64, half), loss_tail_floats(n, last, p.d64, half)});
  p.part = a.take<float>(p.part_floats);
  p.bytes = a.used();
  return p;
}

static bool loss_sizes_ok(int64_t n, int64_t d, int64_t vocab) {
  const int64_t lim = (int64_t)1 << 31;
  return n > 0 && d > 0 && vocab > 0 && n <= MOST_PITCH - 64 && d <= (1 << 20) && vocab <= lim - 65536;
}

// ---- adapter products ---------------------------------------------------------------------------------
struct AdapterPlan {
  int64_t r32, r64, in64, m64;               // in64: the large product's reduction
  uint16_t *b[3], *a2[3], *b2[3], *ut[3], *tt[3], *q[2], *x[2];
  float *thin, *part, *inv; uint32_t* top;
  size_t part_floats, bytes;
};
// The planes of the large product: `features` rows of weights, m rows of activations, and the low-rank operands of both.
static void plan_product(AdapterPlan& p, Arena& a, int64_t m, int64_t features, int64_t depth, int dtype) {
  const bool half = dtype == LQ_T_FP32;
  p.in64 = up_to(depth, 64);
  for (int h = 0; h < 2; ++h) {
    p.q[h] = a.take<uint16_t>(h == 0 || half ? features * p.in64 : 0);
    p.x[h] = a.take<uint16_t>(half || (h == 0 && depth % 64) ? m * p.in64 : 0);
  }
  for (int h = 0; h < 3; ++h) {
    p.a2[h] = a.take<uint16_t>(features * p.r64);
    p.b2[h] = a.take<uint16_t>(m * p.r64);
  }
  p.inv = a.take<float>(half ? m : 0);
  p.top = a.take<uint32_t>(TOP_WORDS);
  p.part_floats = adapter_part_floats(features, m, p.in64, p.r64, dtype);
  p.part = a.take<float>(p.part_floats);
}
static AdapterPlan plan_forward(void* ws, int64_t m, int64_t d, int64_t k, int rank, int dtype) {
  AdapterPlan p{};
  Arena a(ws);
  p.r32 = up_to(rank, 32); p.r64 = up_to(rank, 64);
  for (int h = 0; h < 3; ++h) p.b[h] = a.take<uint16_t>(p.r32 * up_to(d, 64));         // L1^T
  p.thin = a.take<float>((size_t)thin_project_splits(m, d) * m * p.r32);
  plan_product(p, a, m, k, d, dtype);
  p.bytes = a.used();
  return p;
}
static AdapterPlan plan_backward(void* ws, int64_t m, int64_t d, int64_t k, int rank, int dtype) {
  AdapterPlan p{};
  Arena a(ws);
  p.r32 = up_to(rank, 32); p.r64 = up_to(rank, 64); p.m64 = up_to(m, 64);
  for (int h = 0; h < 3; ++h) {
    p.b[h] = a.take<uint16_t>(p.r32 * up_to(k, 64));                                   // L2
    p.ut[h] = a.take<uint16_t>(p.r32 * p.m64);
    p.tt[h] = a.take<uint16_t>(p.r32 * p.m64);
  }
  p.thin = a.take<float>(std::max((size_t)thin_project_splits(m, k) * m, (size_t)thin_gram_splits(m, k, d) * (k + d)) * p.r32);
  plan_product(p, a, m, d, k, dtype);
  p.bytes = a.used();
  return p;
}

// What the large product takes its activations from (bf16 ones of whole pairs of steps are read where they are), and the passes
// for it and for the weights' scale.
static int activation_planes(const AdapterPlan& p, const MvWeights& q, int64_t weights, const void* x, int64_t m, int64_t depth, int dtype,
                             PrepareJobs& jobs, Planes* act) {
  if (dtype == LQ_T_BF16 && depth % 64 == 0) {
    *act = Planes{{static_cast<const uint16_t*>(x), nullptr, nullptr}, depth};
    return LQ_OK;
  }
  const PlaneTarget t{{p.x[0], dtype == LQ_T_FP32 ? p.x[1] : nullptr, nullptr}, p.in64, m};
  const PlaneSource s{x, dtype, depth, m, depth, nullptr};
  *act = planes_of(t);
  if (dtype == LQ_T_BF16) return jobs.rows(s, t);
  const int64_t group = (int64_t)q.block * q.scale_block;
  LQ_TRY(jobs.tops(q.v, (weights + group - 1) / group, p.top));       // no weight is larger than its group's scale
  return jobs.rows_scaled(s, t, p.inv);
}
static WeightPlanes weight_planes(const AdapterPlan& p, const MvWeights& q, int64_t d, int64_t k, bool transposed, int dtype) {
  return WeightPlanes{q, d, k, transposed, p.top, p.q[0], dtype == LQ_T_FP32 ? p.q[1] : nullptr, p.in64};
}
static Planes planes_of(const WeightPlanes& w) { return Planes{{w.hi, w.lo, nullptr}, w.pitch}; }

// The low-rank part in the large product: two of its planes (16 bits) where the result is bf16, all three where it is fp32.
static Planes low_rank_planes(const PlaneTarget& t, int dtype) {
  Planes p = planes_of(t);
  if (dtype == LQ_T_BF16) p.p[2] = nullptr;
  return p;
}

static int check_adapter(int64_t m, int64_t d, int64_t k, int rank, int dtype, lq_config& c) {
  if (rank < 1 || rank > ADAPTER_MAX_RANK) return LQ_ERR_RANK;
  const int64_t lim = (int64_t)1 << 31;
  if (m <= 0 || d <= 0 || k <= 0 || m >= lim || d >= lim || k >= lim || d % 32) return LQ_ERR_SHAPE;
  LQ_TRY(check_quant_args(d * k, c));
  if (k % c.block) return LQ_ERR_SHAPE;
  if (bad_type(dtype)) return LQ_ERR_ARG;
  if (m >= (1 << 24) || up_to(m, 256) * d >= lim || up_to(m, 256) * k >= lim || d * k >= lim) return LQ_ERR_SHAPE;
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
  const bool half = dtype == LQ_T_FP32;
  const PlaneKind kind = half ? PLANE_HALF_2 : PLANE_BF16;
  const LossScales scales{half ? p.x_inv : nullptr, half ? p.tops : nullptr, half && dW ? p.tops + 1 : nullptr};
  // bf16 operands whose rows are whole pairs of steps on 16-byte addresses are read where they are
  auto in_place = [&](const void* a, int64_t ld) { return !half && d % 64 == 0 && ld % 8 == 0 && ld <= MOST_PITCH && !misaligned(a, 16); };
  const char* w0 = static_cast<const char*>(W);
  const bool few = few_by_size(n, d, vocab, half, dW != nullptr);
  if (half && !few) LQ_TRY(launch_zero_words(p.tops, 2, st));
  Planes x{{static_cast<const uint16_t*>(X), nullptr, nullptr}, ldx};
  if (!few && !in_place(X, ldx)) {
    const PlaneTarget t{{p.x[0], p.x[1], nullptr}, p.d64, n};
    LQ_TRY(launch_row_planes({X, dtype, ldx, n, d, nullptr}, kind, t, half ? p.x_inv : nullptr, st));
    x = planes_of(t);
  }
  if (!few && half) LQ_TRY(launch_top_magnitude(W, ldw, vocab, d, nullptr, 0, p.tops, st));
  const bool w_in_place = in_place(W, ldw);
  auto piece_source = [&](int64_t v0, int64_t classes) {
    return PlaneSource{w0 + (size_t)v0 * (size_t)ldw * size, dtype, ldw, classes, d, p.tops};
  };
  auto piece_planes = [&](int64_t v0, int64_t classes, Planes* w) -> int {
    const PlaneSource from = piece_source(v0, classes);
    *w = Planes{{static_cast<const uint16_t*>(from.src), nullptr, nullptr}, ldw};
    if (w_in_place) return LQ_OK;
    const PlaneTarget t{{p.w[0], p.w[1], nullptr}, p.d64, classes};
    *w = planes_of(t);
    return launch_row_planes(from, kind, t, nullptr, st);
  };
  const LossPiece all{n, 0, vocab, vocab, targets};
  const bool join_rows = few && n <= 16;
  if (few) {
    const int vec = d % 8 == 0 && ldx % 8 == 0 && ldw % 8 == 0 && !misaligned(X, 8 * size) && !misaligned(W, 8 * size);
    const LossOperands operands{X, ldx, W, ldw, d, dtype, vec};
    const PlaneTarget t{{p.few_x[0], p.few_x[1], p.few_x[2]}, p.d64, few_rows(n)};
    uint16_t* const e[3] = {dX ? p.few_e[0] : nullptr, dX ? p.few_e[1] : nullptr, dX ? p.few_e[2] : nullptr};
    uint16_t* const none[2] = {nullptr, nullptr};
    LQ_TRY(launch_row_planes({X, dtype, ldx, n, d, nullptr}, half ? PLANE_BF16_3 : PLANE_BF16, t, nullptr, st));
    LQ_TRY(launch_few_logits(W, ldw, dtype, d, planes_of(t), all, p.part_ref, p.part_sum, e, p.v64, st));
    if (join_rows)
      LQ_TRY(launch_loss_join_rows(all, p.rows, p.part_ref, p.part_sum, LOSS_FEW_TILE, mean == 1, operands, loss, row_loss, lse, p.factors, st));
    else
      LQ_TRY(launch_loss_join(all, p.rows, half, false, p.part_ref, p.part_sum, LOSS_FEW_TILE, none, 0, operands, st));
  }
  uint16_t* const none[2] = {nullptr, nullptr};
  if (!few && !half) LQ_TRY(launch_loss_reference(X, ldx, W, ldw, d, all, p.rows, st));
  const bool late = half && dW && p.whole;      // the pass that makes dW's operand of E makes E's planes as well
  uint16_t* const* e = (dX || (dW && p.whole)) && !late ? p.e : none;
  auto accumulate = [&](const LossPiece& piece, const Planes& w) {
    return launch_loss_accumulate(Planes{{p.e[0], half ? p.e[1] : nullptr, nullptr}, p.classes}, w, piece.classes, n, d, p.rows.shift,
                                  piece.v0 == 0, p.acc, p.part, p.part_floats, st);
  };
  Planes whole;
  for (int64_t v0 = 0; !few && v0 < vocab; v0 += p.classes) {
    const LossPiece piece{n, v0, std::min(p.classes, vocab - v0), vocab, targets};
    Planes w;
    LQ_TRY(piece_planes(v0, piece.classes, &w));
    LQ_TRY(launch_loss_logits(w, x, p.d64, piece, p.rows, scales, p.part_ref, p.part_sum, e,
                              late ? p.e32 : nullptr, p.classes, p.part, p.part_floats, st));
    LQ_TRY(launch_loss_join(piece, p.rows, half, !half, p.part_ref, p.part_sum, SEG_T, e, p.classes, LossOperands{}, st));
    if (late) whole = w;
    else if (dX) LQ_TRY(accumulate(piece, w));
  }
  if (scales.xt_top) LQ_TRY(launch_top_magnitude(X, ldx, n, d, targets, vocab, p.tops + 1, st));
  if (!join_rows) LQ_TRY(launch_loss_rows(p.rows, scales, targets, n, vocab, mean == 1, loss, row_loss, lse, p.factors, st));
  if (dW && p.whole)
    LQ_TRY(launch_loss_gradient_from_e(all, p.rows, p.part_ref, p.e32, p.e, p.classes, p.g, p.n64, p.class_tops, p.class_inv, st));
  if (late && dX) LQ_TRY(accumulate(all, whole));
  if (dX && few) {
    LQ_TRY(launch_few_dx(W, ldw, dtype, d, Planes{{p.few_e[0], p.few_e[1], p.few_e[2]}, p.v64}, all, p.rows, p.part_ref, p.factors,
                         p.few_part, dX, st));
  } else if (dX) {
    LQ_TRY(launch_loss_dx(p.rows, scales, targets, n, d, vocab, p.acc, W, ldw, dtype, p.factors, dX, st));
  }
  if (!dW) return LQ_OK;
  const PlaneTarget xt{{p.xt[0], p.xt[1], nullptr}, p.n64, d};
  LQ_TRY(launch_column_planes({X, dtype, ldx, n, d, p.tops + 1}, kind, xt, targets, vocab, st));
  for (int64_t v0 = 0; v0 < vocab; v0 += p.classes) {
    const LossPiece piece{n, v0, std::min(p.classes, vocab - v0), vocab, targets};
    if (!p.whole) {
      Planes w;
      LQ_TRY(piece_planes(v0, piece.classes, &w));
      LQ_TRY(launch_loss_gradient(w, x, p.d64, piece, p.rows, scales, half ? (void*)p.g32 : p.g[0], p.n64, st));
      if (half)
        LQ_TRY(launch_row_planes({p.g32, LQ_T_FP32, p.n64, piece.classes, n, nullptr}, PLANE_HALF_2,
                                 {{p.g[0], p.g[1], nullptr}, p.n64, piece.classes}, p.class_inv, st));
    }
    LQ_TRY(launch_loss_dw(Planes{{p.g[0], p.g[1], nullptr}, p.n64}, planes_of(xt), p.n64, piece.classes, d, p.factors + 1, p.class_inv, dtype,
                          static_cast<char*>(dW) + (size_t)v0 * (size_t)d * size, p.part, p.part_floats, st));
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
  const PlaneTarget l1{{w.b[0], w.b[1], w.b[2]}, up_to(d, 64), w.r32}, none{};
  const PlaneTarget t{{w.b2[0], w.b2[1], w.b2[2]}, w.r64, m}, l2{{w.a2[0], w.a2[1], w.a2[2]}, w.r64, k};
  PrepareJobs jobs{};
  Planes act;
  LQ_TRY(jobs.columns3({L1, LQ_T_FP32, rank, d, rank, nullptr}, l1));
  LQ_TRY(jobs.columns3({L2, LQ_T_FP32, k, rank, k, nullptr}, l2));
  LQ_TRY(activation_planes(w, q, d * k, X, m, d, dtype, jobs, &act));
  LQ_TRY(jobs.launch(st));
  LQ_TRY(launch_thin_project(X, dtype, m, d, planes_of(l1), r32, mask, w.thin, st));
  const WeightPlanes weights = weight_planes(w, q, d, k, true, dtype);
  LQ_TRY(launch_finish({w.thin, thin_project_splits(m, d), m, rank, r32, mask.scale, T, t, none}, &weights, st));
  return launch_adapter_product(planes_of(weights), act, w.in64, low_rank_planes(l2, dtype), low_rank_planes(t, dtype), w.r64, {w.inv, w.top}, k, m,
                                nullptr, dtype, Y, w.part, w.part_floats, st);
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
  const MvWeights q{codes_packed, scale_idx, v, c.bits, c.block, c.scale_block, scale_levels(c)};
  const PlaneTarget l2{{w.b[0], w.b[1], w.b[2]}, up_to(k, 64), w.r32}, none{};
  const PlaneTarget u{{w.b2[0], w.b2[1], w.b2[2]}, w.r64, m}, l1{{w.a2[0], w.a2[1], w.a2[2]}, w.r64, d};
  const PlaneTarget ut{{w.ut[0], w.ut[1], w.ut[2]}, w.m64, w.r32}, tt{{w.tt[0], w.tt[1], w.tt[2]}, w.m64, w.r32};
  PrepareJobs jobs{};
  Planes act;
  LQ_TRY(jobs.rows3({L2, LQ_T_FP32, k, rank, k, nullptr}, l2));
  LQ_TRY(jobs.columns3({T, LQ_T_FP32, rank, m, rank, nullptr}, tt));
  if (dX) {
    LQ_TRY(jobs.rows3({L1, LQ_T_FP32, rank, d, rank, nullptr}, l1));
    LQ_TRY(activation_planes(w, q, d * k, dY, m, k, dtype, jobs, &act));
  }
  LQ_TRY(jobs.launch(st));
  LQ_TRY(launch_thin_project(dY, dtype, m, k, planes_of(l2), r32, DropoutMask{}, w.thin, st));
  const ThinFinish finish{w.thin, thin_project_splits(m, k), m, rank, r32, 1.0f, nullptr, u, ut};
  const WeightPlanes weights = weight_planes(w, q, d, k, false, dtype);
  const bool sums = thin_gram_splits(m, k, d) > 1;
  LQ_TRY(launch_finish(finish, dX && !sums ? &weights : nullptr, st));
  ThinGramSum sum;
  LQ_TRY(launch_thin_grams(dY, k, planes_of(tt), dL2, X, d, planes_of(ut), mask, dL1, dtype, m, rank, r32, w.thin, &sum, st));
  if (sums) LQ_TRY(launch_gram_sum(sum, dX ? &weights : nullptr, st));
  if (!dX) return LQ_OK;
  return launch_adapter_product(planes_of(weights), act, w.in64, low_rank_planes(l1, dtype), low_rank_planes(u, dtype), w.r64, {w.inv, w.top}, d, m,
                                mask.cut ? &mask : nullptr, dtype, dX, w.part, w.part_floats, st);
}

}  // extern "C"
