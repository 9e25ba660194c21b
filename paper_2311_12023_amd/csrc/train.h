// Launchers of the training operators (host-callable, all asynchronous on the given stream): dropout, the adapter product with
// dropout and its gradients, softmax cross entropy with its gradients.
#pragma once

#include <algorithm>

#include "kernels.h"
#include "philox_device.h"

namespace lq {

inline size_t type_bytes(int dtype) { return dtype == LQ_T_BF16 ? 2 : 4; }
inline size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }
inline int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
// Planes that an operand of this type takes: bf16 goes in as it is, fp32 as hi + lo.
inline int type_planes(int dtype) { return dtype == LQ_T_BF16 ? 1 : 2; }

// Checks p (0 <= p <= 1) and fills the mask's parameters.
int dropout_mask(double p, uint64_t seed, uint64_t offset, DropoutMask* d);
int launch_dropout(const void* x, int64_t n, int dtype, const DropoutMask& d, void* y, hipStream_t st);

// ---- the product of planes that the operators share (segment_gemm.h) ---------------------------------
constexpr int SEG_T = 256, SEG_STAGES = 4, SEG_THREADS = 512;
constexpr uint32_t SEG_TILE = SEG_T * 64, SEG_STAGE = 2 * SEG_TILE;           // bytes
constexpr size_t SEG_LDS = (size_t)SEG_STAGES * SEG_STAGE;

struct Segment {
  const uint16_t* A; const uint16_t* B;
  int64_t pitch_a, pitch_b;      // elements from row to row, multiples of 8; the planes begin on 16 bytes
  int end;                       // 32-deep steps of this segment and those before it
};
struct SegArgs {
  Segment seg[6];
  int64_t rows_a, rows_b;
  int tiles_m, tiles_n, splits;
};

// One or two planes of an operand.
struct Planes {
  const uint16_t* hi; const uint16_t* lo;       // lo: NULL where hi is all there is
  int64_t pitch;
};
// Appends the segments of A B^T over `depth` (a multiple of 32) reduction indices, from step `first` on; -> the step behind
// them.  The number of segments in use is *count.
inline int add_segments(SegArgs& s, int* count, int first, const Planes& a, const Planes& b, int64_t depth) {
  const int steps = (int)(depth / 32);
  auto add = [&](const uint16_t* pa, const uint16_t* pb) {
    first += steps;
    s.seg[(*count)++] = Segment{pa, pb, a.pitch, b.pitch, first};
  };
  add(a.hi, b.hi);
  if (a.lo) add(a.lo, b.hi);
  if (b.lo) add(a.hi, b.lo);
  return first;
}
inline unsigned seg_grid(const SegArgs& a) { return (unsigned)(((int64_t)a.tiles_m * a.tiles_n * a.splits + 7) / 8 * 8); }
// Ranges that the reduction of a product with few tiles is cut into: the parts fill the chip, each keeps 16 steps.
inline int seg_splits(int64_t tiles, int steps, int most) {
  const int64_t want = 256 / std::max<int64_t>(1, tiles);
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, (int64_t)steps / 16, (int64_t)most}));
}

// ---- planes of an operand (train_planes_kernels.hip) --------------------------------------------------
// rows x cols values of type dtype, ld elements from row to row -> planes with rows of `pitch` elements, zero beyond cols up to
// up_to(cols, 32) and in rows from `rows` to out_rows; lo may be NULL (bf16 sources have nothing there).
int launch_row_planes(const void* src, int dtype, int64_t ld, int64_t rows, int64_t cols, int64_t out_rows, uint16_t* hi,
                      uint16_t* lo, int64_t pitch, hipStream_t st);
// The transpose: planes of out_rows rows, zero from `cols` on, the source's rows contiguous, zero beyond `rows` up to
// up_to(rows, 64).  keep: one int64 per source row; rows whose value lies outside [0, keep_below) are taken as zero, whatever they hold (NULL: all are taken).
int launch_column_planes(const void* src, int dtype, int64_t ld, int64_t rows, int64_t cols, int64_t out_rows,
                         const int64_t* keep, int64_t keep_below, uint16_t* hi, uint16_t* lo, int64_t pitch, hipStream_t st);

// ---- softmax cross entropy (loss_kernels.hip) -----------------------------------------------------------
struct LossRows {            // per-row state, n values each
  float* ref;                // power of two that the sum and E are relative to, as an exponent; -inf: nothing summed yet
  float* sum;                // sum over the classes seen so far, the target left out, of 2^(s log2 e - ref)
  float* shift;              // 2^(ref before the last piece - ref)
  float* target;             // the target's logit times log2 e
  float* wrong;              // 1 - p[target]; 0 for rows that do not count
  float* lse2;               // log2 of the sum over all classes
};
struct LossPiece {           // the classes v0 .. v0 + classes - 1 of a call
  int64_t n, v0, classes, vocab;
  const int64_t* targets;
};
int launch_loss_begin(const LossRows& r, int64_t n, hipStream_t st);
// E[i][j] = 2^(s_ij log2 e - part_ref), 0 for the target and beyond the piece, as planes (hi NULL: not wanted), and per tile of 256
// classes and row: part_ref, part_sum.
int launch_loss_logits(const Planes& w, const Planes& x, int64_t depth, const LossPiece& p, const LossRows& r, float* part_ref,
                       float* part_sum, uint16_t* e_hi, uint16_t* e_lo, int64_t e_pitch, hipStream_t st);
// Joins the tiles' sums with the row's, brings E to one power of two per row.
int launch_loss_join(const LossPiece& p, const LossRows& r, const float* part_ref, const float* part_sum, uint16_t* e_hi,
                     uint16_t* e_lo, int64_t e_pitch, hipStream_t st);
// acc (n x d) = acc shift + E W; first: acc = E W.  part: splits x n x d floats.
int loss_accumulate_splits(int64_t n, int64_t d, int64_t depth, int planes);
int launch_loss_accumulate(const Planes& e, const Planes& wt, int64_t depth, int64_t n, int64_t d, const float* shift, bool first,
                           float* acc, float* part, size_t part_floats, hipStream_t st);
// Row losses, log-sum-exps, their total and what the gradients need (r.wrong, r.lse2).
int launch_loss_rows(const LossRows& r, const int64_t* targets, int64_t n, int64_t vocab, bool mean, float* loss, float* row_loss,
                     float* lse, float* factor, hipStream_t st);
int launch_loss_dx(const LossRows& r, const int64_t* targets, int64_t n, int64_t d, int64_t vocab, const float* acc, const void* W,
                   int64_t ldw, int dtype, const float* factor, void* dX, hipStream_t st);
// Gt[j][i] = factor (p_ij - [j = target_i]) as planes of `classes` rows, zero for rows that do not count and up to up_to(n, 64).
int launch_loss_gradient(const Planes& w, const Planes& x, int64_t depth, const LossPiece& p, const LossRows& r,
                         const float* factor, uint16_t* g_hi, uint16_t* g_lo, int64_t g_pitch, hipStream_t st);
// out (rows x cols, contiguous, of type dtype) = A B^T + A2 B2^T (depth2 == 0: without).  part: splits x rows x cols floats.
int plain_product_splits(int64_t rows, int64_t cols, int64_t depth, int planes);
int launch_plain_product(const Planes& a, const Planes& b, int64_t depth, const Planes& a2, const Planes& b2, int64_t depth2,
                         int64_t rows, int64_t cols, int dtype, void* out, float* part, size_t part_floats, hipStream_t st);

// ---- adapter products (adapter_kernels.hip) ---------------------------------------------------------------
constexpr int ADAPTER_MAX_RANK = 128;
// part[z] (m x r32) = drop(A) B over range z of the reduction: A m x K of type dtype, contiguous, K a multiple of 8, B as planes of
// r32 rows x K (pitch), zero rows beyond the rank.  d: NULL without dropout (its factor is left to launch_thin_finish).
int thin_project_splits(int64_t m, int64_t K);
int launch_thin_project(const void* A, int dtype, int64_t m, int64_t K, const Planes& b, int r32, const DropoutMask* d, float* part,
                        hipStream_t st);
// T = scale * sum of the partial results: fp32 m x rank (NULL: not wanted), planes m x r32 and planes of its transpose r32 x
// up_to(m, 64) (hi NULL: not wanted).  splits == 0: T is given (m x rank in `part`).
int launch_thin_finish(const float* part, int splits, int64_t m, int rank, int r32, float scale, float* T, uint16_t* hi,
                       uint16_t* lo, uint16_t* t_hi, uint16_t* t_lo, int64_t t_pitch, hipStream_t st);
// out = scale * drop(A)^T B: A m x K as above, B^T as planes of r32 rows x up_to(m, 64).  out: K x rank, or rank x K (transposed).
int thin_gram_splits(int64_t m, int64_t K);
int launch_thin_gram(const void* A, int dtype, int64_t m, int64_t K, const Planes& bt, int rank, int r32, const DropoutMask* d,
                     float scale, bool transposed, float* part, float* out, hipStream_t st);
// The stored weights (K x N, row-major) as bf16 planes with rows of `pitch` elements, zero from N to up_to(N, 32); lo may be NULL.
int launch_weight_rows(const MvWeights& q, int64_t K, int64_t N, uint16_t* hi, uint16_t* lo, int64_t pitch, hipStream_t st);
// dX (m x d, of type dtype) = dY Q^T + mask .* (U L1^T) from planes: Q d x k, dY m x k, L1 d x r32, U m x r32 (mask factor not in).
int adapter_dx_splits(int64_t m, int64_t d, int64_t k, int planes);
int launch_adapter_dx(const Planes& q, const Planes& dy, int64_t depth, const Planes& l1, const Planes& u, int r32, int64_t m,
                      int64_t d, const DropoutMask& mask, int dtype, void* dX, float* part, size_t part_floats, hipStream_t st);

}  // namespace lq
