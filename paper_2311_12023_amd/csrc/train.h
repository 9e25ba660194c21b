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

// Checks p (0 <= p <= 1) and fills the mask's parameters.
int dropout_mask(double p, uint64_t seed, uint64_t offset, DropoutMask* d);
int launch_dropout(const void* x, int64_t n, int dtype, const DropoutMask& d, void* y, hipStream_t st);

// ---- the product of planes that the operators share (segment_gemm.h) ---------------------------------
constexpr int SEG_T = 256, SEG_SLOTS = 5, SEG_THREADS = 512;
constexpr uint32_t SEG_TILE = SEG_T * 64, SEG_STAGE = 2 * SEG_TILE;           // bytes
constexpr size_t SEG_LDS = (size_t)SEG_SLOTS * SEG_STAGE;                     // all of a CU's

struct Segment {
  const uint16_t* A; const uint16_t* B;
  int64_t pitch_a, pitch_b;      // elements from row to row, multiples of 8; the planes begin on 16 bytes
  int end;                       // pairs of 32-deep steps of this segment and those before it
};
struct SegArgs {
  Segment seg[6];
  int64_t rows_a, rows_b;
  int64_t depth_a;               // reduction indices that A has, where it is read turned
  int tiles_m, tiles_n, splits, pairs;
};

// The planes of an operand, the leading one first; those that are not there are NULL.  One: bf16 as it is.  Two: fp16 hi + lo of a
// value times a power of two (22 bits).  Three: bf16 (24 bits).
struct Planes {
  const uint16_t* p[3];
  int64_t pitch;
};
// The segments of A B^T over `depth` (a multiple of 64) reduction indices: products of planes whose places add up to less than
// the larger number of planes.
inline void add_segments(SegArgs& s, int* count, const Planes& a, const Planes& b, int64_t depth) {
  const int na = a.p[2] ? 3 : a.p[1] ? 2 : 1, nb = b.p[2] ? 3 : b.p[1] ? 2 : 1, most = na > nb ? na : nb;
  for (int i = 0; i < na; ++i)
    for (int j = 0; j < nb && i + j < most; ++j) {
      s.pairs += (int)(depth / 64);
      s.seg[(*count)++] = Segment{a.p[i], b.p[j], a.pitch, b.pitch, s.pairs};
    }
}
inline int64_t seg_tiles(int64_t rows, int64_t cols) { return ((rows + SEG_T - 1) / SEG_T) * ((cols + SEG_T - 1) / SEG_T); }
// Ranges that the reduction of a product with few tiles is cut into: the parts fill the chip, each keeps eight pairs of steps.
inline int seg_splits(int64_t tiles, int64_t pairs, int most) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({256 / std::max<int64_t>(1, tiles), pairs / 8, (int64_t)most}));
}
inline int seg_shape(SegArgs& g, int64_t rows, int64_t cols, int splits) {
  if (rows < 1 || cols < 1 || seg_tiles(rows, cols) * splits >= (1ll << 30)) return LQ_ERR_SHAPE;
  g.rows_a = rows; g.rows_b = cols; g.splits = splits;
  g.tiles_m = (int)((rows + SEG_T - 1) / SEG_T); g.tiles_n = (int)((cols + SEG_T - 1) / SEG_T);
  return LQ_OK;
}
inline unsigned seg_grid(const SegArgs& a) { return (unsigned)(((int64_t)a.tiles_m * a.tiles_n * a.splits + 7) / 8 * 8); }

// ---- planes of an operand (train_planes_kernels.hip) --------------------------------------------------
// What a plane holds.  BF16: one plane, the source's own (a bf16 source) or its rounding.  BF16_3: three planes.  HALF_2: two fp16
// planes of the value times 2^s, where s brings the largest finite magnitude below 2^14: that of the whole operand, whose bits
// `top` holds (launch_top_magnitude), or, with row_inv, of each row by itself, 2^-s of which goes there.
enum PlaneKind { PLANE_BF16, PLANE_BF16_3, PLANE_HALF_2 };
struct PlaneSource {
  const void* src; int dtype; int64_t ld, rows, cols;      // rows x cols values, ld elements from row to row
  const uint32_t* top;                                     // HALF_2
};
struct PlaneTarget {
  uint16_t* p[3]; int64_t pitch;                           // pitch: a multiple of 64
  int64_t rows;                                            // rows written, zero beyond the source's
};
inline Planes planes_of(const PlaneTarget& t) { return {{t.p[0], t.p[1], t.p[2]}, t.pitch}; }
// Planes with the source's rows, zero from cols up to up_to(cols, 64).
int launch_row_planes(const PlaneSource& s, PlaneKind kind, const PlaneTarget& t, float* row_inv, hipStream_t st);
// Planes (BF16 or HALF_2) of the transpose: t.rows rows (zero from `cols` on), zero from `rows` up to up_to(rows, 64).  keep: one int64 per source
// row; rows whose value lies outside [0, keep_below) are taken as zero, whatever they hold (NULL: all are taken).
int launch_column_planes(const PlaneSource& s, PlaneKind kind, const PlaneTarget& t, const int64_t* keep, int64_t keep_below,
                         hipStream_t st);
// *top = bits of the largest finite magnitude (keep as above); *top is zero before.
int launch_top_magnitude(const void* src, int64_t ld, int64_t rows, int64_t cols, const int64_t* keep, int64_t keep_below,
                         uint32_t* top, hipStream_t st);                      // fp32
// Several such passes over small operands in one launch.
constexpr int TOP_WORDS = 64;
struct PrepareJobs {
  struct Job {
    int what; int wgs;
    PlaneSource s; PlaneTarget t; float* row_inv; uint32_t* tops; int tiles_r;
  };
  Job job[5];
  int count;
  int rows3(const PlaneSource& s, const PlaneTarget& t);             // launch_row_planes, PLANE_BF16_3
  int columns3(const PlaneSource& s, const PlaneTarget& t);          // three planes of the transpose
  int rows_scaled(const PlaneSource& s, const PlaneTarget& t, float* row_inv);
  int rows(const PlaneSource& s, const PlaneTarget& t);              // bf16 into a padded plane
  int tops(const float* v, int64_t n, uint32_t* words);              // TOP_WORDS words, the largest of which is v's
  int launch(hipStream_t st) const;
};

// ---- softmax cross entropy (loss_kernels.hip) -----------------------------------------------------------
struct LossRows {            // per-row state, n values each
  float* ref;                // power of two that the sum and E are relative to, as an exponent; -inf: nothing summed yet
  float* sum;                // sum over the classes seen so far, the target left out, of 2^(s log2 e - ref)
  float* shift;              // 2^(ref before the last piece - ref)
  float* target;             // the target's logit times log2 e
  float* wrong;              // 1 - p[target]; 0 for rows that do not count
  float* lse2;               // log2 of the sum over all classes
};
struct LossScales {          // fp32 operands: NULL for bf16
  const float* x_inv;        // per row of X
  const uint32_t* w_top;     // of W
  const uint32_t* xt_top;    // of the rows of X that count (for dW)
};
struct LossPiece {           // the classes v0 .. v0 + classes - 1 of a call
  int64_t n, v0, classes, vocab;
  const int64_t* targets;
};
int launch_zero_words(uint32_t* p, int count, hipStream_t st);
// E[i][j] = 2^(s_ij log2 e - part_ref), 0 for the target and beyond the piece, as planes (NULL: not wanted), and per tile of 256
// classes and row: part_ref, part_sum.  bf16: e[1], what the rounding of E left out, may be NULL.  fp32: E is stored times
// 2^LOSS_E_SHIFT and may reach 2^LOSS_E_ROOM; e32 (the whole vocabulary): in fp32 instead of planes.
constexpr int LOSS_E_SHIFT = 13, LOSS_E_ROOM = 2;
int launch_loss_logits(const Planes& w, const Planes& x, int64_t depth, const LossPiece& p, const LossRows& r, const LossScales& s,
                       float* part_ref, float* part_sum, uint16_t* const e[2], float* e32, int64_t e_pitch, float* part,
                       size_t part_floats, hipStream_t st);
size_t loss_tail_floats(int64_t n, int64_t classes, int64_t depth, bool half);      // of part: the piece's last classes, in ranges
// X and W for the logits of the targets (W NULL: the tiles have found them).
struct LossOperands { const void* X; int64_t ldx; const void* W; int64_t ldw, d; int dtype, vec; };
// Joins the sums of tiles of `tile` classes with the row's; with e (tiles of SEG_T classes) brings E to one power of two per row.
// told: r.ref has been set by launch_loss_reference.
int launch_loss_join(const LossPiece& p, const LossRows& r, bool half, bool told, const float* part_ref, const float* part_sum, int tile,
                     uint16_t* const e[2], int64_t e_pitch, const LossOperands& o, hipStream_t st);
// Joins and finishes up to 16 rows in one launch (the whole vocabulary as one piece, no E to bring to another power of two).
int launch_loss_join_rows(const LossPiece& p, const LossRows& r, const float* part_ref, const float* part_sum, int tile, bool mean,
                          const LossOperands& o, float* loss, float* row_loss, float* lse, float* factors, hipStream_t st);
// acc (n x d) = acc shift + E W; first: acc = E W.  W: `classes` rows of at least up_to(d, 8) elements; E is zero from there to
// up_to(classes, 64).  part: splits x n x d floats.
int loss_accumulate_splits(int64_t n, int64_t d, int64_t depth, bool half);
int launch_loss_accumulate(const Planes& e, const Planes& w, int64_t classes, int64_t n, int64_t d, const float* shift, bool first,
                           float* acc, float* part, size_t part_floats, hipStream_t st);
// What rows of X are relative to before a logit is known (bf16): the power of two of their target's logit, of another class's where
// they have none.  With 64 to spare on either side that serves E (see loss_logits_kernel).
int launch_loss_reference(const void* X, int64_t ldx, const void* W, int64_t ldw, int64_t d, const LossPiece& p, const LossRows& r,
                          hipStream_t st);
// Row losses, log-sum-exps, their total and what the gradients need: r.wrong, r.lse2, factors[0] = the gradient's factor,
// factors[1] = that of dW's product.
int launch_loss_rows(const LossRows& r, const LossScales& s, const int64_t* targets, int64_t n, int64_t vocab, bool mean, float* loss,
                     float* row_loss, float* lse, float* factors, hipStream_t st);
int launch_loss_dx(const LossRows& r, const LossScales& s, const int64_t* targets, int64_t n, int64_t d, int64_t vocab,
                   const float* acc, const void* W, int64_t ldw, int dtype, const float* factors, void* dX, hipStream_t st);
// Gt[j][i] = p_ij - [j = target_i], `classes` rows of g_pitch, zero for rows that do not count and up to up_to(n, 64): bf16, or fp32
// where the operands are.
int launch_loss_gradient(const Planes& w, const Planes& x, int64_t depth, const LossPiece& p, const LossRows& r, const LossScales& s,
                         void* g, int64_t g_pitch, hipStream_t st);
// The same from E where one piece is the whole vocabulary, as planes.  bf16: of both of E's planes.  fp32 (e32, relative to part_ref):
// Gt's rows times a power of two each, whose inverse goes to class_inv (tops: loss_class_ranges(n) x classes floats), and E's
// planes relative to its rows' powers of two (e[0] NULL: not wanted).
int loss_class_ranges(int64_t n);
int launch_loss_gradient_from_e(const LossPiece& p, const LossRows& r, const float* part_ref, const float* e32,
                                uint16_t* const e[2], int64_t e_pitch, uint16_t* const g[2], int64_t g_pitch, float* tops,
                                float* class_inv, hipStream_t st);
// dW's rows: out (rows x cols, contiguous, of type dtype) = *factor A B^T, fp32: times class_inv per row.  part: splits x rows x cols floats.
int loss_dw_splits(int64_t rows, int64_t cols, int64_t depth, bool half);
int launch_loss_dw(const Planes& g, const Planes& xt, int64_t depth, int64_t rows, int64_t cols, const float* factor,
                   const float* class_inv, int dtype, void* out, float* part, size_t part_floats, hipStream_t st);

// ---- the same for few rows (loss_few_kernels.hip) ---------------------------------------------------------
// Up to LOSS_FEW rows the loss is bound by reading W: it is then read where it is, once for the logits and once for dX, the whole
// vocabulary as one piece (which sizes: few_by_size in lq_api_train.cpp).  d = 4096, 32000 classes, bf16, 16 / 64 / 128 rows: 106 / 117 /
// 171 us, by the products of many rows 158 / 169 / 184; d = 1024, 50265 classes, fp32: 114 / 147 / 295 for 286 / 295 / 310.  Planes of X
// (one for bf16, three for fp32) and E have few_rows(n) rows.  Tiles are LOSS_FEW_TILE classes; E is relative to its tile's power of two.
constexpr int64_t LOSS_FEW = 128, LOSS_FEW_TILE = 64;
inline int64_t few_rows(int64_t n) { return n <= 16 ? 16 : n <= 32 ? 32 : n <= 64 ? 64 : 128; }
int launch_few_logits(const void* W, int64_t ldw, int dtype, int64_t d, const Planes& x, const LossPiece& p, float* part_ref,
                      float* part_sum, uint16_t* const e[3], int64_t e_pitch, hipStream_t st);
// dX from E and W once r.wrong is there.  part: few_dx_splits(vocab, d) x d x few_rows(n) floats.
int few_dx_splits(int64_t vocab, int64_t d);
int launch_few_dx(const void* W, int64_t ldw, int dtype, int64_t d, const Planes& e, const LossPiece& p, const LossRows& r,
                  const float* part_ref, const float* factors, float* part, void* dX, hipStream_t st);

// ---- adapter products (adapter_kernels.hip, thin_kernels.hip) ---------------------------------------------
constexpr int ADAPTER_MAX_RANK = 128;
// part[z] (m x r32) = drop(A) B over range z of the reduction: A m x K of type dtype, contiguous, K a multiple of 8, B as three
// bf16 planes of r32 rows x up_to(K, 64).  The mask's factor is left to launch_finish.
int thin_project_splits(int64_t m, int64_t K);
int launch_thin_project(const void* A, int dtype, int64_t m, int64_t K, const Planes& b, int r32, const DropoutMask& d, float* part,
                        hipStream_t st);
// T = scale * sum of the partial results: fp32 m x rank (NULL: not wanted), three planes m x up_to(r32, 64) and three of the
// transpose, r32 x up_to(m, 64) (p[0] NULL: not wanted).
struct ThinFinish {
  const float* part; int splits; int64_t m; int rank, r32; float scale;
  float* T; PlaneTarget rows, cols;
};
// The stored weights (K x N, row-major) as planes, row by row (zero from N to up_to(N, 64)) or transposed (N rows, zero from K to
// up_to(K, 64)): one bf16 plane, or two fp16 planes times the power of two that the largest of the TOP_WORDS words at `top` (of the
// group scales v) gives.
struct WeightPlanes {
  MvWeights q; int64_t K, N; bool transposed;
  const uint32_t* top; uint16_t *hi, *lo; int64_t pitch;
};
// dL2 (rank x k) = T^T dY and dL1 (d x rank) = drop(X)^T U; T^T and U^T as three planes of r32 rows x up_to(m, 64).
// part: thin_gram_splits(m, k, d) x (k + d) x r32 floats; with more than one range the results are left in there, and *sum makes
// them of it.
struct ThinGramSum { const float* part[2]; int splits; int64_t K[2]; int rank, r32; float scale; float* out[2]; };
int thin_gram_splits(int64_t m, int64_t k, int64_t d);
int launch_thin_grams(const void* dY, int64_t k, const Planes& tt, float* dL2, const void* X, int64_t d, const Planes& ut,
                      const DropoutMask& mask, float* dL1, int dtype, int64_t m, int rank, int r32, float* part, ThinGramSum* sum,
                      hipStream_t st);
// A pass over partial results, and the weights' planes beside it in the same launch (adapter_kernels.hip); weights NULL: not wanted.
int launch_finish(const ThinFinish& f, const WeightPlanes* weights, hipStream_t st);
int launch_gram_sum(const ThinGramSum& g, const WeightPlanes* weights, hipStream_t st);
// out (tokens x features, of type dtype) = B A^T + mask .* (B2 A2^T): A the weights (features x depth), B the activations
// (tokens x depth), A2 and B2 the low-rank part (depth2; three planes each).  mask: NULL for none.  fp32: b_inv, a_top scale A B.
struct AdapterScales { const float* b_inv; const uint32_t* a_top; };
size_t adapter_part_floats(int64_t features, int64_t tokens, int64_t depth, int64_t depth2, int dtype);
int launch_adapter_product(const Planes& a, const Planes& b, int64_t depth, const Planes& a2, const Planes& b2, int64_t depth2,
                           const AdapterScales& s, int64_t features, int64_t tokens, const DropoutMask* mask, int dtype, void* out,
                           float* part, size_t part_floats, hipStream_t st);

}  // namespace lq
