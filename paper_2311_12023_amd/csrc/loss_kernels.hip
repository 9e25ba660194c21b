// Softmax cross entropy over a large vocabulary without an array of logits, with its gradients.
//
//   s_ij = <x_i, w_j>,  loss_i = log sum_j e^s_ij - s_it,  dX_i = g (sum_j p_ij w_j - w_t),  dW_j = sum_i g (p_ij - [j = t_i]) x_i
//
// The vocabulary is walked in pieces.  A piece's logits come out of the matrix pipe tile by tile and leave the registers as
// E_ij = 2^(s_ij log2 e - ref) in bf16 with their sums in fp32; E W, added up over the pieces, is the gradient of X up to a factor
// per row that is known at the end.  So the loss and dX take one pass, 4 n d V operations, where a pass for the sums and one
// for the gradient would take six.  References are whole powers of two: a row's E, its sum and its part of dX move from one
// reference to a larger one without a rounding.  The target stays out of E: with S the sum over the other classes and z the
// logit's distance from log S, loss = log(1 + e^-z) and dX_i = g (1 - p_t) (E W / S - w_t), 1 - p_t = 1 / (1 + e^z), which
// are as exact for a row that is certain of its target (p_t = 1 - 1e-9) as for any other; 1 - p_t from p_t would be lost there.
// dW needs p itself, so it takes a second pass over the logits.
#include "mfma_device.h"
#include "profiler.h"
#include "segment_gemm.h"
#include "train.h"

namespace lq {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__global__ __launch_bounds__(256) void loss_begin_kernel(LossRows r, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  r.ref[i] = -__builtin_inff();
  r.sum[i] = 0.0f;
  r.target[i] = 0.0f;
}

int launch_loss_begin(const LossRows& r, int64_t n, hipStream_t st) {
  prof::Scope ps(prof::LOSS_ROWS, st, (double)n * 12.0);
  hipLaunchKernelGGL(loss_begin_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, r, n);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// Logits of a piece.  Classes are the tile's rows and tokens its columns: a lane then holds 64 classes of one token, and the
// maximum and the sum over the tile are reductions inside lanes, one exchange between the halves of a wavefront and one through
// LDS between two wavefronts.
struct LogitsArgs {
  SegArgs g;
  LossPiece p;
  const float* ref; float* target;
  float* part_ref; float* part_sum;
  uint16_t* e_hi; uint16_t* e_lo; int64_t e_pitch;
};

__global__ __launch_bounds__(SEG_THREADS) void loss_logits_kernel(LogitsArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const SegTile t = seg_tile(a.g);
  if (!t.live) return;
  floatx16 acc[4][2];
  seg_clear(acc);
  const int steps = a.g.seg[2].end;
  seg_products(a.g, t, 0, steps, seg_lds, acc);
  __syncthreads();                                   // the LDS now holds exchanges
  float* s_max = reinterpret_cast<float*>(seg_lds);  // [wm][column of the tile]
  float* s_sum = s_max + 2 * SEG_T;
  const int64_t class0 = (int64_t)t.tm * SEG_T + 128 * t.wm;                 // inside the piece
  const int64_t left = a.p.classes - class0;
  const int lim = (int)(left < 0 ? 0 : left < 128 ? left : 128);
  float base[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int col = 64 * t.wn + 32 * j + t.ln;
    const int64_t token = (int64_t)t.tn * SEG_T + col;
    const bool live = token < a.p.n;
    const int64_t target = live ? a.p.targets[token] - a.p.v0 - class0 : -1;
    const int at = target >= 0 && target < lim ? (int)target : -1;
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int row = 32 * i + 8 * (e >> 2) + 4 * t.lh + (e & 3);
        float x = acc[i][j][e] * LOG2E;
        if (row == at) { a.target[token] = x; x = -__builtin_inff(); }
        if (row >= lim) x = -__builtin_inff();
        acc[i][j][e] = x;
        top = fmaxf(top, x);
      }
    top = fmaxf(top, __shfl_xor(top, 32));
    s_max[t.wm * SEG_T + col] = top;
    base[j] = live ? a.ref[token] : 0.0f;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int col = 64 * t.wn + 32 * j + t.ln;
    const int64_t token = (int64_t)t.tn * SEG_T + col;
    const float ref = fmaxf(base[j], ceilf(fmaxf(s_max[col], s_max[SEG_T + col])));
    base[j] = ref;
    const float from = ref == -__builtin_inff() ? 0.0f : ref;                // nothing but the target so far
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        acc[i][j][e] = __builtin_amdgcn_exp2f(acc[i][j][e] - from);
        sum += acc[i][j][e];
      }
    sum += __shfl_xor(sum, 32);
    s_sum[t.wm * SEG_T + col] = sum;
    if (a.e_hi && token < a.p.n) {
      // E in bf16: 2^-9 of each term of a sum that ends up in the type of X, and two planes where that is fp32
      uint16_t* out = a.e_hi + token * a.e_pitch + class0 + 4 * t.lh;
      uint16_t* low = a.e_lo + token * a.e_pitch + class0 + 4 * t.lh;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          bf16x2 h0, l0, h1, l1;
          split_bf16(floatx2{acc[i][j][4 * q], acc[i][j][4 * q + 1]}, h0, l0);
          split_bf16(floatx2{acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]}, h1, l1);
          *reinterpret_cast<bf16x4*>(out + 32 * i + 8 * q) = bf16x4{h0[0], h0[1], h1[0], h1[1]};
          if (a.e_lo) *reinterpret_cast<bf16x4*>(low + 32 * i + 8 * q) = bf16x4{l0[0], l0[1], l1[0], l1[1]};
        }
    }
  }
  __syncthreads();
  if (t.wm == 0 && t.lh == 0) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int col = 64 * t.wn + 32 * j + t.ln;
      const int64_t token = (int64_t)t.tn * SEG_T + col;
      if (token < a.p.n) {
        a.part_ref[(int64_t)t.tm * a.p.n + token] = base[j];
        a.part_sum[(int64_t)t.tm * a.p.n + token] = s_sum[col] + s_sum[SEG_T + col];
      }
    }
  }
}

static void fill_segments(SegArgs& g, const Planes& a, const Planes& b, int64_t depth) {
  int count = 0, end = add_segments(g, &count, 0, a, b, depth);
  for (; count < 6; ++count) { g.seg[count] = g.seg[0]; g.seg[count].end = end; }
}

int launch_loss_logits(const Planes& w, const Planes& x, int64_t depth, const LossPiece& p, const LossRows& r, float* part_ref,
                       float* part_sum, uint16_t* e_hi, uint16_t* e_lo, int64_t e_pitch, hipStream_t st) {
  if (depth < 32 || depth % 32 || p.n < 1 || p.classes < 1) return LQ_ERR_SHAPE;
  LogitsArgs a{};
  fill_segments(a.g, w, x, depth);
  a.g.rows_a = p.classes; a.g.rows_b = p.n;
  a.g.tiles_m = (int)((p.classes + SEG_T - 1) / SEG_T); a.g.tiles_n = (int)((p.n + SEG_T - 1) / SEG_T); a.g.splits = 1;
  a.p = p; a.ref = r.ref; a.target = r.target; a.part_ref = part_ref; a.part_sum = part_sum;
  a.e_hi = e_hi; a.e_lo = e_lo; a.e_pitch = e_pitch;
  static LdsLimit limit;
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(loss_logits_kernel), SEG_LDS));
  prof::Scope ps(prof::LOSS_LOGITS, st, 2.0 * p.n * p.classes * depth);
  hipLaunchKernelGGL(loss_logits_kernel, dim3(seg_grid(a.g)), dim3(SEG_THREADS), SEG_LDS, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// A wavefront joins the tiles' sums of one row.  Tiles whose E lies at a smaller power of two than the row's new one are
// multiplied down, which in bf16 is exact (what leaves the range is below 2^-126 of the largest term).
struct JoinArgs {
  LossPiece p; LossRows r;
  const float* part_ref; const float* part_sum; int tiles;
  uint16_t* e_hi; uint16_t* e_lo; int64_t e_pitch;
};

__device__ __forceinline__ void scale_run(uint16_t* at, float f) {
  bf16x4 v = *reinterpret_cast<const bf16x4*>(at);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = (__bf16)((float)v[k] * f);
  *reinterpret_cast<bf16x4*>(at) = v;
}

__global__ __launch_bounds__(256) void loss_join_kernel(JoinArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= a.p.n) return;
  const float old = a.r.ref[row];
  float ref = old;
  for (int t = lane; t < a.tiles; t += 64) ref = fmaxf(ref, a.part_ref[(int64_t)t * a.p.n + row]);
#pragma unroll
  for (int o = 32; o; o >>= 1) ref = fmaxf(ref, __shfl_xor(ref, o));
  const float from = ref == -__builtin_inff() ? 0.0f : ref;
  float sum = 0.0f;
  for (int t = lane; t < a.tiles; t += 64)
    sum += a.part_sum[(int64_t)t * a.p.n + row] * __builtin_amdgcn_exp2f(a.part_ref[(int64_t)t * a.p.n + row] - from);
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) {
    const float shift = __builtin_amdgcn_exp2f(old - from);
    a.r.sum[row] = a.r.sum[row] * shift + sum;
    a.r.shift[row] = shift;
    a.r.ref[row] = ref;
  }
  if (!a.e_hi) return;
  for (int t = 0; t < a.tiles; ++t) {
    const float mine = a.part_ref[(int64_t)t * a.p.n + row];
    if (mine == ref) continue;
    const float f = __builtin_amdgcn_exp2f(mine - from);
    const int64_t at = row * a.e_pitch + (int64_t)t * SEG_T + 4 * lane;
    scale_run(a.e_hi + at, f);
    if (a.e_lo) scale_run(a.e_lo + at, f);
  }
}

int launch_loss_join(const LossPiece& p, const LossRows& r, const float* part_ref, const float* part_sum, uint16_t* e_hi,
                     uint16_t* e_lo, int64_t e_pitch, hipStream_t st) {
  JoinArgs a{p, r, part_ref, part_sum, (int)((p.classes + SEG_T - 1) / SEG_T), e_hi, e_lo, e_pitch};
  prof::Scope ps(prof::LOSS_ROWS, st, (double)p.n * a.tiles * 8.0);
  hipLaunchKernelGGL(loss_join_kernel, dim3((unsigned)((p.n + 3) / 4)), dim3(256), 0, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// acc = acc shift + E W: tokens are the tile's rows, features its columns.
struct AccumulateArgs {
  SegArgs g;
  int64_t n, d;
  const float* shift; int first;
  float* acc; float* part;
};

__global__ __launch_bounds__(SEG_THREADS) void loss_accumulate_kernel(AccumulateArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const SegTile t = seg_tile(a.g);
  if (!t.live) return;
  floatx16 acc[4][2];
  seg_clear(acc);
  const int steps = a.g.seg[2].end;
  seg_products(a.g, t, (int)((int64_t)steps * t.split / a.g.splits), (int)((int64_t)steps * (t.split + 1) / a.g.splits), seg_lds, acc);
  float* part = a.part + (size_t)t.split * (size_t)a.n * (size_t)a.d;
  seg_each(t, [&](int i, int j, int e, int64_t row, int64_t col) {
    if (row >= a.n || col >= a.d) return;
    if (a.g.splits > 1) part[row * a.d + col] = acc[i][j][e];
    else a.acc[row * a.d + col] = a.first ? acc[i][j][e] : fmaf(a.acc[row * a.d + col], a.shift[row], acc[i][j][e]);
  });
}

__global__ __launch_bounds__(256) void loss_accumulate_sum_kernel(const float* __restrict__ part, int splits, int64_t n, int64_t d,
                                                                  const float* __restrict__ shift, int first, float* __restrict__ acc) {
  const int64_t total = n * d;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    float v = first ? 0.0f : acc[i] * shift[i / d];
    for (int s = 0; s < splits; ++s) v += part[s * total + i];
    acc[i] = v;
  }
}

int loss_accumulate_splits(int64_t n, int64_t d, int64_t depth, int planes) {
  return seg_splits(((n + SEG_T - 1) / SEG_T) * ((d + SEG_T - 1) / SEG_T), (int)(depth / 32) * (planes == 2 ? 3 : 1), 64);
}

int launch_loss_accumulate(const Planes& e, const Planes& wt, int64_t depth, int64_t n, int64_t d, const float* shift, bool first,
                           float* acc, float* part, size_t part_floats, hipStream_t st) {
  if (depth < 32 || depth % 32) return LQ_ERR_SHAPE;
  AccumulateArgs a{};
  fill_segments(a.g, e, wt, depth);
  a.g.rows_a = n; a.g.rows_b = d;
  a.g.tiles_m = (int)((n + SEG_T - 1) / SEG_T); a.g.tiles_n = (int)((d + SEG_T - 1) / SEG_T);
  a.g.splits = loss_accumulate_splits(n, d, depth, e.lo ? 2 : 1);
  if (a.g.splits > 1 && part_floats < (size_t)a.g.splits * (size_t)n * (size_t)d) return LQ_ERR_WORKSPACE;
  a.n = n; a.d = d; a.shift = shift; a.first = first; a.acc = acc; a.part = part;
  static LdsLimit limit;
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(loss_accumulate_kernel), SEG_LDS));
  {
    prof::Scope ps(prof::LOSS_ACCUMULATE, st, 2.0 * n * d * depth);
    hipLaunchKernelGGL(loss_accumulate_kernel, dim3(seg_grid(a.g)), dim3(SEG_THREADS), SEG_LDS, st, a);
    LQ_HIP_TRY(hipGetLastError());
  }
  if (a.g.splits > 1) {
    prof::Scope ps(prof::LOSS_ROWS, st, (double)n * d * 4.0 * (a.g.splits + 2));
    const int64_t wgs = std::min<int64_t>((n * d + 255) / 256, 8192);
    hipLaunchKernelGGL(loss_accumulate_sum_kernel, dim3((unsigned)wgs), dim3(256), 0, st, part, a.g.splits, n, d, shift, (int)first, acc);
    LQ_HIP_TRY(hipGetLastError());
  }
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// One workgroup finishes the rows: a few bytes each, and the total is added up in 64 bits in a fixed order.
__global__ __launch_bounds__(1024) void loss_rows_kernel(LossRows r, const int64_t* __restrict__ targets, int64_t n, int64_t vocab,
                                                         int mean, float* loss, float* row_loss, float* lse, float* factor) {
  __shared__ double s_sum[1024];
  __shared__ unsigned long long s_count[1024];
  double sum = 0.0;
  unsigned long long count = 0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) {
    const bool counts = targets[i] >= 0 && targets[i] < vocab;
    const float others = r.ref[i] + log2f(r.sum[i]);        // log2 of the sum without the target; -inf: there is no other class
    float l = 0.0f, wrong = 0.0f, all = others;
    if (counts) {
      const float z = r.target[i] - others;
      l = fmaxf(-z, 0.0f) * LN2 + log1pf(exp2f(-fabsf(z)));
      if (z != z) l = z;
      wrong = 1.0f / (1.0f + exp2f(z));
      all = fmaxf(r.target[i], others) + log1pf(exp2f(-fabsf(z))) * LOG2E;
      if (z != z) all = z;
      sum += l;
      ++count;
    }
    row_loss[i] = l;
    if (lse) lse[i] = all * LN2;
    r.wrong[i] = wrong;
    r.lse2[i] = all;
  }
  s_sum[threadIdx.x] = sum;
  s_count[threadIdx.x] = count;
  __syncthreads();
  for (int o = 512; o; o >>= 1) {
    if ((int)threadIdx.x < o) { s_sum[threadIdx.x] += s_sum[threadIdx.x + o]; s_count[threadIdx.x] += s_count[threadIdx.x + o]; }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    const double f = mean ? 1.0 / (double)(s_count[0] ? s_count[0] : 1) : 1.0;      // no row counts: the mean is 0
    *loss = (float)(s_sum[0] * f);
    *factor = (float)f;
  }
}

int launch_loss_rows(const LossRows& r, const int64_t* targets, int64_t n, int64_t vocab, bool mean, float* loss, float* row_loss,
                     float* lse, float* factor, hipStream_t st) {
  prof::Scope ps(prof::LOSS_ROWS, st, (double)n * 36.0);
  hipLaunchKernelGGL(loss_rows_kernel, dim3(1), dim3(1024), 0, st, r, targets, n, vocab, (int)mean, loss, row_loss, lse, factor);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// dX_i = g (1 - p_t) (E W / S - w_t): one workgroup per row, its features in turn.
template <typename T>
__global__ __launch_bounds__(256) void loss_dx_kernel(LossRows r, const int64_t* __restrict__ targets, int64_t d, int64_t vocab,
                                                      const float* __restrict__ acc, const T* __restrict__ W, int64_t ldw,
                                                      const float* __restrict__ factor, T* __restrict__ dX) {
  const int64_t row = blockIdx.x, t = targets[row];
  const bool counts = t >= 0 && t < vocab;
  const float s = r.sum[row];
  const float inv = s == 0.0f ? 0.0f : 1.0f / s;             // no other class: acc is zero
  const float g = counts ? r.wrong[row] * *factor : 0.0f;
  for (int64_t c = threadIdx.x; c < d; c += 256)
    dX[row * d + c] = counts ? (T)(g * (acc[row * d + c] * inv - (float)W[t * ldw + c])) : (T)0.0f;
}

int launch_loss_dx(const LossRows& r, const int64_t* targets, int64_t n, int64_t d, int64_t vocab, const float* acc, const void* W,
                   int64_t ldw, int dtype, const float* factor, void* dX, hipStream_t st) {
  prof::Scope ps(prof::LOSS_ROWS, st, (double)n * d * (4.0 + 2.0 * type_bytes(dtype)));
  if (dtype == LQ_T_BF16)
    hipLaunchKernelGGL(loss_dx_kernel<__bf16>, dim3((unsigned)n), dim3(256), 0, st, r, targets, d, vocab, acc,
                       static_cast<const __bf16*>(W), ldw, factor, static_cast<__bf16*>(dX));
  else
    hipLaunchKernelGGL(loss_dx_kernel<float>, dim3((unsigned)n), dim3(256), 0, st, r, targets, d, vocab, acc,
                       static_cast<const float*>(W), ldw, factor, static_cast<float*>(dX));
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// The gradient of a piece's logits, transposed: the rows of Gt are classes, their tokens contiguous, as dW = Gt X reads them.
struct GradientArgs {
  SegArgs g;
  LossPiece p; LossRows r;
  const float* factor;
  uint16_t* hi; uint16_t* lo; int64_t pitch;
};

__global__ __launch_bounds__(SEG_THREADS) void loss_gradient_kernel(GradientArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const SegTile t = seg_tile(a.g);
  if (!t.live) return;
  floatx16 acc[4][2];
  seg_clear(acc);
  seg_products(a.g, t, 0, a.g.seg[2].end, seg_lds, acc);
  const int64_t cols = (a.p.n + 63) / 64 * 64;
  const float factor = *a.factor;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int64_t token = (int64_t)t.tn * SEG_T + 64 * t.wn + 32 * j + t.ln;
    if (token >= cols) continue;
    int64_t target = -1;
    float lse2 = 0.0f, wrong = 0.0f;
    if (token < a.p.n) { target = a.p.targets[token]; lse2 = a.r.lse2[token]; wrong = a.r.wrong[token] * factor; }
    const bool counts = target >= 0 && target < a.p.vocab;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int64_t row = (int64_t)t.tm * SEG_T + 128 * t.wm + 32 * i + 8 * (e >> 2) + 4 * t.lh + (e & 3);
        if (row >= a.p.classes) continue;
        float g = a.p.v0 + row == target ? -wrong : factor * __builtin_amdgcn_exp2f(acc[i][j][e] * LOG2E - lse2);
        g = counts ? g : 0.0f;
        const __bf16 h = (__bf16)g;
        a.hi[row * a.pitch + token] = __builtin_bit_cast(uint16_t, h);
        if (a.lo) a.lo[row * a.pitch + token] = __builtin_bit_cast(uint16_t, (__bf16)(g - (float)h));
      }
  }
}

int launch_loss_gradient(const Planes& w, const Planes& x, int64_t depth, const LossPiece& p, const LossRows& r,
                         const float* factor, uint16_t* g_hi, uint16_t* g_lo, int64_t g_pitch, hipStream_t st) {
  if (depth < 32 || depth % 32 || g_pitch < up_to(p.n, 64)) return LQ_ERR_SHAPE;
  GradientArgs a{};
  fill_segments(a.g, w, x, depth);
  a.g.rows_a = p.classes; a.g.rows_b = p.n;
  a.g.tiles_m = (int)((p.classes + SEG_T - 1) / SEG_T); a.g.tiles_n = (int)((p.n + SEG_T - 1) / SEG_T); a.g.splits = 1;
  a.p = p; a.r = r; a.factor = factor; a.hi = g_hi; a.lo = g_lo; a.pitch = g_pitch;
  static LdsLimit limit;
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(loss_gradient_kernel), SEG_LDS));
  prof::Scope ps(prof::LOSS_LOGITS, st, 2.0 * p.n * p.classes * depth);
  hipLaunchKernelGGL(loss_gradient_kernel, dim3(seg_grid(a.g)), dim3(SEG_THREADS), SEG_LDS, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
