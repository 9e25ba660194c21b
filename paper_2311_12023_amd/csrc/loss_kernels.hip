// Softmax cross entropy over a large vocabulary without an array of logits, with its gradients.
//
//   s_ij = <x_i, w_j>,  loss_i = log sum_j e^s_ij - s_it,  dX_i = g (sum_j p_ij w_j - w_t),  dW_j = sum_i g (p_ij - [j = t_i]) x_i
//
// The vocabulary is walked in pieces.  A piece's logits come out of the matrix pipe tile by tile and leave the registers as
// E_ij = 2^(s_ij log2 e - ref), in bf16 or as two fp16 planes, with their sums in fp32; E W, added up over the pieces, is the gradient
// of X up to a factor per row that is known at the end.  So the loss and dX take one pass, 4 n d V operations, where a pass for the sums and one
// for the gradient would take six.  References are whole powers of two: a row's E, its sum and its part of dX move from one
// reference to a larger one without a rounding.  The target stays out of E: with S the sum over the other classes and z the
// logit's distance from log S, loss = log(1 + e^-z) and dX_i = g (1 - p_t) (E W / S - w_t), 1 - p_t = 1 / (1 + e^z), which
// are as exact for a row that is certain of its target (p_t = 1 - 1e-9) as for any other; 1 - p_t from p_t would be lost there.
// dW needs p itself: it comes from E where one piece is the whole vocabulary, else from a second pass over the logits.
#include "half_planes_device.h"
#include "mfma_device.h"
#include "profiler.h"
#include "segment_gemm.h"
#include "train.h"

namespace lq {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__global__ void zero_words_kernel(uint32_t* p) { p[threadIdx.x] = 0; }
int launch_zero_words(uint32_t* p, int count, hipStream_t st) {
  hipLaunchKernelGGL(zero_words_kernel, dim3(1), dim3(count), 0, st, p);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// What a logit's accumulator is multiplied by to become s log2 e: the operands' powers of two go out with it.
__device__ __forceinline__ float logit_factor(const LossScales& s, int64_t token) {
  return s.x_inv ? LOG2E * s.x_inv[token] * power_of_two(-half_exponent(*s.w_top)) : LOG2E;
}

// Two blocks of four neighbours a lane as planes, eight neighbours a lane (bf16: lo may be NULL).
template <bool HALF>
__device__ __forceinline__ void split_four(floatx4 v, uintx2& hi, uintx2& lo) {
  if constexpr (HALF) {
    halfx4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) { const HalfPair p = split_half(v[e]); h[e] = p.hi; l[e] = p.lo; }
    hi = __builtin_bit_cast(uintx2, h);
    lo = __builtin_bit_cast(uintx2, l);
  } else {
    const bf16x4 h = __builtin_convertvector(v, bf16x4);
    hi = __builtin_bit_cast(uintx2, h);
    lo = __builtin_bit_cast(uintx2, __builtin_convertvector(v - __builtin_convertvector(h, floatx4), bf16x4));
  }
}
template <bool HALF>
__device__ __forceinline__ void store_blocks(uint16_t* hi, uint16_t* lo, floatx4 first, floatx4 second) {
  uintx2 h0, l0, h1, l1;
  split_four<HALF>(first, h0, l0);
  split_four<HALF>(second, h1, l1);
  *reinterpret_cast<uintx4*>(hi) = seg_pair_blocks(h0, h1);
  if (HALF || lo) *reinterpret_cast<uintx4*>(lo) = seg_pair_blocks(l0, l1);
}

// Four neighbours of a row of `width` floats, whose start is on 16 bytes where width is a multiple of four.
__device__ __forceinline__ void store_floats(float* at, floatx4 v, int64_t col, int64_t width) {
  if ((width & 3) == 0) { *reinterpret_cast<floatx4*>(at) = v; return; }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (col + e < width) at[e] = v[e];
}
__device__ __forceinline__ floatx4 load_floats(const float* at, int64_t col, int64_t width) {
  if ((width & 3) == 0) return *reinterpret_cast<const floatx4*>(at);
  floatx4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = col + e < width ? at[e] : 0.0f;
  return v;
}

// ------------------------------------------------------------------------------------------------
// Logits of a piece.  Classes are the tile's rows and tokens its columns: a lane then holds 32 classes of each of its tokens, and
// the maximum and the sum over the tile are reductions inside lanes, two exchanges between lanes and one through LDS between two
// wavefronts.  E is rounded to bf16, 2^-8 of each term of a sum that ends up in the type of X; two fp16 planes where that is fp32.
// Where dW comes from E, what the rounding left out is kept beside it, and E in fp32 instead of the planes: they end 2^-39 below the
// largest of 256 classes, and a class can be less probable than that beside it in every row.  2047 x 4096 by 32000 bf16: 560 us, 0.96
// PFLOP/s; 1000 x 1024 by 50265 fp32, three products: 400 us, 0.77, a quarter of it what becomes of the tiles.
struct LogitsArgs {
  SegArgs g;
  LossPiece p; LossScales s;
  const float* ref; float* target;
  float* part_ref; float* part_sum;
  uint16_t* e[2]; float* e32; int64_t e_pitch;
};

template <typename H>
__global__ __launch_bounds__(SEG_THREADS, 2) void loss_logits_kernel(LogitsArgs a) {
  constexpr bool HALF = !std::is_same<H, __bf16>::value;
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const SegTile t = seg_tile(a.g);
  if (!t.live) return;
  SegAcc acc;
  seg_clear(acc);
  seg_products<H>(a.g, t, 0, a.g.pairs, seg_lds, acc);
  __syncthreads();                                   // the LDS now holds exchanges
  float* s_max = reinterpret_cast<float*>(seg_lds);  // [wm][column of the tile]
  float* s_sum = s_max + 2 * SEG_T;
  const int64_t class0 = (int64_t)t.tm * SEG_T + 128 * t.wm;                 // inside the piece
  const int64_t left = a.p.classes - class0;
  const int lim = (int)(left < 0 ? 0 : left < 128 ? left : 128);
  float base[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int col = 64 * t.wn + 16 * j + t.l16;
    const int64_t token = (int64_t)t.tn * SEG_T + col;
    const bool live = token < a.p.n;
    const int64_t target = live ? a.p.targets[token] - a.p.v0 - class0 : -1;
    const int at = target >= 0 && target < lim ? (int)target : -1;
    const float f = live ? logit_factor(a.s, token) : 0.0f;
    float top = -__builtin_inff();
    if (__any(at >= 0) || lim < 128) {                // a target among these classes, or the vocabulary's end: seldom
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = 16 * i + 4 * t.kg + e;
          float x = acc[i][j][e] * f;
          if (row == at) { a.target[token] = x; x = -__builtin_inff(); }
          if (row >= lim) x = -__builtin_inff();
          acc[i][j][e] = x;
          top = fmaxf(top, x);
        }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        acc[i][j] *= f;
        top = fmaxf(top, fmaxf(fmaxf(acc[i][j][0], acc[i][j][1]), fmaxf(acc[i][j][2], acc[i][j][3])));
      }
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    s_max[t.wm * SEG_T + col] = top;
    base[j] = !live ? 0.0f : a.p.v0 == 0 && HALF ? -__builtin_inff() : a.ref[token];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int col = 64 * t.wn + 16 * j + t.l16;
    const int64_t token = (int64_t)t.tn * SEG_T + col;
    // the row's reference so far serves while E stays inside its type: no tile then has to be brought to another
    const float top = ceilf(fmaxf(s_max[col], s_max[SEG_T + col])), room = HALF ? (float)LOSS_E_ROOM : 64.0f;
    const float ref = top <= base[j] + room ? base[j] : top;
    base[j] = ref;
    // nothing but the target so far: any reference will do
    const float from = (ref == -__builtin_inff() ? 0.0f : ref) - (HALF ? (float)LOSS_E_SHIFT : 0.0f);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[i][j][e] = __builtin_amdgcn_exp2f(acc[i][j][e] - from);
        sum += acc[i][j][e];
      }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    s_sum[t.wm * SEG_T + col] = HALF ? sum * power_of_two(-LOSS_E_SHIFT) : sum;
    if (HALF && a.e32 && token < a.p.n) {
      float* out = a.e32 + token * a.e_pitch + class0 + 4 * t.kg;
#pragma unroll
      for (int i = 0; i < 8; ++i) *reinterpret_cast<floatx4*>(out + 16 * i) = acc[i][j];
    } else if (a.e[0] && token < a.p.n) {
      const int64_t at = token * a.e_pitch + class0 + 16 * (t.kg & 1) + 8 * (t.kg >> 1);
#pragma unroll
      for (int i = 0; i < 8; i += 2) store_blocks<HALF>(a.e[0] + at + 16 * i, a.e[1] ? a.e[1] + at + 16 * i : nullptr, acc[i][j], acc[i + 1][j]);
    }
  }
  __syncthreads();
  if (t.wm == 0 && t.kg == 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = 64 * t.wn + 16 * j + t.l16;
      const int64_t token = (int64_t)t.tn * SEG_T + col;
      if (token < a.p.n) {
        a.part_ref[(int64_t)t.tm * a.p.n + token] = base[j];
        a.part_sum[(int64_t)t.tm * a.p.n + token] = s_sum[col] + s_sum[SEG_T + col];
      }
    }
  }
}

// A wavefront per row.
template <bool VEC>
__global__ __launch_bounds__(256) void loss_reference_kernel(const __bf16* __restrict__ X, int64_t ldx, const __bf16* __restrict__ W,
                                                             int64_t ldw, int64_t d, LossPiece p, float* __restrict__ ref) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= p.n) return;
  int64_t c = p.targets[row];
  if (c < 0 || c >= p.vocab) c = row % p.vocab;
  const __bf16 *x = X + row * ldx, *w = W + c * ldw;
  float sum = 0.0f;
  if constexpr (VEC) {
#pragma unroll 2
    for (int64_t k = 8 * lane; k < d; k += 512) {
      const bf16x8 a = *reinterpret_cast<const bf16x8*>(x + k), b = *reinterpret_cast<const bf16x8*>(w + k);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = fmaf((float)a[j], (float)b[j], sum);
    }
  } else {
    for (int64_t k = lane; k < d; k += 64) sum = fmaf((float)x[k], (float)w[k], sum);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  sum = ceilf(sum * LOG2E);
  if (lane == 0) ref[row] = fabsf(sum) < 1e30f ? sum : -__builtin_inff();       // NaN too: the tiles find one
}

int launch_loss_reference(const void* X, int64_t ldx, const void* W, int64_t ldw, int64_t d, const LossPiece& p, const LossRows& r,
                          hipStream_t st) {
  const bool vec = d % 8 == 0 && ldx % 8 == 0 && ldw % 8 == 0 && (((uintptr_t)X | (uintptr_t)W) & 15) == 0;
  auto kernel = vec ? loss_reference_kernel<true> : loss_reference_kernel<false>;
  prof::Scope ps(prof::LOSS_ROWS, st, (double)p.n * d * 4.0);
  hipLaunchKernelGGL(kernel, dim3((unsigned)((p.n + 3) / 4)), dim3(256), 0, st, static_cast<const __bf16*>(X), ldx,
                     static_cast<const __bf16*>(W), ldw, d, p, r.ref);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

static int fill_segments(SegArgs& g, const Planes& a, const Planes& b, int64_t depth) {
  if (depth < 64 || depth % 64) return LQ_ERR_SHAPE;
  int count = 0;
  add_segments(g, &count, a, b, depth);
  return LQ_OK;
}
template <typename Args>
static int launch_tiles(void (*kernel)(Args), LdsLimit& limit, const Args& a, hipStream_t st) {
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(kernel), SEG_LDS));
  hipLaunchKernelGGL(kernel, dim3(seg_grid(a.g)), dim3(SEG_THREADS), SEG_LDS, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// dW's rows of a piece: features are the tile's rows and classes its columns.  2047 x 4096 by 32000 bf16: 560 us, 0.96 PFLOP/s.
struct DwArgs {
  SegArgs g;
  int64_t rows, cols;
  const float* factor; const float* class_inv;
  void* out; float* part;
};

template <typename H, typename T>
__global__ __launch_bounds__(SEG_THREADS, 2) void loss_dw_kernel(DwArgs a) {
  typedef T vec4 __attribute__((ext_vector_type(4)));
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const SegTile t = seg_tile(a.g);
  if (!t.live) return;
  SegAcc acc;
  seg_clear(acc);
  seg_products<H>(a.g, t, seg_first(a.g.pairs, t.split, a.g.splits), seg_first(a.g.pairs, t.split + 1, a.g.splits), seg_lds, acc);
  const float f = a.g.splits > 1 ? 0.0f : *a.factor;
  float* part = a.part + (size_t)t.split * (size_t)a.rows * (size_t)a.cols;
  seg_each(t, acc, [&](floatx4 v, int64_t col, int64_t row) {
    if (row >= a.rows || col >= a.cols) return;
    if (a.g.splits > 1) { store_floats(part + row * a.cols + col, v, col, a.cols); return; }
    T* at = static_cast<T*>(a.out) + row * a.cols + col;
    if constexpr (sizeof(T) == 4) v *= a.class_inv[row];
    v *= f;
    if ((a.cols & 3) == 0 && ((uintptr_t)a.out & (4 * sizeof(T) - 1)) == 0) { *reinterpret_cast<vec4*>(at) = __builtin_convertvector(v, vec4); return; }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < a.cols) at[e] = (T)v[e];
  });
}

int loss_dw_splits(int64_t rows, int64_t cols, int64_t depth, bool half) {
  return seg_splits(seg_tiles(rows, cols), depth / 64 * (half ? 3 : 1), 16);
}

// part (splits x rows x cols) = ranges of B A^T's reduction.
static int launch_parts(const Planes& a_planes, const Planes& b_planes, int64_t depth, int64_t rows, int64_t cols, bool half, float* part,
                        hipStream_t st) {
  DwArgs a{};
  LQ_TRY(fill_segments(a.g, a_planes, b_planes, depth));
  LQ_TRY(seg_shape(a.g, cols, rows, loss_dw_splits(rows, cols, depth, half)));
  if (a.g.splits < 2) return LQ_ERR_SHAPE;
  a.rows = rows; a.cols = cols; a.part = part;
  static LdsLimit limit[2];
  prof::Scope ps(prof::LOSS_LOGITS, st, 2.0 * rows * cols * depth);
  return half ? launch_tiles(loss_dw_kernel<_Float16, float>, limit[0], a, st) : launch_tiles(loss_dw_kernel<__bf16, __bf16>, limit[1], a, st);
}

// Classes that a piece's logits have beyond whole rounds of 256 tiles (all, if there is none), if those are up to a quarter of a round
// and their reduction can be cut into four ranges or more: their product fills the chip then (into parts, whose sums loss_tail_kernel turns into what the
// tiles of loss_logits_kernel become), where its tiles would leave most of the chip idle for as long as a round takes.  The whole call:
// 1000 x 1024 by 50265 fp32 with dW 1249 us, in one product 1277; 1000 x 4096 by 50265 bf16 789, 820; 300 x 2048 by 33001 bf16 190, 195;
// 200 x 4096 by 1500 (six tiles) fp32 with dW 162, 356; 500 x 4096 by 8000 (64 tiles) bf16 124, 153.
static int64_t tail_classes(int64_t n, int64_t classes, int64_t depth, bool half) {
  const int64_t across = (n + SEG_T - 1) / SEG_T, main = seg_tiles(classes, n) / 256 * 256 / across * SEG_T, rest = classes - main;
  if (rest <= 0 || seg_tiles(rest, n) > 64 || loss_dw_splits(n, rest, depth, half) < 4) return 0;
  return rest;
}
size_t loss_tail_floats(int64_t n, int64_t classes, int64_t depth, bool half) {
  const int64_t rest = tail_classes(n, classes, depth, half);
  return rest ? (size_t)loss_dw_splits(n, rest, depth, half) * (size_t)n * (size_t)rest : 0;
}

// A wavefront per token and tile of 256 classes.
struct TailArgs {
  LogitsArgs l;
  const float* part; int splits; int64_t first, rest;      // first: class of the piece
};
template <typename H>
__global__ __launch_bounds__(256) void loss_tail_kernel(TailArgs a) {
  constexpr bool HALF = !std::is_same<H, __bf16>::value;
  const int lane = threadIdx.x & 63;
  const int64_t token = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), at = (int64_t)blockIdx.y * SEG_T + 4 * lane, cls = a.first + at;
  if (token >= a.l.p.n) return;
  floatx4 x = {0.0f, 0.0f, 0.0f, 0.0f};
  if (at < a.rest) {
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) x += load_floats(a.part + ((size_t)s * a.l.p.n + token) * a.rest + at, at, a.rest);
  }
  const float f = logit_factor(a.l.s, token);
  const int64_t target = a.l.p.targets[token] - a.l.p.v0 - cls;
  float top = -__builtin_inff();
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] *= f;
    if (at + e >= a.rest) x[e] = -__builtin_inff();
    else if (e == target) { a.l.target[token] = x[e]; x[e] = -__builtin_inff(); }
    top = fmaxf(top, x[e]);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  top = ceilf(top);
  const float base = a.l.p.v0 == 0 && HALF ? -__builtin_inff() : a.l.ref[token], room = HALF ? (float)LOSS_E_ROOM : 64.0f;
  const float ref = top <= base + room ? base : top;
  const float from = (ref == -__builtin_inff() ? 0.0f : ref) - (HALF ? (float)LOSS_E_SHIFT : 0.0f);
  float sum = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = __builtin_amdgcn_exp2f(x[e] - from);
    sum += x[e];
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) {
    const int64_t tile = a.first / SEG_T + blockIdx.y;
    a.l.part_ref[tile * a.l.p.n + token] = ref;
    a.l.part_sum[tile * a.l.p.n + token] = HALF ? sum * power_of_two(-LOSS_E_SHIFT) : sum;
  }
  const int64_t to = token * a.l.e_pitch + cls;              // rows of E end on whole tiles
  if (HALF && a.l.e32) {
    *reinterpret_cast<floatx4*>(a.l.e32 + to) = x;
  } else if (a.l.e[0]) {
    uintx2 hi, lo;
    split_four<HALF>(x, hi, lo);
    *reinterpret_cast<uintx2*>(a.l.e[0] + to) = hi;
    if (HALF || a.l.e[1]) *reinterpret_cast<uintx2*>(a.l.e[1] + to) = lo;
  }
}

int launch_loss_logits(const Planes& w, const Planes& x, int64_t depth, const LossPiece& p, const LossRows& r, const LossScales& s,
                       float* part_ref, float* part_sum, uint16_t* const e[2], float* e32, int64_t e_pitch, float* part,
                       size_t part_floats, hipStream_t st) {
  const bool half = s.x_inv != nullptr;
  if (e32 && (!half || p.v0 != 0)) return LQ_ERR_ARG;
  const int64_t rest = tail_classes(p.n, p.classes, depth, half), main = p.classes - rest;
  LogitsArgs a{};
  a.p = p; a.s = s; a.ref = r.ref; a.target = r.target; a.part_ref = part_ref; a.part_sum = part_sum;
  a.e[0] = e[0]; a.e[1] = e[1]; a.e32 = e32; a.e_pitch = e_pitch;
  if (main > 0) {
    static LdsLimit limit[2];
    LQ_TRY(fill_segments(a.g, w, x, depth));
    LQ_TRY(seg_shape(a.g, main, p.n, 1));
    prof::Scope ps(prof::LOSS_LOGITS, st, 2.0 * p.n * main * depth);
    LQ_TRY(half ? launch_tiles(loss_logits_kernel<_Float16>, limit[0], a, st) : launch_tiles(loss_logits_kernel<__bf16>, limit[1], a, st));
  }
  if (!rest) return LQ_OK;
  if (part_floats < loss_tail_floats(p.n, p.classes, depth, half)) return LQ_ERR_WORKSPACE;
  const Planes tail{{w.p[0] + main * w.pitch, w.p[1] ? w.p[1] + main * w.pitch : nullptr, nullptr}, w.pitch};
  LQ_TRY(launch_parts(tail, x, depth, p.n, rest, half, part, st));
  const TailArgs t{a, part, loss_dw_splits(p.n, rest, depth, half), main, rest};
  prof::Scope ps(prof::LOSS_ROWS, st, (double)p.n * rest * (4.0 * t.splits + 4.0));
  hipLaunchKernelGGL(half ? loss_tail_kernel<_Float16> : loss_tail_kernel<__bf16>,
                     dim3((unsigned)((p.n + 3) / 4), (unsigned)((rest + SEG_T - 1) / SEG_T)), dim3(256), 0, st, t);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// What becomes of the rows when all classes have been seen, and their total in 64 bits and a fixed order.  Called by all threads of
// one workgroup of 1024.
struct RowsArgs {
  LossRows r; LossScales s;
  const int64_t* targets; int64_t n, vocab; int mean;
  float* loss; float* row_loss; float* lse; float* factors;
};
__device__ __forceinline__ void finish_rows(const RowsArgs& a) {
  __shared__ double s_sum[1024];
  __shared__ uint32_t s_count[1024];
  double sum = 0.0;
  uint32_t count = 0;
  for (int64_t i = threadIdx.x; i < a.n; i += 1024) {
    const int64_t t = a.targets[i];
    const float size = log2f(a.r.sum[i]), others = a.r.ref[i] + size;      // log2 of the sum without the target; -inf: no other class
    float l = 0.0f, wrong = 0.0f, all = others;
    if (t >= 0 && t < a.vocab) {
      const float z = (a.r.target[i] - a.r.ref[i]) - size;     // the reference is whole: one rounding less than target - others
      l = fmaxf(-z, 0.0f) * LN2 + log1pf(exp2f(-fabsf(z)));
      wrong = 1.0f / (1.0f + exp2f(z));
      all = fmaxf(a.r.target[i], others) + log1pf(exp2f(-fabsf(z))) * LOG2E;
      if (z != z) l = all = z;
      sum += l;
      ++count;
    }
    a.row_loss[i] = l;
    if (a.lse) a.lse[i] = all * LN2;
    a.r.wrong[i] = wrong;
    a.r.lse2[i] = all;
  }
  s_sum[threadIdx.x] = sum;
  s_count[threadIdx.x] = count;
  __syncthreads();
  for (int o = 512; o; o >>= 1) {
    if ((int)threadIdx.x < o) { s_sum[threadIdx.x] += s_sum[threadIdx.x + o]; s_count[threadIdx.x] += s_count[threadIdx.x + o]; }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    const double f = a.mean ? 1.0 / (double)(s_count[0] ? s_count[0] : 1) : 1.0;      // no row counts: the mean is 0
    *a.loss = (float)(s_sum[0] * f);
    a.factors[0] = (float)f;
    a.factors[1] = a.s.xt_top ? (float)f * power_of_two(-half_exponent(*a.s.xt_top)) : (float)f;
  }
}

__global__ __launch_bounds__(1024) void loss_rows_kernel(RowsArgs a) { finish_rows(a); }

int launch_loss_rows(const LossRows& r, const LossScales& s, const int64_t* targets, int64_t n, int64_t vocab, bool mean, float* loss,
                     float* row_loss, float* lse, float* factors, hipStream_t st) {
  const RowsArgs a{r, s, targets, n, vocab, (int)mean, loss, row_loss, lse, factors};
  prof::Scope ps(prof::LOSS_ROWS, st, (double)n * 36.0);
  hipLaunchKernelGGL(loss_rows_kernel, dim3(1), dim3(1024), 0, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// A wavefront joins the tiles' sums of one row.  Tiles whose E lies at a smaller power of two than the row's new one are
// multiplied down, which is exact (what leaves the range of bf16 is below 2^-126 of the largest term, that of fp16 below 2^-37).
// Without a reference from the start that is all of them in the first piece, and a launch of its own does it; else it is a row whose
// logits outgrow its reference.
struct JoinArgs {
  LossPiece p; LossRows r;
  const float* part_ref; const float* part_sum; int tiles;
  uint16_t* e[2]; int64_t e_pitch;
  int told;
  LossOperands o;
};

// v *= 2^e, e <= 0, in two steps: 2^e can leave the range where a value of up to 2^64 times it does not.
template <typename H>
__device__ __forceinline__ void scale_run(uint16_t* at, float e) {
  typedef H hx4 __attribute__((ext_vector_type(4)));
  hx4 v = *reinterpret_cast<const hx4*>(at);
  const float whole = fmaxf(e, -250.0f), half = floorf(0.5f * whole);
  const float f = __builtin_amdgcn_exp2f(half), g = __builtin_amdgcn_exp2f(whole - half);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = (H)((float)v[k] * f * g);
  *reinterpret_cast<hx4*>(at) = v;
}

// The target's logit of a row by a wavefront, whose lanes' sums are short: along the matrix pipe's chain of d / 32 sums it is off by
// some 1e-6, which is most of a row loss's error, since those of the other classes cancel in their sum.
template <typename T>
__device__ __forceinline__ void join_target(const JoinArgs& a, int64_t row, int lane) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  const int64_t t = a.p.targets[row];
  if (t < 0 || t >= a.p.vocab) return;
  const T *x = static_cast<const T*>(a.o.X) + row * a.o.ldx, *w = static_cast<const T*>(a.o.W) + t * a.o.ldw;
  float sum[2] = {0.0f, 0.0f};
  auto add = [&](const vec8& u, const vec8& v) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j & 1] = fmaf((float)u[j], (float)v[j], sum[j & 1]);
  };
  if (a.o.vec) {
#pragma unroll 4
    for (int64_t k = 8 * lane; k < a.o.d; k += 512) add(*reinterpret_cast<const vec8*>(x + k), *reinterpret_cast<const vec8*>(w + k));
  } else {                                            // in the same order: the same bits
#pragma unroll 1
    for (int64_t k = 8 * lane; k < a.o.d; k += 512) {
      vec8 u = {}, v = {};
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j < a.o.d) { u[j] = x[k + j]; v[j] = w[k + j]; }
      add(u, v);
    }
  }
  float s = sum[0] + sum[1];
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  if (lane == 0) a.r.target[row] = s * LOG2E;
}

constexpr int JOIN_LOADS = 8;      // of a lane, under way together
// told: the row has a reference from the start (launch_loss_reference).
template <typename H>
__device__ __forceinline__ void join_row(const JoinArgs& a, int64_t row, int lane) {
  const bool first = a.p.v0 == 0;
  const float old = first && !a.told ? -__builtin_inff() : a.r.ref[row];
  float ref = old;
  for (int t0 = lane; t0 < a.tiles; t0 += 64 * JOIN_LOADS) {
    float mine[JOIN_LOADS];
#pragma unroll
    for (int q = 0; q < JOIN_LOADS; ++q) mine[q] = t0 + 64 * q < a.tiles ? a.part_ref[(int64_t)(t0 + 64 * q) * a.p.n + row] : -__builtin_inff();
#pragma unroll
    for (int q = 0; q < JOIN_LOADS; ++q) ref = fmaxf(ref, mine[q]);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) ref = fmaxf(ref, __shfl_xor(ref, o));
  const float from = ref == -__builtin_inff() ? 0.0f : ref;
  float sum = 0.0f;
  for (int t0 = lane; t0 < a.tiles; t0 += 64 * JOIN_LOADS) {
    float mine[JOIN_LOADS], part[JOIN_LOADS];
#pragma unroll
    for (int q = 0; q < JOIN_LOADS; ++q) {
      const int64_t at = (int64_t)(t0 + 64 * q) * a.p.n + row;
      const bool live = t0 + 64 * q < a.tiles;
      mine[q] = live ? a.part_ref[at] : -__builtin_inff();
      part[q] = live ? a.part_sum[at] : 0.0f;
    }
#pragma unroll
    for (int q = 0; q < JOIN_LOADS; ++q) sum += part[q] * __builtin_amdgcn_exp2f(mine[q] - from);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) {
    const float shift = __builtin_amdgcn_exp2f(old - from);
    a.r.sum[row] = first ? sum : a.r.sum[row] * shift + sum;
    a.r.shift[row] = shift;
    a.r.ref[row] = ref;
  }
  if (!a.e[0] || (first && !a.told)) return;
  for (int t0 = 0; t0 < a.tiles; t0 += 64) {
    const float mine = t0 + lane < a.tiles ? a.part_ref[(int64_t)(t0 + lane) * a.p.n + row] : ref;
    for (uint64_t low = __ballot(mine != ref); low; low &= low - 1) {
      const int t = __builtin_ctzll(low);
      const float ft = __shfl(mine, t) - from;
      const int64_t at = row * a.e_pitch + (int64_t)(t0 + t) * SEG_T + 4 * lane;
      scale_run<H>(a.e[0] + at, ft);
      if (a.e[1]) scale_run<H>(a.e[1] + at, ft);
    }
  }
}

template <typename H>
__global__ __launch_bounds__(256) void loss_join_kernel(JoinArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.p.n) return;
  if (a.o.W && a.o.dtype == LQ_T_BF16) join_target<__bf16>(a, row, threadIdx.x & 63);
  else if (a.o.W) join_target<float>(a, row, threadIdx.x & 63);
  join_row<H>(a, row, threadIdx.x & 63);
}

// Up to 16 rows, whole vocabulary: one workgroup joins and finishes them.
__global__ __launch_bounds__(1024) void loss_join_rows_kernel(JoinArgs a, RowsArgs rows) {
  const int64_t row = threadIdx.x >> 6;
  if (row < a.p.n) {
    if (a.o.dtype == LQ_T_BF16) join_target<__bf16>(a, row, threadIdx.x & 63);
    else join_target<float>(a, row, threadIdx.x & 63);
    join_row<__bf16>(a, row, threadIdx.x & 63);
  }
  __threadfence_block();
  __syncthreads();
  finish_rows(rows);
}

// The first piece's E in fp32: 256 classes x 16 tokens a workgroup.
__global__ __launch_bounds__(256) void loss_shift_kernel(JoinArgs a) {
  const int64_t token = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (token >= a.p.n) return;
  const float ref = a.r.ref[token], mine = a.part_ref[(int64_t)blockIdx.y * a.p.n + token];
  if (mine == ref) return;
  const float f = mine - ref;
  const int64_t at = token * a.e_pitch + (int64_t)blockIdx.y * SEG_T + 4 * (threadIdx.x & 15);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    scale_run<_Float16>(a.e[0] + at + 64 * q, f);
    scale_run<_Float16>(a.e[1] + at + 64 * q, f);
  }
}

int launch_loss_join(const LossPiece& p, const LossRows& r, bool half, bool told, const float* part_ref, const float* part_sum, int tile,
                     uint16_t* const e[2], int64_t e_pitch, const LossOperands& o, hipStream_t st) {
  const JoinArgs a{p, r, part_ref, part_sum, (int)((p.classes + tile - 1) / tile), {e[0], e[1]}, e_pitch, told, o};
  prof::Scope ps(prof::LOSS_ROWS, st, (double)p.n * a.tiles * 8.0);
  auto kernel = half ? loss_join_kernel<_Float16> : loss_join_kernel<__bf16>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((p.n + 3) / 4)), dim3(256), 0, st, a);
  LQ_HIP_TRY(hipGetLastError());
  if (!e[0] || p.v0 != 0 || told) return LQ_OK;
  if (!half || a.tiles > 65535) return LQ_ERR_SHAPE;
  hipLaunchKernelGGL(loss_shift_kernel, dim3((unsigned)((p.n + 15) / 16), (unsigned)a.tiles), dim3(256), 0, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

int launch_loss_join_rows(const LossPiece& p, const LossRows& r, const float* part_ref, const float* part_sum, int tile, bool mean,
                          const LossOperands& o, float* loss, float* row_loss, float* lse, float* factors, hipStream_t st) {
  if (!o.X || !o.W) return LQ_ERR_NULL;
  if (p.n > 16 || p.v0 != 0 || p.classes != p.vocab) return LQ_ERR_SHAPE;
  const JoinArgs a{p, r, part_ref, part_sum, (int)((p.classes + tile - 1) / tile), {nullptr, nullptr}, 0, 0, o};
  const RowsArgs rows{r, LossScales{}, p.targets, p.n, p.vocab, (int)mean, loss, row_loss, lse, factors};
  prof::Scope ps(prof::LOSS_ROWS, st, (double)p.n * a.tiles * 8.0);
  hipLaunchKernelGGL(loss_join_rows_kernel, dim3(1), dim3(1024), 0, st, a, rows);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// acc = acc shift + E W: features are the tile's rows and tokens its columns, so that a lane holds four neighbours of a row of acc.
// 2047 x 4096 by 32000 bf16: 490 us, 1.09 PFLOP/s; in one range without a sum after it the whole call (with dW) 1.84 ms for 1.53.
struct AccumulateArgs {
  SegArgs g;
  int64_t n, d;
  const float* shift; int first;
  float* acc; float* part;
};

template <typename H>
__global__ __launch_bounds__(SEG_THREADS, 2) void loss_accumulate_kernel(AccumulateArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const SegTile t = seg_tile(a.g);
  if (!t.live) return;
  SegAcc acc;
  seg_clear(acc);
  seg_products<H, true>(a.g, t, seg_first(a.g.pairs, t.split, a.g.splits), seg_first(a.g.pairs, t.split + 1, a.g.splits), seg_lds, acc);
  float* out = a.g.splits > 1 ? a.part + (size_t)t.split * (size_t)a.n * (size_t)a.d : a.acc;
  const bool add = a.g.splits == 1 && !a.first;
  seg_each(t, acc, [&](floatx4 v, int64_t col, int64_t token) {
    if (token >= a.n || col >= a.d) return;
    float* at = out + token * a.d + col;
    if (add) v = load_floats(at, col, a.d) * a.shift[token] + v;
    store_floats(at, v, col, a.d);
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

int loss_accumulate_splits(int64_t n, int64_t d, int64_t depth, bool half) {
  return seg_splits(seg_tiles(n, d), depth / 64 * (half ? 3 : 1), 64);
}

int launch_loss_accumulate(const Planes& e, const Planes& w, int64_t classes, int64_t n, int64_t d, const float* shift, bool first,
                           float* acc, float* part, size_t part_floats, hipStream_t st) {
  const bool half = e.p[1] != nullptr;
  const int64_t depth = up_to(classes, 64);
  if (w.pitch % 8 || w.pitch < up_to(d, 8) || e.pitch < depth) return LQ_ERR_SHAPE;
  AccumulateArgs a{};
  LQ_TRY(fill_segments(a.g, w, e, depth));
  LQ_TRY(seg_shape(a.g, d, n, loss_accumulate_splits(n, d, depth, half)));
  a.g.rows_a = up_to(d, 8); a.g.depth_a = classes;           // whole units of W's rows
  if (a.g.splits > 1 && part_floats < (size_t)a.g.splits * (size_t)n * (size_t)d) return LQ_ERR_WORKSPACE;
  a.n = n; a.d = d; a.shift = shift; a.first = first; a.acc = acc; a.part = part;
  static LdsLimit limit[2];
  {
    prof::Scope ps(prof::LOSS_ACCUMULATE, st, 2.0 * n * d * depth);
    LQ_TRY(half ? launch_tiles(loss_accumulate_kernel<_Float16>, limit[0], a, st) : launch_tiles(loss_accumulate_kernel<__bf16>, limit[1], a, st));
  }
  if (a.g.splits > 1) {
    prof::Scope ps(prof::LOSS_ROWS, st, (double)n * d * 4.0 * (a.g.splits + 2));
    const int64_t wgs = std::min<int64_t>((n * d + 255) / 256, 8192);
    hipLaunchKernelGGL(loss_accumulate_sum_kernel, dim3((unsigned)wgs), dim3(256), 0, st, part, a.g.splits, n, d, shift, (int)first, acc);
    LQ_HIP_TRY(hipGetLastError());
  }
  return LQ_OK;
}

// dX_i = g (1 - p_t) (E W / S - w_t): one workgroup per row, its features in turn; VEC: four at a time.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void loss_dx_kernel(LossRows r, LossScales sc, const int64_t* __restrict__ targets, int64_t d,
                                                      int64_t vocab, const float* __restrict__ acc, const T* __restrict__ W,
                                                      int64_t ldw, const float* __restrict__ factor, T* __restrict__ dX) {
  typedef T vec4 __attribute__((ext_vector_type(4)));
  const int64_t row = blockIdx.x, t = targets[row];
  const bool counts = t >= 0 && t < vocab;
  const float s = r.sum[row];
  float inv = s == 0.0f ? 0.0f : 1.0f / s;                   // no other class: acc is zero
  if (sc.w_top) inv *= power_of_two(-LOSS_E_SHIFT) * power_of_two(-half_exponent(*sc.w_top));
  const float g = counts ? r.wrong[row] * *factor : 0.0f;
  if constexpr (VEC) {
    for (int64_t c = 4 * threadIdx.x; c < d; c += 1024) {
      vec4 out = {};
      if (counts) {
        const floatx4 w = __builtin_convertvector(*reinterpret_cast<const vec4*>(W + t * ldw + c), floatx4);
        out = __builtin_convertvector(g * (*reinterpret_cast<const floatx4*>(acc + row * d + c) * inv - w), vec4);
      }
      *reinterpret_cast<vec4*>(dX + row * d + c) = out;
    }
  } else {
    for (int64_t c = threadIdx.x; c < d; c += 256)
      dX[row * d + c] = counts ? (T)(g * (acc[row * d + c] * inv - (float)W[t * ldw + c])) : (T)0.0f;
  }
}

template <typename T>
static void dx_of(const LossRows& r, const LossScales& s, const int64_t* targets, int64_t n, int64_t d, int64_t vocab, const float* acc,
                  const void* W, int64_t ldw, const float* factor, void* dX, hipStream_t st) {
  const bool vec = d % 4 == 0 && ldw % 4 == 0 && (((uintptr_t)W | (uintptr_t)dX) & (4 * sizeof(T) - 1)) == 0;
  auto kernel = vec ? loss_dx_kernel<T, true> : loss_dx_kernel<T, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(256), 0, st, r, s, targets, d, vocab, acc, static_cast<const T*>(W), ldw, factor,
                     static_cast<T*>(dX));
}

int launch_loss_dx(const LossRows& r, const LossScales& s, const int64_t* targets, int64_t n, int64_t d, int64_t vocab,
                   const float* acc, const void* W, int64_t ldw, int dtype, const float* factor, void* dX, hipStream_t st) {
  prof::Scope ps(prof::LOSS_ROWS, st, (double)n * d * (4.0 + 2.0 * type_bytes(dtype)));
  if (dtype == LQ_T_BF16) dx_of<__bf16>(r, s, targets, n, d, vocab, acc, W, ldw, factor, dX, st);
  else dx_of<float>(r, s, targets, n, d, vocab, acc, W, ldw, factor, dX, st);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// The gradient of a piece's logits, transposed: the rows of Gt are classes, their tokens contiguous, as dW = Gt X reads them.
// Tokens are the tile's rows here, so that a lane holds four neighbours of a row of Gt.  fp32: a class can be improbable in every row,
// and its planes need a power of two of its own; Gt goes out in fp32 and a pass over its rows makes the planes.
// 4096 x 4096 by 16128 classes, bf16: 450 us, 1.2 PFLOP/s.
struct GradientArgs {
  SegArgs g;
  LossPiece p; LossRows r; LossScales s;
  void* out; int64_t pitch;
};

template <typename H>
__global__ __launch_bounds__(SEG_THREADS, 2) void loss_gradient_kernel(GradientArgs a) {
  constexpr bool HALF = !std::is_same<H, __bf16>::value;
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const SegTile t = seg_tile(a.g);
  if (!t.live) return;
  SegAcc acc;
  seg_clear(acc);
  seg_products<H>(a.g, t, 0, a.g.pairs, seg_lds, acc);
  __syncthreads();
  // per token of the tile: factor of the logit, log2 of the sum, 1 - p of the target, the target's class inside the piece
  float* s_f = reinterpret_cast<float*>(seg_lds);
  float *s_lse = s_f + SEG_T, *s_wrong = s_lse + SEG_T;
  int* s_at = reinterpret_cast<int*>(s_wrong + SEG_T);
  if (threadIdx.x < SEG_T) {
    const int64_t token = (int64_t)t.tm * SEG_T + threadIdx.x;
    const int64_t target = token < a.p.n ? a.p.targets[token] : -1;
    const bool counts = target >= 0 && target < a.p.vocab;
    const int64_t at = target - a.p.v0;
    s_f[threadIdx.x] = counts ? logit_factor(a.s, token) : 0.0f;
    s_lse[threadIdx.x] = counts ? a.r.lse2[token] : 0.0f;
    s_wrong[threadIdx.x] = counts ? a.r.wrong[token] : 0.0f;
    s_at[threadIdx.x] = !counts ? -2 : at >= 0 && at < a.p.classes ? (int)at : -1;
  }
  __syncthreads();
  const int64_t cols = (a.p.n + 63) / 64 * 64;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t cls = (int64_t)t.tn * SEG_T + 64 * t.wn + 16 * j + t.l16;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      floatx4 g[2];
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = 128 * t.wm + 16 * (i + q) + 4 * t.kg + e, at = s_at[row];
          const float p = __builtin_amdgcn_exp2f(acc[i + q][j][e] * s_f[row] - s_lse[row]);
          g[q][e] = at == -2 ? 0.0f : at == (int)cls ? -s_wrong[row] : p;     // rows that do not count: whatever they hold
        }
      // a block of 32 tokens lies inside the padded rows or beyond them
      const int64_t token = (int64_t)t.tm * SEG_T + 128 * t.wm + 16 * i, to = cls * a.pitch + token;
      const bool live = cls < a.p.classes && token < cols;
      if constexpr (HALF) {
        if (!live) continue;
        float* out = static_cast<float*>(a.out) + to + 4 * t.kg;
        *reinterpret_cast<floatx4*>(out) = g[0];
        *reinterpret_cast<floatx4*>(out + 16) = g[1];
      } else {
        uintx2 h0, l0, h1, l1;
        split_four<false>(g[0], h0, l0);
        split_four<false>(g[1], h1, l1);
        const uintx4 h = seg_pair_blocks(h0, h1);
        if (live) *reinterpret_cast<uintx4*>(static_cast<uint16_t*>(a.out) + to + 16 * (t.kg & 1) + 8 * (t.kg >> 1)) = h;
      }
    }
  }
}

int launch_loss_gradient(const Planes& w, const Planes& x, int64_t depth, const LossPiece& p, const LossRows& r, const LossScales& s,
                         void* g, int64_t g_pitch, hipStream_t st) {
  if (g_pitch < up_to(p.n, 64)) return LQ_ERR_SHAPE;
  GradientArgs a{};
  LQ_TRY(fill_segments(a.g, x, w, depth));
  LQ_TRY(seg_shape(a.g, p.n, p.classes, 1));
  a.p = p; a.r = r; a.s = s; a.out = g; a.pitch = g_pitch;
  static LdsLimit limit[2];
  prof::Scope ps(prof::LOSS_LOGITS, st, 2.0 * p.n * p.classes * depth);
  return s.x_inv ? launch_tiles(loss_gradient_kernel<_Float16>, limit[0], a, st) : launch_tiles(loss_gradient_kernel<__bf16>, limit[1], a, st);
}

// ------------------------------------------------------------------------------------------------
// The same from E, where one piece is the whole vocabulary: p = E (1 - p_t) / S, a pass over E for a product less (2047 x 32000: 74 us;
// 1000 x 50265 fp32: 113 us, 5.3 TB/s).  A workgroup turns 64 tokens x 64 classes in LDS, a thread two tokens of eight classes.  bf16: E
// is both planes.  fp32: E is one array relative to its tiles' powers of two; where dX needs them (e[0]), its planes relative to the
// rows' go out in the same pass.  Gt's planes are times a power of two per class, of the largest magnitudes that
// loss_class_tops_kernel found, and class_inv gets its inverse.
struct FromEArgs {
  LossPiece p; LossRows r;
  const float* part_ref; const float* e32;
  uint16_t* e[2]; int64_t e_pitch;
  uint16_t* out[2]; int64_t pitch;
  int tiles_r;
  float* tops; int ranges; float* class_inv;
};
// What a token's E is to be multiplied by to be p: to the row's power of two (shift) and by (1 - p_t) / S.
__device__ __forceinline__ float tile_shift(const FromEArgs& a, int64_t token, int64_t c) {
  const float ref = a.r.ref[token], mine = a.part_ref[c / SEG_T * a.p.n + token];
  return mine == ref ? 1.0f : __builtin_amdgcn_exp2f(mine - ref);
}
template <bool HALF>
__device__ __forceinline__ float row_factor(const FromEArgs& a, int64_t token) {
  const float s = a.r.sum[token];
  return s == 0.0f ? 0.0f : a.r.wrong[token] / s * (HALF ? power_of_two(-LOSS_E_SHIFT) : 1.0f);
}

// tops[range][class] = the largest |Gt| among a range of tokens: a thread reads eight classes of every fourth token (1000 x
// 50265: 39 us, 5.2 TB/s).
constexpr int TOPS_TOKENS = 64, TOPS_CLASSES = 512;
__global__ __launch_bounds__(256) void loss_class_tops_kernel(FromEArgs a) {
  typedef float floatx8 __attribute__((ext_vector_type(8)));
  __shared__ float s_f[2][TOPS_TOKENS];                     // per tile of 256 classes
  __shared__ int64_t s_t[TOPS_TOKENS];
  __shared__ uint32_t s_top[4][TOPS_CLASSES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c0 = (int64_t)blockIdx.x * TOPS_CLASSES, c = c0 + 8 * lane;
  const int64_t blocks = (a.p.n + TOPS_TOKENS - 1) / TOPS_TOKENS, b0 = blocks * blockIdx.y / a.ranges, b1 = blocks * (blockIdx.y + 1) / a.ranges;
  uint32_t top[8] = {};
  for (int64_t b = b0; b < b1; ++b) {
    __syncthreads();
    if (threadIdx.x < TOPS_TOKENS) {
      const int64_t token = b * TOPS_TOKENS + threadIdx.x, t = token < a.p.n ? a.p.targets[token] : -1;
      const bool counts = t >= 0 && t < a.p.vocab;
      s_t[threadIdx.x] = counts ? t : -1;
#pragma unroll
      for (int k = 0; k < 2; ++k)
        s_f[k][threadIdx.x] = counts && c0 + SEG_T * k < a.e_pitch ? tile_shift(a, token, c0 + SEG_T * k) * row_factor<true>(a, token) : 0.0f;
    }
    __syncthreads();
    if (c >= a.e_pitch) continue;
#pragma unroll 4
    for (int i = wave; i < TOPS_TOKENS; i += 4) {
      const int64_t token = b * TOPS_TOKENS + i, t = s_t[i];
      if (t < 0) continue;                                  // rows that do not count: whatever they hold
      const floatx8 e = *reinterpret_cast<const floatx8*>(a.e32 + token * a.e_pitch + c);
      const float f = s_f[lane >> 5][i];
#pragma unroll
      for (int j = 0; j < 8; ++j) top[j] = max(top[j], finite_magnitude(e[j] * f));
      if (t >= c && t < c + 8) {
        const uint32_t w = finite_magnitude(a.r.wrong[token]);
#pragma unroll
        for (int j = 0; j < 8; ++j) top[j] = t == c + j ? max(top[j], w) : top[j];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) s_top[wave][8 * lane + j] = top[j];
  __syncthreads();
  for (int i = threadIdx.x; i < TOPS_CLASSES; i += 256)
    if (c0 + i < a.p.classes)
      a.tops[(int64_t)blockIdx.y * a.p.classes + c0 + i] = __uint_as_float(max(max(s_top[0][i], s_top[1][i]), max(s_top[2][i], s_top[3][i])));
}

template <typename H>
__global__ __launch_bounds__(256) void loss_gradient_from_e_kernel(FromEArgs a) {
  constexpr bool HALF = !std::is_same<H, __bf16>::value;
  constexpr int WORDS = 33;
  typedef H hx8 __attribute__((ext_vector_type(8)));
  typedef float floatx8 __attribute__((ext_vector_type(8)));
  typedef H hx2 __attribute__((ext_vector_type(2)));
  __shared__ uint32_t s_w[HALF ? 2 : 1][64 * WORDS];
  __shared__ uint32_t s_top[HALF ? 4 : 1][64];
  const int c = (threadIdx.x & 7) * 8, pair = threadIdx.x >> 3;
  const int64_t r0 = (int64_t)(blockIdx.x % a.tiles_r) * 64, c0 = (int64_t)(blockIdx.x / a.tiles_r) * 64;
  // all loads first: none waits for another
  floatx8 e[2];
  float f[2], wrong[2], shift[2];
  int64_t target[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t token = r0 + 2 * pair + h, row = token < a.p.n ? token : a.p.n - 1;
    const int64_t at = row * a.e_pitch + c0 + c;             // rows of E end on whole tiles
    if constexpr (HALF) e[h] = *reinterpret_cast<const floatx8*>(a.e32 + at);
    else
      e[h] = __builtin_convertvector(*reinterpret_cast<const hx8*>(a.e[0] + at), floatx8) +
             __builtin_convertvector(*reinterpret_cast<const hx8*>(a.e[1] + at), floatx8);
    target[h] = token < a.p.n ? a.p.targets[row] : -1;
    wrong[h] = a.r.wrong[row];
    f[h] = row_factor<HALF>(a, row);
    shift[h] = HALF ? tile_shift(a, row, c0) : 1.0f;
  }
  float scale[8];
  if constexpr (HALF) {
    const int k = threadIdx.x & 63, q = threadIdx.x >> 6;
    uint32_t top = 0;
    if (c0 + k < a.p.classes) {
#pragma unroll 4
      for (int i = q; i < a.ranges; i += 4) top = max(top, __float_as_uint(a.tops[i * a.p.classes + c0 + k]));
    }
    s_top[q][k] = top;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j)
      scale[j] = power_of_two(half_exponent(max(max(s_top[0][c + j], s_top[1][c + j]), max(s_top[2][c + j], s_top[3][c + j]))));
    if (r0 == 0 && q == 0 && c0 + k < a.p.classes)
      a.class_inv[c0 + k] = power_of_two(-half_exponent(max(max(s_top[0][k], s_top[1][k]), max(s_top[2][k], s_top[3][k]))));
  }
  float g[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t t = target[h];
    if (t < 0 || t >= a.p.vocab) {                           // rows that do not count: whatever they hold
#pragma unroll
      for (int j = 0; j < 8; ++j) g[h][j] = 0.0f;
      continue;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      g[h][j] = e[h][j] * shift[h] * f[h];
      if (c0 + c + j == t) g[h][j] = -wrong[h];
      if constexpr (HALF) g[h][j] *= scale[j];
    }
  }
  if constexpr (HALF) {
    if (a.e[0]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t token = r0 + 2 * pair + h, at = token * a.e_pitch + c0 + c;
        if (token >= a.p.n) continue;
        hx8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {                        // as loss_shift_kernel makes them: dX is the same with and without dW
          const HalfPair v = split_half(e[h][j]);
          hi[j] = (H)((float)v.hi * shift[h]);
          lo[j] = (H)((float)v.lo * shift[h]);
        }
        *reinterpret_cast<hx8*>(a.e[0] + at) = hi;
        *reinterpret_cast<hx8*>(a.e[1] + at) = lo;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const hx2 hi = {(H)g[0][j], (H)g[1][j]};
    s_w[0][(c + j) * WORDS + pair] = __builtin_bit_cast(uint32_t, hi);
    if constexpr (HALF) s_w[HALF ? 1 : 0][(c + j) * WORDS + pair] = __builtin_bit_cast(uint32_t, hx2{(H)(g[0][j] - (float)hi[0]), (H)(g[1][j] - (float)hi[1])});
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int col = (threadIdx.x >> 3) + 32 * h, word = (threadIdx.x & 7) * 4;
    if (c0 + col >= a.p.classes) continue;
#pragma unroll
    for (int k = 0; k < (HALF ? 2 : 1); ++k) {
      uintx4 out;
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = s_w[k][col * WORDS + word + j];
      *reinterpret_cast<uintx4*>(a.out[k] + (c0 + col) * a.pitch + r0 + 2 * word) = out;
    }
  }
}

int loss_class_ranges(int64_t n) { return (int)std::min<int64_t>((n + TOPS_TOKENS - 1) / TOPS_TOKENS, 16); }

int launch_loss_gradient_from_e(const LossPiece& p, const LossRows& r, const float* part_ref, const float* e32,
                                uint16_t* const e[2], int64_t e_pitch, uint16_t* const g[2], int64_t g_pitch, float* tops,
                                float* class_inv, hipStream_t st) {
  const int64_t tr = (p.n + 63) / 64, tc = (p.classes + 63) / 64;
  if (p.v0 != 0 || p.classes != p.vocab || g_pitch < up_to(p.n, 64) || tr * tc >= (1ll << 31) || e_pitch % SEG_T) return LQ_ERR_SHAPE;
  const bool half = e32 != nullptr;
  if (half ? !tops || !class_inv || !part_ref : !e[0] || !e[1]) return LQ_ERR_ARG;
  const FromEArgs a{p, r, part_ref, e32, {e[0], e[1]}, e_pitch, {g[0], g[1]}, g_pitch, (int)tr, tops, loss_class_ranges(p.n), class_inv};
  prof::Scope ps(prof::TRAIN_PLANES, st, (double)p.n * p.classes * (half ? 8.0 : 6.0));      // fp32 with dX: its planes of E beside
  if (half) {
    const dim3 grid((unsigned)((p.classes + TOPS_CLASSES - 1) / TOPS_CLASSES), (unsigned)a.ranges);
    hipLaunchKernelGGL(loss_class_tops_kernel, grid, dim3(256), 0, st, a);
    LQ_HIP_TRY(hipGetLastError());
  }
  auto kernel = half ? loss_gradient_from_e_kernel<_Float16> : loss_gradient_from_e_kernel<__bf16>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(tr * tc)), dim3(256), 0, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void loss_dw_sum_kernel(const float* __restrict__ part, int splits, int64_t total, int64_t cols,
                                                          const float* __restrict__ factor, const float* __restrict__ class_inv,
                                                          T* __restrict__ out) {
  const float f = *factor;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    float v = 0.0f;
    for (int s = 0; s < splits; ++s) v += part[s * total + i];
    if constexpr (sizeof(T) == 4) v *= class_inv[i / cols];
    out[i] = (T)(v * f);
  }
}

static int dw_of(const Planes& g, const Planes& xt, int64_t depth, int64_t rows, int64_t cols, const float* factor,
                 const float* class_inv, int dtype, void* out, float* part, size_t part_floats, hipStream_t st) {
  const bool half = g.p[1] != nullptr;
  DwArgs a{};
  LQ_TRY(fill_segments(a.g, xt, g, depth));
  LQ_TRY(seg_shape(a.g, cols, rows, loss_dw_splits(rows, cols, depth, half)));
  if (a.g.splits > 1 && part_floats < (size_t)a.g.splits * (size_t)rows * (size_t)cols) return LQ_ERR_WORKSPACE;
  if (half != (dtype == LQ_T_FP32) || (half && !class_inv)) return LQ_ERR_ARG;
  a.rows = rows; a.cols = cols; a.factor = factor; a.class_inv = class_inv; a.out = out; a.part = part;
  static LdsLimit limit[2];
  {
    prof::Scope ps(prof::LOSS_ACCUMULATE, st, 2.0 * rows * cols * depth);
    LQ_TRY(dtype == LQ_T_FP32 ? launch_tiles(loss_dw_kernel<_Float16, float>, limit[0], a, st)
                              : launch_tiles(loss_dw_kernel<__bf16, __bf16>, limit[1], a, st));
  }
  if (a.g.splits == 1) return LQ_OK;
  prof::Scope ps(prof::LOSS_ROWS, st, (double)rows * cols * (4.0 * a.g.splits + type_bytes(dtype)));
  const dim3 grid((unsigned)std::min<int64_t>((rows * cols + 255) / 256, 8192));
  if (dtype == LQ_T_BF16)
    hipLaunchKernelGGL(loss_dw_sum_kernel<__bf16>, grid, dim3(256), 0, st, part, a.g.splits, rows * cols, cols, factor,
                       class_inv, static_cast<__bf16*>(out));
  else
    hipLaunchKernelGGL(loss_dw_sum_kernel<float>, grid, dim3(256), 0, st, part, a.g.splits, rows * cols, cols, factor,
                       class_inv, static_cast<float*>(out));
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// Whole rounds of 256 tiles, and what is left over in a product of its own where that is up to a quarter of a round and its reduction
// can be cut into four ranges or more: they fill the chip where the tiles would leave most of it idle for as long as a round takes.
// 1000 x 1024 by 50265 (788 tiles), the whole call, fp32 with six ranges: 1250 us, in one product 1283; bf16 with two: 510, 504.
int launch_loss_dw(const Planes& g, const Planes& xt, int64_t depth, int64_t rows, int64_t cols, const float* factor,
                   const float* class_inv, int dtype, void* out, float* part, size_t part_floats, hipStream_t st) {
  const int64_t across = (cols + SEG_T - 1) / SEG_T, tiles = seg_tiles(rows, cols), main = tiles / 256 * 256 / across * SEG_T;
  const int64_t rest = rows - main;
  if (main <= 0 || rest <= 0 || seg_tiles(rest, cols) > 64 || loss_dw_splits(rest, cols, depth, g.p[1] != nullptr) < 4)
    return dw_of(g, xt, depth, rows, cols, factor, class_inv, dtype, out, part, part_floats, st);
  LQ_TRY(dw_of(g, xt, depth, main, cols, factor, class_inv, dtype, out, part, part_floats, st));
  const Planes tail{{g.p[0] + main * g.pitch, g.p[1] ? g.p[1] + main * g.pitch : nullptr, nullptr}, g.pitch};
  return dw_of(tail, xt, depth, rest, cols, factor, class_inv ? class_inv + main : nullptr, dtype,
               static_cast<char*>(out) + (size_t)main * (size_t)cols * type_bytes(dtype), part, part_floats, st);
}

}  // namespace lq
