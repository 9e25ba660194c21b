// Softmax cross entropy for few rows (up to 128): W is read where it is, as rows for the logits and as columns for dX = E W, by the
// products of thin_device.h; both are bound by that reading (the second out of the memory-side cache where W fits it).  Definitions,
// references and the target's part are those of loss_kernels.hip.  E (n x vocab, one bf16 plane, three for fp32) keeps the power of
// two of its tile of 64 classes, which is one step of the product that reads it: the shift to the row's goes in there.
#include "profiler.h"
#include "thin_device.h"
#include "train.h"

namespace lq {

constexpr float LOG2E = 1.4426950408889634f;

struct FewLogitsArgs {
  ThinSource w; Planes x;
  LossPiece p;
  float* part_ref; float* part_sum;
  uint16_t* e[3]; int64_t e_pitch;
  int steps;
};

// A workgroup owns H tiles of 64 classes, a wavefront 16 of each, and all tokens.  In fp32 X's three planes outweigh W's 64 classes:
// two tiles share them up to 64 tokens (above, their sums would not fit the registers): 50 rows, d = 1024, 50265 classes 62 us, with
// one 66.  One row of bf16, d = 4096, 32000 classes: 44 us, 5.9 TB/s.
template <typename T, int RT> constexpr int few_tiles() { return sizeof(T) == 4 && RT <= 4 ? 2 : 1; }
template <typename T, int RT, bool VEC>
__global__ __launch_bounds__(256) void few_logits_kernel(FewLogitsArgs a) {
  constexpr int NB = thin_planes<T>(), H = few_tiles<T, RT>(), TILE = LOSS_FEW_TILE;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ float s_max[H][4][16 * RT], s_sum[H][4][16 * RT];
  const int wave = threadIdx.x >> 6, l16 = threadIdx.x & 15, kg = (threadIdx.x & 63) >> 4;
  const int64_t tile0 = (int64_t)blockIdx.x * H, class0 = tile0 * TILE + 16 * wave + 4 * kg;         // of this lane's four
  floatx4 acc[H][RT];
  thin_clear(acc);
  thin_rows<T, H, TILE, RT, NB, false, VEC>(a.w, a.x, tile0 * TILE + 16 * wave, 0, a.steps, lds, acc);
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int64_t token = 16 * r + l16;
    const int64_t target = token < a.p.n ? a.p.targets[token] : -1;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      float top = -__builtin_inff();
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t c = class0 + TILE * h + e;
        float x = acc[h][r][e];
        if (c >= a.p.vocab) x = -__builtin_inff();
        else if (c == target) x = -__builtin_inff();      // its logit: when the rows are joined
        acc[h][r][e] = x;
        top = fmaxf(top, x * LOG2E);
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      s_max[h][wave][token] = top;
    }
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < H; ++h) {
    if ((tile0 + h) * TILE >= a.p.vocab) break;          // the same for all of the workgroup
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int64_t token = 16 * r + l16;
      const float ref = ceilf(fmaxf(fmaxf(s_max[h][0][token], s_max[h][1][token]), fmaxf(s_max[h][2][token], s_max[h][3][token])));
      const float from = ref == -__builtin_inff() ? 0.0f : ref;
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[h][r][e] = __builtin_amdgcn_exp2f(fmaf(acc[h][r][e], LOG2E, -from));
        sum += acc[h][r][e];
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      s_sum[h][wave][token] = sum;
      if (wave == 0 && kg == 0 && token < a.p.n) a.part_ref[(tile0 + h) * a.p.n + token] = ref;
      if (a.e[0] && token < a.p.n) {                     // rows of E end on whole tiles
        bf16x2 p0[3], p1[3];
        split_bf16_3(floatx2{acc[h][r][0], acc[h][r][1]}, p0);
        split_bf16_3(floatx2{acc[h][r][2], acc[h][r][3]}, p1);
#pragma unroll
        for (int k = 0; k < NB; ++k)
          *reinterpret_cast<bf16x4*>(a.e[k] + token * a.e_pitch + class0 + TILE * h) = bf16x4{p0[k][0], p0[k][1], p1[k][0], p1[k][1]};
      }
    }
  }
  __syncthreads();
  const int h = threadIdx.x / (16 * RT), token = threadIdx.x % (16 * RT);
  if (h < H && token < a.p.n && (tile0 + h) * TILE < a.p.vocab)
    a.part_sum[(tile0 + h) * a.p.n + token] = (s_sum[h][0][token] + s_sum[h][1][token]) + (s_sum[h][2][token] + s_sum[h][3][token]);
}

static bool rows_fit(const void* W, int64_t ldw, int dtype, int64_t d) {
  return ((uintptr_t)W & 15) == 0 && ldw * type_bytes(dtype) % 16 == 0 && d % 8 == 0;
}

template <typename T, int RT, bool VEC>
static int few_logits(const FewLogitsArgs& a, hipStream_t st) {
  static LdsLimit limit;
  constexpr size_t lds = 2 * ThinStage<RT, thin_planes<T>()>::BYTES;
  constexpr int64_t classes = few_tiles<T, RT>() * LOSS_FEW_TILE;
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(few_logits_kernel<T, RT, VEC>), lds));
  hipLaunchKernelGGL((few_logits_kernel<T, RT, VEC>), dim3((unsigned)((a.p.vocab + classes - 1) / classes)), dim3(256), lds, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}
template <typename T>
static int few_logits_of(const FewLogitsArgs& a, bool vec, hipStream_t st) {
  switch (few_rows(a.p.n)) {
    case 16: return vec ? few_logits<T, 1, true>(a, st) : few_logits<T, 1, false>(a, st);
    case 32: return vec ? few_logits<T, 2, true>(a, st) : few_logits<T, 2, false>(a, st);
    case 64: return vec ? few_logits<T, 4, true>(a, st) : few_logits<T, 4, false>(a, st);
    default: return vec ? few_logits<T, 8, true>(a, st) : few_logits<T, 8, false>(a, st);
  }
}

int launch_few_logits(const void* W, int64_t ldw, int dtype, int64_t d, const Planes& x, const LossPiece& p, float* part_ref,
                      float* part_sum, uint16_t* const e[3], int64_t e_pitch, hipStream_t st) {
  if (p.n > LOSS_FEW || p.v0 != 0 || p.classes != p.vocab || x.pitch < up_to(d, 64) ||
      (e[0] && (e_pitch % LOSS_FEW_TILE || e_pitch < p.vocab)))
    return LQ_ERR_SHAPE;
  FewLogitsArgs a{};
  a.w = ThinSource{W, ldw, p.vocab, d, DropoutMask{}};
  a.x = x; a.p = p; a.part_ref = part_ref; a.part_sum = part_sum;
  for (int k = 0; k < 3; ++k) a.e[k] = e[k];
  a.e_pitch = e_pitch;
  a.steps = (int)((d + 63) / 64);
  prof::Scope ps(prof::LOSS_LOGITS, st, 2.0 * p.n * p.vocab * d);
  const bool vec = rows_fit(W, ldw, dtype, d);
  return dtype == LQ_T_BF16 ? few_logits_of<__bf16>(a, vec, st) : few_logits_of<float>(a, vec, st);
}

// ------------------------------------------------------------------------------------------------
// part[z] (d x tokens) = (E W)^T over a range of classes: a workgroup owns 128 features.  50 rows, d = 1024, 50265 classes, fp32: 64 us,
// 3.2 TB/s, half of which the matrix instructions alone would take (six products for each of W's values).
struct FewDxArgs {
  ThinSource w; Planes e;
  const float* part_ref; const float* ref; int64_t n;
  float* part; int steps, splits;
};

// E's step brought from its tile's power of two to the row's.  A thread brings rows of TOKENS tokens, load q one of token q % TOKENS.
template <int RT, int NB>
struct ShiftStage {
  typedef ThinStage<RT, NB> Stage;
  static constexpr int TOKENS = RT < 2 ? 1 : RT / 2;
  const FewDxArgs& a;
  float to[TOKENS], from[2][TOKENS];
  __device__ __forceinline__ static int token(int i) { return (threadIdx.x / 8 + 32 * i) % (16 * RT); }
  __device__ __forceinline__ explicit ShiftStage(const FewDxArgs& args) : a(args) {
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) {
      to[i] = token(i) < a.n ? a.ref[token(i)] : 0.0f;
      if (to[i] == -__builtin_inff()) to[i] = 0.0f;
    }
  }
  template <class P>
  __device__ __forceinline__ void load(P, int step) {
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) from[P::value][i] = token(i) < a.n ? a.part_ref[(int64_t)step * a.n + token(i)] : 0.0f;
  }
  template <class P>
  __device__ __forceinline__ void operator()(P, Stage& s) {
    float f[TOKENS];
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) f[i] = __builtin_amdgcn_exp2f(from[P::value][i] - to[i]);
#pragma unroll
    for (int q = 0; q < Stage::LOADS; ++q) {
      bf16x8 v = __builtin_bit_cast(bf16x8, s.r[q]);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = (__bf16)((float)v[j] * f[q % TOKENS]);
      s.r[q] = __builtin_bit_cast(uintx4, v);
    }
  }
};

template <typename T, int RT, bool VEC>
__global__ __launch_bounds__(256, (thin_columns_waves<T, RT>())) void few_dx_kernel(FewDxArgs a) {
  constexpr int NB = thin_planes<T>();
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int64_t c0 = (int64_t)blockIdx.x * 128;
  const int s0 = (int)((int64_t)a.steps * blockIdx.y / a.splits), s1 = (int)((int64_t)a.steps * (blockIdx.y + 1) / a.splits);
  floatx4 acc[2][RT];
  thin_clear(acc);
  if (s0 < s1) thin_columns<T, RT, NB, false, VEC>(a.w, a.e, c0, s0, s1, lds, acc, ShiftStage<RT, NB>(a));
  thin_store(acc, a.part + (size_t)blockIdx.y * (size_t)a.w.K * (16 * RT), c0 + 32 * (threadIdx.x >> 6), a.w.K);
}

// dX_i = g (1 - p_t) (E W / S - w_t) from the ranges' parts: 16 features x 16 tokens a workgroup, turned in LDS.
struct FewSumArgs {
  const float* part; int splits, tokens; int64_t n, d, vocab;
  LossRows r; const int64_t* targets; const float* factors; int64_t ldw;
};
template <typename T>
__global__ __launch_bounds__(256) void few_dx_sum_kernel(FewSumArgs a, const T* __restrict__ W, T* __restrict__ dX) {
  __shared__ float s_t[16][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  const size_t stride = (size_t)a.d * a.tokens;
  const int64_t row = (int64_t)blockIdx.x * 16 + r;
  float v = 0.0f;
  if (row < a.d) {
    const float* from = a.part + row * a.tokens + blockIdx.y * 16 + c;
#pragma unroll 16
    for (int s = 0; s < a.splits; ++s) v += from[s * stride];
  }
  s_t[r][c] = v;
  __syncthreads();
  const int64_t col = (int64_t)blockIdx.x * 16 + c, token = (int64_t)blockIdx.y * 16 + r;
  if (token >= a.n || col >= a.d) return;
  const int64_t t = a.targets[token];
  const bool counts = t >= 0 && t < a.vocab;
  const float s = a.r.sum[token], inv = s == 0.0f ? 0.0f : 1.0f / s;         // no other class: the sums are zero
  dX[token * a.d + col] = counts ? (T)(a.r.wrong[token] * a.factors[0] * (s_t[c][r] * inv - (float)W[t * a.ldw + col])) : (T)0.0f;
}

// As many ranges as give every CU two workgroups, each with four steps: 50 rows, d = 1024, 50265 classes, fp32, the whole call 157 us,
// with one workgroup a CU 160, with four 167.
int few_dx_splits(int64_t vocab, int64_t d) {
  const int64_t wgs = (d + 127) / 128, steps = (vocab + 63) / 64;
  return (int)std::max<int64_t>(1, std::min<int64_t>({(512 + wgs - 1) / wgs, steps / 4, 64}));
}

template <typename T, int RT, bool VEC>
static int few_dx(const FewDxArgs& a, dim3 grid, hipStream_t st) {
  static LdsLimit limit;
  constexpr size_t lds = thin_columns_lds<T, RT, thin_planes<T>()>();
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(few_dx_kernel<T, RT, VEC>), lds));
  hipLaunchKernelGGL((few_dx_kernel<T, RT, VEC>), grid, dim3(256), lds, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}
template <typename T>
static int few_dx_of(const FewDxArgs& a, bool vec, dim3 grid, hipStream_t st) {
  switch (few_rows(a.n)) {
    case 16: return vec ? few_dx<T, 1, true>(a, grid, st) : few_dx<T, 1, false>(a, grid, st);
    case 32: return vec ? few_dx<T, 2, true>(a, grid, st) : few_dx<T, 2, false>(a, grid, st);
    case 64: return vec ? few_dx<T, 4, true>(a, grid, st) : few_dx<T, 4, false>(a, grid, st);
    default: return vec ? few_dx<T, 8, true>(a, grid, st) : few_dx<T, 8, false>(a, grid, st);
  }
}

int launch_few_dx(const void* W, int64_t ldw, int dtype, int64_t d, const Planes& e, const LossPiece& p, const LossRows& r,
                  const float* part_ref, const float* factors, float* part, void* dX, hipStream_t st) {
  if (p.n > LOSS_FEW || e.pitch % 64 || e.pitch < p.vocab) return LQ_ERR_SHAPE;
  FewDxArgs a{};
  a.w = ThinSource{W, ldw, p.vocab, d, DropoutMask{}};
  a.e = e; a.part_ref = part_ref; a.ref = r.ref; a.n = p.n; a.part = part;
  a.steps = (int)((p.vocab + 63) / 64);
  a.splits = few_dx_splits(p.vocab, d);
  const dim3 grid((unsigned)((d + 127) / 128), (unsigned)a.splits);
  {
    prof::Scope ps(prof::LOSS_ACCUMULATE, st, 2.0 * p.n * p.vocab * d);
    const bool vec = rows_fit(W, ldw, dtype, d);
    LQ_TRY(dtype == LQ_T_BF16 ? few_dx_of<__bf16>(a, vec, grid, st) : few_dx_of<float>(a, vec, grid, st));
  }
  const FewSumArgs s{part, a.splits, (int)few_rows(p.n), p.n, d, p.vocab, r, p.targets, factors, ldw};
  const dim3 sums((unsigned)((d + 15) / 16), (unsigned)((p.n + 15) / 16));
  prof::Scope ps(prof::LOSS_ROWS, st, (double)p.n * d * (4.0 * a.splits + type_bytes(dtype)));
  if (dtype == LQ_T_BF16)
    hipLaunchKernelGGL(few_dx_sum_kernel<__bf16>, sums, dim3(256), 0, st, s, static_cast<const __bf16*>(W), static_cast<__bf16*>(dX));
  else
    hipLaunchKernelGGL(few_dx_sum_kernel<float>, sums, dim3(256), 0, st, s, static_cast<const float*>(W), static_cast<float*>(dX));
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
