// The thin products of a decomposed layer in training (rank at most 128):  T = drop(X) L1,  U = dY L2^T,  dL1 = drop(X)^T U,
// dL2 = T^T dY.  They read X or dY once and are bound by that and by the operands of the other side, which every workgroup reads.
// The mask is worked out where an element is loaded (the eight neighbours that share a call of the generator are what a lane loads).
// Their results are fp32 whatever the type of X: L1, L2, T and U go in as three bf16 planes, X and dY as one where they are bf16
// and three where they are fp32.
#include "profiler.h"
#include "thin_device.h"
#include "train.h"

namespace lq {

// ------------------------------------------------------------------------------------------------
// part[z] = drop(A) B^T over a range of the reduction, in steps of 64.  A workgroup owns 128 rows, a wavefront 32.
struct ProjectArgs {
  ThinSource a; Planes b;
  float* part; int steps, splits;
};

template <typename T, int RT, bool DROP>
__global__ __launch_bounds__(256) void thin_project_kernel(ProjectArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int64_t row0 = (int64_t)blockIdx.x * 128 + 32 * (threadIdx.x >> 6);
  const int s0 = (int)((int64_t)a.steps * blockIdx.y / a.splits), s1 = (int)((int64_t)a.steps * (blockIdx.y + 1) / a.splits);
  floatx4 acc[2][RT];
  thin_clear(acc);
  if (s0 < s1) thin_rows<T, 2, RT, 3, DROP, true>(a.a, a.b, row0, s0, s1, lds, acc);
  thin_store(acc, a.part + (size_t)blockIdx.y * (size_t)a.a.m * (16 * RT), row0, a.a.m);
}

// Two workgroups a CU; a range keeps four steps.
int thin_project_splits(int64_t m, int64_t K) {
  const int64_t wgs = (m + 127) / 128, steps = (K + 63) / 64;
  return (int)std::max<int64_t>(1, std::min<int64_t>({(512 + wgs - 1) / wgs, steps / 4, 32}));
}

template <typename T, int RT, bool DROP>
static int project(const ProjectArgs& a, dim3 grid, hipStream_t st) {
  static LdsLimit limit;
  constexpr size_t lds = 2 * ThinStage<RT, 3>::BYTES;
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(thin_project_kernel<T, RT, DROP>), lds));
  hipLaunchKernelGGL((thin_project_kernel<T, RT, DROP>), grid, dim3(256), lds, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}
template <typename T>
static int project_of(const ProjectArgs& a, int r32, bool drop, dim3 grid, hipStream_t st) {
  switch (r32 / 32 + (drop ? 4 : 0)) {
    case 1: return project<T, 2, false>(a, grid, st);
    case 2: return project<T, 4, false>(a, grid, st);
    case 3: return project<T, 6, false>(a, grid, st);
    case 4: return project<T, 8, false>(a, grid, st);
    case 5: return project<T, 2, true>(a, grid, st);
    case 6: return project<T, 4, true>(a, grid, st);
    case 7: return project<T, 6, true>(a, grid, st);
    default: return project<T, 8, true>(a, grid, st);
  }
}

int launch_thin_project(const void* A, int dtype, int64_t m, int64_t K, const Planes& b, int r32, const DropoutMask* d, float* part,
                        hipStream_t st) {
  if (K < 8 || K % 8 || m < 1 || r32 < 32 || r32 % 32 || r32 > ADAPTER_MAX_RANK || b.pitch % 64 || b.pitch < K) return LQ_ERR_SHAPE;
  ProjectArgs a{};
  a.a = ThinSource{A, K, m, K, d ? *d : DropoutMask{}};
  a.b = b; a.part = part;
  a.steps = (int)((K + 63) / 64);
  a.splits = thin_project_splits(m, K);
  const dim3 grid((unsigned)((m + 127) / 128), (unsigned)a.splits);
  prof::Scope ps(prof::THIN_PROJECT, st, (double)m * K * type_bytes(dtype));
  return dtype == LQ_T_BF16 ? project_of<__bf16>(a, r32, d != nullptr, grid, st) : project_of<float>(a, r32, d != nullptr, grid, st);
}

// ------------------------------------------------------------------------------------------------
struct FinishArgs {
  const float* part; int splits; int64_t m; int rank, r32; float scale;
  float* T; PlaneTarget rows, cols;
};

// A workgroup finishes 64 rows x 32 columns of T; the transposed planes go through LDS.
__global__ __launch_bounds__(256) void thin_finish_kernel(FinishArgs a) {
  __shared__ float s_t[64][33];
  const int c = threadIdx.x & 31, r0 = threadIdx.x >> 5, col = blockIdx.y * 32 + c;
  const size_t stride = (size_t)a.m * (size_t)a.r32;
  float v[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const int64_t row = (int64_t)blockIdx.x * 64 + r0 + 8 * q;
    v[q] = 0.0f;
    if (a.splits == 0 && row < a.m && col < a.rank) v[q] = a.part[row * a.rank + col];
  }
  for (int s = 0; s < a.splits; ++s)
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int64_t row = (int64_t)blockIdx.x * 64 + r0 + 8 * q;
      if (row < a.m && col < a.r32) v[q] += a.part[s * stride + row * a.r32 + col];
    }
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const int r = r0 + 8 * q;
    const int64_t row = (int64_t)blockIdx.x * 64 + r;
    const float f = a.splits == 0 ? v[q] : v[q] * a.scale;
    s_t[r][c] = f;
    if (row >= a.m) continue;
    if (a.T && col < a.rank) a.T[row * a.rank + col] = f;
    if (a.rows.p[0]) {
      bf16x2 p[3];
      split_bf16_3(floatx2{f, 0.0f}, p);
#pragma unroll
      for (int k = 0; k < 3; ++k) a.rows.p[k][row * a.rows.pitch + col] = __builtin_bit_cast(uint16_t, p[k][0]);
    }
  }
  if (!a.cols.p[0] || (int)blockIdx.y * 32 >= a.r32) return;
  __syncthreads();
  const int pair = threadIdx.x & 31;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int k = (threadIdx.x >> 5) + 8 * q;
    bf16x2 p[3];
    split_bf16_3(floatx2{s_t[2 * pair][k], s_t[2 * pair + 1][k]}, p);
    const int64_t at = (int64_t)(blockIdx.y * 32 + k) * a.cols.pitch + (int64_t)blockIdx.x * 64 + 2 * pair;
#pragma unroll
    for (int j = 0; j < 3; ++j) *reinterpret_cast<bf16x2*>(a.cols.p[j] + at) = p[j];
  }
}

int launch_thin_finish(const float* part, int splits, int64_t m, int rank, int r32, float scale, float* T, const PlaneTarget& rows,
                       const PlaneTarget& cols, hipStream_t st) {
  if ((cols.p[0] && (cols.pitch % 64 || cols.pitch < up_to(m, 64))) || (rows.p[0] && rows.pitch != up_to(r32, 64))) return LQ_ERR_SHAPE;
  const FinishArgs a{part, splits, m, rank, r32, scale, T, rows, cols};
  const int64_t width = rows.p[0] ? rows.pitch : r32;              // the row planes are written to their full pitch
  prof::Scope ps(prof::THIN_FINISH, st, (double)m * r32 * 4.0 * (splits + 2));
  hipLaunchKernelGGL(thin_finish_kernel, dim3((unsigned)((m + 63) / 64), (unsigned)(width / 32)), dim3(256), 0, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// part[z] (K x r32) = drop(A)^T B over a range of rows, in steps of 64.  A workgroup owns 128 columns of A, a wavefront 32.
struct GramArgs {
  ThinSource a; Planes bt;
  float* part; int steps, splits;
};

template <typename T, int RT, bool DROP>
__global__ __launch_bounds__(256) void thin_gram_kernel(GramArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int64_t c0 = (int64_t)blockIdx.x * 128;
  const int s0 = (int)((int64_t)a.steps * blockIdx.y / a.splits), s1 = (int)((int64_t)a.steps * (blockIdx.y + 1) / a.splits);
  floatx4 acc[2][RT];
  thin_clear(acc);
  if (s0 < s1) thin_columns<T, RT, 3, DROP, true>(a.a, a.bt, c0, s0, s1, lds, acc, KeepStage{});
  thin_store(acc, a.part + (size_t)blockIdx.y * (size_t)a.a.K * (16 * RT), c0 + 32 * (threadIdx.x >> 6), a.a.K);
}

struct GramSumArgs { const float* part; int parts; int64_t K; int rank, r32; float scale; int transposed; float* out; };
__global__ __launch_bounds__(256) void thin_gram_sum_kernel(GramSumArgs a) {
  __shared__ float s_t[64][33];
  const int c = threadIdx.x & 31, r0 = threadIdx.x >> 5, col = blockIdx.y * 32 + c;
  const size_t stride = (size_t)a.K * a.r32;
  float v[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = 0.0f;
  for (int s = 0; s < a.parts; ++s)
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int64_t row = (int64_t)blockIdx.x * 64 + r0 + 8 * q;
      if (row < a.K) v[q] += a.part[s * stride + row * a.r32 + col];
    }
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const int64_t row = (int64_t)blockIdx.x * 64 + r0 + 8 * q;
    const float f = v[q] * a.scale;
    s_t[r0 + 8 * q][c] = f;
    if (!a.transposed && row < a.K && col < a.rank) a.out[row * a.rank + col] = f;
  }
  if (!a.transposed) return;
  __syncthreads();
  const int r = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 64 + r;
  for (int k = threadIdx.x >> 6; k < 32; k += 4)
    if (row < a.K && (int)(blockIdx.y * 32 + k) < a.rank) a.out[(int64_t)(blockIdx.y * 32 + k) * a.K + row] = s_t[r][k];
}

int thin_gram_splits(int64_t m, int64_t K) {
  const int64_t wgs = (K + 127) / 128, steps = (m + 63) / 64;
  return (int)std::max<int64_t>(1, std::min<int64_t>({(512 + wgs - 1) / wgs, (steps + 3) / 4, 32}));
}

template <typename T, int RT, bool DROP>
static int gram(const GramArgs& a, dim3 grid, hipStream_t st) {
  static LdsLimit limit;
  constexpr size_t lds = thin_columns_lds<T, RT, 3>();
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(thin_gram_kernel<T, RT, DROP>), lds));
  hipLaunchKernelGGL((thin_gram_kernel<T, RT, DROP>), grid, dim3(256), lds, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}
template <typename T>
static int gram_of(const GramArgs& a, int r32, bool drop, dim3 grid, hipStream_t st) {
  switch (r32 / 32 + (drop ? 4 : 0)) {
    case 1: return gram<T, 2, false>(a, grid, st);
    case 2: return gram<T, 4, false>(a, grid, st);
    case 3: return gram<T, 6, false>(a, grid, st);
    case 4: return gram<T, 8, false>(a, grid, st);
    case 5: return gram<T, 2, true>(a, grid, st);
    case 6: return gram<T, 4, true>(a, grid, st);
    case 7: return gram<T, 6, true>(a, grid, st);
    default: return gram<T, 8, true>(a, grid, st);
  }
}

int launch_thin_gram(const void* A, int dtype, int64_t m, int64_t K, const Planes& bt, int rank, int r32, const DropoutMask* d,
                     float scale, bool transposed, float* part, float* out, hipStream_t st) {
  if (K < 8 || K % 8 || m < 1 || r32 < 32 || r32 % 32 || r32 > ADAPTER_MAX_RANK || bt.pitch % 64 || bt.pitch < up_to(m, 64))
    return LQ_ERR_SHAPE;
  GramArgs a{};
  a.a = ThinSource{A, K, m, K, d ? *d : DropoutMask{}};
  a.bt = bt; a.part = part;
  a.steps = (int)((m + 63) / 64);
  a.splits = thin_gram_splits(m, K);
  const dim3 grid((unsigned)((K + 127) / 128), (unsigned)a.splits);
  {
    prof::Scope ps(prof::THIN_GRAM, st, (double)m * K * type_bytes(dtype));
    LQ_TRY(dtype == LQ_T_BF16 ? gram_of<__bf16>(a, r32, d != nullptr, grid, st) : gram_of<float>(a, r32, d != nullptr, grid, st));
  }
  const GramSumArgs g{part, a.splits, K, rank, r32, scale, (int)transposed, out};
  prof::Scope ps(prof::THIN_FINISH, st, (double)K * r32 * 4.0 * (g.parts + 1));
  hipLaunchKernelGGL(thin_gram_sum_kernel, dim3((unsigned)((K + 63) / 64), (unsigned)(r32 / 32)), dim3(256), 0, st, g);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
