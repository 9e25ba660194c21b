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

template <typename T, int RT>
__global__ __launch_bounds__(256) void thin_project_kernel(ProjectArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int64_t row0 = (int64_t)blockIdx.x * 128 + 32 * (threadIdx.x >> 6);
  const int s0 = (int)((int64_t)a.steps * blockIdx.y / a.splits), s1 = (int)((int64_t)a.steps * (blockIdx.y + 1) / a.splits);
  floatx4 acc[2][RT];
  thin_clear(acc);
  if (s0 < s1) thin_rows<T, 2, RT, 3, true, true>(a.a, a.b, row0, s0, s1, lds, acc);
  thin_store(acc, a.part + (size_t)blockIdx.y * (size_t)a.a.m * (16 * RT), row0, a.a.m);
}

// As many ranges as leave two workgroups a CU, each with two steps.
int thin_project_splits(int64_t m, int64_t K) {
  const int64_t wgs = (m + 127) / 128, steps = (K + 63) / 64;
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / wgs, steps / 2, 16}));
}

template <typename T, int RT>
static int project(const ProjectArgs& a, dim3 grid, hipStream_t st) {
  static LdsLimit limit;
  constexpr size_t lds = 2 * ThinStage<RT, 3>::BYTES;
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(thin_project_kernel<T, RT>), lds));
  hipLaunchKernelGGL((thin_project_kernel<T, RT>), grid, dim3(256), lds, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}
template <typename T>
static int project_of(const ProjectArgs& a, int r32, dim3 grid, hipStream_t st) {
  switch (r32 / 32) {
    case 1: return project<T, 2>(a, grid, st);
    case 2: return project<T, 4>(a, grid, st);
    case 3: return project<T, 6>(a, grid, st);
    default: return project<T, 8>(a, grid, st);
  }
}

int launch_thin_project(const void* A, int dtype, int64_t m, int64_t K, const Planes& b, int r32, const DropoutMask& d, float* part,
                        hipStream_t st) {
  if (K < 8 || K % 8 || m < 1 || r32 < 32 || r32 % 32 || r32 > ADAPTER_MAX_RANK || b.pitch % 64 || b.pitch < K) return LQ_ERR_SHAPE;
  const ProjectArgs a{ThinSource{A, K, m, K, d}, b, part, (int)((K + 63) / 64), thin_project_splits(m, K)};
  const dim3 grid((unsigned)((m + 127) / 128), (unsigned)a.splits);
  prof::Scope ps(prof::THIN_PROJECT, st, (double)m * K * type_bytes(dtype));
  return dtype == LQ_T_BF16 ? project_of<__bf16>(a, r32, grid, st) : project_of<float>(a, r32, grid, st);
}

// ------------------------------------------------------------------------------------------------
struct FinishArgs {
  const float* part; int splits; int64_t m; int rank, r32; float scale;
  float* T; PlaneTarget rows, cols;
};

// A workgroup finishes 16 rows x 32 columns of T, two values a thread with their ranges' loads under way together; the transposed
// planes go through LDS.
__global__ __launch_bounds__(256) void thin_finish_kernel(FinishArgs a) {
  __shared__ float s_t[16][33];
  const int c = threadIdx.x & 31, col = blockIdx.y * 32 + c;
  const size_t stride = (size_t)a.m * (size_t)a.r32;
  float v[2] = {0.0f, 0.0f};
  int64_t row[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) row[q] = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 5) + 8 * q;
  if (col < a.r32) {
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s)
#pragma unroll
      for (int q = 0; q < 2; ++q)
        if (row[q] < a.m) v[q] += a.part[s * stride + row[q] * a.r32 + col];
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const float f = v[q] * a.scale;
    s_t[(threadIdx.x >> 5) + 8 * q][c] = f;
    if (row[q] >= a.m) continue;
    if (a.T && col < a.rank) a.T[row[q] * a.rank + col] = f;
    bf16x2 p[3];
    split_bf16_3(floatx2{f, 0.0f}, p);
#pragma unroll
    for (int k = 0; k < 3; ++k) a.rows.p[k][row[q] * a.rows.pitch + col] = __builtin_bit_cast(uint16_t, p[k][0]);
  }
  if (!a.cols.p[0] || (int)blockIdx.y * 32 >= a.r32) return;
  __syncthreads();
  const int pair = threadIdx.x & 7, k = threadIdx.x >> 3;
  bf16x2 p[3];
  split_bf16_3(floatx2{s_t[2 * pair][k], s_t[2 * pair + 1][k]}, p);
  const int64_t at = (int64_t)(blockIdx.y * 32 + k) * a.cols.pitch + (int64_t)blockIdx.x * 16 + 2 * pair;
#pragma unroll
  for (int j = 0; j < 3; ++j) *reinterpret_cast<bf16x2*>(a.cols.p[j] + at) = p[j];
}

int launch_thin_finish(const float* part, int splits, int64_t m, int rank, int r32, float scale, float* T, const PlaneTarget& rows,
                       const PlaneTarget& cols, hipStream_t st) {
  if ((cols.p[0] && (cols.pitch % 64 || cols.pitch < up_to(m, 64))) || !rows.p[0] || rows.pitch != up_to(r32, 64)) return LQ_ERR_SHAPE;
  const FinishArgs a{part, splits, m, rank, r32, scale, T, rows, cols};
  prof::Scope ps(prof::THIN_FINISH, st, (double)m * r32 * 4.0 * (splits + 2));
  // the row planes are written to their full pitch, the transposed ones up to a multiple of 64 rows
  hipLaunchKernelGGL(thin_finish_kernel, dim3((unsigned)(up_to(m, 64) / 16), (unsigned)(rows.pitch / 32)), dim3(256), 0, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// part[z] (K x r32) = drop(A)^T B over a range of rows, in steps of 64, for two products in one launch.  A workgroup owns 128 columns
// of A, a wavefront 32.
struct GramArgs {
  ThinSource a[2]; Planes bt[2];
  float* part[2]; int splits[2]; int wgs0;
  int steps;
};

template <typename T, int RT>
__global__ __launch_bounds__(256, (thin_columns_waves<T, RT>())) void thin_gram_kernel(GramArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int which = (int)blockIdx.x >= a.wgs0, wg = blockIdx.x - (which ? a.wgs0 : 0);
  const ThinSource& src = a.a[which];
  const int splits = a.splits[which], split = wg % splits;
  const int64_t c0 = (int64_t)(wg / splits) * 128;
  const int s0 = (int)((int64_t)a.steps * split / splits), s1 = (int)((int64_t)a.steps * (split + 1) / splits);
  floatx4 acc[2][RT];
  thin_clear(acc);
  if (s0 < s1) thin_columns<T, RT, 3, true, true>(src, a.bt[which], c0, s0, s1, lds, acc, KeepStage{});
  thin_store(acc, a.part[which] + (size_t)split * (size_t)src.K * (16 * RT), c0 + 32 * (threadIdx.x >> 6), src.K);
}

// The sums over the ranges: 32 rows x 32 columns a workgroup; the first product's result is turned.
struct GramSumArgs { const float* part[2]; int parts[2]; int64_t K[2]; int64_t wgs0; int rank, r32; float scale; float* out[2]; };
__global__ __launch_bounds__(256) void thin_gram_sum_kernel(GramSumArgs a) {
  __shared__ float s_t[32][33];
  const int which = (int64_t)blockIdx.x >= a.wgs0;
  const int64_t row0 = ((int64_t)blockIdx.x - (which ? a.wgs0 : 0)) * 32, K = a.K[which];
  const int c = threadIdx.x & 31, r0 = threadIdx.x >> 5, col = blockIdx.y * 32 + c, parts = a.parts[which];
  const size_t stride = (size_t)K * a.r32;
  const float* part = a.part[which];
  float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = 0; s < parts; ++s)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (row0 + r0 + 8 * q < K) v[q] += part[s * stride + (row0 + r0 + 8 * q) * a.r32 + col];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t row = row0 + r0 + 8 * q;
    if (which) { if (row < K && col < a.rank) a.out[1][row * a.rank + col] = v[q] * a.scale; }
    else s_t[r0 + 8 * q][c] = v[q];
  }
  if (which) return;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int k = r0 + 8 * q;
    if (row0 + c < K && (int)(blockIdx.y * 32 + k) < a.rank) a.out[0][(int64_t)(blockIdx.y * 32 + k) * K + row0 + c] = s_t[c][k];
  }
}

// As many ranges as leave two workgroups a CU for the pair of products, each with four steps.
int thin_gram_splits(int64_t m, int64_t K, int64_t other) {
  const int64_t wgs = (K + 127) / 128 + (other + 127) / 128, steps = (m + 63) / 64;
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / wgs, steps / 4, 16}));
}

template <typename T, int RT>
static int gram(const GramArgs& a, dim3 grid, hipStream_t st) {
  static LdsLimit limit;
  constexpr size_t lds = thin_columns_lds<T, RT, 3>();
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(thin_gram_kernel<T, RT>), lds));
  hipLaunchKernelGGL((thin_gram_kernel<T, RT>), grid, dim3(256), lds, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}
template <typename T>
static int gram_of(const GramArgs& a, int r32, dim3 grid, hipStream_t st) {
  switch (r32 / 32) {
    case 1: return gram<T, 2>(a, grid, st);
    case 2: return gram<T, 4>(a, grid, st);
    case 3: return gram<T, 6>(a, grid, st);
    default: return gram<T, 8>(a, grid, st);
  }
}

int launch_thin_grams(const void* dY, int64_t k, const Planes& tt, float* dL2, const void* X, int64_t d, const Planes& ut,
                      const DropoutMask& mask, float* dL1, int dtype, int64_t m, int rank, int r32, float* part, hipStream_t st) {
  if (k < 8 || k % 8 || d < 8 || d % 8 || m < 1 || r32 < 32 || r32 % 32 || r32 > ADAPTER_MAX_RANK || tt.pitch % 64 ||
      ut.pitch % 64 || tt.pitch < up_to(m, 64) || ut.pitch < up_to(m, 64))
    return LQ_ERR_SHAPE;
  const int splits = thin_gram_splits(m, k, d);
  float* part1 = part + (size_t)splits * (size_t)k * r32;
  const int64_t wgs0 = (k + 127) / 128 * splits, wgs1 = (d + 127) / 128 * splits;
  const GramArgs a{{ThinSource{dY, k, m, k, DropoutMask{}}, ThinSource{X, d, m, d, mask}}, {tt, ut}, {part, part1}, {splits, splits},
                   (int)wgs0, (int)((m + 63) / 64)};
  {
    prof::Scope ps(prof::THIN_GRAM, st, (double)m * (k + d) * type_bytes(dtype));
    const dim3 grid((unsigned)(wgs0 + wgs1));
    LQ_TRY(dtype == LQ_T_BF16 ? gram_of<__bf16>(a, r32, grid, st) : gram_of<float>(a, r32, grid, st));
  }
  const int64_t sums0 = (k + 31) / 32, sums1 = (d + 31) / 32;
  const GramSumArgs g{{part, part1}, {splits, splits}, {k, d}, sums0, rank, r32, mask.scale, {dL2, dL1}};
  prof::Scope ps(prof::THIN_FINISH, st, (double)(k + d) * r32 * 4.0 * (splits + 1));
  hipLaunchKernelGGL(thin_gram_sum_kernel, dim3((unsigned)(sums0 + sums1), (unsigned)(r32 / 32)), dim3(256), 0, st, g);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
