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
// part[z] = drop(A) B^T over a range of the reduction, in steps of 64.  A workgroup owns 128 rows, a wavefront 32.  4096 x 11008 bf16
// by 64: 31 us, 2.9 TB/s: three planes of B for one of A make the LDS reads and matrix instructions of B's operands the larger part.
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
  if (s0 < s1) thin_rows<T, 2, 16, RT, 3, true, true>(a.a, a.b, row0, s0, s1, lds, acc);
  thin_store(acc, a.part + (size_t)blockIdx.y * (size_t)a.a.m * (16 * RT), row0, a.a.m);
}

// As many ranges as give every CU a workgroup, each with two steps.  The whole call, 4096 x 4096, 4096 features, bf16: 145 us, with two
// workgroups a CU 151.
int thin_project_splits(int64_t m, int64_t K) {
  const int64_t wgs = (m + 127) / 128, steps = (K + 63) / 64;
  return (int)std::max<int64_t>(1, std::min<int64_t>({256 / wgs, steps / 2, 16}));
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
// part[z] (K x r32) = drop(A)^T B over a range of rows, in steps of 64, for two products in one launch.  A workgroup owns 128 columns
// of A, a wavefront 32.  4096 rows of 4096 and 11008 columns, bf16, rank 64: 50 us, 2.5 TB/s.
struct GramArgs {
  ThinSource a[2]; Planes bt[2];
  float* part[2]; int splits[2]; int wgs0;
  int steps;
  int rank; float scale; float* out[2];
};

// One range is the whole: the first product's result is turned, the second's is scaled.
template <int RT>
__device__ __forceinline__ void gram_store(const GramArgs& a, int which, const floatx4 (&acc)[2][RT], int64_t row0) {
  const int l16 = threadIdx.x & 15, kg = (threadIdx.x & 63) >> 4;
  const int64_t K = a.a[which].K;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t o = row0 + 16 * h + 4 * kg;          // of four neighbours: K is a multiple of eight
    if (o >= K) continue;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int col = 16 * r + l16;
      if (col >= a.rank) continue;
      if (which == 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) a.out[0][col * K + o + e] = acc[h][r][e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) a.out[1][(o + e) * a.rank + col] = acc[h][r][e] * a.scale;
      }
    }
  }
}

template <typename T, int RT>
__global__ __launch_bounds__(256, (thin_columns_waves<T, RT>())) void thin_gram_kernel(GramArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int which = (int)blockIdx.x >= a.wgs0, wg = blockIdx.x - (which ? a.wgs0 : 0);
  const ThinSource src = which ? a.a[1] : a.a[0];     // copies: else their fields are loaded again and again in the loop
  const Planes bt = which ? a.bt[1] : a.bt[0];
  const int splits = a.splits[which], split = wg % splits;
  const int64_t c0 = (int64_t)(wg / splits) * 128;
  const int s0 = (int)((int64_t)a.steps * split / splits), s1 = (int)((int64_t)a.steps * (split + 1) / splits);
  floatx4 acc[2][RT];
  thin_clear(acc);
  if (s0 < s1) thin_columns<T, RT, 3, true, true>(src, bt, c0, s0, s1, lds, acc, KeepStage{});
  const int64_t row0 = c0 + 32 * (threadIdx.x >> 6);
  if (splits == 1) gram_store(a, which, acc, row0);
  else thin_store(acc, a.part[which] + (size_t)split * (size_t)src.K * (16 * RT), row0, src.K);
}

// As many ranges as give every CU two workgroups for the pair of products, each with eight steps.  4096 rows of 4096 and 11008, bf16,
// the whole call: 394 us, with one workgroup a CU 406; 1000 rows, fp32: 378 us, with four steps a range 386.
int thin_gram_splits(int64_t m, int64_t K, int64_t other) {
  const int64_t wgs = (K + 127) / 128 + (other + 127) / 128, steps = (m + 63) / 64;
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / wgs, steps / 8, 16}));
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
                      const DropoutMask& mask, float* dL1, int dtype, int64_t m, int rank, int r32, float* part, ThinGramSum* sum,
                      hipStream_t st) {
  if (k < 8 || k % 8 || d < 8 || d % 8 || m < 1 || r32 < 32 || r32 % 32 || r32 > ADAPTER_MAX_RANK || tt.pitch % 64 ||
      ut.pitch % 64 || tt.pitch < up_to(m, 64) || ut.pitch < up_to(m, 64))
    return LQ_ERR_SHAPE;
  const int splits = thin_gram_splits(m, k, d);
  float* part1 = part + (size_t)splits * (size_t)k * r32;
  const int64_t wgs0 = (k + 127) / 128 * splits, wgs1 = (d + 127) / 128 * splits;
  const GramArgs a{{ThinSource{dY, k, m, k, DropoutMask{}}, ThinSource{X, d, m, d, mask}}, {tt, ut}, {part, part1}, {splits, splits},
                   (int)wgs0, (int)((m + 63) / 64), rank, mask.scale, {dL2, dL1}};
  {
    prof::Scope ps(prof::THIN_GRAM, st, (double)m * (k + d) * type_bytes(dtype));
    const dim3 grid((unsigned)(wgs0 + wgs1));
    LQ_TRY(dtype == LQ_T_BF16 ? gram_of<__bf16>(a, r32, grid, st) : gram_of<float>(a, r32, grid, st));
  }
  *sum = ThinGramSum{{part, part1}, splits, {k, d}, rank, r32, mask.scale, {dL2, dL1}};
  return LQ_OK;
}

}  // namespace lq
