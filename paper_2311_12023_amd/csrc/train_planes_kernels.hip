// Operands of the training operators as 16-bit planes: rows as they are, or transposed, so that the reduction index of the product
// that reads them is contiguous.  All passes are bound by the bytes they move (50265 x 1024 fp32 into two planes: 61 us, 6.7 TB/s, the
// source out of the memory-side cache; its largest magnitude: 54 us, 3.8 TB/s).
#include "half_planes_device.h"
#include "mfma_device.h"
#include "profiler.h"
#include "train.h"

namespace lq {

// Eight values of a row from column c on, zero beyond `cols`.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* __restrict__ row, int64_t c, int64_t cols, float (&v)[8]) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  if (VEC && c + 8 <= cols) {
    const vec8 in = *reinterpret_cast<const vec8*>(row + c);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)in[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? (float)row[c + j] : 0.0f;
  }
}

template <int KIND>
constexpr int plane_count() { return KIND == PLANE_BF16 ? 1 : KIND == PLANE_HALF_2 ? 2 : 3; }

// Two neighbours as they lie in each plane.
template <int KIND>
__device__ __forceinline__ void split_pair(float a, float b, float scale, uint32_t (&w)[3]) {
  if constexpr (KIND == PLANE_HALF_2) {
    const HalfPair p = split_half(a * scale), q = split_half(b * scale);
    typedef _Float16 half2 __attribute__((ext_vector_type(2)));
    w[0] = __builtin_bit_cast(uint32_t, half2{p.hi, q.hi});
    w[1] = __builtin_bit_cast(uint32_t, half2{p.lo, q.lo});
  } else {
    bf16x2 p[3];
    split_bf16_3(floatx2{a, b}, p);
#pragma unroll
    for (int k = 0; k < 3; ++k) w[k] = __builtin_bit_cast(uint32_t, p[k]);
  }
}

struct RowArgs {
  const void* src; int64_t ld, rows, cols;
  PlaneTarget t; const uint32_t* top; float* row_inv;
};

template <int KIND>
__device__ __forceinline__ void store_split(const RowArgs& a, int64_t row, int64_t c, const float (&v)[8], float scale) {
  uintx4 out[3];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w[3] = {0, 0, 0};
    split_pair<KIND>(v[2 * j], v[2 * j + 1], scale, w);
#pragma unroll
    for (int k = 0; k < plane_count<KIND>(); ++k) out[k][j] = w[k];
  }
#pragma unroll
  for (int k = 0; k < plane_count<KIND>(); ++k) *reinterpret_cast<uintx4*>(a.t.p[k] + row * a.t.pitch + c) = out[k];
}

template <typename T, int KIND, bool VEC>
__device__ __forceinline__ void row_planes(const RowArgs& a, int64_t block, int64_t blocks) {
  const int64_t units = (a.cols + 63) / 64 * 8, total = a.t.rows * units;
  const float scale = KIND == PLANE_HALF_2 ? power_of_two(half_exponent(*a.top)) : 1.0f;
  for (int64_t u = block * 256 + threadIdx.x; u < total; u += blocks * 256) {
    const int64_t row = u / units, c = (u - row * units) * 8;
    float v[8];
    load8<T, VEC>(static_cast<const T*>(a.src) + row * a.ld, c, row < a.rows ? a.cols : 0, v);
    store_split<KIND>(a, row, c, v, scale);
  }
}

template <typename T, int KIND, bool VEC>
__global__ __launch_bounds__(256) void row_planes_kernel(RowArgs a) { row_planes<T, KIND, VEC>(a, blockIdx.x, gridDim.x); }

// fp16 planes with a power of two per row: a wavefront walks its row for the largest magnitude and again, out of the cache, to
// split it.
template <bool VEC>
__device__ __forceinline__ void row_scaled_planes(const RowArgs& a, int64_t block) {
  const int64_t row = block * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= a.rows) return;
  const float* x = static_cast<const float*>(a.src) + row * a.ld;
  float v[8];
  uint32_t top = 0;
  for (int64_t c = 8 * lane; c < a.cols; c += 512) {
    load8<float, VEC>(x, c, a.cols, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, finite_magnitude(v[j]));
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  const int e = half_exponent(top);
  if (lane == 0) a.row_inv[row] = power_of_two(-e);
  const float scale = power_of_two(e);
  for (int64_t c = 8 * lane; c < (a.cols + 63) / 64 * 64; c += 512) {
    load8<float, VEC>(x, c, a.cols, v);
    store_split<PLANE_HALF_2>(a, row, c, v, scale);
  }
}

template <bool VEC>
__global__ __launch_bounds__(256) void row_scaled_planes_kernel(RowArgs a) { row_scaled_planes<VEC>(a, blockIdx.x); }

// A workgroup turns 64 x 64 values in LDS: a thread packs two rows of eight columns, so that words are written, in rows of 33
// words: the eight columns and eight row pairs of a wavefront meet 64 different banks.
struct ColumnArgs {
  const void* src; int64_t ld, rows, cols;
  PlaneTarget t; const uint32_t* top;
  const int64_t* keep; int64_t keep_below;
  int tiles_r;
};
constexpr int CP = 64, CP_WORDS = 33;

template <typename T, int KIND, bool VEC>
__device__ __forceinline__ void column_planes(const ColumnArgs& a, uint32_t block, uint32_t (*s_w)[CP * CP_WORDS]) {
  constexpr int N = plane_count<KIND>();
  const int tid = threadIdx.x;
  const int64_t r0 = (int64_t)(block % a.tiles_r) * CP, c0 = (int64_t)(block / a.tiles_r) * CP;
  const float scale = KIND == PLANE_HALF_2 ? power_of_two(half_exponent(*a.top)) : 1.0f;
  const int c = (tid & 7) * 8, pair = tid >> 3;
  float v[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t row = r0 + 2 * pair + h;
    bool take = row < a.rows;
    if (take && a.keep) { const int64_t t = a.keep[row]; take = t >= 0 && t < a.keep_below; }
    load8<T, VEC>(static_cast<const T*>(a.src) + row * a.ld, c0 + c, take ? a.cols : 0, v[h]);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t w[3] = {0, 0, 0};
    split_pair<KIND>(v[0][j], v[1][j], scale, w);
#pragma unroll
    for (int k = 0; k < N; ++k) s_w[k][(c + j) * CP_WORDS + pair] = w[k];
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int col = (tid >> 3) + 32 * h, word = (tid & 7) * 4;
    if (c0 + col >= a.t.rows) continue;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      uintx4 out;
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = s_w[k][col * CP_WORDS + word + j];
      *reinterpret_cast<uintx4*>(a.t.p[k] + (c0 + col) * a.t.pitch + r0 + 2 * word) = out;
    }
  }
}

template <typename T, int KIND, bool VEC>
__global__ __launch_bounds__(256) void column_planes_kernel(ColumnArgs a) {
  __shared__ uint32_t s_w[plane_count<KIND>()][CP * CP_WORDS];
  column_planes<T, KIND, VEC>(a, blockIdx.x, s_w);
}

static bool vectors_fit(const void* src, int64_t ld, int dtype) {
  return ((uintptr_t)src & 15) == 0 && ld * type_bytes(dtype) % 16 == 0;
}
static int check_target(const PlaneSource& s, PlaneKind kind, const PlaneTarget& t, int64_t least) {
  if (s.rows < 1 || s.cols < 1 || t.pitch % 64 || t.pitch < least) return LQ_ERR_SHAPE;
  const int n = kind == PLANE_BF16 ? 1 : kind == PLANE_HALF_2 ? 2 : 3;
  for (int k = 0; k < n; ++k)
    if (!t.p[k]) return LQ_ERR_NULL;
  return kind == PLANE_HALF_2 && s.dtype != LQ_T_FP32 ? LQ_ERR_ARG : LQ_OK;
}
static double plane_bytes(const PlaneSource& s, PlaneKind kind) {
  return (double)s.rows * (double)s.cols * (type_bytes(s.dtype) + (kind == PLANE_BF16 ? 2.0 : kind == PLANE_HALF_2 ? 4.0 : 6.0));
}

template <typename T, int KIND>
static void rows_of(const RowArgs& a, bool vec, hipStream_t st) {
  auto kernel = vec ? row_planes_kernel<T, KIND, true> : row_planes_kernel<T, KIND, false>;
  const int64_t units = a.t.rows * ((a.cols + 63) / 64 * 8);
  hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>((units + 255) / 256, 1 << 16)), dim3(256), 0, st, a);
}

int launch_row_planes(const PlaneSource& s, PlaneKind kind, const PlaneTarget& t, float* row_inv, hipStream_t st) {
  LQ_TRY(check_target(s, kind, t, up_to(s.cols, 64)));
  const RowArgs a{s.src, s.ld, s.rows, s.cols, t, s.top, row_inv};
  const bool vec = vectors_fit(s.src, s.ld, s.dtype);
  prof::Scope ps(prof::TRAIN_PLANES, st, plane_bytes(s, kind));
  if (kind == PLANE_HALF_2 && row_inv) {
    auto kernel = vec ? row_scaled_planes_kernel<true> : row_scaled_planes_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((s.rows + 3) / 4)), dim3(256), 0, st, a);
  } else if (kind == PLANE_HALF_2) {
    if (!s.top) return LQ_ERR_NULL;
    rows_of<float, PLANE_HALF_2>(a, vec, st);
  } else if (kind == PLANE_BF16_3) {
    if (s.dtype != LQ_T_FP32) return LQ_ERR_ARG;
    rows_of<float, PLANE_BF16_3>(a, vec, st);
  } else if (s.dtype == LQ_T_BF16) {
    rows_of<__bf16, PLANE_BF16>(a, vec, st);
  } else {
    return LQ_ERR_ARG;
  }
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

template <typename T, int KIND>
static void columns_of(const ColumnArgs& a, bool vec, unsigned grid, hipStream_t st) {
  auto kernel = vec ? column_planes_kernel<T, KIND, true> : column_planes_kernel<T, KIND, false>;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, st, a);
}

int launch_column_planes(const PlaneSource& s, PlaneKind kind, const PlaneTarget& t, const int64_t* keep, int64_t keep_below,
                         hipStream_t st) {
  LQ_TRY(check_target(s, kind, t, up_to(s.rows, CP)));
  const int64_t tr = (s.rows + CP - 1) / CP, tc = (t.rows + CP - 1) / CP;
  if (tr * tc >= (1ll << 31)) return LQ_ERR_SHAPE;
  const ColumnArgs a{s.src, s.ld, s.rows, s.cols, t, s.top, keep, keep_below, (int)tr};
  const bool vec = vectors_fit(s.src, s.ld, s.dtype);
  const unsigned grid = (unsigned)(tr * tc);
  prof::Scope ps(prof::TRAIN_PLANES, st, plane_bytes(s, kind));
  if (kind == PLANE_HALF_2) {
    if (!s.top) return LQ_ERR_NULL;
    columns_of<float, PLANE_HALF_2>(a, vec, grid, st);
  } else if (kind == PLANE_BF16 && s.dtype == LQ_T_BF16) {
    columns_of<__bf16, PLANE_BF16>(a, vec, grid, st);
  } else {
    return LQ_ERR_ARG;
  }
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// The largest of integers does not depend on the order in which an atomic takes them.
// FLAT: rows one after the other without a gap, each of them taken, as one long row of whole vectors.
template <bool VEC, bool FLAT>
__global__ __launch_bounds__(256) void top_magnitude_kernel(const float* __restrict__ src, int64_t ld, int64_t rows, int64_t cols,
                                                            const int64_t* __restrict__ keep, int64_t keep_below,
                                                            uint32_t* __restrict__ out) {
  __shared__ uint32_t s_top[4];
  const int64_t units = (cols + 7) / 8, total = FLAT ? rows * cols / 8 : rows * units, step = (int64_t)gridDim.x * 256;
  uint32_t top = 0;
#pragma unroll 4
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += step) {
    float v[8];
    if constexpr (FLAT) {
      load8<float, true>(src, 8 * u, 8 * total, v);
    } else {
      const int64_t row = u / units, c = (u - row * units) * 8;
      if (keep) { const int64_t t = keep[row]; if (t < 0 || t >= keep_below) continue; }
      load8<float, VEC>(src + row * ld, c, cols, v);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, finite_magnitude(v[j]));
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) atomicMax(out, max(max(s_top[0], s_top[1]), max(s_top[2], s_top[3])));
}

int launch_top_magnitude(const void* src, int64_t ld, int64_t rows, int64_t cols, const int64_t* keep, int64_t keep_below,
                         uint32_t* top, hipStream_t st) {
  const bool vec = vectors_fit(src, ld, LQ_T_FP32), flat = vec && !keep && ld == cols && cols % 8 == 0;
  const int64_t units = rows * ((cols + 7) / 8);
  auto kernel = flat ? top_magnitude_kernel<true, true> : vec ? top_magnitude_kernel<true, false> : top_magnitude_kernel<false, false>;
  prof::Scope ps(prof::TRAIN_PLANES, st, (double)rows * (double)cols * 4.0);
  hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>((units + 1023) / 1024, 2048)), dim3(256), 0, st,
                     static_cast<const float*>(src), ld, rows, cols, keep, keep_below, top);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
enum { JOB_ROWS3, JOB_COLUMNS3, JOB_ROWS_SCALED, JOB_ROWS, JOB_TOPS };

__global__ __launch_bounds__(256) void prepare_kernel(PrepareJobs jobs) {
  __shared__ uint32_t s_w[3][CP * CP_WORDS];
  int block = blockIdx.x, j = 0;
  while (block >= jobs.job[j].wgs) { block -= jobs.job[j].wgs; ++j; }       // the grid has no workgroup beyond the last job's
  const PrepareJobs::Job& job = jobs.job[j];
  const RowArgs r{job.s.src, job.s.ld, job.s.rows, job.s.cols, job.t, nullptr, job.row_inv};
  switch (job.what) {
    case JOB_ROWS3: row_planes<float, PLANE_BF16_3, false>(r, block, job.wgs); break;
    case JOB_COLUMNS3:
      column_planes<float, PLANE_BF16_3, false>(ColumnArgs{job.s.src, job.s.ld, job.s.rows, job.s.cols, job.t, nullptr, nullptr, 0, job.tiles_r},
                                                (uint32_t)block, s_w);
      break;
    case JOB_ROWS_SCALED: row_scaled_planes<true>(r, block); break;
    case JOB_ROWS: row_planes<__bf16, PLANE_BF16, true>(r, block, job.wgs); break;
    default: {
      const float* v = static_cast<const float*>(job.s.src);
      uint32_t top = 0;
      for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < job.s.cols; i += (int64_t)TOP_WORDS * 256) top = max(top, finite_magnitude(v[i]));
#pragma unroll
      for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
      if ((threadIdx.x & 63) == 0) s_w[0][threadIdx.x >> 6] = top;
      __syncthreads();
      if (threadIdx.x == 0) job.tops[block] = max(max(s_w[0][0], s_w[0][1]), max(s_w[0][2], s_w[0][3]));
    }
  }
}

static int add_job(PrepareJobs& p, int what, int64_t wgs, const PlaneSource& s, const PlaneTarget& t, float* row_inv, uint32_t* tops, int tiles_r) {
  if (p.count >= 5 || wgs < 1 || wgs >= (1ll << 30)) return LQ_ERR_SHAPE;
  p.job[p.count++] = PrepareJobs::Job{what, (int)wgs, s, t, row_inv, tops, tiles_r};
  return LQ_OK;
}
int PrepareJobs::rows3(const PlaneSource& s, const PlaneTarget& t) {
  LQ_TRY(check_target(s, PLANE_BF16_3, t, up_to(s.cols, 64)));
  return add_job(*this, JOB_ROWS3, std::min<int64_t>((t.rows * ((s.cols + 63) / 64 * 8) + 255) / 256, 1024), s, t, nullptr, nullptr, 0);
}
int PrepareJobs::columns3(const PlaneSource& s, const PlaneTarget& t) {
  LQ_TRY(check_target(s, PLANE_BF16_3, t, up_to(s.rows, CP)));
  const int64_t tr = (s.rows + CP - 1) / CP;
  return add_job(*this, JOB_COLUMNS3, tr * ((t.rows + CP - 1) / CP), s, t, nullptr, nullptr, (int)tr);
}
int PrepareJobs::rows_scaled(const PlaneSource& s, const PlaneTarget& t, float* row_inv) {
  LQ_TRY(check_target(s, PLANE_HALF_2, t, up_to(s.cols, 64)));
  if (!vectors_fit(s.src, s.ld, s.dtype)) return LQ_ERR_ARG;
  return add_job(*this, JOB_ROWS_SCALED, (s.rows + 3) / 4, s, t, row_inv, nullptr, 0);
}
int PrepareJobs::rows(const PlaneSource& s, const PlaneTarget& t) {
  LQ_TRY(check_target(s, PLANE_BF16, t, up_to(s.cols, 64)));
  if (s.dtype != LQ_T_BF16 || !vectors_fit(s.src, s.ld, s.dtype)) return LQ_ERR_ARG;
  return add_job(*this, JOB_ROWS, std::min<int64_t>((t.rows * ((s.cols + 63) / 64 * 8) + 255) / 256, 8192), s, t, nullptr, nullptr, 0);
}
int PrepareJobs::tops(const float* v, int64_t n, uint32_t* words) {
  return add_job(*this, JOB_TOPS, TOP_WORDS, PlaneSource{v, LQ_T_FP32, n, 1, n, nullptr}, PlaneTarget{}, nullptr, words, 0);
}
int PrepareJobs::launch(hipStream_t st) const {
  int64_t wgs = 0;
  double bytes = 0.0;
  for (int j = 0; j < count; ++j) { wgs += job[j].wgs; bytes += (double)job[j].s.rows * (double)job[j].s.cols * 8.0; }
  if (wgs < 1 || wgs >= (1ll << 31)) return LQ_ERR_SHAPE;
  prof::Scope ps(prof::TRAIN_PLANES, st, bytes);
  hipLaunchKernelGGL(prepare_kernel, dim3((unsigned)wgs), dim3(256), 0, st, *this);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
