// Operands of the training operators as bf16 planes: rows as they are, or transposed, so that the reduction index of the product
// that reads them is contiguous.  Both passes are bound by the bytes they move.
#include "mfma_device.h"
#include "profiler.h"
#include "train.h"

namespace lq {

template <typename T>
__device__ __forceinline__ floatx2 pair_of(T a, T b) { return floatx2{(float)a, (float)b}; }

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

__device__ __forceinline__ void split8(const float (&v)[8], bf16x8& hi, bf16x8& lo) {
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    bf16x2 h, l;
    split_bf16(floatx2{v[j], v[j + 1]}, h, l);
    hi[j] = h[0]; hi[j + 1] = h[1];
    lo[j] = l[0]; lo[j + 1] = l[1];
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void row_planes_kernel(const T* __restrict__ src, int64_t ld, int64_t rows, int64_t cols,
                                                         int64_t out_rows, uint16_t* __restrict__ hi, uint16_t* __restrict__ lo, int64_t pitch) {
  const int64_t units = (cols + 31) / 32 * 4, total = out_rows * units;
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
    const int64_t row = u / units, c = (u - row * units) * 8;
    float v[8];
    load8<T, VEC>(src + row * ld, c, row < rows ? cols : 0, v);
    bf16x8 h, l;
    split8(v, h, l);
    *reinterpret_cast<bf16x8*>(hi + row * pitch + c) = h;
    if (lo) *reinterpret_cast<bf16x8*>(lo + row * pitch + c) = l;
  }
}

// A workgroup turns 64 x 64 values in LDS; rows of 33 words, so that reading down a column meets different banks.
constexpr int CP = 64, CP_PITCH = 66;
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void column_planes_kernel(const T* __restrict__ src, int64_t ld, int64_t rows, int64_t cols,
                                                            int64_t out_rows, const int64_t* __restrict__ keep, int64_t keep_below,
                                                            uint16_t* __restrict__ hi, uint16_t* __restrict__ lo, int64_t pitch,
                                                            int tiles_r) {
  __shared__ uint32_t s_hi[CP * CP_PITCH / 2], s_lo[CP * CP_PITCH / 2];
  const int tid = threadIdx.x;
  const int64_t r0 = (int64_t)(blockIdx.x % tiles_r) * CP, c0 = (int64_t)(blockIdx.x / tiles_r) * CP;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = (tid >> 3) + 32 * h, c = (tid & 7) * 8;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    bool take = r0 + r < rows;
    if (take && keep) { const int64_t t = keep[r0 + r]; take = t >= 0 && t < keep_below; }
    if (take && c0 + c < cols) load8<T, VEC>(src + (r0 + r) * ld, c0 + c, cols, v);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      bf16x2 a, b;
      split_bf16(floatx2{v[j], v[j + 1]}, a, b);
      s_hi[r * (CP_PITCH / 2) + (c + j) / 2] = __builtin_bit_cast(uint32_t, a);
      if (lo) s_lo[r * (CP_PITCH / 2) + (c + j) / 2] = __builtin_bit_cast(uint32_t, b);
    }
  }
  __syncthreads();
  const uint16_t* th = reinterpret_cast<const uint16_t*>(s_hi);
  const uint16_t* tl = reinterpret_cast<const uint16_t*>(s_lo);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int c = (tid >> 3) + 32 * h, r = (tid & 7) * 8;
    if (c0 + c >= out_rows) continue;
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
    u16x8 out;
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = th[(r + j) * CP_PITCH + c];
    *reinterpret_cast<u16x8*>(hi + (c0 + c) * pitch + r0 + r) = out;
    if (lo) {
#pragma unroll
      for (int j = 0; j < 8; ++j) out[j] = tl[(r + j) * CP_PITCH + c];
      *reinterpret_cast<u16x8*>(lo + (c0 + c) * pitch + r0 + r) = out;
    }
  }
}

template <typename T>
static void rows_of(const void* src, int64_t ld, int64_t rows, int64_t cols, int64_t out_rows, uint16_t* hi, uint16_t* lo,
                    int64_t pitch, hipStream_t st) {
  const bool vec = ((uintptr_t)src & 15) == 0 && ld * sizeof(T) % 16 == 0;
  auto kernel = vec ? row_planes_kernel<T, true> : row_planes_kernel<T, false>;
  const int64_t units = out_rows * ((cols + 31) / 32 * 4);
  hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>((units + 255) / 256, 1 << 16)), dim3(256), 0, st,
                     static_cast<const T*>(src), ld, rows, cols, out_rows, hi, lo, pitch);
}

int launch_row_planes(const void* src, int dtype, int64_t ld, int64_t rows, int64_t cols, int64_t out_rows, uint16_t* hi,
                      uint16_t* lo, int64_t pitch, hipStream_t st) {
  if (pitch % 8 || pitch < (cols + 31) / 32 * 32) return LQ_ERR_SHAPE;
  prof::Scope ps(prof::TRAIN_PLANES, st, (double)rows * cols * (type_bytes(dtype) + (lo ? 4.0 : 2.0)));
  if (dtype == LQ_T_BF16) rows_of<__bf16>(src, ld, rows, cols, out_rows, hi, lo, pitch, st);
  else rows_of<float>(src, ld, rows, cols, out_rows, hi, lo, pitch, st);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

template <typename T>
static int columns_of(const void* src, int64_t ld, int64_t rows, int64_t cols, int64_t out_rows, const int64_t* keep, int64_t below,
                      uint16_t* hi, uint16_t* lo, int64_t pitch, hipStream_t st) {
  const bool vec = ((uintptr_t)src & 15) == 0 && ld * sizeof(T) % 16 == 0;
  auto kernel = vec ? column_planes_kernel<T, true> : column_planes_kernel<T, false>;
  const int64_t tr = (rows + CP - 1) / CP, tc = (out_rows + CP - 1) / CP;
  if (tr * tc >= (1ll << 31)) return LQ_ERR_SHAPE;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(tr * tc)), dim3(256), 0, st, static_cast<const T*>(src), ld, rows, cols, out_rows, keep, below,
                     hi, lo, pitch, (int)tr);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

int launch_column_planes(const void* src, int dtype, int64_t ld, int64_t rows, int64_t cols, int64_t out_rows,
                         const int64_t* keep, int64_t keep_below, uint16_t* hi, uint16_t* lo, int64_t pitch, hipStream_t st) {
  if (pitch % 8 || pitch < up_to(rows, CP)) return LQ_ERR_SHAPE;
  prof::Scope ps(prof::TRAIN_PLANES, st, (double)rows * cols * (type_bytes(dtype) + (lo ? 4.0 : 2.0)));
  if (dtype == LQ_T_BF16) return columns_of<__bf16>(src, ld, rows, cols, out_rows, keep, keep_below, hi, lo, pitch, st);
  return columns_of<float>(src, ld, rows, cols, out_rows, keep, keep_below, hi, lo, pitch, st);
}

}  // namespace lq
