// Codes and scales of a matrix and of its transpose in one pass.
#include "fp8.h"
#include "fp8_device.h"
#include "profiler.h"

namespace lq {

constexpr int QT = 128;                  // a workgroup's tile: one block in either direction
constexpr int TURN_PITCH = QT + 16;      // bytes between rows of the turned tile in LDS

// Thread t holds columns 8 (t % 16) .. + 7 of rows 8 (t / 16) .. + 7 in registers, so that a line of X is read by sixteen neighbours,
// a row's block is theirs alone, and eight rows of a column are one store into the turned tile.
template <typename T, bool VEC, bool TILES>
__global__ __launch_bounds__(256) void fp8_quantize_kernel(Fp8Quantize q) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  __shared__ uint32_t tops[4][QT];
  __shared__ float inverse[QT];
  __shared__ __align__(16) uint8_t turned[QT * TURN_PITCH];
  const int tid = threadIdx.x, c = tid & 15, r = tid >> 4, wave = tid >> 6;
  const int64_t blocks_d = (q.d + QT - 1) / QT;
  const int64_t tile = blockIdx.x, bi = tile / blocks_d, bj = tile - bi * blocks_d;
  const int64_t i0 = bi * QT + 8 * r, j0 = bj * QT + 8 * c;
  const T* x = static_cast<const T*>(q.x);
  float v[8][8];
#pragma unroll
  for (int a = 0; a < 8; ++a) {
    const int64_t i = i0 + a;
    if (VEC && i < q.m && j0 + 8 <= q.d) {
      const vec8 in = *reinterpret_cast<const vec8*>(x + i * q.ldx + j0);
#pragma unroll
      for (int b = 0; b < 8; ++b) v[a][b] = (float)in[b];
    } else {
#pragma unroll
      for (int b = 0; b < 8; ++b) v[a][b] = i < q.m && j0 + b < q.d ? (float)x[i * q.ldx + j0 + b] : 0.0f;
    }
  }
  uint32_t row_top[8], column_top[8];
#pragma unroll
  for (int a = 0; a < 8; ++a) row_top[a] = column_top[a] = 0;
#pragma unroll
  for (int a = 0; a < 8; ++a)
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const uint32_t g = magnitude(v[a][b]);
      row_top[a] = max(row_top[a], g);
      column_top[b] = max(column_top[b], g);
    }
  float row_inverse[8], column_inverse[8];
  if constexpr (TILES) {
    uint32_t top = 0;
#pragma unroll
    for (int a = 0; a < 8; ++a) top = max(top, row_top[a]);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s));
    if ((tid & 63) == 0) tops[wave][0] = top;
    __syncthreads();
    top = max(max(tops[0][0], tops[1][0]), max(tops[2][0], tops[3][0]));
    const float s = fp8_scale(top);
    if (tid == 0) q.scale[bi * blocks_d + bj] = s;
#pragma unroll
    for (int a = 0; a < 8; ++a) row_inverse[a] = column_inverse[a] = 1.0f / s;
  } else {
    if (q.codes) {
#pragma unroll
      for (int a = 0; a < 8; ++a) {
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) row_top[a] = max(row_top[a], (uint32_t)__shfl_xor((int)row_top[a], s));
        const float s = fp8_scale(row_top[a]);
        row_inverse[a] = 1.0f / s;
        if (c == 0 && i0 + a < q.m) q.scale[bj * q.m + i0 + a] = s;
      }
    }
    if (q.codes_t) {
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        column_top[b] = max(column_top[b], (uint32_t)__shfl_xor((int)column_top[b], 16));
        column_top[b] = max(column_top[b], (uint32_t)__shfl_xor((int)column_top[b], 32));
        if ((tid & 63) < 16) tops[wave][8 * c + b] = column_top[b];
      }
      __syncthreads();
      if (tid < QT) {
        const float s = fp8_scale(max(max(tops[0][tid], tops[1][tid]), max(tops[2][tid], tops[3][tid])));
        inverse[tid] = 1.0f / s;
        if (bj * QT + tid < q.d) q.scale_t[bi * q.d + bj * QT + tid] = s;
      }
      __syncthreads();
#pragma unroll
      for (int b = 0; b < 8; ++b) column_inverse[b] = inverse[8 * c + b];
    }
  }
  if (q.codes) {
    const int64_t end = (q.d + 15) & ~(int64_t)15;
#pragma unroll
    for (int a = 0; a < 8; ++a) {
      const float f = row_inverse[a];
      const uintx2 w = {fp8_four(v[a][0] * f, v[a][1] * f, v[a][2] * f, v[a][3] * f),
                        fp8_four(v[a][4] * f, v[a][5] * f, v[a][6] * f, v[a][7] * f)};
      if (i0 + a < q.m && j0 < end) *reinterpret_cast<uintx2*>(q.codes + (i0 + a) * q.ld + j0) = w;
    }
  }
  if (!q.codes_t) return;
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const float f = column_inverse[b];
    const uintx2 w = {fp8_four(v[0][b] * f, v[1][b] * f, v[2][b] * f, v[3][b] * f),
                      fp8_four(v[4][b] * f, v[5][b] * f, v[6][b] * f, v[7][b] * f)};
    *reinterpret_cast<uintx2*>(turned + (8 * c + b) * TURN_PITCH + 8 * r) = w;
  }
  __syncthreads();
  const int64_t end = (q.m + 15) & ~(int64_t)15;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int j = 32 * a + (tid >> 3), i = 16 * (tid & 7);
    if (bj * QT + j < q.d && bi * QT + i < end)
      *reinterpret_cast<uintx4*>(q.codes_t + (bj * QT + j) * q.ld_t + bi * QT + i) = *reinterpret_cast<const uintx4*>(turned + j * TURN_PITCH + i);
  }
}

template <typename T, bool TILES>
static void launch(const Fp8Quantize& q, hipStream_t st) {
  const unsigned wgs = (unsigned)(fp8_blocks(q.m) * fp8_blocks(q.d));
  const bool vec = ((uintptr_t)q.x & (8 * sizeof(T) - 1) & 15) == 0 && q.ldx % (16 / (int64_t)sizeof(T)) == 0;
  auto kernel = vec ? fp8_quantize_kernel<T, true, TILES> : fp8_quantize_kernel<T, false, TILES>;
  hipLaunchKernelGGL(kernel, dim3(wgs), dim3(256), 0, st, q);
}

int launch_fp8_quantize(const Fp8Quantize& q, bool tiles, hipStream_t st) {
  if (fp8_blocks(q.m) * fp8_blocks(q.d) >= ((int64_t)1 << 31)) return LQ_ERR_SHAPE;
  prof::Scope ps(prof::FP8_QUANTIZE, st, (double)q.m * q.d * (type_bytes(q.dtype) + (q.codes != nullptr) + (q.codes_t != nullptr)));
  if (q.dtype == LQ_T_BF16) tiles ? launch<__bf16, true>(q, st) : launch<__bf16, false>(q, st);
  else tiles ? launch<float, true>(q, st) : launch<float, false>(q, st);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
