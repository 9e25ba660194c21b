// Products of matrices in 8 bits.
#include "fp8.h"
#include "fp8_device.h"
#include "profiler.h"

namespace lq {

// 32 bytes of a row from byte `at` on, zero past its length k; what lies past the last 16 bytes that hold a value is not read.
__device__ __forceinline__ intx8 fp8_load(const uint8_t* row, int64_t at, int64_t k) {
  uintx4 half[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t left = k - (at + 16 * h);
    half[h] = left > 0 ? *reinterpret_cast<const uintx4*>(row + at + 16 * h) : uintx4{0, 0, 0, 0};
    if (left < 16) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int64_t bytes = left - 4 * w;
        half[h][w] = bytes >= 4 ? half[h][w] : bytes <= 0 ? 0u : half[h][w] & ((1u << (8 * bytes)) - 1u);
      }
    }
  }
  return intx8{(int)half[0][0], (int)half[0][1], (int)half[0][2], (int)half[0][3], (int)half[1][0], (int)half[1][1], (int)half[1][2], (int)half[1][3]};
}

// A wavefront makes 16 rows x 16 NC columns; lane l brings byte 32 (l / 16) .. + 31 of a block of row (column) l % 16.
template <int NC>
__global__ __launch_bounds__(256) void fp8_rows_kernel(Fp8Product p) {
  const int lane = threadIdx.x & 63, l16 = lane & 15, kg = lane >> 4;
  const int64_t row_tiles = (p.rows.count + 15) / 16;
  const int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), rt = u % row_tiles, ct = u / row_tiles;
  const int64_t r0 = 16 * rt, c0 = 16 * NC * ct;
  if (c0 >= p.columns.count) return;
  const uint8_t* row = p.rows.codes + min(r0 + l16, p.rows.count - 1) * p.rows.ld;
  const uint8_t* column[NC];
  const float* column_scale[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int64_t i = min(c0 + 16 * j + l16, p.columns.count - 1);
    column[j] = p.columns.codes + i * p.columns.ld;
    column_scale[j] = p.columns.scale + (i >> p.columns.shift) * p.columns.scale_row;
  }
  const float* row_scale[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) row_scale[e] = p.rows.scale + (min(r0 + 4 * kg + e, p.rows.count - 1) >> p.rows.shift) * p.rows.scale_row;
  floatx4 acc[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) acc[j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t blocks = (p.k + FP8_BLOCK - 1) / FP8_BLOCK;
  for (int64_t b = 0; b < blocks; ++b) {
    const int64_t at = b * FP8_BLOCK + 32 * kg;
    const intx8 x = fp8_load(row, at, p.k);
    float s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = row_scale[e][b * p.rows.scale_block] * FP8_LIFT;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const intx8 y = fp8_load(column[j], at, p.k);
      const float t = column_scale[j][b * p.columns.scale_block];
      const floatx4 z = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, floatx4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] = fmaf(z[e], s[e] * t, acc[j][e]);
    }
  }
  __bf16* out = static_cast<__bf16*>(p.out);
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int64_t i = c0 + 16 * j + l16;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i < p.columns.count && r0 + 4 * kg + e < p.rows.count) out[i * p.ld + r0 + 4 * kg + e] = (__bf16)(acc[j][e] * FP8_DROP);
  }
}

constexpr int64_t FEW_COLUMNS = 128;
size_t fp8_product_part_floats(int64_t rows, int64_t columns, int64_t k) {
  return columns > FEW_COLUMNS ? fp8_tiles_part_floats(rows, columns, k) : 0;
}

int launch_fp8_product(const Fp8Product& p, float* part, size_t part_floats, hipStream_t st) {
  if (p.columns.count > FEW_COLUMNS) return launch_fp8_tiles(p, part, part_floats, st);
  const int64_t row_tiles = (p.rows.count + 15) / 16;
  const int nc = p.columns.count > 16 ? 4 : 1;
  const int64_t waves = row_tiles * ((p.columns.count + 16 * nc - 1) / (16 * nc));
  if (waves >= ((int64_t)1 << 32)) return LQ_ERR_SHAPE;
  prof::Scope ps(prof::FP8_ROWS, st, (double)p.rows.count * p.k);
  auto kernel = nc == 4 ? fp8_rows_kernel<4> : fp8_rows_kernel<1>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, p);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
