// Codes and scales of a matrix and of its transpose in one pass.  Bound by its bytes, X once and the codes once or twice: a tile is one
// block in either direction, so whatever is wanted comes out of the registers that hold it (11008 x 4096 fp32 to both forms 49 us, 5.5 TB/s;
// 4096 x 4096 and 11008 x 4096 bf16 in rows, the first both ways, in one launch 48 us, 4.2 TB/s; 1000 x 50265 bf16 on odd addresses 37 us,
// 4.0 TB/s, by single values 108).  Small ones are a chain of latencies: 1001 x 1027 9 us.  bf16 values stay packed until they are scaled (74
// registers for 176, six wavefronts a SIMD for two: 4096 x 4096 in rows 19 -> 12 us).
#include "dense_device.h"
#include "fp8.h"
#include "fp8_device.h"
#include "profiler.h"

namespace lq {

constexpr int QT = 128;                  // a workgroup's tile: one block in either direction
constexpr int TURN_PITCH = QT + 16;      // bytes between rows of the turned tile in LDS

typedef uint16_t ushortx2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b) {      // of 16-bit halves
  const ushortx2 x = __builtin_bit_cast(ushortx2, a), y = __builtin_bit_cast(ushortx2, b);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, false); }

// Eight rows x eight columns of a matrix in a thread's registers as they are stored, and their largest magnitudes' bits.
template <typename T>
struct Patch;
template <>
struct Patch<float> {
  float v[8][8];
  __device__ __forceinline__ void load(int a, const float* x, int count) {
    typedef floatx4 unit __attribute__((aligned(4)));
    if (count >= 8) {
      const floatx4 p = *reinterpret_cast<const unit*>(x), q = *reinterpret_cast<const unit*>(x + 4);
#pragma unroll
      for (int b = 0; b < 4; ++b) { v[a][b] = p[b]; v[a][4 + b] = q[b]; }
    } else {
#pragma unroll
      for (int b = 0; b < 8; ++b) v[a][b] = 0.0f;
      if (count > 0)
#pragma unroll
        for (int b = 0; b < 7; ++b)
          if (b < count) v[a][b] = x[b];
    }
  }
  __device__ __forceinline__ float value(int a, int b) const { return v[a][b]; }
  // over the 16 lanes that share the rows
  __device__ __forceinline__ void row_tops(uint32_t (&top)[8]) const {
#pragma unroll
    for (int a = 0; a < 8; ++a) {
      uint32_t m = 0;
#pragma unroll
      for (int b = 0; b < 8; ++b) m = max(m, magnitude(v[a][b]));
      m = max(m, moved<XOR1>(m));
      m = max(m, moved<XOR2>(m));
      m = max(m, moved<XOR7>(m));
      top[a] = max(m, moved<XOR15>(m));
    }
  }
  // over the four lanes of a wavefront that share the columns
  __device__ __forceinline__ void column_tops(uint32_t (&top)[8]) const {
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      uint32_t m = 0;
#pragma unroll
      for (int a = 0; a < 8; ++a) m = max(m, magnitude(v[a][b]));
      m = max(m, (uint32_t)__shfl_xor((int)m, 16));
      top[b] = max(m, (uint32_t)__shfl_xor((int)m, 32));
    }
  }
};
// bf16: pairs of neighbours in a word, so one instruction compares two.
template <>
struct Patch<__bf16> {
  uint32_t w[8][4];
  __device__ __forceinline__ void load(int a, const __bf16* x, int count) {
    typedef uintx4 unit __attribute__((aligned(2)));
    if (count >= 8) {
      const uintx4 p = *reinterpret_cast<const unit*>(x);
#pragma unroll
      for (int b = 0; b < 4; ++b) w[a][b] = p[b];
    } else {
#pragma unroll
      for (int b = 0; b < 4; ++b) w[a][b] = 0;
      if (count > 0)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const uint32_t lo = 2 * b < count ? __builtin_bit_cast(uint16_t, x[2 * b]) : 0u;
        const uint32_t hi = 2 * b + 1 < count ? __builtin_bit_cast(uint16_t, x[2 * b + 1]) : 0u;
        w[a][b] = lo | hi << 16;
      }
    }
  }
  __device__ __forceinline__ float value(int a, int b) const { return __uint_as_float(b & 1 ? w[a][b >> 1] & 0xffff0000u : w[a][b >> 1] << 16); }
  __device__ __forceinline__ void row_tops(uint32_t (&top)[8]) const {
#pragma unroll
    for (int a = 0; a < 8; a += 2) {
      uint32_t m[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        m[h] = pair_max(pair_max(w[a + h][0] & 0x7fff7fffu, w[a + h][1] & 0x7fff7fffu), pair_max(w[a + h][2] & 0x7fff7fffu, w[a + h][3] & 0x7fff7fffu));
      }
      // the two rows' in one word from here on
      uint32_t both = pair_max((m[0] & 0xffffu) | m[1] << 16, m[0] >> 16 | (m[1] & 0xffff0000u));
      both = pair_max(both, moved<XOR1>(both));
      both = pair_max(both, moved<XOR2>(both));
      both = pair_max(both, moved<XOR7>(both));
      both = pair_max(both, moved<XOR15>(both));
      top[a] = both << 16;
      top[a + 1] = both & 0xffff0000u;
    }
  }
  __device__ __forceinline__ void column_tops(uint32_t (&top)[8]) const {
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      uint32_t m = 0;
#pragma unroll
      for (int a = 0; a < 8; ++a) m = pair_max(m, w[a][b] & 0x7fff7fffu);
      m = pair_max(m, (uint32_t)__shfl_xor((int)m, 16));
      m = pair_max(m, (uint32_t)__shfl_xor((int)m, 32));
      top[2 * b] = m << 16;
      top[2 * b + 1] = m & 0xffff0000u;
    }
  }
};

// Thread t holds columns 8 (t % 16) .. + 7 of rows 8 (t / 16) .. + 7 in registers, so that a line of X is read by sixteen neighbours,
// a row's block is theirs alone, and eight rows of a column are one store into the turned tile.  Two matrices may share a launch.
template <typename T, bool TILES>
__global__ __launch_bounds__(256) void fp8_quantize_kernel(Fp8Quantize one, Fp8Quantize two, int64_t tiles_one) {
  __shared__ uint32_t tops[4][QT];
  __shared__ float inverse[QT];
  __shared__ __align__(16) uint8_t turned[QT * TURN_PITCH];
  const int tid = threadIdx.x, c = tid & 15, r = tid >> 4, wave = tid >> 6;
  const bool second = (int64_t)blockIdx.x >= tiles_one;
  const Fp8Quantize q = second ? two : one;
  const int64_t blocks_d = (q.d + QT - 1) / QT;
  const int64_t tile = (int64_t)blockIdx.x - (second ? tiles_one : 0), bi = tile / blocks_d, bj = tile - bi * blocks_d;
  const int64_t i0 = bi * QT + 8 * r, j0 = bj * QT + 8 * c;
  const T* x = static_cast<const T*>(q.x);
  const int columns = (int)max((int64_t)0, min((int64_t)8, q.d - j0));
  Patch<T> p;
#pragma unroll
  for (int a = 0; a < 8; ++a) p.load(a, x + (i0 + a) * q.ldx + j0, i0 + a < q.m ? columns : 0);
  float row_inverse[8], column_inverse[8];
  if constexpr (TILES) {
    uint32_t row_top[8], top = 0;
    p.row_tops(row_top);
#pragma unroll
    for (int a = 0; a < 8; ++a) top = max(top, row_top[a]);
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    if ((tid & 63) == 0) tops[wave][0] = top;
    __syncthreads();
    top = max(max(tops[0][0], tops[1][0]), max(tops[2][0], tops[3][0]));
    const float s = fp8_scale(top), f = fp8_inverse(s);
    if (tid == 0) q.scale[bi * blocks_d + bj] = s;
#pragma unroll
    for (int a = 0; a < 8; ++a) row_inverse[a] = column_inverse[a] = f;
  } else {
    if (q.codes) {
      uint32_t top[8];
      p.row_tops(top);
#pragma unroll
      for (int a = 0; a < 8; ++a) {
        const float s = fp8_scale(top[a]);
        row_inverse[a] = fp8_inverse(s);
        if (c == a && i0 + a < q.m) q.scale[bj * q.m + i0 + a] = s;
      }
    }
    if (q.codes_t) {
      uint32_t top[8];
      p.column_tops(top);
#pragma unroll
      for (int b = 0; b < 8; ++b)
        if ((tid & 63) < 16) tops[wave][8 * c + b] = top[b];
      __syncthreads();
      if (tid < QT) {
        const float s = fp8_scale(max(max(tops[0][tid], tops[1][tid]), max(tops[2][tid], tops[3][tid])));
        inverse[tid] = fp8_inverse(s);
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
      const uintx2 w = {fp8_four(p.value(a, 0) * f, p.value(a, 1) * f, p.value(a, 2) * f, p.value(a, 3) * f),
                        fp8_four(p.value(a, 4) * f, p.value(a, 5) * f, p.value(a, 6) * f, p.value(a, 7) * f)};
      if (i0 + a < q.m && j0 < end) *reinterpret_cast<uintx2*>(q.codes + (i0 + a) * q.ld + j0) = w;
    }
  }
  if (!q.codes_t) return;
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const float f = column_inverse[b];
    const uintx2 w = {fp8_four(p.value(0, b) * f, p.value(1, b) * f, p.value(2, b) * f, p.value(3, b) * f),
                      fp8_four(p.value(4, b) * f, p.value(5, b) * f, p.value(6, b) * f, p.value(7, b) * f)};
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

template <typename T>
static void launch(const Fp8Quantize& one, const Fp8Quantize& two, bool tiles, hipStream_t st) {
  auto kernel = tiles ? fp8_quantize_kernel<T, true> : fp8_quantize_kernel<T, false>;
  const int64_t first = fp8_blocks(one.m) * fp8_blocks(one.d), second = fp8_blocks(two.m) * fp8_blocks(two.d);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(first + second)), dim3(256), 0, st, one, two, first);
}

int launch_fp8_quantize(const Fp8Quantize* q, int count, bool tiles, hipStream_t st) {
  double bytes = 0;
  for (int i = 0; i < count; ++i) {
    if (fp8_blocks(q[i].m) * fp8_blocks(q[i].d) >= ((int64_t)1 << 23)) return LQ_ERR_SHAPE;
    bytes += (double)q[i].m * q[i].d * (type_bytes(q[i].dtype) + (q[i].codes != nullptr) + (q[i].codes_t != nullptr));
  }
  if (count == 2 && q[0].dtype != q[1].dtype) {
    LQ_TRY(launch_fp8_quantize(q, 1, tiles, st));
    return launch_fp8_quantize(q + 1, 1, tiles, st);
  }
  prof::Scope ps(prof::FP8_QUANTIZE, st, bytes);
  const Fp8Quantize none{}, & two = count == 2 ? q[1] : none;
  if (q[0].dtype == LQ_T_BF16) launch<__bf16>(q[0], two, tiles, st);
  else launch<float>(q[0], two, tiles, st);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
