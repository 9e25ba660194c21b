// Products of matrices in 8 bits for few columns (tokens): bound by reading the rows' operand (the weights) once.
#include "dense_device.h"
#include "fp8.h"
#include "fp8_device.h"
#include "profiler.h"

namespace lq {

// Whether these kernels are taken, us by them and by 256 x 256 tiles (rows x depth, columns): up to 64 columns 4096 x 4096, 64 17 and 23,
// 4096 x 11008, 64 33 and 32, 1024 x 50265, 64 42 and 40, 32 31 and 38; up to 128 where the sum is short: 768 x 768, 128 11 and 17,
// 32000 x 1024, 128 30 and 36, 768 x 3000, 128 20 and 19, 11008 x 4096, 128 46 and 34.
static bool few_columns(int64_t columns, int64_t k) { return columns <= 64 || (columns <= 128 && k <= 3000); }
constexpr int R_WAVES = 4;
// Columns that are quantized where they are used, us for 8 rows so and in a launch before: bf16 768 x 768 3.3 and 7.3, 4096 x 4096 7.8 and
// 12.5, 11008 x 4096 14.6 and 17.2, 1024 x 50265 26.1 and 25.6; one row 2.9 and 7.3, 5.7 and 9.6, 10.1 and 14.5, 16.1 and 23.3.
constexpr int RAW_MOST = 8;

struct RowsArgs {
  Fp8Operand rows, columns;                // columns.codes is not read where x is
  const void* x; int64_t ldx;              // the columns' operand before its quantization
  int64_t k;
  void* out; int64_t ld;
  float* part;
  int64_t row_groups;
  int splits, blocks;
};

// 32 bytes of a row from byte `at` on, in units of 16; units past the row's last one are the last one again.
__device__ __forceinline__ intx8 rows_load(const uint8_t* row, int64_t at, int64_t last) {
  const uintx4 x = *reinterpret_cast<const uintx4*>(row + min(at, last)), y = *reinterpret_cast<const uintx4*>(row + min(at + 16, last));
  return intx8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
}
// The bytes of those that lie past k become 0.
__device__ __forceinline__ void rows_clear(intx8& v, int64_t at, int64_t k) {
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    const int64_t bytes = k - at - 4 * w;
    v[w] = bytes >= 4 ? v[w] : bytes <= 0 ? 0 : v[w] & ((1 << (8 * (int)bytes)) - 1);
  }
}

// ---- the columns' operand quantized by the wavefronts that use it -------------------------------------------------
// A step of U blocks: a lane takes 16 neighbours of a column, eight lanes a block, 8 U a column.  A column's codes are followed by 16
// bytes (reads of 16 columns x 16 bytes touch every bank alike), all codes by the scales.
constexpr int x_pitch(int u) { return u * 128 + 16; }
constexpr int x_bytes(int columns, int u) { return (columns * (x_pitch(u) + u * 4) + 15) & ~15; }      // of a wavefront

template <typename T>
struct RawColumn;
template <>
struct RawColumn<__bf16> {
  uint32_t w[8];
  __device__ __forceinline__ void load(const __bf16* x, int64_t i, int64_t k) {
    typedef uintx4 unit __attribute__((aligned(2)));
    if (i + 16 <= k) {
      const uintx4 a = *reinterpret_cast<const unit*>(x + i), b = *reinterpret_cast<const unit*>(x + i + 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) { w[j] = a[j]; w[4 + j] = b[j]; }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t lo = i + 2 * j < k ? __builtin_bit_cast(uint16_t, x[i + 2 * j]) : 0u;
        const uint32_t hi = i + 2 * j + 1 < k ? __builtin_bit_cast(uint16_t, x[i + 2 * j + 1]) : 0u;
        w[j] = lo | hi << 16;
      }
    }
  }
  __device__ __forceinline__ float value(int j) const { return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16); }
};
template <>
struct RawColumn<float> {
  float v[16];
  __device__ __forceinline__ void load(const float* x, int64_t i, int64_t k) {
    typedef floatx4 unit __attribute__((aligned(4)));
    if (i + 16 <= k) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const floatx4 a = *reinterpret_cast<const unit*>(x + i + 4 * q);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * q + j] = a[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = i + j < k ? x[i + j] : 0.0f;
    }
  }
  __device__ __forceinline__ float value(int j) const { return v[j]; }
};

// The lane's 16 values of a column, from the `at`th of the step on.
template <int U, typename T>
__device__ __forceinline__ void quantize_column(const RawColumn<T>& raw, int column, unsigned char* codes, float* scales, int at) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 16; ++j) top = max(top, magnitude(raw.value(j)));
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, XOR1, 0xf, 0xf, false));
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, XOR2, 0xf, 0xf, false));
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, XOR7, 0xf, 0xf, false));
  const float s = fp8_scale(top), f = fp8_inverse(s);
  uintx4 c;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    c[q] = fp8_four(raw.value(4 * q) * f, raw.value(4 * q + 1) * f, raw.value(4 * q + 2) * f, raw.value(4 * q + 3) * f);
  *reinterpret_cast<uintx4*>(codes + column * x_pitch(U) + at) = c;
  if (at % 128 == 0) scales[column * U + at / 128] = s;
}

// Lanes read from LDS what other lanes of their wavefront have written, and write what those have read.  The wavefront's LDS accesses are
// carried out in order; this keeps the compiler to it, and costs no instruction.
__device__ __forceinline__ void wavefront_turn() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ---- the product ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ void rows_store(const RowsArgs& a, floatx4 v, int64_t row, int64_t column) {
  if (column >= a.columns.count) return;
  __bf16* out = static_cast<__bf16*>(a.out) + column * a.ld + row;
  const bf16x4 w = {(__bf16)(v[0] * FP8_DROP), (__bf16)(v[1] * FP8_DROP), (__bf16)(v[2] * FP8_DROP), (__bf16)(v[3] * FP8_DROP)};
  if (row + 4 <= a.rows.count && ((uintptr_t)out & 7) == 0) {
    *reinterpret_cast<bf16x4*>(out) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (row + e < a.rows.count) out[e] = w[e];
  }
}

// A workgroup makes 16 RT rows x 16 NC columns over its range of the sum, each of its wavefronts a quarter of the range: lane l
// brings 32 bytes (l / 16) of a block of row (column) l % 16 straight into registers, U blocks of the rows' operand under way at
// once (32000 x 1024, one row: with eight blocks a wavefront by more rows 8.3 us, 4 TB/s; 11008 x 4096 10.1 us, 4.5 TB/s).  With T (not
// void) the up to RAWS columns are quantized on the way, by every workgroup for itself: a launch less.  From 17 columns on it is their codes,
// which every 16 RT rows ask for again, that take longer than the weights (11008 x 4096, 64 columns 25 us); four wavefronts that share them did
// not help.
template <int NC, int RT, int U, bool TILED, int RAWS, typename T>
__global__ __launch_bounds__(64 * R_WAVES) void fp8_rows_kernel(RowsArgs a) {
  constexpr bool RAW = !std::is_void<T>::value;
  static_assert(!RAW || (RAWS <= 16 * NC && U <= 8 && RAWS % (8 / U) == 0), "a step's layout");
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = threadIdx.x & 63, l16 = lane & 15, kg = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t group = blockIdx.x / a.splits;
  const int split = (int)(blockIdx.x - group * a.splits);
  const int w0 = split * R_WAVES + wave, shares = a.splits * R_WAVES;
  const int b0 = (int)((int64_t)a.blocks * w0 / shares), b1 = (int)((int64_t)a.blocks * (w0 + 1) / shares);
  const int64_t r0 = group * 16 * RT, last = (a.k - 1) & ~(int64_t)15;
  const bool ragged = a.k % 128 != 0;
  const uint8_t* row[RT];
  constexpr int RS = TILED ? 1 : 4;                  // scales that a lane's four rows of a block have
  const float* row_scale[RT][RS];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    row[t] = a.rows.codes + min(r0 + 16 * t + l16, a.rows.count - 1) * a.rows.ld;
#pragma unroll
    for (int e = 0; e < RS; ++e)
      row_scale[t][e] = a.rows.scale + (TILED ? r0 >> 7 : min(r0 + 16 * t + 4 * kg + e, a.rows.count - 1) >> a.rows.shift) * a.rows.scale_row;
  }
  const uint8_t* column[NC];
  const float* column_scale[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int64_t i = min((int64_t)16 * j + l16, a.columns.count - 1);
    column[j] = a.columns.codes + i * a.columns.ld;
    column_scale[j] = a.columns.scale + (i >> a.columns.shift) * a.columns.scale_row;
  }
  floatx4 acc[RT][NC];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int j = 0; j < NC; ++j) acc[t][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  const int columns = (int)a.columns.count;
  unsigned char* codes = lds + wave * x_bytes(columns, U);
  float* scales = reinterpret_cast<float*>(codes + columns * x_pitch(U));

  for (int b = b0; b < b1; b += U) {
    intx8 w[U][RT];
    float s[U][RT][RS], f[U][NC];
    auto load_rows = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int t = 0; t < RT; ++t) w[u][t] = rows_load(row[t], (int64_t)min(b + u, b1 - 1) * 128 + 32 * kg, last);
    };
    if constexpr (RAW) {
      const T* x = static_cast<const T*>(a.x);
      constexpr int G = 8 / U, N = RAWS / G < 4 || RAWS <= RAW_MOST ? RAWS / G : 4;         // columns at a time, times
      const int at = 16 * (lane % (8 * U)), own = lane / (8 * U);
      RawColumn<T> raw[N];
      auto ask = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < N; ++c)
          if (c0 + G * c + own < columns) raw[c].load(x + (c0 + G * c + own) * a.ldx, (int64_t)b * 128 + at, a.k);
      };
      auto take = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < N; ++c)
          if (c0 + G * c + own < columns) quantize_column<U>(raw[c], c0 + G * c + own, codes, scales, at);
      };
      ask(0);                                        // before the weights, which these values would otherwise wait for
      load_rows();
      take(0);
      if constexpr (RAWS > G * N)
        for (int c0 = G * N; c0 < columns; c0 += G * N) {
          ask(c0);
          take(c0);
        }
      wavefront_turn();
    } else {
      load_rows();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = min(b + u, b1 - 1);
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int e = 0; e < RS; ++e) s[u][t][e] = row_scale[t][e][at * a.rows.scale_block];
      if constexpr (!RAW) {
#pragma unroll
        for (int j = 0; j < NC; ++j) f[u][j] = column_scale[j][at * a.columns.scale_block];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (b + u < b1) {
        const int64_t at = (int64_t)(b + u) * 128 + 32 * kg;
        const bool end = ragged && b + u == a.blocks - 1;
        intx8 y[NC];
        if constexpr (RAW) {
#pragma unroll
          for (int j = 0; j < NC; ++j) {
            const int mine = min(16 * j + l16, columns - 1);
            const unsigned char* from = codes + mine * x_pitch(U) + 128 * u + 32 * kg;
            const uintx4 lo = *reinterpret_cast<const uintx4*>(from), hi = *reinterpret_cast<const uintx4*>(from + 16);
            y[j] = intx8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
            f[u][j] = scales[mine * U + u];
          }
        } else {
#pragma unroll
          for (int j = 0; j < NC; ++j) y[j] = rows_load(column[j], at, last);
          if (end)
#pragma unroll
            for (int j = 0; j < NC; ++j) rows_clear(y[j], at, a.k);
        }
        if (end)
#pragma unroll
          for (int t = 0; t < RT; ++t) rows_clear(w[u][t], at, a.k);
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const floatx4 z = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[u][t], y[j], floatx4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][j][e] = fmaf(z[e], fp8_lifted(s[u][t][e & (RS - 1)], f[u][j]), acc[t][j][e]);
          }
      }
    }
    if constexpr (RAW) wavefront_turn();             // the next step's codes take these ones' place
  }

  // the wavefronts' sums in order
  floatx4* sums = reinterpret_cast<floatx4*>(lds);
  if (RAW) __syncthreads();                          // everyone has read the codes
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int j = 0; j < NC; ++j) sums[((t * NC + j) * R_WAVES + wave) * 64 + lane] = acc[t][j];
  __syncthreads();
  for (int q = wave; q < RT * NC; q += R_WAVES) {
    floatx4 v = sums[q * R_WAVES * 64 + lane];
#pragma unroll
    for (int i = 1; i < R_WAVES; ++i) v += sums[(q * R_WAVES + i) * 64 + lane];
    const int t = q / NC, j = q - t * NC;
    if (a.splits > 1) reinterpret_cast<floatx4*>(a.part)[((group * RT * NC + q) * a.splits + split) * 64 + lane] = v;
    else rows_store(a, v, r0 + 16 * t + 4 * kg, 16 * j + l16);
  }
}

// The ranges' sums in order.
template <int NC, int RT>
__global__ __launch_bounds__(256) void fp8_rows_join_kernel(RowsArgs a) {
  const int lane = threadIdx.x & 63, l16 = lane & 15, kg = lane >> 4;
  const int64_t q = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (q >= a.row_groups * RT * NC) return;
  const floatx4* part = reinterpret_cast<const floatx4*>(a.part) + q * a.splits * 64 + lane;
  floatx4 v = part[0];
  for (int i = 1; i < a.splits; ++i) v += part[i * 64];
  const int64_t group = q / (RT * NC);
  const int t = (int)(q - group * RT * NC) / NC, j = (int)(q - group * RT * NC) % NC;
  rows_store(a, v, group * 16 * RT + 16 * t + 4 * kg, 16 * j + l16);
}

struct RowsShape { int nc, rt, splits; int64_t groups; };
static RowsShape rows_shape(int64_t rows, int64_t columns, int64_t k) {
  RowsShape s{};
  const int64_t blocks = fp8_blocks(k);
  s.nc = columns <= 16 ? 1 : columns <= 32 ? 2 : columns <= 64 ? 4 : 8;
  s.rt = s.nc > 1 && rows >= 32 * 256 ? 2 : 1;
  // up to 16 columns: eight blocks under way a wavefront also where its share of the sum is shorter, by more rows
  if (s.nc == 1)
    while (s.rt < 4 && blocks * s.rt <= 4 * R_WAVES && rows >= 32 * s.rt * 256) s.rt *= 2;
  s.groups = (rows + 16 * s.rt - 1) / (16 * s.rt);
  // Ranges only where workgroups would leave CUs idle, each wavefront's a step (or half of one, where the columns take their time) at
  // least; their join is a launch: one row, 4096 x 4096, 5.7 us whole and 9.0 in two ranges.
  s.splits = (int)std::max<int64_t>(1, std::min<int64_t>(256 / s.groups, blocks / ((s.nc == 1 ? 8 : 4) * R_WAVES)));
  return s;
}
size_t fp8_product_part_floats(int64_t rows, int64_t columns, int64_t k) {
  if (!few_columns(columns, k)) return fp8_tiles_part_floats(rows, columns, k);
  const RowsShape s = rows_shape(rows, columns, k);
  return s.splits > 1 ? (size_t)s.groups * s.rt * s.nc * s.splits * 256 : 0;
}
bool fp8_needs_codes(int64_t columns) { return columns > RAW_MOST; }
// More of them than RAW_MOST where the sum is short, us so and in two launches: 768 x 768, 9, 16, 32, 64 rows 3.6, 3.9, 5.7, 8.6 and 7.3, 7.5, 8.1,
// 9.2; 4096 x 256, 16, 32, 64 rows 5.3, 8.3, 13.2 and 6.9, 7.2, 7.8 (fewer wavefronts have a part of the sum); 32000 x 1024, 16, 32, 64 rows
// 9.1, 16.9, 24.9 and 13.3, 19.0, 20.0.  Up to 16 rows also several such steps one after the other: 1024 x 2000, 16 rows 6.7 and 8.8, 4096 x 4096
// 10.5 and 12.9, 11008 x 4096 15.1 and 19.1, 4096 x 11008 23.6 and 23.1 (with four blocks a step 9.1, 11.9, 17.5, 31.4).
bool fp8_quantizes_columns(const Fp8Product& p) {
  const int64_t columns = p.columns.count, blocks = fp8_blocks(p.k);
  if (columns <= RAW_MOST) return true;
  if (!p.rows.shift || blocks > 32) return false;
  if (blocks > 2 * R_WAVES) return columns <= 16;
  return columns <= 16 || (columns <= 32 && blocks > 2) || (columns <= 64 && blocks > R_WAVES && p.rows.count < 32 * 256);
}

template <int NC, int RT, int U, bool TILED, int RAWS, typename T>
static int launch(const RowsArgs& a, hipStream_t st) {
  constexpr size_t sums = (size_t)NC * RT * R_WAVES * 1024, most = std::max<size_t>(sums, R_WAVES * x_bytes(RAWS, U));
  const size_t bytes = std::is_void<T>::value ? sums : std::max<size_t>(sums, R_WAVES * x_bytes((int)a.columns.count, U));
  static LdsLimit limit;
  if (most > 65536) LQ_TRY(limit.raise(reinterpret_cast<const void*>(fp8_rows_kernel<NC, RT, U, TILED, RAWS, T>), most));
  hipLaunchKernelGGL((fp8_rows_kernel<NC, RT, U, TILED, RAWS, T>), dim3((unsigned)(a.row_groups * a.splits)), dim3(64 * R_WAVES), bytes, st, a);
  LQ_HIP_TRY(hipGetLastError());
  if (a.splits == 1) return LQ_OK;
  hipLaunchKernelGGL((fp8_rows_join_kernel<NC, RT>), dim3((unsigned)((a.row_groups * NC * RT + 3) / 4)), dim3(256), 0, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}
// Up to 16 columns.  Half as many columns in registers leave room for half as many wavefronts again: one row, 11008 x 4096, bf16 10.1 and
// 11.6 us.
template <int RT, int U, bool TILED>
static int launch_one(const RowsArgs& a, int dtype, hipStream_t st) {
  if (!a.x) return launch<1, RT, U, TILED, 0, void>(a, st);
  if (a.columns.count <= 4) return dtype == LQ_T_BF16 ? launch<1, RT, U, TILED, 4, __bf16>(a, st) : launch<1, RT, U, TILED, 4, float>(a, st);
  return dtype == LQ_T_BF16 ? launch<1, RT, U, TILED, RAW_MOST, __bf16>(a, st) : launch<1, RT, U, TILED, RAW_MOST, float>(a, st);
}
// 9 to 64 columns quantized where they are used, two blocks of the sum a step.
template <int NC, int RT>
static int launch_short(const RowsArgs& a, int dtype, hipStream_t st) {
  return dtype == LQ_T_BF16 ? launch<NC, RT, 2, true, 16 * NC, __bf16>(a, st) : launch<NC, RT, 2, true, 16 * NC, float>(a, st);
}
template <bool TILED>
static int launch_shape(const RowsArgs& a, int nc, int rt, int dtype, hipStream_t st) {
  // no more blocks at once than a wavefront has: the others would be asked for again
  const int share = (a.blocks + a.splits * R_WAVES - 1) / (a.splits * R_WAVES);
  if (a.x && a.columns.count > RAW_MOST) {
    if constexpr (TILED) {
      if (nc == 1) return rt == 4 ? launch_short<1, 4>(a, dtype, st) : rt == 2 ? launch_short<1, 2>(a, dtype, st) : launch_short<1, 1>(a, dtype, st);
      if (nc == 2) return rt == 2 ? launch_short<2, 2>(a, dtype, st) : launch_short<2, 1>(a, dtype, st);
      if (nc == 4 && rt == 1) return launch_short<4, 1>(a, dtype, st);
    }
    return LQ_ERR_SHAPE;
  }
  if (nc == 1) {
    if (rt == 4) return launch_one<4, 2, TILED>(a, dtype, st);
    if (rt == 2) return launch_one<2, 4, TILED>(a, dtype, st);
    return share <= 2 ? launch_one<1, 2, TILED>(a, dtype, st) : share <= 4 ? launch_one<1, 4, TILED>(a, dtype, st) : launch_one<1, 8, TILED>(a, dtype, st);
  }
  if (nc == 2 && share <= 2) return rt == 2 ? launch<2, 2, 2, TILED, 0, void>(a, st) : launch<2, 1, 2, TILED, 0, void>(a, st);
  if (nc == 2) return rt == 2 ? launch<2, 2, 4, TILED, 0, void>(a, st) : launch<2, 1, 4, TILED, 0, void>(a, st);
  if (nc == 4) return rt == 2 ? launch<4, 2, 2, TILED, 0, void>(a, st) : share <= 2 ? launch<4, 1, 2, TILED, 0, void>(a, st) : launch<4, 1, 4, TILED, 0, void>(a, st);
  return rt == 2 ? launch<8, 2, 2, TILED, 0, void>(a, st) : launch<8, 1, 2, TILED, 0, void>(a, st);
}

static int launch_rows(const Fp8Product& p, const void* x, int64_t ldx, int dtype, float* part, size_t part_floats, hipStream_t st) {
  const RowsShape s = rows_shape(p.rows.count, p.columns.count, p.k);
  if (part_floats < fp8_product_part_floats(p.rows.count, p.columns.count, p.k)) return LQ_ERR_WORKSPACE;
  if (s.groups * s.splits >= ((int64_t)1 << 31)) return LQ_ERR_SHAPE;
  const RowsArgs a{p.rows, p.columns, x, ldx, p.k, p.out, p.ld, part, s.groups, s.splits, (int)fp8_blocks(p.k)};
  prof::Scope ps(prof::FP8_ROWS, st, (double)p.rows.count * p.k);
  return p.rows.shift ? launch_shape<true>(a, s.nc, s.rt, dtype, st) : launch_shape<false>(a, s.nc, s.rt, dtype, st);
}

int launch_fp8_product(const Fp8Product& p, float* part, size_t part_floats, hipStream_t st) {
  if (!few_columns(p.columns.count, p.k)) return launch_fp8_tiles(p, part, part_floats, st);
  return launch_rows(p, nullptr, 0, 0, part, part_floats, st);
}
int launch_fp8_product_raw(const Fp8Product& p, const void* x, int64_t ldx, int dtype, float* part, size_t part_floats, hipStream_t st) {
  if (!fp8_quantizes_columns(p)) return LQ_ERR_SHAPE;
  return launch_rows(p, x, ldx, dtype, part, part_floats, st);
}

}  // namespace lq
