// The products of a decomposed layer in training:  T = drop(X) L1,  Y = X Q + T L2,  and backwards  U = dY L2^T,
// dX = dY Q^T + mask .* (U L1^T),  dL1 = drop(X)^T U,  dL2 = T^T dY.
//
// The thin products (rank at most 128) read X or dY once and are bound by that; the mask is worked out where an element is
// loaded (eight neighbours share one call of the generator, and are what a lane holds of an operand).
#include "mfma_device.h"
#include "nf_device.h"
#include "profiler.h"
#include "segment_gemm.h"
#include "train.h"

namespace lq {

// Eight neighbours of a row, masked, as bf16 hi (+ lo for fp32).  group: their index in units of eight.
template <typename T, bool DROP>
__device__ __forceinline__ void masked8(const T* __restrict__ at, const DropoutMask& d, uint64_t group, bf16x8& hi, bf16x8& lo) {
  typedef T vec8 __attribute__((ext_vector_type(8)));
  vec8 v = *reinterpret_cast<const vec8*>(at);
  if constexpr (DROP) {
    const PhiloxWords w = philox_words(d, group);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = philox_kept(w, j, d.cut) ? v[j] : (T)0.0f;
  }
  if constexpr (sizeof(T) == 2) hi = v;
  else {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      bf16x2 h, l;
      split_bf16(floatx2{v[j], v[j + 1]}, h, l);
      hi[j] = h[0]; hi[j + 1] = h[1];
      lo[j] = l[0]; lo[j + 1] = l[1];
    }
  }
}

// ------------------------------------------------------------------------------------------------
// part[z] = drop(A) B^T over a range of the reduction: a wavefront owns 32 rows and all columns; operands go from global memory
// into registers (a lane's eight values of A are eight neighbours, B comes out of the L2).
struct ProjectArgs {
  const void* A; int64_t m, K;
  Planes b; DropoutMask d;
  float* part; int steps, splits;      // steps of 16
};

template <typename T, int RT, bool DROP>
__global__ __launch_bounds__(256) void thin_project_kernel(ProjectArgs a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, ln = lane & 31, lh = lane >> 5;
  const int64_t row0 = ((int64_t)blockIdx.x * 4 + wave) * 32;
  if (row0 >= a.m) return;
  const int64_t row = row0 + ln < a.m ? row0 + ln : a.m - 1;
  const int s0 = (int)((int64_t)a.steps * blockIdx.y / a.splits), s1 = (int)((int64_t)a.steps * (blockIdx.y + 1) / a.splits);
  const T* x = static_cast<const T*>(a.A) + row * a.K;
  const uint64_t group0 = (uint64_t)row * (uint64_t)(a.K >> 3);
  floatx16 acc[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[r][e] = 0.0f;
  for (int s = s0; s < s1; ++s) {
    const int64_t k = 16 * (int64_t)s + 8 * lh;
    const bool in = k < a.K;                          // K is a multiple of 8
    bf16x8 hi = {}, lo = {};
    if (in) masked8<T, DROP>(x + k, a.d, group0 + (uint64_t)(k >> 3), hi, lo);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      bf16x8 bh = {}, bl = {};
      if (in) {
        bh = *reinterpret_cast<const bf16x8*>(a.b.hi + (int64_t)(32 * r + ln) * a.b.pitch + k);
        bl = *reinterpret_cast<const bf16x8*>(a.b.lo + (int64_t)(32 * r + ln) * a.b.pitch + k);
      }
      if constexpr (sizeof(T) == 4) acc[r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo, bh, acc[r], 0, 0, 0);
      acc[r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, bl, acc[r], 0, 0, 0);
      acc[r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, bh, acc[r], 0, 0, 0);
    }
  }
  float* out = a.part + (size_t)blockIdx.y * (size_t)a.m * (32 * RT);
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t o = row0 + 8 * (e >> 2) + 4 * lh + (e & 3);
      if (o < a.m) out[o * (32 * RT) + 32 * r + ln] = acc[r][e];
    }
}

int thin_project_splits(int64_t m, int64_t K) {
  const int64_t wgs = (m + 127) / 128, steps = (K + 15) / 16;
  return (int)std::max<int64_t>(1, std::min<int64_t>({(1024 + wgs - 1) / wgs, steps / 8, 32}));
}

template <typename T, int RT>
static void project(const ProjectArgs& a, bool drop, dim3 grid, hipStream_t st) {
  auto kernel = drop ? thin_project_kernel<T, RT, true> : thin_project_kernel<T, RT, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
}

int launch_thin_project(const void* A, int dtype, int64_t m, int64_t K, const Planes& b, int r32, const DropoutMask* d, float* part,
                        hipStream_t st) {
  if (K < 8 || K % 8 || m < 1 || r32 < 32 || r32 % 32 || r32 > ADAPTER_MAX_RANK) return LQ_ERR_SHAPE;
  ProjectArgs a{};
  a.A = A; a.m = m; a.K = K; a.b = b; a.part = part;
  if (d) a.d = *d;
  a.steps = (int)((K + 15) / 16);
  a.splits = thin_project_splits(m, K);
  const dim3 grid((unsigned)((m + 127) / 128), (unsigned)a.splits);
  prof::Scope ps(prof::THIN_PROJECT, st, (double)m * K * type_bytes(dtype));
  const bool drop = d != nullptr;
  switch ((dtype == LQ_T_BF16 ? 0 : 4) + r32 / 32 - 1) {
    case 0: project<__bf16, 1>(a, drop, grid, st); break;
    case 1: project<__bf16, 2>(a, drop, grid, st); break;
    case 2: project<__bf16, 3>(a, drop, grid, st); break;
    case 3: project<__bf16, 4>(a, drop, grid, st); break;
    case 4: project<float, 1>(a, drop, grid, st); break;
    case 5: project<float, 2>(a, drop, grid, st); break;
    case 6: project<float, 3>(a, drop, grid, st); break;
    default: project<float, 4>(a, drop, grid, st); break;
  }
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
struct FinishArgs {
  const float* part; int splits; int64_t m; int rank, r32; float scale;
  float* T; uint16_t* hi; uint16_t* lo; uint16_t* t_hi; uint16_t* t_lo; int64_t t_pitch;
};

// A workgroup finishes 64 rows x 32 columns of T; the transposed planes go through LDS.
__global__ __launch_bounds__(256) void thin_finish_kernel(FinishArgs a) {
  __shared__ float s_t[64][33];
  const int c = threadIdx.x & 31, r0 = threadIdx.x >> 5, col = blockIdx.y * 32 + c;
  const size_t stride = (size_t)a.m * (size_t)(a.splits ? a.r32 : a.rank);
  for (int r = r0; r < 64; r += 8) {
    const int64_t row = (int64_t)blockIdx.x * 64 + r;
    float v = 0.0f;
    if (row < a.m && col < a.rank) {
      if (a.splits == 0) v = a.part[row * a.rank + col];
      else
        for (int s = 0; s < a.splits; ++s) v += a.part[s * stride + row * a.r32 + col];
      if (a.splits != 0) v *= a.scale;
    }
    s_t[r][c] = v;
    if (row >= a.m) continue;
    if (a.T && col < a.rank) a.T[row * a.rank + col] = v;
    if (a.hi) {
      const __bf16 h = (__bf16)v;
      a.hi[row * a.r32 + col] = __builtin_bit_cast(uint16_t, h);
      a.lo[row * a.r32 + col] = __builtin_bit_cast(uint16_t, (__bf16)(v - (float)h));
    }
  }
  if (!a.t_hi) return;
  __syncthreads();
  const int row = threadIdx.x & 63;
  for (int k = threadIdx.x >> 6; k < 32; k += 4) {
    const float v = s_t[row][k];
    const __bf16 h = (__bf16)v;
    const int64_t at = (int64_t)(blockIdx.y * 32 + k) * a.t_pitch + (int64_t)blockIdx.x * 64 + row;
    a.t_hi[at] = __builtin_bit_cast(uint16_t, h);
    a.t_lo[at] = __builtin_bit_cast(uint16_t, (__bf16)(v - (float)h));
  }
}

int launch_thin_finish(const float* part, int splits, int64_t m, int rank, int r32, float scale, float* T, uint16_t* hi,
                       uint16_t* lo, uint16_t* t_hi, uint16_t* t_lo, int64_t t_pitch, hipStream_t st) {
  if (t_hi && t_pitch < up_to(m, 64)) return LQ_ERR_SHAPE;
  FinishArgs a{part, splits, m, rank, r32, scale, T, hi, lo, t_hi, t_lo, t_pitch};
  prof::Scope ps(prof::THIN_FINISH, st, (double)m * r32 * 4.0 * (splits + 2));
  hipLaunchKernelGGL(thin_finish_kernel, dim3((unsigned)((m + 63) / 64), (unsigned)(r32 / 32)), dim3(256), 0, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// part[z] (K x r32) = drop(A)^T B over a range of rows: a workgroup owns 64 columns of A, turned in LDS so that a lane finds eight
// rows of a column together; two wavefronts take the columns' halves, two more the other half of each 64 rows.
struct GramArgs {
  const void* A; int64_t m, K;
  Planes bt; DropoutMask d;
  float* part; int steps, splits;      // steps of 64 rows
};
constexpr int TG_PITCH = 72;

template <typename T, int RT, bool DROP>
__global__ __launch_bounds__(256) void thin_gram_kernel(GramArgs a) {
  constexpr bool SPLIT = sizeof(T) == 4;
  __shared__ __attribute__((aligned(16))) __bf16 s_a[SPLIT ? 2 : 1][64 * TG_PITCH];     // [hi, lo][column][row]
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, ln = lane & 31, lh = lane >> 5;
  const int64_t c0 = (int64_t)blockIdx.x * 64;
  const int s0 = (int)((int64_t)a.steps * blockIdx.y / a.splits), s1 = (int)((int64_t)a.steps * (blockIdx.y + 1) / a.splits);
  const T* x = static_cast<const T*>(a.A);
  floatx16 acc[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[r][e] = 0.0f;
  for (int s = s0; s < s1; ++s) {
    __syncthreads();                                  // the tile of the step before has been read
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = (tid >> 3) + 32 * h, c = (tid & 7) * 8;
      const int64_t row = 64 * (int64_t)s + r;
      bf16x8 hi = {}, lo = {};
      if (row < a.m && c0 + c < a.K)
        masked8<T, DROP>(x + row * a.K + c0 + c, a.d, (uint64_t)row * (uint64_t)(a.K >> 3) + (uint64_t)((c0 + c) >> 3), hi, lo);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s_a[0][(c + j) * TG_PITCH + r] = hi[j];
        if constexpr (SPLIT) s_a[SPLIT ? 1 : 0][(c + j) * TG_PITCH + r] = lo[j];
      }
    }
    __syncthreads();
    const int col = 32 * (wave & 1) + ln;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int r = 32 * (wave >> 1) + 16 * g + 8 * lh;
      const bf16x8 hi = *reinterpret_cast<const bf16x8*>(&s_a[0][col * TG_PITCH + r]);
      bf16x8 lo = {};
      if constexpr (SPLIT) lo = *reinterpret_cast<const bf16x8*>(&s_a[SPLIT ? 1 : 0][col * TG_PITCH + r]);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int64_t at = (int64_t)(32 * t + ln) * a.bt.pitch + 64 * (int64_t)s + r;
        const bf16x8 bh = *reinterpret_cast<const bf16x8*>(a.bt.hi + at), bl = *reinterpret_cast<const bf16x8*>(a.bt.lo + at);
        if constexpr (SPLIT) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo, bh, acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, bl, acc[t], 0, 0, 0);
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, bh, acc[t], 0, 0, 0);
      }
    }
  }
  float* out = a.part + ((size_t)blockIdx.y * 2 + (wave >> 1)) * (size_t)a.K * (32 * RT);
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t o = c0 + 32 * (wave & 1) + 8 * (e >> 2) + 4 * lh + (e & 3);
      if (o < a.K) out[o * (32 * RT) + 32 * t + ln] = acc[t][e];
    }
}

struct GramSumArgs { const float* part; int parts; int64_t K; int rank, r32; float scale; bool transposed; float* out; };
__global__ __launch_bounds__(256) void thin_gram_sum_kernel(GramSumArgs a) {
  __shared__ float s_t[64][33];
  const int c = threadIdx.x & 31, r0 = threadIdx.x >> 5, col = blockIdx.y * 32 + c;
  const size_t stride = (size_t)a.K * a.r32;
  for (int r = r0; r < 64; r += 8) {
    const int64_t row = (int64_t)blockIdx.x * 64 + r;
    float v = 0.0f;
    if (row < a.K && col < a.rank) {
      for (int s = 0; s < a.parts; ++s) v += a.part[s * stride + row * a.r32 + col];
      v *= a.scale;
      if (!a.transposed) a.out[row * a.rank + col] = v;
    }
    s_t[r][c] = v;
  }
  if (!a.transposed) return;
  __syncthreads();
  const int r = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 64 + r;
  for (int k = threadIdx.x >> 6; k < 32; k += 4)
    if (row < a.K && (int)(blockIdx.y * 32 + k) < a.rank) a.out[(int64_t)(blockIdx.y * 32 + k) * a.K + row] = s_t[r][k];
}

int thin_gram_splits(int64_t m, int64_t K) {
  const int64_t wgs = (K + 63) / 64, steps = (m + 63) / 64;
  return (int)std::max<int64_t>(1, std::min<int64_t>({(1024 + wgs - 1) / wgs, steps, 16}));
}

template <typename T, int RT>
static void gram(const GramArgs& a, bool drop, dim3 grid, hipStream_t st) {
  auto kernel = drop ? thin_gram_kernel<T, RT, true> : thin_gram_kernel<T, RT, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
}

int launch_thin_gram(const void* A, int dtype, int64_t m, int64_t K, const Planes& bt, int rank, int r32, const DropoutMask* d,
                     float scale, bool transposed, float* part, float* out, hipStream_t st) {
  if (K < 8 || K % 8 || m < 1 || r32 < 32 || r32 % 32 || r32 > ADAPTER_MAX_RANK || bt.pitch < up_to(m, 64)) return LQ_ERR_SHAPE;
  GramArgs a{};
  a.A = A; a.m = m; a.K = K; a.bt = bt; a.part = part;
  if (d) a.d = *d;
  a.steps = (int)((m + 63) / 64);
  a.splits = thin_gram_splits(m, K);
  const dim3 grid((unsigned)((K + 63) / 64), (unsigned)a.splits);
  const bool drop = d != nullptr;
  {
    prof::Scope ps(prof::THIN_GRAM, st, (double)m * K * type_bytes(dtype));
    switch ((dtype == LQ_T_BF16 ? 0 : 4) + r32 / 32 - 1) {
      case 0: gram<__bf16, 1>(a, drop, grid, st); break;
      case 1: gram<__bf16, 2>(a, drop, grid, st); break;
      case 2: gram<__bf16, 3>(a, drop, grid, st); break;
      case 3: gram<__bf16, 4>(a, drop, grid, st); break;
      case 4: gram<float, 1>(a, drop, grid, st); break;
      case 5: gram<float, 2>(a, drop, grid, st); break;
      case 6: gram<float, 3>(a, drop, grid, st); break;
      default: gram<float, 4>(a, drop, grid, st); break;
    }
    LQ_HIP_TRY(hipGetLastError());
  }
  GramSumArgs g{part, 2 * a.splits, K, rank, r32, scale, transposed, out};
  prof::Scope ps(prof::THIN_FINISH, st, (double)K * r32 * 4.0 * (g.parts + 1));
  hipLaunchKernelGGL(thin_gram_sum_kernel, dim3((unsigned)((K + 63) / 64), (unsigned)(r32 / 32)), dim3(256), 0, st, g);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// The stored weights as planes, row by row: 16 weights a thread.
struct WeightRowsArgs {
  const uint8_t* codes; const uint8_t* sidx; const float* v;
  int64_t K, N, pitch;
  uint16_t* hi; uint16_t* lo;
  int block_shift, group_shift, levels; float inv_levels;
  const DevTables* tables;
};

template <int BITS>
__global__ __launch_bounds__(256) void weight_rows_kernel(WeightRowsArgs a) {
  __shared__ float s_code[1 << BITS];
  for (int i = threadIdx.x; i < (1 << BITS); i += 256) s_code[i] = a.tables->code[Slot<BITS>::value][i];
  __syncthreads();
  const int64_t runs = (a.N + 31) / 32 * 2, total = a.K * runs;       // runs of 16 up to a multiple of 32 weights
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
    const int64_t row = u / runs, c = (u - row * runs) * 16;
    float w[16];
    if (c < a.N) {
      const int64_t e = row * a.N + c, blk = e >> a.block_shift;
      uint32_t code[16];
      load_codes<BITS>(a.codes, e >> 4, code);
      const float scale = block_scale_by_reciprocal(a.sidx[blk], a.v[blk >> a.group_shift], a.levels, a.inv_levels);
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = s_code[code[j]] * scale;
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = 0.0f;
    }
    bf16x8 hi[2], lo[2];
#pragma unroll
    for (int j = 0; j < 16; j += 2) {
      bf16x2 h, l;
      split_bf16(floatx2{w[j], w[j + 1]}, h, l);
      hi[j >> 3][j & 7] = h[0]; hi[j >> 3][(j & 7) + 1] = h[1];
      lo[j >> 3][j & 7] = l[0]; lo[j >> 3][(j & 7) + 1] = l[1];
    }
    bf16x8* o = reinterpret_cast<bf16x8*>(a.hi + row * a.pitch + c);
    o[0] = hi[0]; o[1] = hi[1];
    if (a.lo) {
      o = reinterpret_cast<bf16x8*>(a.lo + row * a.pitch + c);
      o[0] = lo[0]; o[1] = lo[1];
    }
  }
}

int launch_weight_rows(const MvWeights& q, int64_t K, int64_t N, uint16_t* hi, uint16_t* lo, int64_t pitch, hipStream_t st) {
  if (N % 16 || pitch % 8 || pitch < up_to(N, 32)) return LQ_ERR_SHAPE;
  if (q.block < 16 || (q.block & (q.block - 1)) || q.scale_block < 1 || (q.scale_block & (q.scale_block - 1)) || N % q.block)
    return LQ_ERR_CONFIG;
  WeightRowsArgs a{};
  a.codes = q.codes; a.sidx = q.sidx; a.v = q.v; a.K = K; a.N = N; a.pitch = pitch; a.hi = hi; a.lo = lo;
  a.block_shift = __builtin_ctz((unsigned)q.block);
  a.group_shift = __builtin_ctz((unsigned)q.scale_block);
  a.levels = q.levels;
  a.inv_levels = 1.0f / (float)q.levels;
  LQ_TRY(device_tables(&a.tables));
  const dim3 grid((unsigned)std::min<int64_t>((K * (N / 16) + 255) / 256, 1 << 14));
  prof::Scope ps(prof::WEIGHT_PLANE, st, (double)K * (double)N * (q.bits / 8.0 + (lo ? 4.0 : 2.0)));
  switch (q.bits) {
    case 2: hipLaunchKernelGGL(weight_rows_kernel<2>, grid, dim3(256), 0, st, a); break;
    case 3: hipLaunchKernelGGL(weight_rows_kernel<3>, grid, dim3(256), 0, st, a); break;
    case 4: hipLaunchKernelGGL(weight_rows_kernel<4>, grid, dim3(256), 0, st, a); break;
    case 8: hipLaunchKernelGGL(weight_rows_kernel<8>, grid, dim3(256), 0, st, a); break;
    default: return LQ_ERR_CONFIG;
  }
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// out = A B^T from up to six segments.
struct ProductArgs {
  SegArgs g;
  int64_t rows, cols;
  void* out; float* part;
};

template <typename T>
__global__ __launch_bounds__(SEG_THREADS) void plain_product_kernel(ProductArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const SegTile t = seg_tile(a.g);
  if (!t.live) return;
  floatx16 acc[4][2];
  seg_clear(acc);
  const int steps = a.g.seg[5].end;
  seg_products(a.g, t, (int)((int64_t)steps * t.split / a.g.splits), (int)((int64_t)steps * (t.split + 1) / a.g.splits), seg_lds, acc);
  float* part = a.part + (size_t)t.split * (size_t)a.rows * (size_t)a.cols;
  seg_each(t, [&](int i, int j, int e, int64_t row, int64_t col) {
    if (row >= a.rows || col >= a.cols) return;
    if (a.g.splits > 1) part[row * a.cols + col] = acc[i][j][e];
    else static_cast<T*>(a.out)[row * a.cols + col] = (T)acc[i][j][e];
  });
}

template <typename T>
__global__ __launch_bounds__(256) void part_sum_kernel(const float* __restrict__ part, int splits, int64_t total, T* __restrict__ out) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    float v = 0.0f;
    for (int s = 0; s < splits; ++s) v += part[s * total + i];
    out[i] = (T)v;
  }
}

static int launch_part_sum(const float* part, int splits, int64_t total, int dtype, void* out, hipStream_t st) {
  prof::Scope ps(prof::THIN_FINISH, st, (double)total * (4.0 * splits + type_bytes(dtype)));
  const dim3 grid((unsigned)std::min<int64_t>((total + 255) / 256, 8192));
  if (dtype == LQ_T_BF16)
    hipLaunchKernelGGL(part_sum_kernel<__bf16>, grid, dim3(256), 0, st, part, splits, total, static_cast<__bf16*>(out));
  else
    hipLaunchKernelGGL(part_sum_kernel<float>, grid, dim3(256), 0, st, part, splits, total, static_cast<float*>(out));
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

static int64_t tiles_of(int64_t rows, int64_t cols) { return ((rows + SEG_T - 1) / SEG_T) * ((cols + SEG_T - 1) / SEG_T); }

int plain_product_splits(int64_t rows, int64_t cols, int64_t depth, int planes) {
  return seg_splits(tiles_of(rows, cols), (int)(depth / 32) * (planes == 2 ? 3 : 1), 16);
}

static int tile_grid(SegArgs& g, int64_t rows, int64_t cols, int splits) {
  if (tiles_of(rows, cols) * splits >= (1ll << 30)) return LQ_ERR_SHAPE;
  g.rows_a = rows; g.rows_b = cols; g.splits = splits;
  g.tiles_m = (int)((rows + SEG_T - 1) / SEG_T); g.tiles_n = (int)((cols + SEG_T - 1) / SEG_T);
  return LQ_OK;
}

int launch_plain_product(const Planes& a, const Planes& b, int64_t depth, const Planes& a2, const Planes& b2, int64_t depth2,
                         int64_t rows, int64_t cols, int dtype, void* out, float* part, size_t part_floats, hipStream_t st) {
  if (depth < 32 || depth % 32 || depth2 % 32) return LQ_ERR_SHAPE;
  ProductArgs p{};
  int count = 0, end = add_segments(p.g, &count, 0, a, b, depth);
  if (depth2 > 0) end = add_segments(p.g, &count, end, a2, b2, depth2);
  for (; count < 6; ++count) { p.g.seg[count] = p.g.seg[0]; p.g.seg[count].end = end; }
  LQ_TRY(tile_grid(p.g, rows, cols, plain_product_splits(rows, cols, depth, a.lo || b.lo ? 2 : 1)));
  if (p.g.splits > 1 && part_floats < (size_t)p.g.splits * (size_t)rows * (size_t)cols) return LQ_ERR_WORKSPACE;
  p.rows = rows; p.cols = cols; p.out = out; p.part = part;
  {
    prof::Scope ps(prof::SEGMENT_GEMM, st, 2.0 * rows * cols * (depth + depth2));
    if (dtype == LQ_T_BF16) {
      static LdsLimit limit;
      LQ_TRY(limit.raise(reinterpret_cast<const void*>(plain_product_kernel<__bf16>), SEG_LDS));
      hipLaunchKernelGGL(plain_product_kernel<__bf16>, dim3(seg_grid(p.g)), dim3(SEG_THREADS), SEG_LDS, st, p);
    } else {
      static LdsLimit limit;
      LQ_TRY(limit.raise(reinterpret_cast<const void*>(plain_product_kernel<float>), SEG_LDS));
      hipLaunchKernelGGL(plain_product_kernel<float>, dim3(seg_grid(p.g)), dim3(SEG_THREADS), SEG_LDS, st, p);
    }
    LQ_HIP_TRY(hipGetLastError());
  }
  return p.g.splits > 1 ? launch_part_sum(part, p.g.splits, rows * cols, dtype, out, st) : LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// dX: the low-rank part goes into the accumulators first and is masked there, then the weights' part is added to it: no second
// set of accumulators, no array of U L1^T.  Features are the tile's rows and tokens its columns, so that a lane holds four
// neighbouring features of a token and its other half the next four: a group of the generator.
struct DxArgs {
  SegArgs g, low;
  int64_t m, d;
  DropoutMask mask;
  void* out; float* part;
};

template <typename T>
__global__ __launch_bounds__(SEG_THREADS) void adapter_dx_kernel(DxArgs a) {
  typedef T vec4 __attribute__((ext_vector_type(4)));
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const SegTile t = seg_tile(a.g);
  if (!t.live) return;
  floatx16 acc[4][2];
  seg_clear(acc);
  const int64_t row0 = (int64_t)t.tm * SEG_T + 128 * t.wm, col0 = (int64_t)t.tn * SEG_T + 64 * t.wn + t.ln;
  if (t.split == 0) {
    seg_products(a.low, t, 0, a.low.seg[2].end, seg_lds, acc);
    if (a.mask.cut > 0) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint64_t group = (uint64_t)(col0 + 32 * j) * (uint64_t)(a.d >> 3) + (uint64_t)(row0 >> 3);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const PhiloxWords w = philox_words(a.mask, group + 4 * i + q);
            const uint32_t w0 = t.lh ? w.w[2] : w.w[0], w1 = t.lh ? w.w[3] : w.w[1];
            floatx16& v = acc[i][j];
            v[4 * q + 0] = (w0 & 0xffffu) >= a.mask.cut ? v[4 * q + 0] * a.mask.scale : 0.0f;
            v[4 * q + 1] = (w0 >> 16) >= a.mask.cut ? v[4 * q + 1] * a.mask.scale : 0.0f;
            v[4 * q + 2] = (w1 & 0xffffu) >= a.mask.cut ? v[4 * q + 2] * a.mask.scale : 0.0f;
            v[4 * q + 3] = (w1 >> 16) >= a.mask.cut ? v[4 * q + 3] * a.mask.scale : 0.0f;
          }
      }
    }
    __syncthreads();                                  // the LDS has been read by everyone
  }
  const int steps = a.g.seg[2].end;
  seg_products(a.g, t, (int)((int64_t)steps * t.split / a.g.splits), (int)((int64_t)steps * (t.split + 1) / a.g.splits), seg_lds, acc);
  float* part = a.part + (size_t)t.split * (size_t)a.m * (size_t)a.d;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int64_t token = col0 + 32 * j;
    if (token >= a.m) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t row = row0 + 32 * i + 8 * q + 4 * t.lh;
        if (row >= a.d) continue;                     // d is a multiple of 32
        const floatx4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        if (a.g.splits > 1) *reinterpret_cast<floatx4*>(part + token * a.d + row) = v;
        else *reinterpret_cast<vec4*>(static_cast<T*>(a.out) + token * a.d + row) = __builtin_convertvector(v, vec4);
      }
  }
}

int adapter_dx_splits(int64_t m, int64_t d, int64_t k, int planes) { return plain_product_splits(d, m, up_to(k, 32), planes); }

int launch_adapter_dx(const Planes& q, const Planes& dy, int64_t depth, const Planes& l1, const Planes& u, int r32, int64_t m,
                      int64_t d, const DropoutMask& mask, int dtype, void* dX, float* part, size_t part_floats, hipStream_t st) {
  if (depth < 32 || depth % 32 || d % 32 || r32 < 32 || r32 % 32) return LQ_ERR_SHAPE;
  DxArgs a{};
  int count = 0, end = add_segments(a.g, &count, 0, q, dy, depth);
  for (; count < 6; ++count) { a.g.seg[count] = a.g.seg[0]; a.g.seg[count].end = end; }
  count = 0;
  end = add_segments(a.low, &count, 0, l1, u, r32);
  for (; count < 6; ++count) { a.low.seg[count] = a.low.seg[0]; a.low.seg[count].end = end; }
  const int splits = adapter_dx_splits(m, d, depth, q.lo ? 2 : 1);
  LQ_TRY(tile_grid(a.g, d, m, splits));
  LQ_TRY(tile_grid(a.low, d, m, splits));
  if (splits > 1 && part_floats < (size_t)splits * (size_t)m * (size_t)d) return LQ_ERR_WORKSPACE;
  a.m = m; a.d = d; a.mask = mask; a.out = dX; a.part = part;
  {
    prof::Scope ps(prof::SEGMENT_GEMM, st, 2.0 * m * d * (depth + r32));
    if (dtype == LQ_T_BF16) {
      static LdsLimit limit;
      LQ_TRY(limit.raise(reinterpret_cast<const void*>(adapter_dx_kernel<__bf16>), SEG_LDS));
      hipLaunchKernelGGL(adapter_dx_kernel<__bf16>, dim3(seg_grid(a.g)), dim3(SEG_THREADS), SEG_LDS, st, a);
    } else {
      static LdsLimit limit;
      LQ_TRY(limit.raise(reinterpret_cast<const void*>(adapter_dx_kernel<float>), SEG_LDS));
      hipLaunchKernelGGL(adapter_dx_kernel<float>, dim3(seg_grid(a.g)), dim3(SEG_THREADS), SEG_LDS, st, a);
    }
    LQ_HIP_TRY(hipGetLastError());
  }
  return splits > 1 ? launch_part_sum(part, splits, m * d, dtype, dX, st) : LQ_OK;
}

}  // namespace lq
