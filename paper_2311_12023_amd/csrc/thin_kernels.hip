// The thin products of a decomposed layer in training (rank at most 128):  T = drop(X) L1,  U = dY L2^T,  dL1 = drop(X)^T U,
// dL2 = T^T dY.  They read X or dY once and are bound by that and by the operands of the other side, which every workgroup reads.
// The mask is worked out where an element is loaded (the eight neighbours that share a call of the generator are what a lane loads).
// Their results are fp32 whatever the type of X: L1, L2, T and U go in as three bf16 planes, X and dY as one where they are bf16
// and three where they are fp32.
#include "half_planes_device.h"
#include "lds_transfer.h"
#include "mfma_device.h"
#include "profiler.h"
#include "train.h"

namespace lq {

template <typename T> constexpr int thin_planes() { return sizeof(T) == 2 ? 1 : 3; }

// Eight neighbours of a row as a lane loads them.
template <typename T>
struct Eight { typedef T vec8 __attribute__((ext_vector_type(8))); vec8 v; };

template <typename T, bool DROP>
__device__ __forceinline__ void apply_mask(Eight<T>& x, const DropoutMask& d, uint64_t group) {
  if constexpr (DROP) {
    const PhiloxWords w = philox_words(d, group);
#pragma unroll
    for (int j = 0; j < 8; ++j) x.v[j] = philox_kept(w, j, d.cut) ? x.v[j] : (T)0.0f;
  }
}

template <typename T>
__device__ __forceinline__ void to_planes(const Eight<T>& x, bf16x8 (&p)[thin_planes<T>()]) {
  if constexpr (sizeof(T) == 2) p[0] = x.v;
  else {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      bf16x2 s[3];
      split_bf16_3(floatx2{x.v[j], x.v[j + 1]}, s);
#pragma unroll
      for (int k = 0; k < 3; ++k) { p[k][j] = s[k][0]; p[k][j + 1] = s[k][1]; }
    }
  }
}

// acc += a b over the products of planes that count, the smallest first.
template <int NA>
__device__ __forceinline__ void thin_multiply(const bf16x8 (&a)[NA], const bf16x8 (&b)[3], floatx4& acc) {
#pragma unroll
  for (int s = 2; s >= 0; --s)
#pragma unroll
    for (int k = 0; k < NA; ++k)
      if (s - k >= 0) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[k], b[s - k], acc, 0, 0, 0);
}

// The other operand's step: 64 reduction indices of r32 rows of three planes, straight into LDS, rows of 128 bytes with unit u of
// a row at u ^ (row % 8): the 16 rows of an operand read meet different banks.
template <int RT>
constexpr uint32_t thin_stage() { return 3u * RT * 16 * 128; }
template <int RT>
__device__ __forceinline__ void thin_transfer(const Planes& b, int64_t k, uint32_t lds, int wave, int lane) {
#pragma unroll
  for (int q = 0; q < (3 * RT * 2 + 3) / 4; ++q) {                 // pieces of eight rows, dealt to the four wavefronts
    const int piece = 4 * q + wave;
    if (piece >= 3 * RT * 2) break;
    const int plane = piece / (RT * 2), row = (piece - plane * (RT * 2)) * 8 + (lane >> 3), unit = (lane & 7) ^ (row & 7);
    transfer_to_lds(b.p[plane] + k, (uint32_t)(row * b.pitch * 2 + unit * 16), lds + (uint32_t)piece * 1024u);
  }
}
template <int RT>
__device__ __forceinline__ void thin_read(const unsigned char* lds, int r, int sub, int l16, int kg, bf16x8 (&b)[3]) {
#pragma unroll
  for (int k = 0; k < 3; ++k)
    b[k] = *reinterpret_cast<const bf16x8*>(lds + (uint32_t)(k * RT * 16 + 16 * r + l16) * 128u + (uint32_t)((4 * sub + kg) ^ (l16 & 7)) * 16u);
}

// ------------------------------------------------------------------------------------------------
// part[z] = drop(A) B^T over a range of the reduction, in steps of 64.  A workgroup owns 128 rows, a wavefront 32; A goes from global
// memory into registers, a step ahead; B through two LDS stages, shared.
struct ProjectArgs {
  const void* A; int64_t m, K;
  Planes b; DropoutMask d;
  float* part; int steps, splits;
};

template <typename T, int RT, bool DROP>
__global__ __launch_bounds__(256) void thin_project_kernel(ProjectArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char thin_lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l16 = lane & 15, kg = lane >> 4;
  const int64_t row0 = (int64_t)blockIdx.x * 128 + 32 * wave;
  const int s0 = (int)((int64_t)a.steps * blockIdx.y / a.splits), s1 = (int)((int64_t)a.steps * (blockIdx.y + 1) / a.splits);
  const T* x[2];
  uint64_t group[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t r = row0 + 16 * h + l16, row = r < a.m ? r : a.m - 1;
    x[h] = static_cast<const T*>(a.A) + row * a.K;
    group[h] = (uint64_t)row * (uint64_t)(a.K >> 3);
  }
  floatx4 acc[2][RT];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[h][r] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  Eight<T> v[2][2];                                   // [half of the step][row tile]
  auto load = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      const int64_t k = 64 * (int64_t)s + 32 * sub + 8 * kg;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        v[sub][h].v = {};
        if (k < a.K) v[sub][h].v = *reinterpret_cast<const typename Eight<T>::vec8*>(x[h] + k);      // K is a multiple of 8
      }
    }
  };
  if (s0 < s1) {
    thin_transfer<RT>(a.b, 64 * (int64_t)s0, 0, wave, lane);
    load(s0);
  }
  for (int s = s0; s < s1; ++s) {
    const uint32_t stage = (uint32_t)((s - s0) & 1) * thin_stage<RT>();
    bf16x8 p[2][2][thin_planes<T>()];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        apply_mask<T, DROP>(v[sub][h], a.d, group[h] + (uint64_t)(8 * (int64_t)s + 4 * sub + kg));
        to_planes<T>(v[sub][h], p[sub][h]);
      }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                                  // this step's B is there, and the other stage has been read
    if (s + 1 < s1) {
      thin_transfer<RT>(a.b, 64 * (int64_t)(s + 1), thin_stage<RT>() - stage, wave, lane);
      load(s + 1);
    }
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        bf16x8 b[3];
        thin_read<RT>(thin_lds + stage, r, sub, l16, kg, b);
#pragma unroll
        for (int h = 0; h < 2; ++h) thin_multiply<thin_planes<T>()>(p[sub][h], b, acc[h][r]);
      }
  }
  float* out = a.part + (size_t)blockIdx.y * (size_t)a.m * (16 * RT);
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t o = row0 + 16 * h + 4 * kg + e;
      if (o < a.m) {
#pragma unroll
        for (int r = 0; r < RT; ++r) out[o * (16 * RT) + 16 * r + l16] = acc[h][r][e];
      }
    }
}

// Two workgroups a CU; a range keeps four steps.
int thin_project_splits(int64_t m, int64_t K) {
  const int64_t wgs = (m + 127) / 128, steps = (K + 63) / 64;
  return (int)std::max<int64_t>(1, std::min<int64_t>({(512 + wgs - 1) / wgs, steps / 4, 32}));
}

template <typename T, int RT, bool DROP>
static int project(const ProjectArgs& a, dim3 grid, hipStream_t st) {
  static LdsLimit limit;
  constexpr size_t lds = 2 * thin_stage<RT>();
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
  a.A = A; a.m = m; a.K = K; a.b = b; a.part = part;
  if (d) a.d = *d;
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
// part[z] (K x r32) = drop(A)^T B over a range of rows, in steps of 64.  A workgroup owns 128 columns of A, a wavefront 32.  A thread
// loads four rows of eight columns, a step ahead, and writes them turned, four rows of a column at a time, into LDS rows of 64 + 8.
struct GramArgs {
  const void* A; int64_t m, K;
  Planes bt; DropoutMask d;
  float* part; int steps, splits;
};
constexpr int TG_PITCH = 72;
template <typename T, int RT>
constexpr uint32_t gram_lds() { return 2 * thin_stage<RT>() + thin_planes<T>() * 128u * TG_PITCH * 2u; }

template <typename T, int RT, bool DROP>
__global__ __launch_bounds__(256) void thin_gram_kernel(GramArgs a) {
  constexpr int NP = thin_planes<T>();
  extern __shared__ __attribute__((aligned(16))) unsigned char thin_lds[];
  __bf16* s_a = reinterpret_cast<__bf16*>(thin_lds + 2 * thin_stage<RT>());             // [plane][column][row]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l16 = lane & 15, kg = lane >> 4;
  const int c8 = (threadIdx.x & 15) * 8, r4 = (threadIdx.x >> 4) * 4;
  const int64_t c0 = (int64_t)blockIdx.x * 128;
  const int s0 = (int)((int64_t)a.steps * blockIdx.y / a.splits), s1 = (int)((int64_t)a.steps * (blockIdx.y + 1) / a.splits);
  const bool in = c0 + c8 < a.K;                                                        // K is a multiple of 8
  const T* x = static_cast<const T*>(a.A) + c0 + c8;
  floatx4 acc[2][RT];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[h][r] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  Eight<T> v[4];
  auto load = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t row = 64 * (int64_t)s + r4 + q;
      v[q].v = {};
      if (in && row < a.m) v[q].v = *reinterpret_cast<const typename Eight<T>::vec8*>(x + row * a.K);
    }
  };
  if (s0 < s1) {
    thin_transfer<RT>(a.bt, 64 * (int64_t)s0, 0, wave, lane);
    load(s0);
  }
  for (int s = s0; s < s1; ++s) {
    const uint32_t stage = (uint32_t)((s - s0) & 1) * thin_stage<RT>();
    bf16x8 p[4][NP];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t row = 64 * (int64_t)s + r4 + q;
      apply_mask<T, DROP>(v[q], a.d, (uint64_t)row * (uint64_t)(a.K >> 3) + (uint64_t)((c0 + c8) >> 3));
      to_planes<T>(v[q], p[q]);
    }
    __syncthreads();                                  // the tile of the step before has been read
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *reinterpret_cast<bf16x4*>(s_a + (k * 128 + c8 + j) * TG_PITCH + r4) = bf16x4{p[0][k][j], p[1][k][j], p[2][k][j], p[3][k][j]};
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                                  // this step's tile and B are there
    if (s + 1 < s1) {
      thin_transfer<RT>(a.bt, 64 * (int64_t)(s + 1), thin_stage<RT>() - stage, wave, lane);
      load(s + 1);
    }
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      bf16x8 t[2][NP];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < NP; ++k)
          t[h][k] = *reinterpret_cast<const bf16x8*>(s_a + (k * 128 + 32 * wave + 16 * h + l16) * TG_PITCH + 32 * sub + 8 * kg);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        bf16x8 b[3];
        thin_read<RT>(thin_lds + stage, r, sub, l16, kg, b);
#pragma unroll
        for (int h = 0; h < 2; ++h) thin_multiply<NP>(t[h], b, acc[h][r]);
      }
    }
  }
  float* out = a.part + (size_t)blockIdx.y * (size_t)a.K * (16 * RT);
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t o = c0 + 32 * wave + 16 * h + 4 * kg + e;
      if (o < a.K) {
#pragma unroll
        for (int r = 0; r < RT; ++r) out[o * (16 * RT) + 16 * r + l16] = acc[h][r][e];
      }
    }
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
  constexpr size_t lds = gram_lds<T, RT>();
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
  a.A = A; a.m = m; a.K = K; a.bt = bt; a.part = part;
  if (d) a.d = *d;
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
