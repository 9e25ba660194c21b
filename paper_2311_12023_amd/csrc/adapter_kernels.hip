// The large product of a decomposed layer in training:  Y = X Q + T L2  and  dX = dY Q^T + mask .* (U L1^T).
#include "half_planes_device.h"
#include "mfma_device.h"
#include "nf_device.h"
#include "profiler.h"
#include "segment_gemm.h"
#include "train.h"

namespace lq {

// ------------------------------------------------------------------------------------------------
// The stored weights as planes, 16 weights a thread and row.  bf16 activations meet weights rounded to bf16 (2^-9, as much as their
// results are rounded by), fp32 ones meet two fp16 planes.
struct WeightArgs {
  const uint8_t* codes; const uint8_t* sidx; const float* v;
  int64_t K, N, pitch;
  uint16_t* hi; uint16_t* lo;
  int block_shift, group_shift, levels; float inv_levels;
  const DevTables* tables; const uint32_t* top;
};

template <int BITS>
__device__ __forceinline__ void decode_run(const WeightArgs& a, const float* s_code, int64_t row, int64_t c, float scale, float (&w)[16]) {
  const int64_t e = row * a.N + c, blk = e >> a.block_shift;
  uint32_t code[16];
  load_codes<BITS>(a.codes, e >> 4, code);
  const float s = block_scale_by_reciprocal(a.sidx[blk], a.v[blk >> a.group_shift], a.levels, a.inv_levels);
#pragma unroll
  for (int j = 0; j < 16; ++j) w[j] = s_code[code[j]] * s * scale;
}

template <int BITS>
__device__ __forceinline__ void load_codebook(const WeightArgs& a, float* s_code) {
  for (int i = threadIdx.x; i < (1 << BITS); i += 256) s_code[i] = a.tables->code[Slot<BITS>::value][i];
  __syncthreads();
}

// Two values as they lie in the planes.
template <bool HALF>
__device__ __forceinline__ void weight_pair(float a, float b, uint32_t& hi, uint32_t& lo) {
  if constexpr (HALF) {
    typedef _Float16 half2 __attribute__((ext_vector_type(2)));
    const HalfPair p = split_half(a), q = split_half(b);
    hi = __builtin_bit_cast(uint32_t, half2{p.hi, q.hi});
    lo = __builtin_bit_cast(uint32_t, half2{p.lo, q.lo});
  } else {
    hi = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, b}, bf16x2));
    lo = 0;
  }
}

template <int BITS, bool HALF>
__global__ __launch_bounds__(256) void weight_rows_kernel(WeightArgs a) {
  __shared__ float s_code[1 << BITS];
  load_codebook<BITS>(a, s_code);
  const float scale = HALF ? power_of_two(half_exponent_of(a.top, TOP_WORDS)) : 1.0f;
  const int64_t runs = (a.N + 63) / 64 * 4, total = a.K * runs;       // runs of 16 up to a multiple of 64 weights
  for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
    const int64_t row = u / runs, c = (u - row * runs) * 16;
    float w[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = 0.0f;
    if (c < a.N) decode_run<BITS>(a, s_code, row, c, scale, w);
    uintx4 hi[2], lo[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t h, l;
      weight_pair<HALF>(w[2 * j], w[2 * j + 1], h, l);
      hi[j >> 2][j & 3] = h; lo[j >> 2][j & 3] = l;
    }
    uintx4* o = reinterpret_cast<uintx4*>(a.hi + row * a.pitch + c);
    o[0] = hi[0]; o[1] = hi[1];
    if constexpr (HALF) {
      o = reinterpret_cast<uintx4*>(a.lo + row * a.pitch + c);
      o[0] = lo[0]; o[1] = lo[1];
    }
  }
}

// Transposed: a workgroup decodes 64 rows x 128 columns, a thread two rows of 16, and turns them in LDS.
constexpr int WC_K = 64, WC_N = 128, WC_WORDS = 33;
template <int BITS, bool HALF>
__global__ __launch_bounds__(256) void weight_columns_kernel(WeightArgs a) {
  __shared__ float s_code[1 << BITS];
  __shared__ uint32_t s_w[HALF ? 2 : 1][WC_N * WC_WORDS];
  load_codebook<BITS>(a, s_code);
  const float scale = HALF ? power_of_two(half_exponent_of(a.top, TOP_WORDS)) : 1.0f;
  const int tid = threadIdx.x, run = tid & 7, pair = tid >> 3;
  const int64_t n0 = (int64_t)blockIdx.x * WC_N, k0 = (int64_t)blockIdx.y * WC_K, col = n0 + 16 * run;
  float w[2][16];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int j = 0; j < 16; ++j) w[h][j] = 0.0f;
    const int64_t k = k0 + 2 * pair + h;
    if (k < a.K && col < a.N) decode_run<BITS>(a, s_code, k, col, scale, w[h]);      // N is a multiple of 16
  }
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    uint32_t h, l;
    weight_pair<HALF>(w[0][j], w[1][j], h, l);
    s_w[0][(16 * run + j) * WC_WORDS + pair] = h;
    if constexpr (HALF) s_w[HALF ? 1 : 0][(16 * run + j) * WC_WORDS + pair] = l;
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < WC_N / 32; ++h) {
    const int n = (tid >> 3) + 32 * h, word = (tid & 7) * 4;
    if (n0 + n >= a.N) continue;
    uintx4 out;
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = s_w[0][n * WC_WORDS + word + j];
    *reinterpret_cast<uintx4*>(a.hi + (n0 + n) * a.pitch + k0 + 2 * word) = out;
    if constexpr (HALF) {
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = s_w[HALF ? 1 : 0][n * WC_WORDS + word + j];
      *reinterpret_cast<uintx4*>(a.lo + (n0 + n) * a.pitch + k0 + 2 * word) = out;
    }
  }
}

template <int BITS>
static void launch_weights(const WeightArgs& a, bool transposed, hipStream_t st) {
  if (transposed) {
    auto kernel = a.lo ? weight_columns_kernel<BITS, true> : weight_columns_kernel<BITS, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.N + WC_N - 1) / WC_N), (unsigned)((a.K + WC_K - 1) / WC_K)), dim3(256), 0, st, a);
  } else {
    auto kernel = a.lo ? weight_rows_kernel<BITS, true> : weight_rows_kernel<BITS, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>((a.K * (a.N / 16) + 255) / 256, 1 << 14)), dim3(256), 0, st, a);
  }
}

int launch_weight_planes(const MvWeights& q, int64_t K, int64_t N, bool transposed, const uint32_t* top, uint16_t* hi, uint16_t* lo,
                         int64_t pitch, hipStream_t st) {
  if (N % 16 || pitch % 64 || pitch < (transposed ? K : N) || (K + WC_K - 1) / WC_K > 65535 * 64ll) return LQ_ERR_SHAPE;
  if (transposed && (K + WC_K - 1) / WC_K > 65535) return LQ_ERR_SHAPE;
  if (q.block < 16 || (q.block & (q.block - 1)) || q.scale_block < 1 || (q.scale_block & (q.scale_block - 1)) || N % q.block)
    return LQ_ERR_CONFIG;
  if (lo && !top) return LQ_ERR_NULL;
  WeightArgs a{};
  a.codes = q.codes; a.sidx = q.sidx; a.v = q.v; a.K = K; a.N = N; a.pitch = pitch; a.hi = hi; a.lo = lo; a.top = top;
  a.block_shift = __builtin_ctz((unsigned)q.block);
  a.group_shift = __builtin_ctz((unsigned)q.scale_block);
  a.levels = q.levels;
  a.inv_levels = 1.0f / (float)q.levels;
  LQ_TRY(device_tables(&a.tables));
  prof::Scope ps(prof::WEIGHT_PLANE, st, (double)K * (double)N * (q.bits / 8.0 + (lo ? 4.0 : 2.0)));
  switch (q.bits) {
    case 2: launch_weights<2>(a, transposed, st); break;
    case 3: launch_weights<3>(a, transposed, st); break;
    case 4: launch_weights<4>(a, transposed, st); break;
    case 8: launch_weights<8>(a, transposed, st); break;
    default: return LQ_ERR_CONFIG;
  }
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ------------------------------------------------------------------------------------------------
// The low-rank part goes into the accumulators first and is masked there, then the weights' part is added to it: no second set of
// accumulators, no array of U L1^T.  Features are the tile's rows and tokens its columns, so that a lane holds four neighbouring
// features of a token and the lane 16 further the next four: a group of the generator.
struct AdapterArgs {
  SegArgs g, low;
  AdapterScales s;
  int64_t features, tokens;
  int masked; DropoutMask mask;
  void* out; float* part;
};

template <typename H, typename T>
__global__ __launch_bounds__(SEG_THREADS, 2) void adapter_product_kernel(AdapterArgs a) {
  constexpr bool HALF = !std::is_same<H, __bf16>::value;
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const SegTile t = seg_tile(a.g);
  if (!t.live) return;
  SegAcc acc;
  seg_clear(acc);
  const int64_t row0 = (int64_t)t.tm * SEG_T + 128 * t.wm + 4 * t.kg, col0 = (int64_t)t.tn * SEG_T + 64 * t.wn + t.l16;
  const float a_inv = HALF ? power_of_two(-half_exponent_of(a.s.a_top, TOP_WORDS)) : 1.0f;
  float inv[4];                                       // what a token's sums of the fp16 planes are to be multiplied by
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t token = col0 + 16 * j;
    inv[j] = HALF && token < a.tokens ? a.s.b_inv[token] * a_inv : 1.0f;
  }
  if (t.split == 0 && a.low.pairs > 0) {
    seg_products<__bf16>(a.low, t, 0, a.low.pairs, seg_lds, acc);
    if (HALF || a.masked) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t group = (uint64_t)(col0 + 16 * j) * (uint64_t)(a.features >> 3) + (uint64_t)(row0 >> 3);
        const float scale = (a.masked ? a.mask.scale : 1.0f) * (HALF ? 1.0f / inv[j] : 1.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (a.masked) {
            const PhiloxWords w = philox_words(a.mask, group + 2 * i);
            const uint32_t w0 = t.kg & 1 ? w.w[2] : w.w[0], w1 = t.kg & 1 ? w.w[3] : w.w[1];
            acc[i][j][0] = (w0 & 0xffffu) >= a.mask.cut ? acc[i][j][0] * scale : 0.0f;
            acc[i][j][1] = (w0 >> 16) >= a.mask.cut ? acc[i][j][1] * scale : 0.0f;
            acc[i][j][2] = (w1 & 0xffffu) >= a.mask.cut ? acc[i][j][2] * scale : 0.0f;
            acc[i][j][3] = (w1 >> 16) >= a.mask.cut ? acc[i][j][3] * scale : 0.0f;
          } else {
            acc[i][j] *= scale;
          }
        }
      }
    }
    __syncthreads();                                  // the LDS has been read by everyone
  }
  seg_products<H>(a.g, t, seg_first(a.g.pairs, t.split, a.g.splits), seg_first(a.g.pairs, t.split + 1, a.g.splits), seg_lds, acc);
  float* part = a.part + (size_t)t.split * (size_t)a.tokens * (size_t)a.features;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t token = col0 + 16 * j;
    const bool live = token < a.tokens;
    if (sizeof(T) == 2 && a.g.splits == 1) {          // eight neighbouring features a lane: blocks i and i + 1
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const uintx4 v = seg_pair_blocks(__builtin_bit_cast(uintx2, __builtin_convertvector(acc[i][j], bf16x4)),
                                         __builtin_bit_cast(uintx2, __builtin_convertvector(acc[i + 1][j], bf16x4)));
        const int64_t row = row0 - 4 * t.kg + 16 * (i + (t.kg & 1)) + 8 * (t.kg >> 1);
        if (live && row < a.features) *reinterpret_cast<uintx4*>(static_cast<uint16_t*>(a.out) + token * a.features + row) = v;
      }
      continue;
    }
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = row0 + 16 * i;
      if (row >= a.features) continue;                // features are a multiple of 16
      const floatx4 v = HALF ? acc[i][j] * inv[j] : acc[i][j];
      float* out = a.g.splits > 1 ? part : static_cast<float*>(a.out);
      *reinterpret_cast<floatx4*>(out + token * a.features + row) = v;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void adapter_sum_kernel(const float* __restrict__ part, int splits, int64_t quads, T* __restrict__ out) {
  typedef T vec4 __attribute__((ext_vector_type(4)));
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < quads; i += (int64_t)gridDim.x * 256) {
    floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < splits; ++s) v += reinterpret_cast<const floatx4*>(part)[s * quads + i];
    reinterpret_cast<vec4*>(out)[i] = __builtin_convertvector(v, vec4);
  }
}

int adapter_product_splits(int64_t features, int64_t tokens, int64_t depth, int dtype) {
  return seg_splits(seg_tiles(features, tokens), up_to(depth, 64) / 64 * (dtype == LQ_T_FP32 ? 3 : 1), 16);
}

template <typename H, typename T>
static int launch_adapter(const AdapterArgs& a, hipStream_t st) {
  static LdsLimit limit;
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(adapter_product_kernel<H, T>), SEG_LDS));
  hipLaunchKernelGGL((adapter_product_kernel<H, T>), dim3(seg_grid(a.g)), dim3(SEG_THREADS), SEG_LDS, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

int launch_adapter_product(const Planes& a, const Planes& b, int64_t depth, const Planes& a2, const Planes& b2, int64_t depth2,
                           const AdapterScales& s, int64_t features, int64_t tokens, const DropoutMask* mask, int dtype, void* out,
                           float* part, size_t part_floats, hipStream_t st) {
  if (depth < 64 || depth % 64 || depth2 < 64 || depth2 % 64 || features % 16 || (mask && features % 32)) return LQ_ERR_SHAPE;
  AdapterArgs p{};
  int count = 0;
  add_segments(p.g, &count, a, b, depth);
  count = 0;
  add_segments(p.low, &count, a2, b2, depth2);
  const int splits = adapter_product_splits(features, tokens, depth, dtype);
  LQ_TRY(seg_shape(p.g, features, tokens, splits));
  LQ_TRY(seg_shape(p.low, features, tokens, splits));
  if (splits > 1 && part_floats < (size_t)splits * (size_t)tokens * (size_t)features) return LQ_ERR_WORKSPACE;
  p.s = s; p.features = features; p.tokens = tokens; p.out = out; p.part = part;
  p.masked = mask != nullptr;
  if (mask) p.mask = *mask;
  {
    prof::Scope ps(prof::ADAPTER_PRODUCT, st, 2.0 * features * tokens * (depth + depth2));
    LQ_TRY(dtype == LQ_T_BF16 ? (launch_adapter<__bf16, __bf16>(p, st)) : (launch_adapter<_Float16, float>(p, st)));
  }
  if (splits == 1) return LQ_OK;
  const int64_t quads = tokens * features / 4;
  prof::Scope ps(prof::THIN_FINISH, st, (double)quads * 4 * (4.0 * splits + type_bytes(dtype)));
  const dim3 grid((unsigned)std::min<int64_t>((quads + 255) / 256, 8192));
  if (dtype == LQ_T_BF16)
    hipLaunchKernelGGL(adapter_sum_kernel<__bf16>, grid, dim3(256), 0, st, part, splits, quads, static_cast<__bf16*>(out));
  else
    hipLaunchKernelGGL(adapter_sum_kernel<float>, grid, dim3(256), 0, st, part, splits, quads, static_cast<float*>(out));
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
