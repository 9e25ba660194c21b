// The large product of a decomposed layer in training:  Y = X Q + T L2  and  dX = dY Q^T + mask .* (U L1^T).
#include "half_planes_device.h"
#include "mfma_device.h"
#include "nf_device.h"
#include "profiler.h"
#include "segment_gemm.h"
#include "train.h"

namespace lq {

// ------------------------------------------------------------------------------------------------
// A workgroup finishes 16 rows x 32 columns of T, two values a thread with their ranges' loads under way together; the transposed
// planes go through LDS.
__device__ __forceinline__ void finish_block(const ThinFinish& a, uint32_t bx, uint32_t by, float (&s_t)[32][33]) {
  const int c = threadIdx.x & 31, col = by * 32 + c;
  const size_t stride = (size_t)a.m * (size_t)a.r32;
  float v[2] = {0.0f, 0.0f};
  int64_t row[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) row[q] = (int64_t)bx * 16 + (threadIdx.x >> 5) + 8 * q;
  if (col < a.r32) {
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s)
#pragma unroll
      for (int q = 0; q < 2; ++q)
        if (row[q] < a.m) v[q] += a.part[s * stride + row[q] * a.r32 + col];
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const float f = v[q] * a.scale;
    s_t[(threadIdx.x >> 5) + 8 * q][c] = f;
    if (row[q] >= a.m) continue;
    if (a.T && col < a.rank) a.T[row[q] * a.rank + col] = f;
    bf16x2 p[3];
    split_bf16_3(floatx2{f, 0.0f}, p);
#pragma unroll
    for (int k = 0; k < 3; ++k) a.rows.p[k][row[q] * a.rows.pitch + col] = __builtin_bit_cast(uint16_t, p[k][0]);
  }
  if (!a.cols.p[0] || (int)by * 32 >= a.r32) return;
  __syncthreads();
  const int pair = threadIdx.x & 7, k = threadIdx.x >> 3;
  bf16x2 p[3];
  split_bf16_3(floatx2{s_t[2 * pair][k], s_t[2 * pair + 1][k]}, p);
  const int64_t at = (int64_t)(by * 32 + k) * a.cols.pitch + (int64_t)bx * 16 + 2 * pair;
#pragma unroll
  for (int j = 0; j < 3; ++j) *reinterpret_cast<bf16x2*>(a.cols.p[j] + at) = p[j];
}

// The sums over the ranges: 32 rows x 32 columns a workgroup; the first product's result is turned.
__device__ __forceinline__ void gram_sum_block(const ThinGramSum& a, uint32_t bx, uint32_t by, float (&s_t)[32][33]) {
  const uint32_t wgs0 = (uint32_t)((a.K[0] + 31) / 32);
  const int which = bx >= wgs0;
  const int64_t row0 = (int64_t)(bx - (which ? wgs0 : 0)) * 32, K = a.K[which];
  const int c = threadIdx.x & 31, r0 = threadIdx.x >> 5, col = by * 32 + c;
  const size_t stride = (size_t)K * a.r32;
  const float* part = a.part[which];
  float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = 0; s < a.splits; ++s)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (row0 + r0 + 8 * q < K) v[q] += part[s * stride + (row0 + r0 + 8 * q) * a.r32 + col];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t row = row0 + r0 + 8 * q;
    if (which) { if (row < K && col < a.rank) a.out[1][row * a.rank + col] = v[q] * a.scale; }
    else s_t[r0 + 8 * q][c] = v[q];
  }
  if (which) return;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int k = r0 + 8 * q;
    if (row0 + c < K && (int)(by * 32 + k) < a.rank) a.out[0][(int64_t)(by * 32 + k) * K + row0 + c] = s_t[c][k];
  }
}

// ------------------------------------------------------------------------------------------------
// The stored weights as planes, 16 weights a thread and row.  bf16 activations meet weights rounded to bf16 (2^-9, as much as their
// results are rounded by), fp32 ones meet two fp16 planes.  Bound by what is written: 4096 x 11008 in one plane 30 us, 11008 x 4096 in
// two 50 us, 3.7 TB/s.
struct WeightArgs {
  const uint8_t* codes; const uint8_t* sidx; const float* v;
  int64_t K, N, pitch;
  uint16_t* hi; uint16_t* lo;
  int block_shift, group_shift, levels; float inv_levels;
  const DevTables* tables; const uint32_t* top;
};

// The exponent that fp32 weights go into their planes with.  At most 80: the low-rank part is brought to the accumulators' unit, 2^14
// from it per row of activations and this from the weights, and stays below 2^128 unless it is 2^34 times its row's largest value.
// Weights lose bits to that only if all of them are below 2^-82.
__device__ __forceinline__ int weight_exponent(const uint32_t* __restrict__ top) {
  const int e = half_exponent_of(top, TOP_WORDS);
  return e < 80 ? e : 80;
}

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
__device__ __forceinline__ void weight_rows(const WeightArgs& a, uint32_t block, uint32_t wgs, float* s_code) {
  load_codebook<BITS>(a, s_code);
  const float scale = HALF ? power_of_two(weight_exponent(a.top)) : 1.0f;
  const int64_t runs = (a.N + 63) / 64 * 4, total = a.K * runs;       // runs of 16 up to a multiple of 64 weights
  for (int64_t u = (int64_t)block * 256 + threadIdx.x; u < total; u += (int64_t)wgs * 256) {
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
__device__ __forceinline__ void weight_columns(const WeightArgs& a, uint32_t bx, uint32_t by, float* s_code,
                                               uint32_t (&s_w)[HALF ? 2 : 1][WC_N * WC_WORDS]) {
  load_codebook<BITS>(a, s_code);
  const float scale = HALF ? power_of_two(weight_exponent(a.top)) : 1.0f;
  const int tid = threadIdx.x, run = tid & 7, pair = tid >> 3;
  const int64_t n0 = (int64_t)bx * WC_N, k0 = (int64_t)by * WC_K, col = n0 + 16 * run;
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

// A pass over partial results and the weights in one launch: neither waits for the other, and the first hides behind the decoding.
// The backward call's weights go with the sums of its gradients where there are some, right before the product that reads them:
// decoded before the gradients' products, the whole call took 402 us for 381 (1000 x 4096, 11008 features, fp32).
struct FinishArgs { ThinFinish f; ThinGramSum g; int sums; WeightArgs w; uint32_t first, first_x, weight_wgs, weight_x; };

__device__ __forceinline__ void first_block(const FinishArgs& a, float (&s_t)[32][33]) {
  const uint32_t bx = blockIdx.x % a.first_x, by = blockIdx.x / a.first_x;
  if (a.sums) gram_sum_block(a.g, bx, by, s_t);
  else finish_block(a.f, bx, by, s_t);
}
__global__ __launch_bounds__(256) void thin_finish_kernel(FinishArgs a) {
  __shared__ float s_t[32][33];
  first_block(a, s_t);
}
template <int BITS, bool HALF, bool TRANSPOSED>
__global__ __launch_bounds__(256) void finish_weights_kernel(FinishArgs a) {
  struct Columns { float code[1 << BITS]; uint32_t w[HALF ? 2 : 1][WC_N * WC_WORDS]; };
  struct Rows { float code[1 << BITS]; };
  typedef typename std::conditional<TRANSPOSED, Columns, Rows>::type Weights;
  __shared__ union { float t[32][33]; Weights w; } s;
  if (blockIdx.x < a.first) {
    first_block(a, s.t);
    return;
  }
  const uint32_t block = blockIdx.x - a.first;
  if constexpr (TRANSPOSED) weight_columns<BITS, HALF>(a.w, block % a.weight_x, block / a.weight_x, s.w.code, s.w.w);
  else weight_rows<BITS, HALF>(a.w, block, a.weight_wgs, s.w.code);
}

template <int BITS>
static void launch_weights(const FinishArgs& a, bool transposed, hipStream_t st) {
  auto kernel = transposed ? (a.w.lo ? finish_weights_kernel<BITS, true, true> : finish_weights_kernel<BITS, false, true>)
                           : (a.w.lo ? finish_weights_kernel<BITS, true, false> : finish_weights_kernel<BITS, false, false>);
  hipLaunchKernelGGL(kernel, dim3(a.first + a.weight_wgs), dim3(256), 0, st, a);
}

static int launch_first(FinishArgs& a, double bytes, const WeightPlanes* w, hipStream_t st) {
  if (!w) {
    prof::Scope ps(prof::THIN_FINISH, st, bytes);
    hipLaunchKernelGGL(thin_finish_kernel, dim3(a.first), dim3(256), 0, st, a);
    LQ_HIP_TRY(hipGetLastError());
    return LQ_OK;
  }
  const MvWeights& q = w->q;
  const int64_t K = w->K, N = w->N;
  if (N % 16 || w->pitch % 64 || w->pitch < (w->transposed ? K : N) || K * N >= (1ll << 31)) return LQ_ERR_SHAPE;
  if (q.block < 16 || (q.block & (q.block - 1)) || q.scale_block < 1 || (q.scale_block & (q.scale_block - 1)) || N % q.block)
    return LQ_ERR_CONFIG;
  if (w->lo && !w->top) return LQ_ERR_NULL;
  a.w.codes = q.codes; a.w.sidx = q.sidx; a.w.v = q.v; a.w.K = K; a.w.N = N; a.w.pitch = w->pitch; a.w.hi = w->hi; a.w.lo = w->lo;
  a.w.top = w->top;
  a.w.block_shift = __builtin_ctz((unsigned)q.block);
  a.w.group_shift = __builtin_ctz((unsigned)q.scale_block);
  a.w.levels = q.levels;
  a.w.inv_levels = 1.0f / (float)q.levels;
  a.weight_x = (uint32_t)((N + WC_N - 1) / WC_N);
  a.weight_wgs = w->transposed ? a.weight_x * (uint32_t)((K + WC_K - 1) / WC_K)
                               : (uint32_t)std::min<int64_t>((K * ((N + 63) / 64 * 4) + 255) / 256, 1 << 14);
  LQ_TRY(device_tables(&a.w.tables));
  prof::Scope ps(prof::WEIGHT_PLANE, st, bytes + (double)K * (double)N * (q.bits / 8.0 + (w->lo ? 4.0 : 2.0)));
  switch (q.bits) {
    case 2: launch_weights<2>(a, w->transposed, st); break;
    case 3: launch_weights<3>(a, w->transposed, st); break;
    case 4: launch_weights<4>(a, w->transposed, st); break;
    case 8: launch_weights<8>(a, w->transposed, st); break;
    default: return LQ_ERR_CONFIG;
  }
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

int launch_finish(const ThinFinish& f, const WeightPlanes* weights, hipStream_t st) {
  if ((f.cols.p[0] && (f.cols.pitch % 64 || f.cols.pitch < up_to(f.m, 64))) || !f.rows.p[0] || f.rows.pitch != up_to(f.r32, 64))
    return LQ_ERR_SHAPE;
  // the row planes are written to their full pitch, the transposed ones up to a multiple of 64 rows
  FinishArgs a{};
  a.f = f;
  a.first_x = (uint32_t)(up_to(f.m, 64) / 16);
  a.first = a.first_x * (uint32_t)(f.rows.pitch / 32);
  return launch_first(a, (double)f.m * f.r32 * 4.0 * (f.splits + 2), weights, st);
}

int launch_gram_sum(const ThinGramSum& g, const WeightPlanes* weights, hipStream_t st) {
  FinishArgs a{};
  a.g = g;
  a.sums = 1;
  a.first_x = (uint32_t)((g.K[0] + 31) / 32 + (g.K[1] + 31) / 32);
  a.first = a.first_x * (uint32_t)(g.r32 / 32);
  return launch_first(a, (double)(g.K[0] + g.K[1]) * g.r32 * 4.0 * (g.splits + 1), weights, st);
}

// ------------------------------------------------------------------------------------------------
// The low-rank part goes into the accumulators first and is masked there, then the weights' part is added to it: no second set of
// accumulators, no array of U L1^T.  Features are the tile's rows and tokens its columns, so that a lane holds four neighbouring
// features of a token and the lane 16 further the next four: a group of the generator.  4096 x 4096 by 4096, bf16: 109 us, 1.32
// PFLOP/s with the low-rank part; 1000 x 4096 by 11008, fp32 (three products): 300 us, 0.92, 172 tiles on 256 CUs.
//
// Work is dealt out in stretches of pairs of steps, all tiles' one after the other, a tile's low-rank pairs before its others: a
// stretch may end inside a tile, whose parts a second kernel then adds up (the mask goes onto each part of the low-rank sum).
struct AdapterArgs {
  SegArgs g, low;
  AdapterScales s;
  int64_t features, tokens;
  int masked; DropoutMask mask;
  int stretches, per, more;        // pairs of a stretch, and how many of the first have one more
  void* out; float* part;          // two tiles a stretch: of the tile it begins in, of the tile it ends in
};
constexpr int64_t PART_TILE = (int64_t)SEG_T * SEG_T;

__device__ __forceinline__ int stretch_begin(const AdapterArgs& a, int w) { return a.per * w + (w < a.more ? w : a.more); }

// The sums of the fp16 planes of a token are 2^exps times what they stand for.  The power of two itself need not be a float, nor its
// inverse: rows of gradients below 2^-97 are ordinary (a token that is certain of its target), so sums are moved by exponents.
template <bool HALF>
__device__ __forceinline__ void token_exponents(const AdapterArgs& a, int64_t col0, int (&exps)[4]) {
  const int of_weights = HALF ? weight_exponent(a.s.a_top) : 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t token = col0 + 16 * j;
    exps[j] = HALF && token < a.tokens ? of_weights + 127 - (int)(__float_as_uint(a.s.b_inv[token]) >> 23) : 0;
  }
}
__device__ __forceinline__ floatx4 times_power_of_two(floatx4 v, int e) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = __builtin_ldexpf(v[k], e);
  return v;
}

// A finished tile's blocks to `out`.
template <typename T>
__device__ __forceinline__ void store_tile(const AdapterArgs& a, const SegAcc& acc, const SegTile& t, int64_t row0, int64_t col0,
                                           const int (&exps)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t token = col0 + 16 * j;
    const bool live = token < a.tokens;
    if constexpr (sizeof(T) == 2) {                   // eight neighbouring features a lane: blocks i and i + 1
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const uintx4 v = seg_pair_blocks(__builtin_bit_cast(uintx2, __builtin_convertvector(acc[i][j], bf16x4)),
                                         __builtin_bit_cast(uintx2, __builtin_convertvector(acc[i + 1][j], bf16x4)));
        const int64_t row = row0 - 4 * t.kg + 16 * (i + (t.kg & 1)) + 8 * (t.kg >> 1);
        if (live && row < a.features) *reinterpret_cast<uintx4*>(static_cast<uint16_t*>(a.out) + token * a.features + row) = v;
      }
    } else if (live) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t row = row0 + 16 * i;            // features are a multiple of 16
        if (row < a.features) *reinterpret_cast<floatx4*>(static_cast<float*>(a.out) + token * a.features + row) = times_power_of_two(acc[i][j], -exps[j]);
      }
    }
  }
}

template <typename H, typename T>
__global__ __launch_bounds__(SEG_THREADS, 2) void adapter_product_kernel(AdapterArgs a) {
  constexpr bool HALF = !std::is_same<H, __bf16>::value;
  extern __shared__ __attribute__((aligned(16))) unsigned char seg_lds[];
  const int w = seg_piece(a.stretches);
  if (w < 0) return;
  const int low = a.low.pairs, pairs = low + a.g.pairs;       // of a tile
  const int begin = stretch_begin(a, w), stop = stretch_begin(a, w + 1);
  for (int pos = begin; pos < stop;) {
    const int u = pos / pairs, s0 = pos - u * pairs, s1 = stop - pos < pairs - s0 ? s0 + stop - pos : pairs;
    const SegTile t = seg_tile_at(a.g, u);
    const int64_t row0 = (int64_t)t.tm * SEG_T + 128 * t.wm + 4 * t.kg, col0 = (int64_t)t.tn * SEG_T + 64 * t.wn + t.l16;
    SegAcc acc;
    seg_clear(acc);
    int exps[4];
    token_exponents<HALF>(a, col0, exps);
    if (s0 < low) {
      seg_products<__bf16>(a.low, t, s0, s1 < low ? s1 : low, seg_lds, acc);
      if (HALF || a.masked) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t group = (uint64_t)(col0 + 16 * j) * (uint64_t)(a.features >> 3) + (uint64_t)(row0 >> 3);
          const float scale = a.mask.scale;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (a.masked) {
              const PhiloxWords p = philox_words(a.mask, group + 2 * i);
              const uint32_t w0 = t.kg & 1 ? p.w[2] : p.w[0], w1 = t.kg & 1 ? p.w[3] : p.w[1];
              acc[i][j][0] = (w0 & 0xffffu) >= a.mask.cut ? acc[i][j][0] * scale : 0.0f;
              acc[i][j][1] = (w0 >> 16) >= a.mask.cut ? acc[i][j][1] * scale : 0.0f;
              acc[i][j][2] = (w1 & 0xffffu) >= a.mask.cut ? acc[i][j][2] * scale : 0.0f;
              acc[i][j][3] = (w1 >> 16) >= a.mask.cut ? acc[i][j][3] * scale : 0.0f;
            }
            if constexpr (HALF) acc[i][j] = times_power_of_two(acc[i][j], exps[j]);
          }
        }
      }
      __syncthreads();                                // the LDS has been read by everyone
    }
    if (s1 > low) seg_products<H>(a.g, t, s0 > low ? s0 - low : 0, s1 - low, seg_lds, acc);
    if (s0 == 0 && s1 == pairs) {
      store_tile<T>(a, acc, t, row0, col0, exps);
    } else {
      floatx4* part = reinterpret_cast<floatx4*>(a.part + (2 * (int64_t)w + (pos == begin ? 0 : 1)) * PART_TILE) + threadIdx.x;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col0 + 16 * j < a.tokens) {
#pragma unroll
          for (int i = 0; i < 8; ++i) part[(4 * i + j) * SEG_THREADS] = acc[i][j];
        }
    }
    pos += s1 - s0;
    __syncthreads();                                  // the LDS has been read by everyone
  }
}

// The parts of a tile that stretches end in, added in their order, the loads of four under way together.  A workgroup takes one of the
// eight block rows.
template <typename T>
__global__ __launch_bounds__(SEG_THREADS) void adapter_join_kernel(AdapterArgs a) {
  constexpr bool HALF = sizeof(T) == 4;
  typedef T vec4 __attribute__((ext_vector_type(4)));
  const int pairs = a.low.pairs + a.g.pairs, u = blockIdx.x, first = u * pairs, last = first + pairs, i = blockIdx.y;
  int w = first / (a.per + 1);                        // not behind the stretch that the tile begins in
  while (stretch_begin(a, w + 1) <= first) ++w;
  if (stretch_begin(a, w + 1) >= last) return;        // whole: stored by the product
  int end = w + 1;
  while (end < a.stretches && stretch_begin(a, end) < last) ++end;
  const SegTile t = seg_tile_at(a.g, u);
  const int64_t row = (int64_t)t.tm * SEG_T + 128 * t.wm + 16 * i + 4 * t.kg, col0 = (int64_t)t.tn * SEG_T + 64 * t.wn + t.l16;
  // of the tile that a stretch begins in, or, for the first one here, of that it ends in
  const int head = stretch_begin(a, w) < first ? 1 : 0;
  const floatx4* part = reinterpret_cast<const floatx4*>(a.part + 2 * (int64_t)w * PART_TILE) + threadIdx.x;
  constexpr int64_t NEXT = 2 * PART_TILE / 4;
  int exps[4];
  token_exponents<HALF>(a, col0, exps);
  floatx4 v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int p = 0; p < end - w; p += 4) {
    floatx4 x[4][4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[q][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        if (p + q < end - w && col0 + 16 * j < a.tokens)
          x[q][j] = part[(p + q) * NEXT + (p + q == 0 ? head : 0) * (PART_TILE / 4) + (4 * i + j) * SEG_THREADS];
      }
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += x[q][j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t token = col0 + 16 * j;
    if (token < a.tokens && row < a.features)
      *reinterpret_cast<vec4*>(static_cast<T*>(a.out) + token * a.features + row) = __builtin_convertvector(times_power_of_two(v[j], -exps[j]), vec4);
  }
}

// A stretch for every tile where that keeps half the chip busy, else up to one for every CU, of six pairs of steps at least (50 tokens x
// 4096 features, depth 1024, fp32, the whole call 42 us; of three, with twice the parts to join, 48), of three where that leaves less
// than 64 stretches (37 x 768, depth 768: 44 us, of six 45).  Leaving CUs idle costs less than their share, since the others then hold a
// higher clock: 1000 tokens x 11008 features, 172 tiles, fp32, the whole call 402 us with a tile each, 432 with 256 stretches.
static int tile_pairs(int64_t depth, int64_t depth2, int dtype) {
  return (int)(depth / 64 * (dtype == LQ_T_FP32 ? 3 : 1) + depth2 / 64 * (dtype == LQ_T_FP32 ? 6 : 3));
}
static int adapter_stretches(int64_t features, int64_t tokens, int64_t depth, int64_t depth2, int dtype) {
  const int64_t tiles = seg_tiles(features, tokens), rounds = (tiles + 255) / 256;
  if (2 * tiles >= 256 * rounds) return (int)tiles;
  const int64_t pairs = tiles * tile_pairs(depth, depth2, dtype);
  return (int)std::max<int64_t>(1, std::min<int64_t>(256, std::max(pairs / 6, std::min<int64_t>(pairs / 3, 64))));
}
size_t adapter_part_floats(int64_t features, int64_t tokens, int64_t depth, int64_t depth2, int dtype) {
  const int s = adapter_stretches(features, tokens, depth, depth2, dtype);
  return s == seg_tiles(features, tokens) ? 0 : (size_t)2 * s * PART_TILE;
}

template <typename H, typename T>
static int launch_adapter(const AdapterArgs& a, hipStream_t st) {
  static LdsLimit limit;
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(adapter_product_kernel<H, T>), SEG_LDS));
  hipLaunchKernelGGL((adapter_product_kernel<H, T>), dim3((unsigned)((a.stretches + 7) / 8 * 8)), dim3(SEG_THREADS), SEG_LDS, st, a);
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
  LQ_TRY(seg_shape(p.g, features, tokens, 1));
  LQ_TRY(seg_shape(p.low, features, tokens, 1));
  if (part_floats < adapter_part_floats(features, tokens, depth, depth2, dtype)) return LQ_ERR_WORKSPACE;
  p.s = s; p.features = features; p.tokens = tokens; p.out = out; p.part = part;
  p.masked = mask != nullptr;
  if (mask) p.mask = *mask;
  const int64_t total = seg_tiles(features, tokens) * (p.low.pairs + p.g.pairs);
  if (total >= (1ll << 31) - 256) return LQ_ERR_SHAPE;
  p.stretches = adapter_stretches(features, tokens, depth, depth2, dtype);
  p.per = (int)(total / p.stretches);
  p.more = (int)(total % p.stretches);
  {
    prof::Scope ps(prof::ADAPTER_PRODUCT, st, 2.0 * features * tokens * (depth + depth2));
    LQ_TRY(dtype == LQ_T_BF16 ? (launch_adapter<__bf16, __bf16>(p, st)) : (launch_adapter<_Float16, float>(p, st)));
  }
  const int64_t tiles = seg_tiles(features, tokens);
  if (p.stretches == tiles) return LQ_OK;
  prof::Scope ps(prof::THIN_FINISH, st, (double)tiles * PART_TILE * 12.0);
  const dim3 grid((unsigned)tiles, 8);
  if (dtype == LQ_T_BF16) hipLaunchKernelGGL(adapter_join_kernel<__bf16>, grid, dim3(SEG_THREADS), 0, st, p);
  else hipLaunchKernelGGL(adapter_join_kernel<float>, grid, dim3(SEG_THREADS), 0, st, p);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
