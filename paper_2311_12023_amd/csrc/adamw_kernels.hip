// The optimizer's step over many tensors: the gradients' norm and AdamW with states in 32 or 8 bits.  Bound by bytes: 28 a value in fp32
// (480 tensors, 1.7e8 values: 925 us, 5.1 TB/s), 16 with 8-bit states, bf16 gradients and a bf16 copy (1.3e8 values, median 403 us,
// 5.2 TB/s, smallest 382); the norm reads 4: 5.1e7 values 47 us, 4.4 TB/s (36 where the memory-side cache still holds them), 1.6e8 in 448
// tensors 160 us in three launches, 4.0 TB/s, whose last workgroups end one after the other; and the join of the workgroups' sums, 5 us.
#include <cmath>

#include "fp8.h"
#include "fp8_device.h"
#include "profiler.h"

namespace lq {

// Descriptions of tensors travel as kernel arguments (4 KB at most), a launch for every so many of them: nothing has to be uploaded
// that a running kernel may still read, and a captured graph keeps its own.
constexpr int GRADS_A_LAUNCH = 193, TENSORS_A_LAUNCH = 54;
// Elements a workgroup takes.  AdamW: one pass of its threads (480 tensors of 1.7e8 values, 32 bits, 925 us, with four passes 956; one
// of 1.3e8 values, 8 bits, 397 and 408).  The norm: one for few values (a chain of passes is what a small call waits for), several for many,
// whose sums have to be joined.
constexpr int STEP_CHUNK = 2048;
constexpr int64_t NORM_CHUNK_MOST = 16384;
static int64_t norm_chunk(const lq_gradient* g, int64_t count) {
  double n = 0;
  for (int64_t i = 0; i < count; ++i) n += (double)g[i].n;
  int64_t chunk = 2048;
  while (chunk < NORM_CHUNK_MOST && n > (double)chunk * 2048) chunk *= 2;
  return chunk;
}

// ---- the gradients' norm ------------------------------------------------------------------------------------
struct GradTable {
  const void* g[GRADS_A_LAUNCH];
  int64_t n[GRADS_A_LAUNCH];
  uint32_t first[GRADS_A_LAUNCH + 1];      // first workgroup of each
  uint8_t bf16[GRADS_A_LAUNCH];
  int count, chunk;
};

static_assert(sizeof(GradTable) + 24 <= 4096, "kernel arguments");

template <typename Table>
__device__ __forceinline__ int tensor_of(const Table& t, uint32_t wg) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= wg) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Eight neighbours, on addresses that are checked for 16 bytes: the vector type's own alignment is its size, 32 for fp32.
template <typename T>
struct Eight {
  typedef T values __attribute__((ext_vector_type(8)));
  typedef values unit __attribute__((aligned(16)));
};
static_assert(alignof(Eight<float>::unit) == 16 && alignof(Eight<__bf16>::unit) == 16, "addresses that the host checks");

template <int THREADS, typename T>
__device__ __forceinline__ double squares(const T* g, int64_t from, int64_t to) {
  typedef typename Eight<T>::unit vec8;
  double sum = 0.0;
  const bool vec = ((uintptr_t)g & 15) == 0;
  int64_t i = from + 8 * threadIdx.x;
  if (vec) {                                          // four loads under way together
    for (; i + 3 * 8 * THREADS + 8 <= to; i += 4 * 8 * THREADS) {
      vec8 v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = *reinterpret_cast<const vec8*>(g + i + q * 8 * THREADS);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fma((double)(float)v[q][j], (double)(float)v[q][j], sum);
    }
  }
  for (; i < to; i += 8 * THREADS) {
    if (vec && i + 8 <= to) {
      const vec8 v = *reinterpret_cast<const vec8*>(g + i);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = fma((double)(float)v[j], (double)(float)v[j], sum);
    } else {
      for (int j = 0; j < 8 && i + j < to; ++j) sum = fma((double)(float)g[i + j], (double)(float)g[i + j], sum);
    }
  }
  return sum;
}

template <int THREADS>
__device__ __forceinline__ double workgroup_sum(double x) {
  __shared__ double part[THREADS / 64];
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x += __shfl_xor(x, s);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) sum += part[i];
  return sum;
}

__device__ __forceinline__ void write_norm(double sum, float most, float* norm) {
  const float x = (float)sqrt(sum);
  norm[0] = x;
  norm[1] = magnitude(x) >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : fminf(1.0f, most / (x + 1e-6f));
}

template <int THREADS>
__device__ __forceinline__ double tensor_squares(const GradTable& t, int i, int64_t from, int64_t to) {
  return t.bf16[i] ? squares<THREADS>(static_cast<const __bf16*>(t.g[i]), from, to) : squares<THREADS>(static_cast<const float*>(t.g[i]), from, to);
}

__global__ __launch_bounds__(256) void grad_squares_kernel(GradTable t, double* part) {
  const int i = __builtin_amdgcn_readfirstlane(tensor_of(t, blockIdx.x));
  const int64_t from = (int64_t)(blockIdx.x - t.first[i]) * t.chunk;
  const double sum = workgroup_sum<256>(tensor_squares<256>(t, i, from, min(from + t.chunk, t.n[i])));
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

constexpr int NORM_THREADS = 1024;
__global__ __launch_bounds__(NORM_THREADS) void grad_norm_kernel(const double* part, int64_t parts, float most, float* norm) {
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < parts; i += 4 * NORM_THREADS) {      // four loads under way together
    double x[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = i + q * NORM_THREADS < parts ? part[i + q * NORM_THREADS] : 0.0;
#pragma unroll
    for (int q = 0; q < 4; ++q) sum += x[q];
  }
  sum = workgroup_sum<NORM_THREADS>(sum);
  if (threadIdx.x == 0) write_norm(sum, most, norm);
}

// Few values: one workgroup and one launch for all.
constexpr int FEW_PASSES = 4, FEW_THREADS = 1024;
__global__ __launch_bounds__(FEW_THREADS) void grad_norm_few_kernel(GradTable t, float most, float* norm) {
  double sum = 0.0;
  for (int i = 0; i < t.count; ++i) sum += tensor_squares<FEW_THREADS>(t, i, 0, t.n[i]);
  sum = workgroup_sum<FEW_THREADS>(sum);
  if (threadIdx.x == 0) write_norm(sum, most, norm);
}

size_t grad_norm_parts(const lq_gradient* grads, int64_t count) {
  size_t parts = 0;
  const int64_t chunk = norm_chunk(grads, count);
  for (int64_t i = 0; i < count; ++i) parts += (size_t)((grads[i].n + chunk - 1) / chunk);
  return parts;
}

int launch_grad_norm(const lq_gradient* grads, int64_t count, float max_norm, float* norm, double* part, hipStream_t st) {
  double bytes = 0;
  for (int64_t i = 0; i < count; ++i) bytes += (double)grads[i].n * type_bytes(grads[i].dtype);
  prof::Scope ps(prof::GRAD_NORM, st, bytes);
  int64_t passes = 0;
  for (int64_t i = 0; i < count && passes <= FEW_PASSES; ++i) passes += (grads[i].n + 8 * FEW_THREADS - 1) / (8 * FEW_THREADS);
  if (passes <= FEW_PASSES) {
    GradTable t{};
    for (int64_t i = 0; i < count; ++i) {
      if (!grads[i].n) continue;
      t.g[t.count] = grads[i].g;
      t.n[t.count] = grads[i].n;
      t.bf16[t.count++] = grads[i].dtype == LQ_T_BF16;
    }
    hipLaunchKernelGGL(grad_norm_few_kernel, dim3(1), dim3(FEW_THREADS), 0, st, t, max_norm, norm);
    LQ_HIP_TRY(hipGetLastError());
    return LQ_OK;
  }
  size_t done = 0;
  const int64_t chunk = norm_chunk(grads, count);
  for (int64_t i = 0; i < count;) {
    GradTable t{};
    t.chunk = (int)chunk;
    uint64_t wgs = 0;
    for (; i < count && t.count < GRADS_A_LAUNCH; ++i) {
      if (!grads[i].n) continue;
      const uint64_t more = (uint64_t)((grads[i].n + chunk - 1) / chunk);
      if (t.count && wgs + more > 0xffffffull) break;      // fewer than 2^32 threads
      t.g[t.count] = grads[i].g;
      t.n[t.count] = grads[i].n;
      t.bf16[t.count] = grads[i].dtype == LQ_T_BF16;
      t.first[t.count++] = (uint32_t)wgs;
      wgs += more;
    }
    if (!t.count) break;
    hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)wgs), dim3(256), 0, st, t, part + done);
    LQ_HIP_TRY(hipGetLastError());
    done += wgs;
  }
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(NORM_THREADS), 0, st, part, (int64_t)done, max_norm, norm);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

// ---- AdamW ----------------------------------------------------------------------------------------------------
struct StepTensor {
  void* p; const void* g; void* m; void* v;
  float* m_scale; float* v_scale;
  void* copy;
  int64_t n;
};
struct StepTable {
  StepTensor t[TENSORS_A_LAUNCH];
  uint32_t first[TENSORS_A_LAUNCH + 1];
  uint8_t kind[TENSORS_A_LAUNCH];          // bit 0: p bf16, 1: g bf16, 2: on 16-byte addresses
  uint32_t index[TENSORS_A_LAUNCH];        // in the call
  int count;
};
struct StepFactors {
  float beta1, rest1, beta2, rest2, eps, keep, size, root;     // root: (1 - beta2^step)^-1/2, size: lr / (1 - beta1^step)
  uint64_t seed;
  uint32_t step;
};
struct StepArgs {
  StepFactors f;
  double lr, beta1, beta2, decay;          // where lr or step are read on the device
  int64_t step;
  const float* lr_device; const int64_t* step_device; const float* coef;
};

static_assert(sizeof(StepTable) + sizeof(StepArgs) <= 4096, "kernel arguments");

__host__ __device__ inline void step_factors(StepFactors& f, double lr, double beta1, double beta2, double decay, int64_t step) {
  f.keep = (float)(1.0 - lr * decay);
  f.size = (float)(lr / (1.0 - pow(beta1, (double)step)));
  f.root = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
  f.step = (uint32_t)step;
}

// STREAMED: past the caches' replacement, which the 8-bit step's values gain from (1.3e8 values with a bf16 copy 381 us, else 397) and the
// 32-bit one's lose by (954 and 925).
template <bool STREAMED, typename T>
__device__ __forceinline__ void load8(const T* x, int64_t i, int count, bool vec, float (&v)[8]) {
  typedef typename Eight<T>::unit vec8;
  if (vec && count == 8) {
    const vec8* from = reinterpret_cast<const vec8*>(x + i);
    const vec8 in = STREAMED ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)in[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < count ? (float)x[i + j] : 0.0f;
  }
}
template <bool STREAMED, typename T>
__device__ __forceinline__ void store8(T* x, int64_t i, int count, bool vec, const float (&v)[8]) {
  typedef typename Eight<T>::unit vec8;
  if (vec && count == 8) {
    vec8 out;
#pragma unroll
    for (int j = 0; j < 8; ++j) out[j] = (T)v[j];
    if (STREAMED) __builtin_nontemporal_store(out, reinterpret_cast<vec8*>(x + i));
    else *reinterpret_cast<vec8*>(x + i) = out;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < count) x[i + j] = (T)v[j];
  }
}
__device__ __forceinline__ void load_codes(const uint8_t* x, int64_t i, int count, bool vec, float scale, float (&v)[8]) {
  uint32_t w[2] = {0, 0};
  if (vec && count == 8) {
    const uintx2 in = *reinterpret_cast<const uintx2*>(x + i);
    w[0] = in[0]; w[1] = in[1];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < count) w[j >> 2] |= (uint32_t)x[i + j] << (8 * (j & 3));
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const floatx4 c = fp8_values(w[h]);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[4 * h + j] = c[j] * scale;
  }
}
__device__ __forceinline__ void store_codes(uint8_t* x, int64_t i, int count, bool vec, const float (&v)[8]) {
  const uint32_t w[2] = {fp8_four(v[0], v[1], v[2], v[3]), fp8_four(v[4], v[5], v[6], v[7])};
  if (vec && count == 8) {
    *reinterpret_cast<uintx2*>(x + i) = uintx2{w[0], w[1]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < count) x[i + j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
  }
}
// Largest magnitude over the 32 lanes that hold a block of a state.
__device__ __forceinline__ uint32_t block_top(const float (&v)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[j]));
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s));
  return top;
}
// The code's value that stands for 0 <= x <= 448: one of its two neighbours, so that the square is right on average over u.
__device__ __forceinline__ float round_square(float x, uint32_t u) {
  const bool small = x < 0x1p-6f;
  const uint32_t bits = __float_as_uint(x);
  const float step = small ? 0x1p-9f : __uint_as_float((bits & 0x7f800000u) - (3u << 23));
  const float lo = small ? floorf(x * 512.0f) * 0x1p-9f : __uint_as_float(bits & 0xfff00000u);
  const bool up = ((x - lo) * (x + lo)) * 65536.0f > (float)u * (step * (lo + lo + step));
  const float y = up ? lo + step : lo;
  return x > 0.0f ? fmaxf(y, 0x1p-9f) : y;
}

// A thread takes eight neighbours: one call of the generator for its eight roundings, one 8-byte word of codes of either state, and a
// block of 256 lies in 32 lanes, which find its largest magnitude by five exchanges.  Every operation is rounded (no contraction): square
// roots and quotients are the exact ones, some 90 instructions a value, a third of what the bytes leave time for.
template <bool CODES, typename P, typename G>
__device__ __forceinline__ void step_chunk(const StepTensor& t, uint32_t index, bool vec, const StepFactors& f, float coef, bool scaled, int64_t from) {
  const int64_t to = min(from + STEP_CHUNK, t.n);
  // Whole blocks of a state for every group of 32 lanes, so that its lanes stay together.  One pass; left as a loop the 32-bit one takes
  // eight registers less (61, eight wavefronts a SIMD: 925 us, 945 without), the 8-bit one eighteen more.
  for (int64_t i = from + 8 * threadIdx.x; i - 8 * (threadIdx.x & 31) < to; i += 8 * 256) {
    const int count = (int)max((int64_t)0, min((int64_t)8, t.n - i));
    float p[8], g[8], m[8], v[8], r[8];
    load8<CODES>(static_cast<const P*>(t.p), i, count, vec, p);
    // behind the norm the gradients may still be in the memory-side cache (5.1e7 values, norm and step, 160 us, streamed 164)
    if (scaled) load8<false>(static_cast<const G*>(t.g), i, count, vec, g);
    else load8<CODES>(static_cast<const G*>(t.g), i, count, vec, g);
    if constexpr (CODES) {
      load_codes(static_cast<const uint8_t*>(t.m), i, count, vec, t.m_scale[i / STATE_BLOCK], m);
      load_codes(static_cast<const uint8_t*>(t.v), i, count, vec, t.v_scale[i / STATE_BLOCK], v);
    } else {
      load8<false>(static_cast<const float*>(t.m), i, count, vec, m);
      load8<false>(static_cast<const float*>(t.v), i, count, vec, v);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = scaled ? g[j] * coef : g[j];
      const float old = CODES ? v[j] * v[j] : v[j];
      m[j] = m[j] * f.beta1 + x * f.rest1;
      v[j] = old * f.beta2 + (x * f.rest2) * x;
      r[j] = sqrtf(v[j]);
      p[j] = p[j] * f.keep - (m[j] / (r[j] * f.root + f.eps)) * f.size;
    }
    store8<CODES>(static_cast<P*>(t.p), i, count, vec, p);
    if (t.copy) store8<CODES>(static_cast<__bf16*>(t.copy), i, count, vec, p);
    if constexpr (!CODES) {
      store8<false>(static_cast<float*>(t.m), i, count, vec, m);
      store8<false>(static_cast<float*>(t.v), i, count, vec, v);
    } else {
      const float ms = fp8_scale(block_top(m)), vs = fp8_scale(block_top(r));
      const float mi = 1.0f / ms, vi = 1.0f / vs;
      const PhiloxWords w = philox_words({f.seed, ((uint64_t)index << 32) | f.step, 0, 0.0f}, (uint64_t)(i >> 3));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] *= mi;
        r[j] = round_square(fminf(r[j] * vi, 448.0f), (j & 1) ? w.w[j >> 1] >> 16 : w.w[j >> 1] & 0xffffu);
      }
      store_codes(static_cast<uint8_t*>(t.m), i, count, vec, m);
      store_codes(static_cast<uint8_t*>(t.v), i, count, vec, r);
      if ((threadIdx.x & 31) == 0) {
        t.m_scale[i / STATE_BLOCK] = ms;
        t.v_scale[i / STATE_BLOCK] = vs;
      }
    }
    if constexpr (CODES) break;
  }
}

template <bool CODES>
__global__ __launch_bounds__(256) void adamw_kernel(StepTable table, StepArgs a) {
  StepFactors f = a.f;
  const float coef = a.coef ? *a.coef : 1.0f, lr = a.lr_device ? *a.lr_device : 0.0f;
  const int64_t step = a.step_device ? *a.step_device : a.step;
  if (max(magnitude(coef), magnitude(lr)) >= 0x7f800000u || step < 1) return;
  if (a.lr_device || a.step_device) step_factors(f, a.lr_device ? (double)lr : a.lr, a.beta1, a.beta2, a.decay, step);
  const int i = __builtin_amdgcn_readfirstlane(tensor_of(table, blockIdx.x));
  const StepTensor t = table.t[i];
  const int64_t from = (int64_t)(blockIdx.x - table.first[i]) * STEP_CHUNK;
  const int kind = table.kind[i];
  const bool vec = kind & 4, scaled = a.coef != nullptr;
  const uint32_t index = table.index[i];
  if ((kind & 3) == 0) step_chunk<CODES, float, float>(t, index, vec, f, coef, scaled, from);
  else if ((kind & 3) == 1) step_chunk<CODES, __bf16, float>(t, index, vec, f, coef, scaled, from);
  else if ((kind & 3) == 2) step_chunk<CODES, float, __bf16>(t, index, vec, f, coef, scaled, from);
  else step_chunk<CODES, __bf16, __bf16>(t, index, vec, f, coef, scaled, from);
}

int launch_adamw(const lq_adamw_tensor* tensors, int64_t count, int state_bits, const lq_adamw_params& h, const float* coef, hipStream_t st) {
  const bool codes = state_bits == 8;
  StepArgs a{};
  a.f.beta1 = (float)h.beta1; a.f.rest1 = (float)(1.0 - h.beta1);
  a.f.beta2 = (float)h.beta2; a.f.rest2 = (float)(1.0 - h.beta2);
  a.f.eps = (float)h.eps; a.f.seed = h.seed;
  step_factors(a.f, h.lr, h.beta1, h.beta2, h.weight_decay, h.step);
  a.lr = h.lr; a.beta1 = h.beta1; a.beta2 = h.beta2; a.decay = h.weight_decay; a.step = h.step;
  a.lr_device = h.lr_device; a.step_device = h.step_device; a.coef = coef;
  double bytes = 0;
  for (int64_t i = 0; i < count; ++i)
    bytes += (double)tensors[i].n * (2 * type_bytes(tensors[i].p_dtype) + type_bytes(tensors[i].g_dtype) + (codes ? 4 : 16) + (tensors[i].copy ? 2 : 0));
  prof::Scope ps(prof::ADAMW, st, bytes);
  for (int64_t i = 0; i < count;) {
    StepTable t{};
    uint64_t wgs = 0;
    for (; i < count && t.count < TENSORS_A_LAUNCH; ++i) {
      const lq_adamw_tensor& x = tensors[i];
      if (!x.n) continue;
      const uint64_t more = (uint64_t)((x.n + STEP_CHUNK - 1) / STEP_CHUNK);
      if (t.count && wgs + more > 0xffffffull) break;      // fewer than 2^32 threads
      uintptr_t low = (uintptr_t)x.p | (uintptr_t)x.g | (uintptr_t)x.copy;
      const uintptr_t states = (uintptr_t)x.m | (uintptr_t)x.v;
      const bool vec = (low & 15) == 0 && (states & (codes ? 7 : 15)) == 0;
      t.t[t.count] = {x.p, x.g, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.n};
      t.kind[t.count] = (uint8_t)((x.p_dtype == LQ_T_BF16) | (x.g_dtype == LQ_T_BF16) << 1 | vec << 2);
      t.index[t.count] = (uint32_t)i;
      t.first[t.count++] = (uint32_t)wgs;
      wgs += more;
    }
    if (!t.count) break;
    if (codes) hipLaunchKernelGGL(adamw_kernel<true>, dim3((unsigned)wgs), dim3(256), 0, st, t, a);
    else hipLaunchKernelGGL(adamw_kernel<false>, dim3((unsigned)wgs), dim3(256), 0, st, t, a);
    LQ_HIP_TRY(hipGetLastError());
  }
  return LQ_OK;
}

}  // namespace lq
