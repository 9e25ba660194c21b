// Products of a tall matrix A (read once, from global memory) with a narrow one: A B^T over A's rows, and A^T B over its columns.
// B comes as planes with the reduction index contiguous and goes through two LDS stages of 64 reduction indices; A goes through
// registers, where it is masked and split.  Both are loaded two steps ahead, B before A: loads are waited for in their order.
// Barriers are written out: the compiler's own would wait for all that are under way.
#pragma once
#include "dense_device.h"
#include "half_planes_device.h"
#include "mfma_device.h"
#include "philox_device.h"
#include "train.h"

namespace lq {

template <typename T> constexpr int thin_planes() { return sizeof(T) == 2 ? 1 : 3; }

// Eight neighbours of a row as a lane loads them.
template <typename T>
struct Eight { typedef T vec8 __attribute__((ext_vector_type(8))); vec8 v; };

// Eight neighbours from `at` on; without VEC one by one, zero from `left` values on.
template <bool VEC, typename T>
__device__ __forceinline__ void load_eight(const T* at, int64_t left, Eight<T>& x) {
  x.v = {};
  if constexpr (VEC) {
    if (left > 0) x.v = *reinterpret_cast<const typename Eight<T>::vec8*>(at);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) x.v[j] = at[j];
  }
}

// MASKED: there may be a mask (a cut of zero keeps everything).
template <typename T, bool MASKED>
__device__ __forceinline__ void apply_mask(Eight<T>& x, const DropoutMask& d, uint64_t group) {
  if constexpr (MASKED) {
    if (d.cut == 0) return;
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
template <int NA, int NB>
__device__ __forceinline__ void thin_multiply(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], floatx4& acc) {
  constexpr int most = NA > NB ? NA : NB;
#pragma unroll
  for (int s = most - 1; s >= 0; --s)
#pragma unroll
    for (int k = 0; k < NA; ++k)
      if (s - k >= 0 && s - k < NB) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[k], b[s - k], acc, 0, 0, 0);
}

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A stage of B: 64 reduction indices of 16 RT rows of NB planes, rows of 128 bytes with unit u of a row at u ^ (row % 8): the 16
// rows of an operand read meet different banks.
template <int RT, int NB>
struct ThinStage {
  static constexpr int ROWS = 16 * RT * NB, LOADS = (ROWS * 8 + 255) / 256;
  static constexpr uint32_t BYTES = ROWS * 128u;
  uintx4 r[LOADS];
  __device__ __forceinline__ void load(const Planes& b, int64_t k) {
#pragma unroll
    for (int q = 0; q < LOADS; ++q) {
      const int u = threadIdx.x + 256 * q, row = u >> 3;
      if (ROWS * 8 % 256 == 0 || row < ROWS)
        r[q] = *reinterpret_cast<const uintx4*>(b.p[row / (16 * RT)] + (int64_t)(row % (16 * RT)) * b.pitch + k + 8 * (u & 7));
    }
  }
  __device__ __forceinline__ void store(unsigned char* lds) const {
#pragma unroll
    for (int q = 0; q < LOADS; ++q) {
      const int u = threadIdx.x + 256 * q, row = u >> 3;
      if (ROWS * 8 % 256 == 0 || row < ROWS) *reinterpret_cast<uintx4*>(lds + row * 128u + ((u ^ row) & 7) * 16u) = r[q];
    }
  }
};
template <int RT, int NB>
__device__ __forceinline__ void thin_read(const unsigned char* lds, int r, int sub, int l16, int kg, bf16x8 (&b)[NB]) {
#pragma unroll
  for (int k = 0; k < NB; ++k)
    b[k] = *reinterpret_cast<const bf16x8*>(lds + (uint32_t)(k * RT * 16 + 16 * r + l16) * 128u + (uint32_t)((4 * sub + kg) ^ (l16 & 7)) * 16u);
}

// A (m x K, lda elements from row to row) and the mask of its elements where there is one (K a multiple of 8 then).  VEC: rows on
// 16-byte addresses and K a multiple of 8.
struct ThinSource { const void* A; int64_t lda, m, K; DropoutMask d; };

// acc[h][r] += drop(A) B^T over steps s0 .. s1 - 1 (s0 < s1) for rows row0 + 16 h ..: element e is row 4 kg + e, column 16 r + l16.
template <typename T, int H, int RT, int NB, bool MASKED, bool VEC>
__device__ __forceinline__ void thin_rows(const ThinSource& a, const Planes& b, int64_t row0, int s0, int s1, unsigned char* lds,
                                          floatx4 (&acc)[H][RT]) {
  typedef ThinStage<RT, NB> Stage;
  const int lane = threadIdx.x & 63, l16 = lane & 15, kg = lane >> 4;
  const T* x[H];
  uint64_t group[H];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    const int64_t r = row0 + 16 * h + l16, row = r < a.m ? r : a.m - 1;
    x[h] = static_cast<const T*>(a.A) + row * a.lda;
    group[h] = (uint64_t)row * (uint64_t)(a.K >> 3);
  }
  Eight<T> v[2][2][H];                                // [parity of the step][half of it][row tile]
  Stage stage[2];
  auto load = [&](auto odd, int s) __attribute__((always_inline)) {
    constexpr int u = decltype(odd)::value;
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      const int64_t k = 64 * (int64_t)s + 32 * sub + 8 * kg;
#pragma unroll
      for (int h = 0; h < H; ++h) {
        load_eight<VEC, T>(x[h] + k, a.K - k, v[u][sub][h]);
      }
    }
  };
  const auto even = std::integral_constant<int, 0>{};
  const auto odd = std::integral_constant<int, 1>{};
  const int last = s1 - 1;
  const int second = s0 + 1 < last ? s0 + 1 : last;
  stage[0].load(b, 64 * (int64_t)s0);
  load(even, s0);
  stage[1].load(b, 64 * (int64_t)second);
  load(odd, second);
  stage[0].store(lds);
  auto step = [&](auto parity, int s) __attribute__((always_inline)) {
    constexpr int u = decltype(parity)::value;
    bf16x8 p[2][H][thin_planes<T>()];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int h = 0; h < H; ++h) {
        apply_mask<T, MASKED>(v[u][sub][h], a.d, group[h] + (uint64_t)(8 * (int64_t)s + 4 * sub + kg));
        to_planes<T>(v[u][sub][h], p[sub][h]);
      }
    const int ahead = s + 2 < last ? s + 2 : last;    // past the end: the last step again, never used
    stage[u].load(b, 64 * (int64_t)ahead);
    load(parity, ahead);
    lds_barrier();                                    // this step's B is there, and the other stage has been read
    stage[u ^ 1].store(lds + (u ? 0 : Stage::BYTES));
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        bf16x8 w[NB];
        thin_read<RT, NB>(lds + (u ? Stage::BYTES : 0), r, sub, l16, kg, w);
#pragma unroll
        for (int h = 0; h < H; ++h) thin_multiply<thin_planes<T>(), NB>(p[sub][h], w, acc[h][r]);
      }
  };
  int s = s0;
  for (; s + 2 <= s1; s += 2) { step(even, s); step(odd, s + 1); }
  if (s < s1) step(even, s);
}

// acc[h][r] += drop(A)^T B over steps s0 .. s1 - 1 (s0 < s1) of 64 rows for columns c0 + 32 wave + 16 h ..: element e is column
// 4 kg + e, column 16 r + l16 of B.  A thread loads four rows of eight columns and writes them turned, four rows of a column at a
// time.  A column's 64 rows are 128 bytes, its unit u of 16 at u ^ turn(column): the sixteen columns, eight apart, of a write and
// the sixteen neighbours of an operand read both spread over the banks (rows of 64 + 8 instead, without the turn, met eight at a
// time in a bank when written).
__device__ __forceinline__ uint32_t thin_turn(int column) { return (uint32_t)((column >> 3) ^ (column >> 1)) & 7u; }
template <typename T, int RT, int NB>
constexpr uint32_t thin_columns_lds() { return 2 * ThinStage<RT, NB>::BYTES + thin_planes<T>() * 128u * 128u; }

// adjust.load(parity, s) is called where step s's B is loaded, adjust(parity, stage) before it goes into LDS.
struct KeepStage {
  template <class P> __device__ __forceinline__ void load(P, int) {}
  template <class P, class S> __device__ __forceinline__ void operator()(P, S&) {}
};
template <typename T, int RT, int NB, bool MASKED, bool VEC, class Adjust>
__device__ __forceinline__ void thin_columns(const ThinSource& a, const Planes& b, int64_t c0, int s0, int s1, unsigned char* lds,
                                             floatx4 (&acc)[2][RT], Adjust&& adjust) {
  typedef ThinStage<RT, NB> Stage;
  constexpr int NP = thin_planes<T>();
  unsigned char* s_a = lds + 2 * Stage::BYTES;                                          // [plane][column][row]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l16 = lane & 15, kg = lane >> 4;
  const int c8 = (threadIdx.x & 15) * 8, r4 = (threadIdx.x >> 4) * 4;
  const T* x = static_cast<const T*>(a.A) + c0 + c8;
  const int col[2] = {32 * wave + l16, 32 * wave + 16 + l16};
  Eight<T> v[2][4];
  Stage stage[2];
  auto load = [&](auto parity, int s) __attribute__((always_inline)) {
    constexpr int u = decltype(parity)::value;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t row = 64 * (int64_t)s + r4 + q;
      load_eight<VEC, T>(x + row * a.lda, row < a.m ? a.K - c0 - c8 : 0, v[u][q]);
    }
  };
  const auto even = std::integral_constant<int, 0>{};
  const auto odd = std::integral_constant<int, 1>{};
  const int last = s1 - 1;
  const int second = s0 + 1 < last ? s0 + 1 : last;
  stage[0].load(b, 64 * (int64_t)s0);
  adjust.load(even, s0);
  load(even, s0);
  stage[1].load(b, 64 * (int64_t)second);
  adjust.load(odd, second);
  load(odd, second);
  adjust(even, stage[0]);
  stage[0].store(lds);
  auto step = [&](auto parity, int s) __attribute__((always_inline)) {
    constexpr int u = decltype(parity)::value;
    bf16x8 p[4][NP];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t row = 64 * (int64_t)s + r4 + q;
      apply_mask<T, MASKED>(v[u][q], a.d, (uint64_t)row * (uint64_t)(a.K >> 3) + (uint64_t)((c0 + c8) >> 3));
      to_planes<T>(v[u][q], p[q]);
    }
    const int ahead = s + 2 < last ? s + 2 : last;    // past the end: the last step again, never used
    stage[u].load(b, 64 * (int64_t)ahead);
    adjust.load(parity, ahead);
    load(parity, ahead);
    lds_barrier();                                    // the tile and the stage of the step before have been read
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *reinterpret_cast<bf16x4*>(s_a + (k * 128 + c8 + j) * 128 + (((uint32_t)(r4 >> 3) ^ thin_turn(c8 + j)) * 16u) + (r4 & 4) * 2) =
            bf16x4{p[0][k][j], p[1][k][j], p[2][k][j], p[3][k][j]};
    adjust(std::integral_constant<int, u ^ 1>{}, stage[u ^ 1]);
    stage[u ^ 1].store(lds + (u ? 0 : Stage::BYTES));
    lds_barrier();                                    // this step's tile is there
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      bf16x8 t[2][NP];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < NP; ++k)
          t[h][k] = *reinterpret_cast<const bf16x8*>(s_a + (k * 128 + col[h]) * 128 + (((uint32_t)(4 * sub + kg) ^ thin_turn(col[h])) * 16u));
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        bf16x8 w[NB];
        thin_read<RT, NB>(lds + (u ? Stage::BYTES : 0), r, sub, l16, kg, w);
#pragma unroll
        for (int h = 0; h < 2; ++h) thin_multiply<NP, NB>(t[h], w, acc[h][r]);
      }
    }
  };
  int s = s0;
  for (; s + 2 <= s1; s += 2) { step(even, s); step(odd, s + 1); }
  if (s < s1) step(even, s);
}

template <int H, int RT>
__device__ __forceinline__ void thin_clear(floatx4 (&acc)[H][RT]) {
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[h][r] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
}
// part (rows x 16 RT) of a range: rows row0 + 16 h + ..
template <int H, int RT>
__device__ __forceinline__ void thin_store(const floatx4 (&acc)[H][RT], float* out, int64_t row0, int64_t rows) {
  const int l16 = threadIdx.x & 15, kg = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t o = row0 + 16 * h + 4 * kg + e;
      if (o < rows) {
#pragma unroll
        for (int r = 0; r < RT; ++r) out[o * (16 * RT) + 16 * r + l16] = acc[h][r][e];
      }
    }
}

}  // namespace lq
