// Products of a tall matrix A (read once, from global memory) with a narrow one: A B^T over A's rows, and A^T B over its columns.
// B comes as planes with the reduction index contiguous and goes through LDS in stages of 64 reduction indices; A goes through
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

// Wavefronts a SIMD should hold of the columns' product: two, one's products covering the other's loads and splitting; the sums of more
// than 64 columns leave registers for one.
template <typename T, int RT> constexpr int thin_columns_waves() { return RT <= 4 ? 2 : 1; }

// acc[h][r] += a[h] b[r] over the products of planes that count, the smallest first; neighbouring products go to different sums.
template <int NA, int NB, int H, int R, int RT>
__device__ __forceinline__ void thin_multiply(const bf16x8 (&a)[H][NA], const bf16x8 (&b)[R][NB], floatx4 (&acc)[H][RT], int r0) {
  constexpr int most = NA > NB ? NA : NB;
#pragma unroll
  for (int s = most - 1; s >= 0; --s)
#pragma unroll
    for (int k = 0; k < NA; ++k)
      if (s - k >= 0 && s - k < NB) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int h = 0; h < H; ++h) acc[h][r0 + r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[h][k], b[r][s - k], acc[h][r0 + r], 0, 0, 0);
      }
}

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A stage of B: 64 reduction indices of 16 RT rows of NB planes, rows of 128 bytes with unit u of a row at u ^ (row % 8): the 16
// rows of an operand read meet different banks.  A load brings 32 rows, of one plane where RT is even.
template <int RT, int NB>
struct ThinPlace {
  static constexpr int ROWS = 16 * RT * NB, LOADS = (ROWS * 8 + 255) / 256;
  uint32_t at[LOADS];              // bytes into the plane
  __device__ __forceinline__ static constexpr int plane(int q) { return 32 * q / (16 * RT); }
  __device__ __forceinline__ explicit ThinPlace(const Planes& b) {
#pragma unroll
    for (int q = 0; q < LOADS; ++q) {
      const int row = (threadIdx.x >> 3) + 32 * q;
      at[q] = (uint32_t)((row % (16 * RT)) * b.pitch * 2 + 16 * (threadIdx.x & 7));
    }
  }
};
template <int RT, int NB>
struct ThinStage {
  typedef ThinPlace<RT, NB> Place;
  static constexpr int ROWS = Place::ROWS, LOADS = Place::LOADS;
  static constexpr uint32_t BYTES = ROWS * 128u;
  uintx4 r[LOADS];
  __device__ __forceinline__ void load(const Planes& b, const Place& place, int64_t k) {
#pragma unroll
    for (int q = 0; q < LOADS; ++q) {
      const int row = (threadIdx.x >> 3) + 32 * q;
      if (ROWS % 32 == 0 || row < ROWS) {
        const uint16_t* from = (RT % 2 == 0 ? b.p[Place::plane(q)] : b.p[row / (16 * RT)]) + k;
        r[q] = *reinterpret_cast<const uintx4*>(reinterpret_cast<const char*>(from) + place.at[q]);
      }
    }
  }
  __device__ __forceinline__ void store(unsigned char* lds) const {
#pragma unroll
    for (int q = 0; q < LOADS; ++q) {
      const int u = threadIdx.x + 256 * q, row = u >> 3;
      if (ROWS % 32 == 0 || row < ROWS) *reinterpret_cast<uintx4*>(lds + row * 128u + ((u ^ row) & 7) * 16u) = r[q];
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

// acc[h][r] += drop(A) B^T over steps s0 .. s1 - 1 (s0 < s1) for rows row0 + APART h ..: element e is row 4 kg + e, column 16 r + l16.
template <typename T, int H, int APART, int RT, int NB, bool MASKED, bool VEC>
__device__ __forceinline__ void thin_rows(const ThinSource& a, const Planes& b, int64_t row0, int s0, int s1, unsigned char* lds,
                                          floatx4 (&acc)[H][RT]) {
  typedef ThinStage<RT, NB> Stage;
  constexpr int R = RT > 1 ? 2 : 1;
  const int lane = threadIdx.x & 63, l16 = lane & 15, kg = lane >> 4;
  const T* x[H];
  uint64_t group[H];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    const int64_t r = row0 + APART * h + l16, row = r < a.m ? r : a.m - 1;
    x[h] = static_cast<const T*>(a.A) + row * a.lda;
    group[h] = (uint64_t)row * (uint64_t)(a.K >> 3);
  }
  Eight<T> v[2][2][H];                                // [parity of the step][half of it][row tile]
  Stage stage[2];
  const typename Stage::Place place(b);
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
  stage[0].load(b, place, 64 * (int64_t)s0);
  load(even, s0);
  stage[1].load(b, place, 64 * (int64_t)second);
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
    stage[u].load(b, place, 64 * (int64_t)ahead);
    load(parity, ahead);
    lds_barrier();                                    // this step's B is there, and the other stage has been read
    stage[u ^ 1].store(lds + (u ? 0 : Stage::BYTES));
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int r = 0; r < RT; r += R) {
        bf16x8 w[R][NB];
#pragma unroll
        for (int q = 0; q < R; ++q) thin_read<RT, NB>(lds + (u ? Stage::BYTES : 0), r + q, sub, l16, kg, w[q]);
        thin_multiply(p[sub], w, acc, r);
      }
  };
  int s = s0;
  for (; s + 2 <= s1; s += 2) { step(even, s); step(odd, s + 1); }
  if (s < s1) step(even, s);
}

// acc[h][r] += drop(A)^T B over steps s0 .. s1 - 1 (s0 < s1) of 64 rows for columns c0 + 32 wave + 16 h ..: element e is column
// 4 kg + e, column 16 r + l16 of B.  A tile of 64 rows x 128 columns lies in LDS as it comes, and operands come out of it by
// transposed reads: 16 lanes read four rows of 16 columns, a lane gets the four of its own.  The 32-byte chunk c of row m is stored
// at c ^ (m % 4 + 4 (m / 8 % 2)): the sixteen rows that a read touches spread over the banks.  1000 x 11008 fp32 by 64: 27 us, 4096 x 11008
// bf16: 49; with the tile turned on its way into LDS, in 8-byte pieces, 42 and 60.
template <typename T, int RT, int NB>
constexpr uint32_t thin_columns_lds() { return ThinStage<RT, NB>::BYTES + thin_planes<T>() * 64u * 256u; }
__device__ __forceinline__ bf16x8 thin_turned_read(const unsigned char* tile, int sub, int chunk, int l16, int kg) {
  typedef short shortx4 __attribute__((ext_vector_type(4)));
  const uint32_t at = (uint32_t)(32 * sub + 8 * kg + (l16 >> 2)) * 256u + (uint32_t)(chunk ^ ((l16 >> 2) + 4 * (kg & 1))) * 32u + 8u * (l16 & 3);
  const bf16x4 lo = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)(tile + at)));
  const bf16x4 hi = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)(tile + at + 1024u)));
  return bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// adjust.load(parity, s) is called where step s's B is loaded, adjust(parity, stage) before it goes into LDS.
struct KeepStage {
  template <class P> __device__ __forceinline__ void load(P, int) {}
  template <class P, class S> __device__ __forceinline__ void operator()(P, S&) {}
};
template <typename T, int RT, int NB, bool MASKED, bool VEC, class Adjust>
__device__ __forceinline__ void thin_columns(const ThinSource& a, const Planes& b, int64_t c0, int s0, int s1, unsigned char* lds,
                                             floatx4 (&acc)[2][RT], Adjust&& adjust) {
  typedef ThinStage<RT, NB> Stage;
  constexpr int NP = thin_planes<T>(), R = RT > 1 ? 2 : 1;
  unsigned char* s_a = lds + Stage::BYTES;                                              // [plane][row][column]
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l16 = lane & 15, kg = lane >> 4;
  const int c8 = (threadIdx.x & 15) * 8, r4 = (threadIdx.x >> 4) * 4;
  const T* x = static_cast<const T*>(a.A) + c0 + r4 * a.lda + c8;      // rows may be any distance apart: 64-bit offsets
  Eight<T> v[2][4];
  Stage stage[2];
  const typename Stage::Place place(b);
  auto load = [&](auto parity, int s) __attribute__((always_inline)) {
    constexpr int u = decltype(parity)::value;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t row = 64 * (int64_t)s + r4 + q;
      load_eight<VEC, T>(x + (64 * (int64_t)s + q) * a.lda, row < a.m ? a.K - c0 - c8 : 0, v[u][q]);
    }
  };
  const auto even = std::integral_constant<int, 0>{};
  const auto odd = std::integral_constant<int, 1>{};
  const int last = s1 - 1;
  const int second = s0 + 1 < last ? s0 + 1 : last;
  stage[0].load(b, place, 64 * (int64_t)s0);
  adjust.load(even, s0);
  load(even, s0);
  stage[1].load(b, place, 64 * (int64_t)second);
  adjust.load(odd, second);
  load(odd, second);
  auto step = [&](auto parity, int s) __attribute__((always_inline)) {
    constexpr int u = decltype(parity)::value;
    bf16x8 p[4][NP];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t row = 64 * (int64_t)s + r4 + q;
      apply_mask<T, MASKED>(v[u][q], a.d, (uint64_t)row * (uint64_t)(a.K >> 3) + (uint64_t)((c0 + c8) >> 3));
      to_planes<T>(v[u][q], p[q]);
    }
    adjust(parity, stage[u]);
    lds_barrier();                                    // the tile and the stage of the step before have been read
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int m = r4 + q;
      const uint32_t at = (uint32_t)m * 256u + (uint32_t)((c8 >> 3) ^ (((m & 3) + 4 * ((m >> 3) & 1)) * 2)) * 16u;
#pragma unroll
      for (int k = 0; k < NP; ++k) *reinterpret_cast<bf16x8*>(s_a + k * 16384u + at) = p[q][k];
    }
    stage[u].store(lds);
    const int ahead = s + 2 < last ? s + 2 : last;    // past the end: the last step again, never used
    stage[u].load(b, place, 64 * (int64_t)ahead);
    adjust.load(parity, ahead);
    load(parity, ahead);
    lds_barrier();                                    // this step's are there
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      bf16x8 t[2][NP];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < NP; ++k) t[h][k] = thin_turned_read(s_a + k * 16384u, sub, 2 * wave + h, l16, kg);
#pragma unroll
      for (int r = 0; r < RT; r += R) {
        bf16x8 w[R][NB];
#pragma unroll
        for (int q = 0; q < R; ++q) thin_read<RT, NB>(lds, r + q, sub, l16, kg, w[q]);
        thin_multiply(t, w, acc, r);
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
