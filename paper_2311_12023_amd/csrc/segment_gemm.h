// The matrix product that the training operators share:  C = sum over segments of A_s B_s^T  for 16-bit planes with the reduction
// index contiguous.  A segment is a pair of planes; an operand in fp32 is two fp16 planes (hi + lo, 22 bits) or three bf16 planes
// (24 bits) and goes in as the pairs of planes whose product counts.  What becomes of a tile of C is up to the kernel that
// calls it.
#pragma once
#include "dense_device.h"
#include "lds_transfer.h"
#include "mfma_device.h"
#include "train.h"

namespace lq {

// One workgroup of 512 threads owns a 256 x 256 tile, a wavefront 128 x 64 of it (2 x 4), in blocks of 16 x 16.  Accumulator element
// e of acc[i][j] is row 16 i + 4 kg + e, column 16 j + l16 of the wavefront's part (l16 = lane % 16, kg = lane / 16).
struct SegTile {
  int tm, tn, split;
  int wm, wn, l16, kg;
  bool live;
};
typedef floatx4 SegAcc[8][4];

// (tile, range) pairs are dealt to the 8 XCDs in contiguous stretches, four row tiles down before the next column, so that the
// tiles an XCD works on at a time share operands in its L2.
__device__ __forceinline__ SegTile seg_tile(const SegArgs& a) {
  SegTile t;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  t.wm = wave >> 2; t.wn = wave & 3; t.l16 = lane & 15; t.kg = lane >> 4;
  const int items = a.tiles_m * a.tiles_n * a.splits, per = (items + 7) / 8;
  const int item = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  t.live = (int)(blockIdx.x >> 3) < per && item < items;
  const int u = item / a.splits;
  t.split = item - u * a.splits;
  const int band = u / (4 * a.tiles_n), rows = a.tiles_m - 4 * band < 4 ? a.tiles_m - 4 * band : 4;
  const int inside = u - band * 4 * a.tiles_n;
  t.tm = 4 * band + inside % rows;
  t.tn = inside / rows;
  return t;
}

__device__ __forceinline__ void seg_clear(SegAcc& acc) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
}

// The share of a range: pairs of steps first .. last - 1 out of `pairs`.
__device__ __forceinline__ int seg_first(int pairs, int split, int splits) { return (int)((int64_t)pairs * split / splits); }

// acc += pairs of steps s0 .. s1 - 1 (s0 < s1) of the segments.  Rows past the ends of the planes are the last row again: what they
// give lands in rows and columns of C that nobody stores.  All transfers have landed and all operands have been read when it
// returns, but wavefronts come out one by one: a barrier has to stand before the LDS is used for anything else.
//
// Tiles of 32-deep steps go from global memory straight into LDS, into a ring of five slots, and the two steps of a pair together:
// the halves of a 128-byte line one after the other, so that the line comes out of the L2 once (4096 x 8192 x 4096, transfers
// without products: 128 us, with steps on their own 167).  One barrier per step: past it everyone has the operands of the step in
// registers, and its slot is free; the operands of the next step are read between the products.  Products are 16 x 16 x 32: blocks
// of 32 x 32 x 16 take the same cycles, but the chip, which lowers its clock under this load, holds 1.9 GHz with these and 1.65 with
// those (1368 against 1220 TFLOP/s, call after call).  Rows are 64 bytes, unit u of a row stored at u ^ ((row / 4) % 4): the
// 16 lanes that read one unit of 16 rows fall into different banks.
template <typename H>
__device__ __forceinline__ void seg_products(const SegArgs& a, const SegTile& t, int s0, int s1, unsigned char* lds, SegAcc& acc) {
  typedef H hx8 __attribute__((ext_vector_type(8)));
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  // this wavefront's transfers: rows 32 wave .. + 31 of both tiles; lane l brings unit l % 4 ^ swizzle of row l / 4
  const int lrow = lane >> 2, unit = (lane & 3) ^ ((lrow >> 2) & 3);
  const int64_t arow = (int64_t)t.tm * SEG_T, brow = (int64_t)t.tn * SEG_T;
  int ra[2], rb[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int r = 32 * wave + 16 * q + lrow;
    const int64_t la = a.rows_a - 1 - arow, lb = a.rows_b - 1 - brow;
    ra[q] = r < la ? r : (int)la;
    rb[q] = r < lb ? r : (int)lb;
  }
  const uint16_t *pa, *pb;
  uint32_t va[2], vb[2];
  int next = s0, seg = 0, end;
  auto enter = [&](int64_t k) {
    const Segment& g = a.seg[seg];
    pa = g.A + arow * g.pitch_a + k;
    pb = g.B + brow * g.pitch_b + k;
    end = g.end;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      va[q] = (uint32_t)(ra[q] * g.pitch_a * 2 + unit * 16);
      vb[q] = (uint32_t)(rb[q] * g.pitch_b * 2 + unit * 16);
    }
  };
  while (s0 >= a.seg[seg].end) ++seg;
  enter(64 * (int64_t)(s0 - (seg ? a.seg[seg - 1].end : 0)));
  auto transfer = [&](int part, int half, uint32_t slot) __attribute__((always_inline)) {     // a quarter of a step's transfers
    transfer_to_lds((part < 2 ? pa : pb) + 32 * half, part < 2 ? va[part & 1] : vb[part & 1],
                    slot + (part < 2 ? 0u : SEG_TILE) + (uint32_t)wave * 2048u + 1024u * (part & 1));
  };
  auto advance = [&]() {                         // past the end: the last pair again, into slots that nobody reads any more
    if (next + 1 >= s1) return;
    ++next;
    if (next == end) { ++seg; enter(0); }
    else { pa += 64; pb += 64; }
  };
  const uint32_t u0 = (uint32_t)(t.kg ^ ((t.l16 >> 2) & 3)) * 16u;
  const uint32_t aoff = (uint32_t)(128 * t.wm + t.l16) * 64u + u0, boff = SEG_TILE + (uint32_t)(64 * t.wn + t.l16) * 64u + u0;
  hx8 x[2][8], y[2][4];                          // operands of the present and the next step
  auto read = [&](uint32_t slot, int g, int part) __attribute__((always_inline)) {     // one of twelve, in the order of their use
    if (part == 0 || part > 4) {
      const int i = part ? part - 4 : 0;
      x[g][i] = *reinterpret_cast<const hx8*>(lds + (slot + aoff) + 1024u * i);
    } else {
      y[g][part - 1] = *reinterpret_cast<const hx8*>(lds + (slot + boff) + 1024u * (part - 1));
    }
  };
  auto after = [](uint32_t slot) { return slot == (SEG_SLOTS - 1) * SEG_STAGE ? 0u : slot + SEG_STAGE; };
#pragma unroll
  for (int p = 0; p < 2; ++p) {
#pragma unroll
    for (int part = 0; part < 4; ++part) {
      transfer(part, 0, 2 * p * SEG_STAGE);
      transfer(part, 1, (2 * p + 1) * SEG_STAGE);
    }
    advance();
  }
  asm volatile("s_waitcnt vmcnt(8)\n\ts_barrier" ::: "memory");     // 8 transfers a pair: the first pair's are done
#pragma unroll
  for (int part = 0; part < 12; ++part) read(0, 0, part);
  uint32_t rd = SEG_STAGE, wr = 4 * SEG_STAGE;   // the slot read next; the first of the two that are refilled next
  auto step = [&](auto odd) __attribute__((always_inline)) {
    constexpr int u = decltype(odd)::value;
    // The step after an odd one begins a pair: it has arrived when at most the transfers of the pair behind it are outstanding.
    if (u) asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const uint32_t w2 = after(wr);
#pragma unroll
    for (int n = 0; n < 32; ++n) {
      const int i = n >> 2, j = n & 3;
      if constexpr (std::is_same<H, __bf16>::value)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[u][i], y[u][j], acc[i][j], 0, 0, 0);
      else
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[u][i], y[u][j], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if ((n % 5 == 1 || n % 5 == 3) && n < 30) {                  // past the end: a slot's old contents, never used
        read(rd, u ^ 1, n / 5 * 2 + (n % 5 == 3));
        __builtin_amdgcn_sched_barrier(0);
      }
      if (n % 4 == 2 && u == 0) {
        transfer(n / 8, (n / 4) & 1, (n / 4) & 1 ? w2 : wr);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    rd = after(rd);
    if (u == 0) { wr = after(w2); advance(); }
  };
  for (int s = s0; s < s1; ++s) {
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");       // nothing lands in LDS any more
}

// f(v, row, column) for the wavefront's blocks: v holds rows row .. row + 3 of one column.
template <class F>
__device__ __forceinline__ void seg_each(const SegTile& t, const SegAcc& acc, F&& f) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      f(acc[i][j], (int64_t)t.tm * SEG_T + 128 * t.wm + 16 * i + 4 * t.kg, (int64_t)t.tn * SEG_T + 64 * t.wn + 16 * j + t.l16);
}

}  // namespace lq
