// The matrix product that the training operators share:  C = sum over segments of A_s B_s^T  for bf16 planes with the reduction
// index contiguous.  A segment is a pair of planes; operands in fp32 are split into bf16 hi + lo and go in as the three segments
// hi hi, lo hi, hi lo (the products that are left out are below 2^-16 of those kept).  What becomes of a tile of C is up to the
// kernel that calls it.
#pragma once
#include "dense_device.h"
#include "lds_transfer.h"
#include "mfma_device.h"
#include "train.h"

namespace lq {

// One workgroup of 512 threads owns a 256 x 256 tile, a wavefront 128 x 64 of it (2 x 4); the loop is that of plane_gemm_kernel:
// 32-deep steps through four LDS stages, one barrier per step.  Accumulator element e of acc[i][j] is row
// 32 i + 8 (e / 4) + 4 lh + e % 4, column 32 j + ln of the wavefront's part (ln = lane % 32, lh = lane / 32).
struct SegTile {
  int tm, tn, split;
  int wm, wn, ln, lh;
  bool live;
};

// (tile, range) pairs are dealt to the 8 XCDs in contiguous stretches, four row tiles down before the next column, so that the
// tiles an XCD works on at a time share operands in its L2.
__device__ __forceinline__ SegTile seg_tile(const SegArgs& a) {
  SegTile t;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  t.wm = wave >> 2; t.wn = wave & 3; t.ln = lane & 31; t.lh = lane >> 5;
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

__device__ __forceinline__ void seg_clear(floatx16 (&acc)[4][2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
}

// acc += steps s0 .. s1 - 1 (s0 < s1) of the segments.  Rows past the ends of the planes are the last row again: what they
// give lands in rows and columns of C that nobody stores.  All transfers have landed and been read when it returns, but
// wavefronts come out one by one: a barrier has to stand before the LDS is used for anything else.
__device__ __forceinline__ void seg_products(const SegArgs& a, const SegTile& t, int s0, int s1, unsigned char* lds,
                                             floatx16 (&acc)[4][2]) {
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int ln = t.ln, lh = t.lh;
  // this wavefront's transfers: rows 16 wave .. + 15 and 128 further of both tiles; lane l brings unit l % 4 ^ swizzle of row l / 4
  const int lrow = lane >> 2, unit = (lane & 3) ^ ((lrow >> 2) & 3);
  const int64_t arow = (int64_t)t.tm * SEG_T, brow = (int64_t)t.tn * SEG_T;
  int ra[2], rb[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = 16 * wave + lrow + 128 * h;
    const int64_t la = a.rows_a - 1 - arow, lb = a.rows_b - 1 - brow;
    ra[h] = r < la ? r : (int)la;
    rb[h] = r < lb ? r : (int)lb;
  }
  const uint16_t *pa, *pb;
  uint32_t va[2], vb[2];
  int next = s0, seg = 0;
  auto enter = [&](int64_t k) {
    const Segment& g = a.seg[seg];
    pa = g.A + arow * g.pitch_a + k;
    pb = g.B + brow * g.pitch_b + k;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      va[h] = (uint32_t)(ra[h] * g.pitch_a * 2 + unit * 16);
      vb[h] = (uint32_t)(rb[h] * g.pitch_b * 2 + unit * 16);
    }
  };
  while (s0 >= a.seg[seg].end) ++seg;
  enter(32 * (int64_t)(s0 - (seg ? a.seg[seg - 1].end : 0)));
  auto transfer = [&](int part, int stage) {
    const uint32_t at = (uint32_t)stage * SEG_STAGE + (uint32_t)wave * 1024u + 8192u * part;
    transfer_to_lds(part < 2 ? pa : pb, part < 2 ? va[part & 1] : vb[part & 1], at);
  };
  auto advance = [&]() {                         // past the end: the last step again, into a stage that nobody reads any more
    if (next + 1 >= s1) return;
    ++next;
    if (next == a.seg[seg].end) { ++seg; enter(0); }
    else { pa += 32; pb += 32; }
  };
  uint32_t aoff[2], boff[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const uint32_t u = (uint32_t)((2 * g + lh) ^ ((ln >> 2) & 3)) * 16u;
    aoff[g] = (uint32_t)(128 * t.wm + ln) * 64u + u;
    boff[g] = SEG_TILE + (uint32_t)(64 * t.wn + ln) * 64u + u;
  }
  bf16x8 x[2][4], b[2][2];                       // operands of the two halves of a step
  auto read = [&](int stage, int g) __attribute__((always_inline)) {
    const unsigned char* from = lds + (uint32_t)stage * SEG_STAGE;
#pragma unroll
    for (int j = 0; j < 2; ++j) b[g][j] = *reinterpret_cast<const bf16x8*>(from + boff[g] + 2048u * j);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[g][i] = *reinterpret_cast<const bf16x8*>(from + aoff[g] + 2048u * i);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](int g, int i) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[g][i], b[g][j], acc[i][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int p = 0; p < SEG_STAGES; ++p) {
#pragma unroll
    for (int part = 0; part < 4; ++part) transfer(part, p);
    advance();
  }
  asm volatile("s_waitcnt vmcnt(12)\n\ts_barrier" ::: "memory");
  read(0, 0);
  auto step = [&](auto stage) __attribute__((always_inline)) {
    constexpr int u = decltype(stage)::value;
    read(u, 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) multiply(0, i);
    asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    read((u + 1) % SEG_STAGES, 0);               // past the end: never used
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      multiply(1, i);
      transfer(i, u);
      __builtin_amdgcn_sched_barrier(0);
    }
    advance();
  };
  int s = s0;
  for (; s + SEG_STAGES <= s1; s += SEG_STAGES) for_each_block<SEG_STAGES>(step);
  for_each_block<SEG_STAGES - 1>([&](auto stage) { if (s + decltype(stage)::value < s1) step(stage); });
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// f(i, j, e, row, column) for every element of the wavefront's part of the tile.
template <class F>
__device__ __forceinline__ void seg_each(const SegTile& t, F&& f) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        f(i, j, e, (int64_t)t.tm * SEG_T + 128 * t.wm + 32 * i + 8 * (e >> 2) + 4 * t.lh + (e & 3),
          (int64_t)t.tn * SEG_T + 64 * t.wn + 32 * j + t.ln);
}

}  // namespace lq
