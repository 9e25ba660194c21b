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

// The wavefront's part of tile u, tiles in an order that goes down four row tiles before the next column.
__device__ __forceinline__ SegTile seg_tile_at(const SegArgs& a, int u) {
  SegTile t;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  t.wm = wave >> 2; t.wn = wave & 3; t.l16 = lane & 15; t.kg = lane >> 4;
  t.split = 0;
  t.live = true;
  const int band = u / (4 * a.tiles_n), rows = a.tiles_m - 4 * band < 4 ? a.tiles_m - 4 * band : 4;
  const int inside = u - band * 4 * a.tiles_n;
  t.tm = 4 * band + inside % rows;
  t.tn = inside / rows;
  return t;
}

// `count` pieces of work are dealt to the 8 XCDs in contiguous stretches, so that the tiles an XCD works on at a time share operands
// in its L2.  -> this workgroup's piece, or -1.
__device__ __forceinline__ int seg_piece(int count) {
  const int per = (count + 7) / 8, item = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  return (int)(blockIdx.x >> 3) < per && item < count ? item : -1;
}

// One (tile, range) pair a workgroup.
__device__ __forceinline__ SegTile seg_tile(const SegArgs& a) {
  const int item = seg_piece(a.tiles_m * a.tiles_n * a.splits), u = item < 0 ? 0 : item / a.splits;
  SegTile t = seg_tile_at(a, u);
  t.split = item - u * a.splits;
  t.live = item >= 0;
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
// those (1368 against 1220 TFLOP/s, call after call).  Rows are 64 bytes, unit u of a row stored at u ^ ((row / 2) % 4): reads
// of 16 rows x 4 units take 4 cycles of the LDS (with (row / 4) % 4, which serves 32 rows x 2 units, 8).
//
// TURNED: A's planes have its rows contiguous and the reduction index from row to row (W as it is stored, for E W), so a step is 32
// rows of 512 bytes in LDS and operands come out by transposed reads: 16 lanes read four reduction indices of 16 rows of A, a
// lane gets the four of its own.  The 32-byte chunk c of reduction index k is stored at c ^ (k % 4 + 4 (k / 8 % 2)): the sixteen
// indices that a read touches spread over the banks.  A pass that turned W beforehand took 47 us per 16384 x 4096 of it.
template <typename H, bool TURNED = false>
__device__ __forceinline__ void seg_products(const SegArgs& a, const SegTile& t, int s0, int s1, unsigned char* lds, SegAcc& acc) {
  typedef H hx8 __attribute__((ext_vector_type(8)));
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  // this wavefront's transfers: rows 32 wave .. + 31 of both tiles; lane l brings unit l % 4 ^ swizzle of row l / 4
  const int lrow = lane >> 2, unit = (lane & 3) ^ ((lrow >> 1) & 3);
  const int64_t arow = (int64_t)t.tm * SEG_T, brow = (int64_t)t.tn * SEG_T;
  int ra[2], rb[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int r = 32 * wave + 16 * q + lrow;
    const int64_t la = a.rows_a - 1 - arow, lb = a.rows_b - 1 - brow;
    ra[q] = r < la ? r : (int)la;
    rb[q] = r < lb ? r : (int)lb;
    if constexpr (TURNED) {
      // reduction indices 4 wave + 2 q + l / 32 of a step, unit l % 32 ^ chunk swizzle; a unit past the rows is the last one again
      const int k = 4 * wave + 2 * q + (lane >> 5), u = (lane & 31) ^ (((k & 3) + 4 * ((k >> 3) & 1)) * 2);
      ra[q] = 8 * u <= la - 7 ? 8 * u : (int)la - 7;
    }
  }
  const uint16_t *pa, *pb;
  uint32_t va[TURNED ? 4 : 2], vb[2];
  int next = s0, seg = 0, end, left = 0;         // left: TURNED, reduction indices of A from the present pair on
  auto place = [&]() __attribute__((always_inline)) {      // TURNED: indices past the end are the last one again (B is zero there)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int k = 4 * wave + 2 * (q & 1) + (lane >> 5) + 32 * (q >> 1);
      va[TURNED ? q : 0] = (uint32_t)((k < left ? k : left - 1) * a.seg[seg].pitch_a * 2 + ra[q & 1] * 2);
    }
  };
  auto enter = [&](int64_t k) {
    const Segment& g = a.seg[seg];
    if constexpr (TURNED) {
      pa = g.A + k * g.pitch_a + arow;
      left = (int)(a.depth_a - k);
      place();
    } else {
      pa = g.A + arow * g.pitch_a + k;
    }
    pb = g.B + brow * g.pitch_b + k;
    end = g.end;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      if constexpr (!TURNED) va[q] = (uint32_t)(ra[q] * g.pitch_a * 2 + unit * 16);
      vb[q] = (uint32_t)(rb[q] * g.pitch_b * 2 + unit * 16);
    }
  };
  while (s0 >= a.seg[seg].end) ++seg;
  enter(64 * (int64_t)(s0 - (seg ? a.seg[seg - 1].end : 0)));
  auto transfer = [&](int part, int half, uint32_t slot) __attribute__((always_inline)) {     // a quarter of a step's transfers
    if (part < 2)
      transfer_to_lds(TURNED ? pa : pa + 32 * half, va[TURNED ? part + 2 * half : part], slot + (uint32_t)wave * 2048u + 1024u * part);
    else
      transfer_to_lds(pb + 32 * half, vb[part & 1], slot + SEG_TILE + (uint32_t)wave * 2048u + 1024u * (part & 1));
  };
  auto advance = [&]() {                         // past the end: the last pair again, into slots that nobody reads any more
    if (next + 1 >= s1) return;
    ++next;
    if (next == end) { ++seg; enter(0); return; }
    pb += 64;
    if constexpr (TURNED) {
      pa += 64 * a.seg[seg].pitch_a;
      left -= 64;
      if (left < 64) place();
    } else {
      pa += 64;
    }
  };
  const uint32_t u0 = (uint32_t)(t.kg ^ ((t.l16 >> 1) & 3)) * 16u;
  // TURNED: index 8 kg + l16 / 4 of a step (and four further), chunk 8 wm + i: the swizzle takes in the indices' low bits and kg
  const uint32_t turn = (uint32_t)((t.l16 >> 2) + 4 * (t.kg & 1));
  const uint32_t aoff = TURNED ? (uint32_t)(8 * t.kg + (t.l16 >> 2)) * 512u + 8u * (t.l16 & 3) : (uint32_t)(128 * t.wm + t.l16) * 64u + u0, boff = SEG_TILE + (uint32_t)(64 * t.wn + t.l16) * 64u + u0;
  hx8 x[2][8], y[2][4];                          // operands of the present and the next step
  auto read_x = [&](uint32_t slot, int g, int i, int half) __attribute__((always_inline)) {
    if constexpr (TURNED) {
      typedef short shortx4 __attribute__((ext_vector_type(4)));
      typedef H hx4 __attribute__((ext_vector_type(4)));
      const uint32_t at = slot + aoff + (((uint32_t)(8 * t.wm + i) ^ turn) * 32u) + 2048u * half;
      const hx4 v = __builtin_bit_cast(hx4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)(lds + at)));
#pragma unroll
      for (int e = 0; e < 4; ++e) x[g][i][4 * half + e] = v[e];
    } else {
      x[g][i] = *reinterpret_cast<const hx8*>(lds + (slot + aoff) + 1024u * i);
    }
  };
  constexpr int XR = TURNED ? 2 : 1, READS = 8 * XR + 4;         // operand reads of a step, in the order of their use
  auto read = [&](uint32_t slot, int g, int part) __attribute__((always_inline)) {
    if (part < XR) read_x(slot, g, 0, part);
    else if (part < XR + 4) y[g][part - XR] = *reinterpret_cast<const hx8*>(lds + (slot + boff) + 1024u * (part - XR));
    else read_x(slot, g, (part - 4) / XR, (part - 4) % XR);
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
  for (int part = 0; part < READS; ++part) read(0, 0, part);
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
      if (n < 30 && (n + 1) * READS / 30 > n * READS / 30) {       // past the end: a slot's old contents, never used
        read(rd, u ^ 1, n * READS / 30);
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

// Two blocks of 16-bit values, four neighbours (of 16) a lane, become one block of eight neighbours a lane: lanes of even kg hold
// values 8 (kg / 2) .. of the first block then, those of odd kg the same of the second.
__device__ __forceinline__ uintx4 seg_pair_blocks(uintx2 first, uintx2 second) {
  const auto a = __builtin_amdgcn_permlane16_swap(first[0], second[0], false, false);
  const auto b = __builtin_amdgcn_permlane16_swap(first[1], second[1], false, false);
  return uintx4{a[0], b[0], a[1], b[1]};
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
