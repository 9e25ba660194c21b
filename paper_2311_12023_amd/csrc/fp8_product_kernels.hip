// The product of matrices in 8 bits for many rows: 256 x 256 tiles on the matrix unit.
#include "dense_device.h"
#include "fp8.h"
#include "fp8_device.h"
#include "lds_transfer.h"
#include "profiler.h"
#include "segment_gemm.h"

namespace lq {

constexpr int PT = 256, P_THREADS = 512;
constexpr uint32_t P_SIDE = PT * 128, P_STAGE = 2 * P_SIDE;         // bytes of an operand's block, of both
constexpr uint32_t P_SCALES = 2 * P_STAGE;                          // behind the stages: scales of the rows and columns of each
constexpr size_t P_LDS = P_SCALES + 2 * (2 * PT * 4);

struct ProductArgs {
  Fp8Operand rows, columns;
  int64_t k;
  void* out; int64_t ld;
  float* part;
  int tiles_r, tiles_c, splits, blocks;
  bool vec;                                                         // whole 16-byte stores
};
struct ProductTile { int tr, tc; };
__device__ __forceinline__ ProductTile product_tile(const ProductArgs& a, int u) {
  const int band = u / (4 * a.tiles_c), high = min(a.tiles_r - 4 * band, 4), inside = u - band * 4 * a.tiles_c;
  return {4 * band + inside % high, inside / high};
}

// Four rows of one column as they go into the output.
__device__ __forceinline__ uintx2 product_result(floatx4 v) {
  return __builtin_bit_cast(uintx2, bf16x4{(__bf16)(v[0] * FP8_DROP), (__bf16)(v[1] * FP8_DROP), (__bf16)(v[2] * FP8_DROP), (__bf16)(v[3] * FP8_DROP)});
}

// 4096 columns x 11008 rows, median and smallest of 40 launches: depth 4096 174 and 161 us (2.12 and 2.29 PFLOP/s), depth 11008 424 and 409
// (2.34 and 2.43); rows with scales of their own, depth 4096, 205 and 195 (1.80 and 1.89).  The chip's power is the
// limit: the clock is 2.1 GHz and the matrix units are busy for half of its cycles, waits and barriers taken out change nothing, transfers or
// sums taken out 17 % and 11 %.  Where rows have scales of their own these have to be below 2^98 in the columns' operand and 2^103 in the
// rows' one, or a factor on the way overflows: splitting them too would be a third vector instruction for every sum.
//
// A workgroup of eight wavefronts makes a tile, a wavefront 128 x 64 of it (2 x 4) in blocks of 16 x 16.  A block of 128 along k is one
// matrix instruction, whose four sums a lane are multiplied by the two scales into the accumulators: one vector instruction each where
// the rows' scales are of tiles (one scale for the wavefront's 128 rows), else two.
//
// LDS holds two blocks of both operands.  Rows are 128 bytes, unit u of 16 bytes of row r stored at u ^ (r % 8): a read of 16 rows
// x 4 units touches every bank alike.  Blocks of 16 rows are taken two at a time; before the last two of a block of 128, all its operands are
// in registers, so one barrier there tells that the next block has landed and that this one's place is free, and the next block's
// first operands are read under the last products.
template <bool ROW_TILES>
__global__ __launch_bounds__(P_THREADS) void fp8_product_kernel(ProductArgs a) {
  extern __shared__ __align__(16) unsigned char lds[];
  const int item = seg_piece(a.tiles_r * a.tiles_c * a.splits);
  if (item < 0) return;
  // ranges first: the tiles of a range share its operands in an XCD's L2
  const int tiles = a.tiles_r * a.tiles_c, split = item / tiles, u = item - split * tiles;
  const ProductTile t = product_tile(a, u);
  const int b0 = (int)((int64_t)a.blocks * split / a.splits), b1 = (int)((int64_t)a.blocks * (split + 1) / a.splits);
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int wm = wave >> 2, wn = wave & 3, l16 = lane & 15, kg = lane >> 4;
  const int64_t row0 = (int64_t)t.tr * PT, column0 = (int64_t)t.tc * PT;

  // transfers: rows 32 wave + 8 q + lane / 8 of either operand, unit lane % 8 ^ (row % 8); rows past the end are the last one again
  const int unit = (lane & 7) ^ (lane >> 3);
  uint32_t va[4], vb[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int r = 32 * wave + 8 * q + (lane >> 3);
    const int64_t la = a.rows.count - 1 - row0, lb = a.columns.count - 1 - column0;
    va[q] = (uint32_t)((r < la ? r : la) * a.rows.ld + 16 * unit);
    vb[q] = (uint32_t)((r < lb ? r : lb) * a.columns.ld + 16 * unit);
  }
  // units past the row's end read its last one
  const int rest = (int)(a.k - (int64_t)(a.blocks - 1) * 128);      // bytes of the last block, 1 .. 128
  const int past = 16 * unit - ((rest - 1) & ~15);
  const uint32_t back = past > 0 ? (uint32_t)past : 0u;
  const uint8_t* pa = a.rows.codes + row0 * a.rows.ld;
  const uint8_t* pb = a.columns.codes + column0 * a.columns.ld;
  // scales: wavefronts 0 .. 3 those of 64 rows each, 4 .. 7 of the columns
  const Fp8Operand& so = wave < 4 ? a.rows : a.columns;
  const int64_t s0 = wave < 4 ? row0 : column0, sr = min(s0 + 64 * (wave & 3) + lane, so.count - 1);
  const float* ps = so.scale + (s0 >> so.shift) * so.scale_row;
  const uint32_t vs = (uint32_t)(((sr >> so.shift) - (s0 >> so.shift)) * so.scale_row * 4);
  const int64_t sblock = so.scale_block;
  auto transfer = [&](int n, int b, uint32_t stage) __attribute__((always_inline)) {      // piece n of 9 of block b
    const uint32_t less = b == a.blocks - 1 ? back : 0u;
    const uint32_t to = stage * P_STAGE + (uint32_t)wave * 4096u;
    if (n < 4) transfer_to_lds(reinterpret_cast<const uint16_t*>(pa + (int64_t)b * 128), va[n & 3] - less, to + 1024u * n);
    else if (n < 8) transfer_to_lds(reinterpret_cast<const uint16_t*>(pb + (int64_t)b * 128), vb[n & 3] - less, to + P_SIDE + 1024u * (n - 4));
    else transfer_word_to_lds(ps + b * sblock, vs, P_SCALES + stage * (2 * PT * 4) + 256u * wave);
  };
  // The last block's bytes past k become 0: everyone in what they brought themselves.
  auto clear_past = [&](uint32_t stage) __attribute__((always_inline)) {
    // one after the other: all operands are in registers meanwhile, few are left
    const int left = rest - 16 * unit;
    if (left < 16) {
      unsigned char* at = lds + stage * P_STAGE + wave * 4096 + 16 * lane;
#pragma unroll 1
      for (int n = 0; n < 8; ++n) {
        uintx4* v = reinterpret_cast<uintx4*>(at + (n >> 2) * P_SIDE + (n & 3) * 1024);
        uintx4 w = {0, 0, 0, 0};
        if (left > 0) {
          w = *v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int bytes = left - 4 * e;
            w[e] = bytes >= 4 ? w[e] : bytes <= 0 ? 0u : w[e] & ((1u << (8 * bytes)) - 1u);
          }
        }
        *v = w;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };

  // operands: row 16 i + l16 (of the wavefront's), units kg and 4 + kg of the block
  const uint32_t sw = (uint32_t)(l16 & 7), u0 = ((uint32_t)kg ^ sw) * 16u, u1 = ((uint32_t)(4 + kg) ^ sw) * 16u;
  uint32_t xa = (uint32_t)(128 * wm + l16) * 128u + u0, xb = xa - u0 + u1;
  uint32_t ya = P_SIDE + (uint32_t)(64 * wn + l16) * 128u + u0, yb = ya - u0 + u1;
  uint32_t sa = P_SCALES + 4u * (128 * wm + (ROW_TILES ? 0 : 4 * kg)), sb = P_SCALES + 4u * (PT + 64 * wn + l16);
  auto operand = [&](uint32_t first, uint32_t second) __attribute__((always_inline)) -> intx8 {
    const uintx4 x = *reinterpret_cast<const uintx4*>(lds + first), y = *reinterpret_cast<const uintx4*>(lds + second);
    return intx8{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
  };
  float acc[8][4][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
  auto sums = [&](int i, int j) __attribute__((always_inline)) { return floatx4{acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]}; };
  intx8 x[4], y[4];
  floatx4 p[2][2], r[4];
  float s[4], last;                                  // last: the fourth scale of the block before, for its last sums
  float row_scale = 0.0f;                            // of the rows' tile, from its first use in a block on the fraction
  int row_exponent = 0;
  auto read_x = [&](int i) __attribute__((always_inline)) {
    x[i & 3] = operand(xa + 2048u * i, xb + 2048u * i);
    if constexpr (!ROW_TILES) r[i & 3] = *reinterpret_cast<const floatx4*>(lds + sa + 64 * i);
  };
  auto read_y = [&](int j) __attribute__((always_inline)) { y[j] = operand(ya + 2048u * j, yb + 2048u * j); };
  auto read_s = [&](int j) __attribute__((always_inline)) { s[j] = *reinterpret_cast<const float*>(lds + sb + 64 * j); };
  auto read_row_scale = [&]() __attribute__((always_inline)) {
    if constexpr (ROW_TILES) row_scale = *reinterpret_cast<const float*>(lds + sa);
  };
  // The product of both with its lift, as in fp8_lifted, by the fraction and the exponent of the rows' scale: neither may be lifted alone,
  // which overflows from 2^98 on (depth 11008 144.3 -> 145.4 us for it, 146.2 by a choice of the one to lift).
  auto split_row_scale = [&]() __attribute__((always_inline)) {
    row_exponent = __builtin_amdgcn_frexp_expf(row_scale) + 30;
    row_scale = __builtin_amdgcn_frexp_mantf(row_scale);
  };
  auto turn = [&]() __attribute__((always_inline)) {
    xa ^= P_STAGE; xb ^= P_STAGE; ya ^= P_STAGE; yb ^= P_STAGE;
    sa ^= 2 * PT * 4; sb ^= 2 * PT * 4;
  };
  auto add = [&](int ii, int j, int h, float f) __attribute__((always_inline)) {       // sums of block 2 ii + h and column block j
    const int i = 2 * ii + h;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(ROW_TILES ? p[j & 1][h][e] : p[j & 1][h][e] * r[i & 3][e], f, acc[i][j][e]);
    // kept here: moved behind a later branch they would leave all of p alive
    asm volatile("" : "+v"(acc[i][j][0]), "+v"(acc[i][j][1]), "+v"(acc[i][j][2]), "+v"(acc[i][j][3]));
  };
  // pieces 4 .. 7 are the columns', the others the rows' and the scales
#pragma unroll
  for (int n = 0; n < 9; ++n) transfer(n, b0, 0);
#pragma unroll
  for (int n = 0; n < 9; ++n) transfer(n, min(b0 + 1, b1 - 1), 1);
  asm volatile("s_waitcnt vmcnt(9)" ::: "memory");
  if (b0 == a.blocks - 1 && rest < 128) clear_past(0);
  asm volatile("s_barrier" ::: "memory");
  read_row_scale();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    read_y(j);
    if (j < 2) read_x(j);
    read_s(j);
  }
  last = 0.0f;
#pragma unroll
  for (int h = 0; h < 2; ++h) p[1][h] = r[2 + h] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  uint32_t stage = 0;
  // Past the last block the last one comes again, into a place whose contents nobody uses any more.
  // All columns' operands of a block are in registers when it begins, so their place is free then and takes those of two blocks on while
  // this one is under way; the rows' is free before its last products.
  for (int b = b0; b < b1; ++b) {
    const int next = min(b + 2, b1 - 1);
#pragma unroll
    for (int ii = 0; ii < 4; ++ii) {
      if (ii == 1) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (ii == 3) {
        // outstanding are at most the four transfers of this block
        asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)" ::: "memory");
        if (rest < 128 && b + 2 == a.blocks) clear_past(stage ^ 1);
        asm volatile("s_barrier" ::: "memory");
        turn();
        last = s[3];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        auto product = [&](int h) __attribute__((always_inline)) {
          p[j & 1][h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x[(2 * ii + h) & 3], y[j], floatx4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        };
        auto sum = [&](int h) __attribute__((always_inline)) {
          if (j) add(ii, j - 1, h, s[j - 1]);
          else if (ii) add(ii - 1, 3, h, s[3]);
          else add(3, 3, h, last);                   // of the block before
          __builtin_amdgcn_sched_barrier(0);
        };
        // 4096 x 4096 by 11008, smallest: products and sums in turn 161 us, two by two 164; with scales of rows 196 and 193
        if constexpr (ROW_TILES) {
          product(0); sum(0); product(1); sum(1);
        } else {
          product(0); product(1); sum(0); sum(1);
        }
        if (ii < 3) {
          if (ii == 0) {
            if (ROW_TILES && j == 0) split_row_scale();
            s[j] = ROW_TILES ? __builtin_amdgcn_ldexpf(s[j] * row_scale, row_exponent) : s[j] * FP8_LIFT;
          }
          if (j < 2) read_x(2 * ii + 2 + j);
          if (ii == 1) transfer(4 + j, next, stage);
        } else {
          // a scale's place is free once its last sums are through
          if (j == 0) read_row_scale();
          read_s((j + 3) & 3);
          read_y(j);
          if (j < 2) read_x(j);
          transfer(j, next, stage);
          if (j == 3) transfer(8, next, stage);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    stage ^= 1;
  }
  add(3, 3, 0, last);
  add(3, 3, 1, last);
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");

  const int64_t row = row0 + 128 * wm;
  if (a.splits > 1) {
    floatx4* part = reinterpret_cast<floatx4*>(a.part) + ((size_t)u * a.splits + split) * (PT * PT / 4) + tid;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) part[(i * 4 + j) * P_THREADS] = sums(i, j);
    return;
  }
  // The output by way of the LDS, a wavefront's 64 columns of 128 rows (256 bytes, units of 16 bytes turned by the column) for itself: whole
  // lines of a column, and little code, which a kernel this large otherwise waits for more than for its stores.
  asm volatile("s_barrier" ::: "memory");            // everyone has read their operands
  unsigned char* mine = lds + wave * 16384;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uintx2*>(mine + (16 * j + l16) * 256 + ((32 * i + 8 * kg) ^ (16 * l16))) = product_result(sums(i, j));
  __bf16* out = static_cast<__bf16*>(a.out);
  const int64_t first = column0 + 64 * wn, rows_left = a.rows.count - row, columns_left = a.columns.count - first;
  if (a.vec && rows_left >= 128) {
    const int unit16 = lane & 15, c = lane >> 4;
#pragma unroll 2
    for (int n = 0; n < 16; ++n) {
      const int at = 4 * n + c;
      const uintx4 w = *reinterpret_cast<const uintx4*>(mine + at * 256 + ((16 * unit16) ^ (16 * (at & 15))));
      if (at < columns_left) *reinterpret_cast<uintx4*>(out + (first + at) * a.ld + row + 8 * unit16) = w;
    }
  } else {
    // Odd lengths or addresses, or a last tile: halves of lines, value by value, eight of them read from the LDS before the first is stored
    // (4096 x 11007 x 4096: 174 us, one after the other 201; 1000 x 50265 x 1024: 91, 126).
#pragma unroll 1
    for (int n = 0; n < 128; n += 8) {
      __bf16 v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int at = (n + q) >> 1, r16 = 64 * (q & 1) + lane;
        v[q] = *reinterpret_cast<const __bf16*>(mine + at * 256 + ((2 * r16) ^ (16 * (at & 15))));
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int at = (n + q) >> 1, r16 = 64 * (q & 1) + lane;
        if (at < columns_left && r16 < rows_left) out[(first + at) * a.ld + row + r16] = v[q];
      }
    }
  }
}

// Sum of a tile's ranges in order; a workgroup takes one block of 16 rows and 16 columns of every wavefront's part.
__global__ __launch_bounds__(P_THREADS) void fp8_join_kernel(ProductArgs a) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, wm = wave >> 2, wn = wave & 3, l16 = lane & 15, kg = lane >> 4;
  const int u = blockIdx.x, i = blockIdx.y >> 2, j = blockIdx.y & 3;
  const ProductTile t = product_tile(a, u);
  const floatx4* part = reinterpret_cast<const floatx4*>(a.part) + (size_t)u * a.splits * (PT * PT / 4) + (i * 4 + j) * P_THREADS + tid;
  const int64_t row = (int64_t)t.tr * PT + 128 * wm + 16 * i + 4 * kg, column = (int64_t)t.tc * PT + 64 * wn + 16 * j + l16;
  if (row >= a.rows.count || column >= a.columns.count) return;
  floatx4 v = {};
  for (int s = 0; s < a.splits; s += 8) {            // eight under way together
    floatx4 x[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = part[(size_t)min(s + q, a.splits - 1) * (PT * PT / 4)];
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (s + q < a.splits) v += x[q];
  }
  const uintx2 w = product_result(v);
  __bf16* out = static_cast<__bf16*>(a.out) + column * a.ld + row;
  if (a.vec && row + 4 <= a.rows.count) {
    *reinterpret_cast<uintx2*>(out) = w;
  } else {
    const bf16x4 each = __builtin_bit_cast(bf16x4, w);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (row + e < a.rows.count) out[e] = each[e];
  }
}

static int64_t product_tiles(int64_t rows, int64_t columns) { return ((rows + PT - 1) / PT) * ((columns + PT - 1) / PT); }
// Ranges that the sum is cut into where there are few tiles: they fill the chip, each keeps four blocks (1024 x 1000, depth 50265: 16
// tiles in 16 ranges 56 us, their join 11; with the ranges of a tile next to one another, which then share nothing in an L2, 75 us).
static int product_splits(int64_t rows, int64_t columns, int64_t k) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(256 / std::max<int64_t>(1, product_tiles(rows, columns)), fp8_blocks(k) / 4));
}
size_t fp8_tiles_part_floats(int64_t rows, int64_t columns, int64_t k) {
  const int s = product_splits(rows, columns, k);
  return s > 1 ? (size_t)s * product_tiles(rows, columns) * PT * PT : 0;
}

template <bool ROW_TILES>
static int launch(const ProductArgs& a, hipStream_t st) {
  static LdsLimit limit;
  LQ_TRY(limit.raise(reinterpret_cast<const void*>(fp8_product_kernel<ROW_TILES>), P_LDS));
  const unsigned wgs = (unsigned)(((int64_t)a.tiles_r * a.tiles_c * a.splits + 7) / 8 * 8);
  hipLaunchKernelGGL(fp8_product_kernel<ROW_TILES>, dim3(wgs), dim3(P_THREADS), P_LDS, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

int launch_fp8_tiles(const Fp8Product& p, float* part, size_t part_floats, hipStream_t st) {
  if (product_tiles(p.rows.count, p.columns.count) >= ((int64_t)1 << 28)) return LQ_ERR_SHAPE;
  ProductArgs a{p.rows, p.columns, p.k, p.out, p.ld, part, (int)((p.rows.count + PT - 1) / PT), (int)((p.columns.count + PT - 1) / PT),
                product_splits(p.rows.count, p.columns.count, p.k), (int)fp8_blocks(p.k), p.ld % 8 == 0 && ((uintptr_t)p.out & 15) == 0};
  if (part_floats < fp8_tiles_part_floats(p.rows.count, p.columns.count, p.k)) return LQ_ERR_WORKSPACE;
  {
    prof::Scope ps(prof::FP8_PRODUCT, st, 2.0 * p.rows.count * p.columns.count * p.k);
    LQ_TRY(p.rows.shift ? launch<true>(a, st) : launch<false>(a, st));
  }
  if (a.splits == 1) return LQ_OK;
  prof::Scope ps(prof::FP8_JOIN, st, (double)fp8_tiles_part_floats(p.rows.count, p.columns.count, p.k) * 4);
  hipLaunchKernelGGL(fp8_join_kernel, dim3((unsigned)(a.tiles_r * a.tiles_c), 32), dim3(P_THREADS), 0, st, a);
  LQ_HIP_TRY(hipGetLastError());
  return LQ_OK;
}

}  // namespace lq
