// Matrix products of e2m1 operands (4 bits) with a power-of-two scale for each 32 values along k, and the quantisation into them.
//
//   out[i][j] = sum over blocks kb of 32 of 2^(ea[i][kb] + eb[j][kb]) sum over k in kb of a[i][k] b[j][k]  + bias[j]
//
// The scaled MFMA of gfx950 takes 32 values of a row in 16 bytes of a lane, with the scale byte of that lane: a block of 32 is what a lane has.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "jenga_device.h"
#include "jenga_internal.h"
#include "jenga_tiles.h"

namespace {

using namespace jenga;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

int status() { return hipGetLastError() == hipSuccess ? JENGA_OK : JENGA_EHIP; }

// ---- quantisation: bound by memory

// Eight values a lane, four lanes to a block, 512 columns a wavefront at a time.  33272 x 5120 bf16: 82 us, 5.2 TB/s.
template <typename X>
__global__ __launch_bounds__(256) void quantize_mx_kernel(const X* __restrict__ x, int64_t x_stride, uint8_t* __restrict__ q,
                                                          uint8_t* __restrict__ scale, int64_t units, int cols, int quads) {
  const int lane = threadIdx.x & 63, padded = (cols + 127) >> 7 << 7;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); unit < units; unit += (int64_t)gridDim.x * 4) {
    const int64_t row = unit / quads;
    const int col = (int)(unit - row * quads) * 512 + lane * 8;
    const f32x8 v = Eight<X>::wide(load_eight(x + row * x_stride + col, cols - col));
    const uint32_t byte = mx_scale_byte(quad_max(magnitude_of(v)));
    if (col < padded) {
      *(uint32_t*)(q + row * (padded >> 1) + (col >> 1)) = to_e2m1(v, byte);
      if ((lane & 3) == 0) scale[row * (padded >> 5) + (col >> 5)] = (uint8_t)byte;
    }
  }
}

// ---- products

struct MatmulArgs {
  const uint8_t *a, *a_scale, *b, *b_scale;
  const float* bias;
  void* out;
  int64_t m, out_stride;
  int n, halves, steps;   // halves: blocks of 128 along k, 64 bytes of a row and four of its scales; steps: two of them
  int tiles_m, tiles_n;
};

// 16 bytes a lane: a row in lanes l and l + 32, 32 columns each, with the scale in byte B of xs or ys.
template <int B>
__device__ __forceinline__ f32x16 multiply(const i32x4& x, int xs, const i32x4& y, int ys, f32x16 acc) {
#if defined(__HIP_DEVICE_COMPILE__)
  const i32x8 wx = {x[0], x[1], x[2], x[3], 0, 0, 0, 0}, wy = {y[0], y[1], y[2], y[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wx, wy, acc, 4, 4, B, xs, B, ys);
#else
  return acc;
#endif
}
// The same for 16 rows, a row in lanes l, l + 16, l + 32 and l + 48.
__device__ __forceinline__ f32x4 multiply16(const i32x4& x, int xs, const i32x4& y, int ys, f32x4 acc) {
#if defined(__HIP_DEVICE_COMPILE__)
  const i32x8 wx = {x[0], x[1], x[2], x[3], 0, 0, 0, 0}, wy = {y[0], y[1], y[2], y[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wx, wy, acc, 4, 4, 0, xs, 0, ys);
#else
  return acc;
#endif
}

// Up to 16 R rows of a: the weight is read once and is what takes the time, so there are no tiles.  A workgroup makes 16 columns; its eight
// wavefronts take 128 columns of k each in turn, straight from memory into registers, four turns ahead, and add their sums up in LDS.
// 1 x 9216 x 1536: 4.7 us, 1.6 TB/s: a launch, a read and its sums.
template <typename O, int R>
__global__ __launch_bounds__(512) void matmul_mx_rows_kernel(MatmulArgs g) {
  constexpr int WAVES = 8, AHEAD = 4;
  __shared__ float sums[WAVES][R * 256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, part = lane >> 4;
  const int col0 = blockIdx.x * 16;
  const size_t pitch = (size_t)g.halves * 64, scales = (size_t)g.halves * 4;
  // rows and columns past the end: the last one again, and not stored
  const uint8_t *a[R], *a_scale[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t row = min((int64_t)(16 * r + i16), g.m - 1);
    a[r] = g.a + row * pitch + part * 16;
    a_scale[r] = g.a_scale + row * scales + part;
  }
  const size_t col = (size_t)min(col0 + i16, g.n - 1);
  const uint8_t *b = g.b + col * pitch + part * 16, *b_scale = g.b_scale + col * scales + part;
  f32x4 acc[R] = {};
  for (int s0 = wave; s0 < g.halves; s0 += AHEAD * WAVES) {
    i32x4 fb[AHEAD], fa[AHEAD][R];
    int sb[AHEAD], sa[AHEAD][R];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int s = s0 + u * WAVES;
      if (s < g.halves) {
        fb[u] = *(const i32x4*)(b + (size_t)s * 64);
        sb[u] = b_scale[s * 4];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          fa[u][r] = *(const i32x4*)(a[r] + (size_t)s * 64);
          sa[u][r] = a_scale[r][s * 4];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s0 + u * WAVES < g.halves)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r] = multiply16(fb[u], sb[u], fa[u][r], sa[u][r], acc[r]);
  }
#pragma unroll
  for (int r = 0; r < R; ++r)   // lane l holds row l % 16 of a, columns 4 (l / 16) to + 3
    *(f32x4*)&sums[wave][(16 * r + i16) * 16 + (lane >> 4) * 4] = acc[r];
  __syncthreads();
  for (int i = threadIdx.x; i < R * 256; i += 512) {
    const int row = i >> 4, to = col0 + (i & 15);
    if (row >= g.m || to >= g.n) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += sums[w][i];
    ((O*)g.out)[row * g.out_stride + to] = (O)(g.bias ? v + g.bias[to] : v);
  }
}

// 64 lanes x 4 or 16 bytes from a buffer, or nothing: without a branch, which would part the products from the reads and copies between them.
// Pieces of 16 bytes may lie on any multiple of four.
__device__ __forceinline__ void copy_dwords(bool wanted, const u32x4& buffer, uint32_t lane_offset, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_lo, %4\n\ts_mov_b32 exec_hi, %4\n\tbuffer_load_dword %1, %2, %3 offen lds\n\ts_mov_b64 exec, -1"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(lane_offset), "s"(buffer), "s"(__builtin_amdgcn_readfirstlane(offset)),
                 "s"(__builtin_amdgcn_readfirstlane(wanted ? -1 : 0))
               : "memory", "m0");
}
__device__ __forceinline__ void copy_pieces(bool wanted, const u32x4& buffer, uint32_t lane_offset, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_lo, %4\n\ts_mov_b32 exec_hi, %4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds\n\ts_mov_b64 exec, -1"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(lane_offset), "s"(buffer), "s"(__builtin_amdgcn_readfirstlane(offset)),
                 "s"(__builtin_amdgcn_readfirstlane(wanted ? -1 : 0))
               : "memory", "m0");
}

// Four wavefronts, 2 x 2, make BM x BN results, one tile after the other.  Blocks of 256 columns (128 bytes) of either operand are copied
// into one of STAGES LDS tiles while another is multiplied; within a block the products of one half of the columns run while the
// fragments of the next half are read into registers.  So the reads of an LDS tile end in the middle of its block, and that is where
// the barrier is: behind it the next tile is complete, and the one STAGES blocks on goes over this one.
//
// 33272 x 15360 x 5120 to bf16: 1.40 to 1.48 ms, 3.5 to 3.7 PFLOP/s (all-zero operands 1.15); without copies of operands 1.13, without scales
// 1.24, without stores 1.45 where it took 1.65: no part bounds it alone.  A wavefront a SIMD does them one after the other.  Products of one half before those of the other
// (two accumulations into a tile apart) and starts spread over a tile's time changed nothing; scales shifted at their first use 1.54.
//
// A copy instruction takes 8 whole rows of 128 bytes: first their left halves, then the right ones.  Where k has an odd number of halves,
// the last right one is taken from behind the buffer, as zeros.  The 16-byte pieces of a half row are rotated by an exclusive or with bits of the
// row, so that the rows of a fragment fall on all banks.  The rows of b are the rows of the matrix instruction, taken in an order that puts eight
// neighbouring results of a row of out into a lane: two fragments j, j + 1 hold columns 16 q + 8 (lane / 32) + 4 (j & 1) + 0..3 of 64.
// A lane has pieces 2 h and 2 h + 1 of a half row, h = lane / 32: two products, whose scales are those two bytes of the half row's four.
// Scales are copied 16 bytes a row, which serve four halves, in every other block; the last ones of a row end with it.  (Four bytes a row
// and instruction, 64 cache lines each: 33272 x 15360 x 5120 1646 us; 32 bytes 1483 where 16 take 1474.)  SHORT: rows of less than 16 bytes.  In LDS
// the rows of b lie as fragments want them, and a lane reads both halves' scales of a row at once: four bytes from every second row's, as they lie in
// memory, had up to four lanes on a bank.
template <typename O, int BM, int BN, int STAGES, bool SHORT>
__global__ __launch_bounds__(256) void matmul_mx_kernel(MatmulArgs g) {
  constexpr int WM = 2, WN = 2, MT = BM / WM / 32, NT = BN / WN / 32, COPIES = (BM + BN) / 32, STAGE = (BM + BN) * 128;
  constexpr int SCALE_COPIES = SHORT ? 6 : 2, ALL = COPIES + SCALE_COPIES;   // of a wavefront and block
  constexpr int SCALE_ROOM = (BM + BN) * 16, SCALE_ROOMS = STAGES / 2 + 1;
  static_assert(STAGES >= 2 && STAGES <= 4 && BM % 64 == 0 && BN % 64 == 0 && BN / WN <= 128 && 128 % (BN / WN) == 0 && NT % 2 == 0, "");
  // the results of 32 rows of each wavefront go where the tiles but the first are
  constexpr int PITCH = BN / WN * sizeof(O), REST = (STAGES - 1) * STAGE, SECOND = REST > 4 * 32 * PITCH ? REST : 4 * 32 * PITCH;
  constexpr int SCALES = STAGE + SECOND;   // [SCALE_ROOMS][BM + BN][16], SHORT: [.][4][BM + BN][4]
  __shared__ __attribute__((aligned(128))) uint8_t tiles[SCALES + SCALE_ROOMS * SCALE_ROOM + 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % WM, wn = wave / WM;
  const uint32_t pitch = (uint32_t)g.halves * 64, scale_pitch = (uint32_t)g.halves * 4,
                 lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)tiles;
  const int n_tiles = g.tiles_m * g.tiles_n, xcd = blockIdx.x & 7;
  const int end = (int)((int64_t)n_tiles * (xcd + 1) >> 3);
  int t = (int)((int64_t)n_tiles * xcd >> 3) + (blockIdx.x >> 3);
  if (t >= end) return;

  // of this lane, for the copies of its wavefront: 8 rows each, 32 rows apart, so that the rotations are the same for all
  const uint32_t from = (uint32_t)(wave * 8 + (lane >> 2 & 7)) * pitch + (lane >> 5) * 64;
  const uint32_t from_a = from + ((lane & 3) ^ ((2 * wave + (lane >> 4 & 1)) & 3)) * 16, from_b = from + ((lane & 3) ^ wave) * 16;
  const int cut = g.halves & 1 ? g.steps - 1 : -1;   // the block without a right half
  const int i32 = lane & 31, turn = (i32 >> 2 & 3) * 16, piece = (lane >> 5) * 32;
  const int ra = wm * (BM / WM) + i32;                                     // + 32 i
  const int rb = wn * (BN / WN) + 2 * (i32 & ~3) + (i32 & 3);              // + 64 (j / 2) + 4 (j & 1)
  const int at_a = (ra >> 3) * 1024 + (ra & 7) * 64, at_b = BM * 128 + (rb >> 3) * 1024 + (rb & 7) * 64;   // rb & 4 is 0

  // the tile whose operands are copied: that of the products, and behind its last block the next one
  u32x4 a_rows, b_rows, a_scales, b_scales;
  int64_t row0;
  int col0, rows, cols;
  auto begin_copies = [&](int tile) {
    int tm, tn;
    tile_at(tile, g.tiles_m, g.tiles_n, &tm, &tn);
    row0 = (int64_t)tm * BM;
    col0 = tn * BN;
    rows = (int)min(g.m - row0, (int64_t)BM);
    cols = min(g.n - col0, BN);
    a_rows = buffer_of(g.a + row0 * pitch, (uint32_t)rows * pitch);
    b_rows = buffer_of(g.b + (int64_t)col0 * pitch, (uint32_t)cols * pitch);
    a_scales = buffer_of(g.a_scale + row0 * scale_pitch, (uint32_t)rows * scale_pitch);
    b_scales = buffer_of(g.b_scale + (int64_t)col0 * scale_pitch, (uint32_t)cols * scale_pitch);
  };
  const uint32_t scales_a = lane * scale_pitch, scales_b = (4 * (lane >> 5) + 2 * (lane & 28) + (lane & 3)) * scale_pitch;
  auto copy_one = [&](int s, int c) {
    if (c < COPIES) {
      const bool of_a = c * 32 < BM;
      uint32_t lane_from = of_a ? from_a : from_b;
      if (s == cut && lane >= 32) lane_from = 0x80000000u;   // outside
      copy_1kb(of_a ? a_rows : b_rows, lane_from,
               s < g.steps ? (of_a ? c : c - BM / 32) * 32 * pitch + s * 128 : 0x80000000u,   // past the end: outside
               lds0 + (uint32_t)s % STAGES * STAGE + (c * 4 + wave) * 1024);
    } else {   // of 64 rows of an operand; where that has less than four times 64, of some of them twice
      const bool of_a = (c & 1) == 0;
      const int r = wave * 64 % (of_a ? BM : BN), half = (c - COPIES) >> 1;
      const uint32_t to = lds0 + SCALES + (uint32_t)(s >> 1) % SCALE_ROOMS * SCALE_ROOM;
      const u32x4& scales = of_a ? a_scales : b_scales;
      const int row = r + (of_a ? 0 : BM);
      if constexpr (SHORT)
        copy_dwords((s & 1) == 0, scales, of_a ? scales_a : scales_b,
                    half < g.halves - 2 * s ? (uint32_t)r * scale_pitch + (uint32_t)(s * 8 + half * 4) : 0x80000000u,
                    to + (half * (BM + BN) + row) * 4);
      else
        copy_pieces((s & 1) == 0, scales, of_a ? scales_a : scales_b, (uint32_t)r * scale_pitch + (uint32_t)min(2 * s, g.halves - 4) * 4, to + row * 16);
    }
  };

  f32x16 acc[MT][NT];
  i32x4 fa[2][MT][2], fb[2][NT][2];
  struct __attribute__((packed, aligned(4))) Two {
    uint32_t h[2];
  };
  Two both[MT + NT];       // as they come: four bytes a half
  int scale[2][MT + NT];   // this lane's two of them
  // Fragment r of half h of block s: those of b and a in the order in which the products want them.
  auto read_one = [&](int s, auto half, auto index) {
    constexpr int H = decltype(half)::value, R = decltype(index)::value;
    constexpr bool OF_A = R >= 1 && R <= MT;
    constexpr int I = OF_A ? R - 1 : 0, J = R == 0 || OF_A ? 0 : R - MT;
    const uint8_t* p = tiles + (uint32_t)s % STAGES * STAGE + H * 512 + (OF_A ? at_a + I * 4096 : at_b + (J >> 1) * 8192 + (J & 1) * 256);
    const uint4 v[2] = {*(const uint4*)(p + (piece ^ turn)), *(const uint4*)(p + ((piece + 16) ^ turn))};
    __builtin_memcpy(OF_A ? &fa[H][I] : &fb[H][J], v, 32);
    if constexpr (H == 0) {   // the scales of both halves; what stands for a half behind the last one is another's
      const int u = s >> 1, at = (u % SCALE_ROOMS) * SCALE_ROOM + (SHORT ? (2 * s & 3) * (BM + BN) * 4 : ((2 * s - min(4 * u, g.halves - 4)) & 3) * 4);
      const uint8_t* scales = tiles + SCALES + (OF_A ? (ra + 32 * I) : BM + wn * (BN / WN) + 32 * J + i32) * (SHORT ? 4 : 16) + at;
      if constexpr (SHORT) both[R] = {*(const uint32_t*)scales, *(const uint32_t*)(scales + (BM + BN) * 4)};
      else both[R] = *(const Two*)scales;
    }
  };
  using std::integral_constant;
  constexpr integral_constant<int, 0> n0;
  constexpr integral_constant<int, 1> n1;
  constexpr int PRODUCTS = MT * NT, READS = MT + NT;
  constexpr auto of_a = [](int i) { return i + 1; };
  constexpr auto of_b = [](int j) { return j == 0 ? 0 : j + MT; };
  const int by = (lane >> 5) * 16;
  // Multiplies block s.  Between the products are the reads of the next half and the copies of the block STAGES on.  (Left alone,
  // the compiler reads after the products and waits; all reads and copies before them leave the matrix core without work meanwhile:
  // 8192 x 8192 x 8192 585 -> 445 us.)  What is read and copied behind the last block is not used and not fetched: other code there
  // would cost more, in moves between registers.
  auto block = [&](int s) {
    const uint32_t there = 2 * s + 1 < g.halves ? ~0u : 0u;
#pragma unroll
    for (int r = 0; r < READS; ++r) {
      scale[0][r] = (int)(both[r].h[0] >> by);
      scale[1][r] = (int)((both[r].h[1] & there) >> by);
    }
    each<PRODUCTS>([&](auto index) {
      constexpr int N = decltype(index)::value;
      constexpr int I = N % MT, J = N / MT;
      acc[I][J] = multiply<0>(fb[0][J][0], scale[0][of_b(J)], fa[0][I][0], scale[0][of_a(I)], acc[I][J]);
      acc[I][J] = multiply<1>(fb[0][J][1], scale[0][of_b(J)], fa[0][I][1], scale[0][of_a(I)], acc[I][J]);
      each<READS>([&](auto r) {
        if constexpr (decltype(r)::value * (PRODUCTS - 1) / READS == N) read_one(s, n1, r);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    // this wavefront's copies of the next block are done (those of later blocks may be on their way), and its reads of this one;
    // then everybody's are
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((STAGES - 2) * COPIES) : "memory");
    __builtin_amdgcn_sched_barrier(0);
    each<PRODUCTS>([&](auto index) {
      constexpr int N = decltype(index)::value;
      constexpr int I = N % MT, J = N / MT;
      acc[I][J] = multiply<0>(fb[1][J][0], scale[1][of_b(J)], fa[1][I][0], scale[1][of_a(I)], acc[I][J]);
      acc[I][J] = multiply<1>(fb[1][J][1], scale[1][of_b(J)], fa[1][I][1], scale[1][of_a(I)], acc[I][J]);
      each<READS>([&](auto r) {
        if constexpr (decltype(r)::value * (PRODUCTS - 1) / READS == N) read_one(s + 1, n0, r);
      });
      each<ALL>([&](auto c) {
        if constexpr (decltype(c)::value * PRODUCTS / ALL == N) copy_one(s + STAGES, decltype(c)::value);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  // The results go through LDS, so that a store takes whole rows of the wavefront's columns.  Room for each wavefront in the second LDS
  // tile, for ROWS of its rows at a time.  They are not kept in the caches: the operands that they would drive out cost more (33272 x
  // 15360 x 5120: 2.40 -> 2.17 ms).
  constexpr int COLS = BN / WN, PIECES = PITCH / 16, FIT = SECOND / 4 / PITCH / 32 * 32,
                ROWS = FIT < MT * 32 ? FIT : MT * 32, AT_ONCE = 64 / PIECES;   // rows that a store takes
  constexpr int STORES = MT * 32 / AT_ONCE;
  static_assert(ROWS >= 32 && MT * 32 % ROWS == 0 && PIECES <= 64 && (STAGES - 1) * ALL <= 63, "");
  auto store_results = [&](int64_t row0, int col0, int rows, int cols) {
    uint8_t* room = tiles + STAGE + wave * (SECOND / 4);
    const int out_col = col0 + wn * COLS, left = g.n - out_col;
    const bool inside = rows == BM && cols == BN;
    each<MT * 32 / ROWS>([&](auto part) {
      constexpr int I0 = decltype(part)::value * (ROWS / 32);
      each<NT * 2>([&](auto index) {
        constexpr int J = decltype(index)::value / 4 * 2, Q = decltype(index)::value % 4;
        const int col = 32 * J + 16 * Q + 8 * (lane >> 5);
        f32x8 bias = 0.f;
        if (g.bias) {
#pragma unroll
          for (int e = 0; e < 8; ++e) bias[e] = g.bias[out_col + min(col + e, left - 1)];   // those past the end are not stored
        }
        each<ROWS / 32>([&](auto tile) {
          constexpr int I = decltype(tile)::value;
          const f32x16 &x = acc[I0 + I][J], &y = acc[I0 + I][J + 1];
          const f32x8 v = {x[4 * Q], x[4 * Q + 1], x[4 * Q + 2], x[4 * Q + 3], y[4 * Q], y[4 * Q + 1], y[4 * Q + 2], y[4 * Q + 3]};
          const auto raw = Eight<O>::narrow(v + bias);
          uint4 piece16[sizeof(O) / 2];
          __builtin_memcpy(piece16, &raw, sizeof(raw));
#pragma unroll
          for (int h = 0; h < (int)sizeof(O) / 2; ++h)
            *(uint4*)(room + (32 * I + i32) * PITCH + ((col * (int)sizeof(O) / 16 + h) ^ (i32 & (PIECES - 1) & 15)) * 16) = piece16[h];
        });
      });
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const int64_t out_row = row0 + wm * (BM / WM) + 32 * I0;
      const int r0 = lane / PIECES, c = lane % PIECES, per = 16 / (int)sizeof(O);
      auto piece_of = [&](int r) { return *(const uint4*)(room + r * PITCH + (c ^ (r & (PIECES - 1) & 15)) * 16); };
      O* out = (O*)g.out + (out_row + r0) * g.out_stride + out_col + c * per;
      if (inside) {
#pragma unroll
        for (int r = 0; r < ROWS; r += AT_ONCE) store_once(out + r * g.out_stride, piece_of(r + r0));
      } else {
#pragma unroll 1
        for (int r = 0; r < ROWS && out_row + r + r0 < g.m; r += AT_ONCE) {
          const uint4 v = piece_of(r + r0);
          O one[16 / sizeof(O)];
          __builtin_memcpy(one, &v, 16);
          if (c * per + per <= left) {
            store_once(out + r * g.out_stride, v);
          } else {
#pragma unroll
            for (int i = 0; i < per; ++i)
              if (c * per + i < left) out[r * g.out_stride + i] = one[i];
          }
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    });
    return inside;
  };

  begin_copies(t);
  each<ALL>([&](auto c) { copy_one(0, decltype(c)::value); });
  constexpr int BEHIND = (STAGES - 1) * COPIES + STORES < 63 ? (STAGES - 1) * COPIES + STORES : 63;   // what was issued behind block 0 at least: a copy of scales may be none
  bool stores_under_way = false;
  for (;;) {
    each<(STAGES - 1) * ALL>([&](auto c) { copy_one(1 + decltype(c)::value / ALL, decltype(c)::value % ALL); });
    if (stores_under_way) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(BEHIND) : "memory");   // they are behind block 0
    else asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((STAGES - 1) * COPIES) : "memory");
    each<READS>([&](auto r) { read_one(0, n0, r); });
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = 0.f;
    for (int s = 0; s < g.steps; ++s) block(s);
    // everybody has read the last fragments, and nothing is on its way to LDS
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
    const int64_t row = row0;
    const int col = col0, height = rows, width = cols;
    t += gridDim.x >> 3;
    const bool more = t < end;
    if (more) {
      begin_copies(t);
      each<ALL>([&](auto c) { copy_one(0, decltype(c)::value); });
    }
    stores_under_way = store_results(row, col, height, width);
    if (!more) break;
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");   // everybody's results have left LDS
  }
}

// per_cu: workgroups that a compute unit holds, by LDS.  A workgroup makes several tiles, so that the first block of the next one is on its
// way while the results of the last one are stored.
template <typename O, int BM, int BN, int STAGES, bool SHORT = false>
int run_tiles(MatmulArgs g, int per_cu, hipStream_t st) {
  g.tiles_m = (int)((g.m + BM - 1) / BM);
  g.tiles_n = (g.n + BN - 1) / BN;
  const int tiles = (g.tiles_m * g.tiles_n + 7) / 8 * 8;
  matmul_mx_kernel<O, BM, BN, STAGES, SHORT><<<std::min(tiles, 256 * per_cu), 256, 0, st>>>(g);
  return status();
}

template <typename O, int R>
int run_rows(const MatmulArgs& g, hipStream_t st) {
  matmul_mx_rows_kernel<O, R><<<(g.n + 15) / 16, 512, 0, st>>>(g);
  return status();
}

template <typename O>
int run_matmul(const MatmulArgs& g, hipStream_t st) {
  const jenga::MatmulTiles t = jenga::matmul_mx_tiles(g.m, g.n, g.halves * 128, sizeof(O) == 4);
  if (t.rows == 16) return run_rows<O, 1>(g, st);
  if (t.rows == 32) return run_rows<O, 2>(g, st);
  if (g.halves < 4) return run_tiles<O, 64, 128, 4, true>(g, 1, st);
  if (t.bm == 256) return run_tiles<O, 256, 256, 2>(g, t.per_cu, st);
  if (t.bm == 64) return run_tiles<O, 64, 128, 4>(g, t.per_cu, st);
  if (t.stages == 4) return run_tiles<O, 128, 128, 4>(g, t.per_cu, st);
  return run_tiles<O, 128, 128, 2>(g, t.per_cu, st);
}

template <typename X>
int run_quantize(const void* x, int64_t x_stride, int64_t rows, int cols, void* q, uint8_t* scale, hipStream_t st) {
  const int quads = (cols + 511) / 512;
  const int64_t units = rows * quads;
  quantize_mx_kernel<X><<<(unsigned)std::min<int64_t>((units + 3) / 4, 1 << 20), 256, 0, st>>>((const X*)x, x_stride, (uint8_t*)q, scale,
                                                                                             units, cols, quads);
  return status();
}

}  // namespace

extern "C" {

int jenga_quantize_mx(const void* x, int64_t x_stride, int32_t x_type, int64_t rows, int32_t cols, void* q, uint8_t* scale, void* stream) {
  const int why = jenga::quantize_mx_args_ok(x, x_stride, x_type, rows, cols, q, scale);
  if (why != JENGA_OK) return why;
  if (rows == 0) return JENGA_OK;
  hipStream_t st = (hipStream_t)stream;
  if (x_type == JENGA_BF16) return run_quantize<__bf16>(x, x_stride, rows, cols, q, scale, st);
  if (x_type == JENGA_F16) return run_quantize<_Float16>(x, x_stride, rows, cols, q, scale, st);
  return run_quantize<float>(x, x_stride, rows, cols, q, scale, st);
}

int jenga_matmul_mx(const jenga_matmul_config* cfg, const void* a, const uint8_t* a_scale, const void* b, const uint8_t* b_scale,
                    const float* bias_or_null, void* out, void* stream) {
  const int why = jenga::matmul_mx_args_ok(cfg, a, a_scale, b, b_scale, bias_or_null, out);
  if (why != JENGA_OK) return why;
  if (cfg->m == 0) return JENGA_OK;
  MatmulArgs g = {};
  g.a = (const uint8_t*)a;
  g.a_scale = a_scale;
  g.b = (const uint8_t*)b;
  g.b_scale = b_scale;
  g.bias = bias_or_null;
  g.out = out;
  g.m = cfg->m;
  g.n = cfg->n;
  g.halves = cfg->k / 128;
  g.steps = (g.halves + 1) / 2;
  g.out_stride = cfg->out_stride;
  hipStream_t st = (hipStream_t)stream;
  if (cfg->out_type == JENGA_BF16) return run_matmul<__bf16>(g, st);
  if (cfg->out_type == JENGA_F16) return run_matmul<_Float16>(g, st);
  return run_matmul<float>(g, st);
}

}  // extern "C"
