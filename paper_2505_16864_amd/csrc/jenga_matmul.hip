// Matrix products of e4m3 operands with a power-of-two scale for each block of 128 values along k, and the quantisation into them.
//
//   out[i][j] = sum over blocks kb of 2^(ea[i][kb] + eb[j / 128][kb]) sum over k in kb of a[i][k] b[j][k]  + bias[j]
//
// The scales are bytes e + 127, what the scaled MFMA of gfx950 takes with its operands: scaling costs no vector instruction.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "jenga_device.h"
#include "jenga_internal.h"
#include "jenga_tiles.h"

namespace {

using namespace jenga;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

int status() { return hipGetLastError() == hipSuccess ? JENGA_OK : JENGA_EHIP; }

// ---- quantisation: bound by memory

// A scale for each row and 128 columns: 16 lanes hold a block, a wavefront four, which is what a group of four scale bytes is for.
// 33272 x 5120 bf16: 89 us, 5.7 TB/s.
template <typename X>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const X* __restrict__ x, int64_t x_stride, uint8_t* __restrict__ q,
                                                            uint8_t* __restrict__ scale, int64_t units, int cols, int quads) {
  const int lane = threadIdx.x & 63, blocks = (cols + 127) >> 7;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); unit < units; unit += (int64_t)gridDim.x * 4) {
    const int64_t row = unit / quads;
    const int col = (int)(unit - row * quads) * 512 + lane * 8, block = col >> 7;
    const f32x8 v = Eight<X>::wide(load_eight(x + row * x_stride + col, cols - col));
    const uint32_t byte = scale_byte(row_max_f32(largest_of(v)));
    if (block < blocks) *(uint2*)(q + row * blocks * 128 + col) = to_e4m3(v, inverse_scale(byte));
    if ((lane & 15) == 0) scale[row * quads * 4 + block] = block < blocks ? (uint8_t)byte : 0;
  }
}

// A scale for each 128 rows and 128 columns: a workgroup each, 16 rows at a time, the values in registers from the maximum to the conversion.  Bound
// by memory: 15360 x 5120 bf16 50 us, 4.7 TB/s; 4608 x 1536 7.0 us, 3.0 TB/s, 432 workgroups on 256 units.
template <typename X>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const X* __restrict__ x, int64_t x_stride, uint8_t* __restrict__ q,
                                                              uint8_t* __restrict__ scale, int64_t rows, int cols, int quads) {
  __shared__ float room[4];
  const int blocks = (cols + 127) >> 7, block = blockIdx.y, col = block * 128 + (threadIdx.x & 15) * 8;
  const int64_t row0 = (int64_t)blockIdx.x * 128 + (threadIdx.x >> 4);
  if (block >= blocks) {   // the bytes that fill up the last group of four
    if (threadIdx.x == 0) scale[(int64_t)blockIdx.x * quads * 4 + block] = 0;
    return;
  }
  f32x8 v[8];
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = row0 + 16 * i;
    v[i] = 0.f;
    if (row < rows) v[i] = Eight<X>::wide(load_eight(x + row * x_stride + col, cols - col));
    m = fmaxf(m, largest_of(v[i]));
  }
  m = row_max_f32(m);
  m = fmaxf(m, __shfl_xor(m, 16));
  m = fmaxf(m, __shfl_xor(m, 32));
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = m;
  __syncthreads();
  const uint32_t byte = scale_byte(fmaxf(fmaxf(room[0], room[1]), fmaxf(room[2], room[3])));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = row0 + 16 * i;
    if (row < rows) *(uint2*)(q + row * blocks * 128 + col) = to_e4m3(v[i], inverse_scale(byte));
  }
  if (threadIdx.x == 0) scale[(int64_t)blockIdx.x * quads * 4 + block] = (uint8_t)byte;
}

// ---- products

struct MatmulArgs {
  const uint8_t *a, *a_scale, *b, *b_scale;
  const float* bias;
  void* out;
  int64_t m, out_stride;
  int n, steps, quads;   // steps: blocks of 128 along k
  int tiles_m, tiles_n;
};

// 32 rows of an operand and 64 columns (half a block), a row in lanes l and l + 32, with the scale byte of each row.  The product of
// two is 32 x 32 results.  Which half of a block's columns lie in which lane, and in which order, does not matter as long as it is the same
// for both operands.
//
// EXACT: the eight products that the f8 matrix core adds at a time are cut off at 2^-13 of the largest of them (1.5e-5 of the result's norm
// for normal values, 6e-5 for long tails), far below the rounding of a 16-bit result and of e4m3 itself, but not below that of a
// float32 result: there the operands go to bf16, which holds e4m3 times 2^e exactly (from 2^-126 on), and through the bf16 matrix core,
// whose sums are float32.
template <bool EXACT>
struct Fragment;
template <>
struct Fragment<false> {
  i32x8 v;
};
__device__ __forceinline__ f32x16 multiply(const Fragment<false>& x, int xs, const Fragment<false>& y, int ys, f32x16 acc) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x.v, y.v, acc, 0, 0, 0, xs, 0, ys);
#else
  return acc;
#endif
}
template <>
struct Fragment<true> {
  i32x8 v;
  // columns 8 i to 8 i + 7 of the lane's 32
  __device__ __forceinline__ bf16x8 wide(int i, int s) const {
    bf16x8 r = {};
#if defined(__HIP_DEVICE_COMPILE__)
    const float f = __builtin_bit_cast(float, s == 0 ? 0x400000u : (uint32_t)s << 23);   // 2^-127 is a subnormal number
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * i], f, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * i], f, true);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * i + 1], f, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * i + 1], f, true);
    r = (bf16x8){p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
#endif
    return r;
  }
};
__device__ __forceinline__ f32x16 multiply(const Fragment<true>& x, int xs, const Fragment<true>& y, int ys, f32x16 acc) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
  for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.wide(i, xs & 255), y.wide(i, ys & 255), acc, 0, 0, 0);
#endif
  return acc;
}

// The same for 16 rows and a whole block, a row in lanes l, l + 16, l + 32 and l + 48.
__device__ __forceinline__ f32x4 multiply16(const Fragment<false>& x, int xs, const Fragment<false>& y, int ys, f32x4 acc) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x.v, y.v, acc, 0, 0, 0, xs, 0, ys);
#else
  return acc;
#endif
}
__device__ __forceinline__ f32x4 multiply16(const Fragment<true>& x, int xs, const Fragment<true>& y, int ys, f32x4 acc) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
  for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.wide(i, xs & 255), y.wide(i, ys & 255), acc, 0, 0, 0);
#endif
  return acc;
}

__device__ __forceinline__ i32x8 bytes32(const uint8_t* p) {
  const uint4 v[2] = {*(const uint4*)p, *(const uint4*)(p + 16)};
  i32x8 r;
  __builtin_memcpy(&r, v, 32);
  return r;
}

// Up to 16 R rows of a: the weight is read once and is what takes the time, so there are no tiles.  A workgroup makes 16 columns; its eight
// wavefronts take a block of k each in turn, straight from memory into registers, four turns ahead, and add their sums up in LDS.
// 1 x 15360 x 5120: 14.3 us, 5.5 TB/s.
template <typename O, bool EXACT, int R>
__global__ __launch_bounds__(512) void matmul_rows_kernel(MatmulArgs g) {
  constexpr int WAVES = 8, AHEAD = 4;
  __shared__ float sums[WAVES][R * 256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, piece = (lane >> 4) * 32;
  const int col0 = blockIdx.x * 16;
  const size_t pitch = (size_t)g.steps * 128;
  // rows and columns past the end: the last one again, and not stored
  const uint8_t *a[R], *a_scale[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t row = min((int64_t)(16 * r + i16), g.m - 1);
    a[r] = g.a + row * pitch + piece;
    a_scale[r] = g.a_scale + row * g.quads * 4;
  }
  const uint8_t *b = g.b + (size_t)min(col0 + i16, g.n - 1) * pitch + piece, *b_scale = g.b_scale + (size_t)(col0 >> 7) * g.quads * 4;
  f32x4 acc[R] = {};
  for (int s0 = wave; s0 < g.steps; s0 += AHEAD * WAVES) {
    Fragment<EXACT> fb[AHEAD], fa[AHEAD][R];
    int sb[AHEAD], sa[AHEAD][R];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int s = s0 + u * WAVES;
      if (s < g.steps) {
        fb[u].v = bytes32(b + (size_t)s * 128);
        sb[u] = b_scale[s];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          fa[u][r].v = bytes32(a[r] + (size_t)s * 128);
          sa[u][r] = a_scale[r][s];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s0 + u * WAVES < g.steps)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r] = multiply16(fb[u], sb[u], fa[u][r], sa[u][r], acc[r]);
  }
#pragma unroll
  for (int r = 0; r < R; ++r)   // lane l holds row l % 16 of a, columns 4 (l / 16) to + 3
    *(f32x4*)&sums[wave][(16 * r + i16) * 16 + (lane >> 4) * 4] = acc[r];
  __syncthreads();
  for (int i = threadIdx.x; i < R * 256; i += 512) {
    const int row = i >> 4, col = col0 + (i & 15);
    if (row >= g.m || col >= g.n) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += sums[w][i];
    ((O*)g.out)[row * g.out_stride + col] = (O)(g.bias ? v + g.bias[col] : v);
  }
}

// Four wavefronts, 2 x 2, make BM x BN results, one tile after the other.  Blocks of 128 columns (bytes) of either operand are copied
// into one of STAGES LDS tiles while another is multiplied; within a block the products of one half of the columns run while the
// fragments of the next half are read into registers.  So the reads of an LDS tile end in the middle of its block, and that is where
// the barrier is: behind it the next tile is complete, and the one STAGES blocks on goes over this one.
//
// 33272 x 15360 x 5120 to bf16: 1.95 to 2.0 ms, 2.65 to 2.69 PFLOP/s, where the library's product with one scale for each operand takes
// 1.84 to 1.97; the matrix cores are busy 70 % of the cycles at the 1.67 GHz that the package power leaves (all-zero operands: 1.77 ms), no
// bank conflicts.  Float32 results, through the bf16 matrix core: 1.15 PFLOP/s.  16 x 16 x 128 products, eight wavefronts, results in
// LDS room of their own and wider or narrower stripes were slower or the same.
//
// A copy instruction takes 8 whole rows of 128 bytes: first their left halves, then the right ones.  The 16-byte pieces of a half row are
// rotated by an exclusive or with bits of the row, so that the rows of a fragment fall on all banks.  The rows of b are the rows of
// the matrix instruction, taken in an order that puts eight neighbouring results of a row of out into a lane: two fragments j,
// j + 1 hold columns 16 q + 8 (lane / 32) + 4 (j & 1) + 0..3 of 64.
template <typename O, bool EXACT, int BM, int BN, int STAGES>
__global__ __launch_bounds__(256) void matmul_kernel(MatmulArgs g) {
  constexpr int WM = 2, WN = 2, MT = BM / WM / 32, NT = BN / WN / 32, COPIES = (BM + BN) / 32, STAGE = (BM + BN) * 128;
  static_assert(STAGES >= 2 && STAGES <= 4 && BM % 64 == 0 && BN % 64 == 0 && BN / WN <= 128 && 128 % (BN / WN) == 0 && NT % 2 == 0, "");
  // the results of 32 rows of each wavefront go where the tiles but the first are
  constexpr int PITCH = BN / WN * sizeof(O), REST = (STAGES - 1) * STAGE, SECOND = REST > 4 * 32 * PITCH ? REST : 4 * 32 * PITCH;
  constexpr int SCALES = STAGE + SECOND;   // two times four blocks' scales of a
  __shared__ __attribute__((aligned(128))) uint8_t tiles[SCALES + 2 * BM * 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % WM, wn = wave / WM;
  const uint32_t pitch = (uint32_t)g.steps * 128,
                 lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)tiles;
  const int n_tiles = g.tiles_m * g.tiles_n, xcd = blockIdx.x & 7;
  const int end = (int)((int64_t)n_tiles * (xcd + 1) >> 3);
  int t = (int)((int64_t)n_tiles * xcd >> 3) + (blockIdx.x >> 3);
  if (t >= end) return;

  // of this lane, for the copies of its wavefront: 8 rows each, 32 rows apart, so that the rotations are the same for all
  const uint32_t from = (uint32_t)(wave * 8 + (lane >> 2 & 7)) * pitch + (lane >> 5) * 64;
  const uint32_t from_a = from + ((lane & 3) ^ ((2 * wave + (lane >> 4 & 1)) & 3)) * 16, from_b = from + ((lane & 3) ^ wave) * 16;
  const int i32 = lane & 31, turn = (i32 >> 2 & 3) * 16, piece = (lane >> 5) * 32;
  const int ra = wm * (BM / WM) + i32;                                     // + 32 i
  const int rb = wn * (BN / WN) + 2 * (i32 & ~3) + (i32 & 3);              // + 64 (j / 2) + 4 (j & 1)
  const int at_a = (ra >> 3) * 1024 + (ra & 7) * 64, at_b = BM * 128 + (rb >> 3) * 1024 + (rb & 7) * 64;   // rb & 4 is 0

  // the tile whose operands are copied: that of the products, and behind its last block the next one
  u32x4 a_rows, b_rows;
  const uint8_t* s0;
  uint32_t scale_from;
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
    s0 = g.a_scale + row0 * g.quads * 4;
    scale_from = (uint32_t)min(wave % (BM / 64) * 64 + lane, rows - 1) * (uint32_t)(g.quads * 4);   // past the end: the last row's again
  };
  auto copy_one = [&](int s, int c) {
    const bool of_a = c * 32 < BM;
    copy_1kb(of_a ? a_rows : b_rows, of_a ? from_a : from_b,
             s < g.steps ? (of_a ? c : c - BM / 32) * 32 * pitch + s * 128 : 0x80000000u,   // past the end: outside
             lds0 + (uint32_t)s % STAGES * STAGE + (c * 4 + wave) * 1024);
  };
  auto copy_scales = [&](int s) {
    const int k = min(s, g.steps - 1);
    copy_256b(s % 4 == 0 && wave < BM / 64, s0 + (k & ~3), scale_from,
              lds0 + SCALES + (k >> 2 & 1) * BM * 4 + wave % (BM / 64) * 256);
  };

  f32x16 acc[MT][NT];
  Fragment<EXACT> fa[2][MT], fb[2][NT];
  int scale_a[MT], scale_b = 0;
  const __attribute__((address_space(4))) uint32_t* sb;   // read with scalar loads
  // Fragment r of half h of block s: those of b and a in the order in which the products want them.
  auto read_one = [&](int s, auto half, auto index) {
    constexpr int H = decltype(half)::value, R = decltype(index)::value;
    constexpr bool OF_A = R >= 1 && R <= MT;
    constexpr int I = OF_A ? R - 1 : 0, J = R == 0 || OF_A ? 0 : R - MT;
    const uint8_t* p = tiles + (uint32_t)s % STAGES * STAGE + H * 512 + (OF_A ? at_a + I * 4096 : at_b + (J >> 1) * 8192 + (J & 1) * 256);
    const uint4 v[2] = {*(const uint4*)(p + (piece ^ turn)), *(const uint4*)(p + ((piece + 16) ^ turn))};
    __builtin_memcpy(OF_A ? &fa[H][I].v : &fb[H][J].v, v, 32);
  };
  auto read_scales = [&](int s) {
    const int k = min(s, g.steps - 1);
    const uint8_t* sa = tiles + SCALES + ((k >> 2 & 1) * BM + ra) * 4 + (k & 3);
#pragma unroll
    for (int i = 0; i < MT; ++i) scale_a[i] = sa[128 * i];
    scale_b = sb[k >> 2] >> (k & 3) * 8;
  };
  using std::integral_constant;
  constexpr integral_constant<int, 0> n0;
  constexpr integral_constant<int, 1> n1;
  constexpr int PRODUCTS = MT * NT, READS = MT + NT;
  // Multiplies block s.  Between the products are the reads of the next half and the copies of the block STAGES on.  (Left alone,
  // the compiler reads after the products and waits; all reads and copies before them leave the matrix core without work meanwhile:
  // 8192 x 8192 x 8192 585 -> 445 us.)  What is read and copied behind the last block is not used and not fetched: other code there
  // would cost more, in moves between registers.
  auto block = [&](int s) {
    int now_a[MT], now_b = scale_b;
#pragma unroll
    for (int i = 0; i < MT; ++i) now_a[i] = scale_a[i];
    each<PRODUCTS>([&](auto index) {
      constexpr int N = decltype(index)::value;
      acc[N % MT][N / MT] = multiply(fb[0][N / MT], now_b, fa[0][N % MT], now_a[N % MT], acc[N % MT][N / MT]);
      each<READS>([&](auto r) {
        if constexpr (decltype(r)::value * (PRODUCTS - 1) / READS == N) read_one(s, n1, r);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    // this wavefront's copies of the next block are done (those of later blocks may be on their way), and its reads of this one;
    // then everybody's are
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((STAGES - 2) * COPIES) : "memory");
    read_scales(s + 1);
    __builtin_amdgcn_sched_barrier(0);
    each<PRODUCTS>([&](auto index) {
      constexpr int N = decltype(index)::value;
      acc[N % MT][N / MT] = multiply(fb[1][N / MT], now_b, fa[1][N % MT], now_a[N % MT], acc[N % MT][N / MT]);
      each<READS>([&](auto r) {
        if constexpr (decltype(r)::value * (PRODUCTS - 1) / READS == N) read_one(s + 1, n0, r);
      });
      each<COPIES>([&](auto c) {
        if constexpr (decltype(c)::value * PRODUCTS / COPIES == N) copy_one(s + STAGES, decltype(c)::value);
      });
      if constexpr (N == PRODUCTS - 1) copy_scales(s + STAGES);
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  // The results go through LDS, so that a store takes whole rows of the wavefront's columns.  Room for each wavefront in the second LDS
  // tile, for ROWS of its rows at a time.  They are not kept in the caches: the operands that they would drive out cost more (33272 x
  // 15360 x 5120: 2.40 -> 2.17 ms).
  constexpr int COLS = BN / WN, PIECES = PITCH / 16, FIT = SECOND / 4 / PITCH / 32 * 32,
                ROWS = FIT < MT * 32 ? FIT : MT * 32, AT_ONCE = 64 / PIECES;   // rows that a store takes
  constexpr int STORES = MT * 32 / AT_ONCE;
  static_assert(ROWS >= 32 && MT * 32 % ROWS == 0 && PIECES <= 64 && (STAGES - 1) * COPIES + STORES <= 63, "");
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
  each<COPIES>([&](auto c) { copy_one(0, decltype(c)::value); });
  copy_scales(0);
  bool stores_under_way = false;
  for (;;) {
    each<(STAGES - 1) * COPIES>([&](auto c) { copy_one(1 + decltype(c)::value / COPIES, decltype(c)::value % COPIES); });
    if (stores_under_way) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((STAGES - 1) * COPIES + STORES) : "memory");   // they are behind block 0
    else asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((STAGES - 1) * COPIES) : "memory");
    sb = (const __attribute__((address_space(4))) uint32_t*)uniform(g.b_scale + (size_t)((col0 + min(wn * (BN / WN), cols - 1)) >> 7) * g.quads * 4);
    each<READS>([&](auto r) { read_one(0, n0, r); });
    read_scales(0);
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
      each<COPIES>([&](auto c) { copy_one(0, decltype(c)::value); });
      copy_scales(0);
    }
    stores_under_way = store_results(row, col, height, width);
    if (!more) break;
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");   // everybody's results have left LDS
  }
}

// per_cu: workgroups that a compute unit holds, by LDS.  A workgroup makes several tiles, so that the first block of the next one is on its
// way while the results of the last one are stored.
template <typename O, bool EXACT, int BM, int BN, int STAGES>
int run_tiles(MatmulArgs g, int per_cu, hipStream_t st) {
  g.tiles_m = (int)((g.m + BM - 1) / BM);
  g.tiles_n = (g.n + BN - 1) / BN;
  const int tiles = (g.tiles_m * g.tiles_n + 7) / 8 * 8;
  matmul_kernel<O, EXACT, BM, BN, STAGES><<<std::min(tiles, 256 * per_cu), 256, 0, st>>>(g);
  return status();
}

template <typename O, bool EXACT, int R>
int run_rows(const MatmulArgs& g, hipStream_t st) {
  matmul_rows_kernel<O, EXACT, R><<<(g.n + 15) / 16, 512, 0, st>>>(g);
  return status();
}

template <typename O, bool EXACT>
int run_matmul(const MatmulArgs& g, hipStream_t st) {
  const jenga::MatmulTiles t = jenga::matmul_tiles(g.m, g.n, EXACT);
  if (t.rows == 16) return run_rows<O, EXACT, 1>(g, st);
  if (t.rows == 32) return run_rows<O, EXACT, 2>(g, st);
  if constexpr (!EXACT)
    if (t.bm == 256) return run_tiles<O, EXACT, 256, 256, 2>(g, t.per_cu, st);
  if (t.bm == 64) return run_tiles<O, EXACT, 64, 128, 4>(g, t.per_cu, st);
  if (t.stages == 4) return run_tiles<O, EXACT, 128, 128, 4>(g, t.per_cu, st);
  return run_tiles<O, EXACT, 128, 128, 2>(g, t.per_cu, st);
}

template <typename X>
int run_quantize(const void* x, int64_t x_stride, int64_t rows, int cols, int block_rows, void* q, uint8_t* scale, hipStream_t st) {
  const int quads = (cols + 511) / 512;
  if (block_rows == 1) {
    const int64_t units = rows * quads;
    quantize_rows_kernel<X><<<(unsigned)std::min<int64_t>((units + 3) / 4, 1 << 20), 256, 0, st>>>((const X*)x, x_stride, (uint8_t*)q,
                                                                                                scale, units, cols, quads);
  } else {
    quantize_blocks_kernel<X><<<dim3((unsigned)((rows + 127) / 128), quads * 4), 256, 0, st>>>((const X*)x, x_stride, (uint8_t*)q, scale,
                                                                                              rows, cols, quads);
  }
  return status();
}

}  // namespace

extern "C" {

int jenga_quantize(const void* x, int64_t x_stride, int32_t x_type, int64_t rows, int32_t cols, int32_t block_rows, void* q,
                   uint8_t* scale, void* stream) {
  const int why = jenga::quantize_args_ok(x, x_stride, x_type, rows, cols, block_rows, q, scale);
  if (why != JENGA_OK) return why;
  if (rows == 0) return JENGA_OK;
  hipStream_t st = (hipStream_t)stream;
  if (x_type == JENGA_BF16) return run_quantize<__bf16>(x, x_stride, rows, cols, block_rows, q, scale, st);
  if (x_type == JENGA_F16) return run_quantize<_Float16>(x, x_stride, rows, cols, block_rows, q, scale, st);
  return run_quantize<float>(x, x_stride, rows, cols, block_rows, q, scale, st);
}

int jenga_matmul(const jenga_matmul_config* cfg, const void* a, const uint8_t* a_scale, const void* b, const uint8_t* b_scale,
                 const float* bias_or_null, void* out, void* stream) {
  const int why = jenga::matmul_args_ok(cfg, a, a_scale, b, b_scale, bias_or_null, out);
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
  g.steps = cfg->k / 128;
  g.quads = (cfg->k + 511) / 512;
  g.out_stride = cfg->out_stride;
  hipStream_t st = (hipStream_t)stream;
  if (cfg->out_type == JENGA_BF16) return run_matmul<__bf16, false>(g, st);
  if (cfg->out_type == JENGA_F16) return run_matmul<_Float16, false>(g, st);
  return run_matmul<float, true>(g, st);
}

}  // extern "C"
