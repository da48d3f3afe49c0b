// Layer norm over the columns of each row, with a weight and a bias per group of rows, and its gradient.
//
//   mu = sum x / C    var = sum (x - mu)^2 / C    r = 1 / sqrt(var + eps)    h = (x - mu) r    y = h (w0 + w) + b
//   g = dy (w0 + w)   dx = r (g - mean(g) - h mean(g h))   dw = sum over the group's rows of dy h   db = sum of dy
//
// Bound by memory: a row is read once into registers, as it lies in memory, and summed twice from there (the second sum is of
// (x - mu)^2, so that a large mean costs no digits).  All sums are float32.  33272 x 5120 bf16: 144 us, 4.73 TB/s (a copy: 4.88); to
// e4m3 179 us, 2.86 TB/s, by its vector instructions: 30 a value against 20, which keep the ALUs busy 77 % of the cycles; gradient of 63424 x 1536
// in two groups 129 us, 4.5 TB/s, and 5 us for the sums.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "jenga_device.h"
#include "jenga_internal.h"

namespace {

using namespace jenga;

struct NormArgs {
  const void *x, *dy, *weight, *bias;
  void *y, *dx;
  uint8_t* y_scale;
  float *mean, *rstd;
  float* parts;
  int64_t rows, group_rows, x_stride, y_stride, param_stride;
  int32_t cols, scale_cols, row_parts;
  float eps, w0;
};

// The row's weight and bias: eight of each.
template <typename P>
__device__ __forceinline__ void params(const NormArgs& a, int64_t group, int col, f32x8* w, f32x8* b) {
  const int64_t at = group * a.param_stride + col;
  *w = a.w0;
  *b = 0.f;
  if (a.weight) *w += Eight<P>::wide(load_eight((const P*)a.weight + at, a.cols - col));
  if (a.bias) *b = Eight<P>::wide(load_eight((const P*)a.bias + at, a.cols - col));
}

// Eight results of a row from column `col` on, at most n of them in the row; 16 lanes hold a block of 128 columns.
template <typename X, bool E4M3>
__device__ __forceinline__ void put(const NormArgs& a, int64_t row, int col, const f32x8& y) {
  const int n = a.cols - col;
  if (!E4M3) {
    if (n > 0) store_eight((X*)a.y + row * a.y_stride + col, y, n);
    return;
  }
  f32x8 v = y;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i >= n) v[i] = 0.f;   // the columns that fill up the last block
  const uint32_t byte = scale_byte(row_max_f32(largest_of(v)));
  const int block = col >> 7, blocks = (a.cols + 127) >> 7;
  if (block < blocks) *(uint2*)((uint8_t*)a.y + row * a.y_stride + col) = to_e4m3(v, inverse_scale(byte));
  if ((threadIdx.x & 15) == 0 && block < a.scale_cols) a.y_scale[row * a.scale_cols + block] = block < blocks ? (uint8_t)byte : 0;
}

// Rows in registers are taken in pieces of eight columns.  Where their number is no multiple of eight, the last piece ends with the row
// and overlaps the one before it: both compute and store the same results there, and the sums take only what is `own`.  (Columns one
// by one at the end of a row cost a branch each in every piece: 33272 x 5120 bf16 177 us.)  E4M3 results have their places in
// blocks, so there it has to be a multiple of eight.
struct Piece {
  int col;     // of the first value; 8 of them
  int skip;    // so many are the piece's before
  bool here;
};
__device__ __forceinline__ Piece piece_at(int col, int cols) {
  const int c = min(col, cols - 8);
  return {c, col - c, col < cols};
}
template <typename T>
__device__ __forceinline__ typename Eight<T>::raw take(const T* p, bool here) {
  typename Eight<T>::raw r = {};
  if (here) r = *(const typename Eight<T>::raw*)p;
  return r;
}

// Sum over the WPR wavefronts of a row; all of them get it.  `room` is not written again before everybody has read it.
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float* room) {
  v = wave_sum_f32(v);
  if (WPR == 1) return v;
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) room[wave] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < WPR; ++i) s += room[wave / WPR * WPR + i];
  return s;
}

// Workgroups of norm_kernel on a compute unit, by the registers that it needs.  The grid is as many and no more: with 8 a CU
// where 5 have room, the last ones run on a chip that is half empty.  (16-bit rows to e4m3, 4 -> 5 a unit, us: 20000 x 4096 71.7 -> 66.4;
// 20000 x 6144, where 12 registers go to scratch for it, 107 -> 127.)
template <typename X, typename P, bool E4M3, int NV>
constexpr int norm_per_cu() {
  constexpr bool HALF = sizeof(X) + sizeof(P) == 4;   // both of 16 bits
  return NV == 1 ? (HALF ? 8 : 6) : NV == 2 ? (HALF ? 5 : 4) : NV == 3 ? (HALF ? (E4M3 ? 4 : 5) : 3) : HALF ? 3 : 2;
}

// WPR wavefronts to a row, up to NV pieces of WPR * 512 columns, cols >= 8.  A workgroup takes rows a grid apart; it keeps the weight and the
// bias in registers, and the next row is on its way while one is worked on.  (A wavefront alone with 80 columns a lane: 33272 x
// 5120 bf16 177 us.)
template <typename X, typename P, bool E4M3, int NV, int WPR>
__global__ __launch_bounds__(256, (norm_per_cu<X, P, E4M3, NV>())) void norm_kernel(NormArgs a) {
  constexpr int STEP = WPR * 512, AT_ONCE = 4 / WPR;
  __shared__ float room[2][2][4];
  const int slot = (threadIdx.x >> 6) / WPR, col0 = (threadIdx.x % (WPR * 64)) * 8;
  typename Eight<P>::raw weight[NV], bias[NV];
  int64_t have = -1;   // whose group's they are
  typename Eight<X>::raw next[NV];
  auto fetch = [&](int64_t row) {   // zeros for a row that is not there
    const X* x = (const X*)a.x + row * a.x_stride;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        const Piece p = piece_at(v * STEP + col0, a.cols);
        next[v] = take(x + p.col, p.here && row < a.rows);
      }
  };
  const int64_t step = (int64_t)gridDim.x * AT_ONCE;
  fetch((int64_t)blockIdx.x * AT_ONCE + slot);
  int turn = 0;
  // every wavefront takes every turn (there are barriers in it); one without a row has zeros and nothing to store
  for (int64_t row0 = (int64_t)blockIdx.x * AT_ONCE; row0 < a.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool mine = row < a.rows;
    const int64_t group = a.rows > a.group_rows && mine ? row / a.group_rows : 0;
    if (group != have) {
      have = group;
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (v * STEP < a.cols) {
          const Piece p = piece_at(v * STEP + col0, a.cols);
          weight[v] = take((const P*)a.weight + group * a.param_stride + p.col, p.here && a.weight);
          bias[v] = take((const P*)a.bias + group * a.param_stride + p.col, p.here && a.bias);
        }
    }
    f32x8 f[NV];   // x, then x - mean
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        f[v] = Eight<X>::wide(next[v]);
        if (v * STEP + STEP <= a.cols) {
          sum += ((f[v][0] + f[v][1]) + (f[v][2] + f[v][3])) + ((f[v][4] + f[v][5]) + (f[v][6] + f[v][7]));
        } else {
          const Piece p = piece_at(v * STEP + col0, a.cols);
#pragma unroll
          for (int i = 0; i < 8; ++i) sum += i >= p.skip ? f[v][i] : 0.f;   // zeros where there is no piece
        }
      }
    fetch(row + step);
    const float mean = row_sum<WPR>(sum, room[turn][0]) / (float)a.cols;
    float square = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        f[v] -= mean;
        if (v * STEP + STEP <= a.cols) {
#pragma unroll
          for (int i = 0; i < 8; ++i) square = fmaf(f[v][i], f[v][i], square);
        } else {
          const Piece p = piece_at(v * STEP + col0, a.cols);
#pragma unroll
          for (int i = 0; i < 8; ++i) square = fmaf(f[v][i], p.here && i >= p.skip ? f[v][i] : 0.f, square);
        }
      }
    const float rstd = 1.0f / sqrtf(row_sum<WPR>(square, room[turn][1]) / (float)a.cols + a.eps);
    if (mine && threadIdx.x % (WPR * 64) == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    if (mine) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (v * STEP < a.cols) {
          const Piece p = piece_at(v * STEP + col0, a.cols);
          const f32x8 w = Eight<P>::wide(weight[v]) + a.w0, b = Eight<P>::wide(bias[v]);
          f32x8 y;
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = fmaf(f[v][i] * rstd, w[i], b[i]);
          if (E4M3) put<X, true>(a, row, v * STEP + col0, y);
          else if (p.here) *(typename Eight<X>::raw*)((X*)a.y + row * a.y_stride + p.col) = Eight<X>::narrow(y);
        }
    }
  }
}

// Sum over the threads of a workgroup, up to 1024; all of them get it.
__device__ __forceinline__ float block_sum(float v, float* room) {
  v = wave_sum_f32(v);
  __syncthreads();   // the room is free
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
  for (int i = 0; i < (int)blockDim.x / 64; ++i) s += room[i];
  return s;
}

// Rows too long for registers, and those that norm_kernel's pieces do not fit: a workgroup each, read again for each of the three
// passes.  3000 x 10001 bf16: 57 to 67 us, 2.1 to 1.8 TB/s: three passes through the L2, rows off the 16-byte grid.
template <typename X, typename P, bool E4M3>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  __shared__ float room[16];
  const int step = blockDim.x * 8, whole = (a.cols + step - 1) / step * step;   // every thread takes every turn: a block's scale is 16 lanes' work
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const X* x = (const X*)a.x + row * a.x_stride;
    float sum = 0.f, square = 0.f;
    for (int col = threadIdx.x * 8; col < a.cols; col += step) {
      const f32x8 f = Eight<X>::wide(load_eight(x + col, a.cols - col));
      sum += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
    }
    const float mean = block_sum(sum, room) / (float)a.cols;
    for (int col = threadIdx.x * 8; col < a.cols; col += step) {
      const f32x8 f = Eight<X>::wide(load_eight(x + col, a.cols - col));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = f[i] - mean;
        if (col + i < a.cols) square = fmaf(d, d, square);
      }
    }
    const float rstd = 1.0f / sqrtf(block_sum(square, room) / (float)a.cols + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    const int64_t group = row / a.group_rows;
    for (int col = threadIdx.x * 8; col < whole; col += step) {
      f32x8 w = 0.f, b = 0.f, y = 0.f;
      if (col < a.cols) {
        const f32x8 f = Eight<X>::wide(load_eight(x + col, a.cols - col));
        params<P>(a, group, col, &w, &b);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fmaf((f[i] - mean) * rstd, w[i], b[i]);
      }
      put<X, E4M3>(a, row, col, y);
    }
  }
}

// ---- gradient

// The rows of part `part` of group `group`.
__device__ __forceinline__ void part_rows(const NormArgs& a, int64_t group, int part, int64_t* first, int64_t* end) {
  const int64_t start = group * a.group_rows, n = min(a.group_rows, a.rows - start);
  *first = start + n * part / a.row_parts;
  *end = start + n * (part + 1) / a.row_parts;
}

// Wavefronts of norm_grad_kernel on a SIMD, by the registers that it needs.
template <int NV>
constexpr int grad_per_cu() {
  return NV == 1 ? 4 : NV == 2 ? 3 : 2;
}

// A workgroup takes a part of a group's rows, WPR wavefronts to a row, up to NV pieces of WPR * 512 columns, and keeps the weight and
// the sums of its columns in registers; the sums go to parts[workgroup][2][cols].  The next row is on its way while one is worked on.
constexpr int grad_waves(int wpr) { return wpr > 4 ? wpr : 4; }
template <typename X, typename P, int NV, int WPR>
__global__ __launch_bounds__(64 * grad_waves(WPR), (grad_per_cu<NV>())) void norm_grad_kernel(NormArgs a) {
  constexpr int STEP = WPR * 512, WAVES = grad_waves(WPR), AT_ONCE = WAVES / WPR;
  __shared__ float room[2][WAVES][2];
  extern __shared__ float sums[];   // [2][cols], for the rows of AT_ONCE wavefronts
  const int64_t group = blockIdx.x / a.row_parts;
  const int part = blockIdx.x - (int)(group * a.row_parts);
  const int wave = threadIdx.x >> 6, slot = wave / WPR;
  const int col0 = (threadIdx.x % (WPR * 64)) * 8;
  int64_t first, end;
  part_rows(a, group, part, &first, &end);
  f32x8 dw[NV], db[NV];
  typename Eight<P>::raw weight[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    dw[v] = db[v] = 0.f;
    const Piece p = piece_at(v * STEP + col0, a.cols);
    if (a.weight) weight[v] = take((const P*)a.weight + group * a.param_stride + p.col, p.here);
  }
  typename Eight<X>::raw next_x[NV], next_d[NV];
  float next_mean = 0.f, next_rstd = 0.f;
  auto fetch = [&](int64_t row) {   // zeros for a row that is not there
    const X *x = (const X*)a.x + row * a.x_stride, *dy = (const X*)a.dy + row * a.y_stride;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        const Piece p = piece_at(v * STEP + col0, a.cols);
        next_x[v] = take(x + p.col, p.here && row < end);
        next_d[v] = take(dy + p.col, p.here && row < end);
      }
    next_mean = next_rstd = 0.f;
    if (row < end) next_mean = a.mean[row], next_rstd = a.rstd[row];
  };
  fetch(first + slot);
  int turn = 0;
  // every wavefront takes every turn (there are barriers in it); one without a row has zeros and nothing to store
  for (int64_t row0 = first; row0 < end; row0 += AT_ONCE, turn ^= 1) {
    const int64_t row = row0 + slot;
    const float mean = next_mean, rstd = next_rstd;
    f32x8 h[NV], g[NV];
    float sum_g = 0.f, sum_gh = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        const f32x8 x = Eight<X>::wide(next_x[v]), d = Eight<X>::wide(next_d[v]);
        f32x8 w = a.w0;
        if (a.weight) w += Eight<P>::wide(weight[v]);
        int skip = 0;
        float r = rstd;
        if (v * STEP + STEP > a.cols) {
          const Piece p = piece_at(v * STEP + col0, a.cols);
          skip = p.skip;
          if (!p.here) r = 0.f;   // h is 0 where there is no piece: -mean * rstd may be infinite, and 0 times that is NaN
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[v][i] = (x[i] - mean) * r;
          g[v][i] = d[i] * w[i];   // 0 where there is no piece
          dw[v][i] = fmaf(d[i], h[v][i], dw[v][i]);
          db[v][i] += d[i];
          const float own = i >= skip ? g[v][i] : 0.f;
          sum_g += own;
          sum_gh = fmaf(own, h[v][i], sum_gh);
        }
      }
    fetch(row + AT_ONCE);
    sum_g = wave_sum_f32(sum_g);
    sum_gh = wave_sum_f32(sum_gh);
    if (WPR > 1) {
      if ((threadIdx.x & 63) == 0) room[turn][wave][0] = sum_g, room[turn][wave][1] = sum_gh;
      __syncthreads();   // the other turn's room was read before the barrier of this one
      sum_g = sum_gh = 0.f;
#pragma unroll
      for (int i = 0; i < WPR; ++i) sum_g += room[turn][slot * WPR + i][0], sum_gh += room[turn][slot * WPR + i][1];
    }
    const float mg = sum_g / (float)a.cols, mgh = sum_gh / (float)a.cols;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        const Piece p = piece_at(v * STEP + col0, a.cols);
        f32x8 d;
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = rstd * (g[v][i] - mg - h[v][i] * mgh);
        if (p.here && row < end) *(typename Eight<X>::raw*)((X*)a.dx + row * a.x_stride + p.col) = Eight<X>::narrow(d);
      }
  }
  if (!a.parts) return;
  float* to = a.parts + (int64_t)blockIdx.x * 2 * a.cols;
  for (int s = 0; s < AT_ONCE; ++s) {   // the slots add theirs one after the other, in this order
    if (slot == s) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const Piece p = piece_at(v * STEP + col0, a.cols);
          const int col = p.col + i;
          if (p.here && i >= p.skip) {
            float w = dw[v][i], b = db[v][i];
            if (s > 0) w += sums[col], b += sums[a.cols + col];
            if (s == AT_ONCE - 1) to[col] = w, to[a.cols + col] = b;
            else sums[col] = w, sums[a.cols + col] = b;
          }
        }
    }
    if (AT_ONCE > 1) __syncthreads();
  }
}

// Rows too long for that, or of less than eight columns: dx by a workgroup per row, the sums of the columns by a thread per column.
// 3000 x 10001 bf16: 67 us for dx, 2.7 TB/s, 40 for the sums: x and dy are read once for each of the three passes.
template <typename X, typename P>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormArgs a) {
  __shared__ float room[16];
  const int step = blockDim.x * 8;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const X *x = (const X*)a.x + row * a.x_stride, *dy = (const X*)a.dy + row * a.y_stride;
    const P* weight = (const P*)a.weight + row / a.group_rows * a.param_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float sum_g = 0.f, sum_gh = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      for (int col = threadIdx.x * 8; col < a.cols; col += step) {
        const int n = a.cols - col;
        f32x8 w = a.w0, d;
        if (a.weight) w += Eight<P>::wide(load_eight(weight + col, n));
        const f32x8 f = Eight<X>::wide(load_eight(x + col, n)), g = Eight<X>::wide(load_eight(dy + col, n)) * w;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float h = (f[i] - mean) * rstd;
          if (pass == 0) sum_g += g[i], sum_gh = fmaf(g[i], i < n ? h : 0.f, sum_gh);   // g is 0 past the end, -mean * rstd may be infinite
          else d[i] = rstd * (g[i] - sum_g - h * sum_gh);
        }
        if (pass == 1) store_eight((X*)a.dx + row * a.x_stride + col, d, n);
      }
      if (pass == 0) {
        sum_g = block_sum(sum_g, room) / (float)a.cols;
        sum_gh = block_sum(sum_gh, room) / (float)a.cols;
      }
    }
  }
}
template <typename X>
__global__ __launch_bounds__(256) void norm_grad_columns_kernel(NormArgs a) {
  const int col = blockIdx.y * 256 + threadIdx.x;
  if (col >= a.cols) return;
  const int64_t group = blockIdx.x / a.row_parts;
  int64_t first, end;
  part_rows(a, group, blockIdx.x - (int)(group * a.row_parts), &first, &end);
  float dw = 0.f, db = 0.f;
  for (int64_t row = first; row < end; ++row) {
    const float d = (float)((const X*)a.dy)[row * a.y_stride + col];
    dw = fmaf(d, ((float)((const X*)a.x)[row * a.x_stride + col] - a.mean[row]) * a.rstd[row], dw);
    db += d;
  }
  float* to = a.parts + (int64_t)blockIdx.x * 2 * a.cols;
  to[col] = dw;
  to[a.cols + col] = db;
}

// Adds up the parts of each group: WIDE columns a workgroup, the parts in slices of consecutive ones that follow each other.
template <int WIDE>
__global__ __launch_bounds__(1024) void norm_grad_sum_kernel(const float* __restrict__ parts, float* __restrict__ dweight,
                                                             float* __restrict__ dbias, int cols, int row_parts) {
  constexpr int SLICES = 1024 / WIDE;
  __shared__ float room[SLICES][WIDE];
  const int x = threadIdx.x % WIDE, c = blockIdx.y * WIDE + x, slice = threadIdx.x / WIDE;   // column of [2][cols]
  const int64_t group = blockIdx.x;
  float s = 0.f;
  if (c < 2 * cols) {
    const float* from = parts + group * row_parts * 2 * cols + c;
#pragma unroll 4
    for (int p = row_parts * slice / SLICES; p < row_parts * (slice + 1) / SLICES; ++p) s += from[(int64_t)p * 2 * cols];
  }
  room[slice][x] = s;
  __syncthreads();
  if (slice != 0 || c >= 2 * cols) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < SLICES; ++i) s += room[i][x];
  float* to = c < cols ? dweight : dbias;
  if (to) to[group * cols + (c < cols ? c : c - cols)] = s;
}

// ---- launches

constexpr int MOST_COLS = 8192;   // of a row kept in registers

int status() { return hipGetLastError() == hipSuccess ? JENGA_OK : JENGA_EHIP; }

// Eight columns a thread, whole wavefronts, 1024 threads at most.  (1024 for short rows too: 12068 x 777 float32
// to 8 bits 143 us instead of 25, 60000 x 5 690 instead of 64.)
int long_threads(int cols) { return std::min((cols + 511) / 512 * 64, 1024); }

template <typename X, typename P, bool E4M3, int NV, int WPR>
void run_norm_rows(const NormArgs& a, hipStream_t st) {
  const int64_t rows_at_once = 4 / WPR, wanted = (a.rows + rows_at_once - 1) / rows_at_once;
  norm_kernel<X, P, E4M3, NV, WPR><<<(unsigned)std::min<int64_t>(wanted, 256 * norm_per_cu<X, P, E4M3, NV>()), 256, 0, st>>>(a);
}

template <typename X, typename P, bool E4M3>
int run_norm(const NormArgs& a, hipStream_t st) {
  if (a.cols > MOST_COLS || a.cols < 8 || (E4M3 && a.cols % 8 != 0)) {
    norm_long_kernel<X, P, E4M3><<<(unsigned)std::min<int64_t>(a.rows, 1 << 20), long_threads(a.cols), 0, st>>>(a);
    return status();
  }
  if (a.cols <= 512) run_norm_rows<X, P, E4M3, 1, 1>(a, st);
  else if (a.cols <= 1024) run_norm_rows<X, P, E4M3, 1, 2>(a, st);
  else if (a.cols <= 1536) run_norm_rows<X, P, E4M3, 3, 1>(a, st);
  else if (a.cols <= 2048) run_norm_rows<X, P, E4M3, 1, 4>(a, st);
  else if (a.cols <= 4096) run_norm_rows<X, P, E4M3, 2, 4>(a, st);
  else if (a.cols <= 6144) run_norm_rows<X, P, E4M3, 3, 4>(a, st);
  else run_norm_rows<X, P, E4M3, 4, 4>(a, st);
  return status();
}

template <typename X, typename P, int NV, int WPR>
void run_grad_rows(const NormArgs& a, unsigned groups, hipStream_t st) {
  constexpr int WAVES = grad_waves(WPR);
  norm_grad_kernel<X, P, NV, WPR><<<groups * (unsigned)a.row_parts, 64 * WAVES, WAVES > WPR ? (size_t)a.cols * 8 : 0, st>>>(a);
}

template <typename X, typename P>
int run_grad(NormArgs a, unsigned groups, float* dweight, float* dbias, hipStream_t st) {
  // as many workgroups as the chip holds, eight rows each at least
  const bool in_registers = a.cols <= MOST_COLS && a.cols >= 8;
  const int per_cu = !in_registers ? 4 : a.cols <= 1024 ? grad_per_cu<1>() : a.cols <= 1536 ? grad_per_cu<3>() : a.cols <= 2048 ? grad_per_cu<1>() :
                     a.cols <= 4096 ? grad_per_cu<2>() : a.cols <= 6144 ? grad_per_cu<3>() : 1;
  const int64_t rows = std::min(a.rows, a.group_rows);
  a.row_parts = (int)std::max<int64_t>(1, std::min<int64_t>(256 * per_cu / groups, (rows + 7) / 8));
  if (!in_registers) {
    norm_grad_long_kernel<X, P><<<(unsigned)std::min<int64_t>(a.rows, 1 << 20), long_threads(a.cols), 0, st>>>(a);
    if (a.parts) norm_grad_columns_kernel<X><<<dim3(groups * a.row_parts, (a.cols + 255) / 256), 256, 0, st>>>(a);
  } else if (a.cols <= 512) {
    run_grad_rows<X, P, 1, 1>(a, groups, st);
  } else if (a.cols <= 1024) {
    run_grad_rows<X, P, 1, 2>(a, groups, st);
  } else if (a.cols <= 1536) {
    run_grad_rows<X, P, 3, 1>(a, groups, st);
  } else if (a.cols <= 2048) {
    run_grad_rows<X, P, 1, 4>(a, groups, st);
  } else if (a.cols <= 4096) {
    run_grad_rows<X, P, 2, 4>(a, groups, st);
  } else if (a.cols <= 6144) {
    run_grad_rows<X, P, 3, 4>(a, groups, st);
  } else {
    run_grad_rows<X, P, 2, 8>(a, groups, st);
  }
  if (!a.parts) return status();
  // 64 columns a workgroup, 32 while that leaves compute units idle.  Gradient in us, 64 -> 32: 12068 x 777 (25 workgroups of 64) 31.7 ->
  // 29.5; 2000 x 1536 (48) 20.2 -> 19.9; 600 x 8192 in 5 groups (1280) 28.7 -> 31.8.
  const unsigned wide = (2 * a.cols + 63) / 64;
  if (groups * wide < 256) norm_grad_sum_kernel<32><<<dim3(groups, 2 * wide), 1024, 0, st>>>(a.parts, dweight, dbias, a.cols, a.row_parts);
  else norm_grad_sum_kernel<64><<<dim3(groups, wide), 1024, 0, st>>>(a.parts, dweight, dbias, a.cols, a.row_parts);
  return status();
}

NormArgs args_of(const jenga_norm_config& c) {
  NormArgs a = {};
  a.rows = c.rows;
  a.group_rows = c.group_rows;
  a.x_stride = c.x_stride;
  a.y_stride = c.y_stride;
  a.param_stride = c.param_stride;
  a.cols = c.cols;
  a.scale_cols = (c.cols + 511) / 512 * 4;
  a.eps = c.eps;
  a.w0 = c.weight_offset;
  return a;
}

}  // namespace

extern "C" {

int jenga_layer_norm(const jenga_norm_config* cfg, const void* x, const void* weight_or_null, const void* bias_or_null, void* y,
                     uint8_t* y_scale_or_null, float* mean_or_null, float* rstd_or_null, void* stream) {
  const int why = jenga::norm_args_ok(cfg, x, weight_or_null, bias_or_null, y, y_scale_or_null, mean_or_null, rstd_or_null);
  if (why != JENGA_OK) return why;
  if (cfg->rows == 0) return JENGA_OK;
  NormArgs a = args_of(*cfg);
  a.x = x;
  a.weight = weight_or_null;
  a.bias = bias_or_null;
  a.y = y;
  a.y_scale = y_scale_or_null;
  a.mean = mean_or_null;
  a.rstd = rstd_or_null;
  hipStream_t st = (hipStream_t)stream;
  const bool f32_params = cfg->param_type == JENGA_F32, e4m3 = cfg->y_type == JENGA_E4M3;
#define JENGA_NORM(X, P) return e4m3 ? run_norm<X, P, true>(a, st) : run_norm<X, P, false>(a, st)
  switch (cfg->x_type) {
    case JENGA_BF16:
      if (f32_params) JENGA_NORM(__bf16, float);
      JENGA_NORM(__bf16, __bf16);
    case JENGA_F16:
      if (f32_params) JENGA_NORM(_Float16, float);
      JENGA_NORM(_Float16, _Float16);
    default: JENGA_NORM(float, float);
  }
#undef JENGA_NORM
}

int jenga_layer_norm_grad(const jenga_norm_config* cfg, const void* x, const void* dy, const void* weight_or_null, const float* mean,
                          const float* rstd, void* dx, float* dweight_or_null, float* dbias_or_null, void* workspace,
                          size_t workspace_bytes, void* stream) {
  const int why = jenga::norm_grad_args_ok(cfg, x, dy, weight_or_null, mean, rstd, dx, dweight_or_null, dbias_or_null, workspace,
                                           workspace_bytes);
  if (why != JENGA_OK) return why;
  if (cfg->rows == 0) return JENGA_OK;
  NormArgs a = args_of(*cfg);
  const int64_t groups = (cfg->rows + cfg->group_rows - 1) / cfg->group_rows;
  a.x = x;
  a.dy = dy;
  a.weight = weight_or_null;
  a.mean = (float*)mean;
  a.rstd = (float*)rstd;
  a.dx = dx;
  a.parts = dweight_or_null || dbias_or_null ? (float*)workspace : nullptr;
  hipStream_t st = (hipStream_t)stream;
  const bool f32_params = cfg->param_type == JENGA_F32;
#define JENGA_NORM_GRAD(X, P) return run_grad<X, P>(a, (unsigned)groups, dweight_or_null, dbias_or_null, st)
  switch (cfg->x_type) {
    case JENGA_BF16:
      if (f32_params) JENGA_NORM_GRAD(__bf16, float);
      JENGA_NORM_GRAD(__bf16, __bf16);
    case JENGA_F16:
      if (f32_params) JENGA_NORM_GRAD(_Float16, float);
      JENGA_NORM_GRAD(_Float16, _Float16);
    default: JENGA_NORM_GRAD(float, float);
  }
#undef JENGA_NORM_GRAD
}

}  // extern "C"
