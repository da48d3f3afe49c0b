// Root-mean-square norm of each row (or of each head of a row) behind the addition of a residual, and its gradient.
//
//   s = round(x + add)   r = 1 / sqrt(sum s^2 / C + eps)   y = s r (w0 + w)
//   h = s r   g = dy (w0 + w)   dx = r (g - h mean(g h)) + dtotal   dw = sum over rows and heads of dy h
//
// Bound by memory: a row is read once into registers, and everything that is made of it is made from there.  All sums are float32.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "jenga_device.h"
#include "jenga_internal.h"
#include "jenga_tiles.h"

namespace {

using namespace jenga;

enum Out { SAME, EIGHT_BITS, FOUR_BITS };

struct Strided {
  void* at;
  int64_t row, head;
};

struct RmsArgs {
  Strided x, add, sum, y;      // in the gradient: the normed sum, dtotal, dx, dy
  const void* weight;
  uint8_t* y_scale;
  float *rstd, *parts;
  int64_t rows;                // with their heads
  uint32_t heads, by_heads, heads_shift;
  int32_t cols, scale_cols, y_bytes;
  float eps, w0;
  // Results of 16 bits of more than 64 MiB go past the caches: 33272 x 5120 267 -> 262 us, gradient 268 -> 255; 60000 x 1024 99 -> 79; Q and K of
  // 33272 x 40 x 128 160 -> 148 each.  (Smaller ones may be read again from there; float32 rows off the 16-byte grid lose, 12068 x 777 24 -> 31.)
  bool past;
};


// Row n of a tensor; n / heads by multiplication, exact below 2^31.
struct Place {
  int64_t row;
  uint32_t head;
};
__device__ __forceinline__ Place place_of(const RmsArgs& a, int64_t n) {
  if (a.heads == 1) return {n, 0};
  const uint32_t i = (uint32_t)n, token = (__umulhi(i, a.by_heads) + i) >> a.heads_shift;
  return {token, i - token * a.heads};
}
template <typename X>
__device__ __forceinline__ X* row_of(const Strided& t, const Place& p) {
  return (X*)t.at + p.row * t.row + (int64_t)p.head * t.head;
}

// Rows are taken in pieces of eight columns.  Where their number is no multiple of eight, the last piece ends with the row and overlaps the one
// before it: both compute and store the same results there, and sums take only what is a piece's own.  Nothing of a row is stored before all of
// it has been read, by whichever wavefront.  Results of few bits have their places in blocks: there, and in rows of less than eight columns,
// the last piece is read and written one by one (40000 x 2500 bf16: one by one 199 us, its gradient 328; so 164 and 164).
enum Ends { EVEN, OVER, ONE_BY_ONE };
struct Piece {
  int col, skip;   // of the first value; so many are the piece's before
};
template <Out OUT>
__device__ __forceinline__ Ends ends_of(int cols) {
  return cols % 8 == 0 ? EVEN : OUT == SAME && cols > 8 ? OVER : ONE_BY_ONE;
}
__device__ __forceinline__ Piece piece_at(int col, int cols, Ends ends) {
  const int c = ends == OVER ? min(col, cols - 8) : col;
  return {c, col - c};
}
// Zeros past the row's end.
template <typename T>
__device__ __forceinline__ typename Eight<T>::raw piece(const T* p, int col, int cols, Ends ends) {
  typename Eight<T>::raw r = {};
  if (ends != ONE_BY_ONE) {
    if (col < cols) r = *(const typename Eight<T>::raw*)(p + piece_at(col, cols, ends).col);
    return r;
  }
  return load_eight(p + col, cols - col);
}
// past: not to be kept in the caches.
template <typename T>
__device__ __forceinline__ void put_piece(T* p, int col, int cols, Ends ends, bool past, const f32x8& f) {
  if (ends != ONE_BY_ONE) {
    if (col >= cols) return;
    T* to = p + piece_at(col, cols, ends).col;
    const auto r = Eight<T>::narrow(f);
    if constexpr (sizeof(T) == 2) {
      if (past) {
        store_once(to, make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]));
        return;
      }
    }
    *(typename Eight<T>::raw*)to = r;
    return;
  }
  store_eight(p + col, f, cols - col);
}

// Sum over LANES neighbouring lanes; all of them get it.  LANES > 64: over the wavefronts of a row, through `room`, which is not
// written again before everybody has read it.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v, float* room) {
  if constexpr (LANES < 64) {
    v += dpp_f32<0xB1, 0xF>(0.f, v);     // quad_perm 1 0 3 2
    v += dpp_f32<0x4E, 0xF>(0.f, v);     // quad_perm 2 3 0 1
    v += dpp_f32<0x141, 0xF>(0.f, v);    // row_half_mirror
    if constexpr (LANES >= 16) v += dpp_f32<0x140, 0xF>(0.f, v);   // row_mirror
    if constexpr (LANES >= 32) v += __shfl_xor(v, 16);
    return v;
  } else {
    constexpr int WAVES = LANES / 64;
    v = wave_sum_f32(v);
    if constexpr (WAVES == 1) return v;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) room[wave] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) s += room[wave / WAVES * WAVES + i];
    return s;
  }
}

// Eight results of a row from column `col` on; in 8 bits 16 lanes hold a block of 128 columns, in 4 bits four lanes one of 32.
template <typename X, Out OUT>
__device__ __forceinline__ void put(const RmsArgs& a, const Place& p, int col, Ends ends, bool mine, f32x8 y) {
  if constexpr (OUT == SAME) {
    if (mine) put_piece(row_of<X>(a.y, p), col, a.cols, ends, a.past, y);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (col + i >= a.cols) y[i] = 0.f;   // the columns that fill up the last block: an infinite r makes NaN of their zeros
  uint8_t* to = (uint8_t*)a.y.at + p.row * a.y_bytes;
  uint8_t* scales = a.y_scale + p.row * a.scale_cols;
  if constexpr (OUT == EIGHT_BITS) {
    const uint32_t byte = scale_byte(row_max_f32(largest_of(y)));
    const int block = col >> 7;
    if (mine && col < a.y_bytes) {
      *(uint2*)(to + col) = to_e4m3(y, inverse_scale(byte));
      if ((threadIdx.x & 15) == 0) scales[block] = (uint8_t)byte;
    }
  } else {
    const uint32_t byte = mx_scale_byte(quad_max(magnitude_of(y)));
    if (mine && col < 2 * a.y_bytes) {
      *(uint32_t*)(to + (col >> 1)) = to_e2m1(y, byte);
      if ((threadIdx.x & 3) == 0) scales[col >> 5] = (uint8_t)byte;
    }
  }
}

// The bytes, three at most, that fill up the last group of four scales.
__device__ __forceinline__ void fill_scales(const RmsArgs& a, const Place& p, int lane) {
  const int block = (a.y_bytes >> 7) + lane;
  if (block < a.scale_cols) a.y_scale[p.row * a.scale_cols + block] = 0;
}

constexpr int threads_of(int lanes) { return lanes > 128 ? lanes : 256; }

// LANES threads to a row, NV pieces of eight columns each.  33272 x 5120 bf16 with residual and sum 262 us, 5.2 TB/s (a plain copy: 4.88);
// Q and K of 33272 x 40 x 128 148 each, 4.6 TB/s out of a projection's rows.  A workgroup takes rows a grid apart; it keeps the weight in registers, and the next row
// is on its way while one is worked on.
template <typename X, typename P, Out OUT, int LANES, int NV>
__global__ __launch_bounds__(threads_of(LANES)) void rms_kernel(RmsArgs a) {
  constexpr int THREADS = threads_of(LANES), STEP = LANES * 8, AT_ONCE = THREADS / LANES;
  __shared__ float room[2][THREADS / 64];
  const int slot = threadIdx.x / LANES, col0 = threadIdx.x % LANES * 8;
  const Ends ends = ends_of<OUT>(a.cols);
  // of piece v: one that no row's end is in is an even one
  auto ends_at = [&](int v) { return v * STEP + STEP <= a.cols ? EVEN : ends; };
  typename Eight<P>::raw weight[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    weight[v] = {};
    if (a.weight) weight[v] = piece((const P*)a.weight, v * STEP + col0, a.cols, ends_at(v));
  }
  typename Eight<X>::raw next[NV], next_add[NV];
  Place next_place = {};
  auto fetch = [&](int64_t row) {   // zeros for a row that is not there
#pragma unroll
    for (int v = 0; v < NV; ++v) next[v] = next_add[v] = {};
    if (row >= a.rows) return;
    next_place = place_of(a, row);
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        next[v] = piece(row_of<X>(a.x, next_place), v * STEP + col0, a.cols, ends_at(v));
        if (a.add.at) next_add[v] = piece(row_of<X>(a.add, next_place), v * STEP + col0, a.cols, ends_at(v));
      }
  };
  const int64_t step = (int64_t)gridDim.x * AT_ONCE;
  fetch((int64_t)blockIdx.x * AT_ONCE + slot);
  int turn = 0;
  // every thread takes every turn (there are barriers in it); one without a row has zeros and nothing to store
  for (int64_t row0 = (int64_t)blockIdx.x * AT_ONCE; row0 < a.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool mine = row < a.rows;
    const Place place = next_place;
    f32x8 f[NV];
    float square = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        f[v] = Eight<X>::wide(next[v]);
        if (a.add.at) f[v] = Eight<X>::wide(Eight<X>::narrow(f[v] + Eight<X>::wide(next_add[v])));
        if (ends_at(v) != OVER) {
#pragma unroll
          for (int i = 0; i < 8; ++i) square = fmaf(f[v][i], f[v][i], square);
        } else {
          const int skip = piece_at(v * STEP + col0, a.cols, OVER).skip;
#pragma unroll
          for (int i = 0; i < 8; ++i) square = fmaf(f[v][i], i >= skip ? f[v][i] : 0.f, square);
        }
      }
    fetch(row + step);
    const float rstd = 1.0f / sqrtf(lanes_sum<LANES>(square, room[turn]) / (float)a.cols + a.eps);
    if (mine && a.rstd && threadIdx.x % LANES == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        const f32x8 w = Eight<P>::wide(weight[v]) + a.w0;
        f32x8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = f[v][i] * rstd * w[i];
        if (a.sum.at && mine) put_piece(row_of<X>(a.sum, place), v * STEP + col0, a.cols, ends_at(v), a.past, f[v]);
        put<X, OUT>(a, place, v * STEP + col0, ends_at(v), mine, y);
      }
    if (OUT == EIGHT_BITS && mine) fill_scales(a, place, threadIdx.x % LANES);
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

// Rows too long for registers: a workgroup each, read again for the results.  A thread reads only what it has written itself.
template <typename X, typename P, Out OUT>
__global__ __launch_bounds__(1024) void rms_long_kernel(RmsArgs a) {
  __shared__ float room[16];
  const int padded = (a.cols + 511) / 512 * 512;   // every lane of a wavefront takes every turn: a block's scale is several lanes' work
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const Place p = place_of(a, row);
    auto value = [&](int col) {
      f32x8 f = Eight<X>::wide(load_eight(row_of<X>(a.x, p) + col, a.cols - col));
      if (a.add.at) f = Eight<X>::wide(Eight<X>::narrow(f + Eight<X>::wide(load_eight(row_of<X>(a.add, p) + col, a.cols - col))));
      return f;
    };
    float square = 0.f;
    for (int col = threadIdx.x * 8; col < a.cols; col += 8192) {
      const f32x8 f = value(col);
      if (a.sum.at) store_eight(row_of<X>(a.sum, p) + col, f, a.cols - col);
#pragma unroll
      for (int i = 0; i < 8; ++i) square = fmaf(f[i], f[i], square);
    }
    const float rstd = 1.0f / sqrtf(block_sum(square, room) / (float)a.cols + a.eps);
    if (threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
    for (int col = threadIdx.x * 8; col < padded; col += 8192) {
      f32x8 w = a.w0, y = 0.f;
      if (col < a.cols) {
        const f32x8 f = a.sum.at ? Eight<X>::wide(load_eight(row_of<X>(a.sum, p) + col, a.cols - col)) : value(col);
        if (a.weight) w += Eight<P>::wide(load_eight((const P*)a.weight + col, a.cols - col));
        y = f * rstd * w;
      }
      put<X, OUT>(a, p, col, ONE_BY_ONE, true, y);
    }
    if (OUT == EIGHT_BITS) fill_scales(a, p, threadIdx.x);
  }
}

// ---- gradient

// The same shape; a workgroup leaves the sums of its rows for the weight's gradient in parts[workgroup][cols].
template <typename X, typename P, int LANES, int NV>
__global__ __launch_bounds__(threads_of(LANES)) void rms_grad_kernel(RmsArgs a) {
  constexpr int THREADS = threads_of(LANES), STEP = LANES * 8, AT_ONCE = THREADS / LANES;
  __shared__ float room[2][THREADS / 64];
  __shared__ float sums[AT_ONCE > 1 ? AT_ONCE * STEP * NV : 1];
  const int slot = threadIdx.x / LANES, col0 = threadIdx.x % LANES * 8;
  const Ends ends = ends_of<SAME>(a.cols);
  auto ends_at = [&](int v) { return v * STEP + STEP <= a.cols ? EVEN : ends; };
  typename Eight<P>::raw weight[NV];
  f32x8 dw[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    dw[v] = 0.f;
    weight[v] = {};
    if (a.weight) weight[v] = piece((const P*)a.weight, v * STEP + col0, a.cols, ends_at(v));
  }
  typename Eight<X>::raw next_s[NV], next_d[NV], next_t[NV];
  float next_r = 0.f;
  Place next_place = {};
  auto fetch = [&](int64_t row) {   // zeros for a row that is not there
    next_r = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) next_s[v] = next_d[v] = next_t[v] = {};
    if (row >= a.rows) return;
    next_place = place_of(a, row);
    next_r = a.rstd[row];
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        const int col = v * STEP + col0;
        next_s[v] = piece(row_of<X>(a.x, next_place), col, a.cols, ends_at(v));
        next_d[v] = piece(row_of<X>(a.y, next_place), col, a.cols, ends_at(v));
        if (a.add.at) next_t[v] = piece(row_of<X>(a.add, next_place), col, a.cols, ends_at(v));
      }
  };
  const int64_t step = (int64_t)gridDim.x * AT_ONCE;
  fetch((int64_t)blockIdx.x * AT_ONCE + slot);
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * AT_ONCE; row0 < a.rows; row0 += step, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool mine = row < a.rows;
    const Place place = next_place;
    const float rstd = next_r;
    f32x8 h[NV], g[NV];
    typename Eight<X>::raw t[NV];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols) {
        const f32x8 s = Eight<X>::wide(next_s[v]), d = Eight<X>::wide(next_d[v]), w = Eight<P>::wide(weight[v]) + a.w0;
        t[v] = next_t[v];
        // it is there: dx may go over it
#pragma unroll
        for (int i = 0; i < (int)sizeof(t[v]) / 4; ++i) asm volatile("" : "+v"(t[v].w[i]));
        // rstd may be infinite, and 0 times that is NaN: columns that are not there have h = 0.  Of a piece's before, the sums take nothing
        const int col = v * STEP + col0, skip = piece_at(col, a.cols, ends_at(v)).skip;
        const float r = col < a.cols ? rstd : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[v][i] = s[i] * r;
          if (ends_at(v) == ONE_BY_ONE && col + i >= a.cols) h[v][i] = 0.f;
          g[v][i] = d[i] * w[i];
          dw[v][i] = fmaf(d[i], h[v][i], dw[v][i]);
          sum = fmaf(i >= skip ? g[v][i] : 0.f, h[v][i], sum);
        }
      }
    fetch(row + step);
    const float mean = lanes_sum<LANES>(sum, room[turn]) / (float)a.cols;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * STEP < a.cols && mine) {
        f32x8 d;
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = rstd * fmaf(-h[v][i], mean, g[v][i]);
        if (a.add.at) d += Eight<X>::wide(t[v]);
        put_piece(row_of<X>(a.sum, place), v * STEP + col0, a.cols, ends_at(v), a.past, d);
      }
  }
  if (!a.parts) return;
  float* to = a.parts + (int64_t)blockIdx.x * a.cols;
  // a piece's own columns: to memory, or to LDS where several rows at a time have sums
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int col = v * STEP + col0;
    const Piece p = piece_at(col, a.cols, ends_at(v));
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (col < a.cols && i >= p.skip && p.col + i < a.cols) {
        if constexpr (AT_ONCE == 1) to[p.col + i] = dw[v][i];
        else sums[slot * STEP * NV + p.col + i] = dw[v][i];
      }
  }
  if constexpr (AT_ONCE > 1) {
    __syncthreads();
    for (int col = threadIdx.x; col < a.cols; col += THREADS) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) s += sums[i * STEP * NV + col];
      to[col] = s;
    }
  }
}

// Rows too long for registers: dx by a workgroup per row, the sums of the columns by a thread per column.
template <typename X, typename P>
__global__ __launch_bounds__(1024) void rms_grad_long_kernel(RmsArgs a) {
  __shared__ float room[16];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const Place p = place_of(a, row);
    const float rstd = a.rstd[row];
    float mean = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      float sum = 0.f;
      for (int col = threadIdx.x * 8; col < a.cols; col += 8192) {
        const int n = a.cols - col;
        f32x8 w = a.w0;
        if (a.weight) w += Eight<P>::wide(load_eight((const P*)a.weight + col, n));
        const f32x8 g = Eight<X>::wide(load_eight(row_of<X>(a.y, p) + col, n)) * w;
        f32x8 h = Eight<X>::wide(load_eight(row_of<X>(a.x, p) + col, n));
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] *= i < n ? rstd : 0.f;
        if (pass == 0) {
#pragma unroll
          for (int i = 0; i < 8; ++i) sum = fmaf(g[i], h[i], sum);
        } else {
          f32x8 d;
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] = rstd * fmaf(-h[i], mean, g[i]);
          if (a.add.at) d += Eight<X>::wide(load_eight(row_of<X>(a.add, p) + col, n));
          store_eight(row_of<X>(a.sum, p) + col, d, n);
        }
      }
      if (pass == 0) mean = block_sum(sum, room) / (float)a.cols;
    }
  }
}
template <typename X>
__global__ __launch_bounds__(256) void rms_grad_columns_kernel(RmsArgs a) {
  const int col = blockIdx.y * 256 + threadIdx.x;
  if (col >= a.cols) return;
  const int64_t first = a.rows * blockIdx.x / gridDim.x, end = a.rows * (blockIdx.x + 1) / gridDim.x;
  float dw = 0.f;
  for (int64_t row = first; row < end; ++row) {
    const Place p = place_of(a, row);
    dw = fmaf((float)row_of<X>(a.y, p)[col], (float)row_of<X>(a.x, p)[col] * a.rstd[row], dw);
  }
  a.parts[(int64_t)blockIdx.x * a.cols + col] = dw;
}

// Adds up the parts: 32 columns a workgroup, the parts in 32 slices of consecutive ones that follow each other.
__global__ __launch_bounds__(1024) void rms_grad_sum_kernel(const float* __restrict__ parts, float* __restrict__ dweight, int cols,
                                                            int n_parts) {
  __shared__ float room[32][33];
  const int x = threadIdx.x & 31, col = blockIdx.x * 32 + x, slice = threadIdx.x >> 5;
  float s = 0.f;
  if (col < cols) {
#pragma unroll 4
    for (int p = n_parts * slice / 32; p < n_parts * (slice + 1) / 32; ++p) s += parts[(int64_t)p * cols + col];
  }
  room[slice][x] = s;
  __syncthreads();
  if (slice != 0 || col >= cols) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) s += room[i][x];
  dweight[col] = s;
}

// ---- launches

constexpr int MOST_COLS = 16384;   // of a row kept in registers

int status() { return hipGetLastError() == hipSuccess ? JENGA_OK : JENGA_EHIP; }

// Workgroups that the chip holds: as many as the grid has, at most.
template <typename K>
unsigned resident(K kernel, int threads) {
  int n = 0;
  if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, (const void*)kernel, threads, 0) != hipSuccess) n = 1;
  return 256u * (unsigned)std::max(n, 1);
}

template <typename X, typename P, Out OUT, int LANES, int NV>
void run_rows(const RmsArgs& a, hipStream_t st) {
  constexpr int THREADS = threads_of(LANES), AT_ONCE = THREADS / LANES;
  static const unsigned most = resident(rms_kernel<X, P, OUT, LANES, NV>, THREADS);
  rms_kernel<X, P, OUT, LANES, NV><<<(unsigned)std::min<int64_t>((a.rows + AT_ONCE - 1) / AT_ONCE, most), THREADS, 0, st>>>(a);
}

// One piece a thread up to 2048 columns, but three pieces of a wavefront for 1025 to 1536 (63424 x 1536 bf16 150 us, one piece of three wavefronts 178); beyond, shapes of
// whole wavefronts without many idle lanes.  120 M values bf16 with residual and sum, us, to the same type / 8 bits / 4 bits, with the shape taken and with another:
// 1536 columns 64 x 3 182 / 153 / 145, 192 x 1 194 / 193 / 181; 4096 256 x 2 181 / 153 / 141, 512 x 1 185 / 160 / 147; 5120 768 x 1 185 / 162 / 156, 640 x 1
// 188 / 162 / 153; 8192 512 x 2 176 / 155 / 146, 1024 x 1 178 / 169 / 165; 12288 512 x 3 184 / 158 / 149, 768 x 2 178 / 196 / 192.
template <typename X, typename P, Out OUT>
int run_rms(const RmsArgs& a, hipStream_t st) {
  if (a.cols > MOST_COLS)
    rms_long_kernel<X, P, OUT><<<(unsigned)std::min<int64_t>(a.rows, 1 << 20), 1024, 0, st>>>(a);
  else if (a.cols <= 64 && OUT == SAME) run_rows<X, P, OUT, 8, 1>(a, st);
  else if (a.cols <= 128) run_rows<X, P, OUT, 16, 1>(a, st);
  else if (a.cols <= 256) run_rows<X, P, OUT, 32, 1>(a, st);
  else if (a.cols <= 512) run_rows<X, P, OUT, 64, 1>(a, st);
  else if (a.cols <= 1024) run_rows<X, P, OUT, 128, 1>(a, st);
  else if (a.cols <= 1536) run_rows<X, P, OUT, 64, 3>(a, st);
  else if (a.cols <= 2048) run_rows<X, P, OUT, 256, 1>(a, st);
  else if (a.cols <= 4096) run_rows<X, P, OUT, 256, 2>(a, st);
  else if (a.cols <= 6144) run_rows<X, P, OUT, 768, 1>(a, st);
  else if (a.cols <= 8192) run_rows<X, P, OUT, 512, 2>(a, st);
  else if (a.cols <= 12288) run_rows<X, P, OUT, 512, 3>(a, st);
  else run_rows<X, P, OUT, 1024, 2>(a, st);
  return status();
}

template <typename X, typename P, int LANES, int NV>
int run_grad_rows(const RmsArgs& a, hipStream_t st) {
  constexpr int THREADS = threads_of(LANES), AT_ONCE = THREADS / LANES;
  static const unsigned most = std::min(resident(rms_grad_kernel<X, P, LANES, NV>, THREADS), 1024u);
  // four rows a slot at least, so that the sums are not what takes the time
  const unsigned n = (unsigned)std::min<int64_t>((a.rows + 4 * AT_ONCE - 1) / (4 * AT_ONCE), most);
  rms_grad_kernel<X, P, LANES, NV><<<n, THREADS, 0, st>>>(a);
  return (int)n;
}

// One piece a thread where rows have exact shapes for it: gradient of 63424 x 1536 bf16 in three pieces of a wavefront 225 us, in one of
// three 158; 33272 x 5120 510 -> 266, 12000 x 8192 234 -> 146.  2049 to 3584 columns take two pieces of four wavefronts, which differ little from one of
// eight (120 M values bf16, 2560 columns 165 and 159 us, 3584 141 and 136, 4096, which takes the latter, 146 and 136; 60 M float32 140 and 138, 140 and 140).  The last
// two shapes keep 10 to 21 registers in scratch, and still beat the kernel that reads rows again: 6000 x 10000 float32 304 and 337, 6000 x 16000 bf16 228 and 348
// (4000 x 16000 float32, with 68, does not: 414 and 335).
template <typename X, typename P>
int run_grad(const RmsArgs& a, float* dweight, hipStream_t st) {
  int parts;
  if (a.cols > (sizeof(X) == 4 ? 12288 : MOST_COLS)) {
    rms_grad_long_kernel<X, P><<<(unsigned)std::min<int64_t>(a.rows, 1 << 20), 1024, 0, st>>>(a);
    parts = (int)std::min<int64_t>((a.rows + 7) / 8, 64);
    if (a.parts) rms_grad_columns_kernel<X><<<dim3(parts, (a.cols + 255) / 256), 256, 0, st>>>(a);
  } else if (a.cols <= 64) parts = run_grad_rows<X, P, 8, 1>(a, st);
  else if (a.cols <= 128) parts = run_grad_rows<X, P, 16, 1>(a, st);
  else if (a.cols <= 256) parts = run_grad_rows<X, P, 32, 1>(a, st);
  else if (a.cols <= 512) parts = run_grad_rows<X, P, 64, 1>(a, st);
  else if (a.cols <= 1024) parts = run_grad_rows<X, P, 128, 1>(a, st);
  else if (a.cols <= 1536) parts = run_grad_rows<X, P, 192, 1>(a, st);
  else if (a.cols <= 2048) parts = run_grad_rows<X, P, 256, 1>(a, st);
  else if (a.cols <= 3584) parts = run_grad_rows<X, P, 256, 2>(a, st);
  else if (a.cols <= 4096) parts = run_grad_rows<X, P, 512, 1>(a, st);
  else if (a.cols <= 5120) parts = run_grad_rows<X, P, 640, 1>(a, st);
  else if (a.cols <= 6144) parts = run_grad_rows<X, P, 768, 1>(a, st);
  else if (a.cols <= 8192) parts = run_grad_rows<X, P, 1024, 1>(a, st);
  else if (a.cols <= 12288) parts = run_grad_rows<X, P, 768, 2>(a, st);
  else if constexpr (sizeof(X) == 2) parts = run_grad_rows<X, P, 1024, 2>(a, st);
  else return JENGA_EUNSUPPORTED;   // not reached
  if (a.parts) rms_grad_sum_kernel<<<(a.cols + 31) / 32, 1024, 0, st>>>(a.parts, dweight, a.cols, parts);
  return status();
}

RmsArgs args_of(const jenga_rms_config& c) {
  RmsArgs a = {};
  a.x = {nullptr, c.x_row, c.x_head};
  a.add = {nullptr, c.add_row, c.add_head};
  a.sum = {nullptr, c.sum_row, c.sum_head};
  a.y = {nullptr, c.y_row, c.y_head};
  a.rows = c.rows * c.heads;
  a.heads = (uint32_t)c.heads;
  if (c.heads > 1) {   // n / heads = (n * floor(2^32 (2^l - heads) / heads + 1) / 2^32 + n) / 2^l, 2^l >= heads
    int l = 0;
    while ((1ll << l) < c.heads) ++l;
    a.heads_shift = (uint32_t)l;
    a.by_heads = (uint32_t)((((1ull << l) - (uint64_t)c.heads) << 32) / (uint64_t)c.heads + 1);
  }
  a.cols = c.cols;
  const int blocks = (c.cols + 127) / 128;
  a.y_bytes = c.y_type == JENGA_E4M3 ? blocks * 128 : blocks * 64;
  a.scale_cols = c.y_type == JENGA_E4M3 ? (blocks + 3) / 4 * 4 : blocks * 4;
  a.eps = c.eps;
  a.w0 = c.weight_offset;
  a.past = (double)a.rows * c.cols * 2 > 64.0 * (1 << 20);
  return a;
}

}  // namespace

extern "C" {

int jenga_rms_norm(const jenga_rms_config* cfg, const void* x, const void* residual_or_null, const void* weight_or_null,
                   void* total_or_null, void* y, uint8_t* y_scale_or_null, float* rstd_or_null, void* stream) {
  const int why = jenga::rms_args_ok(cfg, x, residual_or_null, weight_or_null, total_or_null, y, y_scale_or_null, rstd_or_null);
  if (why != JENGA_OK) return why;
  if (cfg->rows == 0) return JENGA_OK;
  RmsArgs a = args_of(*cfg);
  a.x.at = (void*)x;
  a.add.at = (void*)residual_or_null;
  a.sum.at = total_or_null;
  a.y.at = y;
  a.weight = weight_or_null;
  a.y_scale = y_scale_or_null;
  a.rstd = rstd_or_null;
  hipStream_t st = (hipStream_t)stream;
  const bool f32_params = cfg->param_type == JENGA_F32;
#define JENGA_RMS(X, P)                                             \
  return cfg->y_type == JENGA_E4M3   ? run_rms<X, P, EIGHT_BITS>(a, st) \
         : cfg->y_type == JENGA_E2M1 ? run_rms<X, P, FOUR_BITS>(a, st)  \
                                     : run_rms<X, P, SAME>(a, st)
  switch (cfg->x_type) {
    case JENGA_BF16:
      if (f32_params) JENGA_RMS(__bf16, float);
      JENGA_RMS(__bf16, __bf16);
    case JENGA_F16:
      if (f32_params) JENGA_RMS(_Float16, float);
      JENGA_RMS(_Float16, _Float16);
    default: JENGA_RMS(float, float);
  }
#undef JENGA_RMS
}

int jenga_rms_norm_grad(const jenga_rms_config* cfg, const void* x, const void* dy, const void* weight_or_null, const float* rstd,
                        const void* dtotal_or_null, void* dx, float* dweight_or_null, void* workspace, size_t workspace_bytes,
                        void* stream) {
  const int why = jenga::rms_grad_args_ok(cfg, x, dy, weight_or_null, rstd, dtotal_or_null, dx, dweight_or_null, workspace, workspace_bytes);
  if (why != JENGA_OK) return why;
  if (cfg->rows == 0) return JENGA_OK;
  RmsArgs a = args_of(*cfg);
  a.x.at = (void*)x;
  a.y.at = (void*)dy;
  a.add.at = (void*)dtotal_or_null;
  a.sum.at = dx;
  a.weight = weight_or_null;
  a.rstd = (float*)rstd;
  a.parts = dweight_or_null ? (float*)workspace : nullptr;
  hipStream_t st = (hipStream_t)stream;
  const bool f32_params = cfg->param_type == JENGA_F32;
  switch (cfg->x_type) {
    case JENGA_BF16: return f32_params ? run_grad<__bf16, float>(a, dweight_or_null, st) : run_grad<__bf16, __bf16>(a, dweight_or_null, st);
    case JENGA_F16: return f32_params ? run_grad<_Float16, float>(a, dweight_or_null, st) : run_grad<_Float16, _Float16>(a, dweight_or_null, st);
    default: return run_grad<float, float>(a, dweight_or_null, st);
  }
}

}  // extern "C"
