// Layer norm over the columns of each row, with a weight and a bias per group of rows, and its gradient.
//
//   mu = sum x / C    var = sum (x - mu)^2 / C    r = 1 / sqrt(var + eps)    h = (x - mu) r    y = h (w0 + w) + b
//   g = dy (w0 + w)   dx = r (g - mean(g) - h mean(g h))   dw = sum over the group's rows of dy h   db = sum of dy
//
// Bound by memory: a row is read once into registers, as it lies in memory, and summed twice from there (the second sum is of
// (x - mu)^2, so that a large mean costs no digits).  All sums are float32.
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

// A wavefront per row, up to NV pieces of 512 columns.
template <typename X, typename P, bool E4M3, int NV>
__global__ __launch_bounds__(256) void norm_kernel(NormArgs a) {
  const int lane = threadIdx.x & 63;
  for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < a.rows; row += (int64_t)gridDim.x * 4) {
    const X* x = (const X*)a.x + row * a.x_stride;
    typename Eight<X>::raw raw[NV];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * 512 < a.cols) raw[v] = load_eight(x + v * 512 + lane * 8, a.cols - v * 512 - lane * 8);
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * 512 < a.cols) {
        const f32x8 f = Eight<X>::wide(raw[v]);
        sum += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
      }
    const float mean = wave_sum_f32(sum) / (float)a.cols;
    float square = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * 512 < a.cols) {
        const f32x8 f = Eight<X>::wide(raw[v]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float d = f[i] - mean;
          if (v * 512 + lane * 8 + i < a.cols) square = fmaf(d, d, square);
        }
      }
    const float rstd = 1.0f / sqrtf(wave_sum_f32(square) / (float)a.cols + a.eps);
    if (lane == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    const int64_t group = row / a.group_rows;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * 512 < a.cols) {
        const int col = v * 512 + lane * 8;
        const f32x8 f = Eight<X>::wide(raw[v]);
        f32x8 w, b, y;
        params<P>(a, group, col, &w, &b);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fmaf((f[i] - mean) * rstd, w[i], b[i]);
        put<X, E4M3>(a, row, col, y);
      }
  }
}

// Sum over the 1024 threads of a workgroup; all of them get it.
__device__ __forceinline__ float block_sum(float v, float* room) {
  v = wave_sum_f32(v);
  __syncthreads();   // the room is free
  if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += room[i];
  return s;
}

// Rows too long for a wavefront's registers: a workgroup each, read again for each of the three passes.
template <typename X, typename P, bool E4M3>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  __shared__ float room[16];
  const int whole = (a.cols + 8191) & ~8191;   // every thread takes every turn: the scales of a block are 16 lanes' work
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const X* x = (const X*)a.x + row * a.x_stride;
    float sum = 0.f, square = 0.f;
    for (int col = threadIdx.x * 8; col < a.cols; col += 8192) {
      const f32x8 f = Eight<X>::wide(load_eight(x + col, a.cols - col));
      sum += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
    }
    const float mean = block_sum(sum, room) / (float)a.cols;
    for (int col = threadIdx.x * 8; col < a.cols; col += 8192) {
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
    for (int col = threadIdx.x * 8; col < whole; col += 8192) {
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

// A workgroup takes a part of a group's rows, WPR wavefronts to a row, up to NV pieces of WPR * 512 columns, and keeps the sums of
// its columns in registers; they go to parts[workgroup][2][cols].
template <typename X, typename P, int NV, int WPR>
__global__ __launch_bounds__(256) void norm_grad_kernel(NormArgs a) {
  constexpr int STEP = WPR * 512, AT_ONCE = 4 / WPR;
  __shared__ float room[2][4][2];
  extern __shared__ float sums[];   // [2][cols], for the rows of AT_ONCE wavefronts
  const int64_t group = blockIdx.x / a.row_parts;
  const int part = blockIdx.x - (int)(group * a.row_parts);
  const int wave = threadIdx.x >> 6, slot = wave / WPR;
  const int col0 = (threadIdx.x % (WPR * 64)) * 8;
  int64_t first, end;
  part_rows(a, group, part, &first, &end);
  f32x8 dw[NV], db[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) dw[v] = db[v] = 0.f;
  int turn = 0;
  // every wavefront takes every turn (there are barriers in it); one without a row has nothing to store
  for (int64_t row0 = first; row0 < end; row0 += AT_ONCE, turn ^= 1) {
    const int64_t row = row0 + slot;
    const bool mine = row < end;
    f32x8 h[NV], g[NV];
    float rstd = 0.f, mean = 0.f, sum_g = 0.f, sum_gh = 0.f;
    if (mine) mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      h[v] = g[v] = 0.f;
      const int col = v * STEP + col0, n = a.cols - col;
      if (mine && n > 0) {
        f32x8 w = a.w0;
        if (a.weight) w += Eight<P>::wide(load_eight((const P*)a.weight + group * a.param_stride + col, n));
        const f32x8 x = Eight<X>::wide(load_eight((const X*)a.x + row * a.x_stride + col, n));
        const f32x8 d = Eight<X>::wide(load_eight((const X*)a.dy + row * a.y_stride + col, n));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[v][i] = i < n ? (x[i] - mean) * rstd : 0.f;
          g[v][i] = d[i] * w[i];   // d is 0 past the end
          dw[v][i] = fmaf(d[i], h[v][i], dw[v][i]);
          db[v][i] += d[i];
          sum_g += g[v][i];
          sum_gh = fmaf(g[v][i], h[v][i], sum_gh);
        }
      }
    }
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
    for (int v = 0; v < NV; ++v) {
      const int col = v * STEP + col0, n = a.cols - col;
      if (mine && n > 0) {
        f32x8 d;
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = rstd * (g[v][i] - mg - h[v][i] * mgh);
        store_eight((X*)a.dx + row * a.x_stride + col, d, n);
      }
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
          const int col = v * STEP + col0 + i;
          if (col < a.cols) {
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

// Rows too long for that: dx by a workgroup per row, the sums of the columns by a thread per column.
template <typename X, typename P>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormArgs a) {
  __shared__ float room[16];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const X *x = (const X*)a.x + row * a.x_stride, *dy = (const X*)a.dy + row * a.y_stride;
    const P* weight = (const P*)a.weight + row / a.group_rows * a.param_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float sum_g = 0.f, sum_gh = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      for (int col = threadIdx.x * 8; col < a.cols; col += 8192) {
        const int n = a.cols - col;
        f32x8 w = a.w0, d;
        if (a.weight) w += Eight<P>::wide(load_eight(weight + col, n));
        const f32x8 f = Eight<X>::wide(load_eight(x + col, n)), g = Eight<X>::wide(load_eight(dy + col, n)) * w;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float h = (f[i] - mean) * rstd;
          if (pass == 0) sum_g += g[i], sum_gh = fmaf(g[i], h, sum_gh);   // g is 0 past the end
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

// Adds up the parts of each group, in order: 64 columns a workgroup, four of its wavefronts a quarter of the parts each.
__global__ __launch_bounds__(256) void norm_grad_sum_kernel(const float* __restrict__ parts, float* __restrict__ dweight,
                                                            float* __restrict__ dbias, int cols, int row_parts) {
  __shared__ float room[4][64];
  const int c = blockIdx.y * 64 + (threadIdx.x & 63), quarter = threadIdx.x >> 6;   // column of [2][cols]
  const int64_t group = blockIdx.x;
  float s = 0.f;
  if (c < 2 * cols)
    for (int p = row_parts * quarter / 4; p < row_parts * (quarter + 1) / 4; ++p) s += parts[(group * row_parts + p) * 2 * cols + c];
  room[quarter][threadIdx.x & 63] = s;
  __syncthreads();
  if (quarter != 0 || c >= 2 * cols) return;
  s = (room[0][c & 63] + room[1][c & 63]) + (room[2][c & 63] + room[3][c & 63]);
  float* to = c < cols ? dweight : dbias;
  if (to) to[group * cols + (c < cols ? c : c - cols)] = s;
}

// ---- launches

constexpr int MOST_COLS = 8192;   // of a row kept in registers

int status() { return hipGetLastError() == hipSuccess ? JENGA_OK : JENGA_EHIP; }

template <typename X, typename P, bool E4M3>
int run_norm(const NormArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)std::min<int64_t>((a.rows + 3) / 4, 1 << 20);
  if (a.cols <= 512) norm_kernel<X, P, E4M3, 1><<<grid, 256, 0, st>>>(a);
  else if (a.cols <= 2048) norm_kernel<X, P, E4M3, 4><<<grid, 256, 0, st>>>(a);
  else if (a.cols <= 5120) norm_kernel<X, P, E4M3, 10><<<grid, 256, 0, st>>>(a);
  else if (a.cols <= MOST_COLS) norm_kernel<X, P, E4M3, 16><<<grid, 256, 0, st>>>(a);
  else norm_long_kernel<X, P, E4M3><<<(unsigned)std::min<int64_t>(a.rows, 1 << 20), 1024, 0, st>>>(a);
  return status();
}

template <typename X, typename P>
int run_grad(const NormArgs& a, unsigned groups, float* dweight, float* dbias, hipStream_t st) {
  const unsigned wgs = groups * (unsigned)a.row_parts;
  const size_t lds = (size_t)a.cols * 8;
  if (a.cols <= 512) norm_grad_kernel<X, P, 1, 1><<<wgs, 256, lds, st>>>(a);
  else if (a.cols <= 2048) norm_grad_kernel<X, P, 4, 1><<<wgs, 256, lds, st>>>(a);
  else if (a.cols <= 4096) norm_grad_kernel<X, P, 2, 4><<<wgs, 256, 0, st>>>(a);
  else if (a.cols <= MOST_COLS) norm_grad_kernel<X, P, 4, 4><<<wgs, 256, 0, st>>>(a);
  else {
    norm_grad_long_kernel<X, P><<<(unsigned)std::min<int64_t>(a.rows, 1 << 20), 1024, 0, st>>>(a);
    if (a.parts) norm_grad_columns_kernel<X><<<dim3(wgs, (a.cols + 255) / 256), 256, 0, st>>>(a);
  }
  if (a.parts)
    norm_grad_sum_kernel<<<dim3(groups, (2 * a.cols + 63) / 64), 256, 0, st>>>(a.parts, dweight, dbias, a.cols, a.row_parts);
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
  a.row_parts = jenga::norm_grad_parts(*cfg);
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
