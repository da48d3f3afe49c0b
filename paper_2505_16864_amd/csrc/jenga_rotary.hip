// Rotary positions over the three axes of the token grid.
//
// Pair i of an axis with d channels turns by the angle (origin + step * cell) * theta^(-2i/d); cos and sin of every pair and cell come
// from a table of T d_t + H d_h + W d_w floats that stays in the caches, so the tensors themselves are what is moved: bound by memory.
// A thread keeps the angles of its channels of one token in registers and walks over the heads.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "jenga_device.h"
#include "jenga_internal.h"

namespace {

using namespace jenga;

struct RotaryArgs {
  const void* src[2];
  void* dst[2];
  int64_t src_batch[2], src_token[2], src_head[2], dst_batch[2], dst_token[2], dst_head[2];
  int heads[2];
  int count;
  const float2* table;
  const int32_t *src_of_pos, *cells;
  int64_t tokens, units;   // units: batch * tokens
  GridCells grid;
  int pairs[3];            // of each axis
  int base[3];             // of each axis in the table
  int head_dim;
  int heads_per_wg;
  float sign;              // -1: the inverse rotation
};

// The cell of token n of batch entry b on each axis; false: not rotated.  -1 on an axis: its channels are not.
__device__ __forceinline__ bool cells_of(const RotaryArgs& a, int64_t b, int64_t n, int cell[3]) {
  if (a.cells) {
    const int32_t* c = a.cells + (b * a.tokens + n) * 3;
    const int most[3] = {a.grid.T - 1, a.grid.H - 1, a.grid.W - 1};
#pragma unroll
    for (int i = 0; i < 3; ++i) cell[i] = min(c[i], most[i]);
    return true;
  }
  if (a.src_of_pos) n = a.src_of_pos[n];
  if (n < 0 || n >= a.grid.cells) return false;
  a.grid.split((uint32_t)n, cell);
  return true;
}

// Channel c: its axis, pair and whether it is the pair's second one.  Axis 3: not rotated.
struct Channel {
  int axis, pair, second;
};
template <bool HALVES>
__device__ __forceinline__ Channel channel(const RotaryArgs& a, int c) {
  Channel r;
  const int d0 = 2 * a.pairs[0], d1 = d0 + 2 * a.pairs[1], d2 = d1 + 2 * a.pairs[2];
  r.axis = c < d0 ? 0 : c < d1 ? 1 : c < d2 ? 2 : 3;
  const int i = c - (r.axis == 0 ? 0 : r.axis == 1 ? d0 : d1), half = r.axis == 0 ? a.pairs[0] : r.axis == 1 ? a.pairs[1] : a.pairs[2];
  r.second = HALVES ? i >= half : i & 1;
  r.pair = HALVES ? i - (r.second ? half : 0) : i >> 1;
  return r;
}
__device__ __forceinline__ float2 turn_of(const RotaryArgs& a, const Channel& c, const int cell[3], bool rotated) {
  if (!rotated || c.axis == 3) return make_float2(1.f, 0.f);
  const int at = c.axis == 0 ? cell[0] : c.axis == 1 ? cell[1] : cell[2];
  if (at < 0) return make_float2(1.f, 0.f);
  const int pairs = c.axis == 0 ? a.pairs[0] : c.axis == 1 ? a.pairs[1] : a.pairs[2];
  const int base = c.axis == 0 ? a.base[0] : c.axis == 1 ? a.base[1] : a.base[2];
  float2 t = a.table[base + at * pairs + c.pair];
  t.y *= a.sign;
  return t;
}

// Any even head_dim: a thread per pair of channels.
template <typename X, bool HALVES>
__global__ __launch_bounds__(256) void rotary_pairs_kernel(RotaryArgs a) {
  const int half = a.head_dim / 2;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, unit = id / half;
  if (unit >= a.units) return;
  const int p = (int)(id - unit * half);
  const int64_t b = unit / a.tokens, n = unit - b * a.tokens;
  int c0 = 2 * p, c1 = 2 * p + 1;
  if (HALVES) {   // pair p of the axis it falls on; behind the axes neighbours
    const int e0 = a.pairs[0], e1 = e0 + a.pairs[1], e2 = e1 + a.pairs[2];
    if (p < e0) c0 = p, c1 = p + a.pairs[0];
    else if (p < e1) c0 = p + e0, c1 = c0 + a.pairs[1];
    else if (p < e2) c0 = p + e1, c1 = c0 + a.pairs[2];
  }
  int cell[3] = {0, 0, 0};
  const bool rotated = cells_of(a, b, n, cell);
  const float2 t = turn_of(a, channel<HALVES>(a, c0), cell, rotated);
  const int h0 = blockIdx.y * a.heads_per_wg;
  for (int k = 0; k < a.count; ++k) {
    const X* src = (const X*)a.src[k] + b * a.src_batch[k] + n * a.src_token[k];
    X* dst = (X*)a.dst[k] + b * a.dst_batch[k] + n * a.dst_token[k];
    const int h1 = min(h0 + a.heads_per_wg, a.heads[k]);
    for (int h = h0; h < h1; ++h) {
      const float x = (float)src[h * a.src_head[k] + c0], y = (float)src[h * a.src_head[k] + c1];
      dst[h * a.dst_head[k] + c0] = (X)(x * t.x - y * t.y);
      dst[h * a.dst_head[k] + c1] = (X)(x * t.y + y * t.x);
    }
  }
}

int status() { return hipGetLastError() == hipSuccess ? JENGA_OK : JENGA_EHIP; }

template <typename X>
int run_rotary(const RotaryArgs& a, bool halves, hipStream_t st) {
  const int most = a.count > 1 ? std::max(a.heads[0], a.heads[1]) : a.heads[0];
  const int64_t wgs = (a.units * (a.head_dim / 2) + 255) / 256;
  if (wgs >= 1 << 24) return JENGA_EUNSUPPORTED;   // 2^32 threads are more than a grid has in x
  const dim3 grid((unsigned)wgs, (most + a.heads_per_wg - 1) / a.heads_per_wg);
  if (halves) rotary_pairs_kernel<X, true><<<grid, 256, 0, st>>>(a);
  else rotary_pairs_kernel<X, false><<<grid, 256, 0, st>>>(a);
  return status();
}

}  // namespace

extern "C" int jenga_rotary(const jenga_rotary_config* cfg, const jenga_plan* plan_or_null, const int32_t* cells_or_null,
                            const float* table, const jenga_rotary_tensor* tensors, int32_t count, int64_t batch, int64_t tokens,
                            void* stream) {
  const int why = jenga::rotary_args_ok(cfg, plan_or_null, cells_or_null, table, tensors, count, batch, tokens);
  if (why != JENGA_OK) return why;
  if (plan_or_null) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != plan_or_null->device) return JENGA_EINVAL;
  }
  if (batch == 0 || tokens == 0) return JENGA_OK;
  RotaryArgs a = {};
  for (int k = 0; k < count; ++k) {
    a.src[k] = tensors[k].src;
    a.dst[k] = tensors[k].dst;
    a.heads[k] = tensors[k].heads;
    a.src_batch[k] = tensors[k].src_batch;
    a.src_token[k] = tensors[k].src_token;
    a.src_head[k] = tensors[k].src_head;
    a.dst_batch[k] = tensors[k].dst_batch;
    a.dst_token[k] = tensors[k].dst_token;
    a.dst_head[k] = tensors[k].dst_head;
  }
  a.count = count;
  a.table = (const float2*)table;
  a.cells = cells_or_null;
  a.src_of_pos = plan_or_null ? plan_or_null->d_src_of_pos : nullptr;
  a.tokens = tokens;
  a.units = batch * tokens;
  a.grid = jenga::GridCells(cfg->T, cfg->H, cfg->W);
  const int cells[3] = {cfg->T, cfg->H, cfg->W};
  for (int i = 0, base = 0; i < 3; ++i) {
    a.pairs[i] = cfg->dim[i] / 2;
    a.base[i] = base;
    base += cells[i] * a.pairs[i];
  }
  a.head_dim = cfg->head_dim;
  a.heads_per_wg = 8;
  a.sign = cfg->flags & JENGA_ROTARY_INVERSE ? -1.f : 1.f;
  const bool halves = (cfg->flags & JENGA_ROTARY_HALVES) != 0;
  hipStream_t st = (hipStream_t)stream;
  if (cfg->type == JENGA_BF16) return run_rotary<__bf16>(a, halves, st);
  if (cfg->type == JENGA_F16) return run_rotary<_Float16>(a, halves, st);
  return run_rotary<float>(a, halves, st);
}
