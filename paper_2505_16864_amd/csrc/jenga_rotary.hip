// Rotary positions over the three axes of the token grid.
//
// Pair i of an axis with d channels turns by the angle (origin + step * cell) * theta^(-2i/d); cos and sin of every pair and cell come
// from a table of T d_t + H d_h + W d_w floats that stays in the caches, so the tensors themselves are what is moved: bound by memory.
// A thread keeps the angles of its channels of one token in registers and walks over the heads.  Q and K of 119056 tokens x 24 heads x 128
// bf16: 576 us, 5.08 TB/s, either way of pairing; in place 4.9 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "jenga_device.h"
#include "jenga_internal.h"
#include "jenga_pool.h"

namespace {

using namespace jenga;

struct Turns {
  const float2* table;
  GridCells grid;
  int pairs[3];   // of each axis
  int base[3];    // of each axis in the table
  float sign;     // -1: the inverse rotation
};

struct RotaryArgs {
  const void* src[2];
  void* dst[2];
  int64_t src_batch[2], src_token[2], src_head[2], dst_batch[2], dst_token[2], dst_head[2];
  int heads[2];
  int count;
  Turns turns;
  const int32_t *src_of_pos, *cells;
  uint32_t tokens, units;   // units: batch * tokens, times the pairs of a head below 2^32
  int head_dim;
  int heads_per_wg;
};

// A pair's place: its axis (3: none, it stays) and where cell 0 of it is in the table.  The checks of arguments hold the pairs of all
// cells below 2^31 - 1024, so that 32 bits take any place.
struct Pair {
  int axis, at, step;
};

// Channel c: the pair that it belongs to, the other channel of it, and whether it is the second one.
template <bool HALVES>
__device__ __forceinline__ Pair pair_of(const Turns& t, int c, int* other, bool* second) {
  const int e0 = 2 * t.pairs[0], e1 = e0 + 2 * t.pairs[1], e2 = e1 + 2 * t.pairs[2];
  Pair p;
  p.axis = c < e0 ? 0 : c < e1 ? 1 : c < e2 ? 2 : 3;
  const int start = p.axis == 0 ? 0 : p.axis == 1 ? e0 : e1, i = c - start;
  p.step = p.axis == 0 ? t.pairs[0] : p.axis == 1 ? t.pairs[1] : t.pairs[2];
  *second = HALVES ? i >= p.step : i & 1;
  *other = p.axis == 3 ? c : HALVES ? (*second ? c - p.step : c + p.step) : c ^ 1;
  p.at = (p.axis == 0 ? t.base[0] : p.axis == 1 ? t.base[1] : t.base[2]) + (HALVES ? (*second ? i - p.step : i) : i >> 1);
  return p;
}

// Halves paired: the first channel of pair p of a head; behind the axes the channels 2 p of neighbours that stay.
__device__ __forceinline__ int first_of_pair(const Turns& t, int p) {
  const int e0 = t.pairs[0], e1 = e0 + t.pairs[1], e2 = e1 + t.pairs[2];
  return p < e0 ? p : p < e1 ? p + e0 : p < e2 ? p + e1 : 2 * p;
}

// cos and sin for a pair of a token in these cells; false: the pair stays as it is, to the last bit.
__device__ __forceinline__ bool turn_of(const Turns& t, const Pair& p, const int cell[3], float2* turn) {
  const int n = p.axis == 0 ? cell[0] : p.axis == 1 ? cell[1] : cell[2];
  const bool turned = p.axis < 3 && n >= 0;
  *turn = make_float2(1.f, 0.f);
  if (turned) {
    *turn = t.table[p.at + n * p.step];
    turn->y *= t.sign;
  }
  return turned;
}

// The cell of token n, unit `unit`, on each axis, -1: not turned.
__device__ __forceinline__ void cells_of(const RotaryArgs& a, uint32_t unit, int64_t n, int cell[3]) {
  cell[0] = cell[1] = cell[2] = -1;
  if (a.cells) {
    const int32_t* c = a.cells + (size_t)unit * 3;
    cell[0] = min(c[0], a.turns.grid.T - 1);
    cell[1] = min(c[1], a.turns.grid.H - 1);
    cell[2] = min(c[2], a.turns.grid.W - 1);
    return;
  }
  if (a.src_of_pos) n = a.src_of_pos[n];
  if (n >= 0 && n < a.turns.grid.cells) a.turns.grid.split((uint32_t)n, cell);
}

// Neighbours paired, head_dim a multiple of 8: a thread turns eight channels of a token, in registers, four heads at a time.
template <typename X>
__global__ __launch_bounds__(256) void rotary_neighbours_kernel(RotaryArgs a) {
  const int pieces = a.head_dim / 8;
  const uint32_t id = blockIdx.x * 256u + threadIdx.x, unit = id / (uint32_t)pieces;
  if (unit >= a.units) return;
  const int c = (int)(id - unit * (uint32_t)pieces) * 8;
  const int64_t b = unit / a.tokens, n = unit % a.tokens;
  int cell[3];
  cells_of(a, unit, n, cell);
  float2 turn[4];
  bool turned[4], any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int other;
    bool second;
    turned[i] = turn_of(a.turns, pair_of<false>(a.turns, c + 2 * i, &other, &second), cell, &turn[i]);
    any |= turned[i];
  }
  const int h0 = blockIdx.y * a.heads_per_wg;
  for (int k = 0; k < a.count; ++k) {
    const X* src = (const X*)a.src[k] + b * a.src_batch[k] + n * a.src_token[k] + c;
    X* dst = (X*)a.dst[k] + b * a.dst_batch[k] + n * a.dst_token[k] + c;
    const int h1 = min(h0 + a.heads_per_wg, a.heads[k]);
    if (!any && src == dst && a.src_head[k] == a.dst_head[k]) continue;   // in place: nothing to do
    for (int h = h0; h < h1; h += 4) {
      typename Eight<X>::raw raw[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (h + u < h1) raw[u] = *(const typename Eight<X>::raw*)(src + (h + u) * a.src_head[k]);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (h + u >= h1) break;
        f32x8 v = Eight<X>::wide(raw[u]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = v[2 * i], y = v[2 * i + 1];
          v[2 * i] = turned[i] ? fmaf(x, turn[i].x, -(y * turn[i].y)) : x;
          v[2 * i + 1] = turned[i] ? fmaf(x, turn[i].y, y * turn[i].x) : y;
        }
        *(typename Eight<X>::raw*)(dst + (h + u) * a.dst_head[k]) = Eight<X>::narrow(v);
      }
    }
  }
}

// Channels half an axis apart paired, head_dim a multiple of 8 up to 512: a thread turns eight channels of a token; the other channel
// of each pair comes from the wavefront's LDS, where the lanes of a token put theirs.  (The two of a pair may lie anywhere against
// the 16-byte pieces: an axis of 42 channels has halves of 21.)
template <typename X>
__global__ __launch_bounds__(256) void rotary_halves_kernel(RotaryArgs a) {
  __shared__ __attribute__((aligned(16))) X room[4][4][64 * 8];   // wavefront, head
  const int pieces = a.head_dim / 8, per_wave = 64 / pieces, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = lane / pieces, c = (lane - row * pieces) * 8;
  const uint32_t unit = (blockIdx.x * 4u + wave) * per_wave + row;
  if (row >= per_wave || unit >= a.units) return;
  const int64_t b = unit / a.tokens, n = unit % a.tokens;
  int cell[3];
  cells_of(a, unit, n, cell);
  float2 turn[8];
  int other[8];
  bool turned[8], any = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    bool second;
    turned[i] = turn_of(a.turns, pair_of<true>(a.turns, c + i, &other[i], &second), cell, &turn[i]);
    if (!second) turn[i].y = -turn[i].y;   // x cos - y sin, y cos + x sin
    other[i] += row * a.head_dim;
    any |= turned[i];
  }
  const int h0 = blockIdx.y * a.heads_per_wg;
  for (int k = 0; k < a.count; ++k) {
    const X* src = (const X*)a.src[k] + b * a.src_batch[k] + n * a.src_token[k] + c;
    X* dst = (X*)a.dst[k] + b * a.dst_batch[k] + n * a.dst_token[k] + c;
    const int h1 = min(h0 + a.heads_per_wg, a.heads[k]);
    for (int h = h0; h < h1; h += 4) {
      typename Eight<X>::raw raw[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (h + u < h1) raw[u] = *(const typename Eight<X>::raw*)(src + (h + u) * a.src_head[k]);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (h + u < h1) __builtin_memcpy(&room[wave][u][row * a.head_dim + c], &raw[u], sizeof(raw[u]));
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (h + u >= h1) break;
        f32x8 v = Eight<X>::wide(raw[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y = (float)room[wave][u][other[i]];
          v[i] = turned[i] ? fmaf(v[i], turn[i].x, y * turn[i].y) : v[i];
        }
        if (any || src != dst) *(typename Eight<X>::raw*)(dst + (h + u) * a.dst_head[k]) = Eight<X>::narrow(v);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Any even head_dim: a thread per pair of channels, two values at a time: what its instructions move bounds it.  Q and K of 31712 tokens x 12
// heads x 66 bf16: 65 us, 3.1 TB/s, halves paired 78; x 90 86 and 98 (128 channels, eight a thread: 84).
template <typename X, bool HALVES>
__global__ __launch_bounds__(256) void rotary_pairs_kernel(RotaryArgs a) {
  const int half = a.head_dim / 2;
  const uint32_t id = blockIdx.x * 256u + threadIdx.x, unit = id / (uint32_t)half;
  if (unit >= a.units) return;
  const int p = (int)(id - unit * (uint32_t)half);
  const int64_t b = unit / a.tokens, n = unit % a.tokens;
  int cell[3], other;
  bool second;
  cells_of(a, unit, n, cell);
  float2 t;
  const int c0 = HALVES ? first_of_pair(a.turns, p) : 2 * p;
  const Pair pair = pair_of<HALVES>(a.turns, c0, &other, &second);
  const int c1 = pair.axis == 3 ? c0 + 1 : other;
  const bool turned = turn_of(a.turns, pair, cell, &t);
  const int h0 = blockIdx.y * a.heads_per_wg;
  for (int k = 0; k < a.count; ++k) {
    const X* src = (const X*)a.src[k] + b * a.src_batch[k] + n * a.src_token[k];
    X* dst = (X*)a.dst[k] + b * a.dst_batch[k] + n * a.dst_token[k];
    const int h1 = min(h0 + a.heads_per_wg, a.heads[k]);
    for (int h = h0; h < h1; ++h) {
      const X *s = src + h * a.src_head[k];
      X* d = dst + h * a.dst_head[k];
      const X x = s[c0], y = s[c1];
      d[c0] = turned ? (X)fmaf((float)x, t.x, -((float)y * t.y)) : x;
      d[c1] = turned ? (X)fmaf((float)x, t.y, (float)y * t.x) : y;
    }
  }
}

int status() { return hipGetLastError() == hipSuccess ? JENGA_OK : JENGA_EHIP; }

// A workgroup takes eight heads of its tokens, so that a token's angles are looked up for eight, but four while that makes fewer than four
// workgroups a compute unit.  us, 8 -> 4: 2 x 6034 tokens x 8 heads x 64 (378 workgroups) 13.2 -> 12.5, halves 17.0 -> 14.1, float32
// halves 24.8 -> 22.2; 31712 x 12 x 128 (3964) 80.8 -> 83.5, halves 84.6 -> 85.7.
template <typename X>
int run_rotary(RotaryArgs a, bool halves, hipStream_t st) {
  const int most = a.count > 1 ? std::max(a.heads[0], a.heads[1]) : a.heads[0], pieces = a.head_dim / 8;
  const bool by_pairs = a.head_dim % 8 != 0 || (halves && pieces > 64);
  const int64_t per_wg = by_pairs || !halves ? 256 : 64 / pieces * 4;   // threads, or tokens
  const int64_t work = by_pairs ? (int64_t)a.units * (a.head_dim / 2) : halves ? a.units : (int64_t)a.units * pieces;
  const int64_t wgs = (work + per_wg - 1) / per_wg;
  a.heads_per_wg = wgs * ((most + 7) / 8) < 1024 ? 4 : 8;
  const dim3 grid((unsigned)wgs, (most + a.heads_per_wg - 1) / a.heads_per_wg);
  if (by_pairs && halves) rotary_pairs_kernel<X, true><<<grid, 256, 0, st>>>(a);
  else if (by_pairs) rotary_pairs_kernel<X, false><<<grid, 256, 0, st>>>(a);
  else if (halves) rotary_halves_kernel<X><<<grid, 256, 0, st>>>(a);
  else rotary_neighbours_kernel<X><<<grid, 256, 0, st>>>(a);
  return status();
}

Turns turns_of(const jenga_rotary_config& c, const float* table) {
  Turns t;
  t.table = (const float2*)table;
  t.grid = GridCells(c.T, c.H, c.W);
  const int cells[3] = {c.T, c.H, c.W};
  for (int i = 0, base = 0; i < 3; ++i) {
    t.pairs[i] = c.dim[i] / 2;
    t.base[i] = base;
    base += cells[i] * t.pairs[i];
  }
  t.sign = c.flags & JENGA_ROTARY_INVERSE ? -1.f : 1.f;
  return t;
}

// ---- Q, K and V into curve order, Q and K turned on the way, with the block means of Q and K: the first launch of
// jenga_forward_rotary.  As permute_pool_kernel (jenga_select.hip), a workgroup for a block of one (batch, head), tokens `token` elements
// apart.  The turn is rounded to bf16 before it is stored and summed, so that the results are those of jenga_rotary and
// jenga_forward one after the other.  Three tensors of 119056 tokens x 24 heads x 128: 1.10 ms, 4.0 TB/s, the lookups of angles; 0.86 without
// the turn, and 0.58 for a turn by itself.
struct TurnedMoves {
  const uint16_t* src[3];
  Piece16* dst[3];
  double* mean[2];
  int64_t token;
};
template <int M_TOK, int D, bool HALVES>
__global__ __launch_bounds__(256) void permute_turn_pool_kernel(TurnedMoves moves, Turns turns, const int32_t* __restrict__ src_of_pos,
                                                                const int32_t* __restrict__ blk_valid, int n_src, int M_v, int batch) {
  constexpr int CH = D / 8, G = 256 / CH, ROWS = M_TOK / G;   // pieces of a row, rows at a time, rows of a thread
  __shared__ double red[G][D];
  __shared__ __attribute__((aligned(16))) __bf16 room[HALVES ? 256 * 8 : 8];
  const int h = blockIdx.x, j = blockIdx.y, heads = gridDim.x, M = gridDim.y;
  const int tensor = blockIdx.z / batch, b = blockIdx.z - tensor * batch;
  const int c = threadIdx.x % CH, g = threadIdx.x / CH;
  const uint16_t* src = moves.src[tensor] + (size_t)b * n_src * moves.token + h * D + c * 8;
  Piece16* dst = moves.dst[tensor] + (((size_t)b * heads + h) * M + j) * (M_TOK * CH) + threadIdx.x;
  int s[ROWS];
#pragma unroll
  for (int u = 0; u < ROWS; ++u) s[u] = src_of_pos[j * M_TOK + u * G + g];
  Piece16 v[ROWS];
#pragma unroll
  for (int u = 0; u < ROWS; ++u) {
    v[u] = Piece16{{0, 0, 0, 0}};
    if (s[u] >= 0) v[u] = *(const Piece16*)(src + (size_t)s[u] * moves.token);
  }
  if (tensor < 2 && j < M_v) {   // blocks of vision tokens hold no text
    // The thread's four pairs of each row: of its piece, or, halves paired, those CH apart, so that the lanes of a row read neighbouring
    // angles; they take both channels from LDS then and put them back.
    Pair pair[4];
    int first[4], other[4];
    bool second;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      first[i] = HALVES ? first_of_pair(turns, c + i * CH) : c * 8 + 2 * i;
      pair[i] = pair_of<HALVES>(turns, first[i], &other[i], &second);
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
      int cell[3] = {-1, -1, -1};
      if (s[u] >= 0) turns.grid.split((uint32_t)s[u], cell);
      float2 t;
      if (HALVES) {
        __bf16* row = room + g * D;
        __builtin_memcpy(row + c * 8, &v[u], 16);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // a row is 8 or 16 lanes of one wavefront
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!turn_of(turns, pair[i], cell, &t)) continue;
          const float x = (float)row[first[i]], y = (float)row[other[i]];
          row[first[i]] = (__bf16)fmaf(x, t.x, -(y * t.y));
          row[other[i]] = (__bf16)fmaf(y, t.x, x * t.y);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_memcpy(&v[u], row + c * 8, 16);
      } else {
        f32x8 f = Eight<__bf16>::wide(v[u]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = f[2 * i], y = f[2 * i + 1];
          if (turn_of(turns, pair[i], cell, &t)) f[2 * i] = fmaf(x, t.x, -(y * t.y)), f[2 * i + 1] = fmaf(x, t.y, y * t.x);
        }
        v[u] = Eight<__bf16>::narrow(f);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < ROWS; ++u) dst[u * 256] = v[u];
  if (tensor == 2 || (tensor == 0 && j >= M_v)) return;
  double acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0;
#pragma unroll
  for (int u = 0; u < ROWS; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      acc[2 * e] += bf16_bits_to_double(v[u].w[e] & 0xFFFFu);
      acc[2 * e + 1] += bf16_bits_to_double(v[u].w[e] >> 16);
    }
#pragma unroll
  for (int e = 0; e < 8; ++e) red[g][c * 8 + e] = acc[e];
  __syncthreads();
  if (threadIdx.x < D) {
    double sum = 0.0;
#pragma unroll
    for (int gg = 0; gg < G; ++gg) sum += red[gg][threadIdx.x];
    const size_t row = ((size_t)b * heads + h) * (tensor == 0 ? M_v : M) + j;
    moves.mean[tensor][row * D + pooled_pos<D>(j, threadIdx.x)] = sum / (double)blk_valid[j];
  }
}

template <int M_TOK, int D>
void run_permute_turn_pool(const jenga_plan* p, TurnedMoves moves, const Turns& turns, bool halves, void* ws, hipStream_t st) {
  pooled_rows<D>(p, ws, &moves.mean[0], &moves.mean[1]);
  const dim3 grid(p->cfg.heads, p->info.M, 3 * p->cfg.batch);
  const int n_src = p->info.N_v + p->cfg.n_text;
  if (halves)
    permute_turn_pool_kernel<M_TOK, D, true><<<grid, 256, 0, st>>>(moves, turns, p->d_src_of_pos, p->d_blk_valid, n_src, p->info.M_v, p->cfg.batch);
  else
    permute_turn_pool_kernel<M_TOK, D, false><<<grid, 256, 0, st>>>(moves, turns, p->d_src_of_pos, p->d_blk_valid, n_src, p->info.M_v, p->cfg.batch);
}

}  // namespace

namespace jenga {

int launch_permute_turn_pool(const jenga_plan* p, const jenga_rotary_config& c, const float* table, const void* const src[3],
                             int64_t token_stride, void* const dst[3], void* select_ws, void* stream) {
  TurnedMoves moves = {{(const uint16_t*)src[0], (const uint16_t*)src[1], (const uint16_t*)src[2]},
                       {(Piece16*)dst[0], (Piece16*)dst[1], (Piece16*)dst[2]}, {nullptr, nullptr}, token_stride};
  const Turns turns = turns_of(c, table);
  const bool halves = (c.flags & JENGA_ROTARY_HALVES) != 0;
  hipStream_t st = (hipStream_t)stream;
  const int m = p->cfg.block;
  if (p->cfg.head_dim == 128) {
    if (m == 128) run_permute_turn_pool<128, 128>(p, moves, turns, halves, select_ws, st);
    else if (m == 64) run_permute_turn_pool<64, 128>(p, moves, turns, halves, select_ws, st);
    else run_permute_turn_pool<32, 128>(p, moves, turns, halves, select_ws, st);
  } else {
    if (m == 128) run_permute_turn_pool<128, 64>(p, moves, turns, halves, select_ws, st);
    else if (m == 64) run_permute_turn_pool<64, 64>(p, moves, turns, halves, select_ws, st);
    else run_permute_turn_pool<32, 64>(p, moves, turns, halves, select_ws, st);
  }
  return status();
}

}  // namespace jenga

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
  a.turns = turns_of(*cfg, table);
  a.cells = cells_or_null;
  a.src_of_pos = plan_or_null ? plan_or_null->d_src_of_pos : nullptr;
  a.tokens = (uint32_t)tokens;
  a.units = (uint32_t)(batch * tokens);
  a.head_dim = cfg->head_dim;
  const bool halves = (cfg->flags & JENGA_ROTARY_HALVES) != 0;
  hipStream_t st = (hipStream_t)stream;
  if (cfg->type == JENGA_BF16) return run_rotary<__bf16>(a, halves, st);
  if (cfg->type == JENGA_F16) return run_rotary<_Float16>(a, halves, st);
  return run_rotary<float>(a, halves, st);
}
