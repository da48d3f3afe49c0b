// Softmax attention of packed sequences to all of their keys, causal or not, with heads that share keys.
//
//   o_i = sum over j of p_ij v_j / sum over j of p_ij,   p_ij = 2^(c q_i k_j - m_i),   c = scale log2(e)
//
// The rows of a sequence and of the heads that share keys are packed: row n is token n / group, head n % group.  A tile of packed rows walks
// its keys once; the reference m_i of a row moves only when the sum of a step leaves its range (see SUM_MAX), and cancels.  The transposed
// products S^T = K Q^T and O^T = V^T P^T keep a row in one lane of every accumulator, and the accumulators of S^T are the operand of
// the second product as they are.
//
// Lengths are on the device.  A workgroup finds its tile from them; where there are more than 64 sequences, which is what a wavefront looks at
// in one go, a first launch makes a list instead.  Where there are few tiles, long ones are cut along their keys, and a second launch joins the
// parts in the order of the keys.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "jenga_device.h"
#include "jenga_internal.h"
#include "jenga_tiles.h"

namespace {

using namespace jenga;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct DenseArgs {
  const uint16_t *q, *k, *v;
  uint16_t* out;
  const int32_t *q_start, *kv_start, *kv_len;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, out_row, out_head;
  int32_t q_rows, kv_rows, sequences, kv_heads, group;
  uint32_t by_group, group_shift;
  int32_t causal, take_out;   // take_out: steps that some rows do not see whole may hold values of keys that they do not see, or that are not there
  float scale_log2e;
  int32_t tile, keys, max_tiles, max_slots, workgroups, may_split;   // keys: of a step
  int32_t *counts, *bins;   // of a list: items and merges; tiles of the sequences in front of each
  DenseItem* items;         // or NULL
  DenseMerge* merges;
  float *stat, *part;       // [slot][kv_heads][tile][2]: reference, sum; [slot][kv_heads][tile][D], 128 rows in the order of the accumulators
};

// ---- the two types

template <typename T>
struct Type;
template <>
struct Type<__bf16> {
  typedef bf16x8 eight;
  static constexpr float SUM_MAX = 1073741824.0f;   // 2^30
  static constexpr bool WIDE = true;                // values may be as large as float32 holds
  static constexpr uint32_t EXPONENT = 0x7F807F80u;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  }
  static __device__ __forceinline__ f32x16 mul32(const eight& a, const eight& b, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
#endif
    return c;
  }
  static __device__ __forceinline__ f32x4 mul16(const eight& a, const eight& b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#endif
    return c;
  }
};
template <>
struct Type<_Float16> {
  typedef f16x8 eight;
  static constexpr float SUM_MAX = 32768.0f;   // below the largest fp16
  static constexpr bool WIDE = false;
  static constexpr uint32_t EXPONENT = 0x7C007C00u;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
  }
  static __device__ __forceinline__ f32x16 mul32(const eight& a, const eight& b, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
#endif
    return c;
  }
  static __device__ __forceinline__ f32x4 mul16(const eight& a, const eight& b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
#endif
    return c;
  }
};

// Whether one of the 16-bit values is an infinity or a NaN: a halfword whose exponent bits are all set.
template <typename T>
__device__ __forceinline__ bool not_finite(uint32_t w) {
  const uint32_t v = (w & Type<T>::EXPONENT) ^ Type<T>::EXPONENT;
  return ((v - 0x00010001u) & ~v & 0x80008000u) != 0;
}

// The finite ones of two values, 0 for the others.
template <typename T>
__device__ __forceinline__ uint32_t finite_part(uint32_t w) {
  const uint32_t e = w & Type<T>::EXPONENT;
  return ((e & 0xFFFFu) == (Type<T>::EXPONENT & 0xFFFFu) ? 0u : w & 0xFFFFu) | ((e >> 16) == (Type<T>::EXPONENT >> 16) ? 0u : w & 0xFFFF0000u);
}
// A value that is not finite, 0 for others.
template <typename T>
__device__ __forceinline__ float rest_of(T v) {
  const float f = (float)v;
  return fabsf(f) < __builtin_inff() ? 0.f : f;
}
// Values that are not finite, of keys that some rows of a tile do not see: a probability of 0 is not enough there.  They are taken out of LDS,
// 16 bytes a lane, by the wavefront that has copied them; rows that see them get them behind the loop.  Returns whether there were any.
template <typename T>
__device__ __forceinline__ bool take_out(uint32_t lds) {
  u32x4 w = *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)lds;
  const bool found = not_finite<T>(w[0]) | not_finite<T>(w[1]) | not_finite<T>(w[2]) | not_finite<T>(w[3]);
  if (found) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = finite_part<T>(w[i]);
    *(__attribute__((address_space(3))) u32x4*)(uintptr_t)lds = w;
  }
  return found;
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// The reference that a part's results are joined by: of an undefined sum the largest, so that it is not lost beside others.
__device__ __forceinline__ float reference_of(float m, float l) { return l == l ? m : __builtin_inff(); }

// Four rows x 16 channels of 16 bits, a row by four lanes of 8 bytes, to the 16 lanes of a group: lane i gets channel i, row 0 first.
__device__ __forceinline__ u32x2 columns(uint32_t lds) {
  u32x2 r = {};
#if defined(__HIP_DEVICE_COMPILE__)
  r = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)lds));
#endif
  return r;
}
__device__ __forceinline__ u32x4 piece16(uint32_t lds) {
  return *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)lds;
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
__device__ __forceinline__ uint32_t token_of(const DenseArgs& a, uint32_t row) {   // row / group, exact below 2^31
  return a.group == 1 ? row : (__umulhi(row, a.by_group) + row) >> a.group_shift;
}

// ---- the list of work

struct Lengths {
  int q0, nq, kv0, nk;
};
__device__ __forceinline__ Lengths lengths_of(const DenseArgs& a, int s) {
  Lengths n;
  n.q0 = min(max(a.q_start[s], 0), a.q_rows);
  n.nq = max(min(max(a.q_start[s + 1], 0), a.q_rows) - n.q0, 0);
  n.kv0 = min(max(a.kv_start[s], 0), a.kv_rows);
  n.nk = a.kv_len ? min(max(a.kv_len[s], 0), a.kv_rows - n.kv0) : max(min(max(a.kv_start[s + 1], 0), a.kv_rows) - n.kv0, 0);
  return n;
}
__device__ __forceinline__ int keys_of_tile(const DenseArgs& a, const Lengths& n, int row0) {
  if (!a.causal) return n.nk;
  const int last = min((int)token_of(a, (uint32_t)row0 + a.tile - 1), n.nq - 1);
  return max(0, min(n.nk, (int)min((int64_t)last + 1 + n.nk - n.nq, (int64_t)n.nk)));
}

__device__ __forceinline__ int tiles_of(const DenseArgs& a, const Lengths& n) {
  return (int)(((int64_t)n.nq * a.group + a.tile - 1) / a.tile);
}
__device__ __forceinline__ int steps_of(const DenseArgs& a, int keys) { return (keys + a.keys - 1) / a.keys; }
// Tile t of a sequence; the last ones, which see the most keys, come first.
__device__ __forceinline__ DenseItem item_of(const DenseArgs& a, const Lengths& n, int tiles, int t) {
  DenseItem item = {n.q0, n.nq, n.kv0, n.nk, (a.causal ? tiles - 1 - t : t) * a.tile, 0, 0, -1};
  item.end = keys_of_tile(a, n, item.row0);
  return item;
}
// Part `part` of `parts` of an item, in whole steps.
__device__ __forceinline__ void take_part(const DenseArgs& a, DenseItem* item, int part, int parts, int slot) {
  if (parts == 1) return;
  const int64_t steps = steps_of(a, item->end);
  item->begin = (int)(steps * part / parts) * a.keys;
  item->end = min(item->end, (int)(steps * (part + 1) / parts) * a.keys);
  item->slot = slot;
}
// Steps of a part at least.  A part costs its start, its results and their joining: shorter ones than 256 keys lose.
__device__ __forceinline__ int least_steps(const DenseArgs& a) { return 256 / a.keys; }
// Parts of a tile: ceil(steps / chunk), but 64 at most, which is as many as are joined in a few us.
constexpr int MOST_PARTS = 64;
__device__ __forceinline__ int parts_of(const DenseArgs& a, int chunk, int keys) {
  return chunk == 0 ? 1 : min(MOST_PARTS, max(1, (steps_of(a, keys) + chunk - 1) / chunk));
}

// Steps of a part where tiles are cut, 0 where not: `tiles` and `steps` of all sequences, for each head of keys.  Uncut, the call lasts as long as the
// longest tile, or as its rounds of workgroups; cut, as a workgroup's share of the steps and the joining.  16 rows, which wait for memory: halves of a
// share, so that the workgroups end together (16 sequences of 1 to 8192 keys x 8 heads 123 us uncut, 51 in shares, 49.5 in halves; 16 x 3000 x 40 217, 220,
// 194; 400 tiles of 500 keys 30, 41, 40).  128 rows: a lone workgroup on a compute unit takes a third of the time a step that it takes
// beside two others, and results of parts are 64 KB (12000 rows, one head, 244 us uncut, 85 in shares, 106 in halves; 4096 x 12 108, 107, 117; 1024 x 40, not
// causal, 47, 58, 64; 6 x 700 x 12 40, 52, 53).
__device__ __forceinline__ int chunk_of(const DenseArgs& a, int64_t tiles, float steps, float longest) {
  const int64_t all = tiles * a.kv_heads;
  if (!a.may_split || all >= 2 * a.workgroups || tiles == 0) return 0;
  const bool rows = a.tile == 16;
  const float share = steps * (float)a.kv_heads / (float)a.workgroups, rounds = (float)((all + a.workgroups - 1) / a.workgroups);
  if (rows ? fmaxf(longest, rounds * steps / (float)tiles) <= 1.15f * share + 4.f : longest <= 3.f * share + 8.f) return 0;
  return max((int)ceilf(rows ? 0.5f * share : share), least_steps(a));
}

// Sum over this lane and those in front of it.
__device__ __forceinline__ int lanes_scan(int v) {
  auto moved = [](int x, auto ctrl, auto mask) { return __builtin_amdgcn_update_dpp(0, x, decltype(ctrl)::value, decltype(mask)::value, 0xF, false); };
  using std::integral_constant;
  v += moved(v, integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});   // row_shr 1, 2, 4, 8
  v += moved(v, integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});
  v += moved(v, integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});
  v += moved(v, integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});
  v += moved(v, integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});   // row_bcast 15 and 31
  v += moved(v, integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});
  return v;
}

// 64 sequences at most, one a lane: what the call's work is.  A tile is cut into ceil(steps / chunk) parts, and all tiles of a sequence have
// as many places as the longest of them has parts.
struct Work {
  Lengths n;
  int tiles, chunk, parts;   // chunk 0: nothing is cut
  int tiles_before, items_before;   // with this lane's own
};
__device__ __forceinline__ Work work_of_lane(const DenseArgs& a) {
  const int lane = threadIdx.x & 63;
  Work w = {};
  if (lane < a.sequences) w.n = lengths_of(a, lane), w.tiles = tiles_of(a, w.n);
  w.tiles_before = lanes_scan(w.tiles);
  w.parts = 1;
  w.items_before = w.tiles_before;
  const int all = __builtin_amdgcn_readlane(w.tiles_before, 63);
  if (!a.may_split || all < 0) return w;
  float steps = 0.f;   // of all tiles of the sequence: from the first one's to the last one's
  if (w.tiles > 0) steps = 0.5f * (float)w.tiles * ((float)steps_of(a, keys_of_tile(a, w.n, 0)) + (float)steps_of(a, w.n.nk));
  float longest = w.tiles > 0 ? (float)steps_of(a, w.n.nk) : 0.f;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) longest = fmaxf(longest, __shfl_xor(longest, d));
  w.chunk = chunk_of(a, all, wave_sum_f32(steps), longest);
  if (w.chunk == 0) return w;
  w.parts = parts_of(a, w.chunk, w.n.nk);
  w.items_before = lanes_scan(w.tiles * w.parts);
  return w;
}
__device__ __forceinline__ Lengths lengths_from(const Lengths& n, int lane) {
  return {__builtin_amdgcn_readlane(n.q0, lane), __builtin_amdgcn_readlane(n.nq, lane), __builtin_amdgcn_readlane(n.kv0, lane),
          __builtin_amdgcn_readlane(n.nk, lane)};
}
// Item `index` of the call, the same for all lanes; false: there is none.  Slots past the last one: starts that do not ascend.
__device__ __forceinline__ bool find_item(const DenseArgs& a, int index, DenseItem* item) {
  if (a.items) {
    if (index >= a.counts[0]) return false;
    *item = a.items[index];
    return true;
  }
  const Work w = work_of_lane(a);
  const uint64_t behind = __ballot(w.items_before > index);
  if (behind == 0) return false;
  const int s = __builtin_ctzll(behind), tiles = __builtin_amdgcn_readlane(w.tiles, s), places = __builtin_amdgcn_readlane(w.parts, s);
  const int chunk = __builtin_amdgcn_readfirstlane(w.chunk), first = __builtin_amdgcn_readlane(w.items_before, s) - tiles * places;
  const int tile = (index - first) / places, part = index - first - tile * places;
  *item = item_of(a, lengths_from(w.n, s), tiles, tile);
  const int parts = parts_of(a, chunk, item->end);
  if (part >= parts || (parts > 1 && index >= a.max_slots)) return false;
  take_part(a, item, part, parts, index);
  return true;
}
// Tile `index` of the call, if it was cut.
__device__ __forceinline__ bool find_merge(const DenseArgs& a, int index, DenseMerge* merge) {
  if (a.items) {
    if (index >= a.counts[1]) return false;
    *merge = a.merges[index];
    return true;
  }
  const Work w = work_of_lane(a);
  const uint64_t behind = __ballot(w.tiles_before > index);
  const int chunk = __builtin_amdgcn_readfirstlane(w.chunk);
  if (behind == 0 || chunk == 0) return false;
  const int s = __builtin_ctzll(behind), tiles = __builtin_amdgcn_readlane(w.tiles, s), places = __builtin_amdgcn_readlane(w.parts, s);
  const int tile = index - (__builtin_amdgcn_readlane(w.tiles_before, s) - tiles);
  const DenseItem item = item_of(a, lengths_from(w.n, s), tiles, tile);
  *merge = {item.q0, item.nq, item.row0, __builtin_amdgcn_readlane(w.items_before, s) - tiles * places + tile * places,
            parts_of(a, chunk, item.end), 0};
  return merge->parts > 1 && merge->slot >= 0 && merge->slot + merge->parts <= a.max_slots;
}

// Sum over the threads in front; *total: over all of them.
__device__ __forceinline__ int64_t scan(int64_t v, int64_t* room, int64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t x = __shfl_up(s, o);
    if (lane >= o) s += x;
  }
  __syncthreads();   // the room is free
  if (lane == 63) room[wave] = s;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int w = 0; w < 16; ++w) {
    if (w < wave) before += room[w];
    all += room[w];
  }
  *total = all;
  return before + s - v;
}
// The last of n ascending numbers that is not above x; the first one is not.
__device__ __forceinline__ int last_below(const int32_t* p, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ __launch_bounds__(1024) void dense_plan_kernel(DenseArgs a) {
  constexpr int IN_LDS = 4096;
  __shared__ int64_t room[16];
  __shared__ int32_t bins_here[IN_LDS];
  __shared__ int32_t of_tile[1024][2];   // parts, first slot
  __shared__ int32_t first_item[1024];
  const int tid = threadIdx.x;
  int32_t* bins = a.sequences <= IN_LDS ? bins_here : a.bins;
  int64_t tiles = 0, total;
  for (int s0 = 0; s0 < a.sequences; s0 += 1024) {
    const int s = s0 + tid;
    int64_t n = 0;
    if (s < a.sequences) n = ((int64_t)lengths_of(a, s).nq * a.group + a.tile - 1) / a.tile;
    const int64_t before = tiles + scan(n, room, &total);
    if (s < a.sequences) bins[s] = (int32_t)min(before, (int64_t)a.max_tiles);
    tiles += total;
  }
  __syncthreads();
  auto tile_at_index = [&](int j) {
    const int s = last_below(bins, a.sequences, j);
    const Lengths n = lengths_of(a, s);
    return item_of(a, n, tiles_of(a, n), j - bins[s]);
  };
  const int n_tiles = (int)min(tiles, (int64_t)a.max_tiles);   // more only where starts do not ascend
  // fewer tiles than may be cut, 1024 at most: their steps
  DenseItem mine = {};
  int steps = 0, chunk = 0;
  if (a.may_split && tiles * a.kv_heads < 2 * a.workgroups && n_tiles <= 1024) {
    if (tid < n_tiles) {
      mine = tile_at_index(tid);
      steps = steps_of(a, mine.end);
    }
    int64_t all;
    scan(steps, room, &all);
    float longest = (float)steps;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) longest = fmaxf(longest, __shfl_xor(longest, d));
    __syncthreads();
    if ((tid & 63) == 0) first_item[tid >> 6] = (int)longest;
    __syncthreads();
    for (int i = 0; i < 16; ++i) longest = fmaxf(longest, (float)first_item[i]);
    __syncthreads();
    chunk = chunk_of(a, n_tiles, (float)all, longest);
  }
  if (chunk == 0) {
    for (int j = tid; j < n_tiles; j += 1024) a.items[j] = tile_at_index(j);
    if (tid == 0) a.counts[0] = n_tiles, a.counts[1] = 0;
    return;
  }
  const int parts = tid < n_tiles ? parts_of(a, chunk, mine.end) : 0;
  int64_t n_items, n_slots, n_merges;
  const int item0 = (int)scan(parts, room, &n_items);
  const int slot0 = (int)scan(parts > 1 ? parts : 0, room, &n_slots);
  const int merge0 = (int)scan(parts > 1 ? 1 : 0, room, &n_merges);
  if (tid < n_tiles) {
    of_tile[tid][0] = parts;
    of_tile[tid][1] = slot0;
    first_item[tid] = item0;
    if (parts > 1) a.merges[merge0] = {mine.q0, mine.nq, mine.row0, slot0, parts, 0};
  }
  __syncthreads();
  for (int i = tid; i < n_items; i += 1024) {
    const int j = last_below(first_item, n_tiles, i), part = i - first_item[j];
    DenseItem item = tile_at_index(j);
    take_part(a, &item, part, of_tile[j][0], of_tile[j][1] + part);
    a.items[i] = item;
  }
  if (tid == 0) a.counts[0] = (int)n_items, a.counts[1] = (int)n_merges;
}

// ---- tiles of 128 rows

// What a lane's row is: its token's place in q and out, how many keys it sees.  Rows behind the last token are the tile's first row once more: what a row
// holds takes part in which way its wavefront goes on, and another tile's rows may be written over by then (out may be q).  (q = 0 for them, by a
// branch around the loads: 12000 rows x 8 heads fp16 344 -> 379 us.)
struct Row {
  int64_t token;   // of all
  int head, limit;
  bool there;
};
__device__ __forceinline__ Row row_at(const DenseArgs& a, const DenseItem& it, int kv_head, int row) {
  const int t = (int)token_of(a, (uint32_t)row), first = (int)token_of(a, (uint32_t)it.row0);
  Row r;
  r.there = t < it.nq;
  const int token = r.there ? t : first;
  r.head = kv_head * a.group + (r.there ? row : it.row0) - token * a.group;
  r.token = (int64_t)it.q0 + token;
  r.limit = a.causal ? (int)min((int64_t)token + 1 + it.nk - it.nq, (int64_t)it.end) : it.end;
  return r;
}

// The keys of a step as a buffer: what lies behind them reads as 0.
__device__ __forceinline__ u32x4 keys_of_step(const uint16_t* base, int64_t row_stride, int64_t first, int count, int D) {
  return buffer_of((const uint8_t*)(base + first * row_stride), (uint32_t)(((count - 1) * row_stride + D) * 2));
}

// ALIGNED: rows of k and v on the 16-byte grid, which the copies into LDS want.
//
// Bound by the matrix cores and the package power where sequences are long: nine causal prompts of 31 to 12000 tokens, 40 heads on 8 of keys, 2.05
// ms, 1.16 PFLOP/s (a bf16 product of the library 1.49); 4096 keys x 62400 rows x 12 heads 1.12, at D = 64 0.99.  Short ones read q and write out:
// 512 keys 219 us, of which 75 are that, with little of it under the products.  A step of 64 keys keeps S, P and O of 32 rows a wavefront in 168
// registers, three workgroups a compute unit.
//
// SUM_MAX: a step forms its probabilities against the reference as it stands and only looks at their sum.  While a lane's 32 add up to at
// most SUM_MAX, they and their float32 sums can be represented.  A sum above it, infinite or
// undefined sends the step down the exact path: logits again, the row's maximum, what has been added up rescaled, probabilities <= 1.  The first
// step of a row starts there, so the reference never exceeds the largest logit seen and the largest term is never lost to underflow.
//
// Sums of such probabilities times values can be represented, too, if the values are fp16, or bf16 below 2^70.  Where a tile of bf16 ends with one
// that is not finite it is made again, lifted: with references 2^32 above the maximum, probabilities <= 2^-32, a lane's sum of a step <= 2^-27 and the sum over
// 2^31 keys <= 1, so that what is added up stays below the largest value.  (Results below 2^-83 lose bits there, and tiles that see an infinity or a NaN take
// twice their time.)  The look at the sums costs 0.6 % of the nine prompts, 2.5 % of 512 keys, a microsecond of 40 of single tokens.
constexpr float LIFT = 32.0f, LIFTED_MAX = 7.450580596923828125e-09f;   // 2^-27
template <int N, typename V>
__device__ __forceinline__ bool any_not_finite(const V (&v)[N]) {   // times 0 these are NaN, others 0
  float sum[4] = {};
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < (int)(sizeof(V) / 4); ++e) sum[e & 3] = fmaf(v[i][e], 0.f, sum[e & 3]);
  return !((sum[0] + sum[1]) + (sum[2] + sum[3]) == 0.f);
}

template <typename T, int D, bool ALIGNED>
__global__ __launch_bounds__(256, D == 128 ? 3 : 4) void dense_tiles_kernel(DenseArgs a) {
  typedef typename Type<T>::eight eight;
  constexpr int KEYS = 64, KS = D / 16, DT = D / 32, MH = KEYS / 32, PH = KEYS / 16, CH = D / 8;
  constexpr int CHUNKS = KEYS * CH, COPIES = CHUNKS / 256, ROWS_PER_COPY = 256 / CH;
  __shared__ __attribute__((aligned(256))) u32x4 Ks[2 * CHUNKS];
  __shared__ int again;
  u32x4* Vs = Ks + CHUNKS;
  const int index = blockIdx.x / a.kv_heads, kv_head = blockIdx.x - index * a.kv_heads;
  DenseItem it;
  if (!find_item(a, index, &it)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hl = lane >> 5, ql = lane & 31;
  if (tid == 0) again = 0;
  int row = it.row0 + 32 * wave + ql;
  Row r = row_at(a, it, kv_head, row);
  // keys that all rows of the tile see
  const int first_token = (int)token_of(a, (uint32_t)it.row0);
  const int all_see = a.causal ? (int)min((int64_t)first_token + 1 + it.nk - it.nq, (int64_t)it.end) : it.end;

  eight qf[KS];
  {
    const uint16_t* qp = a.q + r.token * a.q_row + (int64_t)r.head * a.q_head + 8 * hl;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const Piece16 p = *(const Piece16*)(qp + 16 * ks);
      __builtin_memcpy(&qf[ks], &p, 16);
    }
  }

  // The 16-byte pieces of a row are rotated by an exclusive or on the way.  K: so that the 16 rows that are read at a time fall on different
  // banks.  V is read by columns, which hands a lane four keys of its channel: two of them are a fragment, in the key order of the accumulators.
  auto k_swizzle = [](int n) { return D == 128 ? n & 15 : (n >> 1) & 7; };
  auto v_swizzle = [](int n) { return D == 128 ? (n & 3) * 4 : (n & 2) * 2; };
  const int copy_row = tid / CH, copy_piece = tid % CH;
  const uint32_t k_from = (uint32_t)copy_row * (uint32_t)a.k_row * 2 + (copy_piece ^ k_swizzle(copy_row)) * 16;
  const uint32_t v_from = (uint32_t)copy_row * (uint32_t)a.v_row * 2 + (copy_piece ^ v_swizzle(copy_row)) * 16;
  const uint16_t *k0 = a.k + (int64_t)it.kv0 * a.k_row + kv_head * a.k_head, *v0 = a.v + (int64_t)it.kv0 * a.v_row + kv_head * a.v_head;
  const uint32_t ks_wave = lds_address(Ks) + wave * 1024, vs_wave = lds_address(Vs) + wave * 1024;
  auto copy = [&](const uint16_t* base, int64_t stride, uint32_t from, u32x4* to, uint32_t lds, int key) {
    const u32x4 rows = keys_of_step(base, stride, key, min(KEYS, it.end - key), D);
    if constexpr (ALIGNED) {
#pragma unroll
      for (int c = 0; c < COPIES; ++c) copy_1kb(rows, from, (uint32_t)(c * ROWS_PER_COPY) * (uint32_t)stride * 2, lds + c * 4096);
    } else {
#pragma unroll
      for (int c = 0; c < COPIES; ++c) {
        const int n = copy_row + c * ROWS_PER_COPY;
        Piece16 p = {};
        if (key + n < it.end) p = *(const Piece16*)((const uint8_t*)(base + (int64_t)key * stride) + from + (int64_t)c * ROWS_PER_COPY * stride * 2);
        to[tid + c * 256] = (u32x4){p.w[0], p.w[1], p.w[2], p.w[3]};
      }
    }
  };
  auto landed = []() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); };

  float m_run, l_run;
  bool unset, taken = false, lifted = false;
  f32x16 O[DT];
  auto restart = [&]() {
    uint32_t from = k_from;
    asm volatile("" : "+v"(from));   // addresses of its own: kept for both places they cost 8 registers more than there are
    if (it.begin < it.end) copy(k0, a.k_row, from, Ks, ks_wave, it.begin);
    m_run = r.limit > it.begin ? -__builtin_inff() : 0.f;   // 0: a row that sees none of these keys
    l_run = 0.f;
    unset = true;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) O[dt] = 0.f;
  };

  const uint32_t ks_lane = lds_address(Ks) + ql * (2 * D) + (hl ^ k_swizzle(ql)) * 16;
  const int v_row = 4 * hl + ((lane >> 2) & 3);
  const uint32_t vs_lane = lds_address(Vs) + v_row * (2 * D) + v_swizzle(v_row) * 16 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;

  restart();
  for (int key = it.begin; key < it.end; key += KEYS) {
    landed();
    __syncthreads();   // K of this step is in LDS; every wavefront is past the products of the step before
    copy(v0, a.v_row, v_from, Vs, vs_wave, key);
    const bool masked = key + KEYS > all_see;
    f32x16 S[MH];
    auto logits = [&]() {
#pragma unroll
      for (int m = 0; m < MH; ++m) S[m] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int m = 0; m < MH; ++m)
          S[m] = Type<T>::mul32(__builtin_bit_cast(eight, piece16((ks_lane ^ (ks * 32)) + m * 64 * D)), qf[ks], S[m]);
      if (masked) {
        const int left = r.limit - key - 4 * hl;
#pragma unroll
        for (int m = 0; m < MH; ++m)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (32 * m + 8 * (e / 4) + e % 4 >= left) S[m][e] = -__builtin_inff();
      }
    };
    eight pb[PH];
    auto probabilities = [&](float off) {
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int p = 0; p < PH; ++p) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p0 = exp2_of(fmaf(S[p >> 1][8 * (p & 1) + 2 * e], a.scale_log2e, off));
          const float p1 = exp2_of(fmaf(S[p >> 1][8 * (p & 1) + 2 * e + 1], a.scale_log2e, off));
          w[e] = Type<T>::pack(p0, p1);
          s0 += p0;
          s1 += p1;
        }
        pb[p] = __builtin_bit_cast(eight, w);
      }
      return s0 + s1;
    };
    float sum = 0.f;
    bool in_range = false;
    if (!unset) {
      logits();
      sum = probabilities(-m_run);
      in_range = __ballot(!(sum <= (lifted ? LIFTED_MAX : Type<T>::SUM_MAX))) == 0;
    }
    if (!in_range) {
      logits();
      float top = -__builtin_inff();
#pragma unroll
      for (int m = 0; m < MH; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, S[m][e]);
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m_run, fmaf(top, a.scale_log2e, lifted ? LIFT : 0.f));
      const float alpha = m_new == m_run ? 1.0f : exp2_of(m_run - m_new);
      l_run *= alpha;
      m_run = m_new;
      unset = __ballot(m_run == -__builtin_inff()) != 0;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) O[dt] *= alpha;
      sum = probabilities(m_run == -__builtin_inff() ? 0.f : -m_run);
    }
    l_run += sum;
    landed();
    if (masked && a.take_out) {
#pragma unroll
      for (int c = 0; c < COPIES; ++c) taken |= take_out<T>(vs_wave + c * 4096 + lane * 16);
    }
    __syncthreads();   // V is in LDS; every wavefront has read K
    if (key + KEYS < it.end) copy(k0, a.k_row, k_from, Ks, ks_wave, key + KEYS);
    auto v_fragment = [&](int dt, int p) {
      const uint32_t at = (vs_lane ^ (dt * 64)) + p * 32 * D;
      const u32x2 lo = columns(at), hi = columns(at + 16 * D);
      return (u32x4){lo[0], lo[1], hi[0], hi[1]};
    };
#pragma unroll
    for (int p = 0; p < PH; ++p)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) O[dt] = Type<T>::mul32(__builtin_bit_cast(eight, v_fragment(dt, p)), pb[p], O[dt]);
    if (Type<T>::WIDE && key + KEYS >= it.end && !lifted) {   // after the last step
      if (any_not_finite(O)) again = 1;
      __syncthreads();   // every wavefront has read K and V
      lifted = __builtin_amdgcn_readfirstlane(again);
      if (lifted) {
        restart();
        key = it.begin - KEYS;
      }
    }
  }
  if (a.take_out && __syncthreads_or(taken)) {   // what was taken out, to the rows that see it: it makes of a sum what it is itself
    for (int key = it.begin + max(all_see - it.begin, 0) / KEYS * KEYS; key < min(it.end, r.limit); ++key) {
      const T* v = (const T*)v0 + (int64_t)key * a.v_row + 4 * hl;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[dt][e] += rest_of(v[32 * dt + 8 * (e / 4) + e % 4]);
    }
  }

  // lane holds channels 32 dt + 8 g + 4 hl + 0..3 of its row
  const float l_all = l_run + __shfl_xor(l_run, 32);
  if (it.slot >= 0) {   // as they lie in the registers: whole kilobytes
    const int64_t at = ((int64_t)it.slot * a.kv_heads + kv_head) * 128 + 32 * wave;
    f32x4* o = (f32x4*)(a.part + at * D) + lane;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) o[(dt * 4 + g) * 64] = (f32x4){O[dt][4 * g], O[dt][4 * g + 1], O[dt][4 * g + 2], O[dt][4 * g + 3]};
    if (hl == 0) *(f32x2*)(a.stat + 2 * (at + ql)) = (f32x2){reference_of(m_run, l_all), l_all};
    return;
  }
  // Through LDS, so that a store takes whole rows: stored from here, 16 bytes of 32 rows at a time and through the caches, 62400
  // rows x 12 heads took 98 us for a single key instead of 75, which is what reading q and writing out takes.
  const float inv = l_all > 0.f ? 1.0f / l_all : l_all == 0.f ? 0.f : l_all;   // NaN stays
  if (!Type<T>::WIDE || lifted) __syncthreads();   // as above
  const uint32_t room = lds_address(Ks) + wave * (64 * D);   // 32 rows
  auto turned = [](int row) { return D == 128 ? row & 15 : row & 7; };
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const u32x2 w = {Type<T>::pack(O[dt][4 * g] * inv, O[dt][4 * g + 1] * inv), Type<T>::pack(O[dt][4 * g + 2] * inv, O[dt][4 * g + 3] * inv)};
      *(__attribute__((address_space(3))) u32x2*)(uintptr_t)(room + ql * (2 * D) + ((4 * dt + g) ^ turned(ql)) * 16 + hl * 8) = w;
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int n = lane / CH; n < 32; n += 64 / CH) {
    const Row to = row_at(a, it, kv_head, it.row0 + 32 * wave + n);
    const u32x4 w = piece16(room + n * (2 * D) + ((lane % CH) ^ turned(n)) * 16);
    if (to.there) {
      store_once(a.out + to.token * a.out_row + (int64_t)to.head * a.out_head + lane % CH * 8, make_uint4(w[0], w[1], w[2], w[3]));
    }
  }
}

// ---- tiles of 16 rows

constexpr int ROWS_WAVES = 2;

// Few rows: the keys are read once and are what takes the time.  Each wavefront takes 32 keys of every 32 x WAVES with LDS of its own,
// two steps deep, so that nothing but its own copies makes it wait; they join at the end.  Two wavefronts a workgroup, 64 KB of LDS at D = 128: 16
// sequences of 1 to 8192 keys x 8 heads 41.8 us and 6.6 to join, 4.6 TB/s; 64 x 2000 x 8, whole calls, 4.8 TB/s.  (Four a workgroup, one workgroup on a compute unit: 45.2.)
template <typename T, int D, bool ALIGNED>
__global__ __launch_bounds__(64 * ROWS_WAVES) void dense_rows_kernel(DenseArgs a) {
  typedef typename Type<T>::eight eight;
  constexpr int WAVES = ROWS_WAVES, KEYS = 32, KS = D / 32, DT = D / 16, CH = D / 8, BYTES = KEYS * D * 2, STAGES = 2;
  constexpr int COPIES = BYTES / 1024, ROWS_PER_COPY = 64 / CH;   // of a wavefront, for K
  constexpr int ROOM = STAGES * 2 * BYTES;                        // of a wavefront
  __shared__ __attribute__((aligned(256))) uint8_t tiles[WAVES * ROOM];
  __shared__ float stats[WAVES][16][2];
  static_assert(ROOM >= 16 * D * 4, "");
  const int index = blockIdx.x / a.kv_heads, kv_head = blockIdx.x - index * a.kv_heads;
  DenseItem it;
  if (!find_item(a, index, &it)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, i16 = lane & 15;
  const Row r = row_at(a, it, kv_head, it.row0 + i16);
  const int first_token = (int)token_of(a, (uint32_t)it.row0);
  const int all_see = a.causal ? (int)min((int64_t)first_token + 1 + it.nk - it.nq, (int64_t)it.end) : it.end;
  eight qf[KS];
  {
    const uint16_t* qp = a.q + r.token * a.q_row + (int64_t)r.head * a.q_head + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const Piece16 p = *(const Piece16*)(qp + 32 * ks);
      __builtin_memcpy(&qf[ks], &p, 16);
    }
  }
  auto k_swizzle = [](int n) { return D == 128 ? n & 15 : (n >> 1) & 7; };
  auto v_swizzle = [](int n) { return D == 128 ? (n & 3) * 4 : (n & 2) * 2; };
  const int copy_row = lane / CH, copy_piece = lane % CH;
  const uint16_t *k0 = a.k + (int64_t)it.kv0 * a.k_row + kv_head * a.k_head, *v0 = a.v + (int64_t)it.kv0 * a.v_row + kv_head * a.v_head;
  const uint32_t lds = lds_address(tiles) + wave * ROOM;
  auto copy = [&](const uint16_t* base, int64_t stride, auto swizzle, int key, uint32_t to) {
    const int left = it.end - key;
    const u32x4 rows = keys_of_step(base, stride, left > 0 ? key : it.begin, max(min(KEYS, left), 1), D);
#pragma unroll
    for (int c = 0; c < COPIES; ++c) {
      const int n = c * ROWS_PER_COPY;
      const uint32_t from = (uint32_t)copy_row * (uint32_t)stride * 2 + (copy_piece ^ swizzle(copy_row) ^ swizzle(n)) * 16;
      if constexpr (ALIGNED) {
        copy_1kb(rows, from, left > 0 ? (uint32_t)n * (uint32_t)stride * 2 : 0x80000000u, to + c * 1024);   // past the end: outside
      } else {
        Piece16 p = {};
        if (n + copy_row < left) p = *(const Piece16*)((const uint8_t*)(base + (int64_t)(key + n) * stride) + from);
        *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(to + c * 1024 + lane * 16) = (u32x4){p.w[0], p.w[1], p.w[2], p.w[3]};
      }
    }
  };
  auto copy_step = [&](int key, int stage) {
    copy(k0, a.k_row, k_swizzle, key, lds + stage * 2 * BYTES);
    copy(v0, a.v_row, v_swizzle, key, lds + stage * 2 * BYTES + BYTES);
  };
  float m_run, l_run;
  bool unset, taken = false, lifted = false;
  f32x4 O[DT];
  const uint32_t k_lane = i16 * (2 * D) + (g ^ k_swizzle(i16)) * 16;
  const int v_row = 4 * g + ((lane >> 2) & 3);
  const uint32_t v_lane = BYTES + v_row * (2 * D) + (((lane >> 1) & 1) ^ v_swizzle(v_row)) * 16 + (lane & 1) * 8;

  const int first_key = it.begin + KEYS * wave;
  // two turns that only copy, in front
  for (int key = first_key - 2 * WAVES * KEYS, stage = 0; key < it.end; key += WAVES * KEYS, stage ^= 1) {
    if (key < first_key) {
      m_run = r.limit > it.begin ? -__builtin_inff() : 0.f;
      l_run = 0.f;
      unset = true;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) O[dt] = 0.f;
    } else {
      asm volatile("s_waitcnt vmcnt(%0)" : : "n"(ALIGNED ? 2 * COPIES : 0) : "memory");
      const uint32_t at = lds + stage * 2 * BYTES;
      const bool masked = key + KEYS > all_see;
      if (masked && a.take_out) {
#pragma unroll
        for (int c = 0; c < COPIES; ++c) taken |= take_out<T>(at + BYTES + c * 1024 + lane * 16);
      }
      f32x4 S[2] = {};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int m = 0; m < 2; ++m)
          S[m] = Type<T>::mul16(__builtin_bit_cast(eight, piece16(at + (k_lane ^ (ks * 64)) + m * 32 * D)), qf[ks], S[m]);
      if (masked) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key + 16 * m + 4 * g + e >= r.limit) S[m][e] = -__builtin_inff();
      }
      eight pb;
      auto probabilities = [&](float off) {
        float s = 0.f;
        u32x4 w;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          float p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = exp2_of(fmaf(S[m][e], a.scale_log2e, off));
            s += p[e];
          }
          w[2 * m] = Type<T>::pack(p[0], p[1]);
          w[2 * m + 1] = Type<T>::pack(p[2], p[3]);
        }
        pb = __builtin_bit_cast(eight, w);
        return s;
      };
      float sum = 0.f;
      bool in_range = false;
      if (!unset) {
        sum = probabilities(-m_run);
        in_range = __ballot(!(sum <= (lifted ? LIFTED_MAX : Type<T>::SUM_MAX))) == 0;
      }
      if (!in_range) {
        float top = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])), fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3])));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m_run, fmaf(top, a.scale_log2e, lifted ? LIFT : 0.f));
        const float alpha = m_new == m_run ? 1.0f : exp2_of(m_run - m_new);
        l_run *= alpha;
        m_run = m_new;
        unset = __ballot(m_run == -__builtin_inff()) != 0;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) O[dt] *= alpha;
        sum = probabilities(m_run == -__builtin_inff() ? 0.f : -m_run);
      }
      l_run += sum;
      // channels 16 dt to + 15: pieces 2 dt and 2 dt + 1 of the row, before their rotation
      auto v_fragment = [&](int dt) {
        const uint32_t from = at + (v_lane ^ (dt * 32));
        const u32x2 lo = columns(from), hi = columns(from + 32 * D);
        return (u32x4){lo[0], lo[1], hi[0], hi[1]};
      };
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) O[dt] = Type<T>::mul16(__builtin_bit_cast(eight, v_fragment(dt)), pb, O[dt]);
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // this stage has been read
      if (Type<T>::WIDE && key + WAVES * KEYS >= it.end && !lifted && __ballot(any_not_finite(O)) != 0) {   // after the last step
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        lifted = true;
        key = first_key - 3 * WAVES * KEYS;
        continue;
      }
    }
    if (first_key < it.end) copy_step(key + 2 * WAVES * KEYS, stage);
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");   // nothing is on its way into LDS

  if (a.take_out && __ballot(taken) != 0) {   // what was taken out, to the rows that see it: it makes of a sum what it is itself
    for (int step = first_key; step < it.end; step += WAVES * KEYS) {
      if (step + KEYS <= all_see) continue;
      for (int j = step; j < min(min(step + KEYS, it.end), r.limit); ++j) {
        const T* v = (const T*)v0 + (int64_t)j * a.v_row + 4 * g;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) O[dt][e] += rest_of(v[16 * dt + e]);
      }
    }
  }

  // the wavefronts' results
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);
  if (lane < 16) stats[wave][i16][0] = reference_of(m_run, l_run), stats[wave][i16][1] = l_run;
  float* mine = (float*)(tiles + wave * ROOM) + i16 * D + 4 * g;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) *(f32x4*)(mine + 16 * dt) = O[dt];
  __syncthreads();
  constexpr int PER_ROW = 4 * WAVES, N = D / PER_ROW;   // threads of a row, channels of a thread
  const int row = tid / PER_ROW, c0 = tid % PER_ROW * N;
  const Row to = row_at(a, it, kv_head, it.row0 + row);
  if (!to.there) return;
  float m_all = -__builtin_inff(), l_all = 0.f, o[N] = {};
#pragma unroll
  for (int w = 0; w < WAVES; ++w)
    if (stats[w][row][1] != 0.f) m_all = fmaxf(m_all, stats[w][row][0]);   // NaN is not 0
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const float l = stats[w][row][1];
    if (l == 0.f) continue;
    const float by = exp2_of(stats[w][row][0] - m_all) * (1.0f / WAVES);   // so that the sum of finite results is finite
    l_all = fmaf(l, by, l_all);
    const float* from = (const float*)(tiles + w * ROOM) + row * D + c0;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = fmaf(from[i], by, o[i]);
  }
  if (it.slot >= 0) {
    const int64_t n = ((int64_t)it.slot * a.kv_heads + kv_head) * 16 + row;
#pragma unroll
    for (int i = 0; i < N; i += 4) *(f32x4*)(a.part + n * D + c0 + i) = (f32x4){o[i], o[i + 1], o[i + 2], o[i + 3]};
    if (tid % PER_ROW == 0) a.stat[2 * n] = l_all == 0.f ? 0.f : m_all, a.stat[2 * n + 1] = l_all;
    return;
  }
  const float inv = l_all > 0.f ? 1.0f / l_all : l_all == 0.f ? 0.f : l_all;
  T* out = (T*)a.out + to.token * a.out_row + (int64_t)to.head * a.out_head + c0;
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = (T)(o[i] * inv);
}

// ---- joining

// Tiles of 16 rows: a wavefront a row, a lane looks at a part's reference and sum, 64 of them at a time, then groups of lanes with four
// channels each take a part each.
template <typename T, int D>
__global__ __launch_bounds__(256) void dense_merge_rows_kernel(DenseArgs a) {
  constexpr int TILE = 16, LANES = D / 4, GROUPS = 64 / LANES, BLOCKS = TILE / 4;
  const int block = blockIdx.x % BLOCKS, of = blockIdx.x / BLOCKS, index = of / a.kv_heads, kv_head = of - index * a.kv_heads;
  DenseMerge it;
  if (!find_merge(a, index, &it)) return;
  const int lane = threadIdx.x & 63, row = 4 * block + (threadIdx.x >> 6), group = lane / LANES, c = lane % LANES * 4;
  const uint32_t t = token_of(a, (uint32_t)(it.row0 + row));
  if ((int)t >= it.nq) return;
  const int64_t first = ((int64_t)it.slot * a.kv_heads + kv_head) * TILE + row, step = (int64_t)a.kv_heads * TILE;
  float top = -__builtin_inff(), l = 0.f;
  f32x4 o = 0.f;
  for (int p0 = 0; p0 < it.parts; p0 += 64) {
    float m = 0.f, sum = 0.f;
    if (p0 + lane < it.parts) {
      const float2 s = *(const float2*)(a.stat + 2 * (first + step * (p0 + lane)));
      m = s.x;
      sum = s.y;
    }
    float top_here = sum != 0.f ? m : -__builtin_inff();   // NaN is not 0
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top_here = fmaxf(top_here, __shfl_xor(top_here, d));
    const float top_new = fmaxf(top, top_here), alpha = top_new == top ? 1.0f : exp2_of(top - top_new);
    const float weight = sum != 0.f ? exp2_of(m - top_new) * (1.0f / MOST_PARTS) : 0.f;   // so that the sum of finite results is finite
    top = top_new;
    l = l * alpha + wave_sum_f32(sum * weight);
    o *= alpha;
    const int n = min(64, it.parts - p0);
    // Four at a time; past the last one it again, and not taken.  The turns are the same for all lanes: a lane that had no part left and was out of the
    // loop would hand its weight, of a part that another group takes, to nobody.
    for (int q0 = 0; q0 < n; q0 += 4 * GROUPS) {
      const int q = q0 + group;
      f32x4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *(const f32x4*)(a.part + (first + step * (p0 + min(q + i * GROUPS, n - 1))) * D + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float w = __shfl(weight, min(q + i * GROUPS, 63));   // weights past the last part are 0
        if (w != 0.f && q + i * GROUPS < n) o += x[i] * w;
      }
    }
  }
#pragma unroll
  for (int d = LANES; d < 64; d <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], d);
  if (group != 0) return;
  const float inv = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l;
  const int head = kv_head * a.group + it.row0 + row - (int)t * a.group;
  T* out = (T*)a.out + ((int64_t)it.q0 + t) * a.out_row + (int64_t)head * a.out_head + c;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (T)(o[e] * inv);
}

// Tiles of 128 rows: a workgroup for 32 of them and 32 channels; a lane has a row and four of the channels.
template <typename T, int D>
__global__ __launch_bounds__(256) void dense_merge_tiles_kernel(DenseArgs a) {
  constexpr int TILE = 128, BLOCKS = 4 * (D / 32);
  const int block = blockIdx.x % BLOCKS, of = blockIdx.x / BLOCKS, index = of / a.kv_heads, kv_head = of - index * a.kv_heads;
  DenseMerge it;
  if (!find_merge(a, index, &it)) return;
  const int lane = threadIdx.x & 63, wave = block & 3, unit = block / 4 * 4 + (threadIdx.x >> 6), row = 32 * wave + (lane & 31);
  const int64_t first = ((int64_t)it.slot * a.kv_heads + kv_head) * TILE + 32 * wave, step = (int64_t)a.kv_heads * TILE;
  const f32x2* stat = (const f32x2*)a.stat + first + (lane & 31);
  const f32x4* part = (const f32x4*)(a.part + first * D) + unit * 64 + lane;
  float top = -__builtin_inff(), l = 0.f;
  // four parts at a time; past the last one it again, and not taken
  for (int p = 0; p < it.parts; p += 4) {
    f32x2 s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = stat[step * min(p + i, it.parts - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, s[i][1] != 0.f ? s[i][0] : -__builtin_inff());   // NaN is not 0
  }
  f32x4 o = 0.f;
  for (int p = 0; p < it.parts; p += 4) {
    f32x2 s[4];
    f32x4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = stat[step * min(p + i, it.parts - 1)];
      x[i] = part[step * min(p + i, it.parts - 1) * (D / 4)];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float weight = s[i][1] != 0.f && p + i < it.parts ? exp2_of(s[i][0] - top) * (1.0f / MOST_PARTS) : 0.f;
      if (weight != 0.f) {
        l = fmaf(s[i][1], weight, l);
        o += x[i] * weight;
      }
    }
  }
  const uint32_t t = token_of(a, (uint32_t)(it.row0 + row));
  if ((int)t >= it.nq) return;
  const float inv = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l;
  const int head = kv_head * a.group + it.row0 + row - (int)t * a.group;
  T* out = (T*)a.out + ((int64_t)it.q0 + t) * a.out_row + (int64_t)head * a.out_head + 8 * unit + 4 * (lane >> 5);
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = (T)(o[e] * inv);
}

int status() { return hipGetLastError() == hipSuccess ? JENGA_OK : JENGA_EHIP; }

template <typename T, int D, bool ALIGNED>
int run(const DenseArgs& a, const DenseShape& s, hipStream_t st) {
  const unsigned grid = (unsigned)(s.items * a.kv_heads), merges = (unsigned)(s.split_tiles * a.kv_heads);
  if (a.items) dense_plan_kernel<<<1, 1024, 0, st>>>(a);
  if (s.rows == 16) {
    dense_rows_kernel<T, D, ALIGNED><<<grid, 64 * ROWS_WAVES, 0, st>>>(a);
    if (s.may_split) dense_merge_rows_kernel<T, D><<<4 * merges, 256, 0, st>>>(a);
  } else {
    dense_tiles_kernel<T, D, ALIGNED><<<grid, 256, 0, st>>>(a);
    if (s.may_split) dense_merge_tiles_kernel<T, D><<<D / 8 * merges, 256, 0, st>>>(a);
  }
  return status();
}

}  // namespace

extern "C" {

int jenga_dense_attn(const jenga_dense_config* cfg, const void* q, const void* k, const void* v, const int32_t* q_start,
                     const int32_t* kv_start, const int32_t* kv_len_or_null, void* out, void* workspace, size_t workspace_bytes,
                     void* stream) {
  const int why = jenga::dense_args_ok(cfg, q, k, v, q_start, kv_start, kv_len_or_null, out, workspace, workspace_bytes);
  if (why != JENGA_OK) return why;
  if (cfg->q_rows == 0 || cfg->sequences == 0) return JENGA_OK;
  const DenseShape s = jenga::dense_shape(*cfg);
  const jenga_dense_config& c = *cfg;
  DenseArgs a = {};
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k;
  a.v = (const uint16_t*)v;
  a.out = (uint16_t*)out;
  a.q_start = q_start;
  a.kv_start = kv_start;
  a.kv_len = kv_len_or_null;
  a.q_row = c.q_row;
  a.q_head = c.q_head;
  a.k_row = c.k_row;
  a.k_head = c.k_head;
  a.v_row = c.v_row;
  a.v_head = c.v_head;
  a.out_row = c.out_row;
  a.out_head = c.out_head;
  a.q_rows = (int32_t)c.q_rows;
  a.kv_rows = (int32_t)c.kv_rows;
  a.sequences = c.sequences;
  a.kv_heads = c.kv_heads;
  a.group = c.heads / c.kv_heads;
  int l = 0;
  while ((1ll << l) < a.group) ++l;
  a.group_shift = (uint32_t)l;
  a.by_group = (uint32_t)((((1ull << l) - (uint64_t)a.group) << 32) / (uint64_t)a.group + 1);
  a.causal = (c.flags & JENGA_DENSE_CAUSAL) != 0;
  a.take_out = a.causal || c.v_row < c.head_dim;   // rows over each other: behind the last key's value lie others, not zeros
  a.scale_log2e = c.scale * 1.4426950408889634f;
  a.tile = s.rows;
  a.keys = s.rows == 16 ? 32 * ROWS_WAVES : 64;
  a.max_tiles = (int32_t)s.tiles;
  a.max_slots = (int32_t)s.slots;
  a.workgroups = (int32_t)s.workgroups;
  a.may_split = s.may_split;
  uint8_t* ws = (uint8_t*)workspace;
  a.counts = (int32_t*)ws;
  a.bins = (int32_t*)(ws + s.bins_at);
  a.items = s.listed ? (DenseItem*)(ws + s.items_at) : nullptr;
  a.merges = (DenseMerge*)(ws + s.merge_at);
  a.stat = (float*)(ws + s.stat_at);
  a.part = (float*)(ws + s.part_at);
  hipStream_t st = (hipStream_t)stream;
  const bool aligned = (((uintptr_t)k | (uintptr_t)v) & 15) == 0 && (c.k_row | c.k_head | c.v_row | c.v_head) % 8 == 0;
#define JENGA_DENSE(T)                                                                                     \
  return c.head_dim == 128 ? (aligned ? run<T, 128, true>(a, s, st) : run<T, 128, false>(a, s, st))  \
                           : (aligned ? run<T, 64, true>(a, s, st) : run<T, 64, false>(a, s, st))
  if (c.type == JENGA_BF16) JENGA_DENSE(__bf16);
  JENGA_DENSE(_Float16);
#undef JENGA_DENSE
}

}  // extern "C"
