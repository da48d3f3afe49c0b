// What the tiled products share: copies from global memory straight into LDS, stores past the caches, and the order of the tiles.
#pragma once
#include "jenga_device.h"

namespace jenga {

// 64 lanes x 16 (or 4) bytes from global memory straight into 1 KB (256 bytes) of LDS, complete when vmcnt says so.
__device__ __forceinline__ uint64_t uniform(const uint8_t* p) {
  const uint64_t b = (uint64_t)p;
  return (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
}
// The rows of an operand that a tile has, as a buffer: what lies behind them reads as 0.  The range check is on the sum of the vector and
// the scalar offset, also where the latter alone is past the end (every 4 bytes of 64 lanes, scalar offsets up to 2^31).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4 buffer_of(const uint8_t* base, uint32_t bytes) {
  const uint64_t b = uniform(base);
  return (u32x4){(uint32_t)b, (uint32_t)(b >> 32), (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};   // raw, 32-bit elements
}
__device__ __forceinline__ void copy_1kb(const u32x4& buffer, uint32_t lane_offset, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(lane_offset), "s"(buffer), "s"(offset)
               : "memory", "m0");
}
// 64 lanes x 4 bytes, or nothing: without a branch, which would part the products from the reads and copies between them.
__device__ __forceinline__ void copy_256b(bool wanted, const uint8_t* base, uint32_t lane_offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b64 exec, -1"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(lane_offset), "s"(uniform(base)), "s"(__builtin_amdgcn_readfirstlane(wanted ? -1 : 0))
               : "memory", "m0");
}

// 16 bytes to any address that is a multiple of two, not to be kept in the caches.
typedef uint32_t u32x4_at_2 __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void store_once(void* to, const uint4& v) {
  __builtin_nontemporal_store((u32x4_at_2){v.x, v.y, v.z, v.w}, (u32x4_at_2*)to);
}

// Tile t of all.  Workgroups are dealt round-robin to the 8 XCDs; each XCD gets a run of neighbouring tiles, in stripes of 8 tiles along m,
// so that what runs on it at a time reads few rows of either operand.
__device__ __forceinline__ void tile_at(int t, int tiles_m, int tiles_n, int* tm, int* tn) {
  const int stripe = t / (8 * tiles_n), high = min(8, tiles_m - 8 * stripe), in = t - stripe * 8 * tiles_n;
  *tn = in / high;
  *tm = stripe * 8 + in - *tn * high;
}

}  // namespace jenga
