// The block means that the selection reads: their arithmetic and their place in its workspace.
#pragma once
#include <hip/hip_runtime.h>

#include "jenga_internal.h"

namespace jenga {

__device__ inline double bf16_bits_to_double(uint32_t bits16) {
  return (double)__uint_as_float(bits16 << 16);
}

// Where channel d of block j lies in its pooled row: pieces of 64 bytes, their order rotated by an exclusive or with the
// block index.  select_kernel reads the same piece of 16 consecutive blocks at a time; without the rotation those lie
// a row (1 KB at D = 128) apart and fall on a quarter of the L2's channels (the products of 929 x 931 blocks x 24 heads:
// 175 us without it, 105 us with).
template <int D>
__device__ inline int pooled_pos(int j, int d) {
  return ((((d >> 3) ^ j) & (D / 8 - 1)) << 3) | (d & 7);
}

// Where the pooled rows of Q and K lie in the workspace.
template <int D>
void pooled_rows(const jenga_plan* p, void* ws, double** qh, double** kh) {
  const size_t q_bytes = (size_t)p->cfg.batch * p->cfg.heads * p->info.M_v * D * 8;
  *qh = (double*)ws;
  *kh = (double*)((char*)ws + ((q_bytes + 255) & ~(size_t)255));
}

}  // namespace jenga
