// Test driver for the argument checks of jenga_rotary (CPU only; a call that passes them would launch).  Reads calls from stdin, one per
// line, and prints the status of each:
//     T H W head_dim dim0 dim1 dim2 type batch tokens count, then for each tensor src dst heads and the six strides
// With the argument "tiles" the lines are products, m n and whether the result is float32, and the output is what matmul_tiles() says:
// rows, tile, LDS tiles, workgroups a compute unit.
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "jenga_internal.h"

static int tiles() {
  long long m, n;
  int float32;
  while (std::scanf("%lld %lld %d", &m, &n, &float32) == 3) {
    const jenga::MatmulTiles t = jenga::matmul_tiles(m, n, float32 != 0);
    std::printf("%d %d %d %d %d\n", t.rows, t.bm, t.bn, t.stages, t.per_cu);
  }
  return 0;
}

int main(int argc, char** argv) {
  if (argc > 1 && std::strcmp(argv[1], "tiles") == 0) return tiles();
  jenga_rotary_config c = {};
  c.theta = 10000.0;
  c.step[0] = c.step[1] = c.step[2] = 1.0;
  long long batch, tokens;
  int count;
  while (std::scanf("%d %d %d %d %d %d %d %d %lld %lld %d", &c.T, &c.H, &c.W, &c.head_dim, &c.dim[0], &c.dim[1], &c.dim[2], &c.type,
                    &batch, &tokens, &count) == 11) {
    jenga_rotary_tensor t[2] = {};
    for (int i = 0; i < count && i < 2; ++i) {
      long long src, dst, s[6];
      int heads;
      if (std::scanf("%lld %lld %d %lld %lld %lld %lld %lld %lld", &src, &dst, &heads, s, s + 1, s + 2, s + 3, s + 4, s + 5) != 9) return 1;
      t[i] = {(const void*)(uintptr_t)src, (void*)(uintptr_t)dst, s[0], s[1], s[2], s[3], s[4], s[5], heads, 0};
    }
    std::printf("%d\n", jenga::rotary_args_ok(&c, nullptr, nullptr, (const float*)(uintptr_t)8, t, count, batch, tokens));
  }
  return 0;
}
