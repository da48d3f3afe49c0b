// Test driver for the argument checks of jenga_rotary (CPU only; a call that passes them would launch).  Reads calls from stdin, one per
// line, and prints the status of each:
//     T H W head_dim dim0 dim1 dim2 type batch tokens count, then for each tensor src dst heads and the six strides
#include <cstdint>
#include <cstdio>

#include "jenga_internal.h"

int main() {
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
