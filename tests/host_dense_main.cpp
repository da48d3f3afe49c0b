// Test driver for the sizes of dense attention's launches (CPU only).  Reads configurations from stdin, one per line,
//     q_rows kv_rows sequences heads kv_heads head_dim
// and prints what dense_shape() says of each: rows of a tile, workgroups, whether tiles may be cut, whether there is a list; tiles, items, slots and cut tiles at
// most; where the parts of the workspace begin, and its end.
#include <cstdio>

#include "jenga_internal.h"

int main() {
  jenga_dense_config c = {};
  long long q, kv;
  while (std::scanf("%lld %lld %d %d %d %d", &q, &kv, &c.sequences, &c.heads, &c.kv_heads, &c.head_dim) == 6) {
    c.q_rows = q;
    c.kv_rows = kv;
    const jenga::DenseShape s = jenga::dense_shape(c);
    std::printf("%d %lld %d %d %lld %lld %lld %lld %llu %llu %llu %llu %llu %llu\n", s.rows, (long long)s.workgroups, s.may_split, s.listed, (long long)s.tiles,
                (long long)s.items, (long long)s.slots, (long long)s.split_tiles, (unsigned long long)s.bins_at, (unsigned long long)s.items_at,
                (unsigned long long)s.merge_at, (unsigned long long)s.stat_at, (unsigned long long)s.part_at, (unsigned long long)s.workspace);
  }
  return 0;
}
