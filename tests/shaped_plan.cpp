// Prints for each line of standard input "P heads query_heads_per_head d tokens keys" the plan of the pass over a
// shared prefix ("tile row_tiles pieces units ranges workgroups rows fits"), for "W tile query_heads_per_head
// window" the units that a row tile may touch.
#include <cstdio>

#include "../paper_2609_04105_amd/csrc/cache_plan.hpp"

int main() {
  char what;
  long long x[5];
  while (std::scanf(" %c", &what) == 1) {
    const int n = what == 'P' ? 5 : 3;
    for (int i = 0; i < n; ++i)
      if (std::scanf("%lld", &x[i]) != 1) return 1;
    if (what == 'W') {
      std::printf("%d\n", fp4attn::window_units((int)x[0], (int)x[1], (int)x[2]));
    } else {
      const fp4attn::PrefixPlan p = fp4attn::prefix_plan(x[0], x[1], x[2], x[3], x[4]);
      std::printf("%d %d %d %d %d %lld %lld %d\n", p.plan.tile, p.plan.row_tiles, p.pieces, p.units, p.plan.ranges,
                  (long long)p.plan.workgroups, (long long)p.rows, p.fits);
    }
  }
  return 0;
}
