// Prints the plan of an attention call over the cache ("tile row_tiles tile_rows split ranges min_units
// fits workgroups workspace") for each line of standard input:
//   B heads query_heads_per_head d fp8 max_q max_keys
#include <cstdio>

#include "../paper_2609_04105_amd/csrc/cache_plan.hpp"

int main() {
  long long B, H, G, d, fp8, max_q, max_keys;
  while (std::scanf("%lld %lld %lld %lld %lld %lld %lld", &B, &H, &G, &d, &fp8, &max_q, &max_keys) == 7) {
    const fp4attn::CachePlan p = fp4attn::cache_plan(B, H, G, d, fp8 != 0, max_q, max_keys);
    std::printf("%d %d %d %d %d %d %d %lld %lld\n", p.tile, p.row_tiles, p.tile_rows, p.split, p.ranges, p.min_units, p.fits,
                (long long)p.workgroups, (long long)p.workspace);
  }
  return 0;
}
