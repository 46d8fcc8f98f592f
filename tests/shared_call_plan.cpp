// Prints for each line of standard input "B heads query_heads_per_head d fp8 max_q tokens max_keys shared" the plan of an attention
// call with that many keys in common: "shared prefix_tile pieces rows, tile row_tiles split ranges min_units fits direct
// direct_units workgroups workspace".
#include <cstdio>

#include "../paper_2609_04105_amd/csrc/cache_plan.hpp"

int main() {
  long long B, H, G, d, fp8, max_q, n, keys, shared;
  while (std::scanf("%lld %lld %lld %lld %lld %lld %lld %lld %lld", &B, &H, &G, &d, &fp8, &max_q, &n, &keys, &shared) == 9) {
    const fp4attn::CachePlan plan = fp4attn::cache_plan(B, H, G, d, fp8 != 0, max_q, keys);
    const fp4attn::SharedPlan s = fp4attn::shared_plan(plan, B, H, G, d, fp8 != 0, max_q, n, keys, shared);
    const fp4attn::CachePlan& p = s.plan;
    std::printf("%lld %d %d %lld %d %d %d %d %d %d %d %d %lld %lld\n", (long long)s.shared, s.prefix.plan.tile, s.prefix.pieces,
                (long long)s.prefix.rows, p.tile, p.row_tiles, p.split, p.ranges, p.min_units, p.fits, p.direct, p.direct_units,
                (long long)p.workgroups, (long long)p.workspace);
  }
  return 0;
}
