// Attention over the cache with capped or biased scores, under any mask, also behind a shared prefix.
#include "cache_attention_rows.hpp"
#include "cache_attention_tiles.hpp"

namespace fp4attn {

hipError_t launch_shaped_attention(const ShapedAttentionArgs& a, const CachePlan& plan, hipStream_t stream) {
  for_format(a.c, [&](auto d, auto fp8) {
    if (plan.tile == kRowsTile) launch_rows<d(), fp8()>(a, plan, stream);
    else launch_tiles<d(), fp8()>(a, plan, stream);
    if (plan.split) launch_join<d(), fp8()>(a, plan, stream);
  });
  return hipGetLastError();
}

}  // namespace fp4attn
