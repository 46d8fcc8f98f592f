// Attention over the cache as it stands: causal, or a tree of drafted tokens.
#include "cache_attention_rows.hpp"
#include "cache_attention_tiles.hpp"

namespace fp4attn {

hipError_t launch_cache_attention(const CacheAttentionArgs& a, const CachePlan& plan, hipStream_t stream) {
  for_format(a.c, [&](auto d, auto fp8) {
    if (plan.tile == kRowsTile) launch_rows<d(), fp8()>(a, plan, stream);
    else launch_tiles<d(), fp8()>(a, plan, stream);
    if (plan.split) launch_join<d(), fp8()>(a, plan, stream);
  });
  return hipGetLastError();
}

}  // namespace fp4attn
