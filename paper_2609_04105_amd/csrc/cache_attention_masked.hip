// Attention over the cache with a window or a prefix mask, or behind a shared prefix.  (The kernels for capped and biased
// scores take up to 6 % longer for these where registers are short: chunks behind a window 124 us, here 117.)
#include "cache_attention_rows.hpp"
#include "cache_attention_tiles.hpp"

namespace fp4attn {

hipError_t launch_masked_attention(const MaskedAttentionArgs& a, const CachePlan& plan, hipStream_t stream) {
  for_format(a.c, [&](auto d, auto fp8) {
    if (plan.tile == kRowsTile) launch_rows<d(), fp8()>(a, plan, stream);
    else launch_tiles<d(), fp8()>(a, plan, stream);
    if (plan.split) launch_join<d(), fp8()>(a, plan, stream);
  });
  return hipGetLastError();
}

}  // namespace fp4attn
