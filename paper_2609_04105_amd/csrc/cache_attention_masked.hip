// Attention over the cache with a window or a prefix mask, or behind a shared prefix.
//
// The kernels of cache_attention_tiles.hpp and cache_attention_rows.hpp; a row tile behind a window walks the units of 128 keys that its rows
// see, the longest of them deciding how many places of the line (cache_attention.hpp) a row tile of the sequence has.
// Measured, 8 key heads of 4 query heads, d = 128, MXFP4: 8 tokens behind a window of 4096 keys 17.1 to 17.7 us at 8192 to
// 131072 keys, of sequences of 4096 keys without one 16.4; 64 tokens behind 1024 keys 15.7 for 14.9.  (The kernels for capped and biased
// scores take up to 6 % longer for these where registers are short: chunks behind a window 124 us, here 116.)
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
