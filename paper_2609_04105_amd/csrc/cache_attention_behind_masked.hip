// Attention behind a shared prefix for batches whose members may end inside it: scores as they are.
//
// The kernels of cache_attention_tiles.hpp and cache_attention_rows.hpp, which beside a range for every row tile have others for the rest
// of row tiles of long sequences (own_plan in cache_plan.hpp, which has the figures).  They are kernels of their own: what they hold of their
// piece costs scalar registers, and one token of 700 keys with a cap took 11.5 us instead of 10.8, chunks behind a window 150
// instead of 144.
#include "cache_attention_rows.hpp"
#include "cache_attention_tiles.hpp"

namespace fp4attn {

hipError_t launch_masked_behind(const MaskedBehindArgs& a, const CachePlan& plan, hipStream_t stream) {
  for_format(a.c, [&](auto d, auto fp8) {
    if (plan.tile == kRowsTile) launch_rows<d(), fp8()>(a, plan, stream);
    else launch_tiles<d(), fp8()>(a, plan, stream);
  });
  return hipGetLastError();
}

}  // namespace fp4attn
