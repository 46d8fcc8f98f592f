// Attention over the cache with capped or biased scores, under any mask, also behind a shared prefix.
//
//   O_r = sum_j p_rj V_j / sum_j p_rj,  p_rj = exp(c tanh(s q_r . K_j / c) - slope_r |place_r - j|)
//
// The kernels of cache_attention_tiles.hpp and cache_attention_rows.hpp with their scores replaced between the two products; what
// bounds them is as there, and the vector unit sooner: the cap takes seven instructions a score, a bias two (three with a prefix mask).
// Measured, 8 key heads of 4 query heads, d = 128, MXFP4: one token of 700 keys 8.9 us, with a cap 10.6, with slopes 11.0;
// 838 row tiles of 128 rows behind a window of 1024 keys 116, with a cap 144, with slopes 143, with both 158 (MXFP8 108, 143, 146, 154); MXFP8,
// 4 key heads of 8 query heads, 48 tokens of up to 16384 keys 48.5 us, with slopes 52.1.  The 128-row kernels hold more than the registers:
// with d = 128 the compiler spills 20 (MXFP4) and 50 (MXFP8), for the second in the loop over the keys.
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
