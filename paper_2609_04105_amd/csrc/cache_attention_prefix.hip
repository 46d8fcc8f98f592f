// The pass over a prefix that the sequences of a batch share: the rows of all sequences together, each piece of the
// prefix by itself.
//
// Of every row and piece it leaves (m, l, a) = (a reference, sum 2^(y - m), sum 2^(y - m) V), from which the waves of the row's
// own pass begin (add_piece in cache_attention.hpp): partial states join in any order, a = a_1 2^(m_1 - m) + a_2 2^(m_2 - m).
// With many rows the kernels that it is built from bound it.  Medians of traced launches, 8 key heads, d = 128: 248 rows a key head
// behind 8192 keys in MXFP4 21.5 us, 387 TFLOP/s; 768 behind 65536 keys in MXFP8 301, 684.
#include "cache_attention_rows.hpp"
#include "cache_attention_tiles.hpp"

namespace fp4attn {

hipError_t launch_prefix_attention(const PrefixAttentionArgs& a, const CachePlan& plan, hipStream_t stream) {
  for_format(a.c, [&](auto d, auto fp8) {
    if (plan.tile == kRowsTile) launch_rows<d(), fp8()>(a, plan, stream);
    else launch_tiles<d(), fp8()>(a, plan, stream);
  });
  return hipGetLastError();
}

}  // namespace fp4attn
