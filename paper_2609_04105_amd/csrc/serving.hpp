// Host-side launchers of the operators around a key/value cache:
// rotary positions, the cache's quantizer and reader, attention over it.  Arguments
// are already validated by the C-ABI layer (api.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fp4attn {

struct RotaryArgs {
  const void* x;
  void* out;
  int64_t B, H, N;
  int64_t xb, xh, xn, ob, oh, on;  // strides in elements; d is contiguous
  int d, r;                        // r: rotated channels
  const int64_t* positions;        // (b, n) at b * pos_stride + n
  int64_t pos_stride;
  const double* inv_freq;          // [r / 2] radians per position
  float magnitude;
  int bf16, interleaved, inverse;
};

constexpr int kRotaryMaxDim = 512;

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream);

// The paged cache (layouts in include/fp4attn.h); page_size is a power of two >= 16.
struct CacheView {
  uint8_t* k_codes;
  uint8_t* k_scales;
  uint8_t* v_codes;
  uint8_t* v_scales;
  int64_t pages;
  int page_limit;  // page numbers below it (they are 32-bit in a page table) are in the cache
  int H, d, page_shift, fp8;
};

struct CacheWriteArgs {
  CacheView c;
  const void* k;
  const void* v;
  int64_t n, k_stride, v_stride;  // strides of a token in elements; [H, d] contiguous
  const int64_t* slots;
  int bf16;
};

struct CacheReadArgs {
  CacheView c;
  int64_t n;
  const int64_t* slots;
  void* k;
  void* v;
  int bf16;
};

hipError_t launch_cache_write(const CacheWriteArgs& a, hipStream_t stream);
hipError_t launch_cache_read(const CacheReadArgs& a, hipStream_t stream);

struct CachePlan;  // cache_plan.hpp

struct CacheAttentionArgs {
  CacheView c;
  const void* q;
  int64_t q_stride;  // of a token, in elements
  int64_t n;         // tokens
  int B, Hq, G, max_q, max_pages;
  const int* page_table;  // [B, max_pages]
  const int* lengths;     // [B]
  const int* q_starts;    // [B + 1], or null: n / B tokens each
  const int64_t* tree;    // [n, tree_words], or null: causal
  int tree_words;
  float softmax_scale;
  void* out;
  int out_bf16;
  float* lse;  // [n, Hq] or null
  void* workspace;
};

void launch_cache_rows(const CacheAttentionArgs& a, const CachePlan& plan, hipStream_t stream);
hipError_t launch_cache_attention(const CacheAttentionArgs& a, hipStream_t stream);

}  // namespace fp4attn
