// Host-side launchers of the operators around a key/value cache:
// rotary positions, the cache's quantizer and reader, its pages, attention over it.  Arguments
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

// Pages and slots of a step's tokens (csrc/cache_assign.hip).
struct CacheAssignArgs {
  int* page_table;     // [B, max_pages]
  const int* held;     // [B]
  const int* lengths;  // [B]
  const int* fresh;    // [B] new tokens, or null: `each`
  const int* shared;   // [B] or null: 0
  int* ring;           // [capacity] free pages
  const int64_t* counts;
  int64_t* counts_out;
  int* lengths_out;
  int64_t* slots;      // [tokens]
  int64_t* positions;  // [tokens]
  int* starts;         // [B + 1]
  void* workspace;
  int B, max_pages, page_shift, each, tokens, capacity;
};

// Steps of up to so many sequences and tokens are served by one workgroup, without a workspace.  In one launch / in two, us in a graph:
// 64 sequences, one token each 4.3 / 6.6; 1000 sequences 8.3 / 12.7; 2000 tokens of 256 sequences 7.1 / 8.9.  20 thousand tokens of
// prompts take 8.1 in two.  A step that moves many pages is the worse for it, us a call of 64 sequences that return 4 thousand pages 5.8 / 8.4,
// 16 thousand 9.4 / 8.5, 64 thousand (of 16 keys, a million keys) 28 / 8.5, 300 thousand 119 / 8.5.  How many move only the device knows; a rule on
// those that may would charge every step with a wide table 2.3 us.
constexpr int kAssignOne = 1024, kAssignOneTokens = 4096;
constexpr bool assign_in_one(int64_t B, int64_t tokens) { return B <= kAssignOne && tokens <= kAssignOneTokens; }
constexpr int64_t cache_assign_workspace(int64_t B, int64_t tokens) { return assign_in_one(B, tokens) ? 0 : 16 + 16 * B; }
hipError_t launch_cache_assign(const CacheAssignArgs& a, hipStream_t stream);

struct CachePlan;  // cache_plan.hpp

struct CacheAttentionArgs {
  static constexpr bool kShaped = false, kScores = false, kPrefix = false, kDirect = false;
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

// tanh(x) = x (p_0 + p_1 x^2 ..) for |x| <= 0.6: a least-squares fit, its weights moved until the largest relative errors were
// equal, 7.3e-8, 1.2 half steps of fp32.
constexpr double kTanhNear = 0.6, kTanh[5] = {0.99999992687, -0.333323099773, 0.133101736776, -0.0521014805221, 0.0154754275956};
// c tanh(z / c) in binades, of a product s of codes with z = scale s, with inside = scale / c and C = c log2(e): near zero
// y K(y^2), beyond it C tanh(inside s) by an exponential.  y = s, K's coefficients are k_i = C inside^(2 i + 1) p_i, up to |s| = near.
// Where these leave fp32's normal numbers (caps above some hundred, caps far below the scale) near is -1, which no |s| is at
// most: y = inside s, k_i = C p_i, up to |y| = kTanhNear.
struct CapShape {
  int on;
  float inside, most;  // scale / c, C
  float near, k[5];
};
inline CapShape cap_shape(double scale, double c) {
  CapShape s{};
  if (c == 0.0) return s;
  const double inside = scale / c, most = c * 1.4426950408889634;
  s.on = 1;
  s.inside = (float)inside;
  s.most = (float)most;
  auto coefficients = [&](double first, double step) {
    for (int i = 0; i < 5; ++i, first *= step) s.k[i] = (float)(first * kTanh[i]);
  };
  coefficients(most * inside, inside * inside);
  const bool fits = s.k[4] > 1e-36f && s.k[4] < 1e30f && s.k[0] > 1e-36f && s.k[0] < 1e30f;
  if (!fits) coefficients(most, 1.0);
  s.near = fits ? (float)(kTanhNear / inside) : -1.0f;
  return s;
}

// Attention with shaped scores, other masks, a shared prefix.
struct ShapedAttentionArgs : CacheAttentionArgs {
  static constexpr bool kShaped = true, kScores = true;
  CapShape cap;
  int window;            // keys that a token sees up to its own, 0: all
  const float* slopes;   // [Hq] or null
  const int* open_keys;  // [B] keys that every new token sees, or null
  // the shared prefix: its keys (a multiple of kUnit; 0: none), passed over in pieces of prefix_units units; of every
  // piece and row of q {reference, sum, sum of the rounded values} and the accumulators
  int shared, prefix_pieces, prefix_units;
  // beside direct ranges: row tiles that may be cut; the row tile and direct_units of the sequences' own pass
  int crossings, own_tile, direct_units;
  float4* prefix_stat;  // [pieces][n * Hq]
  float* prefix_acc;    // [pieces][n * Hq][d]
  int* arrived;         // of each of these the pieces that are there, then the units of all; or null (look_for_long)
};
// The same without a cap and slopes.
struct MaskedAttentionArgs : ShapedAttentionArgs {
  static constexpr bool kScores = false;
};
// Either behind a shared prefix, with a plan that has direct ranges.
struct ShapedBehindArgs : ShapedAttentionArgs {
  static constexpr bool kDirect = true;
};
struct MaskedBehindArgs : MaskedAttentionArgs {
  static constexpr bool kDirect = true;
};
// The pass over the shared prefix itself.
struct PrefixAttentionArgs : ShapedAttentionArgs {
  static constexpr bool kPrefix = true;
};

hipError_t launch_cache_attention(const CacheAttentionArgs& a, const CachePlan& plan, hipStream_t stream);
hipError_t launch_shaped_attention(const ShapedAttentionArgs& a, const CachePlan& plan, hipStream_t stream);
hipError_t launch_masked_attention(const MaskedAttentionArgs& a, const CachePlan& plan, hipStream_t stream);
hipError_t launch_shaped_behind(const ShapedBehindArgs& a, const CachePlan& plan, hipStream_t stream);
hipError_t launch_masked_behind(const MaskedBehindArgs& a, const CachePlan& plan, hipStream_t stream);
hipError_t launch_prefix_attention(const PrefixAttentionArgs& a, const CachePlan& plan, hipStream_t stream);

}  // namespace fp4attn
