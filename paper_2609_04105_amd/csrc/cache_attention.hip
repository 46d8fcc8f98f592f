// Attention of new tokens over the paged MXFP4 or MXFP8 cache.
//
//   O_r = sum_j p_rj V_j / sum_j p_rj,  p_rj = exp(s q_r . K_j) over the keys j that row r
// sees; K_j, V_j the values that the cache's codes stand for.  One pass over the keys with
// a running maximum and sums.  A row is one (token, head of a key head's group).
//
// What bounds it: with few rows the cache, 2 (d / 2 + d / 32) bytes of MXFP4 a key and head,
// is read once and nothing else is large, so every choice serves the load path:
// - the waves of a workgroup walk different 32-key tiles and each loads its tile straight
//   into the registers that the matrix products take, one tile ahead: no LDS, no barrier
//   in the loop.  The cache's layouts are made for this.  K: a lane's 16 bytes are 32
//   values of one key under one scale, the A operand of the S^T = K Q^T products (the
//   order of d is free as long as Q's is the same).  V: eight keys of one sixteenth of d lie
//   together, the A operand of the O^T = V^T P^T products;
// - keys enter S^T permuted so that lane group g (lane / 16) ends with scores of keys
//   8 g .. 8 g + 7 of the tile: its probabilities are its B operand of the PV product;
// - codes become bf16 exactly (E2M1 has two significant bits, E4M3 four), scales in the
//   same instruction; 1/6 of MXFP4 goes into the score factor and into the end;
// - the keys of a sequence are cut over workgroups when the rows alone do not fill the
//   chip; partial results meet in a second launch (no atomics: the order is fixed).
//
// Precision: scores and sums fp32.  P is rounded to bf16 for the matrix product, and the
// normaliser sums the same rounded values (a product with ones), so that the rounding of
// a dominant key cancels; the log normaliser that `lse` returns takes the unrounded sum.
// The reference of a row lags its maximum by at most 8 binades (p <= 256), which
// saves most rescalings of the accumulators.
#include "gfx950.hpp"
#include "serving.hpp"

namespace fp4attn {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kTile = 32;       // keys of a wave's step
constexpr float kLag = 8.0f;    // binades that a row's reference may lag its maximum
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

__device__ __forceinline__ v4f mfma_16x16x32(v4i a, v4i b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// max and sum over the four lane groups that share lane % 16
__device__ __forceinline__ float groups_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(as_uint(x), as_uint(x), false, false);
  x = fmaxf(as_float(r[0]), as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(as_uint(x), as_uint(x), false, false);
  return fmaxf(as_float(r[0]), as_float(r[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(as_uint(x), as_uint(x), false, false);
  x = as_float(r[0]) + as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(as_uint(x), as_uint(x), false, false);
  return as_float(r[0]) + as_float(r[1]);
}

// New tokens, keys and chunks of the sequences.
struct Sequence {
  int first, tokens;  // rows of q
  int keys;           // lengths[b], within [0, the table's capacity]
  int prefix;         // keys before the new tokens (may be negative)
};
__device__ __forceinline__ Sequence sequence(const CacheAttentionArgs& a, int b) {
  Sequence s;
  if (a.q_starts) {
    const int64_t n = a.n;
    const int64_t lo = a.q_starts[b], hi = a.q_starts[b + 1];
    const int64_t from = lo < 0 ? 0 : (lo > n ? n : lo), to = hi < from ? from : (hi > n ? n : hi);
    s.first = (int)from;
    s.tokens = (int)(to - from > a.max_q ? a.max_q : to - from);
    const int len = a.lengths[b];
    s.prefix = (len < 0 ? 0 : len) - (int)(to - from);
    s.keys = len;
  } else {
    s.tokens = (int)(a.n / a.B);
    s.first = b * s.tokens;
    s.keys = a.lengths[b];
    s.prefix = (s.keys < 0 ? 0 : s.keys) - s.tokens;
  }
  const int64_t capacity = (int64_t)a.max_pages << a.c.page_shift;
  s.keys = s.keys < 0 ? 0 : (s.keys > capacity ? (int)capacity : s.keys);
  return s;
}

// Chunk `ci` of the batch: its sequence, first key, end, and its place among the
// sequence's chunks.  Every wave finds it by itself.
struct Chunk {
  int b, index, count, first_chunk;  // first_chunk: ci of the sequence's chunk 0
  int begin, end;
  bool none;
};
__device__ __forceinline__ Chunk find_chunk(const CacheAttentionArgs& a, const CachePlan& plan, int ci) {
  Chunk r{};
  const int lane = threadIdx.x & 63;
  if (!plan.split) {
    r.b = ci;
    const Sequence s = sequence(a, ci);
    r.count = 1;
    r.first_chunk = ci;
    r.end = s.keys;
    r.none = s.tokens == 0;
    return r;
  }
  int64_t total = 0;
  for (int b = lane; b < a.B; b += 64) {
    const Sequence s = sequence(a, b);
    total += s.tokens ? s.keys : 0;
  }
#pragma unroll
  for (int i = 1; i < 64; i *= 2) total += __shfl_xor(total, i);
  int64_t chunk64 = (total + plan.target - 1) / plan.target;
  chunk64 = chunk64 < plan.min_chunk ? plan.min_chunk : (chunk64 > kMaxCacheKeys ? kMaxCacheKeys : chunk64);
  const int chunk = uniform((int)((chunk64 + kTile * kWaves - 1) / (kTile * kWaves) * (kTile * kWaves)));
  int before = 0;
  r.none = true;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    int count = 0, keys = 0;
    if (b0 + lane < a.B) {
      const Sequence s = sequence(a, b0 + lane);
      keys = s.keys;
      count = s.tokens == 0 ? 0 : (keys == 0 ? 1 : (int)(((int64_t)keys + chunk - 1) / chunk));
    }
    int sum = count;  // inclusive prefix
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
      const int up = __shfl_up(sum, i);
      if (lane >= i) sum += up;
    }
    const int start = before + sum - count;
    const bool mine = ci >= start && ci < start + count;
    const uint64_t found = __ballot(mine);
    if (found) {
      const int src = __ffsll((unsigned long long)found) - 1;
      r.b = uniform(b0 + src);
      r.count = uniform(__shfl(count, src));
      r.first_chunk = uniform(__shfl(start, src));
      keys = uniform(__shfl(keys, src));
      r.index = ci - r.first_chunk;
      r.begin = r.index * chunk;
      r.end = r.count == 1 ? keys : (r.index + 1 == r.count ? keys : r.begin + chunk);
      r.none = false;
      return r;
    }
    before += uniform(__shfl(sum, 63));
  }
  return r;
}

// Partial results in the workspace: per sequence {first chunk, chunks}, then per tile of
// (chunk, key head, row tile) the accumulators [tile_rows, D] and {reference, sum, sum of
// the rounded values} per row.
struct Partials {
  int2* sequences;
  float* acc;
  float4* stat;
};
__host__ __device__ inline int64_t partial_tiles(const CachePlan& p, int H) { return p.chunks * H * p.row_tiles; }
__device__ __forceinline__ Partials partials(const CacheAttentionArgs& a, const CachePlan& p, int D) {
  char* w = static_cast<char*>(a.workspace);
  Partials r;
  r.sequences = reinterpret_cast<int2*>(w);
  w += ((int64_t)a.B * 8 + 255) / 256 * 256;
  r.stat = reinterpret_cast<float4*>(w);
  w += partial_tiles(p, a.c.H) * p.tile_rows * 16;
  r.acc = reinterpret_cast<float*>(w);
  return r;
}

// N consecutive values, 16 bytes at a time.
template <int N>
__device__ __forceinline__ void store_row(float* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    reinterpret_cast<float4*>(p)[i] = float4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
}
template <int N>
__device__ __forceinline__ void store_row(uint16_t* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 8; ++i) {
    unsigned w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = __builtin_bit_cast(unsigned, v2bf{(__bf16)v[8 * i + 2 * j], (__bf16)v[8 * i + 2 * j + 1]});
    reinterpret_cast<uint4*>(p)[i] = uint4{w[0], w[1], w[2], w[3]};
  }
}

__device__ __forceinline__ bool is_zero(float x) { return (as_uint(x) << 1) == 0u; }

// The log normaliser in nats from a base-2 reference and sum.
__device__ __forceinline__ float log_norm(float ref, float sum) {
  return is_zero(sum) ? -__builtin_inff() : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int D, bool FP8>
struct Format {
  static constexpr int kBits = FP8 ? 8 : 4;
  static constexpr int kSteps = D / 32;                   // QK products per 16 keys
  static constexpr int kDTiles = D / 16;                  // PV products per 32 keys
  static constexpr int kBlocks = D / 32;                  // scales per key
  static constexpr int kKWords = D / 4 * kBits / 32;      // of a lane: D / 4 values of one key
  static constexpr int kVWords = D / 16 * kBits / 8 * 2;  // of a lane: D / 16 values of eight keys
};

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, unsigned (&w)[N]) {
  if constexpr (N == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x;
    w[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 x = reinterpret_cast<const uint4*>(p)[i];
      w[4 * i] = x.x;
      w[4 * i + 1] = x.y;
      w[4 * i + 2] = x.z;
      w[4 * i + 3] = x.w;
    }
  }
}

// What a lane holds of one 32-key tile.
template <int D, bool FP8>
struct Tile {
  using F = Format<D, FP8>;
  unsigned k[2][F::kKWords];  // [half] key 8 (m / 4) + 4 half + m % 4, m = lane % 16: values D / 4 * (lane / 16) ..
  unsigned ks[2];             // their E8M0 byte
  unsigned v[F::kVWords];     // keys 8 (lane / 16) .. + 7, values D / 16 * (lane % 16) ..
  unsigned vs[2];             // their eight E8M0 bytes
};

// The two pages of a tile (the same one unless pages hold 16 keys); -1: no such page.
struct Pages {
  int p0, p1;
};
__device__ __forceinline__ Pages find_pages(const CacheAttentionArgs& a, const int* __restrict__ table, int key0) {
  Pages r;
  r.p0 = table[key0 >> a.c.page_shift];
  r.p1 = r.p0;
  if (a.c.page_shift == 4) {
    const int at = (key0 >> 4) + 1;
    r.p1 = table[at < a.max_pages ? at : a.max_pages - 1];
  }
  r.p0 = (unsigned)r.p0 < (uint64_t)a.c.pages ? r.p0 : -1;
  r.p1 = (unsigned)r.p1 < (uint64_t)a.c.pages ? r.p1 : -1;
  return r;
}

template <int D, bool FP8>
__device__ __forceinline__ void load_tile(const CacheView& c, Pages pages, int key0, int head, int lane, Tile<D, FP8>& t) {
  using F = Format<D, FP8>;
  const int m = lane & 15, g = lane >> 4, shift = c.page_shift;
  const int inside = key0 & ((1 << shift) - 1);
  // rows (page, head, offset) of the tile's two halves of 16 keys; a missing page reads page 0
  const int64_t r0 = (((int64_t)(pages.p0 < 0 ? 0 : pages.p0) * c.H + head) << shift) + inside;
  const int64_t r1 = shift == 4 ? ((int64_t)(pages.p1 < 0 ? 0 : pages.p1) * c.H + head) << 4 : r0 + 16;
  const int64_t krow = (m >= 8 ? r1 : r0) + (m & 4) * 2 + (m & 3);
  const int64_t vgroup = ((g >= 2 ? r1 : r0) >> 3) + (g & 1);
  constexpr int kKBytes = F::kKWords * 4, kVBytes = F::kVWords * 4;
  const uint8_t* kp = c.k_codes + krow * (4 * kKBytes) + g * kKBytes;
  const uint8_t* ksp = c.k_scales + krow * F::kBlocks + g * F::kBlocks / 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    load_words<F::kKWords>(kp + h * 4 * (4 * kKBytes), t.k[h]);
    t.ks[h] = ksp[h * 4 * F::kBlocks];
  }
  load_words<F::kVWords>(c.v_codes + (vgroup * 16 + m) * kVBytes, t.v);
  const uint2 s = *reinterpret_cast<const uint2*>(c.v_scales + (vgroup * F::kBlocks + m * F::kBlocks / 16) * 8);
  t.vs[0] = s.x;
  t.vs[1] = s.y;
}

// The E8M0 byte as the converter's scale operand: a float's exponent field.
__device__ __forceinline__ float scale_of(unsigned byte) { return as_float(byte << 23); }
template <int J>
__device__ __forceinline__ float scale_of_key(const unsigned (&vs)[2]) {
  const unsigned w = vs[J / 4];
  constexpr int j = J % 4;
  return as_float((j == 3 ? w >> 1 : w << (23 - 8 * j)) & 0x7f800000u);
}

// Pair I (values 2 I, 2 I + 1) of packed codes as two bf16.
template <int I, bool FP8>
__device__ __forceinline__ unsigned code_pair(const unsigned* w, float scale) {
  if constexpr (FP8)
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[I / 2], scale, I % 2 != 0));
  else
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[I / 4], scale, I % 4));
}

// E8M0 bytes from which bf16 values may overflow (6 * 2^126, 448 * 2^120): such a V block
// counts as non-finite, as byte 255 does.
template <bool FP8>
constexpr unsigned kHugeScale = FP8 ? 247u : 253u;

// Keys that a row sees: j < limit, or a bit of the tree.
struct Row {
  int limit;            // causal: keys below; tree: the prefix
  const int64_t* bits;  // of the row's token, or null
};
__device__ __forceinline__ unsigned below(int n) { return (1u << (n < 0 ? 0 : (n > 8 ? 8 : n))) - 1u; }
// Which of keys key .. key + 7 the row sees, as bits.  Straight-line code: loads are
// clamped to the row's words instead of branched around.
__device__ __forceinline__ unsigned seen8(const Row& r, int key, int prefix, int tokens, int words) {
  unsigned see = below(r.limit - key);
  if (words) {  // uniform
    const int u = key - prefix, at = u >> 6, shift = u & 63;
    const int i = at < 0 ? 0 : (at >= words ? words - 1 : at), k = i + 1 < words ? i + 1 : i;
    const uint64_t lo = (uint64_t)r.bits[i], hi = (uint64_t)r.bits[k];
    const unsigned inside = (unsigned)(lo >> shift) | (shift > 56 ? (unsigned)(hi << (64 - shift)) : 0u);
    const unsigned up = u > -8 ? (unsigned)lo << (-u & 7) : 0u;  // the first new token is key - u
    see |= (u < 0 ? up : inside) & below(tokens - u);
  }
  return see;
}

template <int D, bool FP8, int NR>
__global__ __launch_bounds__(kThreads, NR == 1 ? 3 : 1) void cache_attention_kernel(const CacheAttentionArgs a, const CachePlan plan) {
  using F = Format<D, FP8>;
  constexpr int kV = D / 4;  // output values of a lane and row
  __shared__ float4 lds_acc[kWaves / 2][NR * F::kDTiles][64];
  __shared__ float lds_stat[kWaves / 2][NR][3][64];

  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  // Row tiles of one (chunk, key head) go to one XCD (workgroups are dealt round-robin to
  // eight), which then reads the chunk once for all of them.
  int item = blockIdx.x, tile = 0;
  if (plan.row_tiles > 1) {
    const int q = item / 8;
    tile = q % plan.row_tiles;
    item = q / plan.row_tiles * 8 + item % 8;
  }
  const int ci = item / a.c.H, head = item - ci * a.c.H;
  if (ci >= plan.chunks) return;
  const Chunk ch = find_chunk(a, plan, ci);
  if (ch.none) return;
  const Sequence seq = sequence(a, ch.b);
  const int rows = seq.tokens * a.G, row0 = tile * 16 * NR;
  if (plan.split && ch.index == 0 && head == 0 && tile == 0 && threadIdx.x == 0)
    partials(a, plan, D).sequences[ch.b] = int2{ch.first_chunk, ch.count};
  if (row0 >= rows) return;

  // this lane's rows (the same for the four lane groups) and its part of their queries
  Row row[NR];
  v4i q[NR][F::kSteps];
  int at[NR];  // row of q and out, as token * Hq + head
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int i = row0 + 16 * r + m, ic = i < rows ? i : rows - 1, t = ic / a.G;
    const int token = seq.first + t, h = head * a.G + (ic - t * a.G);
    at[r] = i < rows ? token * a.Hq + h : -1;
    row[r].limit = a.tree ? seq.prefix : seq.prefix + t + 1;
    row[r].limit = row[r].limit > seq.keys ? seq.keys : row[r].limit;
    row[r].bits = a.tree ? a.tree + (int64_t)token * a.tree_words : nullptr;
    const uint16_t* p = static_cast<const uint16_t*>(a.q) + token * a.q_stride + h * D + g * (D / 4);
#pragma unroll
    for (int s = 0; s < F::kSteps; ++s) q[r][s] = reinterpret_cast<const v4i*>(p)[s];
  }
  // keys below `common` are seen by every row of the sequence
  int common = a.tree ? seq.prefix : seq.prefix + 1;
  common = common > seq.keys ? seq.keys : common;
  int seen_tokens = seq.keys - seq.prefix;  // that have a bit in the tree
  seen_tokens = seen_tokens > 64 * a.tree_words ? 64 * a.tree_words : seen_tokens;

  v4f acc[NR][F::kDTiles], sum16[NR];  // sum16: the rounded probabilities, in every register
  float ref[NR], sum[NR];              // base 2, lags the maximum by at most kLag; this lane's own keys
  const v4i ones = {0x3f803f80, 0x3f803f80, 0x3f803f80, 0x3f803f80};
#pragma unroll
  for (int r = 0; r < NR; ++r) {
#pragma unroll
    for (int t = 0; t < F::kDTiles; ++t) acc[r][t] = v4f{0, 0, 0, 0};
    sum16[r] = v4f{0, 0, 0, 0};
    ref[r] = -__builtin_inff();
    sum[r] = 0.0f;
  }
  const float factor = a.softmax_scale * kLog2e * (FP8 ? 1.0f : 1.0f / 6.0f);
  const int* __restrict__ table = a.page_table + (int64_t)ch.b * a.max_pages;

  auto step = [&](Tile<D, FP8>& t, const Pages& pages, int key0) {
    const bool masked = key0 + kTile > common || pages.p0 < 0 || pages.p1 < 0;  // uniform
    if (masked) {
      // Keys that no row sees hold anything: their V codes and scales become zero.  A
      // non-finite V block that some row sees becomes zero too, and turns the outputs of
      // the rows that see it to NaN here.
      bool huge = false;
      const int base = key0 + 8 * g;
      const bool page_ok = (g >= 2 ? pages.p1 : pages.p0) >= 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool there = page_ok && base + j < seq.keys;
        const unsigned byte = t.vs[j / 4] >> (8 * (j % 4)) & 255u;
        huge |= there && byte >= kHugeScale<FP8>;
        if (!there || byte >= kHugeScale<FP8>) {
          t.vs[j / 4] &= ~(255u << (8 * (j % 4)));
          if constexpr (F::kVWords >= 8) {
#pragma unroll
            for (int w = 0; w < F::kVWords / 8; ++w) t.v[j * (F::kVWords / 8) + w] = 0u;
          } else {
            t.v[j / 2] &= j % 2 ? 0x0000ffffu : 0xffff0000u;
          }
        }
      }
      if (__any(huge)) {  // lane group g holds outputs of d block g (d = 64: g / 2)
        const int blk = g * F::kBlocks / 4;
        for (int k = 0; k < kTile; ++k) {
          const int page = k >= 16 ? pages.p1 : pages.p0, key = key0 + k;
          if (page < 0 || key >= seq.keys) continue;
          const int64_t r8 = ((((int64_t)page * a.c.H + head) << a.c.page_shift) + (key & ((1 << a.c.page_shift) - 1))) >> 3;
          if (a.c.v_scales[(r8 * F::kBlocks + blk) * 8 + (k & 7)] < kHugeScale<FP8>) continue;
#pragma unroll
          for (int r = 0; r < NR; ++r)
            if (seen8(row[r], key & ~7, seq.prefix, seen_tokens, a.tree_words) >> (key & 7) & 1)
#pragma unroll
              for (int tt = 0; tt < F::kDTiles; ++tt)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[r][tt][i] = as_float(0x7fc00000u);
        }
      }
    }
    // S^T: register i of half h is key 8 g + 4 h + i
    v4f s[NR][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float scale = scale_of(t.ks[h]);
#pragma unroll
      for (int r = 0; r < NR; ++r) s[r][h] = v4f{0, 0, 0, 0};
      static_for<F::kSteps>([&](auto S_) {
        constexpr int st = decltype(S_)::value;
        v4i kk;
        static_for<4>([&](auto I_) {
          constexpr int i = decltype(I_)::value;
          kk[i] = (int)code_pair<4 * st + i, FP8>(t.k[h], scale);
        });
#pragma unroll
        for (int r = 0; r < NR; ++r) s[r][h] = mfma_16x16x32(kk, q[r][st], s[r][h]);
      });
    }
    if (masked) {
      const int base = key0 + 8 * g;
      const unsigned there = (g >= 2 ? pages.p1 : pages.p0) >= 0 ? below(seq.keys - base) : 0u;
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const unsigned see = there & seen8(row[r], base, seq.prefix, seen_tokens, a.tree_words);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[r][j / 4][j % 4] = see >> j & 1 ? s[r][j / 4][j % 4] : -__builtin_inff();
      }
    }
    float top[NR];
    bool rise = false;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float x = fmaxf(fmaxf(s[r][0][0], s[r][0][1]), s[r][0][2]);
      x = fmaxf(fmaxf(x, s[r][0][3]), s[r][1][0]);
      x = fmaxf(fmaxf(x, s[r][1][1]), s[r][1][2]);
      top[r] = groups_max(fmaxf(x, s[r][1][3])) * factor;
      rise |= top[r] > ref[r] + kLag;
    }
    if (__any(rise)) {
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const float now = fmaxf(ref[r], top[r]);
        const float down = now == ref[r] ? 1.0f : __builtin_amdgcn_exp2f(ref[r] - now);
        ref[r] = now;
        sum[r] *= down;
        sum16[r] *= down;
#pragma unroll
        for (int tt = 0; tt < F::kDTiles; ++tt) acc[r][tt] *= down;
      }
    }
    v4i p[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const float base = ref[r] == -__builtin_inff() ? 0.0f : -ref[r];
      float e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(fmaf(s[r][j / 4][j % 4], factor, base));
      sum[r] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
#pragma unroll
      for (int j = 0; j < 4; ++j) p[r][j] = (int)__builtin_bit_cast(unsigned, v2bf{(__bf16)e[2 * j], (__bf16)e[2 * j + 1]});
      sum16[r] = mfma_16x16x32(ones, p[r], sum16[r]);
    }
    // O^T: product t takes value t of every lane's part, rows d = D / 16 * m + t
    float vscale[8];
    static_for<8>([&](auto J_) { vscale[decltype(J_)::value] = scale_of_key<decltype(J_)::value>(t.vs); });
    static_for<F::kDTiles / 2>([&](auto E_) {
      constexpr int e = decltype(E_)::value;  // values 2 e, 2 e + 1 of the part
      unsigned w[8];
      static_for<8>([&](auto J_) {
        constexpr int j = decltype(J_)::value;
        // pair index within the lane's run of eight keys
        w[j] = code_pair<j * (F::kDTiles / 2) + e, FP8>(t.v, vscale[j]);
      });
      v4i lo, hi;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lo[j] = (int)__builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x05040100u);
        hi[j] = (int)__builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], 0x07060302u);
      }
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        acc[r][2 * e] = mfma_16x16x32(lo, p[r], acc[r][2 * e]);
        acc[r][2 * e + 1] = mfma_16x16x32(hi, p[r], acc[r][2 * e + 1]);
      }
    });
  };

  // The wave's tiles, one loaded ahead; the page table two ahead.
  constexpr int kStride = kTile * kWaves;
  int key0 = ch.begin + kTile * wave;
  if (key0 < ch.end) {
    Tile<D, FP8> cur, next;
    Pages now = find_pages(a, table, key0), then = now;
    load_tile<D, FP8>(a.c, now, key0, head, lane, cur);
    if (key0 + kStride < ch.end) then = find_pages(a, table, key0 + kStride);
    while (true) {
      const int ahead = key0 + kStride;
      Pages after = then;
      if (ahead < ch.end) {
        load_tile<D, FP8>(a.c, then, ahead, head, lane, next);
        if (ahead + kStride < ch.end) after = find_pages(a, table, ahead + kStride);
      }
      step(cur, now, key0);
      if (ahead >= ch.end) break;
      key0 = ahead;
      cur = next;
      now = then;
      then = after;
    }
  }

#pragma unroll
  for (int r = 0; r < NR; ++r) sum[r] = groups_sum(sum[r]);

  // Join the waves, half of them at a time: same lanes, same rows and columns.
#pragma unroll
  for (int n = kWaves / 2; n >= 1; n /= 2) {
    __syncthreads();
    if (wave >= n && wave < 2 * n) {
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        lds_stat[wave - n][r][0][lane] = ref[r];
        lds_stat[wave - n][r][1][lane] = sum[r];
        lds_stat[wave - n][r][2][lane] = sum16[r][0];
#pragma unroll
        for (int t = 0; t < F::kDTiles; ++t)
          lds_acc[wave - n][r * F::kDTiles + t][lane] = float4{acc[r][t][0], acc[r][t][1], acc[r][t][2], acc[r][t][3]};
      }
    }
    __syncthreads();
    if (wave < n) {
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const float other = lds_stat[wave][r][0][lane], top = fmaxf(ref[r], other);
        const float mine = ref[r] == top ? 1.0f : __builtin_amdgcn_exp2f(ref[r] - top);
        const float its = other == top ? 1.0f : __builtin_amdgcn_exp2f(other - top);
        ref[r] = top;
        sum[r] = sum[r] * mine + lds_stat[wave][r][1][lane] * its;
        sum16[r][0] = sum16[r][0] * mine + lds_stat[wave][r][2][lane] * its;
#pragma unroll
        for (int t = 0; t < F::kDTiles; ++t) {
          const float4 o = lds_acc[wave][r * F::kDTiles + t][lane];
          acc[r][t] = v4f{acc[r][t][0] * mine + o.x * its, acc[r][t][1] * mine + o.y * its,
                          acc[r][t][2] * mine + o.z * its, acc[r][t][3] * mine + o.w * its};
        }
      }
    }
  }
  if (wave != 0) return;

#pragma unroll
  for (int r = 0; r < NR; ++r) {
    if (at[r] < 0) continue;
    float o[kV];  // columns D / 4 * g ..: register i of product t is column D / 16 * (4 g + i) + t
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < F::kDTiles; ++t) o[i * F::kDTiles + t] = acc[r][t][i];
    if (ch.count == 1) {
      const float norm = is_zero(sum16[r][0]) ? 0.0f : (FP8 ? 1.0f : 1.0f / 6.0f) / sum16[r][0];
#pragma unroll
      for (int i = 0; i < kV; ++i) o[i] = is_zero(sum16[r][0]) ? 0.0f : o[i] * norm;
      const int64_t to = (int64_t)at[r] * D + g * kV;
      if (a.out_bf16) store_row<kV>(static_cast<uint16_t*>(a.out) + to, o);
      else store_row<kV>(static_cast<float*>(a.out) + to, o);
      if (a.lse && g == 0) a.lse[at[r]] = log_norm(ref[r], sum[r]);
    } else {
      const Partials w = partials(a, plan, D);
      const int64_t to = (((int64_t)ci * a.c.H + head) * plan.row_tiles + tile) * plan.tile_rows + 16 * r + m;
      store_row<kV>(w.acc + to * D + g * kV, o);
      if (g == 0) w.stat[to] = float4{ref[r], sum[r], sum16[r][0], 0.0f};
    }
  }
}

// Joins the chunks of one row: eight waves take D / 4-lane groups of chunks each.
// grid: (rows of the longest sequence and all heads, B)
constexpr int kJoinThreads = 512;
template <int D, bool FP8>
__global__ __launch_bounds__(kJoinThreads) void cache_join_kernel(const CacheAttentionArgs a, const CachePlan plan) {
  constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes;  // lanes of a row; chunks in flight
  const Partials w = partials(a, plan, D);
  const int b = blockIdx.y;
  const Sequence seq = sequence(a, b);
  const int t = blockIdx.x / a.Hq, hq = blockIdx.x - t * a.Hq;
  if (t >= seq.tokens) return;
  const int2 chunks = w.sequences[b];
  if (chunks.y <= 1) return;
  const int head = hq / a.G, i = t * a.G + (hq - head * a.G);
  const int tile = i / (16 * plan.nr), in_tile = i - tile * 16 * plan.nr;
  const int64_t step = (int64_t)a.c.H * plan.row_tiles * plan.tile_rows;
  const int64_t first = (((int64_t)chunks.x * a.c.H + head) * plan.row_tiles + tile) * plan.tile_rows + in_tile;
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  __shared__ float4 acc_lds[kGroups][kLanes];
  __shared__ float4 stat_lds[kGroups];
  float ref = -__builtin_inff(), sum = 0.0f, sum16 = 0.0f;
  float4 acc = {0, 0, 0, 0};
  auto join = [&](const float4& s, const float4& o) {
    const float top = fmaxf(ref, s.x);
    const float mine = ref == top ? 1.0f : __builtin_amdgcn_exp2f(ref - top);
    const float its = s.x == top ? 1.0f : __builtin_amdgcn_exp2f(s.x - top);
    ref = top;
    sum = sum * mine + s.y * its;
    sum16 = sum16 * mine + s.z * its;
    acc = float4{acc.x * mine + o.x * its, acc.y * mine + o.y * its, acc.z * mine + o.z * its, acc.w * mine + o.w * its};
  };
#pragma unroll 4
  for (int k = group; k < chunks.y; k += kGroups) {
    const int64_t at = first + k * step;
    join(w.stat[at], reinterpret_cast<const float4*>(w.acc + at * D)[lane]);
  }
  acc_lds[group][lane] = acc;
  if (lane == 0) stat_lds[group] = float4{ref, sum, sum16, 0.0f};
  __syncthreads();
  if (group != 0) return;
  const int used = chunks.y < kGroups ? chunks.y : kGroups;
  for (int k = 1; k < used; ++k) join(stat_lds[k], acc_lds[k][lane]);
  const int at = (seq.first + t) * a.Hq + hq;
  const bool empty = is_zero(sum16);
  const float norm = (FP8 ? 1.0f : 1.0f / 6.0f) / sum16;
  const float o[4] = {empty ? 0.0f : acc.x * norm, empty ? 0.0f : acc.y * norm, empty ? 0.0f : acc.z * norm,
                      empty ? 0.0f : acc.w * norm};
  const int64_t to = (int64_t)at * D + lane * 4;
  if (a.out_bf16) {
    const unsigned lo = __builtin_bit_cast(unsigned, v2bf{(__bf16)o[0], (__bf16)o[1]});
    const unsigned hi = __builtin_bit_cast(unsigned, v2bf{(__bf16)o[2], (__bf16)o[3]});
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + to) = uint2{lo, hi};
  } else {
    store_row<4>(static_cast<float*>(a.out) + to, o);
  }
  if (a.lse && lane == 0) a.lse[at] = log_norm(ref, sum);
}

template <int D, bool FP8>
void launch_format(const CacheAttentionArgs& a, const CachePlan& plan, hipStream_t stream) {
  const unsigned grid = (unsigned)plan.workgroups;
  if (plan.nr == 1) cache_attention_kernel<D, FP8, 1><<<grid, kThreads, 0, stream>>>(a, plan);
  else if (plan.nr == 2) cache_attention_kernel<D, FP8, 2><<<grid, kThreads, 0, stream>>>(a, plan);
  else cache_attention_kernel<D, FP8, 4><<<grid, kThreads, 0, stream>>>(a, plan);
  if (plan.split)
    cache_join_kernel<D, FP8><<<dim3((unsigned)(a.max_q * a.Hq), (unsigned)a.B), kJoinThreads, 0, stream>>>(a, plan);
}

}  // namespace

CachePlan cache_plan(int64_t B, int64_t H, int64_t G, int64_t d, int64_t max_q, int64_t max_keys) {
  CachePlan p{};
  const int64_t rows = max_q * G;
  p.nr = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
  p.row_tiles = (int)((rows + 16 * p.nr - 1) / (16 * p.nr));
  p.tile_rows = (int)(rows < 16 * p.nr ? rows : 16 * p.nr);
  p.min_chunk = 1024;
  const int64_t wanted = 1024;  // workgroups
  const int64_t per_chunk = H * p.row_tiles;
  p.split = max_keys > p.min_chunk && B * per_chunk < 2 * wanted;
  p.target = (int)(wanted / per_chunk < 1 ? 1 : wanted / per_chunk);
  const int64_t most = B * ((max_keys + p.min_chunk - 1) / p.min_chunk);
  p.chunks = p.split ? p.target + B : B;
  if (p.split && most < p.chunks) p.chunks = most;
  const int64_t items = p.row_tiles > 1 ? (p.chunks * H + 7) / 8 * 8 : p.chunks * H;
  p.workgroups = items * p.row_tiles;
  p.workspace = 0;
  if (p.split) p.workspace = (B * 8 + 255) / 256 * 256 + p.chunks * per_chunk * p.tile_rows * (d * 4 + 16);
  return p;
}

hipError_t launch_cache_attention(const CacheAttentionArgs& a, hipStream_t stream) {
  const CachePlan plan = cache_plan(a.B, a.c.H, a.G, a.c.d, a.max_q, (int64_t)a.max_pages << a.c.page_shift);
  if (a.c.d == 64 && a.c.fp8) launch_format<64, true>(a, plan, stream);
  else if (a.c.d == 64) launch_format<64, false>(a, plan, stream);
  else if (a.c.fp8) launch_format<128, true>(a, plan, stream);
  else launch_format<128, false>(a, plan, stream);
  return hipGetLastError();
}

}  // namespace fp4attn
