// Device code that the cache attention kernels share: the batch's sequences and how their
// keys are dealt to workgroups, the cache's codes as bf16, masks, partial results.
#pragma once

#include "cache_plan.hpp"
#include "gfx950.hpp"
#include "serving.hpp"

namespace fp4attn {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kTile = 32;   // keys of a wave's step
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

__device__ __forceinline__ unsigned groups_or(unsigned x) {
  auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  x = r[0] | r[1];
  r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return r[0] | r[1];
}

// Largest of a lane's eight scores.
__device__ __forceinline__ float max8(const v4f (&s)[2]) {
  float x = fmaxf(fmaxf(s[0][0], s[0][1]), s[0][2]);
  x = fmaxf(fmaxf(x, s[0][3]), s[1][0]);
  x = fmaxf(fmaxf(x, s[1][1]), s[1][2]);
  return fmaxf(x, s[1][3]);
}

constexpr int kOnes = 0x3f803f80;  // two bf16

// The bf16 probabilities 2^(s factor - ref) of a lane's eight scores; *sum grows by the
// unrounded ones.
__device__ __forceinline__ v4i probabilities(const v4f (&s)[2], float factor, float ref, float* sum) {
  const float base = ref == -__builtin_inff() ? 0.0f : -ref;
  float e[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) e[j] = __builtin_amdgcn_exp2f(fmaf(s[j / 4][j % 4], factor, base));
  *sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
  v4i p;
#pragma unroll
  for (int j = 0; j < 4; ++j) p[j] = (int)__builtin_bit_cast(unsigned, v2bf{(__bf16)e[2 * j], (__bf16)e[2 * j + 1]});
  return p;
}

// The arguments lie in four lines of the scalar cache, each a miss of 0.7 us when it is first used: one
// value of each is read at the start, so that the misses overlap.
template <class Args>
__device__ __forceinline__ void fetch_arguments(const Args& a, const CachePlan& plan) {
  asm volatile("" ::"s"(a.c.H), "s"(a.B), "s"(a.tree), "s"(plan.ranges));
  if constexpr (Args::kShaped) asm volatile("" ::"s"(a.window), "s"(a.prefix_acc));
}

// Of numbers that are not negative (half the instructions of a signed division).
__device__ __forceinline__ int divide(int a, int b) { return (int)((unsigned)a / (unsigned)b); }

// New tokens and keys of a sequence.
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
    s.tokens = a.max_q;  // n = B * max_q
    s.first = b * s.tokens;
    s.keys = a.lengths[b];
    s.prefix = (s.keys < 0 ? 0 : s.keys) - s.tokens;
  }
  const int64_t capacity = (int64_t)a.max_pages << a.c.page_shift;
  s.keys = s.keys < 0 ? 0 : (s.keys > capacity ? (int)capacity : s.keys);
  return s;
}

// Keys at the start of a sequence that its rows have from the shared prefix's pass: those of a sequence whose
// new tokens all come after the prefix.
template <class Args>
__device__ __forceinline__ int shared_keys(const Args& a, const Sequence& s) {
  if constexpr (Args::kShaped && !Args::kPrefix) return s.tokens > 0 && s.prefix >= a.shared && s.keys >= a.shared ? a.shared : 0;
  return 0;
}

// With a window the first key that row tile `tile` sees, or earlier (kUnit-aligned).
template <class Args>
__device__ __forceinline__ int first_key(const Args& a, const CachePlan& plan, const Sequence& s, int tile) {
  if constexpr (Args::kShaped)
    if (a.window) {
      const int low = s.prefix + divide(tile * plan.tile, a.G) + 1 - a.window;
      return low < 0 ? 0 : (low > s.keys ? s.keys : low) & -kUnit;
    }
  return shared_keys(a, s);
}

// Units of kUnit keys that a row tile walks; at least one, so that rows without keys are written.
template <class Args>
__device__ __forceinline__ int units_of(const Args& a, const CachePlan& plan, const Sequence& s) {
  if constexpr (Args::kShaped) {
    const int keys = s.keys - shared_keys(a, s), units = keys == 0 ? 1 : (keys + kUnit - 1) / kUnit;
    // (a prefix that every token sees reaches past the window's end)
    if (a.window == 0 || a.open_keys) return units;
    const int span = window_units(plan.tile, a.G, a.window);
    return units < span ? units : span;
  }
  return s.keys == 0 ? 1 : (s.keys + kUnit - 1) / kUnit;
}
template <class Args>
__device__ __forceinline__ int row_tiles_of(const Args& a, const CachePlan& plan, const Sequence& s) {
  return (s.tokens * a.G + plan.tile - 1) >> __builtin_ctz(plan.tile);
}

// The row tiles of all sequences laid end to end in one line, each as kSetup places for what
// starting one costs and then its keys' units; range w takes places [w per, (w + 1) per): equal parts
// for every workgroup, whatever the lengths and the numbers of rows.  A causal row tile has places for all keys of its
// sequence and walks those up to its last row's: of the last 2048 of 8192 tokens the busiest workgroup has 1.14 times
// the mean work, of a prompt of 8192 twice.  (Places to a start, 64 sequences of 128 to
// 16384 keys: 4 47.9 us, 3 47.3, 2 48.3, 1 50.5; trees of 16 tokens over 8 of 2047 keys: 22.6, 22.2, 24.2, 25.0.)
struct Range {
  int begin, end;
  int b, tile, tiles;  // a row tile of the range, of the sequence's `tiles`
  int at, units;       // its units are at places [at, at + units)
  Sequence seq;
  int per;
  int piece;  // of the shared prefix
  int rest;   // beside direct ranges: the first other range of its row tile, and the one in whose slots it leaves its own piece
  int slot;
};

// Inclusive prefix sum over the wave's lanes: within rows of 16, then across them.
__device__ __forceinline__ int prefix_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr 1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15: rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast 31: rows 2 and 3
  return x;
}

// Every wave finds its range by itself, 64 sequences at a time.
template <class Args>
__device__ __forceinline__ Range find_range(const Args& a, const CachePlan& plan, int w) {
  const int lane = threadIdx.x & 63;
  Range r{};
  Sequence seq{};  // the lane's
  int own = 0, sum = 0, total = 0;
  auto scan = [&](int b0) {  // own: the sequence's places; sum: inclusive prefix over the lanes
    own = 0;
    if (b0 + lane < a.B) {
      seq = sequence(a, b0 + lane);
      own = row_tiles_of(a, plan, seq) * (units_of(a, plan, seq) + kSetup);
    }
    sum = prefix_sum(own);
  };
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    scan(b0);
    total += __builtin_amdgcn_readlane(sum, 63);
  }
  r.per = divide(total + plan.ranges - 1, plan.ranges);
  r.per = r.per < plan.min_units ? plan.min_units : r.per;
  r.begin = w * r.per;
  r.end = r.begin + r.per < total ? r.begin + r.per : total;
  if (r.begin >= total) return r;  // empty: begin >= end
  for (int b0 = 0, before = 0;; b0 += 64) {
    if (a.B > 64) scan(b0);
    const int from = before + sum - own;
    const uint64_t found = __ballot(r.begin >= from && r.begin < from + own);
    if (found) {  // once, as begin < total
      const int src = __ffsll((unsigned long long)found) - 1;
      r.b = b0 + src;
      r.seq.first = __builtin_amdgcn_readlane(seq.first, src);
      r.seq.tokens = __builtin_amdgcn_readlane(seq.tokens, src);
      r.seq.keys = __builtin_amdgcn_readlane(seq.keys, src);
      r.seq.prefix = __builtin_amdgcn_readlane(seq.prefix, src);
      r.units = units_of(a, plan, r.seq);
      r.tiles = row_tiles_of(a, plan, r.seq);
      const int start = __builtin_amdgcn_readlane(from, src), places = r.units + kSetup;
      r.tile = divide(r.begin - start, places);
      r.at = start + r.tile * places + kSetup;
      return r;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
    if (b0 + 64 >= a.B) return r;
  }
}

// Beside direct ranges: row tiles of more than direct_units units are cut after every `per` units, whose size leaves as many pieces as
// there are other ranges.  The row tile's own range takes the first, the others the rest, in the order of the sequences.  The range of
// piece w of those, or (w < 0) of the first piece of row tile `tile` of sequence b.
template <class Args>
__device__ __forceinline__ Range find_cut(const Args& a, const CachePlan& plan, int w, int b, int tile) {
  const int lane = threadIdx.x & 63, ranges = plan.ranges - plan.direct;
  Range r{};
  Sequence seq{};  // the lane's
  const int total = a.arrived[a.crossings];  // (look_for_long)
  if (total == 0) return r;  // empty
  r.per = divide(total + ranges - 1, ranges);
  r.per = r.per < plan.min_units ? plan.min_units : r.per;
  for (int b0 = 0, before = 0; b0 < a.B; b0 += 64) {
    int units = 0, tiles = 0;
    if (b0 + lane < a.B) {
      seq = sequence(a, b0 + lane);
      units = units_of(a, plan, seq);
      tiles = units > a.direct_units ? row_tiles_of(a, plan, seq) : 0;
    }
    const int rests = divide(units + r.per - 1, r.per) - 1, own = tiles * rests, sum = prefix_sum(own);  // (units are at least 1 where tiles are)
    const int from = before + sum - own;
    const uint64_t found = __ballot(w < 0 ? b0 + lane == b : w >= from && w < from + own);
    if (found) {
      const int src = __ffsll((unsigned long long)found) - 1;
      r.b = b0 + src;
      r.seq.first = __builtin_amdgcn_readlane(seq.first, src);
      r.seq.tokens = __builtin_amdgcn_readlane(seq.tokens, src);
      r.seq.keys = __builtin_amdgcn_readlane(seq.keys, src);
      r.seq.prefix = __builtin_amdgcn_readlane(seq.prefix, src);
      r.units = __builtin_amdgcn_readlane(units, src);
      const int start = __builtin_amdgcn_readlane(from, src), n = __builtin_amdgcn_readlane(rests, src);
      r.tile = w < 0 ? tile : divide(w - start, n);
      r.rest = start + r.tile * n;
      r.slot = w < 0 ? r.rest : w;
      r.begin = w < 0 ? 0 : (w - r.rest + 1) * r.per;
      r.end = r.begin + r.per < r.units ? r.begin + r.per : r.units;
      if (r.rest + n > ranges) r.end = r.begin;  // (only if the lengths were changed after the prefix's pass)
      return r;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  return r;  // empty
}

// Partial results in the workspace.  A row tile that crosses from range to range leaves a
// piece in each: its first in slot 1 of its range, the others in slot 0 of theirs.  joins[w], of
// the row tile whose first crossing is into range w: its pieces (0: there is none), its sequence's first
// token and rows, its number.  Then per row of a slot (range, side, key head): {reference, sum,
// sum of the rounded values}, and the accumulators.
struct Partials {
  int4* joins;
  float4* stat;
  float* acc;
};
__device__ __forceinline__ Partials partials(const CacheAttentionArgs& a, const CachePlan& p) {
  char* w = static_cast<char*>(a.workspace);
  const int64_t ranges = p.ranges - p.direct;
  Partials r;
  r.joins = reinterpret_cast<int4*>(w);
  w += ranges * 16;
  r.stat = reinterpret_cast<float4*>(w);
  w += ranges * 2 * a.c.H * p.tile_rows * 16;
  r.acc = reinterpret_cast<float*>(w);
  return r;
}
__device__ __forceinline__ int64_t partial_row(const CacheAttentionArgs& a, const CachePlan& p, int w, int side, int head) {
  return (((int64_t)w * 2 + side) * a.c.H + head) * p.tile_rows;
}

// N consecutive values.
template <int N>
__device__ __forceinline__ void store_row(float* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    reinterpret_cast<float4*>(p)[i] = float4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
}
template <int N>
__device__ __forceinline__ void store_row(uint16_t* p, const float (&v)[N]) {
  static_assert(N == 4 || N == 8, "8 or 16 bytes");
  unsigned w[N / 2];
#pragma unroll
  for (int j = 0; j < N / 2; ++j) w[j] = __builtin_bit_cast(unsigned, v2bf{(__bf16)v[2 * j], (__bf16)v[2 * j + 1]});
  if constexpr (N == 8) *reinterpret_cast<uint4*>(p) = uint4{w[0], w[1], w[2], w[3]};
  else *reinterpret_cast<uint2*>(p) = uint2{w[0], w[1]};
}

// Values that workgroups of other XCDs read in the same launch: stores that go through to the memory that all XCDs share, loads from there.
template <int N>
__device__ __forceinline__ void store_through(float* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i)
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p) + i, (uint64_t)as_uint(v[2 * i + 1]) << 32 | as_uint(v[2 * i]), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float4 load_through(const float* p) {
  uint64_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) w[i] = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p) + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return float4{as_float((unsigned)w[0]), as_float((unsigned)(w[0] >> 32)), as_float((unsigned)w[1]), as_float((unsigned)(w[1] >> 32))};
}

// Of +0 and -0 only.  (The empty asm keeps it a test of bits: as a comparison of floats the compiler,
// told that there are no NaNs, may choose one that holds for them.)
__device__ __forceinline__ bool is_zero(float x) {
  unsigned bits = as_uint(x);
  asm("" : "+v"(bits));
  return (bits << 1) == 0u;
}

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

// The two pages of a tile (the same one unless pages hold 16 keys); -1: no such page.
// The table is read through the scalar path, whose waits leave the tile loads in flight.
struct Pages {
  int p0, p1;
};
typedef const __attribute__((address_space(4))) int* ScalarInts;
__device__ __forceinline__ Pages find_pages(const CacheAttentionArgs& a, ScalarInts table, int key0) {
  Pages r;
  r.p0 = table[key0 >> a.c.page_shift];
  r.p1 = r.p0;
  if (a.c.page_shift == 4) {
    const int at = (key0 >> 4) + 1;
    r.p1 = table[at < a.max_pages ? at : a.max_pages - 1];
  }
  return r;
}
__device__ __forceinline__ bool is_page(const CacheView& c, int p) { return (unsigned)p < (unsigned)c.page_limit; }

// Row (page, head, place); a missing page reads page 0.
__device__ __forceinline__ int64_t row_of(const CacheView& c, int page, int head, int place) {
  return (((int64_t)(is_page(c, page) ? page : 0) * c.H + head) << c.page_shift) + place;
}
// First row of the tile for the lanes of its lower and of its upper 16 keys: the same
// one, or with pages of 16 keys 16 rows before the second page's, so that a lane's
// offset is the same either way.
__device__ __forceinline__ int64_t base_row(const CacheView& c, const Pages& pages, int key0, int head, bool upper) {
  const int64_t row = row_of(c, pages.p0, head, key0 & ((1 << c.page_shift) - 1));
  if (c.page_shift != 4) return row;
  return upper ? row_of(c, pages.p1, head, 0) - 16 : row;
}

// The E8M0 byte as the converter's scale operand: a float's exponent field.
__device__ __forceinline__ float scale_of(unsigned byte) { return as_float(byte << 23); }
template <int J>
__device__ __forceinline__ float scale_of_key(const unsigned (&vs)[2]) {  // byte J of the two words
  const unsigned w = vs[J / 4];
  if constexpr (J % 4 == 3) return as_float(w >> 1 & 0x7f800000u);
  else return as_float(w << (23 - 8 * (J % 4)) & 0x7f800000u);
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

// The top bits of those bytes of w that are E4M3's NaN codes, 0x7f and 0xff (carries stay in their bytes).
__device__ __forceinline__ unsigned nan_codes(unsigned w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ unsigned without_nan_codes(unsigned w) {
  const unsigned n = nan_codes(w);
  return w & ~(n | (n - (n >> 7)));
}

// Of the D / 4 output columns that lane group g holds, D / 16 * (4 g + i) + t as bit D / 16 * i + t, those in which
// key `key` of eight keys' V is no number: all under a huge scale (they lie in one block), else those of NaN codes.
template <int D, bool FP8>
__device__ __forceinline__ unsigned odd_columns(const CacheView& c, int64_t group, int key, int g) {
  constexpr int kCols = D / 16, kBlocks = D / 32;
  if (c.v_scales[(group * kBlocks + g * kBlocks / 4) * 8 + key] >= kHugeScale<FP8>) return ~0u;
  unsigned odd = 0;
  if constexpr (FP8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint8_t* p = c.v_codes + ((group * 16 + 4 * g + i) * 8 + key) * kCols;
#pragma unroll
      for (int j = 0; j < kCols / 4; ++j)  // (the product gathers the four bytes' bits at 24 .. 27, no two terms meet)
        odd |= (nan_codes(reinterpret_cast<const unsigned*>(p)[j]) >> 7) * 0x01020408u >> 24 << (kCols * i + 4 * j);
    }
  }
  return odd;
}

// Which of keys key .. key + 7 a row sees, as bits: those under `limit`, and of the new
// tokens those in its words of the tree (none if words = 0).  Straight-line code: loads are
// clamped to the row's words instead of branched around.
__device__ __forceinline__ unsigned below(int n) { return (1u << (n < 0 ? 0 : (n > 8 ? 8 : n))) - 1u; }
__device__ __forceinline__ unsigned seen8(int limit, const int64_t* bits, int key, int prefix, int tokens, int words) {
  unsigned see = below(limit - key);
  if (words) {  // uniform
    const int u = key - prefix, at = u >> 6, shift = u & 63;
    const int i = at < 0 ? 0 : (at >= words ? words - 1 : at), k = i + 1 < words ? i + 1 : i;
    const uint64_t lo = (uint64_t)bits[i], hi = (uint64_t)bits[k];
    const unsigned inside = (unsigned)(lo >> shift) | (shift > 56 ? (unsigned)(hi << (64 - shift)) : 0u);
    const unsigned up = u > -8 ? (unsigned)lo << (-u & 7) : 0u;  // the first new token is key - u
    see |= (u < 0 ? up : inside) & below(tokens - u);
  }
  return see;
}

// Columns (odd_columns) that a lane's rows see a V in that is no number.  MXFP4 has only whole blocks of them,
// a bit for each row (with a word each, 32 trees of 64 tokens took 365 us instead of 362).
template <bool FP8, int NR>
struct OddMarks {
  unsigned w[FP8 ? NR : 1] = {};
  __device__ __forceinline__ void add(int r, bool sees, unsigned columns) {
    if constexpr (FP8) w[r] |= sees ? columns : 0u;
    else w[0] |= columns & (unsigned)sees << r;
  }
  // D / 16 columns from i-th of four; MXFP4: not zero for all
  template <int COLS>
  __device__ __forceinline__ unsigned of(int r, int i) const {
    return FP8 ? w[r] >> COLS * i : w[0] >> r & 1;
  }
};

// Adds piece k of the shared prefix to what a lane holds of a row (of q and head h): columns D / 16 * (4 g + i) + t in
// register i of product t.  lower: what the bias by distance takes off the piece's reference, which its pass counts
// from the prefix's end.
template <int D, class Args>
__device__ __forceinline__ void add_piece(const Args& a, int k, int64_t row, int g, float lower, float* ref, float* sum, v4f* sum16,
                                          v4f (&acc)[D / 16]) {
  constexpr int kCols = D / 16;
  const int64_t at = k * (a.n * a.Hq) + row;
  const float4 s = a.prefix_stat[at];
  float4 x[4][kCols / 4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < kCols / 4; ++j) x[i][j] = reinterpret_cast<const float4*>(a.prefix_acc + at * D + (4 * g + i) * kCols)[j];
  const float its_ref = s.x - lower, top = fmaxf(*ref, its_ref);
  const float mine = *ref == top ? 1.0f : __builtin_amdgcn_exp2f(*ref - top);
  const float its = its_ref == top ? 1.0f : __builtin_amdgcn_exp2f(its_ref - top);
  *ref = top;
  *sum = *sum * mine + (g == 0 ? s.y * its : 0.0f);  // (the lane groups' sums are added up later)
  *sum16 = *sum16 * mine + s.z * its;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < kCols / 4; ++j) {
      acc[4 * j][i] = acc[4 * j][i] * mine + x[i][j].x * its;
      acc[4 * j + 1][i] = acc[4 * j + 1][i] * mine + x[i][j].y * its;
      acc[4 * j + 2][i] = acc[4 * j + 2][i] * mine + x[i][j].z * its;
      acc[4 * j + 3][i] = acc[4 * j + 3][i] * mine + x[i][j].w * its;
    }
}

// Joins and stores: D / 16 columns from D / 16 * c of row i of the sequence, as output if the
// sequence is whole in this workgroup, else as a piece.  o are sums of probabilities times codes'
// values, `rounded` the sum of the probabilities, ref their base-2 reference, sum the unrounded sum; columns
// whose bit of `odd` is set are NaN (MXFP4: all or none).
template <int D, bool FP8, class Args>
__device__ __forceinline__ void store_columns(const Args& a, const CachePlan& plan, const Sequence& seq, int i, int head, int c,
                                              bool whole, int64_t piece, float ref, float sum, float rounded, unsigned odd,
                                              const float (&o)[D / 16]) {
  constexpr int kCols = D / 16;
  if constexpr (Args::kPrefix) {  // a piece of row (token, head) of the batch
    const int t = divide(i, a.G);
    piece += (int64_t)(seq.first + t) * a.Hq + head * a.G + (i - t * a.G);
  }
  const bool empty = is_zero(rounded);
  const float norm = whole ? (empty ? 0.0f : (FP8 ? 1.0f : 1.0f / 6.0f) / rounded) : 1.0f;
  float x[kCols];
  unsigned nan = 0x7fc00000u;  // as bits: a compiler told that there are no NaNs may drop the choice of one
  asm("" : "+v"(nan));
#pragma unroll
  for (int j = 0; j < kCols; ++j) x[j] = as_float((FP8 ? odd >> j & 1 : odd) ? nan : as_uint(o[j] * norm));
  if (whole) {
    const int t = divide(i, a.G);
    const int64_t at = (int64_t)(seq.first + t) * a.Hq + head * a.G + (i - t * a.G);
    if (a.out_bf16) store_row<kCols>(static_cast<uint16_t*>(a.out) + at * D + c * kCols, x);
    else store_row<kCols>(static_cast<float*>(a.out) + at * D + c * kCols, x);
    if (a.lse && c == 0) a.lse[at] = log_norm(ref, sum);
  } else {
    float4* stat;
    float* acc;
    if constexpr (Args::kPrefix) {
      stat = a.prefix_stat;
      acc = a.prefix_acc;
    } else {
      const Partials p = partials(a, plan);
      stat = p.stat;
      acc = p.acc;
    }
    if constexpr (Args::kDirect) {
      store_through(acc + piece * D + c * kCols, x);
      if (c == 0) store_through(&stat[piece].x, {ref, sum, rounded, 0.0f});
    } else {
      store_row<kCols>(acc + piece * D + c * kCols, x);
      if (c == 0) stat[piece] = float4{ref, sum, rounded, 0.0f};
    }
  }
}

// A row's partial state {reference, sum, sum of the rounded values}, four columns in each lane.
struct RowState {
  float ref = -__builtin_inff(), sum = 0.0f, sum16 = 0.0f;
  float4 acc = {0, 0, 0, 0};
  __device__ __forceinline__ void add(const float4& s, const float4& o) {
    const float top = fmaxf(ref, s.x);
    const float mine = ref == top ? 1.0f : __builtin_amdgcn_exp2f(ref - top);
    const float its = s.x == top ? 1.0f : __builtin_amdgcn_exp2f(s.x - top);
    ref = top;
    sum = sum * mine + s.y * its;
    sum16 = sum16 * mine + s.z * its;
    acc = float4{acc.x * mine + o.x * its, acc.y * mine + o.y * its, acc.z * mine + o.z * its, acc.w * mine + o.w * its};
  }
};
// Adds pieces k, k + step .. of `pieces` of row `in_tile` of the row tile whose first crossing is into range w.
template <int D>
__device__ __forceinline__ void add_pieces(const CacheAttentionArgs& a, const CachePlan& plan, const Partials& part, int w, int head,
                                           int in_tile, int lane, int k, int step, int pieces, RowState& state) {
#pragma unroll 4
  for (; k < pieces; k += step) {
    const int64_t at = partial_row(a, plan, w - 1 + k, k == 0 ? 1 : 0, head) + in_tile;
    state.add(part.stat[at], reinterpret_cast<const float4*>(part.acc + at * D)[lane]);
  }
}
// Stores row i of a sequence whose first token is `first`.
template <int D, bool FP8>
__device__ __forceinline__ void store_state(const CacheAttentionArgs& a, const RowState& s, int first, int i, int head, int lane) {
  const int t = divide(i, a.G);
  const int64_t at = (int64_t)(first + t) * a.Hq + head * a.G + (i - t * a.G);
  const bool empty = is_zero(s.sum16);
  const float norm = (FP8 ? 1.0f : 1.0f / 6.0f) / s.sum16;
  const float o[4] = {empty ? 0.0f : s.acc.x * norm, empty ? 0.0f : s.acc.y * norm, empty ? 0.0f : s.acc.z * norm,
                      empty ? 0.0f : s.acc.w * norm};
  const int64_t to = at * D + lane * 4;
  if (a.out_bf16) store_row<4>(static_cast<uint16_t*>(a.out) + to, o);
  else store_row<4>(static_cast<float*>(a.out) + to, o);
  if (a.lse && lane == 0) a.lse[at] = log_norm(s.ref, s.sum);
}

// Which range and key head a workgroup takes.  Workgroups are dealt round-robin to eight XCDs;
// neighbouring ranges of a key head go to one of them, whose L2 then holds the keys of a
// sequence while its row tiles are at work.
struct Place {
  int w, head;
  bool tile;  // it is a row tile's own
};
template <class Args>
__device__ __forceinline__ Place place_of(const Args& a, const CachePlan& plan) {
  int block = blockIdx.x, grid = gridDim.x, ranges = plan.ranges;
  bool tile = !plan.split;
  if constexpr (Args::kPrefix) {  // the last eight have no range
    grid -= 8;
    if (block >= grid) return {block - grid, a.c.H, false};
  }
  if constexpr (Args::kDirect) {  // those of each kind over all XCDs
    const int direct = (plan.direct * a.c.H + 7) & ~7;
    tile = block < direct;
    block -= tile ? 0 : direct;
    grid = tile ? direct : grid - direct;
    ranges = tile ? plan.direct : ranges - plan.direct;
  }
  const int item = block % 8 * (grid / 8) + block / 8, head = divide(item, ranges);
  return {item - head * ranges, head, tile};
}
// Whether a workgroup comes in the second half of those of its kind that fill the chip.
template <class Args>
__device__ __forceinline__ bool in_second_half(const Args& a, const CachePlan& plan) {
  const unsigned all = Args::kDirect ? (unsigned)(plan.direct * a.c.H) : gridDim.x - (Args::kPrefix ? 8 : 0);
  return blockIdx.x >= all / 2;
}

// For the sequences' own pass with direct ranges, by a workgroup of the shared prefix's that has no range: the units of its row tiles
// of more than direct_units (mostly none: then the ranges beside the direct ones end at once), and no piece of them is there yet.
template <class Args>
__device__ __forceinline__ void look_for_long(const Args& a) {
  if (a.arrived == nullptr) return;
  __shared__ int lds[kWaves];
  int units = 0;
  for (int b = threadIdx.x; b < a.B; b += kThreads) {
    const Sequence s = sequence(a, b);
    const int its = (s.keys + kUnit - 1) / kUnit;
    const bool joins = s.prefix >= a.shared && s.keys >= a.shared;  // (then it has at most direct_units of its own)
    if (!joins && its > a.direct_units) units += divide(s.tokens * a.G + a.own_tile - 1, a.own_tile) * its;
  }
  units = prefix_sum(units);
  if ((threadIdx.x & 63) == 63) lds[threadIdx.x / 64] = units;
  for (int i = threadIdx.x; i < a.crossings; i += kThreads) a.arrived[i] = 0;
  __syncthreads();
  if (threadIdx.x == 0) a.arrived[a.crossings] = lds[0] + lds[1] + lds[2] + lds[3];
}

// The workgroup's range of the shared prefix: piece w / row_tiles of row tile w % row_tiles of all tokens
// together.  Its pages are those of the first sequence that joins it (if there is none, the range is empty).
template <class Args>
__device__ __forceinline__ Range open_prefix(const Args& a, const CachePlan& plan, const Place& p) {
  Range range{};
  const int lane = threadIdx.x & 63;
  int b = -1;
  for (int b0 = 0; b0 < a.B && b < 0; b0 += 64) {
    bool joins = false;
    if (b0 + lane < a.B) {
      const Sequence seq = sequence(a, b0 + lane);
      joins = seq.tokens > 0 && seq.prefix >= a.shared && seq.keys >= a.shared;
    }
    const uint64_t found = __ballot(joins);
    if (found) b = b0 + __ffsll((unsigned long long)found) - 1;
  }
  range.piece = divide(p.w, plan.row_tiles);
  range.tile = p.w - range.piece * plan.row_tiles;
  range.b = b;
  range.tiles = 1;
  int64_t tokens = a.n;
  if (a.q_starts) {  // rows past the last sequence's belong to none
    const int last = a.q_starts[a.B];
    tokens = last < 0 ? 0 : (last < tokens ? last : tokens);
  }
  range.seq = Sequence{0, (int)tokens, a.shared, a.shared};
  range.units = a.shared / kUnit;
  range.begin = range.piece * a.prefix_units;
  range.end = range.begin + a.prefix_units < range.units ? range.begin + a.prefix_units : range.units;
  if (b < 0 || (int64_t)range.tile * plan.tile >= tokens * a.G) range.end = range.begin;
  return range;
}

// The workgroup's range, and (from one of its threads) the record for the row tile that crosses
// into it for the first time.
template <class Args>
__device__ __forceinline__ Range open_range(const Args& a, const CachePlan& plan, const Place& p) {
  if constexpr (Args::kPrefix) return open_prefix(a, plan, p);
  Range range{};
  if constexpr (Args::kDirect)
    if (!p.tile) return find_cut(a, plan, p.w, 0, 0);
  if (!p.tile) {
    range = find_range(a, plan, p.w);
    if (p.head == 0 && threadIdx.x == 0) {
      int4 join = {0, 0, 0, 0};
      if (range.begin < range.end && range.begin > range.at && range.at >= range.begin - range.per)
        join = int4{divide(range.at + range.units - 1, range.per) - p.w + 2, range.seq.first, range.seq.tokens * a.G, range.tile};
      partials(a, plan).joins[p.w] = join;
    }
  } else {  // range w: row tile w % row_tiles of sequence w / row_tiles
    range.b = divide(p.w, plan.row_tiles);
    range.tile = p.w - range.b * plan.row_tiles;
    range.seq = sequence(a, range.b);
    range.tiles = row_tiles_of(a, plan, range.seq);
    range.units = units_of(a, plan, range.seq);
    range.end = range.tile < range.tiles ? range.units : 0;
    if constexpr (Args::kDirect)
      if (range.end > a.direct_units) return find_cut(a, plan, -1, range.b, range.tile);
  }
  return range;
}

// The range's part of its row tile: keys [begin, end).
struct Part {
  int begin, end, stop;  // stop: place of the line where it ends
  bool whole, first;     // all keys of the row tile; its first piece
  int common;            // keys below are seen by every row of the tile (from `from` on)
  int tree_tokens;       // new tokens that have a bit in the tree
  int low, from;         // with a window: keys below are seen by no row, by not every row
};
// Where a row of the range's row tile (for the shared prefix: any row, store_columns adds its number) has its piece.
template <class Args>
__device__ __forceinline__ int64_t piece_row(const Args& a, const CachePlan& plan, const Range& range, const Place& place,
                                             const Part& part, int row) {
  if constexpr (Args::kPrefix) return range.piece * a.n * a.Hq;
  else return partial_row(a, plan, Args::kDirect ? range.slot : place.w, part.first ? 1 : 0, place.head) + row;
}

// Goes on to the next row tile, which begins at place `stop`; false at the end of the range.
template <class Args>
__device__ __forceinline__ bool next_tile(const Args& a, const CachePlan& plan, int stop, Range& range) {
  if (Args::kPrefix || stop >= range.end) return false;
  if (++range.tile >= range.tiles) {
    range.tile = 0;
    do {
      if (++range.b >= a.B) return false;
      range.seq = sequence(a, range.b);
      range.tiles = row_tiles_of(a, plan, range.seq);
    } while (range.tiles == 0);
    range.units = units_of(a, plan, range.seq);
  }
  range.at = stop + kSetup;
  return true;
}

template <class Args>
__device__ __forceinline__ bool open_part(const Args& a, const CachePlan& plan, const Range& range, Part* part) {
  const Sequence& seq = range.seq;
  const int from = range.begin > range.at ? range.begin : range.at, seq_end = range.at + range.units;
  part->stop = seq_end < range.end ? seq_end : range.end;
  if (from >= part->stop) return false;  // only places of its setup are left of the range
  part->first = from == range.at;
  part->whole = part->first && part->stop == seq_end;
  const int key0 = first_key(a, plan, seq, range.tile);
  part->begin = key0 + (from - range.at) * kUnit;
  part->end = part->stop < seq_end ? key0 + (part->stop - range.at) * kUnit : seq.keys;
  part->low = part->from = 0;
  const int rows = seq.tokens * a.G, row0 = range.tile * plan.tile, row1 = row0 + plan.tile < rows ? row0 + plan.tile : rows;
  if (a.tree) {
    part->common = seq.prefix;
  } else {  // causal: the first and the last row's token
    int last = seq.prefix + divide(row1 - 1, a.G) + 1;
    part->common = seq.prefix + divide(row0, a.G) + 1;
    if constexpr (Args::kShaped) {
      if (a.window) {
        part->low = part->common - a.window;
        part->from = last - a.window;
      }
      if (a.open_keys) {
        const int open = a.open_keys[range.b];
        last = last > open ? last : open;
        part->common = part->common > open ? part->common : open;
      }
    }
    part->end = part->end > last ? last : part->end;
  }
  // (a window's units may reach past the keys, and a prefix may be longer than they are)
  if constexpr (Args::kShaped) part->end = part->end > seq.keys ? seq.keys : part->end;
  part->common = part->common > seq.keys ? seq.keys : part->common;
  part->tree_tokens = seq.keys - seq.prefix;
  part->tree_tokens = part->tree_tokens > 64 * a.tree_words ? 64 * a.tree_words : part->tree_tokens;
  return true;
}

// Keys key .. key + 7 that a row of token t of sequence b sees.
template <class Args>
__device__ __forceinline__ unsigned row_sees(const Args& a, const Sequence& seq, const Part& part, int b, int t, int key) {
  int limit = a.tree ? seq.prefix : seq.prefix + t + 1;
  unsigned hidden = 0;
  if constexpr (Args::kShaped) {
    if (a.window) hidden = below(limit - a.window - key);
    if (a.open_keys) {
      const int open = a.open_keys[b];
      limit = limit > open ? limit : open;
    }
  }
  limit = limit > seq.keys ? seq.keys : limit;
  return ~hidden & seen8(limit, a.tree + (int64_t)(seq.first + t) * a.tree_words, key, seq.prefix, part.tree_tokens, a.tree_words);
}

// Whether keys [key, key + n) hide one from some row of the tile (their pages aside).
template <class Args>
__device__ __forceinline__ bool some_hidden(const Args& a, const Part& part, int key, int n) {
  return key + n > part.common || (Args::kShaped && key < part.from);
}
// Of keys key .. key + 7 below `end`, those that some row may see.
template <class Args>
__device__ __forceinline__ unsigned may_see(const Args& a, const Part& part, int end, int key) {
  unsigned see = below(end - key);
  if constexpr (Args::kShaped) see &= ~below(part.low - key);
  return see;
}

// Beside direct ranges: the workgroup has stored a piece of its row tile, and the last of the row tile's to do so joins them, in their
// order.  (A launch for it, as of a plan that is split, would take 4 us in every call; few have such a row tile.)
template <int D, bool FP8, class Args>
__device__ __forceinline__ void join_last(const Args& a, const CachePlan& plan, const Range& range, const Place& place, unsigned* lds) {
  const int pieces = divide(range.units + range.per - 1, range.per);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // every wave's stores are through, before the count
  __syncthreads();
  if (threadIdx.x == 0) *lds = atomicAdd(a.arrived + range.rest * a.c.H + place.head, 1) == pieces - 1;
  __syncthreads();
  if (*lds == 0) return;
  const Partials part = partials(a, plan);
  const int lane = threadIdx.x % (D / 4), row0 = range.tile * plan.tile, rows = range.seq.tokens * a.G - row0;
  constexpr int kAhead = 8;  // loads in flight
  for (int row = threadIdx.x / (D / 4); row < rows && row < plan.tile; row += kThreads / (D / 4)) {
    RowState state;
    for (int k0 = 0; k0 < pieces; k0 += kAhead) {
      float4 stat[kAhead], acc[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int k = k0 + j < pieces ? k0 + j : pieces - 1;
        const int64_t at = partial_row(a, plan, range.rest + (k == 0 ? 0 : k - 1), k == 0 ? 1 : 0, place.head) + row;
        stat[j] = load_through(&part.stat[at].x);
        acc[j] = load_through(part.acc + at * D + 4 * lane);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (k0 + j < pieces) state.add(stat[j], acc[j]);
    }
    store_state<D, FP8>(a, state, range.seq.first, row0 + row, place.head, lane);
  }
}

// How a product of codes s = q . k becomes the exponent of a probability, in binades.  Plain: times `factor`.  Shaped, scores
// are replaced by y = C tanh(x) - slope |distance| with x = z / c, z = softmax_scale q . k, C = c log2(e) (capped), or by z log2(e)
// less the bias; their factor is then 1.
struct ScoreShape {
  float factor;  // of what the scores are
  float plain;   // of a product without a cap
};
template <bool FP8, class Args>
__device__ __forceinline__ ScoreShape score_shape(const Args& a) {
  ScoreShape s{};
  s.factor = a.softmax_scale * kLog2e * (FP8 ? 1.0f : 1.0f / 6.0f);
  if constexpr (Args::kScores) {
    s.plain = s.factor;
    if (a.cap.on || a.slopes) s.factor = 1.0f;
  }
  return s;
}
// The slope of a query head in binades.
template <class Args>
__device__ __forceinline__ float slope_of(const Args& a, int head) {
  if constexpr (Args::kScores)
    if (a.slopes) return a.slopes[head] * kLog2e;
  return 0.0f;
}
// The place of a token that distances count from: in the pass over a shared prefix its end, for all tokens.
template <class Args>
__device__ __forceinline__ int place_of_token(const Sequence& seq, int token) {
  return Args::kPrefix ? seq.keys : seq.prefix + token;
}

// The cap's form near zero, y K(y^2).
__device__ __forceinline__ float cap_form(const CapShape& c, float y) {
  const float u = y * y;
  return y * fmaf(fmaf(fmaf(fmaf(c.k[4], u, c.k[3]), u, c.k[2]), u, c.k[1]), u, c.k[0]);
}
// Capped scores of N times eight products, where |s| is at most cap.near: 7 instructions a score.  Returns the largest |s|.
template <class Args, int N>
__device__ __forceinline__ float cap_near(const Args& a, v4f (&s)[N][2]) {
  float most = 0.0f;
#pragma unroll
  for (int r = 0; r < N; ++r)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = s[r][j / 4][j % 4];
      most = fmaxf(most, fabsf(x));
      s[r][j / 4][j % 4] = cap_form(a.cap, x);
    }
  return most;
}
// Of any products: the same value for those, and beyond the edge C tanh(x) = C (1 - 2 / (e^2x + 1)), in which nothing cancels.  A score
// is what its own product makes it either way: which of the two a wave takes is decided by all its products, those with keys that no row sees
// (whatever they hold, or LDS holds in their place) and of other rows among them.
template <class Args, int N>
__device__ __forceinline__ void cap_all(const Args& a, v4f (&s)[N][2]) {
  int near = (int)as_uint(a.cap.near);
  asm volatile("" : "+s"(near));  // (unit and edge are formed here, not held in scalar registers through the loop)
  const float unit = near >= 0 ? 1.0f : a.cap.inside, edge = near >= 0 ? as_float(near) : (float)kTanhNear;
#pragma unroll
  for (int r = 0; r < N; ++r)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = s[r][j / 4][j % 4], y = x * unit;
      const float e = __builtin_amdgcn_exp2f(x * a.cap.inside * (2.0f * kLog2e));
      float lo = cap_form(a.cap, y);
      float hi = fmaf(-2.0f * a.cap.most, __builtin_amdgcn_rcpf(e + 1.0f), a.cap.most);
      asm("" : "+v"(lo), "+v"(hi));  // both, and a choice: the compiler made a branch for every score of it
      s[r][j / 4][j % 4] = fabsf(y) <= edge ? lo : hi;
    }
}
// Scores without a cap, in binades.
template <int N>
__device__ __forceinline__ void scale_scores(float factor, v4f (&s)[N][2]) {
#pragma unroll
  for (int r = 0; r < N; ++r)
#pragma unroll
    for (int j = 0; j < 8; ++j) s[r][j / 4][j % 4] *= factor;
}
// Scores without a cap, with the bias of keys key .. key + 7 that lie before their tokens (of later ones: any number).
template <class Args, int N>
__device__ __forceinline__ void scale_with_bias(const Sequence& seq, float factor, const float (&slope)[N], const int (&token)[N],
                                                int key, v4f (&s)[N][2]) {
#pragma unroll
  for (int r = 0; r < N; ++r) {
    const float first = slope[r] * (float)(key - place_of_token<Args>(seq, token[r]));
#pragma unroll
    for (int j = 0; j < 8; ++j) s[r][j / 4][j % 4] = fmaf(s[r][j / 4][j % 4], factor, fmaf(slope[r], (float)j, first));
  }
}
// The bias of keys key .. key + 7.
template <class Args, int N>
__device__ __forceinline__ void add_bias(const Sequence& seq, const float (&slope)[N], const int (&token)[N], int key, v4f (&s)[N][2]) {
#pragma unroll
  for (int r = 0; r < N; ++r) {
    const float far = (float)(place_of_token<Args>(seq, token[r]) - key);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[r][j / 4][j % 4] = fmaf(-slope[r], fabsf(far - (float)j), s[r][j / 4][j % 4]);
  }
}

}  // namespace fp4attn
