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
__device__ __forceinline__ void fetch_arguments(const CacheAttentionArgs& a, const CachePlan& plan) {
  asm volatile("" ::"s"(a.c.H), "s"(a.B), "s"(a.tree), "s"(plan.ranges));
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

// Units of kUnit keys; at least one, so that rows without keys are written.
__device__ __forceinline__ int units_of(const Sequence& s) { return s.keys == 0 ? 1 : (s.keys + kUnit - 1) / kUnit; }
__device__ __forceinline__ int row_tiles_of(const CacheAttentionArgs& a, const CachePlan& plan, const Sequence& s) {
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
__device__ __forceinline__ Range find_range(const CacheAttentionArgs& a, const CachePlan& plan, int w) {
  const int lane = threadIdx.x & 63;
  Range r{};
  Sequence seq{};  // the lane's
  int own = 0, sum = 0, total = 0;
  auto scan = [&](int b0) {  // own: the sequence's places; sum: inclusive prefix over the lanes
    own = 0;
    if (b0 + lane < a.B) {
      seq = sequence(a, b0 + lane);
      own = row_tiles_of(a, plan, seq) * (units_of(seq) + kSetup);
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
      r.units = units_of(r.seq);
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
  Partials r;
  r.joins = reinterpret_cast<int4*>(w);
  w += (int64_t)p.ranges * 16;
  r.stat = reinterpret_cast<float4*>(w);
  w += (int64_t)p.ranges * 2 * a.c.H * p.tile_rows * 16;
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

// Joins and stores: D / 16 columns from D / 16 * c of row i of the sequence, as output if the
// sequence is whole in this workgroup, else as a piece.  o are sums of probabilities times codes'
// values, `rounded` the sum of the probabilities, ref their base-2 reference, sum the unrounded sum; columns
// whose bit of `odd` is set are NaN (MXFP4: all or none).
template <int D, bool FP8>
__device__ __forceinline__ void store_columns(const CacheAttentionArgs& a, const CachePlan& plan, const Sequence& seq, int i,
                                              int head, int c, bool whole, int64_t piece, float ref, float sum,
                                              float rounded, unsigned odd, const float (&o)[D / 16]) {
  constexpr int kCols = D / 16;
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
    const Partials p = partials(a, plan);
    store_row<kCols>(p.acc + piece * D + c * kCols, x);
    if (c == 0) p.stat[piece] = float4{ref, sum, rounded, 0.0f};
  }
}

// Which range and key head a workgroup takes.  Workgroups are dealt round-robin to eight XCDs;
// neighbouring ranges of a key head go to one of them, whose L2 then holds the keys of a
// sequence while its row tiles are at work.
struct Place {
  int w, head;
};
__device__ __forceinline__ Place place_of(const CachePlan& plan) {
  const int item = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8, head = divide(item, plan.ranges);
  return {item - head * plan.ranges, head};
}

// The workgroup's range, and (from one of its threads) the record for the row tile that crosses
// into it for the first time.
__device__ __forceinline__ Range open_range(const CacheAttentionArgs& a, const CachePlan& plan, const Place& p) {
  Range range{};
  if (plan.split) {
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
    range.units = units_of(range.seq);
    range.end = range.tile < range.tiles ? range.units : 0;
  }
  return range;
}

// Goes on to the next row tile, which begins at place `stop`; false at the end of the range.
__device__ __forceinline__ bool next_tile(const CacheAttentionArgs& a, const CachePlan& plan, int stop, Range& range) {
  if (stop >= range.end) return false;
  if (++range.tile >= range.tiles) {
    range.tile = 0;
    do {
      if (++range.b >= a.B) return false;
      range.seq = sequence(a, range.b);
      range.tiles = row_tiles_of(a, plan, range.seq);
    } while (range.tiles == 0);
    range.units = units_of(range.seq);
  }
  range.at = stop + kSetup;
  return true;
}

// The range's part of its row tile: keys [begin, end).
struct Part {
  int begin, end, stop;  // stop: place of the line where it ends
  bool whole, first;     // all keys of the row tile; its first piece
  int common;            // keys below are seen by every row of the tile
  int tree_tokens;       // new tokens that have a bit in the tree
};
__device__ __forceinline__ bool open_part(const CacheAttentionArgs& a, const CachePlan& plan, const Range& range,
                                          Part* part) {
  const Sequence& seq = range.seq;
  const int from = range.begin > range.at ? range.begin : range.at, seq_end = range.at + range.units;
  part->stop = seq_end < range.end ? seq_end : range.end;
  if (from >= part->stop) return false;  // only places of its setup are left of the range
  part->first = from == range.at;
  part->whole = part->first && part->stop == seq_end;
  part->begin = (from - range.at) * kUnit;
  part->end = part->stop < seq_end ? (part->stop - range.at) * kUnit : seq.keys;
  const int rows = seq.tokens * a.G, row0 = range.tile * plan.tile, row1 = row0 + plan.tile < rows ? row0 + plan.tile : rows;
  if (a.tree) {
    part->common = seq.prefix;
  } else {  // causal: the first and the last row's token
    const int last = seq.prefix + divide(row1 - 1, a.G) + 1;
    part->common = seq.prefix + divide(row0, a.G) + 1;
    part->end = part->end > last ? last : part->end;
  }
  part->common = part->common > seq.keys ? seq.keys : part->common;
  part->tree_tokens = seq.keys - seq.prefix;
  part->tree_tokens = part->tree_tokens > 64 * a.tree_words ? 64 * a.tree_words : part->tree_tokens;
  return true;
}

// Keys key .. key + 7 that a row of token t sees.
__device__ __forceinline__ unsigned row_sees(const CacheAttentionArgs& a, const Sequence& seq, const Part& part, int t,
                                             int key) {
  int limit = a.tree ? seq.prefix : seq.prefix + t + 1;
  limit = limit > seq.keys ? seq.keys : limit;
  return seen8(limit, a.tree + (int64_t)(seq.first + t) * a.tree_words, key, seq.prefix, part.tree_tokens, a.tree_words);
}

}  // namespace fp4attn
