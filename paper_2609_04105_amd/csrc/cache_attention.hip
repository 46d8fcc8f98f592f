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
constexpr int kUnit = kTile * kWaves;  // keys of a workgroup's step
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

// Units of kUnit keys of sequence s in row tile `tile`: none without rows there, else at
// least one, so that rows without keys are written.
__device__ __forceinline__ int units_of(const CacheAttentionArgs& a, const CachePlan& plan, const Sequence& s, int tile) {
  if (s.tokens * a.G <= tile * 16 * plan.nr) return 0;
  return s.keys == 0 ? 1 : (s.keys + kUnit - 1) / kUnit;
}

// All sequences laid end to end in one line, each as kSetup places for what starting one costs
// and then its units; range w takes places [w per, (w + 1) per): equal parts for every
// workgroup, whatever the lengths.
constexpr int kSetup = 4;
struct Range {
  int begin, end;
  int b, at, units;  // a sequence of the range: units at places [at, at + units)
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
__device__ __forceinline__ Range find_range(const CacheAttentionArgs& a, const CachePlan& plan, int w, int tile) {
  const int lane = threadIdx.x & 63;
  Range r{};
  Sequence seq{};  // the lane's
  int own = 0, sum = 0, total = 0;
  auto scan = [&](int b0) {  // own: the sequence's places; sum: inclusive prefix over the lanes
    own = 0;
    if (b0 + lane < a.B) {
      seq = sequence(a, b0 + lane);
      own = units_of(a, plan, seq, tile);
      own += own > 0 ? kSetup : 0;
    }
    sum = prefix_sum(own);
  };
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    scan(b0);
    total += __builtin_amdgcn_readlane(sum, 63);
  }
  r.per = (total + plan.ranges - 1) / plan.ranges;
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
      r.units = __builtin_amdgcn_readlane(own, src) - kSetup;
      r.at = __builtin_amdgcn_readlane(from, src) + kSetup;
      r.seq.first = __builtin_amdgcn_readlane(seq.first, src);
      r.seq.tokens = __builtin_amdgcn_readlane(seq.tokens, src);
      r.seq.keys = __builtin_amdgcn_readlane(seq.keys, src);
      r.seq.prefix = __builtin_amdgcn_readlane(seq.prefix, src);
      return r;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
    if (b0 + 64 >= a.B) return r;
  }
}

// Partial results in the workspace.  A sequence that crosses from range to range leaves a
// piece in each: its first in slot 1 of its range, the others in slot 0 of theirs.
// joins[tile][w], of the sequence whose first crossing is into range w: its pieces (0: there is
// none), first token and rows.
// Then per row of a slot (range, side, key head, row tile): {reference, sum, sum of the rounded
// values}, and the accumulators.
struct Partials {
  int4* joins;
  float4* stat;
  float* acc;
};
__device__ __forceinline__ Partials partials(const CacheAttentionArgs& a, const CachePlan& p) {
  char* w = static_cast<char*>(a.workspace);
  Partials r;
  r.joins = reinterpret_cast<int4*>(w);
  w += (int64_t)p.ranges * p.row_tiles * 16;
  r.stat = reinterpret_cast<float4*>(w);
  w += (int64_t)p.ranges * 2 * a.c.H * p.row_tiles * p.tile_rows * 16;
  r.acc = reinterpret_cast<float*>(w);
  return r;
}
__device__ __forceinline__ int64_t partial_row(const CacheAttentionArgs& a, const CachePlan& p, int w, int side, int head,
                                               int tile) {
  return ((((int64_t)w * 2 + side) * a.c.H + head) * p.row_tiles + tile) * p.tile_rows;
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
__device__ __forceinline__ bool is_page(const CacheView& c, int p) { return (unsigned)p < (uint64_t)c.pages; }

// What a lane holds of one 32-key tile, and where it finds it.
template <int D, bool FP8>
struct Tile {
  using F = Format<D, FP8>;
  unsigned k[2][F::kKWords];  // [half] key 8 (m / 4) + 4 half + m % 4, m = lane % 16: values D / 4 * (lane / 16) ..
  unsigned ks[2];             // their E8M0 byte
  unsigned v[F::kVWords];     // keys 8 (lane / 16) .. + 7, values D / 16 * (lane % 16) ..
  unsigned vs[2];             // their eight E8M0 bytes
  static constexpr int kKBytes = F::kKWords * 4, kVBytes = F::kVWords * 4;

  // Row (page, head, place); a missing page reads page 0.
  static __device__ __forceinline__ int64_t row_of(const CacheView& c, int page, int head, int place) {
    return (((int64_t)(is_page(c, page) ? page : 0) * c.H + head) << c.page_shift) + place;
  }
  // First row of the tile for the lanes of its lower and of its upper 16 keys: the same
  // one, or with pages of 16 keys 16 rows before the second page's, so that a lane's
  // offset is the same either way.
  static __device__ __forceinline__ int64_t base_row(const CacheView& c, const Pages& pages, int key0, int head, bool upper) {
    const int64_t row = row_of(c, pages.p0, head, key0 & ((1 << c.page_shift) - 1));
    if (c.page_shift != 4) return row;
    return upper ? row_of(c, pages.p1, head, 0) - 16 : row;
  }
  // The lane's byte offsets in a tile are formed from its number at every load (the empty asm
  // keeps them from being held in registers through the loop).
  __device__ __forceinline__ void load_k(const CacheView& c, const Pages& pages, int key0, int head, int lane) {
    asm volatile("" : "+v"(lane));
    const unsigned m = lane & 15, g = (unsigned)lane >> 4, key = (m >> 2) * 8 + (m & 3);
    const int64_t row = base_row(c, pages, key0, head, m >= 8);
    const uint8_t* kp = c.k_codes + row * (4 * kKBytes) + (key * (4 * kKBytes) + g * kKBytes);
    const uint8_t* ksp = c.k_scales + row * F::kBlocks + (key * F::kBlocks + g * F::kBlocks / 4);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      load_words<F::kKWords>(kp + h * 4 * (4 * kKBytes), k[h]);
      ks[h] = ksp[h * 4 * F::kBlocks];
    }
  }
  __device__ __forceinline__ void load_v(const CacheView& c, const Pages& pages, int key0, int head, int lane) {
    asm volatile("" : "+v"(lane));
    const unsigned m = lane & 15, g = (unsigned)lane >> 4;
    const int64_t row = base_row(c, pages, key0, head, g >= 2);
    load_words<F::kVWords>(c.v_codes + row * (2 * kVBytes) + (unsigned)lane * kVBytes, v);
    const uint2 s = *reinterpret_cast<const uint2*>(c.v_scales + row * F::kBlocks + (g * F::kBlocks + m * F::kBlocks / 16) * 8);
    vs[0] = s.x;
    vs[1] = s.y;
  }
};

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

// Waves per SIMD that the registers are kept to.
constexpr int waves_per_simd(int d, bool fp8, int nr) {
  if (nr == 1) return 3;
  if (nr == 2) return d == 64 ? 3 : 2;
  return d == 64 ? 2 : 1;
}

// Joins the waves' results of one row and D / 16 columns, and stores them: as outputs if the
// sequence is whole here, else as a piece.  lds: [wave][product][row, 4 g + i]; stat: the row's
// {reference, sum, sum of the rounded values} of the first wave, 16 rows apart; poison: its mark,
// 64 words apart.
template <int D, bool FP8>
__device__ __forceinline__ void join_waves(const CacheAttentionArgs& a, const CachePlan& plan, const Sequence& seq,
                                           const float* lds, const float* stat, const unsigned* poison, int i, int c,
                                           int head, bool whole, int64_t piece) {
  constexpr int kCols = D / 16;
  if (i >= seq.tokens * a.G) return;
  float top = -__builtin_inff(), sum = 0.0f, rounded = 0.0f, o[kCols];
  unsigned bad = 0;
#pragma unroll
  for (int j = 0; j < kCols; ++j) o[j] = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stat[w * 64]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float ref = stat[w * 64], part = ref == top ? 1.0f : __builtin_amdgcn_exp2f(ref - top);
    sum += stat[w * 64 + 1] * part;
    rounded += stat[w * 64 + 2] * part;
    bad |= poison[w * 64];
#pragma unroll
    for (int j = 0; j < kCols; ++j) o[j] += lds[(w * kCols + j) * 256 + threadIdx.x] * part;
  }
  const bool empty = is_zero(rounded);
  const float norm = whole ? (empty ? 0.0f : (FP8 ? 1.0f : 1.0f / 6.0f) / rounded) : 1.0f;
#pragma unroll
  for (int j = 0; j < kCols; ++j) o[j] = bad ? as_float(0x7fc00000u) : o[j] * norm;
  if (whole) {
    const int t = i / a.G;
    const int64_t at = (int64_t)(seq.first + t) * a.Hq + head * a.G + (i - t * a.G);
    if (a.out_bf16) store_row<kCols>(static_cast<uint16_t*>(a.out) + at * D + c * kCols, o);
    else store_row<kCols>(static_cast<float*>(a.out) + at * D + c * kCols, o);
    if (a.lse && c == 0) a.lse[at] = log_norm(top, sum);
  } else {
    const Partials p = partials(a, plan);
    store_row<kCols>(p.acc + piece * D + c * kCols, o);
    if (c == 0) p.stat[piece] = float4{top, sum, rounded, 0.0f};
  }
}

// blockIdx.x: (range, key head, row tile)
template <int D, bool FP8, int NR>
__global__ __launch_bounds__(kThreads, waves_per_simd(D, FP8, NR)) void cache_attention_kernel(const CacheAttentionArgs a,
                                                                                              const CachePlan plan) {
  using F = Format<D, FP8>;
  constexpr bool kSharedQ = NR > 1;  // Q operands in LDS: NR * D / 8 registers less
  // the waves' results of one 16-row tile, or Q before them
  constexpr int kAccWords = kWaves * F::kDTiles * 64, kQWords = kSharedQ ? NR * F::kSteps * 64 : 0;
  __shared__ float4 lds[kAccWords > kQWords ? kAccWords : kQWords];
  __shared__ float4 lds_stat[kWaves][16];
  __shared__ unsigned lds_poison[kWaves][64];
  v4i* lds_q = reinterpret_cast<v4i*>(lds);

  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  // Row tiles of one (range, key head) go to one XCD (workgroups are dealt round-robin to
  // eight), which then reads the keys once for all of them.
  int item = blockIdx.x, tile = 0;
  if (plan.row_tiles > 1) {
    const int q = item / 8;
    tile = q % plan.row_tiles;
    item = q / plan.row_tiles * 8 + item % 8;
  }
  const int w = item / a.c.H, head = item - w * a.c.H;
  if (w >= plan.ranges) return;

  Range range{};
  if (plan.split) {
    range = find_range(a, plan, w, tile);
    if (head == 0 && threadIdx.x == 0) {  // the sequence that crosses into this range for the first time
      int4 join = {0, 0, 0, 0};
      if (range.begin < range.end && range.begin > range.at && range.at >= range.begin - range.per)
        join = int4{(range.at + range.units - 1) / range.per - w + 2, range.seq.first, range.seq.tokens * a.G, 0};
      partials(a, plan).joins[tile * plan.ranges + w] = join;
    }
    if (range.begin >= range.end) return;
  } else {
    range.b = w;
    range.seq = sequence(a, w);
    range.units = units_of(a, plan, range.seq, tile);
    range.end = range.units;
    if (range.units == 0) return;
  }
  const float factor = a.softmax_scale * kLog2e * (FP8 ? 1.0f : 1.0f / 6.0f);

  while (true) {
    // The range's part of sequence range.b: keys [begin, end).
    const int from = range.begin > range.at ? range.begin : range.at, seq_end = range.at + range.units;
    const int stop = seq_end < range.end ? seq_end : range.end;
    if (from >= stop) break;  // only places of its setup are left of the range
    const Sequence seq = range.seq;
    const int begin = (from - range.at) * kUnit, end = stop < seq_end ? (stop - range.at) * kUnit : seq.keys;
    const bool whole = from == range.at && stop == seq_end;
    const int rows = seq.tokens * a.G, row0 = tile * 16 * NR;

    // this lane's rows (the same for the four lane groups) and its part of their queries
    int token[NR];  // of the sequence
    v4i q[kSharedQ ? 1 : NR][F::kSteps];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int i = row0 + 16 * r + m, ic = i < rows ? i : rows - 1;
      token[r] = ic / a.G;
      const int h = head * a.G + (ic - token[r] * a.G);
      const uint16_t* p = static_cast<const uint16_t*>(a.q) + (int64_t)(seq.first + token[r]) * a.q_stride + h * D + g * (D / 4);
      if constexpr (kSharedQ) {
        if (r % kWaves == wave || NR < kWaves)
#pragma unroll
          for (int s = 0; s < F::kSteps; ++s) lds_q[(r * F::kSteps + s) * 64 + lane] = reinterpret_cast<const v4i*>(p)[s];
      } else {
#pragma unroll
        for (int s = 0; s < F::kSteps; ++s) q[r][s] = reinterpret_cast<const v4i*>(p)[s];
      }
    }
    if constexpr (kSharedQ) __syncthreads();
    // keys below `common` are seen by every row of the sequence
    int common = a.tree ? seq.prefix : seq.prefix + 1;
    common = common > seq.keys ? seq.keys : common;
    int seen_tokens = seq.keys - seq.prefix;  // that have a bit in the tree
    seen_tokens = seen_tokens > 64 * a.tree_words ? 64 * a.tree_words : seen_tokens;
    auto seen = [&](int r, int key) {
      int limit = a.tree ? seq.prefix : seq.prefix + token[r] + 1;
      limit = limit > seq.keys ? seq.keys : limit;
      return seen8(limit, a.tree + (int64_t)(seq.first + token[r]) * a.tree_words, key, seq.prefix, seen_tokens, a.tree_words);
    };

    v4f acc[NR][F::kDTiles];
    v4f sum16 = {0, 0, 0, 0};  // register r: the rounded probabilities of row tile r
    unsigned poisoned = 0;     // bit r: this lane's columns of row r see a non-finite V block
    float ref[NR], sum[NR];    // base 2, lags the maximum by at most kLag; this lane's own keys
#pragma unroll
    for (int r = 0; r < NR; ++r) {
#pragma unroll
      for (int t = 0; t < F::kDTiles; ++t) acc[r][t] = v4f{0, 0, 0, 0};
      ref[r] = -__builtin_inff();
      sum[r] = 0.0f;
    }
    const ScalarInts table = (ScalarInts)(uintptr_t)(a.page_table + (int64_t)range.b * a.max_pages);

    // The wave's tiles.  One set of registers: a tile's K is loaded when the one before has
    // become scores, its V when the one before is in the accumulators.
    constexpr int kStride = kTile * kWaves;
    int key0 = begin + kTile * wave;
    if (key0 < end) {
      Tile<D, FP8> t;
      Pages pages = find_pages(a, table, key0), next = pages;
      t.load_k(a.c, pages, key0, head, lane);
      t.load_v(a.c, pages, key0, head, lane);
      if (key0 + kStride < end) next = find_pages(a, table, key0 + kStride);
      while (true) {
        const int ahead = key0 + kStride;
        const bool page0 = is_page(a.c, pages.p0), page1 = is_page(a.c, pages.p1);
        const bool masked = key0 + kTile > common || !page0 || !page1;  // uniform
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
            for (int r = 0; r < NR; ++r)
              s[r][h] = mfma_16x16x32(kk, kSharedQ ? lds_q[(r * F::kSteps + st) * 64 + lane] : q[kSharedQ ? 0 : r][st], s[r][h]);
          });
        }
        if (ahead < end) t.load_k(a.c, next, ahead, head, lane);
        if (masked) {
          // Hidden scores become -inf.  Keys that no row sees hold anything: their V codes and
          // scales become zero.  A non-finite V block that some row sees becomes zero too, and
          // marks the rows that see it, whose outputs become NaN after the loop.
          const int base = key0 + 8 * g;
          const unsigned there = (g >= 2 ? page1 : page0) ? below(seq.keys - base) : 0u;
          unsigned see[NR];
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            see[r] = there & seen(r, base);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[r][j / 4][j % 4] = see[r] >> j & 1 ? s[r][j / 4][j % 4] : -__builtin_inff();
          }
          unsigned huge = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool in = there >> j & 1, big = (t.vs[j / 4] >> (8 * (j % 4)) & 255u) >= kHugeScale<FP8>;
            huge |= in && big ? 1u : 0u;
            const unsigned keep = in && !big ? ~0u : 0u;
            t.vs[j / 4] &= keep | ~(255u << (8 * (j % 4)));
            if constexpr (F::kVWords >= 8) {
#pragma unroll
              for (int i = 0; i < F::kVWords / 8; ++i) t.v[j * (F::kVWords / 8) + i] &= keep;
            } else {
              t.v[j / 2] &= keep | (j % 2 ? 0x0000ffffu : 0xffff0000u);
            }
          }
          if (__any(huge)) {  // lane group g holds outputs of d block g (d = 64: g / 2)
#pragma unroll
            for (int r = 0; r < NR; ++r) see[r] = groups_or(see[r] << (8 * g));
            const int blk = g * F::kBlocks / 4;
            for (int k = 0; k < kTile; ++k) {
              const int page = k >= 16 ? pages.p1 : pages.p0, key = key0 + k;
              if (!is_page(a.c, page) || key >= seq.keys) continue;
              const int64_t group = Tile<D, FP8>::row_of(a.c, page, head, key & ((1 << a.c.page_shift) - 1)) >> 3;
              const bool big = a.c.v_scales[(group * F::kBlocks + blk) * 8 + (k & 7)] >= kHugeScale<FP8>;
#pragma unroll
              for (int r = 0; r < NR; ++r) poisoned |= big ? (see[r] >> k & 1) << r : 0u;
            }
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
          for (int j = 0; j < 4; ++j)
            p[r][j] = (int)__builtin_bit_cast(unsigned, v2bf{(__bf16)e[2 * j], (__bf16)e[2 * j + 1]});
          // ones in the rows r, r + 4, r + 8, r + 12 of A: register r of every lane group
          const int one = (lane & 3) == r ? 0x3f803f80 : 0;
          sum16 = mfma_16x16x32(v4i{one, one, one, one}, p[r], sum16);
        }
        // O^T: product t takes value t of every lane's part, rows d = D / 16 * m + t
        float vscale[8];
        static_for<8>([&](auto J_) { vscale[decltype(J_)::value] = scale_of_key<decltype(J_)::value>(t.vs); });
        static_for<F::kDTiles / 2>([&](auto E_) {
          constexpr int e = decltype(E_)::value;  // values 2 e, 2 e + 1 of the part
          unsigned x[8];
          static_for<8>([&](auto J_) {
            constexpr int j = decltype(J_)::value;
            x[j] = code_pair<j * (F::kDTiles / 2) + e, FP8>(t.v, vscale[j]);  // pair e of key j
          });
          v4i lo, hi;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            lo[j] = (int)__builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x05040100u);
            hi[j] = (int)__builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x07060302u);
          }
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            acc[r][2 * e] = mfma_16x16x32(lo, p[r], acc[r][2 * e]);
            acc[r][2 * e + 1] = mfma_16x16x32(hi, p[r], acc[r][2 * e + 1]);
          }
          if constexpr (NR > 1) __builtin_amdgcn_sched_barrier(0);
        });
        if (ahead >= end) break;
        t.load_v(a.c, next, ahead, head, lane);
        key0 = ahead;
        pages = next;
        if (ahead + kStride < end) next = find_pages(a, table, ahead + kStride);
      }
    }

    // Join the waves, one 16-row tile at a time: thread (row, c) takes columns D / 16 * c .., which
    // lane (row, g) of each wave holds in register i of its products, c = 4 g + i.
    const int row = threadIdx.x >> 4, c = threadIdx.x & 15;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      __syncthreads();  // Q, or the tile before, is read
      const float total = groups_sum(sum[r]);
#pragma unroll
      for (int t = 0; t < F::kDTiles; ++t)
        lds[(wave * F::kDTiles + t) * 64 + m * 4 + g] = float4{acc[r][t][0], acc[r][t][1], acc[r][t][2], acc[r][t][3]};
      if (g == 0) lds_stat[wave][m] = float4{ref[r], total, sum16[r], 0.0f};
      lds_poison[wave][m * 4 + g] = poisoned >> r & 1;
      __syncthreads();
      join_waves<D, FP8>(a, plan, seq, reinterpret_cast<const float*>(lds), &lds_stat[0][row].x,
                         &lds_poison[0][row * 4 + (c >> 2)], row0 + 16 * r + row, c, head, whole,
                         partial_row(a, plan, w, from == range.at ? 1 : 0, head, tile) + 16 * r + row);
    }
    // the next sequence that has rows here; there is one if the range goes on
    if (stop >= range.end) break;
    do {
      if (++range.b >= a.B) return;
      range.seq = sequence(a, range.b);
      range.units = units_of(a, plan, range.seq, tile);
    } while (range.units == 0);
    range.at = stop + kSetup;
    __syncthreads();
  }
}

// Joins the pieces of the sequences that cross ranges.  A row takes D / 4 lanes of 4
// columns; kSpread = 1: every group of lanes has its own row and walks the pieces;
// else one row a workgroup, the pieces dealt to the groups.
// grid: (rows of a row tile and all key heads / rows of a workgroup, ranges - 1, row tiles)
constexpr int kJoinThreads = 256;
template <int D, bool FP8, bool SPREAD>
__global__ __launch_bounds__(kJoinThreads) void cache_join_kernel(const CacheAttentionArgs a, const CachePlan plan) {
  constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes;
  const Partials part = partials(a, plan);
  const int w = blockIdx.y + 1, tile = blockIdx.z;
  const int4 job = part.joins[tile * plan.ranges + w];
  const int pieces = job.x, first = job.y, rows = job.z;
  if (pieces == 0) return;
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int row = SPREAD ? (int)blockIdx.x : (int)blockIdx.x * kGroups + group;
  const int head = row / plan.tile_rows, in_tile = row - head * plan.tile_rows;
  const int i = tile * 16 * plan.nr + in_tile;
  const bool there = head < a.c.H && i < rows;
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
  if (there) {
#pragma unroll 4
    for (int k = SPREAD ? group : 0; k < pieces; k += SPREAD ? kGroups : 1) {
      const int64_t at = partial_row(a, plan, w - 1 + k, k == 0 ? 1 : 0, head, tile) + in_tile;
      join(part.stat[at], reinterpret_cast<const float4*>(part.acc + at * D)[lane]);
    }
  }
  if constexpr (SPREAD) {
    __shared__ float4 acc_lds[kGroups][kLanes];
    __shared__ float4 stat_lds[kGroups];
    acc_lds[group][lane] = acc;
    if (lane == 0) stat_lds[group] = float4{ref, sum, sum16, 0.0f};
    __syncthreads();
    if (group != 0) return;
    const int used = pieces < kGroups ? pieces : kGroups;
    for (int k = 1; k < used; ++k) join(stat_lds[k], acc_lds[k][lane]);
  }
  if (!there) return;
  const int t = i / a.G;
  const int64_t at = (int64_t)(first + t) * a.Hq + head * a.G + (i - t * a.G);
  const bool empty = is_zero(sum16);
  const float norm = (FP8 ? 1.0f : 1.0f / 6.0f) / sum16;
  const float o[4] = {empty ? 0.0f : acc.x * norm, empty ? 0.0f : acc.y * norm, empty ? 0.0f : acc.z * norm,
                      empty ? 0.0f : acc.w * norm};
  const int64_t to = at * D + lane * 4;
  if (a.out_bf16) store_row<4>(static_cast<uint16_t*>(a.out) + to, o);
  else store_row<4>(static_cast<float*>(a.out) + to, o);
  if (a.lse && lane == 0) a.lse[at] = log_norm(ref, sum);
}

template <int D, bool FP8>
void launch_format(const CacheAttentionArgs& a, const CachePlan& plan, hipStream_t stream) {
  const unsigned grid = (unsigned)plan.workgroups;
  if (plan.nr == 1) cache_attention_kernel<D, FP8, 1><<<grid, kThreads, 0, stream>>>(a, plan);
  else if (plan.nr == 2) cache_attention_kernel<D, FP8, 2><<<grid, kThreads, 0, stream>>>(a, plan);
  else cache_attention_kernel<D, FP8, 4><<<grid, kThreads, 0, stream>>>(a, plan);
  if (!plan.split || plan.ranges == 1) return;
  const unsigned rows = (unsigned)(plan.tile_rows * a.c.H), per = kJoinThreads / (D / 4);
  // many pieces a sequence: a workgroup for each row
  if (plan.ranges >= 4 * a.B)
    cache_join_kernel<D, FP8, true><<<dim3(rows, plan.ranges - 1, plan.row_tiles), kJoinThreads, 0, stream>>>(a, plan);
  else
    cache_join_kernel<D, FP8, false><<<dim3((rows + per - 1) / per, plan.ranges - 1, plan.row_tiles), kJoinThreads, 0,
                                       stream>>>(a, plan);
}

}  // namespace

CachePlan cache_plan(int64_t B, int64_t H, int64_t G, int64_t d, int fp8, int64_t max_q, int64_t max_keys) {
  CachePlan p{};
  const int64_t rows = max_q * G;
  p.nr = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
  const int64_t row_tiles = (rows + 16 * p.nr - 1) / (16 * p.nr);
  p.row_tiles = (int)row_tiles;
  p.tile_rows = (int)(rows < 16 * p.nr ? rows : 16 * p.nr);
  p.min_units = 4;
  // Ranges: as many workgroups as the chip holds at once, so that all end together.
  const int64_t slots = 256 * waves_per_simd((int)d, fp8, p.nr), per_range = H * row_tiles;
  p.split = max_keys > 1024;
  p.ranges = p.split ? (int)(slots / per_range < 1 ? 1 : slots / per_range) : (int)B;
  const int64_t most = B * ((max_keys + kUnit - 1) / kUnit);  // units there can be
  if (p.split && p.ranges > (most + p.min_units - 1) / p.min_units) p.ranges = (int)((most + p.min_units - 1) / p.min_units);
  const int64_t items = row_tiles > 1 ? (p.ranges * H + 7) / 8 * 8 : p.ranges * H;
  p.workgroups = items * row_tiles;
  if (p.split && p.ranges > 1)
    p.workspace = p.ranges * row_tiles * 16 + p.ranges * 2 * per_range * p.tile_rows * (d * 4 + 16);
  return p;
}

hipError_t launch_cache_attention(const CacheAttentionArgs& a, hipStream_t stream) {
  const CachePlan plan = cache_plan(a.B, a.c.H, a.G, a.c.d, a.c.fp8, a.max_q, (int64_t)a.max_pages << a.c.page_shift);
  if (a.c.d == 64 && a.c.fp8) launch_format<64, true>(a, plan, stream);
  else if (a.c.d == 64) launch_format<64, false>(a, plan, stream);
  else if (a.c.fp8) launch_format<128, true>(a, plan, stream);
  else launch_format<128, false>(a, plan, stream);
  return hipGetLastError();
}

}  // namespace fp4attn
