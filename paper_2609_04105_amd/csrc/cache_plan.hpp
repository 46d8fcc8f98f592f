// The launch plan of an attention call over the cache.  Plain C++, so that a host program can ask
// what a call takes.
#pragma once
#include <cstdint>

namespace fp4attn {

// How one attention call is cut up.  Rows (token, head of the group) of a sequence and
// key head go to workgroups in tiles of 16, 32 (their waves split the keys) or 128 rows (their
// waves split the rows).  With split, the row tiles of all sequences, each with its keys in
// units of 128, lie end to end (with a few places between them), and each of `ranges` workgroups
// per key head takes an equal part of that line (fewer ranges if that leaves less than
// min_units each); lengths are known on the device only.  Without, a range is a row tile; beside `direct` ones of that kind
// there may be others, for the rest of row tiles of more than direct_units units (own_plan).
struct CachePlan {
  int tile;       // rows of a row tile
  int row_tiles;  // of the longest sequence and one key head
  int tile_rows;  // rows of a tile that can be in use
  int split, ranges, min_units;
  bool fits;           // the line's places and the workgroups are in range
  int direct, direct_units;
  int64_t workgroups;  // of the first launch
  int64_t workspace;   // bytes
};
constexpr int kUnit = 128;  // keys that ranges are counted in
constexpr int kSetup = 4;   // places of the line that starting a row tile takes (cache_attention.hpp)
constexpr int kRowsTile = 128, kRowsPerCu = 2;  // cache_attention_rows.hpp: rows of a workgroup, workgroups of a CU

constexpr int64_t kMaxCacheKeys = int64_t(1) << 30;  // keys of one sequence

// Waves per SIMD that the registers are kept to.  (Two tiles in flight instead of one, at 2 .. 3 waves:
// within 3 % either way for d = 128, and four waves of d = 64 are faster, 126 us against 130 for 64
// sequences of 16384 keys and 8 key heads; at three waves 140.)
constexpr int waves_per_simd(int d, int nr) { return 6 - d / 64 - nr; }

// Units that a row tile touches of which every token sees `window` keys, wherever they begin.
constexpr int window_units(int tile, int G, int window) {
  return (window + (tile + G - 2) / G + kUnit - 2) / kUnit + 1;
}

inline CachePlan cache_plan(int64_t B, int64_t H, int64_t G, int64_t d, bool fp8, int64_t max_q, int64_t max_keys) {
  CachePlan p{};
  const int64_t rows = max_q * G, units = (max_keys + kUnit - 1) / kUnit;
  auto tiles_of = [&](int64_t tile) { return (rows + tile - 1) / tile; };
  // Rows of a tile.  Up to 16 rows the matrix products have one column tile of them.  More: the 128-row
  // kernel converts a key's codes once for 128 rows, the other once for 32, but
  // - it needs more work to fill the chip: rows for two workgroups on every CU with d = 64 (half the products to a
  //   conversion), for one with d = 128, for half of one if there are many keys to cut up;
  // - a workgroup takes as long with few of its rows in use as with all, as long as three 32-row tiles with d = 64,
  //   two with d = 128, and in a full chip one with MXFP8, whose codes are twice the bytes.
  // 8 key heads of 8 query heads, us at tile 32 / 128:
  //   d = 128, MXFP4, 32 sequences, 64 tokens (rows for 1024 workgroups), 2048 keys 184 / 154, 12 (384), 1024 keys 57 / 46;
  //   24 sequences, 16 tokens (192), 4096 keys 89 / 84, 8192 keys 149 / 135, 2048 keys 53 / 54, 1024 keys 36 / 38;
  //   16 sequences, 16 tokens (128), 8192 keys MXFP4 96 / 95, MXFP8 145 / 108, 4096 keys 60 / 63;
  //   64 sequences, 4096 keys, MXFP4: 4 tokens 78 / 138, 8 126 / 158, 10 164 / 163, 12 173 / 165, 16 222 / 175; MXFP8: 110 / 149,
  //   203 / 162, 247 / 171, 275 / 171, 336 / 184; 32 sequences, MXFP4, 4 tokens 45 / 85, 8 71 / 97, 10 86 / 102, 16 118 / 109;
  //   d = 64, 16 sequences, 64 tokens (512), 1024 keys 45 / 39, 4096 keys 121 / 125; 32, 16 tokens (256), 2048 keys 44 / 53;
  //   64 sequences, 1024 keys, 4 tokens 18 / 35, 12 40 / 40, 16 51 / 40, 17 51 / 76, 24 67 / 76, 32 92 / 77.
  const int64_t wide = B * H * rows / kRowsTile;  // workgroups of 128 rows, if all are in use
  const int64_t least = d == 64 ? 3 : (fp8 && wide >= 256 ? 1 : 2);
  const bool rows128 = tiles_of(32) > least * tiles_of(kRowsTile) &&
                       (wide >= 512 || (d == 128 && (wide >= 256 || (wide >= 128 && wide * max_keys >= 3 << 18))));
  p.tile = rows <= 16 ? 16 : (rows128 ? kRowsTile : 32);
  const int64_t row_tiles = tiles_of(p.tile);
  p.row_tiles = (int)row_tiles;
  p.tile_rows = (int)(rows < p.tile ? rows : p.tile);
  p.min_units = 4;
  // Without the split there is no second launch and a range has no neighbours.  It pays while a
  // workgroup alone walks its keys in the time of that launch, and longer where the row tiles fill the
  // chip anyway (of 128 rows: twice).  Single tokens, d = 128, MXFP4, 8 key heads, us split / not:
  //   1 sequence, 1024 keys 10.9 / 10.4, 2048 keys 10.9 / 16.4; 32 sequences, 2048 keys 23.9 / 20.6, 4096 keys 37.6 / 41.6;
  // of 128 rows: 16 sequences, 64 tokens (512 workgroups), 2048 keys 92 / 81, 8 (256) 60 / 68, 1024 keys 43 / 38;
  // 32, 16 tokens (256), 1040 keys 49 / 39.
  const bool full = B * H * row_tiles >= (p.tile == kRowsTile ? 512 : 256);
  // Ranges: as many workgroups as the chip holds at once, so that all end together.  With so many key heads that
  // this leaves each a single range, nothing can be cut.
  const int64_t slots = 256 * (p.tile == kRowsTile ? kRowsPerCu : waves_per_simd((int)d, p.tile / 16));
  p.split = max_keys > (full ? 2048 : (p.tile == kRowsTile ? 1536 : 1024)) && slots / H >= 2;
  const int64_t places = B * row_tiles * (units + kSetup);  // there can be
  int64_t ranges = slots / H;
  if (ranges > (places + p.min_units - 1) / p.min_units) ranges = (places + p.min_units - 1) / p.min_units;
  if (!p.split) ranges = B * row_tiles;
  p.fits = places + ranges < (int64_t(1) << 31) && ranges * H <= (1 << 24) - 8;  // int places; launches below 2^32 threads
  p.ranges = (int)ranges;
  p.workgroups = (ranges * H + 7) / 8 * 8;
  if (p.split) p.workspace = ranges * 16 + ranges * 2 * H * p.tile_rows * (d * 4 + 16);
  return p;
}

// Microseconds of walking `keys` keys for `tiles` row tiles, all key heads counted, in a chip that they fill, with the
// launch and its start: from the times of 400 batches of 2 to 200 sequences, 1 to 16 tokens, 1 to 8 query heads a key head,
// behind 1024 to 65536 keys (8 heads of d = 128 in MXFP4, 2 of d = 64 in MXFP8), by least squares.  A rough model: d = 128 in MXFP8
// and d = 64 in MXFP4 were not in it, and it knows nothing of a last round that leaves workgroups idle.
inline double walk_time(int tile, int64_t d, int64_t tiles, int64_t keys, bool prefix) {
  const double walks = (double)tiles * (double)keys * 1e-6;
  if (tile == 16) return prefix ? 14 + 30 * walks : 12 + 15 * walks;  // (a pass over a prefix has one tile a key head)
  if (tile == 32) return (prefix ? 18.5 : 16) + (prefix ? (d == 64 ? 20 : 25) : 22) * walks;
  return 28 + (prefix ? 75 : 67) * walks;
}

// The pass over a prefix of `keys` keys (whole units) that the sequences share: all n tokens' rows of a key head together in
// row tiles, each with `pieces` parts of the prefix of `units` units, one to a workgroup.
struct PrefixPlan {
  CachePlan plan;
  int pieces, units;
  bool fits;
  int64_t rows;  // n * H * G: of each piece
};
// Row tiles: 16 where they hold all rows, else 32 or 128, whichever the times above say.  us at tile 32 / 128, 8 key heads, d =
// 128, MXFP4: 192 rows, 4096 keys 23 / 32, 65536 keys 94 / 100; 768 rows, 4096 keys 40 / 44, 16384 keys 110 / 87, 65536 keys 384 / 265.
// Pieces: as many workgroups as the chip holds at once, of four units at least: at least two or eight, 192 rows behind 4096 keys 23.4,
// 23.3 against 23.3; 16 rows behind 16384 keys 21.9, 19.2 against 18.1; 64 rows behind 1024 keys 15.2, 20.9 against 16.9.
inline PrefixPlan prefix_plan(int64_t H, int64_t G, int64_t d, int64_t n, int64_t keys) {
  PrefixPlan p{};
  const int64_t rows = n * G, units = keys / kUnit;
  CachePlan& c = p.plan;
  auto tiles_of = [&](int64_t tile) { return (rows + tile - 1) / tile; };
  c.tile = rows <= 16 ? 16 : 32;
  if (rows > 16 && walk_time(kRowsTile, d, tiles_of(kRowsTile) * H, keys, true) < walk_time(32, d, tiles_of(32) * H, keys, true))
    c.tile = kRowsTile;
  const int64_t row_tiles = tiles_of(c.tile);
  c.row_tiles = (int)row_tiles;
  c.tile_rows = (int)(rows < c.tile ? rows : c.tile);
  const int64_t slots = 256 * (c.tile == kRowsTile ? kRowsPerCu : waves_per_simd((int)d, c.tile / 16));
  constexpr int64_t kLeast = 4, kMost = 64;  // units of a piece, pieces
  int64_t pieces = slots / (row_tiles * H);
  if (pieces > units / kLeast) pieces = units / kLeast;
  pieces = pieces < 1 ? 1 : (pieces > kMost ? kMost : pieces);
  const int64_t per = (units + pieces - 1) / pieces;
  p.units = (int)per;
  p.pieces = (int)((units + per - 1) / per);
  c.ranges = (int)(row_tiles * p.pieces);
  c.workgroups = (row_tiles * p.pieces * H + 7) / 8 * 8 + 8;  // the last eight without a range (place_of, look_for_long)
  p.rows = rows * H;
  p.fits = c.workgroups < 1 << 24;
  return p;
}

// Whether n tokens of B sequences, which a call with `plan` serves one by one, gain by a pass over their shared prefix.  us without it /
// with it, 8 key heads of 4 query heads, d = 128, MXFP4, one token each: 2 sequences behind 65536 keys 29 / 29; 4 31 / 29 of
// 32768; 16 behind 1024 keys 12.9 / 16.9, 4096 keys 21.9 / 18.2; 48 behind 4096 keys 39 / 23, 65536 keys 363 / 94; 16 tokens each: 8
// behind 65536 keys 190 / 177, 48 behind 16384 keys 281 / 314.  The model has to promise a tenth: of 320 other random batches (2 to 128
// sequences, 2 or 8 key heads, both head dimensions and formats, 1 to 16 tokens) that it says gain anything the pass made 52 more than 3 % longer,
// of those that it says gain a tenth 14, 1.43 times at most; on average the calls take 0.622 and 0.618 of what they take one by one.
inline bool shares_prefix(const CachePlan& plan, const PrefixPlan& prefix, int64_t B, int64_t H, int64_t G, int64_t d, int64_t n,
                          int64_t keys) {
  int64_t tiles = n * G / plan.tile + B;  // at most, of ragged sequences
  if (tiles > B * plan.row_tiles) tiles = B * plan.row_tiles;
  // (where row tiles of 128 rows serve the sequences one by one, their own keys lose by the smaller tiles that fewer keys get: trees of
  // 32 tokens, 24 sequences of up to 2048 keys behind 4096, 94 us without the pass, 112 with it)
  const double gain = 0.9 * (plan.tile == kRowsTile ? 0.8 : 1.0);
  return prefix.fits && walk_time(prefix.plan.tile, d, prefix.plan.row_tiles * H, keys, true) <
                            gain * walk_time(plan.tile, d, tiles * H, keys, false);
}

// The plan of the sequences' own pass behind a shared prefix: for `own` keys, which those that join the prefix have at most.
// One that does not join it may have max_keys.  If these would be cut up without the prefix and `own` keys are not, every row tile has a
// direct range, and beside those are others for what is beyond the first pieces of row tiles with more than `own` keys (find_cut,
// join_last in cache_attention.hpp).  us uncut / so / one by one, 8 key heads, d = 128, one token each, one sequence ending after 15/16 of the
// prefix: 16 sequences, 4 query heads a key head, MXFP4, behind 65536 keys 393 / 61 / 128; 96, 8 query heads, MXFP8, 632 / 327 / 1158; 24,
// 8 query heads, MXFP4, behind 16384 keys 121 / 46 / 56; with all sequences behind the prefix uncut 49, 282, 37, so 50, 281, 36.  (Cutting all
// as without a prefix, with a launch that joins, 69, 311, 45, and with all behind 51, 287, 40; over 160 batches 11 % longer, so 1 %.)
inline CachePlan own_plan(int64_t B, int64_t H, int64_t G, int64_t d, bool fp8, int64_t max_q, int64_t own, int64_t max_keys) {
  CachePlan p = cache_plan(B, H, G, d, fp8, max_q, own);
  if (p.split || !cache_plan(B, H, G, d, fp8, max_q, max_keys).split) return p;
  const int64_t units = (max_keys + kUnit - 1) / kUnit, places = B * p.row_tiles * units;
  // A unit takes a workgroup 0.7 us, a piece the workgroup that joins them 0.45.
  while (1.6 * p.min_units * p.min_units < (double)units) ++p.min_units;
  int64_t others = 512 / H;  // (half as many: batches of which half ends inside the prefix 8 % slower; as many as the chip holds: the same)
  if (others > (places + p.min_units - 1) / p.min_units) others = (places + p.min_units - 1) / p.min_units;
  if (others < 2) return p;
  p.direct = p.ranges;
  p.direct_units = (int)((own + kUnit - 1) / kUnit);
  p.ranges += (int)others;
  p.workgroups += (others * H + 7) / 8 * 8;
  p.fits = p.fits && p.workgroups < 1 << 24;
  p.workspace = others * 16 + others * 2 * H * p.tile_rows * (d * 4 + 16);
  return p;
}

// The plan of a call that may pass over the first `shared` keys by themselves, of n tokens; `plan` serves it without.
struct SharedPlan {
  CachePlan plan;  // of the sequences' own pass
  PrefixPlan prefix;
  int64_t shared;  // keys that have a pass of their own; 0: none
};
inline SharedPlan shared_plan(const CachePlan& plan, int64_t B, int64_t H, int64_t G, int64_t d, bool fp8, int64_t max_q, int64_t n,
                              int64_t max_keys, int64_t shared) {
  SharedPlan p{plan, {}, 0};
  const int64_t keys = shared / kUnit * kUnit;
  if (n < 1 || B < 2 || keys < 1) return p;
  p.prefix = prefix_plan(H, G, d, n, keys);
  if (!shares_prefix(plan, p.prefix, B, H, G, d, n, keys)) return p;
  p.shared = keys;
  p.plan = own_plan(B, H, G, d, fp8, max_q, max_keys > keys ? max_keys - keys : 1, max_keys);
  // (smaller row tiles than the call's without the pass, and sequences that do not join the prefix)
  const int64_t places = B * p.plan.row_tiles * ((max_keys + kUnit - 1) / kUnit + kSetup);
  if (!p.plan.fits || places + p.plan.ranges >= int64_t(1) << 31) return SharedPlan{plan, {}, 0};
  return p;
}

}  // namespace fp4attn
