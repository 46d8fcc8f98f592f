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
// min_units each); lengths are known on the device only.  Without, a range is a row tile.
struct CachePlan {
  int tile;       // rows of a row tile
  int row_tiles;  // of the longest sequence and one key head
  int tile_rows;  // rows of a tile that can be in use
  int split, ranges, min_units;
  bool fits;           // the line's places and the workgroups are in range
  int64_t workgroups;  // of the first launch
  int64_t workspace;   // bytes
};
constexpr int kUnit = 128;  // keys that ranges are counted in
constexpr int kSetup = 4;   // places of the line that starting a row tile takes (cache_attention.hpp)
constexpr int kRowsTile = 128, kRowsPerCu = 2;  // cache_attention_rows.hip: rows of a workgroup, workgroups of a CU

constexpr int64_t kMaxCacheKeys = int64_t(1) << 30;  // keys of one sequence

// Waves per SIMD that the registers are kept to.  (Two tiles in flight instead of one, at 2 .. 3 waves:
// within 3 % either way for d = 128, and four waves of d = 64 are faster, 126 us against 130 for 64
// sequences of 16384 keys and 8 key heads; at three waves 140.)
constexpr int waves_per_simd(int d, int nr) { return 6 - d / 64 - nr; }

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

}  // namespace fp4attn
