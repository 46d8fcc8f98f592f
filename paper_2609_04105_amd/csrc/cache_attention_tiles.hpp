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
// - the row tiles of all sequences, each with its keys, are laid end to end and cut into equal parts
//   for as many workgroups as the chip holds; pieces of a row tile that a cut crosses meet in a
//   second launch (no atomics: the order is fixed).
//
// Measured, single tokens, 8 key heads: MXFP4, d = 128, 64 sequences of 16384 keys and four query heads to
// a key head 208 us, 5.5 TB/s of the cache (a large copy: 5.0 .. 5.3); MXFP8, 4 sequences of 131072 keys
// and less (412 thousand in all), eight to a key head 160 us, 5.4 TB/s; d = 64, MXFP4, 64 of 16384 keys, eight to a key head 117 us, 4.9 TB/s
// (half the bytes a key, more than half the instructions).  Short calls are latency: one sequence of 517 keys
// 8.1 us, of which the arguments, the length, the page, the first tile one after the other 2.3 us, the tiles
// 0.74 us each (330 instructions of a wave alone on its SIMD), the join of the waves and the stores 1.2 us.
//
// Precision: scores and sums fp32.  P is rounded to bf16 for the matrix product, and the
// normaliser sums the same rounded values (a product with ones), so that the rounding of
// a dominant key cancels; the log normaliser that `lse` returns takes the unrounded sum.  What is left is at most 2^-8 of
// the weighted mean of |v - o|, less than the formats' own steps of V.  (What the rounding loses as a second operand of
// the PV product brings that to 2^-16, and took 16-row tiles up to 10 % longer: one sequence of 517 keys 7.9 -> 8.4 us, d = 64,
// 16 of 900 8.8 -> 9.7, 64 of 4096 37.3 -> 40.1; long caches of d = 128 the same.)
// The reference of a row lags its maximum by at most 8 binades (p <= 256), which
// saves most rescalings of the accumulators.
#pragma once

#include "cache_attention.hpp"

namespace fp4attn {

namespace {

// What a lane holds of one 32-key tile, and where it finds it.
template <int D, bool FP8>
struct Tile {
  using F = Format<D, FP8>;
  unsigned k[2][F::kKWords];  // [half] key 8 (m / 4) + 4 half + m % 4, m = lane % 16: values D / 4 * (lane / 16) ..
  unsigned ks[2];             // their E8M0 byte
  unsigned v[F::kVWords];     // keys 8 (lane / 16) .. + 7, values D / 16 * (lane % 16) ..
  unsigned vs[2];             // their eight E8M0 bytes
  static constexpr int kKBytes = F::kKWords * 4, kVBytes = F::kVWords * 4;

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

// Joins the waves' results of row i and columns D / 16 * c ..  lds: [wave][product][row, 4 g + i];
// stat: the row's {reference, sum, sum of the rounded values} of the first wave, 16 rows apart;
// odd_marks: its marks, 64 words apart.
template <int D, bool FP8, class Args>
__device__ __forceinline__ void join_waves(const Args& a, const CachePlan& plan, const Sequence& seq,
                                           const float* lds, const float* stat, const unsigned* odd_marks, int i, int c,
                                           int head, bool whole, int64_t piece) {
  constexpr int kCols = D / 16;
  if (i >= seq.tokens * a.G) return;
  float top = -__builtin_inff(), sum = 0.0f, rounded = 0.0f, o[kCols];
  unsigned odd = 0;
#pragma unroll
  for (int j = 0; j < kCols; ++j) o[j] = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stat[w * 64]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float ref = stat[w * 64], part = ref == top ? 1.0f : __builtin_amdgcn_exp2f(ref - top);
    sum += stat[w * 64 + 1] * part;
    rounded += stat[w * 64 + 2] * part;
    odd |= odd_marks[w * 64];
#pragma unroll
    for (int j = 0; j < kCols; ++j) o[j] += lds[(w * kCols + j) * 256 + threadIdx.x] * part;
  }
  store_columns<D, FP8>(a, plan, seq, i, head, c, whole, piece, top, sum, rounded, FP8 ? odd >> kCols * (c % 4) : odd, o);
}

template <int D, bool FP8, int NR, class Args>
__global__ __launch_bounds__(kThreads, waves_per_simd(D, NR)) void cache_attention_kernel(const Args a, const CachePlan plan) {
  using F = Format<D, FP8>;
  constexpr bool kSharedQ = NR > 1;  // Q operands in LDS: NR * D / 8 registers less
  // the waves' results of one 16-row tile, or Q before them
  constexpr int kAccWords = kWaves * F::kDTiles * 64, kQWords = kSharedQ ? NR * F::kSteps * 64 : 0;
  __shared__ float4 lds[kAccWords > kQWords ? kAccWords : kQWords];
  __shared__ float4 lds_stat[kWaves][16];
  __shared__ unsigned lds_odd[kWaves][64];
  v4i* lds_q = reinterpret_cast<v4i*>(lds);

  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  fetch_arguments(a, plan);
  const Place place = place_of(a, plan);
  const int head = place.head;
  if (head >= a.c.H) {
    if constexpr (Args::kPrefix)
      if (head == a.c.H && place.w == 0) look_for_long(a);
    return;
  }
  Range range = open_range(a, plan, place);
  if (range.begin >= range.end) return;
  const ScoreShape shape = score_shape<FP8>(a);
  const float factor = shape.factor;

  // A CU serves the workgroups that came first, of the first half of the grid, before the others, which then end
  // later: those go first in every second tile.  64 sequences of 2768 keys 46.9 -> 45.7 us, of 16384
  // keys 210.3 -> 208.0; d = 64 119.4 -> 117.2; trees of 16 tokens over 8 of 2047 keys 22.6 -> 21.8.
  const bool late = (plan.split || Args::kPrefix) && in_second_half(a, plan);
  Part part;
  while (open_part(a, plan, range, &part)) {
    const Sequence seq = range.seq;
    const int rows = seq.tokens * a.G, row0 = range.tile * plan.tile;

    // this lane's rows (the same for the four lane groups) and its part of their queries
    int token[NR];  // of the sequence
    float slope[NR];
    v4i q[kSharedQ ? 1 : NR][F::kSteps];  // in LDS later: wave r has row tile r
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const int i = row0 + 16 * r + m, ic = i < rows ? i : rows - 1;
      token[r] = divide(ic, a.G);
      const int h = head * a.G + (ic - token[r] * a.G);
      slope[r] = slope_of(a, h);
      const uint16_t* p = static_cast<const uint16_t*>(a.q) + (int64_t)(seq.first + token[r]) * a.q_stride + h * D + g * (D / 4);
      if (!kSharedQ || r == wave)
#pragma unroll
        for (int s = 0; s < F::kSteps; ++s) q[kSharedQ ? 0 : r][s] = reinterpret_cast<const v4i*>(p)[s];
    }
    // the wave's first tile, on its way together with the queries
    const ScalarInts table = (ScalarInts)(uintptr_t)(a.page_table + (int64_t)range.b * a.max_pages);
    constexpr int kStride = kTile * kWaves;
    int key0 = part.begin + kTile * wave;
    Tile<D, FP8> t;
    Pages pages{0, 0}, next{0, 0};
    if (key0 < part.end) {
      pages = find_pages(a, table, key0);
      t.load_k(a.c, pages, key0, head, lane);
      t.load_v(a.c, pages, key0, head, lane);
      if (key0 + kStride < part.end) next = find_pages(a, table, key0 + kStride);
    }
    if constexpr (kSharedQ) {
      if (wave < NR)
#pragma unroll
        for (int s = 0; s < F::kSteps; ++s) lds_q[(wave * F::kSteps + s) * 64 + lane] = q[0][s];
      __syncthreads();
    } else {  // (waits for the queries here; in the loop the compiler would wait for tiles with them)
#pragma unroll
      for (int s = 0; s < F::kSteps; ++s) asm volatile("" : "+v"(q[0][s]));
    }
    v4f acc[NR][F::kDTiles];
    v4f sum16[NR];  // the rounded probabilities (the same in all four)
    OddMarks<FP8, NR> odd_marks;
    float ref[NR], sum[NR];    // base 2, lags the maximum by at most kLag; this lane's own keys
#pragma unroll
    for (int r = 0; r < NR; ++r) {
#pragma unroll
      for (int t = 0; t < F::kDTiles; ++t) acc[r][t] = v4f{0, 0, 0, 0};
      sum16[r] = v4f{0, 0, 0, 0};
      ref[r] = -__builtin_inff();
      sum[r] = 0.0f;
    }

    if constexpr (Args::kShaped && !Args::kPrefix)
      if (part.first && shared_keys(a, seq)) {  // the waves begin with the pieces of the shared prefix
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          const int i = row0 + 16 * r + m, ic = i < rows ? i : rows - 1, h = head * a.G + (ic - token[r] * a.G);
          const int row = (seq.first + token[r]) * a.Hq + h;  // below 2^31
          const float lower = slope[r] * (float)(seq.prefix + token[r] - a.shared);
          for (int k = wave; k < a.prefix_pieces; k += kWaves)
            add_piece<D>(a, k, row, g, lower, &ref[r], &sum[r], &sum16[r], acc[r]);
        }
      }

    // The wave's tiles.  One set of registers: a tile's K is loaded when the one before has
    // become scores, its V when the one before is in the accumulators.
    if (key0 < part.end) {
      while (true) {
        if (late) {
          if (key0 & kStride) __builtin_amdgcn_s_setprio(2);
          else __builtin_amdgcn_s_setprio(0);
        }
        // The last tile is loaded again instead of one behind it: where the loads of a tile depended on
        // a branch, the compiler's waits for K waited for V too, the whole latency of a load in every tile.
        const bool more = key0 + kStride < part.end;
        const int ahead = more ? key0 + kStride : key0;
        if (!more) next = pages;
        const bool page0 = is_page(a.c, pages.p0), page1 = is_page(a.c, pages.p1);
        const bool masked = some_hidden(a, part, key0, kTile) || !page0 || !page1;  // uniform
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
        t.load_k(a.c, next, ahead, head, lane);
        if constexpr (Args::kScores) {
          const int base = key0 + 8 * g;
          if (a.cap.on) {
            float most = 0.0f;
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
              for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(s[r][j / 4][j % 4]));
            // (the near form follows in the code: one token of 700 keys 11.15 -> 10.95 us)
            if (__builtin_expect(__any(most > a.cap.near), 0)) cap_all(a, s);
            else cap_near(a, s);
            if (a.slopes) add_bias<Args>(seq, slope, token, base, s);
          } else if (a.slopes) {
            if (a.open_keys) {
              scale_scores(shape.plain, s);
              add_bias<Args>(seq, slope, token, base, s);
            } else {
              scale_with_bias<Args>(seq, shape.plain, slope, token, base, s);
            }
          }
        }
        if (masked) {
          // Hidden scores become -inf.  Keys that no row sees hold anything: their V codes and
          // scales become zero.  A non-finite V block that some row may see becomes zero too, and a NaN
          // code of MXFP8; they mark the rows that see them, whose outputs become NaN after the loop.
          const int base = key0 + 8 * g;
          const unsigned there = (g >= 2 ? page1 : page0) ? may_see(a, part, seq.keys, base) : 0u;
          unsigned see[NR];
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            see[r] = there & row_sees(a, seq, part, range.b, token[r], base);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[r][j / 4][j % 4] = see[r] >> j & 1 ? s[r][j / 4][j % 4] : -__builtin_inff();
          }
          unsigned odd = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const bool in = there >> j & 1, big = (t.vs[j / 4] >> (8 * (j % 4)) & 255u) >= kHugeScale<FP8>;
            odd |= in && big ? 1u : 0u;
            const unsigned keep = in && !big ? ~0u : 0u;
            t.vs[j / 4] &= keep | ~(255u << (8 * (j % 4)));
            if constexpr (F::kVWords >= 8) {
#pragma unroll
              for (int i = 0; i < F::kVWords / 8; ++i) t.v[j * (F::kVWords / 8) + i] &= keep;
            } else {
              t.v[j / 2] &= keep | (j % 2 ? 0x0000ffffu : 0xffff0000u);
            }
          }
          if constexpr (FP8)
#pragma unroll
            for (int i = 0; i < F::kVWords; ++i) odd |= nan_codes(t.v[i]);
          if (__any(odd)) {
            if constexpr (FP8)
#pragma unroll
              for (int i = 0; i < F::kVWords; ++i) t.v[i] = without_nan_codes(t.v[i]);
#pragma unroll
            for (int r = 0; r < NR; ++r) see[r] = groups_or(see[r] << (8 * g));
            for (int k = 0; k < kTile; ++k) {
              const int page = k >= 16 ? pages.p1 : pages.p0, key = key0 + k;
              if (!is_page(a.c, page) || key >= seq.keys) continue;
              const int64_t group = row_of(a.c, page, head, key & ((1 << a.c.page_shift) - 1)) >> 3;
              const unsigned columns = odd_columns<D, FP8>(a.c, group, k & 7, g);
#pragma unroll
              for (int r = 0; r < NR; ++r) odd_marks.add(r, see[r] >> k & 1, columns);
            }
          }
        }
        float top[NR];
        bool rise = false;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          top[r] = groups_max(max8(s[r])) * factor;
          rise |= top[r] > ref[r] + kLag;
        }
        if (__any(rise)) {
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            const float now = top[r] > ref[r] + kLag ? top[r] : ref[r];  // (a row moves by its own keys alone)
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
          p[r] = probabilities(s[r], factor, ref[r], &sum[r]);
          sum16[r] = mfma_16x16x32(v4i{kOnes, kOnes, kOnes, kOnes}, p[r], sum16[r]);
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
        t.load_v(a.c, next, ahead, head, lane);
        if (!more) break;
        key0 = ahead;
        pages = next;
        if (ahead + kStride < part.end) next = find_pages(a, table, ahead + kStride);
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
      if (g == 0) lds_stat[wave][m] = float4{ref[r], total, sum16[r][0], 0.0f};
      lds_odd[wave][m * 4 + g] = odd_marks.template of<0>(r, 0);
      __syncthreads();
      join_waves<D, FP8>(a, plan, seq, reinterpret_cast<const float*>(lds), &lds_stat[0][row].x,
                         &lds_odd[0][row * 4 + (c >> 2)], row0 + 16 * r + row, c, head,
                         !Args::kPrefix && part.whole,
                         piece_row(a, plan, range, place, part, 16 * r + row));
    }
    if constexpr (Args::kDirect)
      if (!part.whole) join_last<D, FP8>(a, plan, range, place, &lds_odd[0][0]);
    if (!next_tile(a, plan, part.stop, range)) break;
    __syncthreads();
  }
}

// Joins the pieces of the row tiles that cross ranges.  A row takes D / 4 lanes of 4 columns; with
// SPREAD a workgroup has one row and deals the pieces to its groups of lanes, else every group
// has its own row and walks the pieces.
// grid: (rows of a row tile and all key heads / rows of a workgroup, ranges - 1)
constexpr int kJoinThreads = 256;
template <int D, bool FP8, bool SPREAD>
__global__ __launch_bounds__(kJoinThreads) void cache_join_kernel(const CacheAttentionArgs a, const CachePlan plan) {
  constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes;
  fetch_arguments(a, plan);
  const Partials part = partials(a, plan);
  const int w = blockIdx.y + 1;
  const int4 job = part.joins[w];
  const int pieces = job.x, first = job.y, rows = job.z;
  if (pieces == 0) return;
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int row = SPREAD ? (int)blockIdx.x : (int)blockIdx.x * kGroups + group;
  const int head = divide(row, plan.tile_rows), in_tile = row - head * plan.tile_rows;
  const int i = job.w * plan.tile + in_tile;
  const bool there = head < a.c.H && i < rows;
  RowState state;
  if (there) add_pieces<D>(a, plan, part, w, head, in_tile, lane, SPREAD ? group : 0, SPREAD ? kGroups : 1, pieces, state);
  if constexpr (SPREAD) {
    __shared__ float4 acc_lds[kGroups][kLanes];
    __shared__ float4 stat_lds[kGroups];
    acc_lds[group][lane] = state.acc;
    if (lane == 0) stat_lds[group] = float4{state.ref, state.sum, state.sum16, 0.0f};
    __syncthreads();
    if (group != 0) return;
    const int used = pieces < kGroups ? pieces : kGroups;
    for (int k = 1; k < used; ++k) state.add(stat_lds[k], acc_lds[k][lane]);
  }
  if (there) store_state<D, FP8>(a, state, first, i, head, lane);
}

template <int D, bool FP8, class Args>
void launch_tiles(const Args& a, const CachePlan& plan, hipStream_t stream) {
  const unsigned grid = (unsigned)plan.workgroups;
  if (plan.tile == 16) cache_attention_kernel<D, FP8, 1><<<grid, kThreads, 0, stream>>>(a, plan);
  else cache_attention_kernel<D, FP8, 2><<<grid, kThreads, 0, stream>>>(a, plan);
}

template <int D, bool FP8>
void launch_join(const CacheAttentionArgs& a, const CachePlan& plan, hipStream_t stream) {
  const unsigned rows = (unsigned)(plan.tile_rows * a.c.H), per = kJoinThreads / (D / 4);
  // many pieces a row tile: a workgroup for each row
  if (plan.ranges >= 16 * a.B * plan.row_tiles)
    cache_join_kernel<D, FP8, true><<<dim3(rows, plan.ranges - 1), kJoinThreads, 0, stream>>>(a, plan);
  else
    cache_join_kernel<D, FP8, false><<<dim3((rows + per - 1) / per, plan.ranges - 1), kJoinThreads, 0, stream>>>(a, plan);
}

// f(head dimension, format) as constants.
template <class F>
void for_format(const CacheView& c, F&& f) {
  using std::integral_constant;
  if (c.d == 64 && c.fp8) f(integral_constant<int, 64>{}, integral_constant<bool, true>{});
  else if (c.d == 64) f(integral_constant<int, 64>{}, integral_constant<bool, false>{});
  else if (c.fp8) f(integral_constant<int, 128>{}, integral_constant<bool, true>{});
  else f(integral_constant<int, 128>{}, integral_constant<bool, false>{});
}

}  // namespace

}  // namespace fp4attn
