// Attention over the cache for many rows (tokens times heads of a group): trees of drafted
// tokens, chunks of a prompt.
//
// The same mathematics and operand orders as cache_attention_tiles.hpp; what bounds it is another:
// with 128 rows a key costs 128 * 4 D flop and 136 bytes (MXFP4, D 128), so the matrix unit and the
// softmax's vector work do, and turning codes into bf16 must not be repeated by every wave.
// The four waves of a workgroup take 32 rows each and walk the same keys; the codes of a step of 64
// keys are turned into bf16 operands once, a quarter by each wave, into LDS, in the order in which
// every lane reads its own 16 bytes of a product's A operand (no bank conflicts, no transposing).  The
// codes come by copies to LDS that hold no registers, sent one or two steps ahead.  Two barriers
// a step; the second workgroup of a CU fills them.
//
// Measured, d = 128, MXFP4, 32 sequences of 8192 keys and less, trees of 64 tokens, 8 key heads of 8 query heads:
// 362 us, 738 TFLOP/s (a large bf16 matrix product: 1170); the last 2048 of 8192 tokens, causal, 564 us, 854 over the keys
// that their rows see, d = 64 456 us, 527; a prompt of 8192 tokens 2101 us, 523 (its cut is uneven: cache_attention.hpp).
// Counters of the first: the matrix unit is busy 33 % of the time, vector instructions take 42 %, LDS 33 %; two waves a SIMD
// overlap them in part.  Work put between the products of the same wave (converting V and K, the second tile's
// probabilities) made it 1 to 3 % slower, four sums side by side in the K products changed nothing.
#pragma once

#include "cache_attention.hpp"

namespace fp4attn {

namespace {

constexpr int kNr = 2;                    // 16-row tiles of a wave
constexpr int kTiles = 2;                 // 32-key tiles of a step
constexpr int kKeys = kTiles * kTile;
static_assert(kTiles == kWaves / 2 && kUnit % kKeys == 0, "a step that is cut short is the last of its sequence");
static_assert(kRowsTile == 16 * kNr * kWaves, "rows of a workgroup");

// Copies of 16 and 4 bytes a lane from memory to LDS bytes lds + 16 lane, lds + 4 lane: from base + off with
// one base for the wave, or from the lane's p.  Assembly, so that the compiler counts neither the
// copies nor the LDS they write (it would wait for all of them before every LDS read); the wave
// waits for its own with wait_copies.  Nor does it look for hazards in there: a scalar register that
// a vector instruction wrote must be five wait states old.
template <int BYTES>
__device__ __forceinline__ void copy(unsigned lds, const uint8_t* base, unsigned off) {
  static_assert(BYTES == 16 || BYTES == 4, "sizes of the copy instructions");
  if constexpr (BYTES == 16) asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
  else asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}
template <int BYTES>
__device__ __forceinline__ void copy(unsigned lds, const uint8_t* p) {
  if constexpr (BYTES == 16) asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "{m0}"(lds) : "memory");
  else asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, off" ::"v"(p), "{m0}"(lds) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_copies() {  // until at most N vector memory operations are in flight
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// A wave's share of a step's codes, as it lies in LDS: of tile wave / 2, half h = wave % 2 of K (every lane a
// key's D / 4 values) and keys 4 h .. 4 h + 3 of every eight of V (every lane D / 16 values of
// each); then the tile's scales.
template <int D, bool FP8>
struct Share {
  using F = Format<D, FP8>;
  static constexpr int kWords = F::kKWords, kBytes = 4 * kWords;  // of a lane, for K and for V
  static constexpr int kScaleBytes = kTile * F::kBlocks;          // of a tile's K; V as much
  static constexpr int kV = 64 * kBytes, kScales = 2 * kV, kSize = kScales + 2 * kScaleBytes;
  static constexpr int kStep = kWords == 2 ? 4 : 16;
  static constexpr int kCopies = 2 * kBytes / kStep + 1;
  static_assert(F::kVWords == 2 * F::kKWords, "half a V run is a K run");

  static __device__ __forceinline__ void fetch(unsigned lds, const CacheView& c, const Pages& pages, int key0, int head,
                                               int half, int lane) {
    asm volatile("" : "+v"(lane));  // offsets are formed here and not held through the loop
    const unsigned m = lane & 15, g = (unsigned)lane >> 4, key = (m >> 2) * 8 + (m & 3) + 4 * half;
    const unsigned k_off = key * (4 * kBytes) + g * kBytes, v_off = (unsigned)(lane * 2 + half) * kBytes;
    // the scales of 32 keys lie together, 16 keys in a half (K by key, V by eight keys)
    constexpr unsigned n = kScaleBytes / 4;
    const bool of_v = (unsigned)lane >= n;
    const unsigned word = of_v ? lane - n : lane;
    const uint8_t* scales = of_v ? c.v_scales : c.k_scales;
    const int64_t row = base_row(c, pages, key0, head, false);
    if (c.page_shift != 4) {
      const uint8_t *kb = c.k_codes + row * (4 * kBytes), *vb = c.v_codes + row * (4 * kBytes);
#pragma unroll
      for (int i = 0; i < kBytes / kStep; ++i) {
        copy<kStep>(lds + 64 * kStep * i, kb, k_off + kStep * i);
        copy<kStep>(lds + kV + 64 * kStep * i, vb, v_off + kStep * i);
      }
      if ((unsigned)lane < 2 * n) copy<4>(lds + kScales, scales + (row * F::kBlocks + 4 * word));
    } else {
      const int64_t other = base_row(c, pages, key0, head, true);
      const uint8_t *kp = c.k_codes + ((m >= 8 ? other : row) * (4 * kBytes) + k_off);
      const uint8_t *vp = c.v_codes + ((g >= 2 ? other : row) * (4 * kBytes) + v_off);
#pragma unroll
      for (int i = 0; i < kBytes / kStep; ++i) {
        copy<kStep>(lds + 64 * kStep * i, kp + kStep * i);
        copy<kStep>(lds + kV + 64 * kStep * i, vp + kStep * i);
      }
      if ((unsigned)lane < 2 * n) copy<4>(lds + kScales, scales + ((word >= n / 2 ? other : row) * F::kBlocks + 4 * word));
    }
  }

  unsigned k[kWords], v[kWords];
  unsigned k_scale, v_scales;  // an E8M0 byte; four
  static __device__ __forceinline__ void read_words(const uint8_t* lds, int lane, unsigned (&w)[kWords]) {
    if constexpr (kWords == 2) {
      w[0] = reinterpret_cast<const unsigned*>(lds)[lane];
      w[1] = reinterpret_cast<const unsigned*>(lds + 256)[lane];
    } else {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const uint4 x = reinterpret_cast<const uint4*>(lds + 1024 * i)[lane];
        w[4 * i] = x.x;
        w[4 * i + 1] = x.y;
        w[4 * i + 2] = x.z;
        w[4 * i + 3] = x.w;
      }
    }
  }
  __device__ __forceinline__ void read(const uint8_t* lds, int half, int lane) {
    read_words(lds, lane, k);
    read_words(lds + kV, lane, v);
    const unsigned m = lane & 15, g = (unsigned)lane >> 4;
    k_scale = lds[kScales + ((m >> 2) * 8 + (m & 3) + 4 * half) * F::kBlocks + g * F::kBlocks / 4];
    v_scales = *reinterpret_cast<const unsigned*>(lds + kScales + kScaleBytes + (g * F::kBlocks + m * F::kBlocks / 16) * 8 + 4 * half);
  }
};

template <int D, bool FP8, class Args>
__global__ __launch_bounds__(kThreads, kRowsPerCu) void cache_rows_kernel(const Args a, const CachePlan plan) {
  using F = Format<D, FP8>;
  using Codes = Share<D, FP8>;
  constexpr int kRing = FP8 && D == 128 ? 2 : 3;  // steps whose codes are in LDS or on the way (LDS for two workgroups)
  __shared__ v4i k_lds[kTiles][2][F::kSteps][64];  // [tile][half][step of d][lane]
  __shared__ uint2 v_lds[kTiles][F::kDTiles][2][64];  // [tile][product][keys 0-3, 4-7 of eight][lane]
  __shared__ __attribute__((aligned(16))) uint8_t code_lds[kRing][kWaves][Codes::kSize];
  __shared__ unsigned odd_lds[kTiles][2];  // [tile][keys 0-3, 4-7 of eight]: V that is no number, of a key that some row may see

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

  // Of a CU's two workgroups the one that came first, of the first half of the grid, is served first: a step took it
  // 2.17 us and the other 2.62, and it ended 60 us of 370 earlier.  The later one goes before it in every
  // second step: 373 -> 357 us, 8 of 512-token chunks 293 -> 282.
  const bool late = in_second_half(a, plan);
  Part part;
  while (open_part(a, plan, range, &part)) {
    const Sequence seq = range.seq;
    const int rows = seq.tokens * a.G, row0 = range.tile * kRowsTile + 16 * kNr * wave;

    // this lane's rows (the same for the four lane groups) and its part of their queries
    int token[kNr];  // of the sequence
    float slope[kNr];
    v4i q[kNr][F::kSteps];
#pragma unroll
    for (int r = 0; r < kNr; ++r) {
      const int i = row0 + 16 * r + m, ic = i < rows ? i : rows - 1;
      token[r] = divide(ic, a.G);
      const int h = head * a.G + (ic - token[r] * a.G);
      slope[r] = slope_of(a, h);
      const uint16_t* p = static_cast<const uint16_t*>(a.q) + (int64_t)(seq.first + token[r]) * a.q_stride + h * D + g * (D / 4);
#pragma unroll
      for (int s = 0; s < F::kSteps; ++s) q[r][s] = reinterpret_cast<const v4i*>(p)[s];
    }
    // (waits for the queries here: the compiler would wait in the loop, and then for the copies too)
#pragma unroll
    for (int r = 0; r < kNr; ++r)
#pragma unroll
      for (int s = 0; s < F::kSteps; ++s) asm volatile("" : "+v"(q[r][s]));
    v4f acc[kNr][F::kDTiles];
    v4f sum16[kNr];
    OddMarks<FP8, kNr> odd_marks;
    float ref[kNr], sum[kNr];
#pragma unroll
    for (int r = 0; r < kNr; ++r) {
#pragma unroll
      for (int t = 0; t < F::kDTiles; ++t) acc[r][t] = v4f{0, 0, 0, 0};
      sum16[r] = v4f{0, 0, 0, 0};
      ref[r] = -__builtin_inff();
      sum[r] = 0.0f;
    }
    if constexpr (Args::kShaped && !Args::kPrefix)
      if (part.first && shared_keys(a, seq) && row0 < rows) {  // a row begins with the pieces of the shared prefix
#pragma unroll
        for (int r = 0; r < kNr; ++r) {
          const int i = row0 + 16 * r + m, ic = i < rows ? i : rows - 1, h = head * a.G + (ic - token[r] * a.G);
          const int row = (seq.first + token[r]) * a.Hq + h;  // below 2^31
          const float lower = slope[r] * (float)(seq.prefix + token[r] - a.shared);
          for (int k = 0; k < a.prefix_pieces; ++k)
            add_piece<D>(a, k, row, g, lower, &ref[r], &sum[r], &sum16[r], acc[r]);
        }
      }
    const ScalarInts table = (ScalarInts)(uintptr_t)(a.page_table + (int64_t)range.b * a.max_pages);
    auto pages_of = [&](int key) { return key < part.end ? find_pages(a, table, key) : Pages{0, 0}; };
    // the wave's tile of every step and its halves there
    const int my_tile = wave / 2, half = wave % 2;
    auto fetch = [&](const Pages& p, int key, int slot) {
      if (key < part.end)
        Codes::fetch((unsigned)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)code_lds[slot][wave], a.c, p, key, head,
                     half, lane);
    };

    // Keys that all rows of the wave see: [from, common).
    int common = part.common, from = 0;
    if constexpr (Args::kShaped)
      if (!a.tree) {
        const int last = (row0 + 16 * kNr < rows ? row0 + 16 * kNr : rows) - 1;
        common = seq.prefix + divide(row0 < rows ? row0 : rows - 1, a.G) + 1;
        if (a.window) from = seq.prefix + divide(last, a.G) + 1 - a.window;
        if (a.open_keys) common = common > a.open_keys[range.b] ? common : a.open_keys[range.b];
        common = common > seq.keys ? seq.keys : common;
      }

    // The codes of the wave's tile (keys from key0) into operands.  Keys from part.end on are seen by no row.
    auto convert = [&](Codes& raw, const Pages& pages, int key0) {
      const float k_scale = scale_of(raw.k_scale);
      static_for<F::kSteps>([&](auto S_) {
        constexpr int st = decltype(S_)::value;
        v4i kk;
        static_for<4>([&](auto I_) {
          constexpr int i = decltype(I_)::value;
          kk[i] = (int)code_pair<4 * st + i, FP8>(raw.k, k_scale);
        });
        k_lds[my_tile][half][st][lane] = kk;
      });
      const bool page0 = is_page(a.c, pages.p0), page1 = is_page(a.c, pages.p1);
      if (some_hidden(a, part, key0, kTile) || !page0 || !page1) {
        // Keys that no row sees hold anything: their V codes and scales become zero.  A
        // non-finite block of the others becomes zero too, as a NaN code of MXFP8 does, and is looked for by the rows.
        const unsigned there = (g >= 2 ? page1 : page0) ? may_see(a, part, part.end, key0 + 8 * g) >> (4 * half) : 0u;
        unsigned odd = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool in = there >> j & 1, big = (raw.v_scales >> (8 * j) & 255u) >= kHugeScale<FP8>;
          odd |= in && big ? 1u : 0u;
          const unsigned keep = in && !big ? ~0u : 0u;
          raw.v_scales &= keep | ~(255u << (8 * j));
          if constexpr (Codes::kWords >= 4) {
#pragma unroll
            for (int i = 0; i < Codes::kWords / 4; ++i) raw.v[j * (Codes::kWords / 4) + i] &= keep;
          } else {
            raw.v[j / 2] &= keep | (j % 2 ? 0x0000ffffu : 0xffff0000u);
          }
        }
        if constexpr (FP8)
#pragma unroll
          for (int i = 0; i < Codes::kWords; ++i) odd |= nan_codes(raw.v[i]);
        const bool any = __any(odd);
        if (lane == 0) odd_lds[my_tile][half] = any;
        if constexpr (FP8)
          if (any)
#pragma unroll
            for (int i = 0; i < Codes::kWords; ++i) raw.v[i] = without_nan_codes(raw.v[i]);
      }
      const unsigned sc[2] = {raw.v_scales, 0};
      float scale[4];
      static_for<4>([&](auto J_) { scale[decltype(J_)::value] = scale_of_key<decltype(J_)::value>(sc); });
      static_for<F::kDTiles / 2>([&](auto E_) {
        constexpr int e = decltype(E_)::value;  // values 2 e, 2 e + 1 of the part
        unsigned x[4];
        static_for<4>([&](auto J_) {
          constexpr int j = decltype(J_)::value;
          x[j] = code_pair<j * (F::kDTiles / 2) + e, FP8>(raw.v, scale[j]);
        });
        v_lds[my_tile][2 * e][half][lane] =
            uint2{__builtin_amdgcn_perm(x[1], x[0], 0x05040100u), __builtin_amdgcn_perm(x[3], x[2], 0x05040100u)};
        v_lds[my_tile][2 * e + 1][half][lane] =
            uint2{__builtin_amdgcn_perm(x[1], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[2], 0x07060302u)};
      });
    };
    auto read_v = [&](int i) {
      const uint2 lo = v_lds[i / F::kDTiles][i % F::kDTiles][0][lane], hi = v_lds[i / F::kDTiles][i % F::kDTiles][1][lane];
      return v4i{(int)lo.x, (int)lo.y, (int)hi.x, (int)hi.y};
    };

    auto attend = [&](const Pages (&pages)[kTiles], int key0) {
      // S^T: register i of half h of a tile is its key 8 g + 4 h + i
      // (operands are read one half ahead of their products, and kept there)
      v4f s[kTiles][kNr][2];
      auto multiply = [&] {
        v4i kk[2 * kTiles][F::kSteps];
        auto read_k = [&](int i) {
#pragma unroll
          for (int st = 0; st < F::kSteps; ++st) kk[i][st] = k_lds[i / 2][i % 2][st][lane];
        };
        read_k(0);
#pragma unroll
        for (int i = 0; i < 2 * kTiles; ++i) {
          if (i + 1 < 2 * kTiles) read_k(i + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int r = 0; r < kNr; ++r) s[i / 2][r][i % 2] = v4f{0, 0, 0, 0};
#pragma unroll
          for (int st = 0; st < F::kSteps; ++st)
#pragma unroll
            for (int r = 0; r < kNr; ++r) s[i / 2][r][i % 2] = mfma_16x16x32(kk[i][st], q[r][st], s[i / 2][r][i % 2]);
        }
      };
      multiply();
      if constexpr (Args::kScores) {
        const int base = key0 + 8 * g;
        if (a.cap.on) {
          // As if all were near the cap's middle, between the products; where one is not, the products are formed again.  (Asked
          // before: chunks of 1024 tokens behind a window of 1024 160 us instead of 148.)
          float most = 0.0f;
#pragma unroll
          for (int tile = 0; tile < kTiles; ++tile) most = fmaxf(most, cap_near(a, s[tile]));
          if (__any(most > a.cap.near)) {
            multiply();
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile) cap_all(a, s[tile]);
          }
          if (a.slopes)
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile) add_bias<Args>(seq, slope, token, base + kTile * tile, s[tile]);
        } else if (a.slopes) {
          if (a.open_keys) {
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile) {
              scale_scores(shape.plain, s[tile]);
              add_bias<Args>(seq, slope, token, base + kTile * tile, s[tile]);
            }
          } else {
#pragma unroll
            for (int tile = 0; tile < kTiles; ++tile)
              scale_with_bias<Args>(seq, shape.plain, slope, token, base + kTile * tile, s[tile]);
          }
        }
      }
      bool all = !some_hidden(a, part, key0, kKeys);
#pragma unroll
      for (int tile = 0; tile < kTiles; ++tile) all = all && is_page(a.c, pages[tile].p0) && is_page(a.c, pages[tile].p1);
      if (!all) {  // uniform
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile) {
          const int first = key0 + kTile * tile, base = first + 8 * g;
          const bool page0 = is_page(a.c, pages[tile].p0), page1 = is_page(a.c, pages[tile].p1);
          const bool looked = some_hidden(a, part, first, kTile) || !page0 || !page1;  // as convert did
          // The rows of a wave see more in common than those of the workgroup.  (Chunks behind a window 117 -> 112 us; plain chunks the
          // same or 1 % slower, so there every tile of the step is masked.)
          if constexpr (Args::kShaped)
            if (!looked || (page0 && page1 && !(odd_lds[tile][0] | odd_lds[tile][1]) && first >= from && first + kTile <= common)) continue;
          const unsigned there = (g >= 2 ? page1 : page0) ? may_see(a, part, part.end, base) : 0u;
          unsigned see[kNr];
#pragma unroll
          for (int r = 0; r < kNr; ++r) {
            see[r] = there & row_sees(a, seq, part, range.b, token[r], base);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              s[tile][r][j / 4][j % 4] = see[r] >> j & 1 ? s[tile][r][j / 4][j % 4] : -__builtin_inff();
          }
          if (looked && (odd_lds[tile][0] | odd_lds[tile][1])) {
#pragma unroll
            for (int r = 0; r < kNr; ++r) see[r] = groups_or(see[r] << (8 * g));
            for (int k = 0; k < kTile; ++k) {
              const int page = k >= 16 ? pages[tile].p1 : pages[tile].p0, key = first + k;
              if (!is_page(a.c, page) || key >= part.end) continue;
              const int64_t group = row_of(a.c, page, head, key & ((1 << a.c.page_shift) - 1)) >> 3;
              const unsigned columns = odd_columns<D, FP8>(a.c, group, k & 7, g);
#pragma unroll
              for (int r = 0; r < kNr; ++r) odd_marks.add(r, see[r] >> k & 1, columns);
            }
          }
        }
      }
      float top[kNr];
      bool rise = false;
#pragma unroll
      for (int r = 0; r < kNr; ++r) {
        top[r] = groups_max(fmaxf(max8(s[0][r]), max8(s[1][r]))) * factor;
        rise |= top[r] > ref[r] + kLag;
      }
      if (__any(rise)) {
#pragma unroll
        for (int r = 0; r < kNr; ++r) {
          const float now = top[r] > ref[r] + kLag ? top[r] : ref[r];  // (a row moves by its own keys alone)
          const float down = now == ref[r] ? 1.0f : __builtin_amdgcn_exp2f(ref[r] - now);
          ref[r] = now;
          sum[r] *= down;
          sum16[r] *= down;
#pragma unroll
          for (int t = 0; t < F::kDTiles; ++t) acc[r][t] *= down;
        }
      }
      constexpr int kVAhead = 4;
      v4i vv[kTiles * F::kDTiles];
#pragma unroll
      for (int i = 0; i < kVAhead; ++i) vv[i] = read_v(i);
      v4i p[kNr][kTiles];
#pragma unroll
      for (int tile = 0; tile < kTiles; ++tile)
#pragma unroll
        for (int r = 0; r < kNr; ++r) {
          p[r][tile] = probabilities(s[tile][r], factor, ref[r], &sum[r]);
          sum16[r] = mfma_16x16x32(v4i{kOnes, kOnes, kOnes, kOnes}, p[r][tile], sum16[r]);
        }
      // O^T: product t has rows d = D / 16 * m + t
#pragma unroll
      for (int i = 0; i < kTiles * F::kDTiles; ++i) {
        constexpr int n = kTiles * F::kDTiles;
        if (i + kVAhead < n) vv[i + kVAhead] = read_v(i + kVAhead);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int r = 0; r < kNr; ++r)
          acc[r][i % F::kDTiles] = mfma_16x16x32(vv[i], p[r][i / F::kDTiles], acc[r][i % F::kDTiles]);
      }
    };

    // Step i: the codes of step i + kRing - 1 are sent for (their place in the ring was read before the last
    // barrier), the step's own become operands, and after a barrier every wave uses them and reads
    // its codes of the next step.
    if (part.begin < part.end) {
      constexpr int kAhead = kRing - 1;
      const int mine = my_tile * kTile;  // the wave's tile in a step
      Codes raw;
      // the codes of the step at `key`, the first of those on the way
      auto take = [&](int key, int slot) {
        if (key + kAhead * kKeys <= part.end) wait_copies<(kAhead - 1) * Codes::kCopies>();
        else wait_copies<0>();
        raw.read(code_lds[slot][wave], half, lane);
      };
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int key = part.begin + j * kKeys + mine;
        fetch(pages_of(key), key, j);
      }
      Pages send = pages_of(part.begin + kAhead * kKeys + mine);  // of the step to send for
      take(part.begin, 0);
      for (int key0 = part.begin, slot = 0;;) {
        if (late && (key0 / kKeys & 1)) __builtin_amdgcn_s_setprio(2);
        else __builtin_amdgcn_s_setprio(0);
        const int ahead = key0 + kAhead * kKeys;
        Pages pages[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) pages[t] = pages_of(key0 + t * kTile);
        const Pages next = pages_of(ahead + kKeys + mine);
        fetch(send, ahead + mine, slot == 0 ? kRing - 1 : slot - 1);
        send = next;
        convert(raw, my_tile == 0 ? pages[0] : pages[1], key0 + mine);
        __syncthreads();
        if (row0 < rows) attend(pages, key0);
        key0 += kKeys;
        if (key0 >= part.end) break;
        slot = slot + 1 == kRing ? 0 : slot + 1;
        take(key0, slot);
        __syncthreads();
      }
    }

    // Register i of product t is column D / 16 * (4 g + i) + t.
#pragma unroll
    for (int r = 0; r < kNr; ++r) {
      const int i = row0 + 16 * r + m;
      const float total = groups_sum(sum[r]);
      if (i >= rows) continue;
      const int64_t piece = piece_row(a, plan, range, place, part, 16 * kNr * wave + 16 * r + m);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float o[F::kDTiles];
#pragma unroll
        for (int t = 0; t < F::kDTiles; ++t) o[t] = acc[r][t][j];
        store_columns<D, FP8>(a, plan, seq, i, head, 4 * g + j, !Args::kPrefix && part.whole, piece, ref[r], total, sum16[r][0],
                              odd_marks.template of<F::kDTiles>(r, j), o);
      }
    }
    if constexpr (Args::kDirect)
      if (!part.whole) join_last<D, FP8>(a, plan, range, place, &odd_lds[0][0]);
    if (!next_tile(a, plan, part.stop, range)) break;
    __syncthreads();
  }
}

template <int D, bool FP8, class Args>
void launch_rows(const Args& a, const CachePlan& plan, hipStream_t stream) {
  cache_rows_kernel<D, FP8><<<(unsigned)plan.workgroups, kThreads, 0, stream>>>(a, plan);
}

}  // namespace

}  // namespace fp4attn
