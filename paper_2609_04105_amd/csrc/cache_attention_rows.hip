// Attention over the cache for many rows (tokens times heads of a group): trees of drafted
// tokens, chunks of a prompt.
//
// The same mathematics and operand orders as cache_attention.hip; what bounds it is another:
// with 128 rows a key costs 128 * 4 D flop and 136 bytes (MXFP4, D 128), so the matrix unit and the
// softmax's vector work do, and turning codes into bf16 must not be repeated by every wave.
// The four waves of a workgroup take 32 rows each and walk the same keys; each 32-key tile is
// turned into bf16 operands once, K by two waves and V by the other two, into LDS, in the order
// in which every lane reads its own 16 bytes of a product's A operand (no bank conflicts, no
// transposing).  Two buffers: a tile is converted while the one before is used, and loaded
// while the one before that is; one barrier a tile.
#include "cache_attention.hpp"

namespace fp4attn {

namespace {

constexpr int kNr = 2;    // 16-row tiles of a wave
constexpr int kRing = 4;  // tiles whose codes are in LDS or on the way
static_assert(kRowsTile == 16 * kNr * kWaves, "rows of a workgroup");

// Copies of 16 and 4 bytes a lane from memory to LDS bytes lds + 16 lane, lds + 4 lane.  Assembly, so
// that the compiler counts neither the copies nor the LDS they write (it would wait for all of
// them before every LDS read); the wave waits for its own with wait_copies.
__device__ __forceinline__ void copy16(unsigned lds, const uint8_t* p) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "{m0}"(uniform((int)lds)) : "memory");
}
__device__ __forceinline__ void copy4(unsigned lds, const uint8_t* p) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dword %0, off" ::"v"(p), "{m0}"(uniform((int)lds)) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_copies() {  // until at most N vector memory operations are in flight
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// A wave's share of a tile's codes, as it lies in LDS: of K (waves 0, 1: halves 0, 1) every lane a key's
// D / 4 values, of V (waves 2, 3) four keys' D / 16 values; then the tile's K or V scales.
template <int D, bool FP8>
struct Share {
  using F = Format<D, FP8>;
  static constexpr int kWords = F::kKWords, kBytes = 4 * kWords;  // of a lane
  static constexpr int kScaleBytes = kTile * F::kBlocks;
  static constexpr int kSize = 64 * kBytes + kScaleBytes;
  static constexpr int kCopies = (kWords == 2 ? 2 : kWords / 4) + 1;
  static_assert(F::kVWords == 2 * F::kKWords, "half a V run is a K run");

  static __device__ __forceinline__ void copy(unsigned lds, const CacheView& c, const Pages& pages, int key0, int head,
                                              int wave, int lane) {
    asm volatile("" : "+v"(lane));  // offsets are formed here and not held through the loop
    const unsigned m = lane & 15, g = (unsigned)lane >> 4;
    const bool is_k = wave < 2;
    const int64_t row = base_row(c, pages, key0, head, is_k ? m >= 8 : g >= 2);
    const unsigned key = (m >> 2) * 8 + (m & 3) + 4 * wave;
    const uint8_t* p = (is_k ? c.k_codes : c.v_codes) + row * (4 * kBytes) +
                       (is_k ? key * (4 * kBytes) + g * kBytes : (unsigned)(lane * 2 + (wave - 2)) * kBytes);
    if constexpr (kWords == 2) {
      copy4(lds, p);
      copy4(lds + 256, p + 4);
    } else {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) copy16(lds + 1024 * i, p + 16 * i);
    }
    // the scales of 32 keys lie together, 16 keys in a half (K by key, V by eight keys)
    if (lane < kScaleBytes / 4) {
      const int64_t half = base_row(c, pages, key0, head, lane >= kScaleBytes / 8);
      copy4(lds + 64 * kBytes, (is_k ? c.k_scales : c.v_scales) + half * F::kBlocks + 4 * lane);
    }
  }

  unsigned w[kWords];
  unsigned scale;  // K: an E8M0 byte; V: four
  __device__ __forceinline__ void read(const uint8_t* lds, int wave, int lane) {
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
    const unsigned m = lane & 15, g = (unsigned)lane >> 4;
    const uint8_t* sc = lds + 64 * kBytes;
    if (wave < 2) scale = sc[((m >> 2) * 8 + (m & 3) + 4 * wave) * F::kBlocks + g * F::kBlocks / 4];
    else scale = *reinterpret_cast<const unsigned*>(sc + (g * F::kBlocks + m * F::kBlocks / 16) * 8 + 4 * (wave - 2));
  }
};

template <int D, bool FP8>
__global__ __launch_bounds__(kThreads, rows_per_cu(D, FP8)) void cache_rows_kernel(const CacheAttentionArgs a, const CachePlan plan) {
  using F = Format<D, FP8>;
  __shared__ v4i k_lds[2][2][F::kSteps][64];  // [buffer][half][step][lane]
  __shared__ v4i v_lds[2][F::kDTiles][64];    // [buffer][product][lane]
  using Codes = Share<D, FP8>;
  __shared__ __attribute__((aligned(16))) uint8_t code_lds[kRing][kWaves][Codes::kSize];
  __shared__ unsigned huge_lds[2][2];         // [buffer][keys 0-3, 4-7 of eight]: a non-finite V block that some row sees

  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const Place place = place_of(a, plan);
  const int head = place.head;
  if (place.w >= plan.ranges) return;
  Range range = open_range(a, plan, place);
  if (range.begin >= range.end) return;
  const float factor = a.softmax_scale * kLog2e * (FP8 ? 1.0f : 1.0f / 6.0f);

  Part part;
  while (open_part(a, plan, range, place.tile, &part)) {
    const Sequence seq = range.seq;
    const int rows = seq.tokens * a.G, row0 = place.tile * kRowsTile + 16 * kNr * wave;

    // this lane's rows (the same for the four lane groups) and its part of their queries
    int token[kNr];  // of the sequence
    v4i q[kNr][F::kSteps];
#pragma unroll
    for (int r = 0; r < kNr; ++r) {
      const int i = row0 + 16 * r + m, ic = i < rows ? i : rows - 1;
      token[r] = ic / a.G;
      const int h = head * a.G + (ic - token[r] * a.G);
      const uint16_t* p = static_cast<const uint16_t*>(a.q) + (int64_t)(seq.first + token[r]) * a.q_stride + h * D + g * (D / 4);
#pragma unroll
      for (int s = 0; s < F::kSteps; ++s) q[r][s] = reinterpret_cast<const v4i*>(p)[s];
    }
    v4f acc[kNr][F::kDTiles];
    v4f sum16 = {0, 0, 0, 0};
    unsigned poisoned = 0;
    float ref[kNr], sum[kNr];
#pragma unroll
    for (int r = 0; r < kNr; ++r) {
#pragma unroll
      for (int t = 0; t < F::kDTiles; ++t) acc[r][t] = v4f{0, 0, 0, 0};
      ref[r] = -__builtin_inff();
      sum[r] = 0.0f;
    }
    const ScalarInts table = (ScalarInts)(uintptr_t)(a.page_table + (int64_t)range.b * a.max_pages);
    // The wave's codes of the tile at key0, in place `slot` of the ring, into buffer `buf`.
    auto convert = [&](const Pages& pages, int key0, int slot, int buf) {
      Codes raw;
      raw.read(code_lds[slot][wave], wave, lane);
      if (wave < 2) {
        const float scale = scale_of(raw.scale);
        static_for<F::kSteps>([&](auto S_) {
          constexpr int st = decltype(S_)::value;
          v4i kk;
          static_for<4>([&](auto I_) {
            constexpr int i = decltype(I_)::value;
            kk[i] = (int)code_pair<4 * st + i, FP8>(raw.w, scale);
          });
          k_lds[buf][wave][st][lane] = kk;
        });
        return;
      }
      const int half = wave - 2;
      const bool page0 = is_page(a.c, pages.p0), page1 = is_page(a.c, pages.p1);
      if (key0 + kTile > part.common || !page0 || !page1) {
        // Keys that no row sees hold anything: their V codes and scales become zero.  A
        // non-finite block of the others becomes zero too, and is looked for by the rows.
        const unsigned there = (g >= 2 ? page1 : page0) ? below(seq.keys - (key0 + 8 * g)) >> (4 * half) : 0u;
        bool huge = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool in = there >> j & 1, big = (raw.scale >> (8 * j) & 255u) >= kHugeScale<FP8>;
          huge |= in && big;
          const unsigned keep = in && !big ? ~0u : 0u;
          raw.scale &= keep | ~(255u << (8 * j));
          if constexpr (raw.kWords >= 4) {
#pragma unroll
            for (int i = 0; i < raw.kWords / 4; ++i) raw.w[j * (raw.kWords / 4) + i] &= keep;
          } else {
            raw.w[j / 2] &= keep | (j % 2 ? 0x0000ffffu : 0xffff0000u);
          }
        }
        const bool any = __any(huge);
        if (lane == 0) huge_lds[buf][half] = any;
      }
      const unsigned sc[2] = {raw.scale, 0};
      float scale[4];
      static_for<4>([&](auto J_) { scale[decltype(J_)::value] = scale_of_key<decltype(J_)::value>(sc); });
      static_for<F::kDTiles / 2>([&](auto E_) {
        constexpr int e = decltype(E_)::value;  // values 2 e, 2 e + 1 of the part
        unsigned x[4];
        static_for<4>([&](auto J_) {
          constexpr int j = decltype(J_)::value;
          x[j] = code_pair<j * (F::kDTiles / 2) + e, FP8>(raw.w, scale[j]);
        });
        uint2* lo = reinterpret_cast<uint2*>(&v_lds[buf][2 * e][lane]) + half;
        uint2* hi = reinterpret_cast<uint2*>(&v_lds[buf][2 * e + 1][lane]) + half;
        *lo = uint2{__builtin_amdgcn_perm(x[1], x[0], 0x05040100u), __builtin_amdgcn_perm(x[3], x[2], 0x05040100u)};
        *hi = uint2{__builtin_amdgcn_perm(x[1], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[2], 0x07060302u)};
      });
    };

    auto attend = [&](const Pages& pages, int key0, int buf) {
      const bool page0 = is_page(a.c, pages.p0), page1 = is_page(a.c, pages.p1);
      // S^T: register i of half h is key 8 g + 4 h + i
      v4f s[kNr][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int r = 0; r < kNr; ++r) s[r][h] = v4f{0, 0, 0, 0};
#pragma unroll
        for (int st = 0; st < F::kSteps; ++st) {
          const v4i kk = k_lds[buf][h][st][lane];
#pragma unroll
          for (int r = 0; r < kNr; ++r) s[r][h] = mfma_16x16x32(kk, q[r][st], s[r][h]);
        }
      }
      if (key0 + kTile > part.common || !page0 || !page1) {
        const int base = key0 + 8 * g;
        const unsigned there = (g >= 2 ? page1 : page0) ? below(seq.keys - base) : 0u;
        unsigned see[kNr];
#pragma unroll
        for (int r = 0; r < kNr; ++r) {
          see[r] = there & row_sees(a, seq, part, token[r], base);
#pragma unroll
          for (int j = 0; j < 8; ++j) s[r][j / 4][j % 4] = see[r] >> j & 1 ? s[r][j / 4][j % 4] : -__builtin_inff();
        }
        if (huge_lds[buf][0] | huge_lds[buf][1]) {  // lane group g holds outputs of d block g (d = 64: g / 2)
#pragma unroll
          for (int r = 0; r < kNr; ++r) see[r] = groups_or(see[r] << (8 * g));
          const int blk = g * F::kBlocks / 4;
          for (int k = 0; k < kTile; ++k) {
            const int page = k >= 16 ? pages.p1 : pages.p0, key = key0 + k;
            if (!is_page(a.c, page) || key >= seq.keys) continue;
            const int64_t group = row_of(a.c, page, head, key & ((1 << a.c.page_shift) - 1)) >> 3;
            const bool big = a.c.v_scales[(group * F::kBlocks + blk) * 8 + (k & 7)] >= kHugeScale<FP8>;
#pragma unroll
            for (int r = 0; r < kNr; ++r) poisoned |= big ? (see[r] >> k & 1) << r : 0u;
          }
        }
      }
      float top[kNr];
      bool rise = false;
#pragma unroll
      for (int r = 0; r < kNr; ++r) {
        top[r] = groups_max(max8(s[r])) * factor;
        rise |= top[r] > ref[r] + kLag;
      }
      if (__any(rise)) {
#pragma unroll
        for (int r = 0; r < kNr; ++r) {
          const float now = fmaxf(ref[r], top[r]);
          const float down = now == ref[r] ? 1.0f : __builtin_amdgcn_exp2f(ref[r] - now);
          ref[r] = now;
          sum[r] *= down;
          sum16[r] *= down;
#pragma unroll
          for (int t = 0; t < F::kDTiles; ++t) acc[r][t] *= down;
        }
      }
      v4i p[kNr];
#pragma unroll
      for (int r = 0; r < kNr; ++r) {
        p[r] = probabilities(s[r], factor, ref[r], &sum[r]);
        const int one = (lane & 3) == r ? 0x3f803f80 : 0;
        sum16 = mfma_16x16x32(v4i{one, one, one, one}, p[r], sum16);
      }
      // O^T: product t has rows d = D / 16 * m + t
#pragma unroll
      for (int t = 0; t < F::kDTiles; ++t) {
        const v4i vv = v_lds[buf][t][lane];
#pragma unroll
        for (int r = 0; r < kNr; ++r) acc[r][t] = mfma_16x16x32(vv, p[r], acc[r][t]);
      }
    };

    // Tile i of the part: its codes are copied into place i % kRing of the ring from kRing tiles
    // before, when the place's last tile has been converted by every wave, and converted one
    // tile before.  pages[j]: of the tile j ahead.
    int key0 = part.begin, buf = 0, slot = 0;
    if (key0 < part.end) {
      Pages pages[kRing + 1];
      auto pages_at = [&](int key) { return key < part.end ? find_pages(a, table, key) : Pages{0, 0}; };
      auto copy = [&](const Pages& p, int key, int to) {
        if (key < part.end) Codes::copy((unsigned)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)code_lds[to][wave], a.c, p, key, head, wave, lane);
      };
#pragma unroll
      for (int j = 0; j <= kRing; ++j) pages[j] = pages_at(key0 + j * kTile);
#pragma unroll
      for (int j = 0; j < kRing; ++j) copy(pages[j], key0 + j * kTile, j);
      if (key0 + (kRing - 1) * kTile < part.end) wait_copies<(kRing - 1) * Codes::kCopies>();
      else wait_copies<0>();
      convert(pages[0], key0, 0, 0);
      __syncthreads();
      while (true) {
        const int ahead = key0 + kTile;
        const Pages after = pages_at(key0 + (kRing + 1) * kTile);
        if (ahead < part.end) {
          if (key0 + (kRing - 1) * kTile < part.end) wait_copies<(kRing - 2) * Codes::kCopies>();
          else wait_copies<0>();
          convert(pages[1], ahead, slot + 1 == kRing ? 0 : slot + 1, buf ^ 1);
          copy(pages[kRing], key0 + kRing * kTile, slot);
        }
        if (row0 < rows) attend(pages[0], key0, buf);
        if (ahead >= part.end) break;
        __syncthreads();
        buf ^= 1;
        slot = slot + 1 == kRing ? 0 : slot + 1;
        key0 = ahead;
#pragma unroll
        for (int j = 0; j < kRing; ++j) pages[j] = pages[j + 1];
        pages[kRing] = after;
      }
    }

    // Register i of product t is column D / 16 * (4 g + i) + t.
#pragma unroll
    for (int r = 0; r < kNr; ++r) {
      const int i = row0 + 16 * r + m;
      const float total = groups_sum(sum[r]);
      if (i >= rows) continue;
      const int64_t piece = partial_row(a, plan, place.w, part.first ? 1 : 0, head, place.tile) + (16 * kNr * wave + 16 * r + m);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float o[F::kDTiles];
#pragma unroll
        for (int t = 0; t < F::kDTiles; ++t) o[t] = acc[r][t][j];
        store_columns<D, FP8>(a, plan, seq, i, head, 4 * g + j, part.whole, piece, ref[r], total, sum16[r],
                              (poisoned >> r & 1) != 0, o);
      }
    }
    if (!next_sequence(a, plan, place.tile, part.stop, range)) break;
    __syncthreads();
  }
}

}  // namespace

void launch_cache_rows(const CacheAttentionArgs& a, const CachePlan& plan, hipStream_t stream) {
  const unsigned grid = (unsigned)plan.workgroups;
  if (a.c.d == 64 && a.c.fp8) cache_rows_kernel<64, true><<<grid, kThreads, 0, stream>>>(a, plan);
  else if (a.c.d == 64) cache_rows_kernel<64, false><<<grid, kThreads, 0, stream>>>(a, plan);
  else if (a.c.fp8) cache_rows_kernel<128, true><<<grid, kThreads, 0, stream>>>(a, plan);
  else cache_rows_kernel<128, false><<<grid, kThreads, 0, stream>>>(a, plan);
}

}  // namespace fp4attn
