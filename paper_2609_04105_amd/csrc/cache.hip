// The paged key/value cache: quantizing new tokens into it, and reading tokens back.
//
// A block is 32 values of one token and head along d, so that a token can be written
// by itself; the block rules are the operand quantizers' (mx_block.hpp).  Both kernels
// are bound by memory: writing reads 2 or 4 bytes a value and leaves 17/32 (MXFP8
// 33/32), reading back the other way round.  16384 tokens, 8 heads, d = 128, bf16, MXFP4 (85 MB):
// writing 20 us, 4.2 TB/s (choosing the amplitudes, some 400 instructions a block, takes 13 us of the
// vector units by itself), reading 15 us, 5.6 TB/s.
#include "gfx950.hpp"
#include "mx_block.hpp"
#include "serving.hpp"

namespace fp4attn {

namespace {

constexpr int kThreads = 256;

// Byte offsets of one (page, head, offset in the page).
struct Place {
  int64_t row;     // (page * H + head) * page_size + offset: row of the K codes and scales
  int64_t group;   // of eight keys: (page * H + head) * page_size / 8 + offset / 8
  int key;         // offset % 8
  __device__ __forceinline__ Place(const CacheView& c, int64_t slot, int h) {
    const int64_t page = slot >> c.page_shift;
    row = ((page * c.H + h) << c.page_shift) + (slot & ((int64_t(1) << c.page_shift) - 1));
    group = row >> 3;
    key = (int)(row & 7);
  }
};

__device__ __forceinline__ bool in_cache(const CacheView& c, int64_t slot) {
  return (uint64_t)slot < (uint64_t)(c.pages << c.page_shift);
}

// One thread quantizes one block.  blockIdx.y 0: K, blocks in memory order; 1: V, eight
// tokens to consecutive threads, so that the eight keys of a group leave as one run.
template <typename T, int D, bool FP8>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(const CacheWriteArgs a) {
  constexpr unsigned kBlocks = D / 32;
  const unsigned t = blockIdx.x * kThreads + threadIdx.x;
  const bool is_v = blockIdx.y == 1;
  unsigned token, blk, h;
  if (!is_v) {
    const unsigned row = t / kBlocks;
    blk = t % kBlocks;
    token = row / (unsigned)a.c.H;
    h = row - token * (unsigned)a.c.H;
  } else {
    const unsigned row = t / (8 * kBlocks), group = row / (unsigned)a.c.H;
    blk = t / 8 % kBlocks;
    h = row - group * (unsigned)a.c.H;
    token = group * 8 + t % 8;
  }
  if (token >= a.n) return;
  const int64_t slot = a.slots[token];
  Block<T> b;  // (loaded beside the slot, not behind it)
  load_row_block(static_cast<const T*>(is_v ? a.v : a.k) + token * (is_v ? a.v_stride : a.k_stride) + h * D + blk * 32, b);
  if (!in_cache(a.c, slot)) return;
  const Place p(a.c, slot, h);
  unsigned w[FP8 ? 8 : 4], u;
  if constexpr (FP8) u = b.mxfp8(w);
  else u = b.mxfp4(w);
  if (!is_v) {
    uint4* dst = reinterpret_cast<uint4*>(a.c.k_codes + (p.row * kBlocks + blk) * (FP8 ? 32 : 16));
    dst[0] = uint4{w[0], w[1], w[2], w[3]};
    if constexpr (FP8) dst[1] = uint4{w[4], w[5], w[6], w[7]};
    a.c.k_scales[p.row * kBlocks + blk] = (uint8_t)u;
  } else {
    // 16 parts of d, each with its eight keys' bytes side by side
    constexpr int kPart = D / 16 * (FP8 ? 8 : 4) / 8, kParts = 16 / kBlocks;  // bytes of a part; parts of a block
    uint8_t* dst = a.c.v_codes + ((p.group * 16 + blk * kParts) * 8 + p.key) * kPart;
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      uint8_t* at = dst + i * 8 * kPart;
      if constexpr (kPart == 8) *reinterpret_cast<uint2*>(at) = uint2{w[2 * i], w[2 * i + 1]};
      else if constexpr (kPart == 4) *reinterpret_cast<unsigned*>(at) = w[i];
      else *reinterpret_cast<uint16_t*>(at) = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
    }
    a.c.v_scales[(p.group * kBlocks + blk) * 8 + p.key] = (uint8_t)u;
  }
}

// The values of one part (D / 16 values, `w` their codes) under E8M0 byte u.  Codes / 6
// are correctly rounded by one multiplication with fp32(1/6), and the amplitude is
// applied after it, so that no value of the format's range overflows on the way.
template <int N, bool FP8>
__device__ __forceinline__ void decode(const unsigned* w, unsigned u, float (&v)[N]) {
  static_for<N / 2>([&](auto I_) {
    constexpr int i = decltype(I_)::value;
    v2f f;
    if constexpr (FP8) f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i / 2], 1.0f, i % 2 != 0);
    else f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, i);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float x = ldexpf(FP8 ? f[j] : f[j] * (1.0f / 6.0f), (int)u - 127);
      v[2 * i + j] = u == 255u ? __builtin_nanf("") : x;
    }
  });
}

template <int N>
__device__ __forceinline__ void store_values(float* p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    reinterpret_cast<float4*>(p)[i] = float4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
}
template <int N>
__device__ __forceinline__ void store_values(uint16_t* p, const float (&v)[N]) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  unsigned w[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) w[i] = __builtin_bit_cast(unsigned, bf2{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]});
  if constexpr (N == 8) *reinterpret_cast<uint4*>(p) = uint4{w[0], w[1], w[2], w[3]};
  else *reinterpret_cast<uint2*>(p) = uint2{w[0], w[1]};
}

// A thread reads one sixteenth of d of one token and head, K and V.  (With four tokens, all in flight, the
// smallest calls leave compute units without work, 1047 tokens of 8 heads 4.3 us against 3.7, and the
// largest gain nothing, 16384 tokens 16.0 against 15.1.)
constexpr int kReadTokens = kThreads / 16;

template <typename T, int D, bool FP8>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(const CacheReadArgs a) {
  constexpr int kPart = D / 16 * (FP8 ? 8 : 4) / 8, kBlocks = D / 32, kWords = (kPart + 3) / 4;
  const int part = threadIdx.x % 16, h = blockIdx.y;
  const int64_t token = (int64_t)blockIdx.x * kReadTokens + threadIdx.x / 16;
  if (token >= a.n) return;
  const int64_t slot = a.slots[token];
  float k[D / 16], v[D / 16];
  if (in_cache(a.c, slot)) {
    const Place p(a.c, slot, h);
    const int blk = part * kBlocks / 16;
    const uint8_t* kc = a.c.k_codes + (p.row * 16 + part) * kPart;
    const uint8_t* vc = a.c.v_codes + ((p.group * 16 + part) * 8 + p.key) * kPart;
    unsigned kw[kWords], vw[kWords];
    if constexpr (kPart == 2) {
      kw[0] = *reinterpret_cast<const uint16_t*>(kc);
      vw[0] = *reinterpret_cast<const uint16_t*>(vc);
    } else {
#pragma unroll
      for (int j = 0; j < kWords; ++j) {
        kw[j] = reinterpret_cast<const unsigned*>(kc)[j];
        vw[j] = reinterpret_cast<const unsigned*>(vc)[j];
      }
    }
    decode<D / 16, FP8>(kw, a.c.k_scales[p.row * kBlocks + blk], k);
    decode<D / 16, FP8>(vw, a.c.v_scales[(p.group * kBlocks + blk) * 8 + p.key], v);
  } else {
#pragma unroll
    for (int j = 0; j < D / 16; ++j) k[j] = v[j] = 0.0f;
  }
  const int64_t at = (token * a.c.H + h) * D + part * (D / 16);
  store_values(static_cast<T*>(a.k) + at, k);
  store_values(static_cast<T*>(a.v) + at, v);
}

// f(std::integral_constant<int, d>, std::bool_constant<fp8>)
template <class F>
void with_format(const CacheView& c, F&& f) {
  if (c.d == 64 && c.fp8) f(std::integral_constant<int, 64>{}, std::true_type{});
  else if (c.d == 64) f(std::integral_constant<int, 64>{}, std::false_type{});
  else if (c.fp8) f(std::integral_constant<int, 128>{}, std::true_type{});
  else f(std::integral_constant<int, 128>{}, std::false_type{});
}

}  // namespace

hipError_t launch_cache_write(const CacheWriteArgs& a, hipStream_t stream) {
  const int64_t threads = (a.n + 7) / 8 * 8 * a.c.H * (a.c.d / 32);
  const dim3 grid((unsigned)((threads + kThreads - 1) / kThreads), 2);
  with_format(a.c, [&](auto D_, auto FP8_) {
    constexpr int D = decltype(D_)::value;
    constexpr bool kFp8 = decltype(FP8_)::value;
    if (a.bf16) cache_write_kernel<uint16_t, D, kFp8><<<grid, kThreads, 0, stream>>>(a);
    else cache_write_kernel<float, D, kFp8><<<grid, kThreads, 0, stream>>>(a);
  });
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheReadArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.n + kReadTokens - 1) / kReadTokens), (unsigned)a.c.H);
  with_format(a.c, [&](auto D_, auto FP8_) {
    constexpr int D = decltype(D_)::value;
    constexpr bool kFp8 = decltype(FP8_)::value;
    if (a.bf16) cache_read_kernel<uint16_t, D, kFp8><<<grid, kThreads, 0, stream>>>(a);
    else cache_read_kernel<float, D, kFp8><<<grid, kThreads, 0, stream>>>(a);
  });
  return hipGetLastError();
}

}  // namespace fp4attn
