// One MXFP4 or MXFP8 block of 32 values, quantized by one thread: shared by the operand
// quantizers (quantize.hip) and the key/value cache (cache.hip).
//
// MXFP4 (eq. mx-scale): the E8M0 amplitude is 2^floor(log2 a) or 2^ceil(log2 a), a the
// absolute maximum, whichever has the smaller squared error (ties: the ceiling).
#pragma once

#include "gfx950.hpp"

namespace fp4attn {

typedef float v2f __attribute__((ext_vector_type(2)));

// bf16 fast path of the same rule, exact in 32-bit arithmetic.  A bf16 value
// has at most 8 significant bits, so r = 6 v / 2^e_ceil has at most 10 and is
// exact in fp32; the hardware converter's E2M1 rounding (nearest, ties to the
// even code, saturating at 6) gives qc = E2M1(r) and qf = E2M1(2 r) exactly and
// the decode instruction returns their values, so the rule's sum is evaluated
// exactly (see below).  The codes of the chosen amplitude are the ones already
// converted (unless the E8M0 range clamps it).
//   raw[i]: elements 2i (bits 0-15) and 2i + 1 (bits 16-31).  Returns the E8M0
//   byte; codes[j] holds elements 8 j .. 8 j + 7, even element in the low nibble.
__device__ __forceinline__ unsigned mxfp4_block_bf16(const unsigned (&raw)[16], unsigned (&codes)[4]) {
  // Block maximum on the magnitude bits, two bf16 values per packed 16-bit max:
  // magnitudes order as their bit patterns, and Inf and NaN sort above every
  // finite value.
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  u16x2 mx = {0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i) mx = __builtin_elementwise_max(mx, __builtin_bit_cast(u16x2, raw[i] & 0x7fff7fffu));
  const unsigned amax_bits = mx[0] > mx[1] ? mx[0] : mx[1];
  if (amax_bits >= 0x7f80u) {  // a NaN or an infinity in the block
#pragma unroll
    for (int j = 0; j < 4; ++j) codes[j] = 0u;
    return 255u;
  }
  // Signed values go straight into the converter: its codes carry the input's
  // sign bit (-0.0 and negative values that round to zero give 0x8).
  // encode: the codes of 6 v / 2^e, scaled in two exact steps (valid for every
  // E8M0 exponent, where the single factor 6 / 2^e may overflow).
  auto encode = [&](int e, unsigned (&w)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      unsigned acc = 0u;
      static_for<4>([&](auto P_) {
        constexpr int pb = decltype(P_)::value;
        const unsigned word = raw[4 * j + pb];
        const float v0 = __builtin_bit_cast(float, word << 16), v1 = __builtin_bit_cast(float, word & 0xffff0000u);
        acc = cvt_pk_fp4<pb>(pb == 0 ? 0u : acc, 6.0f * ldexpf(v0, -e), 6.0f * ldexpf(v1, -e), 1.0f);
      });
      w[j] = acc;
    }
  };
  if (amax_bits == 0u) {  // zero block: byte 0, every code a signed zero
    encode(0, codes);
    return 0u;
  }
  int x;
  const float m = frexpf(__builtin_bit_cast(float, amax_bits << 16), &x);  // amax = m 2^x, m in [0.5, 1)
  const int e_floor = x - 1, e_ceil = (m == 0.5f) ? x - 1 : x;
  // r = 6 v / 2^e_ceil (one exact multiply), qc = E2M1(r) and qf = E2M1(2 r)
  // (the converter divides by its scale operand and saturates at 6).  The
  // choice compares 4 sum(a r) with sum(a b), a = 2 qc - qf, b = 2 qc + qf: the
  // floor amplitude wins iff sum a (4 r - b) < 0.  Only values with |r| >= 1/8
  // have a != 0; such r are multiples of 2^-12, and |a| <= qc <= 6 because
  // qf >= qc, so both sums are exact in fp32 (multiples of 2^-13 below 2^11, and
  // of 2^-2 below 2^12).
  // The single factor 6 / 2^e_ceil is finite for e_ceil >= -125; blocks below
  // that (amax under 2^-125) take the two-step scaling of encode.
  const float sc = ldexpf(6.0f, -e_ceil);
  unsigned cc[4], cf[4];
  float s_ar = 0.0f, s_ab = 0.0f;
  auto convert = [&](auto TWO_STEP_) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      unsigned wc = 0u, wf = 0u;
      static_for<4>([&](auto P_) {
        constexpr int pb = decltype(P_)::value;
        const unsigned word = raw[4 * j + pb];
        const float v0 = __builtin_bit_cast(float, word << 16), v1 = __builtin_bit_cast(float, word & 0xffff0000u);
        float r0, r1;
        if constexpr (decltype(TWO_STEP_)::value) {
          r0 = 6.0f * ldexpf(v0, -e_ceil);
          r1 = 6.0f * ldexpf(v1, -e_ceil);
        } else {
          r0 = v0 * sc;
          r1 = v1 * sc;
        }
        wc = cvt_pk_fp4<pb>(pb == 0 ? 0u : wc, r0, r1, 1.0f);
        wf = cvt_pk_fp4<pb>(pb == 0 ? 0u : wf, r0, r1, 0.5f);
        const v2f qc = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wc, 1.0f, pb);
        const v2f qf = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(wf, 1.0f, pb);
        const float a0 = fmaf(2.0f, qc[0], -qf[0]), a1 = fmaf(2.0f, qc[1], -qf[1]);
        s_ar = fmaf(a1, r1, fmaf(a0, r0, s_ar));
        s_ab = fmaf(a1, fmaf(2.0f, qc[1], qf[1]), fmaf(a0, fmaf(2.0f, qc[0], qf[0]), s_ab));
      });
      cc[j] = wc;
      cf[j] = wf;
    }
  };
  if (e_ceil >= -125) convert(std::false_type{});
  else convert(std::true_type{});
  int e = (e_floor != e_ceil && 4.0f * s_ar < s_ab) ? e_floor : e_ceil;
  e = e < -127 ? -127 : (e > 127 ? 127 : e);
  if (e == e_ceil) {
#pragma unroll
    for (int j = 0; j < 4; ++j) codes[j] = cc[j];
  } else if (e == e_floor) {
#pragma unroll
    for (int j = 0; j < 4; ++j) codes[j] = cf[j];
  } else {  // amplitude clamped to the E8M0 range
    encode(e, codes);
  }
  return (unsigned)(e + 127);
}

// MXFP8 (E4M3 payload + E8M0 per 32 values): the amplitude is the smallest
// power of two 2^e with amax / 2^e <= 448, so no payload saturates; payloads
// are v / 2^e (exact) rounded to nearest even by the hardware converter, which
// keeps E4M3 subnormals.  Zero block: u = 0; non-finite block: u = 255, codes 0.
// Codes are stored one byte per value, in the same orientation as the MXFP4
// quantizer (axis 0: transposed).
// One MXFP8 block: returns the E8M0 byte; w[i] holds the E4M3 payloads of values
// 4 i .. 4 i + 3.
__device__ __forceinline__ unsigned mxfp8_block(const float (&v)[32], unsigned (&w)[8]) {
  float amax = 0.0f;
  bool finite = true;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    finite = finite && __builtin_isfinite(v[j]);
    amax = fmaxf(amax, fabsf(v[j]));
  }
  unsigned ubyte;
  int e = 0;
  if (!finite) {
    ubyte = 255;
  } else if (amax == 0.0f) {
    ubyte = 0;
  } else {
    int x;
    frexpf(amax, &x);          // amax = m 2^x, m in [0.5, 1)
    e = x - 9;                 // amax / 2^e in [256, 512)
    if (ldexpf(amax, -e) > 448.0f) ++e;
    e = e < -127 ? -127 : (e > 127 ? 127 : e);
    ubyte = (unsigned)(e + 127);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (finite) {
      const float a0 = ldexpf(v[4 * i], -e), a1 = ldexpf(v[4 * i + 1], -e);
      const float a2 = ldexpf(v[4 * i + 2], -e), a3 = ldexpf(v[4 * i + 3], -e);
      w[i] = cvt_pk_fp8<true>(cvt_pk_fp8<false>(0u, a0, a1), a2, a3);
    } else {
      w[i] = 0u;
    }
  }
  return ubyte;
}

// fp32 form of the same rule.  r = 6 v / 2^e has up to 26 significant bits, so
// its fp32 product is rounded to odd: truncated, with the last bit set if
// anything was lost (the fma gives the product's error exactly).  Every E2M1
// boundary (of r and of 2 r) has at most three significant bits, hence an even
// last bit, so a value rounded to odd lies on the same side of each as the exact
// product and meets one only when it is exactly there: the converter's codes
// are those of the exact r.  Values under 2^-126 of the block's scale may lose
// bits in the scaling; their code is a signed zero all the same.
__device__ __forceinline__ float six_to_odd(float m) {
  const float r = 6.0f * m, err = fmaf(6.0f, m, -r);
  const unsigned lost = err != 0.0f ? 1u : 0u, over = (as_uint(err) ^ as_uint(r)) >> 31;  // |r| > |6 m|
  return as_float((as_uint(r) - (lost & over)) | lost);
}

// The rule's sum over the block in fp64, where it is exact, from the codes of
// both amplitudes.
// (The empty asm keeps the values of the common path from staying in registers
// for this rare one, and its terms in order.)
__device__ __forceinline__ bool floor_wins_f64(const float (&v)[32], int e_ceil, const unsigned (&codes_c)[4],
                                               const unsigned (&codes_f)[4]) {
  double delta = 0.0;
  unsigned cc[4], cf[4];
  static_for<16>([&](auto I_) {
    constexpr int i = decltype(I_)::value;
    if constexpr (i % 4 == 0) {
      cc[i / 4] = codes_c[i / 4];
      cf[i / 4] = codes_f[i / 4];
      asm volatile("" : "+v"(cc[i / 4]), "+v"(cf[i / 4]), "+v"(e_ceil), "+v"(delta));
    }
    const v2f qc = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(cc[i / 4], 1.0f, i % 4);
    const v2f qf = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(cf[i / 4], 1.0f, i % 4);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const double r4 = 24.0 * (double)ldexpf(v[2 * i + t], -e_ceil);
      delta += (2.0 * qc[t] - qf[t]) * (r4 - qf[t] - 2.0 * qc[t]);
    }
  });
  return delta < 0.0;
}

// One fp32 block: returns the E8M0 byte; codes as mxfp4_block_bf16.
__device__ __forceinline__ unsigned mxfp4_block_f32(const float (&v)[32], unsigned (&codes)[4]) {
  unsigned amax_bits = 0u;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const unsigned a = as_uint(v[j]) & 0x7fffffffu;
    amax_bits = a > amax_bits ? a : amax_bits;
  }
  if (amax_bits >= 0x7f800000u) {  // a NaN or an infinity in the block
#pragma unroll
    for (int j = 0; j < 4; ++j) codes[j] = 0u;
    return 255u;
  }
  auto encode = [&](int e) {
    static_for<16>([&](auto I_) {
      constexpr int i = decltype(I_)::value;
      const float r0 = six_to_odd(ldexpf(v[2 * i], -e)), r1 = six_to_odd(ldexpf(v[2 * i + 1], -e));
      codes[i / 4] = cvt_pk_fp4<i % 4>(i % 4 == 0 ? 0u : codes[i / 4], r0, r1, 1.0f);
    });
  };
  if (amax_bits == 0u) {  // zero block: byte 0, every code a signed zero
    encode(0);
    return 0u;
  }
  int x;
  const float m = frexpf(as_float(amax_bits), &x);  // amax = m 2^x, m in [0.5, 1)
  const int e_floor = x - 1, e_ceil = (m == 0.5f) ? x - 1 : x;
  unsigned cc[4], cf[4];
  float s_ar = 0.0f, s_ab = 0.0f;
  static_for<16>([&](auto I_) {
    constexpr int i = decltype(I_)::value, w = i / 4, pb = i % 4;
    const float r0 = six_to_odd(ldexpf(v[2 * i], -e_ceil)), r1 = six_to_odd(ldexpf(v[2 * i + 1], -e_ceil));
    cc[w] = cvt_pk_fp4<pb>(pb == 0 ? 0u : cc[w], r0, r1, 1.0f);
    cf[w] = cvt_pk_fp4<pb>(pb == 0 ? 0u : cf[w], r0, r1, 0.5f);
    const v2f qc = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(cc[w], 1.0f, pb);
    const v2f qf = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(cf[w], 1.0f, pb);
    const float a0 = fmaf(2.0f, qc[0], -qf[0]), a1 = fmaf(2.0f, qc[1], -qf[1]);
    s_ar = fmaf(a1, r1, fmaf(a0, r0, s_ar));
    s_ab = fmaf(a1, fmaf(2.0f, qc[1], qf[1]), fmaf(a0, fmaf(2.0f, qc[0], qf[0]), s_ab));
    // (emits nothing: the sums are formed here and not sunk below the branch with
    // every term held in registers)
    if constexpr (pb == 3) asm volatile("" : "+v"(s_ar), "+v"(s_ab));
  });
  // s_ab is exact (see the bf16 form).  s_ar = sum a r <= 32 * 36 carries at most
  // 32 roundings of 2^-24 of it and, from each r, 2^-23: under 0.0025, so the sign
  // of 4 s_ar - s_ab stands when it is 0.0125 or more from zero.  About one block
  // in a thousand is nearer and takes the exact sum.
  bool floor_wins = false;
  if (e_floor != e_ceil) {
    const float diff = 4.0f * s_ar - s_ab;
    floor_wins = diff < 0.0f;
    if (fabsf(diff) < 0.0125f) floor_wins = floor_wins_f64(v, e_ceil, cc, cf);
  }
  int e = floor_wins ? e_floor : e_ceil;
  e = e < -127 ? -127 : (e > 127 ? 127 : e);
  if (e == e_ceil || e == e_floor) {
#pragma unroll
    for (int j = 0; j < 4; ++j) codes[j] = e == e_ceil ? cc[j] : cf[j];
  } else {  // amplitude clamped to the E8M0 range
    encode(e);
  }
  return (unsigned)(e + 127);
}

// A block of 32 values as the block functions take it: bf16 pairs in 16 words,
// fp32 values as they are.
template <typename T>
struct Block;
template <>
struct Block<uint16_t> {
  unsigned raw[16];
  __device__ __forceinline__ unsigned mxfp4(unsigned (&w)[4]) const { return mxfp4_block_bf16(raw, w); }
  __device__ __forceinline__ unsigned mxfp8(unsigned (&w)[8]) const {
    float v[32];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      v[2 * i] = as_float(raw[i] << 16);
      v[2 * i + 1] = as_float(raw[i] & 0xffff0000u);
    }
    return mxfp8_block(v, w);
  }
  // element j from a value in memory (j in order, even first)
  __device__ __forceinline__ void set(int j, uint16_t x) {
    if (j % 2 == 0) raw[j / 2] = x;
    else raw[j / 2] |= (unsigned)x << 16;
  }
};
template <>
struct Block<float> {
  float v[32];
  __device__ __forceinline__ unsigned mxfp4(unsigned (&w)[4]) const { return mxfp4_block_f32(v, w); }
  __device__ __forceinline__ unsigned mxfp8(unsigned (&w)[8]) const { return mxfp8_block(v, w); }
  __device__ __forceinline__ void set(int j, float x) { v[j] = x; }
};

// 32 contiguous values (16-byte aligned).
template <typename T>
__device__ __forceinline__ void load_row_block(const T* p, Block<T>& b) {
  constexpr int kLoads = 32 * sizeof(T) / 16;
  uint4 q[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) q[i] = reinterpret_cast<const uint4*>(p)[i];
  static_assert(sizeof(b) == sizeof(q), "a block is its values' bytes");
  __builtin_memcpy(&b, q, sizeof(q));
}

}  // namespace fp4attn
