// Rotary positions.
//
// Pair j of a head's first r channels turns by t = position * inv_freq[j]:
//   y_a = m (x_a cos t - x_b sin t),  y_b = m (x_a sin t + x_b cos t),
// (a, b) = (j, j + r / 2) or, interleaved, (2 j, 2 j + 1); channels past r pass through.
// The inverse turns by -t: m R^T, which is the gradient of the rotation.
//
// Angles of far positions need more than 24 bits (position 10^6 at one radian a step is
// off by 0.06 in fp32), so t and its reduction to a quarter turn are fp64; what is
// left, |t| <= pi / 4, is exact to 2^-26 quarter turns in fp32.  A workgroup takes 4 or 16 tokens
// and forms each token's angles once, in LDS, for all its heads.
//
// What bounds it is memory: x in, y out.  A thread turns two runs of 16 bytes that lie half the turned (or
// passed-on) channels apart, the two halves' pairs or, interleaved, two lots of whole pairs, so that
// neighbouring lanes load neighbouring 16 bytes either way (runs of 32 bytes in fp32, and with both runs of
// interleaved pairs side by side: 61 us where it is now 48).  Measured, 32 heads of 16384 tokens, d = 128, bf16
// (268 MB): 51 us, 5.3 TB/s, interleaved the same; fp32, 2 x 16 heads of 8192 tokens (268 MB): 48 us, 5.6 TB/s;
// 16 tokens of 40 heads: 3.0 us, a launch.
#include <cmath>

#include "gfx950.hpp"
#include "serving.hpp"

namespace fp4attn {

namespace {

constexpr int kThreads = 256;
template <typename T>
constexpr int kUnit = 32 / sizeof(T);  // elements that a thread turns at once, in two runs of 16 bytes

template <typename T>
struct Unit;
template <>
struct Unit<uint16_t> {
  uint4 a, b;
  __device__ __forceinline__ void load(const uint16_t* pa, const uint16_t* pb) {
    a = *reinterpret_cast<const uint4*>(pa);
    b = *reinterpret_cast<const uint4*>(pb);
  }
  __device__ __forceinline__ void store(uint16_t* pa, uint16_t* pb) const {
    *reinterpret_cast<uint4*>(pa) = a;
    *reinterpret_cast<uint4*>(pb) = b;
  }
  __device__ __forceinline__ void get(float (&v)[16]) const {
    const unsigned w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[2 * i] = as_float(w[i] << 16);
      v[2 * i + 1] = as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&v)[16]) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    unsigned w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __builtin_bit_cast(unsigned, bf2{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]});
    a = uint4{w[0], w[1], w[2], w[3]};
    b = uint4{w[4], w[5], w[6], w[7]};
  }
};
template <>
struct Unit<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* pa, const float* pb) {
    a = *reinterpret_cast<const float4*>(pa);
    b = *reinterpret_cast<const float4*>(pb);
  }
  __device__ __forceinline__ void store(float* pa, float* pb) const {
    *reinterpret_cast<float4*>(pa) = a;
    *reinterpret_cast<float4*>(pb) = b;
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = w[i];
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    a = float4{v[0], v[1], v[2], v[3]};
    b = float4{v[4], v[5], v[6], v[7]};
  }
};

// grid: (token groups, head groups of `heads`, B)
template <typename T, bool INTERLEAVED, int TOKENS>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a, int heads) {
  constexpr int kItems = 4;  // units of a thread in flight
  constexpr int kPairs = kUnit<T> / 2;
  __shared__ __attribute__((aligned(16))) float table[2][TOKENS][kRotaryMaxDim / 2];
  asm volatile("" ::"s"(heads), "s"(a.N), "s"(a.x));  // of each line of the arguments: their misses overlap
  const int tid = threadIdx.x, half = a.r / 2;
  const int64_t n0 = (int64_t)blockIdx.x * TOKENS;
  const int64_t b = blockIdx.z;
  const int tokens = a.N - n0 < TOKENS ? (int)(a.N - n0) : TOKENS;
  for (int i = tid; i < tokens * half; i += kThreads) {
    const int tok = i / half, j = i - tok * half;
    const double t = (double)a.positions[b * a.pos_stride + n0 + tok] * a.inv_freq[j];
    const double quarters = t * 0.63661977236758134308;  // 2 / pi
    const double whole = rint(quarters);
    float s, c;
    sincospif(0.5f * (float)(quarters - whole), &s, &c);
    const int k = (int)(whole - 4.0 * floor(0.25 * whole));  // quarter turns, 0 .. 3
    const float cc = k & 1 ? s : c, ss = k & 1 ? c : s;
    table[0][tok][j] = a.magnitude * (k == 1 || k == 2 ? -cc : cc);
    table[1][tok][j] = a.magnitude * ((k >= 2) != (a.inverse != 0) ? -ss : ss);
  }
  __syncthreads();
  const int h0 = blockIdx.y * heads;
  const int nh = a.H - h0 < heads ? (int)(a.H - h0) : heads;
  const int units = a.d / kUnit<T>, turned = a.r / kUnit<T>;
  const int count = units * nh * TOKENS;
  const T* x = static_cast<const T*>(a.x) + b * a.xb + n0 * a.xn + h0 * a.xh;
  T* out = static_cast<T*>(a.out) + b * a.ob + n0 * a.on + h0 * a.oh;
  const bool in_place = a.x == a.out;
  for (int first = tid; first < count; first += kThreads * kItems) {
    Unit<T> v[kItems];
    int64_t at[kItems];  // of the unit's first run in `out`
    int tok[kItems], u[kItems], gap[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int idx = first + i * kThreads, row = idx / units, h = row / TOKENS;
      u[i] = idx - row * units;
      tok[i] = row % TOKENS;
      const bool turn = u[i] < turned;
      if (idx >= count || tok[i] >= tokens || (in_place && !turn)) tok[i] = -1;
      const int c = turn ? kPairs * u[i] : a.r + kPairs * (u[i] - turned);
      gap[i] = turn ? half : (a.d - a.r) / 2;
      at[i] = h * a.oh + tok[i] * a.on + c;
      if (tok[i] >= 0) {
        const T* p = x + h * a.xh + tok[i] * a.xn + c;
        v[i].load(p, p + gap[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      if (tok[i] < 0) continue;
      if (u[i] < turned) {
        float f[kUnit<T>], y[kUnit<T>], c[kPairs], s[kPairs];
        v[i].get(f);
        // angles of the unit's pairs, or interleaved of the pairs of its first and of its second run
        const int j0 = INTERLEAVED ? kPairs / 2 * u[i] : kPairs * u[i], j1 = INTERLEAVED ? j0 + half / 2 : j0 + kPairs / 2;
        const float *cp = table[0][tok[i]], *sp = table[1][tok[i]];
        constexpr size_t kRun = kPairs / 2 * sizeof(float);
        __builtin_memcpy(c, __builtin_assume_aligned(cp + j0, kRun), kRun);
        __builtin_memcpy(c + kPairs / 2, __builtin_assume_aligned(cp + j1, kRun), kRun);
        __builtin_memcpy(s, __builtin_assume_aligned(sp + j0, kRun), kRun);
        __builtin_memcpy(s + kPairs / 2, __builtin_assume_aligned(sp + j1, kRun), kRun);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
          const int p = INTERLEAVED ? 2 * j : j, q = INTERLEAVED ? 2 * j + 1 : j + kPairs;
          y[p] = fmaf(f[p], c[j], -(f[q] * s[j]));
          y[q] = fmaf(f[p], s[j], f[q] * c[j]);
        }
        v[i].set(y);
      }
      v[i].store(out + at[i], out + at[i] + gap[i]);
    }
  }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  const int units = a.d / (a.bf16 ? kUnit<uint16_t> : kUnit<float>);
  int tokens;
  int64_t groups, heads;
  auto plan = [&](int t, int per_thread) {  // heads of a workgroup: `per_thread` units for each thread
    tokens = t;
    groups = (a.N + t - 1) / t;
    heads = (int64_t)kThreads * per_thread / (units * t);
    heads = heads < 1 ? 1 : (heads > a.H ? a.H : heads);
    return groups * a.B * ((a.H + heads - 1) / heads);
  };
  // Sixteen tokens make longer runs where tokens lie side by side, but fewer workgroups: bf16, d = 128,
  // 32 heads, 16384 tokens 54.3 -> 49.4 us (4096 workgroups), 8 heads 15.3 -> 13.8 (1024), 32 heads of 2048
  // tokens 8.9 -> 9.8 (512); with heads side by side 16384 tokens 50.7 -> 53.8.  One unit a thread where
  // four leave few workgroups: one token of 32 heads 4.0 -> 3.1 us.
  if (!(a.xn < a.xh && plan(16, 4) >= 1024) && plan(4, 4) < 512) plan(4, 1);
  const dim3 grid((unsigned)groups, (unsigned)((a.H + heads - 1) / heads), (unsigned)a.B);
  auto launch = [&](auto T_, auto INTERLEAVED_) {
    using T = decltype(T_);
    constexpr bool kInterleaved = decltype(INTERLEAVED_)::value;
    if (tokens == 16) rotary_kernel<T, kInterleaved, 16><<<grid, kThreads, 0, stream>>>(a, (int)heads);
    else rotary_kernel<T, kInterleaved, 4><<<grid, kThreads, 0, stream>>>(a, (int)heads);
  };
  if (a.bf16 && a.interleaved) launch(uint16_t{}, std::true_type{});
  else if (a.bf16) launch(uint16_t{}, std::false_type{});
  else if (a.interleaved) launch(float{}, std::true_type{});
  else launch(float{}, std::false_type{});
  return hipGetLastError();
}

}  // namespace fp4attn
