// Activations, dropout and the element-wise end of a linear map (internal): what the products'
// epilogues and the dropout kernels do to four neighbouring channels of a row.
//
// Dropout: the mask is a function of (seed, offset, row, channel) and is computed wherever it is
// needed, so that the forward and the backward agree without storing it.  Four channels share one
// counter of Philox 4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", 2011): two 32 x 32 -> 64 bit products and two three-way xors a round.
#pragma once

#include <cuda_bf16.h>
#include <cstdint>

#include "flashslice.h"

namespace fs {
namespace act {

struct Words {
  uint32_t w[4];
};

constexpr uint32_t kM0 = 0xD2511F53u, kM1 = 0xCD9E8D57u, kW0 = 0x9E3779B9u, kW1 = 0xBB67AE85u;

__device__ __forceinline__ void philox_round(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
  const uint64_t p = (uint64_t)kM0 * c[0], q = (uint64_t)kM1 * c[2];
  c[0] = (uint32_t)(q >> 32) ^ c[1] ^ k0;
  c[1] = (uint32_t)q;
  c[2] = (uint32_t)(p >> 32) ^ c[3] ^ k1;
  c[3] = (uint32_t)p;
}

// What a call's dropout needs: a word below `threshold` drops its value, the others scale it.
struct Drop {
  const uint64_t* rng;  // {seed, offset} in device memory, so that a replayed graph draws anew; null: none
  uint32_t threshold;   // floor(p 2^32)
  float scale;          // 1 / (1 - p)
};

// The generator's part that a call's counters share: the offset fills the upper half of each, and
// the quads' upper word is 0 up to 2^34 values.  Two of the first rounds' four products and most of
// their xors are then the same for all, and the words of the key schedule too.  Taken from one
// lane, so that the compiler keeps them in registers that a warp shares.
struct DropKey {
  uint32_t k0, k1, o0, o1;
  uint32_t b, c, d, e;  // rounds 1 to 3, for a quad's upper word of 0
};
__device__ __forceinline__ DropKey drop_key(const uint64_t* rng) {
  const uint64_t seed = rng[0], offset = rng[1];
  DropKey k;
  k.k0 = __shfl_sync(0xffffffffu, (uint32_t)seed, 0);
  k.k1 = __shfl_sync(0xffffffffu, (uint32_t)(seed >> 32), 0);
  k.o0 = __shfl_sync(0xffffffffu, (uint32_t)offset, 0);
  k.o1 = __shfl_sync(0xffffffffu, (uint32_t)(offset >> 32), 0);
  const uint64_t q1 = (uint64_t)kM1 * k.o0, p2 = (uint64_t)kM0 * ((uint32_t)(q1 >> 32) ^ k.k0);
  k.b = k.o1 ^ k.k1;
  k.c = (uint32_t)q1 ^ (k.k0 + kW0);
  k.d = (uint32_t)(p2 >> 32) ^ (k.k1 + kW1);
  k.e = (uint32_t)p2 ^ (k.k1 + 2 * kW1);
  return k;
}

__device__ __forceinline__ Words philox(uint64_t quad, const DropKey& k) {
  uint32_t c[4];
  if ((uint32_t)(quad >> 32) == 0) {
    const uint64_t p1 = (uint64_t)kM0 * (uint32_t)quad, q2 = (uint64_t)kM1 * ((uint32_t)(p1 >> 32) ^ k.b);
    const uint64_t p3 = (uint64_t)kM0 * ((uint32_t)(q2 >> 32) ^ k.c), q3 = (uint64_t)kM1 * ((uint32_t)p1 ^ k.d);
    c[0] = (uint32_t)(q3 >> 32) ^ (uint32_t)q2 ^ (k.k0 + 2 * kW0);
    c[1] = (uint32_t)q3;
    c[2] = (uint32_t)(p3 >> 32) ^ k.e;
    c[3] = (uint32_t)p3;
  } else {
    c[0] = (uint32_t)quad, c[1] = (uint32_t)(quad >> 32), c[2] = k.o0, c[3] = k.o1;
#pragma unroll
    for (uint32_t r = 0; r < 3; r++) philox_round(c, k.k0 + r * kW0, k.k1 + r * kW1);
  }
#pragma unroll
  for (uint32_t r = 3; r < 10; r++) philox_round(c, k.k0 + r * kW0, k.k1 + r * kW1);
  return {{c[0], c[1], c[2], c[3]}};
}

// A word that drops gives 0 whatever the value is (a NaN or an infinity included).
__device__ __forceinline__ void keep4(const Drop& d, const DropKey& k, uint64_t quad, float* v) {
  const Words r = philox(quad, k);
#pragma unroll
  for (int i = 0; i < 4; i++) v[i] = r.w[i] >= d.threshold ? v[i] * d.scale : 0.f;
}

// ---- activations ---------------------------------------------------------------------------
//
// kFast: for values that are rounded to bf16 afterwards (half a step is 2^-9 of the value).
//
// GELU is u Phi(u).  For a = |u|, Phi(-a) = e^(-a^2/2) Q(a) with Q(a) = erfcx(a / sqrt 2) / 2, a
// smooth function that falls from 1/2 to 0.077 over [0, 5]: a polynomial of degree 8 (weighted
// least squares, reweighted towards the minimax fit) is within 1.6e-4 of itself there, and past
// a = 5, where gelu(-a) is below 1.5e-6, Q stays at Q(5) and the Gaussian goes on falling.  One
// exponential and eight fused multiply-adds, and the exponential serves the derivative
// Phi(u) + u e^(-u^2/2) / sqrt(2 pi) too.
__device__ __forceinline__ float gauss_tail(float a, float& e) {
  constexpr float kHalfLog2e = 0.7213475204f;
  float q;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-kHalfLog2e * a * a));
  const float b = fminf(a, 5.f);
  q = 5.7904302e-06f;
  q = fmaf(q, b, -0.00014531538f);
  q = fmaf(q, b, 0.0015831057f);
  q = fmaf(q, b, -0.0099215629f);
  q = fmaf(q, b, 0.040258871f);
  q = fmaf(q, b, -0.11416839f);
  q = fmaf(q, b, 0.24129194f);
  q = fmaf(q, b, -0.39726451f);
  q = fmaf(q, b, 0.49994163f);
  return e * q;
}
constexpr float kInvSqrt2Pi = 0.3989422804014327f;
// Past this a the Gaussian is 0 in fp32; a product of it with an infinite u would be NaN.
constexpr float kGaussEnd = 15.f;
// Past this u the sigmoid is 1 (or 0) in fp32, and with u held there no infinity meets a 0.
constexpr float kSigmoidEnd = 110.f;

template <bool kFast>
__device__ __forceinline__ float gelu(float u) {
  if (u < -kGaussEnd) return 0.f;
  if (!kFast) return u * normcdff(u);
  float e;
  const float a = fabsf(u), t = a * gauss_tail(a, e);  // |u| Phi(-|u|)
  return a > kGaussEnd ? u : fmaxf(u, 0.f) - t;  // a NaN is one in t
}
template <bool kFast>
__device__ __forceinline__ float gelu_slope(float u) {
  if (fabsf(u) > kGaussEnd) return u > 0.f ? 1.f : 0.f;
  if (!kFast) return fmaf(u * kInvSqrt2Pi, expf(-0.5f * u * u), normcdff(u));
  float e;
  const float t = gauss_tail(fabsf(u), e);
  return fmaf(u * kInvSqrt2Pi, e, u > 0.f ? 1.f - t : t);
}

// By e^-|u|, which never overflows, so that the left tail keeps its values.
template <bool kFast>
__device__ __forceinline__ float sigmoid(float u) {
  const float e = kFast ? __expf(-fabsf(u)) : expf(-fabsf(u)), top = u < 0.f ? e : 1.f;
  return kFast ? __fdividef(top, 1.f + e) : top / (1.f + e);
}
template <bool kFast>
__device__ __forceinline__ float silu(float u) {
  const float b = u < -kSigmoidEnd ? -kSigmoidEnd : u;
  return b * sigmoid<kFast>(b);
}
template <bool kFast>
__device__ __forceinline__ float silu_slope(float u) {
  const float b = u > kSigmoidEnd ? kSigmoidEnd : u < -kSigmoidEnd ? -kSigmoidEnd : u;
  const float s = sigmoid<kFast>(b);
  return s * fmaf(b, 1.f - s, 1.f);
}

// v = act(v), n values that one loop walks (so that the chains of several are under way at once).
template <bool kFast, int ACT, int n>
__device__ __forceinline__ void apply(float (&v)[n]) {
#pragma unroll
  for (int i = 0; i < n; i++) {
    if (ACT == FS_ACT_GELU) v[i] = gelu<kFast>(v[i]);
    if (ACT == FS_ACT_SILU) v[i] = silu<kFast>(v[i]);
    if (ACT == FS_ACT_RELU) v[i] = v[i] < 0.f ? 0.f : v[i];
  }
}
// v = g act'(v)
template <bool kFast, int ACT, int n>
__device__ __forceinline__ void slope(float (&v)[n], const float* g) {
#pragma unroll
  for (int i = 0; i < n; i++) {
    if (ACT == FS_ACT_GELU) v[i] = gelu_slope<kFast>(v[i]) * g[i];
    if (ACT == FS_ACT_SILU) v[i] = silu_slope<kFast>(v[i]) * g[i];
    if (ACT == FS_ACT_RELU) v[i] = v[i] > 0.f ? g[i] : v[i] <= 0.f ? 0.f : v[i];
    if (ACT == FS_ACT_NONE) v[i] = g[i];
  }
}
template <bool kFast, int n>
__device__ __forceinline__ void apply(int act, float (&v)[n]) {
  if (act == FS_ACT_GELU) apply<kFast, FS_ACT_GELU>(v);
  else if (act == FS_ACT_SILU) apply<kFast, FS_ACT_SILU>(v);
  else if (act == FS_ACT_RELU) apply<kFast, FS_ACT_RELU>(v);
}
template <bool kFast, int n>
__device__ __forceinline__ void slope(int act, float (&v)[n], const float* g) {
  if (act == FS_ACT_GELU) slope<kFast, FS_ACT_GELU>(v, g);
  else if (act == FS_ACT_SILU) slope<kFast, FS_ACT_SILU>(v, g);
  else if (act == FS_ACT_RELU) slope<kFast, FS_ACT_RELU>(v, g);
  else slope<kFast, FS_ACT_NONE>(v, g);
}

// ---- four neighbouring channels in memory --------------------------------------------------
//
// n of them are there (1..4); whole: all four, at an address that a vector access may take.
template <typename T>
__device__ __forceinline__ void load4(const T* p, int n, bool whole, float (&v)[4]);
template <>
__device__ __forceinline__ void load4<float>(const float* p, int n, bool whole, float (&v)[4]) {
  if (whole) {
    const float4 x = *reinterpret_cast<const float4*>(p);
    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = i < n ? p[i] : 0.f;
  }
}
template <>
__device__ __forceinline__ void load4<__nv_bfloat16>(const __nv_bfloat16* p, int n, bool whole, float (&v)[4]) {
  if (whole) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(x.x << 16), v[1] = __uint_as_float(x.x & 0xFFFF0000u);
    v[2] = __uint_as_float(x.y << 16), v[3] = __uint_as_float(x.y & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = i < n ? __bfloat162float(p[i]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, int n, bool whole, const float (&v)[4]);
template <>
__device__ __forceinline__ void store4<float>(float* p, int n, bool whole, const float (&v)[4]) {
  if (whole) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (i < n) p[i] = v[i];
  }
}
template <>
__device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16* p, int n, bool whole, const float (&v)[4]) {
  if (whole) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (i < n) p[i] = __float2bfloat16_rn(v[i]);
  }
}

}  // namespace act
}  // namespace fs
