// Activations, dropout and the element-wise end of a linear map (internal): what the products'
// epilogues and the dropout kernels do to four neighbouring channels of a row.
//
// Dropout: the mask is a function of (seed, offset, row, channel) and is computed wherever it is
// needed, so that the forward and the backward agree without storing it.  Four channels share one
// counter of Philox 4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", 2011): two 32 x 32 -> 64 bit products and two three-way xors a round, 40 instructions
// for four values, which stay under the memory time of a row that is read and written.
#pragma once

#include <cuda_bf16.h>
#include <cstdint>

#include "flashslice.h"

namespace fs {
namespace act {

struct Words {
  uint32_t w[4];
};

__device__ __forceinline__ Words philox(uint64_t counter, uint64_t offset, uint64_t seed) {
  uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; r++) {
    const uint64_t p = (uint64_t)0xD2511F53u * c0, q = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)q;
    c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

// What a call's dropout needs: a word below `threshold` drops its value, the others scale it.
struct Drop {
  const uint64_t* rng;  // {seed, offset} in device memory, so that a replayed graph draws anew; null: none
  uint32_t threshold;   // floor(p 2^32)
  float scale;          // 1 / (1 - p)
};
// (seed, offset), read once a thread.
struct DropKey {
  uint64_t seed, offset;
};

// A word that drops gives 0 whatever the value is (a NaN or an infinity included).
__device__ __forceinline__ void keep4(const Drop& d, const DropKey& k, uint64_t quad, float (&v)[4]) {
  const Words r = philox(quad, k.offset, k.seed);
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

template <bool kFast>
__device__ __forceinline__ void apply4(int act, float (&v)[4]) {
  if (act == FS_ACT_NONE) return;
#pragma unroll
  for (int i = 0; i < 4; i++)
    v[i] = act == FS_ACT_GELU ? gelu<kFast>(v[i]) : act == FS_ACT_SILU ? silu<kFast>(v[i]) : (v[i] < 0.f ? 0.f : v[i]);
}
// v *= act'(u)
template <bool kFast>
__device__ __forceinline__ void slope4(int act, const float (&u)[4], float (&v)[4]) {
  if (act == FS_ACT_NONE) return;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (act == FS_ACT_RELU) v[i] = u[i] > 0.f ? v[i] : u[i] <= 0.f ? 0.f : u[i];
    else v[i] *= act == FS_ACT_GELU ? gelu_slope<kFast>(u[i]) : silu_slope<kFast>(u[i]);
  }
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
