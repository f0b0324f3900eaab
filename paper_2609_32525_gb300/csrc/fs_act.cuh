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
#include "fs_tc_ptx.cuh"

namespace fs {
namespace act {

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

// n neighbouring quads, round by round for all of them: the chains of n counters are under way at
// once and share the key schedule's additions.  A quad of 32 bits has an upper word of 0.
template <int n, typename Q>
__device__ __forceinline__ void philox(Q quad, const DropKey& k, uint32_t (&c)[n][4]) {
  constexpr bool kLow = sizeof(Q) == 4;
  uint32_t k0 = k.k0, k1 = k.k1;
  if constexpr (kLow) {
    k0 += 2 * kW0;
#pragma unroll
    for (int i = 0; i < n; i++) {
      const uint64_t p1 = (uint64_t)kM0 * (quad + i), q2 = (uint64_t)kM1 * ((uint32_t)(p1 >> 32) ^ k.b);
      const uint64_t p3 = (uint64_t)kM0 * ((uint32_t)(q2 >> 32) ^ k.c), q3 = (uint64_t)kM1 * ((uint32_t)p1 ^ k.d);
      c[i][0] = (uint32_t)(q3 >> 32) ^ (uint32_t)q2 ^ k0;
      c[i][1] = (uint32_t)q3;
      c[i][2] = (uint32_t)(p3 >> 32) ^ k.e;
      c[i][3] = (uint32_t)p3;
    }
    k0 += kW0;
    k1 += 3 * kW1;
  } else {
#pragma unroll
    for (int i = 0; i < n; i++)
      c[i][0] = (uint32_t)(quad + i), c[i][1] = (uint32_t)((uint64_t)(quad + i) >> 32), c[i][2] = k.o0, c[i][3] = k.o1;
  }
#pragma unroll
  for (int r = kLow ? 3 : 0; r < 10; r++) {
#pragma unroll
    for (int i = 0; i < n; i++) philox_round(c[i], k0, k1);
    k0 += kW0;
    k1 += kW1;
  }
}

// r += drop(v), n values from a quad on (a 32-bit one where all of them have an upper word of 0).  A word that
// drops leaves r as it is, whatever the value is (a NaN or an infinity included); else product and sum are one
// instruction under the comparison's predicate.
template <int n, typename Q>
__device__ __forceinline__ void keep_by(const Drop& d, const DropKey& k, Q quad, const float* v, float* r) {
  uint32_t w[n / 4][4];
  philox<n / 4>(quad, k, w);
#pragma unroll
  for (int i = 0; i < n; i++)
    asm("{\n .reg .pred p;\n setp.ge.u32 p, %1, %2;\n @p fma.rn.f32 %0, %3, %4, %0;\n}"
        : "+f"(r[i])
        : "r"(w[i / 4][i % 4]), "r"(d.threshold), "f"(v[i]), "f"(d.scale));
}
template <int n>
__device__ __forceinline__ void keep(const Drop& d, const DropKey& k, uint64_t quad, const float* v, float* r) {
  if (((quad + n / 4 - 1) >> 32) == 0) keep_by<n>(d, k, (uint32_t)quad, v, r);
  else keep_by<n>(d, k, quad, v, r);
}

// ---- activations ---------------------------------------------------------------------------
//
// kFast: for values that are rounded to bf16 afterwards, by half a step of 2^-9 to 2^-8 of the value.  GELU and SILU are
// good to 2^-16 of themselves over the whole range, their derivatives to 2^-19.
//
// All of them two values at a time (f32x2 instructions).
//
// GELU is u Phi(u).  For a = |u|, Phi(-a) = e^(-a^2/2) Q(a) with Q(a) = erfcx(a / sqrt 2) / 2, a smooth function
// that falls slowly; the exponential serves the derivative Phi(u) + u e^(-u^2/2) / sqrt(2 pi) too.
//   kFast: Q(a) (a + k) as a polynomial of degree 6 in (a - k) / (a + k) on [0, 15], within 1.4e-6 of itself.  (A
//   polynomial of degree 8 in a on [0, 5], Q held past 5, has as many instructions but the reciprocal; it was off by
//   1.6e-4, and past 5 by up to the value itself.)
//   else: Q(a) (1 + 2 a) as a polynomial of degree 9 in (a - k) / (a + k) on [0, 15], within 2.7e-8 of itself (the
//   form of Shepherd and Laframboise, "Chebyshev approximation of (1 + 2x) exp(x^2) erfc x in 0 <= x < inf", 1981).
//   Quotients get one Newton step, and the exponent's rounding is put back after the exponential.
// Both polynomials are weighted least-squares fits, reweighted towards the minimax one.
constexpr float kInvSqrt2Pi = 0.3989422804014327f;
// Past this a the Gaussian is 0 in fp32; a product of it with an infinite u would be NaN.
constexpr float kGaussEnd = 15.f;
// Past this u the sigmoid is 1 (or 0) in fp32, and with u held there no infinity meets a 0.
constexpr float kSigmoidEnd = 110.f;
constexpr float kLog2eHi = 1.442695041f, kLog2eLo = 1.925963033e-08f, kLn2 = 0.6931471806f;

__device__ __forceinline__ uint64_t twice(float x) { return tc::pack2(__float_as_uint(x), __float_as_uint(x)); }
__device__ __forceinline__ uint64_t pair(float x, float y) { return tc::pack2(__float_as_uint(x), __float_as_uint(y)); }
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^x, with subnormal results.
__device__ __forceinline__ float ex2_full(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The larger (smaller) of two; NaN where one is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float d;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

template <int n>
__device__ __forceinline__ uint64_t poly2(const float (&c)[n], uint64_t x) {
  uint64_t q = twice(c[n - 1]);
#pragma unroll
  for (int i = n - 2; i >= 0; i--) q = tc::fma2(q, x, twice(c[i]));
  return q;
}
// Phi(-a) for 0 <= a <= kGaussEnd; e: e^(-a^2/2).  kTail: small values are good to their own size; without it (a
// derivative adds them to others) the Newton steps and the exponent's remainder are left out, and fp32's absolute
// error is 2^-21 at most: quotients and polynomial 8 u of 1/2, and a^2/2 e^(-a^2/2) u from the exponent.
template <bool kFast, bool kTail>
__device__ __forceinline__ uint64_t gauss_tail2(float a0, float a1, uint64_t& e) {
  const uint64_t a = pair(a0, a1);
  if constexpr (kFast) {
    constexpr float k = 5.f;
    constexpr float c[7] = {0.769192398f, -0.665391624f, 0.495357752f, -0.313332379f, 0.164524734f, -0.070451133f, 0.0217513554f};
    const uint64_t up = tc::add2(a, twice(k)), r = pair(rcp(tc::lo_f(up)), rcp(tc::hi_f(up)));
    const uint64_t y = tc::mul2(tc::mul2(a, twice(-0.5f * kLog2eHi)), a);
    e = pair(tc::ex2(tc::lo_f(y)), tc::ex2(tc::hi_f(y)));
    return tc::mul2(tc::mul2(e, r), poly2(c, tc::fma2(r, twice(-2.f * k), twice(1.f))));
  } else {
    constexpr float k = 2.8125f;
    constexpr float c[10] = {0.849999964f,     0.0238276552f,  -0.168504149f,   0.131846741f,    -0.0378766023f,
                             -0.00768018235f, 0.00614848454f, 0.00123171532f, -0.000851653749f, -0.000309873198f};
    const uint64_t up = tc::add2(a, twice(k)), down = tc::add2(a, twice(-k)), den = tc::fma2(a, twice(2.f), twice(1.f));
    const uint64_t both = tc::mul2(up, den), minus = twice(-1.f);
    const uint64_t r = pair(rcp(tc::lo_f(both)), rcp(tc::hi_f(both)));
    const uint64_t up_r = tc::mul2(r, den);
    uint64_t t = tc::mul2(down, up_r), s = tc::mul2(r, up);
    if (kTail) {
      t = tc::fma2(tc::fma2(tc::mul2(t, minus), up, down), up_r, t);
      s = tc::fma2(s, tc::fma2(tc::mul2(s, minus), den, twice(1.f)), s);
    }
    // a^2 = h + l; the exponent y = -h log2(e) / 2 and what it leaves out
    const uint64_t h = tc::mul2(a, a), y = tc::mul2(h, twice(-0.5f * kLog2eHi));
    e = pair(tc::ex2(tc::lo_f(y)), tc::ex2(tc::hi_f(y)));
    if (kTail) {
      const uint64_t l = tc::fma2(a, a, tc::mul2(h, minus));
      uint64_t left = tc::fma2(h, twice(-0.5f * kLog2eHi), tc::mul2(y, minus));
      left = tc::fma2(h, twice(-0.5f * kLog2eLo), left);
      left = tc::fma2(l, twice(-0.5f * kLog2eHi), left);
      e = tc::fma2(tc::mul2(e, twice(kLn2)), left, e);
    }
    return tc::mul2(tc::mul2(e, s), poly2(c, t));
  }
}
// max(u, 0) - a Phi(-a)
template <bool kFast>
__device__ __forceinline__ void gelu2(float& u0, float& u1) {
  const float a0 = fminf(fabsf(u0), kGaussEnd), a1 = fminf(fabsf(u1), kGaussEnd);
  uint64_t e;
  const uint64_t t = gauss_tail2<kFast, true>(a0, a1, e);
  const uint64_t y = tc::fma2(t, pair(-a0, -a1), pair(max_nan(u0, 0.f), max_nan(u1, 0.f)));
  u0 = tc::lo_f(y), u1 = tc::hi_f(y);
}
template <bool kFast>
__device__ __forceinline__ void gelu_slope2(float& u0, float& u1) {
  const float v0 = max_nan(min_nan(u0, kGaussEnd), -kGaussEnd), v1 = max_nan(min_nan(u1, kGaussEnd), -kGaussEnd);
  uint64_t e;
  const uint64_t t = gauss_tail2<kFast, false>(fabsf(v0), fabsf(v1), e);
  const float t0 = tc::lo_f(t), t1 = tc::hi_f(t);
  const uint64_t cdf = pair(v0 > 0.f ? 1.f - t0 : t0, v1 > 0.f ? 1.f - t1 : t1);
  const uint64_t y = tc::fma2(tc::mul2(pair(v0, v1), twice(kInvSqrt2Pi)), e, cdf);
  u0 = tc::lo_f(y), u1 = tc::hi_f(y);
}

// SILU by e^-|u|, which never overflows, so that the left tail keeps its values; |u| <= kSigmoidEnd.
template <bool kFast>
__device__ __forceinline__ uint64_t sigmoid2(float u0, float u1) {
  const uint64_t a = pair(fabsf(u0), fabsf(u1)), y = tc::mul2(a, twice(-kLog2eHi));
  uint64_t e;
  if constexpr (kFast) {
    e = pair(tc::ex2(tc::lo_f(y)), tc::ex2(tc::hi_f(y)));
  } else {
    uint64_t left = tc::fma2(a, twice(-kLog2eHi), tc::mul2(y, twice(-1.f)));
    left = tc::fma2(a, twice(-kLog2eLo), left);
    e = pair(ex2_full(tc::lo_f(y)), ex2_full(tc::hi_f(y)));
    e = tc::fma2(tc::mul2(e, twice(kLn2)), left, e);
  }
  const float e0 = tc::lo_f(e), e1 = tc::hi_f(e);
  return tc::mul2(pair(u0 < 0.f ? e0 : 1.f, u1 < 0.f ? e1 : 1.f), pair(rcp(1.f + e0), rcp(1.f + e1)));
}
template <bool kFast>
__device__ __forceinline__ void silu2(float& u0, float& u1) {
  const float b0 = max_nan(u0, -kSigmoidEnd), b1 = max_nan(u1, -kSigmoidEnd);
  // (a large u's own sigmoid is 1)
  const uint64_t y = tc::mul2(pair(b0, b1), sigmoid2<kFast>(min_nan(b0, kSigmoidEnd), min_nan(b1, kSigmoidEnd)));
  u0 = tc::lo_f(y), u1 = tc::hi_f(y);
}
template <bool kFast>
__device__ __forceinline__ void silu_slope2(float& u0, float& u1) {
  const float b0 = max_nan(min_nan(u0, kSigmoidEnd), -kSigmoidEnd), b1 = max_nan(min_nan(u1, kSigmoidEnd), -kSigmoidEnd);
  const uint64_t s = sigmoid2<kFast>(b0, b1), rest = tc::fma2(s, twice(-1.f), twice(1.f));
  const uint64_t y = tc::mul2(s, tc::fma2(pair(b0, b1), rest, twice(1.f)));
  u0 = tc::lo_f(y), u1 = tc::hi_f(y);
}

// v = act(v), n values (an even number) that one loop walks, so that the chains of several are under way at once.
template <bool kFast, int ACT, int n>
__device__ __forceinline__ void apply(float (&v)[n]) {
#pragma unroll
  for (int i = 0; i < n; i++) {
    if (ACT == FS_ACT_GELU && i % 2 == 0) gelu2<kFast>(v[i], v[i + 1]);
    if (ACT == FS_ACT_SILU && i % 2 == 0) silu2<kFast>(v[i], v[i + 1]);
    if (ACT == FS_ACT_RELU) v[i] = max_nan(v[i], 0.f);
  }
}
// v = g act'(v)
template <bool kFast, int ACT, int n>
__device__ __forceinline__ void slope(float (&v)[n], const float* g) {
#pragma unroll
  for (int i = 0; i < n; i++) {
    if (ACT == FS_ACT_GELU && i % 2 == 0) gelu_slope2<kFast>(v[i], v[i + 1]);
    if (ACT == FS_ACT_SILU && i % 2 == 0) silu_slope2<kFast>(v[i], v[i + 1]);
    if (ACT == FS_ACT_RELU) v[i] = v[i] > 0.f ? g[i] : v[i] <= 0.f ? 0.f : v[i];
    if (ACT == FS_ACT_NONE) v[i] = g[i];
  }
  if (ACT == FS_ACT_GELU || ACT == FS_ACT_SILU)
#pragma unroll
    for (int i = 0; i < n; i++) v[i] *= g[i];
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
