// Layer norm forward and backward, and the 8-bit checkpoint, over rows of C channels.
//
//   forward    v = x + res;  mean, var over the row;  y = (v - mean) rstd gamma + beta,
//              rstd = 1 / sqrt(var + eps)
//   backward   xh = (v - mean) rstd, g = dy gamma:
//              dv = rstd (g - avg(g) - xh avg(g xh)) + dres;  dgamma = sum dy xh, dbeta = sum dy
//   checkpoint blocks of 32 channels: v ~ q 2^s, q = v 2^-s rounded, s the smallest >= -126 at
//              which the block's largest magnitude rounds to at most 127; the byte s + 127 is
//              kept, 255 for a block with NaN or infinity.  2^s scales exactly, so that the only
//              rounding is q's: half a step, at most 1/127.5 = 2^-6.994 of the block's largest
//              magnitude (which is 63.75 steps at least: 127.5 of the next smaller ones round up).
//
// Every pass reads each input once and writes each output once: a row lies in the registers of
// its threads between its sums and its outputs, so memory bandwidth bounds all of them.  Sums
// are fp32, the variance from centred values (a second sweep over registers), which stays
// exact where the mean is far larger than the deviation.
//
// The parameter gradients sum over rows.  A thread owns the same channels of every row it
// meets and keeps their sums in registers; a block adds its row groups in order and writes one
// row of partial sums, and a second kernel adds the blocks' rows in order: no atomics, the same
// bits in every run.
#pragma once

#include "fs_internal.h"
#include "fs_launch.h"
#include "fs_rows.h"
#include "fs_tc_ptx.cuh"

#include <algorithm>
#include <cuda_bf16.h>

namespace fs {
namespace rows {

template <int N>
struct Raw;
template <> struct Raw<1> { using type = uint8_t; };
template <> struct Raw<2> { using type = uint16_t; };
template <> struct Raw<4> { using type = uint32_t; };
template <> struct Raw<8> { using type = uint2; };
template <> struct Raw<16> { using type = uint4; };
template <typename T, int VE>
using RawV = typename Raw<sizeof(T) * VE>::type;

template <typename R>
__device__ __forceinline__ R raw_zero() {
  R r;
  memset(&r, 0, sizeof(R));
  return r;
}

template <typename T, int VE>
__device__ __forceinline__ void to_float(const RawV<T, VE>& r, float (&f)[VE]) {
  if constexpr (sizeof(T) == 4) {
    memcpy(f, &r, sizeof(r));
  } else {
    uint16_t u[VE];
    memcpy(u, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < VE; i++) f[i] = __uint_as_float((uint32_t)u[i] << 16);
  }
}
template <typename T, int VE>
__device__ __forceinline__ RawV<T, VE> from_float(const float (&f)[VE]) {
  RawV<T, VE> r;
  if constexpr (sizeof(T) == 4) {
    memcpy(&r, f, sizeof(r));
  } else if constexpr (VE == 1) {
    const __nv_bfloat16 h = __float2bfloat16_rn(f[0]);
    memcpy(&r, &h, sizeof(r));
  } else {
    __nv_bfloat162 h[VE / 2];
#pragma unroll
    for (int i = 0; i < VE / 2; i++) h[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    memcpy(&r, h, sizeof(r));
  }
  return r;
}

template <int TPR>
__host__ __device__ constexpr int block_threads() { return TPR <= 32 ? 256 : TPR; }

// Rows whose loads a thread issues before it uses the first.
template <int K>
__host__ __device__ constexpr int rows_ahead() { return K == 1 ? 2 : 1; }
// Blocks of the backward on an SM: by its registers (16 channels a lane: 300,000 x 384 bf16 from the
// checkpoint 389 us with one block, 240 with two, 283 with three).
template <int TPR, int N>
__host__ __device__ constexpr int bwd_blocks_per_sm() { return TPR > 32 ? 1 : N <= 8 ? 3 : 2; }

// The sum over a row's TPR threads, in every one of them, in a fixed order.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
#pragma unroll
  for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if constexpr (TPR > 32) {
    constexpr int W = TPR / 32;
    __syncthreads();  // the sums before this one have been read
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < W; i++) v += red[i];
  }
  return v;
}

// The byte s + 127 of a block's scale 2^s, from the bits of its largest magnitude (NaN and
// infinity have the largest bits).
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255u;
  // 2^E <= top < 2^(E+1): s = E - 6 puts top in [64, 128), and 127.5 upwards rounds past 127
  const int s = (int)(top >> 23) - 127 - 6;
  const int s1 = s + ((top & 0x7fffffu) >= 0x7f0000u ? 1 : 0);
  return (uint32_t)((s1 < -126 ? -126 : s1) + 127);
}
__device__ __forceinline__ float scale_of(uint32_t byte) {  // 2^s; NaN for 255
  return __uint_as_float(byte == 255u ? 0x7fc00000u : byte << 23);
}
__device__ __forceinline__ float inverse_scale_of(uint32_t byte) {  // 2^-s; 0 for 255
  return __uint_as_float(byte == 255u ? 0u : (254u - byte) << 23);
}

// Two fp32 values in one instruction: these passes are close to the issue rate.
struct F2 {
  unsigned long long v;
};
__device__ __forceinline__ F2 pair(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(F2 x, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v));
}
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ float total(F2 x) {
  float a, b;
  split(x, a, b);
  return a + b;
}

// A thread's N channels of a row as pairs; an odd last one is paired with 0.
template <int N>
struct Vals {
  static constexpr int P = (N + 1) / 2;
  F2 p[P];
};
template <typename T, int VE, int K>
__device__ __forceinline__ Vals<K * VE> vals_of(const RawV<T, VE> (&r)[K]) {
  Vals<K * VE> o;
  float f[K * VE + 1];
  f[K * VE] = 0.f;
#pragma unroll
  for (int k = 0; k < K; k++) to_float<T, VE>(r[k], *reinterpret_cast<float(*)[VE]>(f + k * VE));
#pragma unroll
  for (int i = 0; i < o.P; i++) o.p[i] = pair(f[2 * i], f[2 * i + 1]);
  return o;
}
template <int N>
__device__ __forceinline__ void floats_of(const Vals<N>& v, float (&f)[2 * Vals<N>::P]) {
#pragma unroll
  for (int i = 0; i < v.P; i++) split(v.p[i], f[2 * i], f[2 * i + 1]);
}

// |a|, |b|, |c|: the largest; NaN if one is.
__device__ __forceinline__ float max_abs(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Quantises a vector of a row; the 32 / VE neighbouring lanes that share a block agree on its
// scale.  All lanes of the warp call it.  Adding 1.5 2^23 rounds to whole numbers, ties to
// even, and leaves them in the low byte.
template <int VE>
__device__ __forceinline__ void quantise(const float* f, uint32_t& byte, RawV<uint8_t, VE>& q) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < VE; i += 2) m = max_abs(m, f[i], VE > 1 ? f[i + 1] : 0.f);
#pragma unroll
  for (int o = kCkptBlock / VE / 2; o > 0; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, o), 0.f);
  byte = scale_byte(__float_as_uint(m));
  const float inv = inverse_scale_of(byte);
  uint32_t u[VE];
#pragma unroll
  for (int i = 0; i < VE; i++)
    u[i] = byte == 255u ? 0u : __float_as_uint(fmaf(f[i], inv, 12582912.f));
  if constexpr (VE >= 4) {
    uint32_t w[VE / 4];
#pragma unroll
    for (int i = 0; i < VE / 4; i++)
      w[i] = __byte_perm(__byte_perm(u[4 * i], u[4 * i + 1], 0x0040), __byte_perm(u[4 * i + 2], u[4 * i + 3], 0x0040),
                         0x5410);
    memcpy(&q, w, sizeof(q));
  } else {
    uint8_t b[VE];
#pragma unroll
    for (int i = 0; i < VE; i++) b[i] = (uint8_t)u[i];
    memcpy(&q, b, sizeof(q));
  }
}
// A byte with its sign bit flipped is q + 128; as the low byte of 2^23 it is exact in fp32.
template <int VE>
__device__ __forceinline__ void restore(const RawV<uint8_t, VE>& q, uint32_t byte, float (&f)[VE]) {
  const float size = scale_of(byte);
  if constexpr (VE >= 4) {
    uint32_t w[VE / 4];
    memcpy(w, &q, sizeof(q));
    const F2 minus = pair(-8388736.f, -8388736.f), both = pair(size, size);
#pragma unroll
    for (int i = 0; i < VE; i += 2) {
      const uint32_t u = w[i / 4] ^ 0x80808080u;
      const F2 x = pair(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 + i % 4)),
                        __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7441 + i % 4)));
      split((x + minus) * both, f[i], f[i + 1]);
    }
  } else {
    int8_t b[VE];
    memcpy(b, &q, sizeof(q));
#pragma unroll
    for (int i = 0; i < VE; i++) f[i] = (float)b[i] * size;
  }
}

// ---- rows on their way -------------------------------------------------------------------------
//
// What bounds these passes is memory bandwidth, and what keeps them from it is latency: a row's
// two sums depend on its loads, one on the other.  So every thread fetches the vectors of its
// next rows with cp.async into slots of shared memory that it alone reads: several rows are on
// their way at no cost in registers, and no barrier is needed.  (With the next rows in
// registers instead, 118 of them, 1,048,576 rows of 256 bf16 channels took 315 us in the plain
// forward, against 270 us with one row at a time.)

// N bytes from global to this thread's slot, zeros where !ok (src is then any valid address).
template <int N>
__device__ __forceinline__ void fetch(void* dst, const void* src, bool ok) {
  if constexpr (N >= 4) {
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    const int n = ok ? N : 0;
    if constexpr (N == 16)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(n) : "memory");
    else
      asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(d), "l"(src), "n"(N), "r"(n) : "memory");
  } else {  // below cp.async's smallest size
    using R = typename Raw<N>::type;
    *static_cast<R*>(dst) = ok ? *static_cast<const R*>(src) : R(0);
  }
}
__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void fetch_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A thread's slots for one stage: element (k, thread) of a [K][THREADS] array of R.
template <typename R, int THREADS>
__device__ __forceinline__ R* slot(char* base, int k) {
  return reinterpret_cast<R*>(base) + k * THREADS + threadIdx.x;
}
// Stages: up to 64 KB of slots per block (8 stages of bf16 rows of 256 channels: plain forward
// 181 us, 4 stages 189 us), two at least.
template <int BYTES, int THREADS>
__host__ __device__ constexpr int stages() {
  constexpr int fit = 65536 / (BYTES * THREADS);
  return fit >= 8 ? 8 : fit <= 2 ? 2 : fit;
}

// gamma or beta of a thread's channels; `none` where it is null and past C.
template <int N, int VE, int TPR>
__device__ __forceinline__ Vals<N> channels_of(const float* p, int C, int t, float none) {
  Vals<N> o;
  float f[N + 1];
  f[N] = none;
#pragma unroll
  for (int i = 0; i < N; i++) {
    const int c = (i / VE * TPR + t) * VE + i % VE;
    f[i] = p && c < C ? p[c] : none;
  }
#pragma unroll
  for (int i = 0; i < o.P; i++) o.p[i] = pair(f[2 * i], f[2 * i + 1]);
  return o;
}

// kNorm: the layer norm, with the residual sum and the checkpoint where asked; else the
// checkpoint alone.
template <typename T, int VE, int TPR, int K, bool kNorm>
struct Fwd {
  static constexpr int THREADS = block_threads<TPR>(), NB = VE * (int)sizeof(T);
  static constexpr int BYTES = K * NB * (kNorm ? 2 : 1);  // a thread's slots of a stage
  static constexpr int S = stages<BYTES, THREADS>();
  static constexpr size_t SMEM = (size_t)BYTES * THREADS * S;
};

template <typename T, int VE, int TPR, int K, bool kNorm>
__global__ void __launch_bounds__(block_threads<TPR>()) k_rows_fwd(const RowsArgs args) {
  using F = Fwd<T, VE, TPR, K, kNorm>;
  constexpr int THREADS = F::THREADS, RPB = THREADS / TPR, S = F::S;
  using R = RawV<T, VE>;
  extern __shared__ __align__(16) char slots[];
  __shared__ float red[32];
  RowsArgs a = args;
  grid_begin(a.x, a.res, a.gamma, a.beta);
  const T* x = static_cast<const T*>(a.x);
  const T* res = static_cast<const T*>(a.res);
  const int t = threadIdx.x % TPR, rb = threadIdx.x / TPR;
  const int C = a.C, nb = (C + kCkptBlock - 1) / kCkptBlock;
  const int64_t groups = (a.rows + RPB - 1) / RPB;
  auto issue = [&](int64_t group, int stage) {
    const int64_t row = group * RPB + rb;
    char* base = slots + (size_t)stage * F::BYTES * THREADS;
#pragma unroll
    for (int k = 0; k < K; k++) {
      const int c = (k * TPR + t) * VE;
      const bool ok = row < a.rows && c < C;
      const int64_t at = ok ? row * C + c : 0;
      fetch<F::NB>(slot<R, THREADS>(base, k), x + at, ok);
      if (kNorm && res) fetch<F::NB>(slot<R, THREADS>(base, K + k), res + at, ok);
    }
  };
  int64_t next = blockIdx.x;
#pragma unroll
  for (int s = 0; s < S - 1; s++, next += gridDim.x) {
    if (next < groups) issue(next, s);
    fetch_commit();
  }
  constexpr int N = K * VE, P = Vals<N>::P;
  const Vals<N> gm = channels_of<N, VE, TPR>(kNorm ? a.gamma : nullptr, C, t, 1.f);
  const Vals<N> bt = channels_of<N, VE, TPR>(kNorm ? a.beta : nullptr, C, t, 0.f);
  const bool whole = N % 2 == 0 && ((K - 1) * TPR + t) * VE < C;
  const float invC = 1.f / (float)C;
  int stage = 0;
  for (int64_t group = blockIdx.x; group < groups; group += gridDim.x, next += gridDim.x) {
    if (next < groups) issue(next, stage == 0 ? S - 1 : stage - 1);
    fetch_commit();
    fetch_wait<S - 1>();
    char* base = slots + (size_t)stage * F::BYTES * THREADS;
    stage = stage == S - 1 ? 0 : stage + 1;
    const int64_t row = group * RPB + rb;
    const bool here = row < a.rows;
    R raw[K];
#pragma unroll
    for (int k = 0; k < K; k++) raw[k] = *slot<R, THREADS>(base, k);
    Vals<N> v = vals_of<T, VE, K>(raw);
    if (kNorm && res) {
#pragma unroll
      for (int k = 0; k < K; k++) raw[k] = *slot<R, THREADS>(base, K + k);
      const Vals<N> r = vals_of<T, VE, K>(raw);
#pragma unroll
      for (int i = 0; i < P; i++) v.p[i] = v.p[i] + r.p[i];
      float f[2 * P];
      floats_of(v, f);
      // the stream is kept in its own type, and what is kept is what is normalised
#pragma unroll
      for (int k = 0; k < K; k++) raw[k] = from_float<T, VE>(*reinterpret_cast<float(*)[VE]>(f + k * VE));
      v = vals_of<T, VE, K>(raw);
      if (a.sum && here) {
#pragma unroll
        for (int k = 0; k < K; k++) {
          const int c = (k * TPR + t) * VE;
          if (c < C) *reinterpret_cast<R*>(static_cast<T*>(a.sum) + row * C + c) = raw[k];
        }
      }
    }
    if (!kNorm || a.q8) {
      float f[2 * P];
      floats_of(v, f);
#pragma unroll
      for (int k = 0; k < K; k++) {
        const int c = (k * TPR + t) * VE;
        uint32_t byte;
        RawV<uint8_t, VE> q;
        quantise<VE>(f + k * VE, byte, q);
        if (here && c < C) {
          *reinterpret_cast<RawV<uint8_t, VE>*>(reinterpret_cast<uint8_t*>(a.q8) + row * C + c) = q;
          if (c % kCkptBlock == 0) a.e8[row * nb + c / kCkptBlock] = (uint8_t)byte;
        }
      }
    }
    if constexpr (kNorm) {
      F2 s = v.p[0];  // channels past C hold 0
#pragma unroll
      for (int i = 1; i < P; i++) s = s + v.p[i];
      const float mean = row_sum<TPR>(total(s), red) * invC;
      const F2 minus = pair(-mean, -mean);
      float f[2 * P], d2 = 0.f;
#pragma unroll
      for (int i = 0; i < P; i++) v.p[i] = v.p[i] + minus;
      if (whole) {  // every vector of the thread lies inside C
        F2 q = v.p[0] * v.p[0];
#pragma unroll
        for (int i = 1; i < P; i++) q = fma(v.p[i], v.p[i], q);
        d2 = total(q);
      } else {
        floats_of(v, f);
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
          for (int i = 0; i < VE; i++)
            if ((k * TPR + t) * VE < C) d2 += f[k * VE + i] * f[k * VE + i];
      }
      const float rstd = rsqrtf(row_sum<TPR>(d2, red) * invC + a.eps);
      const F2 r2 = pair(rstd, rstd);
#pragma unroll
      for (int i = 0; i < P; i++) v.p[i] = fma(v.p[i] * r2, gm.p[i], bt.p[i]);
      floats_of(v, f);
      if (here) {
#pragma unroll
        for (int k = 0; k < K; k++) {
          const int c = (k * TPR + t) * VE;
          if (c < C)
            *reinterpret_cast<R*>(static_cast<T*>(a.y) + row * C + c) =
                from_float<T, VE>(*reinterpret_cast<float(*)[VE]>(f + k * VE));
        }
        if (t == 0) {
          if (a.mean) a.mean[row] = mean;
          if (a.rstd) a.rstd[row] = rstd;
        }
      }
    }
  }
}

template <typename T, int VE, int TPR, int K>
__global__ void __launch_bounds__(block_threads<TPR>()) k_ckpt_unpack(const RowsArgs args) {
  constexpr int RPB = block_threads<TPR>() / TPR, RU = K >= 4 ? 1 : 4 / K;  // no sums: loads stay in registers
  RowsArgs a = args;
  grid_begin(a.q8, a.e8);
  const int t = threadIdx.x % TPR, rb = threadIdx.x / TPR;
  const int C = a.C, nb = (C + kCkptBlock - 1) / kCkptBlock;
  const uint8_t* q8 = reinterpret_cast<const uint8_t*>(a.q8);
  for (int64_t r0 = (int64_t)blockIdx.x * (RPB * RU); r0 < a.rows; r0 += (int64_t)gridDim.x * (RPB * RU)) {
    RawV<uint8_t, VE> q[RU][K];
    uint32_t e[RU][K];
#pragma unroll
    for (int u = 0; u < RU; u++) {
      const int64_t row = r0 + u * RPB + rb;
#pragma unroll
      for (int k = 0; k < K; k++) {
        const int c = (k * TPR + t) * VE;
        if (row < a.rows && c < C) {
          q[u][k] = *reinterpret_cast<const RawV<uint8_t, VE>*>(q8 + row * C + c);
          e[u][k] = a.e8[row * nb + c / kCkptBlock];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < RU; u++) {
      const int64_t row = r0 + u * RPB + rb;
#pragma unroll
      for (int k = 0; k < K; k++) {
        const int c = (k * TPR + t) * VE;
        if (row < a.rows && c < C) {
          float f[VE];
          restore<VE>(q[u][k], e[u][k], f);
          *reinterpret_cast<RawV<T, VE>*>(static_cast<T*>(a.y) + row * C + c) = from_float<T, VE>(f);
        }
      }
    }
  }
}

// A row's gradient without its factor rstd, in place of dy in g; xh: v.  Past C, dy is 0: nothing is
// added to the sums there.
template <int TPR, int N>
__device__ __forceinline__ void row_grad(Vals<N>& xh, Vals<N>& g, float mean, float rstd, const Vals<N>& gm, float invC,
                                         float* red, Vals<N>& dg, Vals<N>& db) {
  constexpr int P = Vals<N>::P;
  const F2 minus = pair(-mean, -mean), r2 = pair(rstd, rstd);
  F2 t1 = pair(0.f, 0.f), t2 = t1;
#pragma unroll
  for (int i = 0; i < P; i++) {
    xh.p[i] = (xh.p[i] + minus) * r2;
    db.p[i] = db.p[i] + g.p[i];
    dg.p[i] = fma(g.p[i], xh.p[i], dg.p[i]);
    g.p[i] = g.p[i] * gm.p[i];
    t1 = t1 + g.p[i];
    t2 = fma(g.p[i], xh.p[i], t2);
  }
  const float s1 = row_sum<TPR>(total(t1), red) * invC;
  const float s2 = row_sum<TPR>(total(t2), red) * invC;
  const F2 m1 = pair(-s1, -s1), m2 = pair(-s2, -s2);
#pragma unroll
  for (int i = 0; i < P; i++) g.p[i] = fma(xh.p[i], m2, g.p[i] + m1);
}

// The block's row of partial sums of dgamma (dg) and dbeta (db); acc: W * TPR * N floats.
template <int TPR, int VE, int N, int THREADS>
__device__ __forceinline__ void write_partials(const RowsArgs& a, const Vals<N>& dg, const Vals<N>& db, int t, float* acc) {
  constexpr int W = TPR <= 32 ? THREADS / 32 : 1;  // warps with their own sums of the same channels
  constexpr int WC = TPR * N, P = Vals<N>::P;      // channels a row group covers
  const int C = a.C;
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
  for (int which = 0; which < 2; which++) {
    float sum[2 * P];
    floats_of(which ? db : dg, sum);
    if constexpr (TPR < 32) {  // row groups of a warp
#pragma unroll
      for (int o = TPR; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < N; i++) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
    }
    if constexpr (W > 1) {
      __syncthreads();
      if ((threadIdx.x & 31) < TPR) {
#pragma unroll
        for (int i = 0; i < N; i++) acc[(threadIdx.x >> 5) * WC + (i / VE * TPR + t) * VE + i % VE] = sum[i];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < C; c += THREADS) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < W; w++) s += acc[w * WC + c];
        part[which * C + c] = s;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; i++) {
        const int c = (i / VE * TPR + t) * VE + i % VE;
        if (c < C) part[which * C + c] = sum[i];
      }
    }
  }
}

// kCkpt: v comes from its checkpoint.  Rows on their way stay in registers here, two at a time
// with three blocks of 256 threads on an SM (1,048,576 rows of 256 bf16 channels: 297 us from
// rows, 351 us from the checkpoint with dres; four rows and 126 registers took 467 and 520 us).
template <typename T, int VE, int TPR, int K, bool kCkpt>
__global__ void __launch_bounds__(block_threads<TPR>(), bwd_blocks_per_sm<TPR, K * VE>()) k_norm_bwd(const RowsArgs args) {
  constexpr int THREADS = block_threads<TPR>();
  constexpr int RPB = THREADS / TPR, RU = rows_ahead<K>();
  constexpr int N = K * VE, P = Vals<N>::P;
  using R = RawV<T, VE>;
  using Q = RawV<uint8_t, VE>;
  __shared__ float red[32];
  __shared__ float acc[TPR <= 32 ? THREADS / 32 * TPR * N : 1];
  RowsArgs a = args;
  grid_begin(a.x, a.q8, a.e8, a.gamma, a.mean, a.rstd, a.dy, a.dres);
  if (a.status && blockIdx.x == 0 && threadIdx.x == 0) *a.status = kDevOk;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  const T* dres = static_cast<const T*>(a.dres);
  const uint8_t* q8 = reinterpret_cast<const uint8_t*>(a.q8);
  const int t = threadIdx.x % TPR, rb = threadIdx.x / TPR;
  const int C = a.C, nb = (C + kCkptBlock - 1) / kCkptBlock;
  const Vals<N> gm = channels_of<N, VE, TPR>(a.gamma, C, t, 1.f);
  Vals<N> dg, db;
#pragma unroll
  for (int i = 0; i < P; i++) dg.p[i] = db.p[i] = pair(0.f, 0.f);
  const float invC = 1.f / (float)C;
  for (int64_t r0 = (int64_t)blockIdx.x * (RPB * RU); r0 < a.rows; r0 += (int64_t)gridDim.x * (RPB * RU)) {
    R xr[RU][K], yr[RU][K], rr[RU][K];
    Q q[RU][K];
    uint32_t e[RU][K];
    float mean[RU], rstd[RU];
#pragma unroll
    for (int u = 0; u < RU; u++) {
      const int64_t row = r0 + u * RPB + rb;
      mean[u] = row < a.rows ? a.mean[row] : 0.f;
      rstd[u] = row < a.rows ? a.rstd[row] : 0.f;
#pragma unroll
      for (int k = 0; k < K; k++) {
        const int c = (k * TPR + t) * VE;
        const bool ok = row < a.rows && c < C;
        const int64_t at = row * C + c;
        if constexpr (kCkpt) {
          q[u][k] = ok ? *reinterpret_cast<const Q*>(q8 + at) : raw_zero<Q>();
          e[u][k] = ok ? a.e8[row * nb + c / kCkptBlock] : 0u;
        } else {
          xr[u][k] = ok ? *reinterpret_cast<const R*>(x + at) : raw_zero<R>();
        }
        yr[u][k] = ok ? *reinterpret_cast<const R*>(dy + at) : raw_zero<R>();
        if (dres) rr[u][k] = ok ? *reinterpret_cast<const R*>(dres + at) : raw_zero<R>();
      }
    }
#pragma unroll
    for (int u = 0; u < RU; u++) {
      const int64_t row = r0 + u * RPB + rb;
      Vals<N> xh;
      if constexpr (kCkpt) {
        float f[N + 1];
        f[N] = 0.f;
#pragma unroll
        for (int k = 0; k < K; k++) restore<VE>(q[u][k], e[u][k], *reinterpret_cast<float(*)[VE]>(f + k * VE));
#pragma unroll
        for (int i = 0; i < P; i++) xh.p[i] = pair(f[2 * i], f[2 * i + 1]);
      } else {
        xh = vals_of<T, VE, K>(xr[u]);
      }
      Vals<N> g = vals_of<T, VE, K>(yr[u]);
      row_grad<TPR, N>(xh, g, mean[u], rstd[u], gm, invC, red, dg, db);
      if (dres) {
        const Vals<N> r = vals_of<T, VE, K>(rr[u]);
        const F2 r2 = pair(rstd[u], rstd[u]);
#pragma unroll
        for (int i = 0; i < P; i++) g.p[i] = fma(g.p[i], r2, r.p[i]);
      } else {
        const F2 r2 = pair(rstd[u], rstd[u]);
#pragma unroll
        for (int i = 0; i < P; i++) g.p[i] = g.p[i] * r2;
      }
      if (row < a.rows) {
        float f[2 * P];
        floats_of(g, f);
#pragma unroll
        for (int k = 0; k < K; k++) {
          const int c = (k * TPR + t) * VE;
          if (c < C)
            *reinterpret_cast<R*>(static_cast<T*>(a.y) + row * C + c) =
                from_float<T, VE>(*reinterpret_cast<float(*)[VE]>(f + k * VE));
        }
      }
    }
  }
  write_partials<TPR, VE, N, THREADS>(a, dg, db, t, acc);
}

// The same for rows of one warp each, 16 rows of a block fetched at a time by bulk copies: they
// are one piece of memory per tensor, whatever C is, which one lane fetches into the block's
// stages.  No instruction of the other lanes and no register waits for them.  (Pieces of two rows for
// each warp by itself, 1 KB, took 410 us where these take 333: too many copies.)
struct Bulk {
  int stages, bytes, per_sm;  // of a stage; blocks that an SM holds (0: not for these rows)
};
constexpr int kBulkRows = 16, kBulkStages = 6;
// Dynamic shared memory of a block where per_sm of them share an SM; the rest is for static arrays.
constexpr int bulk_room(int per_sm) { return 232448 / per_sm - 2048; }

// kFull: every lane has K vectors of the row: no lane is masked, and no register zeroed for it (from
// the checkpoint with dres 333 -> 306 us; rows without checkpoint gain nothing).
template <typename T, int VE, int K, bool kCkpt, bool kFull>
__global__ void __launch_bounds__(256, K * VE <= 8 ? 3 : 2) k_norm_bwd_bulk(const RowsArgs args, const Bulk plan) {
  constexpr int N = K * VE, P = Vals<N>::P, RU = kBulkRows / 8;
  using R = RawV<T, VE>;
  using Q = RawV<uint8_t, VE>;
  extern __shared__ __align__(128) char stages[];
  __shared__ uint64_t full[kBulkStages], empty[kBulkStages];
  __shared__ tc::Abort ab;
  __shared__ int issued;  // by thread 0: chunk number i of the block goes to stage i % plan.stages
  RowsArgs a = args;
  const int warp = threadIdx.x >> 5, t = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < plan.stages; s++) {
      tc::mbar_init(&full[s], 1);
      tc::mbar_init(&empty[s], 8);
    }
    ab.flag = 0;
    issued = 0;
    tc::fence_mbar_init();
  }
  __syncthreads();
  grid_begin(a.x, a.q8, a.e8, a.gamma, a.mean, a.rstd, a.dy, a.dres);
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = kDevOk;
  const int C = a.C, nb = (C + kCkptBlock - 1) / kCkptBlock;
  const int64_t chunks = (a.rows + kBulkRows - 1) / kBulkRows;
  const uint32_t nd = (uint32_t)(kBulkRows * C * sizeof(T)), nq = (uint32_t)(kBulkRows * C);
  const uint32_t at_x = a.dres ? 2 * nd : nd, at_e = at_x + nq;  // dy, dres, then v or q8 and e8
  const char* src_dy = static_cast<const char*>(a.dy);
  const char* src_dres = static_cast<const char*>(a.dres);
  const char* src_x = kCkpt ? reinterpret_cast<const char*>(a.q8) : static_cast<const char*>(a.x);
  auto issue = [&](int64_t chunk, int s) {
    if ((chunk + 1) * kBulkRows > a.rows) return;  // a last chunk of fewer rows is read by the lanes
    issued++;
    char* to = stages + (size_t)s * plan.bytes;
    tc::mbar_expect_tx(&full[s], (uint32_t)plan.bytes);
    tc::bulk_load(to, src_dy + chunk * nd, nd, &full[s]);
    if (src_dres) tc::bulk_load(to + nd, src_dres + chunk * nd, nd, &full[s]);
    tc::bulk_load(to + at_x, src_x + chunk * (kCkpt ? nq : nd), kCkpt ? nq : nd, &full[s]);
    if (kCkpt) tc::bulk_load(to + at_e, a.e8 + chunk * kBulkRows * nb, (uint32_t)(kBulkRows * nb), &full[s]);
  };
  const int64_t first = blockIdx.x, step = gridDim.x;
  if (threadIdx.x == 0)
    for (int s = 0; s < plan.stages - 1; s++)
      if (first + s * step < chunks) issue(first + s * step, s);
  auto stat = [&](const float* p, int64_t chunk) {  // lane i: of the warp's row i
    const int64_t row = chunk * kBulkRows + RU * warp + t;
    return t < RU && row < a.rows ? p[row] : 0.f;
  };
  const Vals<N> gm = channels_of<N, VE, 32>(a.gamma, C, t, 1.f);
  Vals<N> dg, db;
#pragma unroll
  for (int i = 0; i < P; i++) dg.p[i] = db.p[i] = pair(0.f, 0.f);
  const float invC = 1.f / (float)C;
  float mean_next = stat(a.mean, first), rstd_next = stat(a.rstd, first);
  int s = 0;
  uint32_t parity = 0;
#pragma unroll 1
  for (int64_t chunk = first; chunk < chunks; chunk += step) {
    const float mean_of = mean_next, rstd_of = rstd_next;
    mean_next = stat(a.mean, chunk + step);
    rstd_next = stat(a.rstd, chunk + step);
    // The stage of the chunk before this one gets the chunk that follows those on their way, once
    // every warp has read it.
    const int64_t ahead = chunk + (plan.stages - 1) * step;
    if (warp == 0 && ahead < chunks) {
      const int w = s == 0 ? plan.stages - 1 : s - 1;
      if (chunk > first && !tc::mbar_wait_w(&empty[w], s == 0 ? parity ^ 1u : parity, &ab, a.status)) break;
      if (t == 0) issue(ahead, w);
    }
    const bool whole = (chunk + 1) * kBulkRows <= a.rows;
    const int64_t row0 = chunk * kBulkRows + RU * warp;
    char* base = stages + (size_t)s * plan.bytes;
    char* b_dy = base + RU * warp * C * sizeof(T);  // the warp's rows
    char* b_dres = b_dy + nd;
    char* b_x = base + at_x + RU * warp * C * (kCkpt ? 1 : sizeof(T));
    uint8_t* b_e = reinterpret_cast<uint8_t*>(base + at_e) + RU * warp * nb;
    if (whole) {
      if (!tc::mbar_wait_w(&full[s], parity, &ab, a.status)) break;
    } else {  // each warp its own, in whose place no other reads; kFull: zeros past the last row
      const int left = (int)max((int64_t)0, min((int64_t)RU, a.rows - row0)) * C;
      const T zero = T(0.f);
#pragma unroll 1
      for (int i = t; i < (kFull ? RU * C : left); i += 32) {
        const int64_t at = row0 * C + i;
        const bool in = !kFull || i < left;
        reinterpret_cast<T*>(b_dy)[i] = in ? static_cast<const T*>(a.dy)[at] : zero;
        if (src_dres) reinterpret_cast<T*>(b_dres)[i] = in ? static_cast<const T*>(a.dres)[at] : zero;
        if (kCkpt) b_x[i] = in ? src_x[at] : 0;
        else reinterpret_cast<T*>(b_x)[i] = in ? static_cast<const T*>(a.x)[at] : zero;
      }
      if (kCkpt)
        for (int i = t; i < (kFull ? RU : left / C) * nb; i += 32) b_e[i] = !kFull || i < left / C * nb ? a.e8[row0 * nb + i] : 0;
      __syncwarp();
    }
#pragma unroll
    for (int u = 0; u < RU; u++) {
      const int64_t row = row0 + u;
      const bool here = row < a.rows;
      const float mean = __shfl_sync(0xffffffffu, mean_of, u), rstd = __shfl_sync(0xffffffffu, rstd_of, u);
      R yr[K], rr[K];
      Vals<N> xh;
      if constexpr (kCkpt) {
        float f[N + 1];
        f[N] = 0.f;
#pragma unroll
        for (int k = 0; k < K; k++) {
          const int c = (k * 32 + t) * VE;
          const bool ok = kFull || (here && c < C);
          const Q q = ok ? *reinterpret_cast<const Q*>(b_x + u * C + c) : raw_zero<Q>();
          const uint32_t e = ok ? b_e[u * nb + c / kCkptBlock] : 0u;
          restore<VE>(q, e, *reinterpret_cast<float(*)[VE]>(f + k * VE));
        }
#pragma unroll
        for (int i = 0; i < P; i++) xh.p[i] = pair(f[2 * i], f[2 * i + 1]);
      } else {
        R xr[K];
#pragma unroll
        for (int k = 0; k < K; k++) {
          const int c = (k * 32 + t) * VE;
          xr[k] = kFull || (here && c < C) ? *reinterpret_cast<const R*>(b_x + (u * C + c) * sizeof(T)) : raw_zero<R>();
        }
        xh = vals_of<T, VE, K>(xr);
      }
#pragma unroll
      for (int k = 0; k < K; k++) {
        const int c = (k * 32 + t) * VE;
        const bool ok = kFull || (here && c < C);
        yr[k] = ok ? *reinterpret_cast<const R*>(b_dy + (u * C + c) * sizeof(T)) : raw_zero<R>();
        if (src_dres) rr[k] = ok ? *reinterpret_cast<const R*>(b_dres + (u * C + c) * sizeof(T)) : raw_zero<R>();
      }
      Vals<N> g = vals_of<T, VE, K>(yr);
      row_grad<32, N>(xh, g, mean, rstd, gm, invC, nullptr, dg, db);
      const F2 r2 = pair(rstd, rstd);
      if (src_dres) {
        const Vals<N> r = vals_of<T, VE, K>(rr);
#pragma unroll
        for (int i = 0; i < P; i++) g.p[i] = fma(g.p[i], r2, r.p[i]);
      } else {
#pragma unroll
        for (int i = 0; i < P; i++) g.p[i] = g.p[i] * r2;
      }
      if (here) {
        float f[2 * P];
        floats_of(g, f);
#pragma unroll
        for (int k = 0; k < K; k++) {
          const int c = (k * 32 + t) * VE;
          if (kFull || c < C)
            *reinterpret_cast<R*>(static_cast<T*>(a.y) + row * C + c) =
                from_float<T, VE>(*reinterpret_cast<float(*)[VE]>(f + k * VE));
        }
      }
    }
    __syncwarp();
    if (t == 0) tc::mbar_arrive(&empty[s]);
    if (++s == plan.stages) {
      s = 0;
      parity ^= 1u;
    }
  }
  // The block keeps its stages until the copies have landed.  (From stage s on: in the order of the
  // numbers the compiler spills 44 bytes more with single loads, 300,000 x 255 bf16 235 -> 241 us.)
  if (threadIdx.x == 0 && ab.flag)
    for (int k = 0, i = s; k < plan.stages; k++, i = i + 1 == plan.stages ? 0 : i + 1)
      if (i < issued) tc::mbar_drain(&full[i], (uint32_t)((issued - 1 - i) / plan.stages) & 1u);
  __syncthreads();  // the stages are free for the sums
  write_partials<32, VE, N, 256>(a, dg, db, t, reinterpret_cast<float*>(stages));
}

// One row of the forward of the norm, from its values in raw; load_res(raw) brings those of res.  The
// same arithmetic as k_rows_fwd's, which keeps its own: sharing this made it slower (1,048,576 x 256
// bf16 188 -> 203 us).
template <typename T, int K, typename F>
__device__ __forceinline__ void forward_row(const RowsArgs& a, int64_t row, int t, bool whole, float invC, const Vals<K>& gm,
                                            const Vals<K>& bt, RawV<T, 1> (&raw)[K], F load_res) {
  constexpr int P = Vals<K>::P;
  using R = RawV<T, 1>;
  const int C = a.C, nb = (C + kCkptBlock - 1) / kCkptBlock;
  Vals<K> v = vals_of<T, 1, K>(raw);
  if (a.res) {
    load_res(raw);
    const Vals<K> r = vals_of<T, 1, K>(raw);
#pragma unroll
    for (int i = 0; i < P; i++) v.p[i] = v.p[i] + r.p[i];
    float f[2 * P];
    floats_of(v, f);
    // the stream is kept in its own type, and what is kept is what is normalised
#pragma unroll
    for (int k = 0; k < K; k++) raw[k] = from_float<T, 1>(*reinterpret_cast<float(*)[1]>(f + k));
    v = vals_of<T, 1, K>(raw);
    if (a.sum) {
#pragma unroll
      for (int k = 0; k < K; k++) {
        const int c = k * 32 + t;
        if (c < C) *reinterpret_cast<R*>(static_cast<T*>(a.sum) + row * C + c) = raw[k];
      }
    }
  }
  if (a.q8) {
    float f[2 * P];
    floats_of(v, f);
#pragma unroll
    for (int k = 0; k < K; k++) {
      const int c = k * 32 + t;
      uint32_t byte;
      uint8_t q;
      quantise<1>(f + k, byte, q);
      if (c < C) {
        reinterpret_cast<uint8_t*>(a.q8)[row * C + c] = q;
        if (c % kCkptBlock == 0) a.e8[row * nb + c / kCkptBlock] = (uint8_t)byte;
      }
    }
  }
  F2 s = v.p[0];  // channels past C hold 0
#pragma unroll
  for (int i = 1; i < P; i++) s = s + v.p[i];
  const float mean = row_sum<32>(total(s), nullptr) * invC;
  const F2 minus = pair(-mean, -mean);
  float f[2 * P], d2 = 0.f;
#pragma unroll
  for (int i = 0; i < P; i++) v.p[i] = v.p[i] + minus;
  if (whole) {  // every value of the thread lies inside C
    F2 q = v.p[0] * v.p[0];
#pragma unroll
    for (int i = 1; i < P; i++) q = fma(v.p[i], v.p[i], q);
    d2 = total(q);
  } else {
    floats_of(v, f);
#pragma unroll
    for (int k = 0; k < K; k++)
      if (k * 32 + t < C) d2 += f[k] * f[k];
  }
  const float rstd = rsqrtf(row_sum<32>(d2, nullptr) * invC + a.eps);
  const F2 r2 = pair(rstd, rstd);
#pragma unroll
  for (int i = 0; i < P; i++) v.p[i] = fma(v.p[i] * r2, gm.p[i], bt.p[i]);
  floats_of(v, f);
#pragma unroll
  for (int k = 0; k < K; k++) {
    const int c = k * 32 + t;
    if (c < C)
      *reinterpret_cast<R*>(static_cast<T*>(a.y) + row * C + c) =
          from_float<T, 1>(*reinterpret_cast<float(*)[1]>(f + k));
  }
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

// The forward for rows of odd C of one warp each, in the same way: single values are below
// cp.async's size for bf16, and each took a load, a store and a load.
//
// No status word here: a warp whose wait gives up (`staged` ends) reads its rows from global memory
// from then on, and so does the last chunk of fewer rows.  Such a warp waits at no barrier of the
// stages again, since a wait for the use after one that it has not seen complete would pass at
// once; and it frees no stage again, so that none is filled anew while a copy may be on its way to it.
template <typename T, int K>
__global__ void __launch_bounds__(256, 3) k_norm_fwd_bulk(const RowsArgs args, const Bulk plan) {
  constexpr int RU = kBulkRows / 8;
  using R = RawV<T, 1>;
  extern __shared__ __align__(128) char stages[];
  __shared__ uint64_t full[kBulkStages], empty[kBulkStages];
  __shared__ tc::Abort ab;
  RowsArgs a = args;
  const int warp = threadIdx.x >> 5, t = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < plan.stages; s++) {
      tc::mbar_init(&full[s], 1);
      tc::mbar_init(&empty[s], 8);
    }
    ab.flag = 0;
    tc::fence_mbar_init();
  }
  __syncthreads();
  grid_begin(a.x, a.res, a.gamma, a.beta);
  const int C = a.C;
  const bool res = a.res != nullptr;
  const int64_t chunks = (a.rows + kBulkRows - 1) / kBulkRows, first = blockIdx.x, step = gridDim.x;
  const uint32_t nd = (uint32_t)(kBulkRows * C * sizeof(T));
  int issued = 0;  // by thread 0: chunk number i of the block goes to stage i % plan.stages
  auto issue = [&](int64_t chunk, int s) {
    if ((chunk + 1) * kBulkRows > a.rows) return;  // a last chunk of fewer rows is read by the lanes
    issued++;
    char* to = stages + (size_t)s * plan.bytes;
    tc::mbar_expect_tx(&full[s], (uint32_t)plan.bytes);
    tc::bulk_load(to, static_cast<const char*>(a.x) + chunk * nd, nd, &full[s]);
    if (res) tc::bulk_load(to + nd, static_cast<const char*>(a.res) + chunk * nd, nd, &full[s]);
  };
  if (threadIdx.x == 0)
    for (int s = 0; s < plan.stages - 1; s++)
      if (first + s * step < chunks) issue(first + s * step, s);
  const Vals<K> gm = channels_of<K, 1, 32>(a.gamma, C, t, 1.f);
  const Vals<K> bt = channels_of<K, 1, 32>(a.beta, C, t, 0.f);
  const bool inside = K % 2 == 0 && (K - 1) * 32 + t < C;
  const float invC = 1.f / (float)C;
  int s = 0;
  uint32_t parity = 0;
  bool staged = true;
#pragma unroll 1
  for (int64_t chunk = first; chunk < chunks; chunk += step) {
    const int64_t ahead = chunk + (plan.stages - 1) * step;
    if (warp == 0 && staged && ahead < chunks) {
      const int w = s == 0 ? plan.stages - 1 : s - 1;
      staged = chunk == first || tc::mbar_wait_w(&empty[w], s == 0 ? parity ^ 1u : parity, &ab, nullptr);
      if (staged && t == 0) issue(ahead, w);
    }
    const int64_t row0 = chunk * kBulkRows + RU * warp;
    const T* x = reinterpret_cast<const T*>(stages + (size_t)s * plan.bytes) + RU * warp * C;  // the warp's rows
    const T* r = reinterpret_cast<const T*>(reinterpret_cast<const char*>(x) + nd);
    const bool whole = (chunk + 1) * kBulkRows <= a.rows;
    if (whole && staged) staged = tc::mbar_wait_w(&full[s], parity, &ab, nullptr);
    if (whole && staged) {
#pragma unroll
      for (int u = 0; u < RU; u++) {
        auto load = [&](R (&to)[K], const T* from) {
#pragma unroll
          for (int k = 0; k < K; k++) {
            const int c = k * 32 + t;
            to[k] = c < C ? *reinterpret_cast<const R*>(from + u * C + c) : R(0);
          }
        };
        R raw[K];
        load(raw, x);
        forward_row<T, K>(a, row0 + u, t, inside, invC, gm, bt, raw, [&](R (&to)[K]) { load(to, r); });
      }
    } else {
#pragma unroll 1
      for (int64_t row = row0; row < min(row0 + RU, a.rows); row++) {
        auto load = [&](R (&to)[K], const void* from) {
#pragma unroll
          for (int k = 0; k < K; k++) {
            const int c = k * 32 + t;
            to[k] = c < C ? *reinterpret_cast<const R*>(static_cast<const T*>(from) + row * C + c) : R(0);
          }
        };
        R raw[K];
        load(raw, a.x);
        forward_row<T, K>(a, row, t, inside, invC, gm, bt, raw, [&](R (&to)[K]) { load(to, a.res); });
      }
    }
    __syncwarp();
    if (t == 0 && staged) tc::mbar_arrive(&empty[s]);
    if (++s == plan.stages) {
      s = 0;
      parity ^= 1u;
    }
  }
  if (threadIdx.x == 0 && !staged)  // the block keeps its stages until the copies have landed
    for (int i = max(0, issued - plan.stages); i < issued; i++)
      tc::mbar_drain(&full[i % plan.stages], (uint32_t)(i / plan.stages) & 1u);
}

// ---- choice of the plan ----------------------------------------------------------------------

// Calls f(VE, TPR, K) as integral constants.  A row goes to the fewest threads that hold it in
// at most 16 channels each (the backward keeps five values of every channel in registers): 8
// or 32 threads of a warp, else a block of 128 or 512.
template <int V>
struct Int { static constexpr int value = V; };
template <typename T, int VE, typename F>
auto with_lanes(int C, F f) {
  const int slots = (C + VE - 1) / VE;
  constexpr int KM = 16 / VE;
  if constexpr (VE >= 4)
    if (slots <= 8) return f(Int<VE>(), Int<8>(), Int<1>());
  if (slots <= 32) return f(Int<VE>(), Int<32>(), Int<1>());
  if (slots <= 64) return f(Int<VE>(), Int<32>(), Int<2>());
  if constexpr (KM >= 4) if (slots <= 128) return f(Int<VE>(), Int<32>(), Int<4>());
  if constexpr (KM >= 8) if (slots <= 256) return f(Int<VE>(), Int<32>(), Int<8>());
  if constexpr (KM < 4) if (slots <= 128) return f(Int<VE>(), Int<128>(), Int<1>());
  if constexpr (KM < 8) if (slots <= 256) return f(Int<VE>(), Int<128>(), Int<2>());
  if constexpr (KM >= 4) if (slots <= 512) return f(Int<VE>(), Int<128>(), Int<4>());
  if constexpr (KM >= 8) if (slots <= 1024) return f(Int<VE>(), Int<128>(), Int<8>());
  if constexpr (KM < 4) if (slots <= 512) return f(Int<VE>(), Int<512>(), Int<1>());
  if constexpr (KM < 8) if (slots <= 1024) return f(Int<VE>(), Int<512>(), Int<2>());
  if constexpr (KM == 4 || KM == 8) if (slots <= 2048) return f(Int<VE>(), Int<512>(), Int<4>());
  if constexpr (KM >= 8) if (slots <= 4096) return f(Int<VE>(), Int<512>(), Int<8>());
  return f(Int<VE>(), Int<512>(), Int<KM>());
}
// Vectors of 16 bytes where every row starts on one; else of four channels, pairs, single ones.
template <typename T, typename F>
auto with_plan(int C, F f) {
  constexpr int V16 = 16 / sizeof(T);
  if (C % V16 == 0) return with_lanes<T, V16>(C, f);
  if constexpr (V16 == 8)
    if (C % 4 == 0) return with_lanes<T, 4>(C, f);
  if (C % 2 == 0) return with_lanes<T, 2>(C, f);
  return with_lanes<T, 1>(C, f);
}

// Blocks for `rows` rows, `ahead` of them a row group at a time: one wave of three (of 256 threads)
// an SM, or, where each still has `least` turns to fill its loads in, up to per_sm, several waves
// that even out.
template <typename V, typename TPR, typename K>
dim3 grid_of(int64_t rows, int per_sm, int ahead, int least) {
  const int64_t per = (int64_t)(block_threads<TPR::value>() / TPR::value) * ahead;
  const int64_t turns = (rows + per - 1) / per, scale = (int64_t)num_sms() * 256;
  const int64_t wave = std::max<int64_t>(1, scale * 3 / block_threads<TPR::value>());
  const int64_t most = std::max<int64_t>(1, scale * per_sm / block_threads<TPR::value>());
  const int64_t many = std::min(most, turns / least);
  return dim3((unsigned)std::min(turns, many >= 3 * wave ? many : wave));
}
constexpr int kFwdPerSm = 24;  // most blocks of 256 threads per SM: several waves, which even out

// Only the kernels that some call reaches are compiled: bulk copies where they may be the faster
// way, rows in registers where they are not always.
template <typename T, int VE, int N>
constexpr bool bulk_always() {
  if (N <= 8 && VE != 1) return false;
  return bulk_room(2) / (kBulkRows * 32 * N * (int)sizeof(T) * 3) >= 2;  // two stages of the widest rows, dy, dres and v
}
template <typename T, int VE, int N>
constexpr bool bulk_ever() { return N > 8 || VE == 1 || VE == 8; }

// Stages that fit with three blocks on an SM, or with two; and whether bulk copies are the faster
// way (us, bulk / rows in registers; r: with dres, q: from the checkpoint):
//   16 channels a lane, of which registers hold few rows: always.  300,000 rows of bf16, C = 512 r
//     183 / 269, 384 rq 149 / 240, with vectors of two 300 rq 214 / 330
//   odd C, single loads: always.  300,000 x 101 bf16 77 / 110, fp32 r 91 / 102
//   8 channels of bf16: with three stages and 32 turns a block.  1,048,576 x 256 274 / 297,
//     r 349 / 350, rq 306 / 351, q 287 / 302; 20,000 x 256 rq 13.6 / 13.2
//   else never: fp32 stages are too long.  524,288 x 256 277 / 244, 60,033 x 198 41 / 35
template <typename T, int VE, int N>
Bulk bulk_plan(const RowsArgs& a) {
  const int nb = (a.C + kCkptBlock - 1) / kCkptBlock, nd = kBulkRows * a.C * (int)sizeof(T);
  const int bytes = nd * (a.dres ? 2 : 1) + (a.q8 ? kBulkRows * (a.C + nb) : nd);
  for (int per_sm = N <= 8 ? 3 : 2; per_sm >= 2; per_sm--) {
    const int fit = bulk_room(per_sm) / bytes;
    if (fit < 2) continue;
    const bool many = a.rows >= (int64_t)num_sms() * per_sm * kBulkRows * 32;
    if (N > 8 || VE == 1 || (fit >= 3 && many)) return {std::min(fit, kBulkStages), bytes, per_sm};
    break;
  }
  return {};
}
inline int64_t bulk_blocks(int64_t rows, int per_sm) {
  return std::min((int64_t)num_sms() * per_sm, (rows + kBulkRows - 1) / kBulkRows);
}

}  // namespace rows

template <typename T>
int64_t norm_bwd_blocks(int64_t rows, int C) {
  return rows::with_plan<T>(C, [&](auto v, auto l, auto k) {
    const int64_t n = rows::grid_of<decltype(v), decltype(l), decltype(k)>(rows, 9, rows::rows_ahead<decltype(k)::value>(), 16).x;
    return decltype(l)::value == 32 ? std::max(n, rows::bulk_blocks(rows, 3)) : n;
  });
}

template <typename T, bool kNorm>
cudaError_t rows_fwd(const RowsArgs& a, cudaStream_t st) {
  return rows::with_plan<T>(a.C, [&](auto v, auto l, auto k) {
    using V = decltype(v); using L = decltype(l); using K = decltype(k);
    // The norm of more than 64 channels, odd C: 300,000 rows of bf16 255 287 -> 86 us, with res and
    // checkpoint 611 -> 225; 101 92 -> 62 and 193 -> 131; 33 channels 50 / 57, the checkpoint alone 74 / 81
    // stay with the slots.  At most 256 channels: two stages always fit.
    if constexpr (kNorm && V::value == 1 && L::value == 32 && K::value >= 4) {
      const int bytes = rows::kBulkRows * a.C * (int)sizeof(T) * (a.res ? 2 : 1);
      const rows::Bulk plan{std::min(rows::bulk_room(3) / bytes, rows::kBulkStages), bytes, 3};
      auto kernel = rows::k_norm_fwd_bulk<T, K::value>;
      const size_t smem = (size_t)plan.stages * plan.bytes;
      if (cudaError_t e = allow_smem<rows::bulk_room(3)>(kernel)) return e;
      return launch(kernel, dim3((unsigned)rows::bulk_blocks(a.rows, plan.per_sm)), dim3(256), smem, st, a, plan);
    } else {
      using F = rows::Fwd<T, V::value, L::value, K::value, kNorm>;
      auto kernel = rows::k_rows_fwd<T, V::value, L::value, K::value, kNorm>;
      if constexpr (F::SMEM > 24576)  // with the static arrays past the default limit
        if (cudaError_t e = allow_smem<F::SMEM>(kernel)) return e;
      return launch(kernel, rows::grid_of<V, L, K>(a.rows, rows::kFwdPerSm, 1, 8), dim3(F::THREADS), F::SMEM, st, a);
    }
  });
}
template <typename T>
cudaError_t norm_fwd(const RowsArgs& a, cudaStream_t st) { return rows_fwd<T, true>(a, st); }
template <typename T>
cudaError_t ckpt_pack(const RowsArgs& a, cudaStream_t st) { return rows_fwd<T, false>(a, st); }

template <typename T>
cudaError_t ckpt_unpack(const RowsArgs& a, cudaStream_t st) {
  return rows::with_plan<T>(a.C, [&](auto v, auto l, auto k) {
    using V = decltype(v); using L = decltype(l); using K = decltype(k);
    return launch(rows::k_ckpt_unpack<T, V::value, L::value, K::value>,
                  rows::grid_of<V, L, K>(a.rows, rows::kFwdPerSm, 1, 8), dim3(rows::block_threads<L::value>()), 0, st, a);
  });
}

template <typename T>
cudaError_t norm_bwd(const RowsArgs& a, int64_t* blocks, cudaStream_t st) {
  return rows::with_plan<T>(a.C, [&](auto v, auto l, auto k) {
    using V = decltype(v); using L = decltype(l); using K = decltype(k);
    constexpr int N = V::value * K::value;
    if constexpr (L::value == 32 && rows::bulk_ever<T, V::value, N>()) {
      const rows::Bulk plan = rows::bulk_plan<T, V::value, N>(a);
      if (plan.per_sm) {
        *blocks = rows::bulk_blocks(a.rows, plan.per_sm);
        const size_t smem = std::max((size_t)plan.stages * plan.bytes, (size_t)8 * 32 * N * sizeof(float));
        constexpr bool kCanBeFull = V::value == 8;
        const auto kernel = !a.q8                             ? rows::k_norm_bwd_bulk<T, V::value, K::value, false, false>
                            : kCanBeFull && a.C == 32 * N ? rows::k_norm_bwd_bulk<T, V::value, K::value, true, kCanBeFull>
                                                              : rows::k_norm_bwd_bulk<T, V::value, K::value, true, false>;
        if (cudaError_t e = allow_smem<rows::bulk_room(2)>(kernel)) return e;  // no plan has fewer blocks an SM
        return launch(kernel, dim3((unsigned)*blocks), dim3(256), smem, st, a, plan);
      }
    }
    if constexpr (L::value == 32 && rows::bulk_always<T, V::value, N>()) {
      return cudaErrorInvalidValue;  // the plan above was not empty
    } else {
      const dim3 grid = rows::grid_of<V, L, K>(a.rows, 9, rows::rows_ahead<K::value>(), 16);
      const dim3 block(rows::block_threads<L::value>());
      *blocks = grid.x;
      return a.q8 ? launch(rows::k_norm_bwd<T, V::value, L::value, K::value, true>, grid, block, 0, st, a)
                  : launch(rows::k_norm_bwd<T, V::value, L::value, K::value, false>, grid, block, 0, st, a);
    }
  });
}

}  // namespace fs
