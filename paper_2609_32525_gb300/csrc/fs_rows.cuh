// Layer norm forward and backward, and the 8-bit checkpoint, over rows of C channels.
//
//   forward    v = x + res;  mean, var over the row;  y = (v - mean) rstd gamma + beta,
//              rstd = 1 / sqrt(var + eps)
//   backward   xh = (v - mean) rstd, g = dy gamma:
//              dv = rstd (g - avg(g) - xh avg(g xh)) + dres;  dgamma = sum dy xh, dbeta = sum dy
//   checkpoint blocks of 32 channels: v ~ q 2^s, q whole in [-127, 127], s the smallest that
//              brings the block's largest magnitude to 127; the byte s + 127 is kept, 255 for a
//              block with NaN or infinity.  2^s scales exactly, so that the only rounding is
//              q's (half a step, at most 2^-7 of the block's largest magnitude).
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

// Quantises a vector of a row; the 32 / VE neighbouring lanes that share a block agree on its
// scale.  All lanes of the warp call it.
template <int VE>
__device__ __forceinline__ void quantise(const float (&f)[VE], uint32_t& byte, RawV<uint8_t, VE>& q) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < VE; i++) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
#pragma unroll
  for (int o = kCkptBlock / VE / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  byte = scale_byte(top);
  const float inv = inverse_scale_of(byte);
  uint8_t b[VE];
#pragma unroll
  for (int i = 0; i < VE; i++) b[i] = (uint8_t)(int8_t)__float2int_rn(byte == 255u ? 0.f : f[i] * inv);
  memcpy(&q, b, sizeof(q));
}
template <int VE>
__device__ __forceinline__ void restore(const RawV<uint8_t, VE>& q, uint32_t byte, float (&f)[VE]) {
  const float size = scale_of(byte);
  int8_t b[VE];
  memcpy(b, &q, sizeof(q));
#pragma unroll
  for (int i = 0; i < VE; i++) f[i] = (float)b[i] * size;
}

// Rows in flight per thread: four vectors' loads are issued before the first is used.
template <int K>
__host__ __device__ constexpr int rows_ahead() { return K >= 4 ? 1 : 4 / K; }

// kNorm: the layer norm, with the residual sum and the checkpoint where asked; else the
// checkpoint alone.
template <typename T, int VE, int TPR, int K, bool kNorm>
__global__ void __launch_bounds__(block_threads<TPR>()) k_rows_fwd(const RowsArgs args) {
  constexpr int RPB = block_threads<TPR>() / TPR, RU = rows_ahead<K>();
  __shared__ float red[32];
  RowsArgs a = args;
  grid_begin(a.x, a.res, a.gamma, a.beta);
  const T* x = static_cast<const T*>(a.x);
  const T* res = static_cast<const T*>(a.res);
  const int t = threadIdx.x % TPR, rb = threadIdx.x / TPR;
  const int C = a.C, nb = (C + kCkptBlock - 1) / kCkptBlock;
  float gm[K][VE], bt[K][VE];
  if constexpr (kNorm) {
#pragma unroll
    for (int k = 0; k < K; k++)
#pragma unroll
      for (int i = 0; i < VE; i++) {
        const int c = (k * TPR + t) * VE + i;
        gm[k][i] = a.gamma && c < C ? a.gamma[c] : 1.f;
        bt[k][i] = a.beta && c < C ? a.beta[c] : 0.f;
      }
  }
  const float invC = 1.f / (float)C;
  for (int64_t r0 = (int64_t)blockIdx.x * (RPB * RU); r0 < a.rows; r0 += (int64_t)gridDim.x * (RPB * RU)) {
    RawV<T, VE> xr[RU][K], rr[RU][K];
#pragma unroll
    for (int u = 0; u < RU; u++) {
      const int64_t row = r0 + u * RPB + rb;
#pragma unroll
      for (int k = 0; k < K; k++) {
        const int c = (k * TPR + t) * VE;
        const bool ok = row < a.rows && c < C;
        xr[u][k] = ok ? *reinterpret_cast<const RawV<T, VE>*>(x + row * C + c) : raw_zero<RawV<T, VE>>();
        if (kNorm && res)
          rr[u][k] = ok ? *reinterpret_cast<const RawV<T, VE>*>(res + row * C + c) : raw_zero<RawV<T, VE>>();
      }
    }
#pragma unroll
    for (int u = 0; u < RU; u++) {
      const int64_t row = r0 + u * RPB + rb;
      const bool here = row < a.rows;
      float v[K][VE];
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < K; k++) {
        const int c = (k * TPR + t) * VE;
        to_float<T, VE>(xr[u][k], v[k]);
        if (kNorm && res) {
          float r[VE];
          to_float<T, VE>(rr[u][k], r);
#pragma unroll
          for (int i = 0; i < VE; i++) r[i] += v[k][i];
          // the stream is kept in its own type, and what is kept is what is normalised
          const RawV<T, VE> w = from_float<T, VE>(r);
          to_float<T, VE>(w, v[k]);
          if (a.sum && here && c < C)
            *reinterpret_cast<RawV<T, VE>*>(static_cast<T*>(a.sum) + row * C + c) = w;
        }
        if constexpr (kNorm) {
#pragma unroll
          for (int i = 0; i < VE; i++) s += v[k][i];  // channels past C hold 0
        }
      }
      if (!kNorm || a.q8) {
#pragma unroll
        for (int k = 0; k < K; k++) {
          const int c = (k * TPR + t) * VE;
          uint32_t byte;
          RawV<uint8_t, VE> q;
          quantise<VE>(v[k], byte, q);
          if (here && c < C) {
            *reinterpret_cast<RawV<uint8_t, VE>*>(reinterpret_cast<uint8_t*>(a.q8) + row * C + c) = q;
            if (c % kCkptBlock == 0) a.e8[row * nb + c / kCkptBlock] = (uint8_t)byte;
          }
        }
      }
      if constexpr (kNorm) {
        const float mean = row_sum<TPR>(s, red) * invC;
        float d2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
          for (int i = 0; i < VE; i++) {
            const int c = (k * TPR + t) * VE + i;
            v[k][i] -= mean;
            if (c < C) d2 += v[k][i] * v[k][i];
          }
        const float rstd = 1.f / sqrtf(row_sum<TPR>(d2, red) * invC + a.eps);
        if (here) {
#pragma unroll
          for (int k = 0; k < K; k++) {
            const int c = (k * TPR + t) * VE;
            float o[VE];
#pragma unroll
            for (int i = 0; i < VE; i++) o[i] = v[k][i] * rstd * gm[k][i] + bt[k][i];
            if (c < C) *reinterpret_cast<RawV<T, VE>*>(static_cast<T*>(a.y) + row * C + c) = from_float<T, VE>(o);
          }
          if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
          }
        }
      }
    }
  }
}

template <typename T, int VE, int TPR, int K>
__global__ void __launch_bounds__(block_threads<TPR>()) k_ckpt_unpack(const RowsArgs args) {
  constexpr int RPB = block_threads<TPR>() / TPR, RU = rows_ahead<K>();
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

// kCkpt: v comes from its checkpoint.
template <typename T, int VE, int TPR, int K, bool kCkpt>
__global__ void __launch_bounds__(block_threads<TPR>()) k_norm_bwd(const RowsArgs args) {
  constexpr int THREADS = block_threads<TPR>();
  constexpr int RPB = THREADS / TPR, RU = rows_ahead<K>();
  constexpr int W = TPR <= 32 ? THREADS / 32 : 1;  // warps with their own sums of the same channels
  constexpr int WC = TPR * K * VE;                 // channels a row group covers
  __shared__ float red[32];
  __shared__ float acc[W > 1 ? W * WC : 1];
  RowsArgs a = args;
  grid_begin(a.x, a.q8, a.e8, a.gamma, a.mean, a.rstd, a.dy, a.dres);
  if (a.status && blockIdx.x == 0 && threadIdx.x == 0) *a.status = kDevOk;
  const T* x = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  const T* dres = static_cast<const T*>(a.dres);
  const uint8_t* q8 = reinterpret_cast<const uint8_t*>(a.q8);
  const int t = threadIdx.x % TPR, rb = threadIdx.x / TPR;
  const int C = a.C, nb = (C + kCkptBlock - 1) / kCkptBlock;
  float gm[K][VE], dg[K][VE], db[K][VE];
#pragma unroll
  for (int k = 0; k < K; k++)
#pragma unroll
    for (int i = 0; i < VE; i++) {
      const int c = (k * TPR + t) * VE + i;
      gm[k][i] = a.gamma && c < C ? a.gamma[c] : 1.f;
      dg[k][i] = db[k][i] = 0.f;
    }
  const float invC = 1.f / (float)C;
  for (int64_t r0 = (int64_t)blockIdx.x * (RPB * RU); r0 < a.rows; r0 += (int64_t)gridDim.x * (RPB * RU)) {
    RawV<T, VE> xr[RU][K], yr[RU][K], rr[RU][K];
    RawV<uint8_t, VE> q[RU][K];
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
          q[u][k] = ok ? *reinterpret_cast<const RawV<uint8_t, VE>*>(q8 + at) : raw_zero<RawV<uint8_t, VE>>();
          e[u][k] = ok ? a.e8[row * nb + c / kCkptBlock] : 0u;
        } else {
          xr[u][k] = ok ? *reinterpret_cast<const RawV<T, VE>*>(x + at) : raw_zero<RawV<T, VE>>();
        }
        yr[u][k] = ok ? *reinterpret_cast<const RawV<T, VE>*>(dy + at) : raw_zero<RawV<T, VE>>();
        if (dres) rr[u][k] = ok ? *reinterpret_cast<const RawV<T, VE>*>(dres + at) : raw_zero<RawV<T, VE>>();
      }
    }
#pragma unroll
    for (int u = 0; u < RU; u++) {
      const int64_t row = r0 + u * RPB + rb;
      float xh[K][VE], g[K][VE];
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int k = 0; k < K; k++) {
        if constexpr (kCkpt) restore<VE>(q[u][k], e[u][k], xh[k]);
        else to_float<T, VE>(xr[u][k], xh[k]);
        float d[VE];
        to_float<T, VE>(yr[u][k], d);
#pragma unroll
        for (int i = 0; i < VE; i++) {
          const bool in = VE > 1 || (k * TPR + t) * VE + i < C;  // vectors lie whole inside or outside C
          xh[k][i] = (xh[k][i] - mean[u]) * rstd[u];
          // past C, dy is 0: nothing is added there
          db[k][i] += d[i];
          dg[k][i] += d[i] * xh[k][i];
          g[k][i] = d[i] * gm[k][i];
          s1 += in ? g[k][i] : 0.f;
          s2 += in ? g[k][i] * xh[k][i] : 0.f;
        }
      }
      s1 = row_sum<TPR>(s1, red) * invC;
      s2 = row_sum<TPR>(s2, red) * invC;
      if (row < a.rows) {
#pragma unroll
        for (int k = 0; k < K; k++) {
          const int c = (k * TPR + t) * VE;
          float o[VE], r[VE];
          if (dres) to_float<T, VE>(rr[u][k], r);
#pragma unroll
          for (int i = 0; i < VE; i++) {
            o[i] = (g[k][i] - s1 - xh[k][i] * s2) * rstd[u];
            if (dres) o[i] += r[i];
          }
          if (c < C) *reinterpret_cast<RawV<T, VE>*>(static_cast<T*>(a.y) + row * C + c) = from_float<T, VE>(o);
        }
      }
    }
  }
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
  for (int which = 0; which < 2; which++) {
    float(&sum)[K][VE] = which ? db : dg;
    if constexpr (TPR < 32) {  // row groups of a warp
#pragma unroll
      for (int o = TPR; o < 32; o <<= 1)
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
          for (int i = 0; i < VE; i++) sum[k][i] += __shfl_xor_sync(0xffffffffu, sum[k][i], o);
    }
    if constexpr (W > 1) {
      __syncthreads();
      if ((threadIdx.x & 31) < TPR) {
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
          for (int i = 0; i < VE; i++) acc[(threadIdx.x >> 5) * WC + (k * TPR + t) * VE + i] = sum[k][i];
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
      for (int k = 0; k < K; k++)
#pragma unroll
        for (int i = 0; i < VE; i++) {
          const int c = (k * TPR + t) * VE + i;
          if (c < C) part[which * C + c] = sum[k][i];
        }
    }
  }
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
// Vectors of 16 bytes where every row starts on one; else pairs of bf16, else single channels.
template <typename T, typename F>
auto with_plan(int C, F f) {
  constexpr int V16 = 16 / sizeof(T);
  if (C % V16 == 0) return with_lanes<T, V16>(C, f);
  if constexpr (sizeof(T) == 2)
    if (C % 2 == 0) return with_lanes<T, 2>(C, f);
  return with_lanes<T, 1>(C, f);
}

template <typename V, typename TPR, typename K>
int64_t rows_per_block() { return (int64_t)(block_threads<TPR::value>() / TPR::value) * rows_ahead<K::value>(); }
template <typename V, typename TPR, typename K>
dim3 grid_of(int64_t rows, int per_sm) {
  const int64_t per = rows_per_block<V, TPR, K>();
  const int64_t most = (int64_t)num_sms() * per_sm * 256 / block_threads<TPR::value>();
  const int64_t want = (rows + per - 1) / per;
  return dim3((unsigned)(want < most ? want : (most < 1 ? 1 : most)));
}
constexpr int kFwdPerSm = 8, kBwdPerSm = 4;  // blocks of 256 threads per SM, by their registers

}  // namespace rows

template <typename T>
int64_t norm_bwd_blocks(int64_t rows, int C) {
  return rows::with_plan<T>(C, [&](auto v, auto l, auto k) {
    return (int64_t)rows::grid_of<decltype(v), decltype(l), decltype(k)>(rows, rows::kBwdPerSm).x;
  });
}

template <typename T>
cudaError_t norm_fwd(const RowsArgs& a, cudaStream_t st) {
  return rows::with_plan<T>(a.C, [&](auto v, auto l, auto k) {
    using V = decltype(v); using L = decltype(l); using K = decltype(k);
    return launch(rows::k_rows_fwd<T, V::value, L::value, K::value, true>,
                  rows::grid_of<V, L, K>(a.rows, rows::kFwdPerSm), dim3(rows::block_threads<L::value>()), 0, st, a);
  });
}

template <typename T>
cudaError_t ckpt_pack(const RowsArgs& a, cudaStream_t st) {
  return rows::with_plan<T>(a.C, [&](auto v, auto l, auto k) {
    using V = decltype(v); using L = decltype(l); using K = decltype(k);
    return launch(rows::k_rows_fwd<T, V::value, L::value, K::value, false>,
                  rows::grid_of<V, L, K>(a.rows, rows::kFwdPerSm), dim3(rows::block_threads<L::value>()), 0, st, a);
  });
}

template <typename T>
cudaError_t ckpt_unpack(const RowsArgs& a, cudaStream_t st) {
  return rows::with_plan<T>(a.C, [&](auto v, auto l, auto k) {
    using V = decltype(v); using L = decltype(l); using K = decltype(k);
    return launch(rows::k_ckpt_unpack<T, V::value, L::value, K::value>,
                  rows::grid_of<V, L, K>(a.rows, rows::kFwdPerSm), dim3(rows::block_threads<L::value>()), 0, st, a);
  });
}

template <typename T>
cudaError_t norm_bwd(const RowsArgs& a, int64_t blocks, cudaStream_t st) {
  return rows::with_plan<T>(a.C, [&](auto v, auto l, auto k) {
    using V = decltype(v); using L = decltype(l); using K = decltype(k);
    const dim3 grid((unsigned)blocks), block(rows::block_threads<L::value>());
    return a.q8 ? launch(rows::k_norm_bwd<T, V::value, L::value, K::value, true>, grid, block, 0, st, a)
                : launch(rows::k_norm_bwd<T, V::value, L::value, K::value, false>, grid, block, 0, st, a);
  });
}

}  // namespace fs
