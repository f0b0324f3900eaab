// Device code that the attention's kernels share: the sides of a call, a pair's score, the exact
// rows for values that are not finite, and the joins of split results.  Internal linkage.
#pragma once

#include "fs_attn.h"
#include "fs_internal.h"
#include "fs_launch.h"

#include <climits>
#include <cmath>

namespace fs {
namespace {

__device__ __forceinline__ uint32_t tf32_hi(float x) {  // to nearest, ties away from zero
  return (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
}
struct Split {
  uint32_t hi, lo;
};
__device__ __forceinline__ Split split(float x) {
  const uint32_t h = tf32_hi(x);
  return {h, __float_as_uint(x - __uint_as_float(h))};
}

// The hardware's 2^x, 2^-22 relative: as much as the rounding of x costs from |x| = 6 on.  Below
// 2^-126 it is 0.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A side of the attention that a block owns or streams: queries (a unit's rows) or keys.
struct Side {
  const float *x0, *x1;  // [n, d]: q and dout, or k and v (x1 null: not needed)
  const float* pos;      // by token, or null
  const int* doc;        // by token, or null
  int n;                 // rows of the unit
  int tokens;            // row r is token r % tokens
  int first;             // the index of token 0 among the keys
  __device__ __forceinline__ int token(int r) const { return r < tokens ? r : r % tokens; }
  __device__ __forceinline__ float place(int tok) const { return pos ? pos[tok] : (float)(first + tok); }
};
struct Unit {
  Side q, k;
  int b, kvh, prefix;
};
__device__ __forceinline__ Unit unit_of(const AttnArgs& a, int unit, int d) {
  Unit u;
  u.b = unit / a.Hkv;
  u.kvh = unit - u.b * a.Hkv;
  const int64_t qo = (int64_t)unit * a.rows * d, ko = (int64_t)unit * a.Gk * d;
  u.q = {a.q + qo, a.dout ? a.dout + qo : nullptr, a.pos_q ? a.pos_q + (int64_t)u.b * a.Gq : nullptr,
         a.doc_q ? a.doc_q + (int64_t)u.b * a.Gq : nullptr, a.rows, a.Gq, a.Gk - a.Gq};
  u.k = {a.k + ko, a.v + ko, a.pos_k ? a.pos_k + (int64_t)u.b * a.Gk : nullptr,
         a.doc_k ? a.doc_k + (int64_t)u.b * a.Gk : nullptr, a.Gk, a.Gk, 0};
  u.prefix = a.causal && a.prefix ? a.prefix[u.b] : 0;
  return u;
}

// The pair's score in base-2 units from the product s = q.k, and the factor of its gradient.
struct Score {
  float a, slope;
};
__device__ __forceinline__ Score score_of(const AttnArgs& p, float s, float slope2, float far) {
  Score r;
  r.slope = p.scale;
  if (p.cap > 0.f) {
    const float t = tanhf(s * p.scale / p.cap);
    r.a = p.cap * kLog2e * t;
    r.slope = p.scale * (1.f - t * t);
  } else {
    r.a = s * (p.scale * kLog2e);
  }
  if (p.slopes) r.a -= slope2 * far;
  return r;
}
// The statistic as the backward subtracts it: a row that saw nothing has weight 0 everywhere.
__device__ __forceinline__ float lse2_of(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }
__device__ __forceinline__ bool sees(const AttnArgs& a, int prefix, int qi, int kj, int qdoc, int kdoc) {
  if (a.causal && kj > qi && kj >= prefix) return false;
  return !a.doc_q || (qdoc == kdoc && kdoc >= 0);
}

// Range of documents and of key indexes that the block's own rows hold.
struct Own {
  int doc_lo, doc_hi, first, last;
};
__device__ __forceinline__ Own own_range(const AttnArgs& a, const Side& s, int r0, int r1) {
  Own o{0x7fffffff, -1, 0, 0};
  r1 = min(r1, s.n);
  const int t0 = s.token(r0), t1 = s.token(r1 - 1);
  const bool wraps = r1 - r0 > t1 - t0 + 1;  // rows of several heads
  o.first = s.first + (wraps ? 0 : t0);
  o.last = s.first + (wraps ? s.tokens - 1 : t1);
  if (s.doc) {
    for (int r = r0 + (threadIdx.x & 31); r < r1; r += 32) {
      const int doc = s.doc[s.token(r)];
      if (doc >= 0) {
        o.doc_lo = min(o.doc_lo, doc);
        o.doc_hi = max(o.doc_hi, doc);
      }
    }
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) {
      o.doc_lo = min(o.doc_lo, __shfl_xor_sync(0xffffffffu, o.doc_lo, m));
      o.doc_hi = max(o.doc_hi, __shfl_xor_sync(0xffffffffu, o.doc_hi, m));
    }
  }
  return o;
}

// ---- rows with values that are not finite -------------------------------------------------

template <int D>
__device__ float dot_row(const float* x, const float* y) {
  float s = 0.f;
  for (int c = 0; c < D; c++) s += x[c] * y[c];
  return s;
}

// Pair (row r, key j) from global memory: false if masked.
template <int D>
__device__ bool slow_pair(const AttnArgs& a, const Unit& u, int r, int j, Score* out) {
  const int ti = u.q.token(r);
  if (!sees(a, u.prefix, u.q.first + ti, j, u.q.doc ? u.q.doc[ti] : 0, u.k.doc ? u.k.doc[j] : 0)) return false;
  const float slope2 = a.slopes ? a.slopes[u.kvh * (a.H / a.Hkv) + r / a.Gq] * kLog2e : 0.f;
  const float far = a.slopes ? fabsf(u.q.place(ti) - u.k.place(j)) : 0.f;
  *out = score_of(a, dot_row<D>(u.q.x0 + (int64_t)r * D, u.k.x0 + (int64_t)j * D), slope2, far);
  return true;
}

// One row's maximum, sum and unnormalised output over keys [j0, j1), visible pairs alone; lane c
// has channels c and c + 32.
template <int D>
__device__ __noinline__ void slow_row(const AttnArgs& a, int unit, int r, int j0, int j1, float* m_out,
                                      float* l_out, float (&o)[2]) {
  const Unit u = unit_of(a, unit, D);
  const int lane = threadIdx.x & 31;
  float m = -INFINITY, l = 0.f;
  Score s;
  for (int j = j0 + lane; j < j1; j += 32)
    if (slow_pair<D>(a, u, r, j, &s)) m = fmaxf(m, s.a);
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
  o[0] = o[1] = 0.f;
  const float base = m == -INFINITY ? 0.f : m;
  for (int jb = j0; jb < j1; jb += 32) {
    const int j = jb + lane;
    float p = 0.f;
    if (j < j1 && slow_pair<D>(a, u, r, j, &s)) p = exp2_fast(s.a - base);
    l += p;
    for (int i = 0; i < 32; i++) {
      const float w = __shfl_sync(0xffffffffu, p, i);
      if (w == 0.f) continue;  // masked, or of no weight
      const float* row = u.k.x1 + (int64_t)(jb + i) * D;
      if (lane < D) o[0] += w * row[lane];
      if (lane + 32 < D) o[1] += w * row[lane + 32];
    }
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
  *m_out = m;
  *l_out = l;
}

// A pair's weight and score gradient from global memory; zeros if masked.
template <int D>
__device__ void slow_grad(const AttnArgs& a, const Unit& u, int unit, int r, int j, float* p, float* ds) {
  Score s;
  *p = *ds = 0.f;
  if (!slow_pair<D>(a, u, r, j, &s)) return;
  const int64_t row = (int64_t)unit * a.rows + r;
  *p = exp2_fast(s.a - lse2_of(a.lse[row]));
  if (*p == 0.f) return;
  const float* g = u.q.x1 + (int64_t)r * D;
  const float delta = a.delta ? a.delta[row] : dot_row<D>(g, a.out + row * D);
  *ds = *p * (dot_row<D>(g, u.k.x1 + (int64_t)j * D) - delta) * s.slope;
}
// One own row's sums over streamed rows [s0, s1).
template <int D, bool kOwnKeys>
__device__ __noinline__ void slow_row_bwd(const AttnArgs& a, int unit, int own, int s0, int s1, float (&o0)[2],
                                          float (&o1)[2]) {
  const Unit u = unit_of(a, unit, D);
  const int lane = threadIdx.x & 31;
  o0[0] = o0[1] = o1[0] = o1[1] = 0.f;
  for (int sb = s0; sb < s1; sb += 32) {
    float p = 0.f, ds = 0.f;
    if (sb + lane < s1) slow_grad<D>(a, u, unit, kOwnKeys ? sb + lane : own, kOwnKeys ? own : sb + lane, &p, &ds);
    for (int i = 0; i < 32; i++) {
      const float wp = __shfl_sync(0xffffffffu, p, i), wd = __shfl_sync(0xffffffffu, ds, i);
      const Side& s = kOwnKeys ? u.q : u.k;
      const int64_t at = (int64_t)(sb + i) * D;
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int c = lane + 32 * h;
        if (c >= D) continue;
        if (wd != 0.f) o0[h] += wd * s.x0[at + c];
        if (kOwnKeys && wp != 0.f) o1[h] += wp * s.x1[at + c];
      }
    }
  }
}

// ---- joins ------------------------------------------------------------------------------------

// Joins the splits' rows in the order of the splits: a warp per row, or (kBlock: many splits) the
// four warps of a block, each a quarter of them.
template <int D, bool kBlock>
__global__ void __launch_bounds__(128) k_attn_join(const AttnArgs args) {
  constexpr int W = kBlock ? 4 : 1;
  __shared__ float part[4][66];
  AttnArgs a = args;
  grid_begin(a.part);
  const int64_t all = (int64_t)a.units * a.rows;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row = kBlock ? blockIdx.x : (int64_t)blockIdx.x * 4 + warp;
  if (row >= all) return;  // whole warps, and whole blocks where they synchronise
  const float2* stat = reinterpret_cast<const float2*>(a.part + (int64_t)a.splits * all * D) + row;
  float m = -INFINITY;
  for (int s = lane; s < a.splits; s += 32) m = fmaxf(m, stat[s * all].x);
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
  const float base = m == -INFINITY ? 0.f : m;
  const int per = (a.splits + W - 1) / W, s0 = kBlock ? warp * per : 0, s1 = min(a.splits, s0 + per);
  float l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll 8
  for (int s = s0; s < s1; s++) {
    const float2 st = stat[s * all];
    const float* o = a.part + (s * all + row) * D;
    const float x0 = lane < D ? o[lane] : 0.f, x1 = lane + 32 < D ? o[lane + 32] : 0.f;
    // A range in which nothing is visible has sum 0 and zeros; one with a NaN among its scores may
    // have no maximum either, but its sum is NaN and stays so.
    const float w = exp2_fast(st.x - base);
    l += st.y * w;
    o0 += x0 * w;
    o1 += x1 * w;
  }
  if constexpr (kBlock) {
    part[warp][lane] = o0;
    part[warp][lane + 32] = o1;
    if (lane == 0) part[warp][64] = l;
    __syncthreads();
    if (warp != 0) return;
    for (int w = 1; w < 4; w++) {
      o0 += part[w][lane];
      o1 += part[w][lane + 32];
      l += part[w][64];
    }
  }
  const float f = l == 0.f ? 0.f : 1.f / l;
  if (lane < D) a.out[row * D + lane] = o0 * f;
  if (lane + 32 < D) a.out[row * D + lane + 32] = o1 * f;
  if (lane == 0) a.lse[row] = (m + log2f(l)) * kLn2;
}
template <int D>
cudaError_t attn_join(const AttnArgs& a, cudaStream_t st) {
  const int64_t all = (int64_t)a.units * a.rows;
  return a.splits > 8 ? launch(k_attn_join<D, true>, dim3((unsigned)all), dim3(128), 0, st, a)
                      : launch(k_attn_join<D, false>, dim3((unsigned)((all + 3) / 4)), dim3(128), 0, st, a);
}

// Sums of the splits' partial gradients, in order, four values a thread: dq's where the keys
// were split, then dk's and dv's where the queries were.
__global__ void __launch_bounds__(256) k_attn_sum(const AttnArgs args, int64_t nq, int64_t nk) {
  AttnArgs a = args;
  grid_begin(a.part, a.part_kv);
  int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 4;
  const bool of_q = a.splits > 1 && i < nq;
  if (a.splits > 1 && !of_q) i -= nq;
  if (!of_q && (a.splits_kv == 1 || i >= 2 * nk)) return;
  const float* src = (of_q ? a.part : a.part_kv) + i;
  float* dst = of_q ? a.dq + i : (i < nk ? a.dk + i : a.dv + (i - nk));
  const int64_t step = of_q ? nq : 2 * nk;
  const int n = of_q ? a.splits : a.splits_kv;
  float4 s = *reinterpret_cast<const float4*>(src);
  for (int p = 1; p < n; p++) {
    const float4 w = *reinterpret_cast<const float4*>(src + p * step);
    s.x += w.x; s.y += w.y; s.z += w.z; s.w += w.w;
  }
  *reinterpret_cast<float4*>(dst) = s;
}

}  // namespace
}  // namespace fs
