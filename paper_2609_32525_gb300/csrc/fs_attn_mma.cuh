// Self-attention of the slice tokens, forward and backward, in fp32.
//
//   s = scale q.k;  c = cap tanh(s / cap) or s;  a = c - slope |pos_q - pos_k|;  masked: weight 0
//   lse_i = log sum_j exp(a_ij),  p = exp(a - lse),  out_i = sum_j p_ij v_j
//   D_i = dout_i . out_i;  ds_ij = p_ij (dout_i . v_j - D_i) (1 - (c/cap)^2) scale
//   dq_i = sum_j ds_ij k_j;  dk_j = sum_i ds_ij q_i;  dv_j = sum_i p_ij dout_i
//
// No score is written to memory.  A warp owns 16 rows (queries; for dk and dv keys) and streams
// the other side through shared memory in tiles of 64 (32 for d = 64), fetched one tile ahead
// by cp.async; the forward keeps a running maximum and sum per row.
//
// The products run on the tensor cores at fp32's accuracy: every fp32 operand is taken as the
// sum of two tf32 values, x = hi + lo with lo = x - hi exact and cut to tf32's 11 bits by the
// product, and x y = hi hi' + hi lo' + lo hi' with fp32 accumulation.  What is dropped is
// 2^-22 of a product.  (bf16 halves drop 2^-16, which the fp32 results of the library's other
// token operations do not allow; the tf32 exponent is fp32's, so no scale is needed.)
//
// Fragments are laid out so that nothing is ever transposed: the order of the contracted index
// is free as long as both operands use the same one.  In S = X Y^T the thread's lane t = lane
// % 4 takes channels 8t..8t+7 of both; the accumulator's columns 2t, 2t + 1 become the
// contracted index of the next product as they lie, with rows 2t, 2t + 1 of Y; and its output
// columns stand for channels 4g + m, so that a lane's results are 8 neighbouring channels.
// Rows of shared tiles have d + 4 words, which makes these reads free of conflicts (but for
// pairs in the first product at d = 16).
//
// Masked pairs get weight 0 by a selection, but 0 times an infinity or a NaN that a masked
// token may hold is NaN inside a product.  Sums over visible pairs alone are what is defined,
// so a row whose result is not finite is computed again by its warp, pair by pair (slow_*);
// with finite inputs that never happens.  Tokens without a document (masked for every row)
// are read as zeros.
//
// Few rows leave most of the machine idle: the streamed side is then split into ranges, each
// block writes a partial result, and a second kernel joins them in order.  No atomics: the
// same bits in every run.
//
// What bounds it: m16n8k8 tf32 runs at 302 TFLOP/s on this chip (a quarter of tcgen05's), so
// three products of parts at 100; the longest calls reached half of that, where the splitting of
// the streamed fragments and the scores take the issue slots (they run on tcgen05 now).  Short
// calls are latency: one query of 4 x 8 heads against 4096 keys takes 12 us in two
// launches, 29 before the chains of products took turns and the join loaded at once.
#pragma once

#include "fs_attn.cuh"

#include <type_traits>

namespace fs {
namespace {

constexpr int kMaxWarps = 4;
template <int D>
__host__ __device__ constexpr int tile_rows() { return D == 64 ? 32 : 64; }
template <int D>
__host__ __device__ constexpr int row_words() { return D + 4; }

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The three products of split operands go to two accumulators, lo += al bh + ah bl and hi += ah bh:
// the tensor core cuts its accumulator towards zero at every step, which drifts over a long chain,
// so the small terms have a chain of their own, and chains are short (product_cols adds a tile's to
// fp32 registers).  A warp issues in order and a product waits some 30 clocks for the one before it
// in its chain, so several chains take turns.

__device__ __forceinline__ void copy16(void* dst, const void* src, bool ok) {
  const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
  const int n = ok ? 16 : 0;  // the rest is filled with zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---- streamed tiles ------------------------------------------------------------------------

template <int D>
struct Tile {
  float y0[tile_rows<D>()][row_words<D>()];
  float y1[tile_rows<D>()][row_words<D>()];
  float pos[tile_rows<D>()];
  float lse[tile_rows<D>()], delta[tile_rows<D>()], slope[tile_rows<D>()];  // of streamed queries
  int doc[tile_rows<D>()], index[tile_rows<D>()];
};

// The first tile from `tile` on that may hold a visible pair; every warp finds the same.
template <int D, bool kKeys>
__device__ __forceinline__ int next_tile(const AttnArgs& a, const Side& s, const Own& o, int prefix, int tile,
                                         int end) {
  constexpr int TR = tile_rows<D>();
  for (; tile < end; tile++) {
    const int r0 = tile * TR, r1 = min(r0 + TR, s.n);
    if (a.causal) {
      if (kKeys) {  // streamed keys: the first of them may be past every own query
        if (r0 > o.last && r0 >= prefix) continue;
      } else {  // streamed queries: all of them may be before every own key
        const int t0 = s.token(r0), t1 = s.token(r1 - 1);
        const int last = s.first + (r1 - r0 > t1 - t0 + 1 ? s.tokens - 1 : t1);
        if (o.first > last && o.first >= prefix) continue;
      }
    }
    if (!s.doc) return tile;
    bool any = false;
    for (int r = r0 + (threadIdx.x & 31); r < r1; r += 32) {
      const int doc = s.doc[s.token(r)];
      any |= doc >= o.doc_lo && doc <= o.doc_hi;
    }
    if (__any_sync(0xffffffffu, any)) return tile;
  }
  return end;
}

template <int D, bool kKeys>
__device__ __forceinline__ void load_tile(Tile<D>& t, const AttnArgs& a, const Unit& u, int unit, int tile) {
  constexpr int TR = tile_rows<D>(), Q = D / 4;
  const Side& s = kKeys ? u.k : u.q;
  const int r0 = tile * TR;
  for (int i = threadIdx.x; i < TR * Q; i += blockDim.x) {
    const int r = i / Q, c = i % Q * 4, row = r0 + r;
    bool ok = row < s.n;
    if (s.doc && ok) ok = s.doc[s.token(row)] >= 0;
    const int64_t at = ok ? (int64_t)row * D + c : 0;
    copy16(&t.y0[r][c], s.x0 + at, ok);
    copy16(&t.y1[r][c], s.x1 + at, ok);
  }
  for (int r = threadIdx.x; r < TR; r += blockDim.x) {
    const int row = r0 + r;
    const bool ok = row < s.n;
    const int tok = ok ? s.token(row) : 0;
    t.index[r] = s.first + tok;
    if (a.slopes) t.pos[r] = ok ? s.place(tok) : 0.f;
    if (s.doc) t.doc[r] = ok ? max(s.doc[tok], -1) : -1;  // any negative number: not in use
    if (!kKeys) {
      t.lse[r] = ok ? lse2_of(a.lse[(int64_t)unit * a.rows + row]) : INFINITY;  // weight 0 past the last row
      if (a.delta) t.delta[r] = ok ? a.delta[(int64_t)unit * a.rows + row] : 0.f;
      if (a.slopes) t.slope[r] = ok ? a.slopes[u.kvh * (a.H / a.Hkv) + row / a.Gq] * kLog2e : 0.f;
    }
  }
}

// D_i = dout_i . out_i of a tile's queries where no kernel has made them (few tiles: a launch
// costs more than the loads), 8 lanes a row.
template <int D>
__device__ __forceinline__ void tile_delta(Tile<D>& t, const AttnArgs& a, const Unit& u, int unit, int tile) {
  constexpr int TR = tile_rows<D>();
  const int l = threadIdx.x & 7;
  for (int r = threadIdx.x >> 3; r < TR; r += blockDim.x >> 3) {
    const int row = tile * TR + r;
    float s = 0.f;
    if (tile * TR + (r & ~3) >= a.rows) {  // none of the warp's four rows
      if (l == 0) t.delta[r] = 0.f;
      continue;
    }
    if (row < a.rows) {
      const float* x = a.out + ((int64_t)unit * a.rows + row) * D;
      const float* y = a.dout + ((int64_t)unit * a.rows + row) * D;
#pragma unroll
      for (int c = 2 * l; c < D; c += 16) {
        const float2 v = *reinterpret_cast<const float2*>(x + c), w = *reinterpret_cast<const float2*>(y + c);
        s += v.x * w.x + v.y * w.y;
      }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (l == 0) t.delta[r] = s;
  }
}

// ---- fragments ------------------------------------------------------------------------------

// Channel of a lane's value: k-step s of the first product, and its output's first channel.
template <int D>
__device__ __forceinline__ int lane_channel(int s, int t) {
  constexpr int PER = D < 32 ? D / 4 : 8;  // neighbouring channels of a lane
  return 32 * (s / (PER / 2)) + PER * t + 2 * (s % (PER / 2));
}

// The 16 own rows of a warp as the first operand, split once (d <= 32) or when used.
template <int D>
struct OwnRows {
  static constexpr bool kOnce = D <= 32;
  float x[kOnce ? 1 : D / 8][4];
  uint32_t hi[kOnce ? D / 8 : 1][4], lo[kOnce ? D / 8 : 1][4];
  __device__ __forceinline__ void load(const float* rows, int r0, int n, int g, int t) {
#pragma unroll
    for (int s = 0; s < D / 8; s++) {
      const int c = lane_channel<D>(s, t);
      float2 v0 = make_float2(0.f, 0.f), v1 = v0;
      if (r0 + g < n) v0 = *reinterpret_cast<const float2*>(rows + (int64_t)(r0 + g) * D + c);
      if (r0 + g + 8 < n) v1 = *reinterpret_cast<const float2*>(rows + (int64_t)(r0 + g + 8) * D + c);
      const float f[4] = {v0.x, v1.x, v0.y, v1.y};
#pragma unroll
      for (int i = 0; i < 4; i++) {
        if constexpr (kOnce) {
          const Split w = split(f[i]);
          hi[s][i] = w.hi;
          lo[s][i] = w.lo;
        } else {
          x[s][i] = f[i];
        }
      }
    }
  }
  __device__ __forceinline__ void get(int s, uint32_t (&h)[4], uint32_t (&l)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if constexpr (kOnce) {
        h[i] = hi[s][i];
        l[i] = lo[s][i];
      } else {
        const Split w = split(x[s][i]);
        h[i] = w.hi;
        l[i] = w.lo;
      }
    }
  }
};

// c[n] (columns: tile rows base + 8n + ..) = X Y^T, two or four columns' chains taking turns
template <int D, int NT>
__device__ __forceinline__ void product_rows(float (&c)[NT][4], const OwnRows<D>& x,
                                             const float (*y)[row_words<D>()], int base, int g, int t) {
  constexpr int PER = D < 32 ? D / 4 : 8, GN = NT < 4 ? NT : 4;
#pragma unroll
  for (int n0 = 0; n0 < NT; n0 += GN) {
    float lo[GN][4];
#pragma unroll
    for (int n = 0; n < GN; n++)
#pragma unroll
      for (int i = 0; i < 4; i++) c[n0 + n][i] = lo[n][i] = 0.f;
#pragma unroll
    for (int blk = 0; blk < (D + 31) / 32; blk++) {
      float f[GN][PER];
#pragma unroll
      for (int n = 0; n < GN; n++)
#pragma unroll
        for (int i = 0; i < PER; i += 4)
          *reinterpret_cast<float4*>(f[n] + i) =
              *reinterpret_cast<const float4*>(&y[base + 8 * (n0 + n) + g][32 * blk + PER * t + i]);
#pragma unroll
      for (int s = 0; s < PER / 2; s++) {
        uint32_t h[4], l[4];
        x.get(blk * (PER / 2) + s, h, l);
        Split b0[GN], b1[GN];
#pragma unroll
        for (int n = 0; n < GN; n++) {
          b0[n] = split(f[n][2 * s]);
          b1[n] = split(f[n][2 * s + 1]);
        }
#pragma unroll
        for (int n = 0; n < GN; n++) mma(lo[n], l, b0[n].hi, b1[n].hi);
#pragma unroll
        for (int n = 0; n < GN; n++) mma(c[n0 + n], h, b0[n].hi, b1[n].hi);
#pragma unroll
        for (int n = 0; n < GN; n++) mma(lo[n], h, b0[n].lo, b1[n].lo);
      }
    }
#pragma unroll
    for (int n = 0; n < GN; n++)
#pragma unroll
      for (int i = 0; i < 4; i++) c[n0 + n][i] += lo[n][i];
  }
}

// acc = keep acc + P Y with P [16 x 8 NT] as product_rows leaves it
template <int D, int NT>
__device__ __forceinline__ void product_cols(float (&acc)[D / 8][4], const float (&keep)[2], const float (&p)[NT][4],
                                             const float (*y)[row_words<D>()], int base, int g, int t) {
  constexpr int V = D < 32 ? D / 8 : 4;  // neighbouring output columns m of a lane's read
#pragma unroll
  for (int blk = 0; blk < (D + 31) / 32; blk++) {
    float hi[V][4], lo[V][4];
#pragma unroll
    for (int m = 0; m < V; m++)
#pragma unroll
      for (int i = 0; i < 4; i++) hi[m][i] = lo[m][i] = 0.f;
#pragma unroll
    for (int n = 0; n < NT; n++) {
      uint32_t h[4], l[4];
      const float f[4] = {p[n][0], p[n][2], p[n][1], p[n][3]};
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const Split w = split(f[i]);
        h[i] = w.hi;
        l[i] = w.lo;
      }
      const float* y0 = y[base + 8 * n + 2 * t];
      const float* y1 = y[base + 8 * n + 2 * t + 1];
      float f0[V], f1[V];
      if constexpr (V == 4) {
        *reinterpret_cast<float4*>(f0) = *reinterpret_cast<const float4*>(y0 + 32 * blk + 4 * g);
        *reinterpret_cast<float4*>(f1) = *reinterpret_cast<const float4*>(y1 + 32 * blk + 4 * g);
      } else {
        *reinterpret_cast<float2*>(f0) = *reinterpret_cast<const float2*>(y0 + 2 * g);
        *reinterpret_cast<float2*>(f1) = *reinterpret_cast<const float2*>(y1 + 2 * g);
      }
      Split b0[V], b1[V];
#pragma unroll
      for (int m = 0; m < V; m++) {
        b0[m] = split(f0[m]);
        b1[m] = split(f1[m]);
      }
#pragma unroll
      for (int m = 0; m < V; m++) mma(lo[m], l, b0[m].hi, b1[m].hi);
#pragma unroll
      for (int m = 0; m < V; m++) mma(hi[m], h, b0[m].hi, b1[m].hi);
#pragma unroll
      for (int m = 0; m < V; m++) mma(lo[m], h, b0[m].lo, b1[m].lo);
    }
#pragma unroll
    for (int m = 0; m < V; m++)
#pragma unroll
      for (int i = 0; i < 4; i++)
        acc[blk * V + m][i] = acc[blk * V + m][i] * keep[i >> 1] + (hi[m][i] + lo[m][i]);
  }
}

// Writes a lane's results, channels 8t..8t+7 (d = 16: 4t..4t+3) of each 32, of rows g and g + 8.
template <int D>
__device__ __forceinline__ void store_rows(float* rows, int r0, int n, const float (&acc)[D / 8][4], float f0,
                                           float f1, bool skip0, bool skip1, int g, int t) {
  constexpr int V = D < 32 ? D / 8 : 4;
#pragma unroll
  for (int half = 0; half < 2; half++) {
    const int r = r0 + g + 8 * half;
    if (r >= n || (half ? skip1 : skip0)) continue;
    const float f = half ? f1 : f0;
#pragma unroll
    for (int blk = 0; blk < (D + 31) / 32; blk++)
#pragma unroll
      for (int j = 0; j < 2; j++) {  // accumulator column 2t + j: channels V (2t + j) + m
        float v[V];
#pragma unroll
        for (int m = 0; m < V; m++) v[m] = acc[blk * V + m][2 * half + j] * f;
        float* dst = rows + (int64_t)r * D + 32 * blk + V * (2 * t + j);
        if constexpr (V == 4) *reinterpret_cast<float4*>(dst) = *reinterpret_cast<float4*>(v);
        else *reinterpret_cast<float2*>(dst) = *reinterpret_cast<float2*>(v);
      }
  }
}

// Bit i: row i of the warp's 16 has a value that is not finite.
template <int D>
__device__ __forceinline__ uint32_t bad_rows(const float (&acc)[D / 8][4]) {
  bool b0 = false, b1 = false;
#pragma unroll
  for (int m = 0; m < D / 8; m++) {
    b0 |= !(fabsf(acc[m][0]) < INFINITY) || !(fabsf(acc[m][1]) < INFINITY);
    b1 |= !(fabsf(acc[m][2]) < INFINITY) || !(fabsf(acc[m][3]) < INFINITY);
  }
  uint32_t lo = __ballot_sync(0xffffffffu, b0), hi = __ballot_sync(0xffffffffu, b1), bad = 0;
#pragma unroll
  for (int g = 0; g < 8; g++) {
    if ((lo >> (4 * g)) & 15u) bad |= 1u << g;
    if ((hi >> (4 * g)) & 15u) bad |= 1u << (g + 8);
  }
  return bad;
}

// ---- scores ---------------------------------------------------------------------------------

// What a lane knows of its two own rows (g and g + 8), and which streamed rows they may see: keys
// below `limit` (own queries), or queries from `limit` on (own keys).
struct OwnPair {
  int limit[2], doc[2];
  float pos[2], slope2[2], lse2[2], delta[2];
};
template <bool kOwnKeys>
__device__ __forceinline__ OwnPair own_pair(const AttnArgs& a, const Unit& u, int unit, int r0, int g, bool backward) {
  const Side& s = kOwnKeys ? u.k : u.q;
  OwnPair o;
#pragma unroll
  for (int h = 0; h < 2; h++) {
    const int r = min(r0 + g + 8 * h, s.n - 1), tok = s.token(r), index = s.first + tok;
    if (kOwnKeys) o.limit[h] = a.causal && index >= u.prefix ? index : INT_MIN;
    else o.limit[h] = a.causal ? min(a.Gk, max(index + 1, u.prefix)) : a.Gk;
    // no streamed row has the document of an own row without one
    o.doc[h] = !s.doc ? 0 : s.doc[tok] >= 0 ? s.doc[tok] : INT_MIN;
    o.pos[h] = a.slopes ? s.place(tok) : 0.f;
    o.slope2[h] = !kOwnKeys && a.slopes ? a.slopes[u.kvh * (a.H / a.Hkv) + r / a.Gq] * kLog2e : 0.f;
    o.lse2[h] = o.delta[h] = 0.f;
    if (!kOwnKeys && backward) {
      o.lse2[h] = lse2_of(a.lse[(int64_t)unit * a.rows + r]);
      o.delta[h] = a.delta ? a.delta[(int64_t)unit * a.rows + r] : 0.f;
    }
  }
  return o;
}

enum Masks { kSeesAll, kByIndex, kByIndexAndDoc };

// The products c of a tile's rows from `base` on (the tile starts at k0) become base-2 scores
// (forward); or weights, and dp score gradients without the factor `scale`, which the sums get
// at the end.  Cap and bias are the kernel's, masks a tile's.
template <int D, int NT, bool kBwd, bool kOwnKeys, bool kCap, bool kBias, int kMask>
__device__ __forceinline__ void scores(const AttnArgs& a, const OwnPair& o, const Tile<D>& T, int k0, int base, int t,
                                       float (&c)[NT][4], float (&dp)[NT][4]) {
  const float f2 = kCap ? a.scale / a.cap : a.scale * kLog2e, cap2 = a.cap * kLog2e;
#pragma unroll
  for (int n = 0; n < NT; n++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int col = base + 8 * n + 2 * t + (i & 1), h = i >> 1;
      float x = c[n][i] * f2, keep = 1.f;
      if (kCap) {
        const float th = tanhf(x);
        x = th * cap2;
        keep = 1.f - th * th;
      }
      if (kBias) x -= (kOwnKeys ? T.slope[col] : o.slope2[h]) * fabsf(o.pos[h] - T.pos[col]);
      bool ok = true;
      if (kMask) ok = kOwnKeys ? T.index[col] >= o.limit[h] : k0 + col < o.limit[h];
      if (kMask == kByIndexAndDoc) ok = ok && T.doc[col] == o.doc[h];
      if (!kBwd) {
        c[n][i] = ok ? x : -INFINITY;
      } else {
        const float p = exp2_fast(x - (kOwnKeys ? T.lse[col] : o.lse2[h]));
        const float w = kCap ? p * keep : p;
        c[n][i] = ok ? p : 0.f;
        dp[n][i] = ok ? w * (dp[n][i] - (kOwnKeys ? T.delta[col] : o.delta[h])) : 0.f;
      }
    }
}
template <int D, int NT, bool kBwd, bool kOwnKeys, bool kCap, bool kBias>
__device__ __forceinline__ void scores_by_mask(const AttnArgs& a, const OwnPair& o, const Tile<D>& T, int k0, int base,
                                               int t, int mask, float (&c)[NT][4], float (&dp)[NT][4]) {
  if (mask == kSeesAll) scores<D, NT, kBwd, kOwnKeys, kCap, kBias, kSeesAll>(a, o, T, k0, base, t, c, dp);
  else if (mask == kByIndex) scores<D, NT, kBwd, kOwnKeys, kCap, kBias, kByIndex>(a, o, T, k0, base, t, c, dp);
  else scores<D, NT, kBwd, kOwnKeys, kCap, kBias, kByIndexAndDoc>(a, o, T, k0, base, t, c, dp);
}

// ---- forward --------------------------------------------------------------------------------

template <int D, bool kCap, bool kBias>
__global__ void __launch_bounds__(kMaxWarps * 32) k_attn_fwd(const __grid_constant__ AttnArgs args) {
  constexpr int TR = tile_rows<D>(), NT = TR / 8;
  __shared__ Tile<D> tiles[2];
  const AttnArgs& a = args;  // in the constant bank: no registers through the loops
  grid_begin();
  if (a.status && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.status = kDevOk;
  const int per = 16 * a.warps, blocks = (a.rows + per - 1) / per;
  const int unit = blockIdx.x / blocks, r_blk = (blockIdx.x - unit * blocks) * per, sp = blockIdx.y;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int r0 = r_blk + 16 * (threadIdx.x >> 5);
  const Unit u = unit_of(a, unit, D);
  const int ntiles = (a.Gk + TR - 1) / TR;
  const int tile0 = (int)((int64_t)ntiles * sp / a.splits), tile1 = (int)((int64_t)ntiles * (sp + 1) / a.splits);
  const Own own = own_range(a, u.q, r_blk, r_blk + per);
  OwnRows<D> x;
  x.load(u.q.x0, r0, a.rows, g, t);
  const OwnPair o = own_pair<false>(a, u, unit, r0, g, false);
  // the first key that some own query does not see
  const int seen_by_all = a.causal ? min(a.Gk, max(own.first + 1, u.prefix)) : a.Gk;
  float acc[D / 8][4];
#pragma unroll
  for (int m = 0; m < D / 8; m++)
#pragma unroll
    for (int i = 0; i < 4; i++) acc[m][i] = 0.f;
  float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};

  int tile = next_tile<D, true>(a, u.k, own, u.prefix, tile0, tile1), stage = 0;
  if (tile < tile1) load_tile<D, true>(tiles[0], a, u, unit, tile);
  copy_commit();
  while (tile < tile1) {
    const int nxt = next_tile<D, true>(a, u.k, own, u.prefix, tile + 1, tile1);
    if (nxt < tile1) load_tile<D, true>(tiles[stage ^ 1], a, u, unit, nxt);
    copy_commit();
    copy_wait<1>();
    __syncthreads();
    const Tile<D>& T = tiles[stage];
    const int k0 = tile * TR;
    float c[NT][4];
    product_rows<D, NT>(c, x, T.y0, 0, g, t);
    const int mask = u.k.doc ? kByIndexAndDoc : k0 + TR > seen_by_all ? kByIndex : kSeesAll;
    scores_by_mask<D, NT, false, false, kCap, kBias>(a, o, T, k0, 0, t, mask, c, c);
    float keep[2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
      float m = top[h];
#pragma unroll
      for (int n = 0; n < NT; n++) m = fmaxf(m, fmaxf(c[n][2 * h], c[n][2 * h + 1]));
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
      const float base = m == -INFINITY ? 0.f : m;  // a row that has seen nothing yet
      keep[h] = exp2_fast(top[h] - base);
      top[h] = m;
      float s = 0.f;
#pragma unroll
      for (int n = 0; n < NT; n++)
#pragma unroll
        for (int j = 0; j < 2; j++) {
          const float p = exp2_fast(c[n][2 * h + j] - base);
          c[n][2 * h + j] = p;
          s += p;
        }
      sum[h] = sum[h] * keep[h] + s;
    }
    product_cols<D, NT>(acc, keep, c, T.y1, 0, g, t);
    __syncthreads();
    tile = nxt;
    stage ^= 1;
  }
#pragma unroll
  for (int h = 0; h < 2; h++) {
    sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
    sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
  }
  const int64_t at = (int64_t)unit * a.rows;
  const int64_t all = (int64_t)a.units * a.rows;
  float* out = a.splits > 1 ? a.part + ((int64_t)sp * all + at) * D : a.out + at * D;
  float* stat = a.splits > 1 ? a.part + (int64_t)a.splits * all * D + ((int64_t)sp * all + at) * 2 : nullptr;
  uint32_t bad = bad_rows<D>(acc);
  float f[2];
#pragma unroll
  for (int h = 0; h < 2; h++) {
    f[h] = a.splits > 1 ? 1.f : (sum[h] == 0.f ? 0.f : 1.f / sum[h]);
    const int r = r0 + g + 8 * h;
    if (t == 0 && r < a.rows && !((bad >> (g + 8 * h)) & 1u)) {
      if (stat) {
        stat[2 * r] = top[h];
        stat[2 * r + 1] = sum[h];
      } else {
        a.lse[at + r] = (top[h] + log2f(sum[h])) * kLn2;
      }
    }
  }
  store_rows<D>(out, r0, a.rows, acc, f[0], f[1], (bad >> g) & 1u, (bad >> (g + 8)) & 1u, g, t);
  for (; bad; bad &= bad - 1) {
    const int r = r0 + __ffs(bad) - 1;
    if (r >= a.rows) break;
    float m, l, o[2];
    slow_row<D>(args, unit, r, tile0 * TR, min(tile1 * TR, a.Gk), &m, &l, o);
    const float w = stat ? 1.f : (l == 0.f ? 0.f : 1.f / l);
    if (lane < D) out[(int64_t)r * D + lane] = o[0] * w;
    if (lane + 32 < D) out[(int64_t)r * D + lane + 32] = o[1] * w;
    if (lane == 0) {
      if (stat) {
        stat[2 * r] = m;
        stat[2 * r + 1] = l;
      } else {
        a.lse[at + r] = (m + log2f(l)) * kLn2;
      }
    }
  }
}

// ---- backward -------------------------------------------------------------------------------

// D_i = dout_i . out_i, 8 lanes per row.
template <int D>
__global__ void __launch_bounds__(256) k_attn_delta(const AttnArgs args) {
  AttnArgs a = args;
  grid_begin(a.out, a.dout);
  if (a.status && blockIdx.x == 0 && threadIdx.x == 0) *a.status = kDevOk;
  const int64_t row = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 3;
  const int l = threadIdx.x & 7;
  const bool ok = row < (int64_t)a.units * a.rows;
  float s = 0.f;
  if (ok)
#pragma unroll
    for (int c = 0; c < D / 8; c += 2) {
      const int at = (c / 2) * 16 + 2 * l;
      const float2 x = *reinterpret_cast<const float2*>(a.out + row * D + at);
      const float2 y = *reinterpret_cast<const float2*>(a.dout + row * D + at);
      s += x.x * y.x + x.y * y.y;
    }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (ok && l == 0) a.delta[row] = s;
}

// kOwnKeys: a block owns keys, streams queries and makes dk, dv; else it owns queries and makes dq.
template <int D, bool kOwnKeys, bool kCap, bool kBias>
__device__ __forceinline__ void backward_block(const AttnArgs& args, const AttnArgs& a, Tile<D> (&tiles)[2], int block,
                                               int sp) {
  constexpr int TR = tile_rows<D>(), NT = D == 64 ? 2 : 4;  // 32 streamed rows at a time (16: registers)
  const int n_own = kOwnKeys ? a.Gk : a.rows, n_str = kOwnKeys ? a.rows : a.Gk;
  const int splits = kOwnKeys ? a.splits_kv : a.splits;
  const int per = 16 * a.warps, blocks = (n_own + per - 1) / per;
  const int unit = block / blocks, r_blk = (block - unit * blocks) * per;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int r0 = r_blk + 16 * (threadIdx.x >> 5);
  const Unit u = unit_of(a, unit, D);
  const Side& own_s = kOwnKeys ? u.k : u.q;
  const Side& str_s = kOwnKeys ? u.q : u.k;
  const int ntiles = (n_str + TR - 1) / TR;
  const int tile0 = (int)((int64_t)ntiles * sp / splits), tile1 = (int)((int64_t)ntiles * (sp + 1) / splits);
  const Own own = own_range(a, own_s, r_blk, r_blk + per);
  OwnRows<D> x0, x1;
  x0.load(own_s.x0, r0, n_own, g, t);
  x1.load(own_s.x1, r0, n_own, g, t);
  OwnPair o = own_pair<kOwnKeys>(a, u, unit, r0, g, true);
  if (!kOwnKeys && !a.delta) {  // a lane has its rows' channels of one k-step of four
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int64_t at = ((int64_t)unit * a.rows + min(r0 + g + 8 * h, n_own - 1)) * D;
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < D / 8; k++) {
        const int c = lane_channel<D>(k, t);
        const float2 v = *reinterpret_cast<const float2*>(a.out + at + c);
        const float2 w = *reinterpret_cast<const float2*>(a.dout + at + c);
        s += v.x * w.x + v.y * w.y;
      }
      s += __shfl_xor_sync(0xffffffffu, s, 1);
      s += __shfl_xor_sync(0xffffffffu, s, 2);
      o.delta[h] = s;
    }
  }
  const int seen_by_all = a.causal ? min(a.Gk, max(own.first + 1, u.prefix)) : a.Gk;
  float acc0[D / 8][4], acc1[kOwnKeys ? D / 8 : 1][4];
#pragma unroll
  for (int m = 0; m < D / 8; m++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      acc0[m][i] = 0.f;
      if (kOwnKeys) acc1[m][i] = 0.f;
    }

  int tile = next_tile<D, !kOwnKeys>(a, str_s, own, u.prefix, tile0, tile1), stage = 0;
  if (tile < tile1) load_tile<D, !kOwnKeys>(tiles[0], a, u, unit, tile);
  copy_commit();
  if (kOwnKeys && !a.delta && tile < tile1) tile_delta<D>(tiles[0], a, u, unit, tile);
  while (tile < tile1) {
    const int nxt = next_tile<D, !kOwnKeys>(a, str_s, own, u.prefix, tile + 1, tile1);
    if (nxt < tile1) load_tile<D, !kOwnKeys>(tiles[stage ^ 1], a, u, unit, nxt);
    copy_commit();
    if (kOwnKeys && !a.delta && nxt < tile1) tile_delta<D>(tiles[stage ^ 1], a, u, unit, nxt);
    copy_wait<1>();
    __syncthreads();
    const Tile<D>& T = tiles[stage];
    const int k0 = tile * TR;
    int mask = kSeesAll;
    if (str_s.doc) {
      mask = kByIndexAndDoc;
    } else if (!kOwnKeys) {
      if (k0 + TR > seen_by_all) mask = kByIndex;
    } else if (a.causal && own.last >= u.prefix) {  // some query of the tile may be before some own key
      const int s1 = min(k0 + TR, n_str), last = u.q.token(s1 - 1), first = u.q.token(k0);
      if (u.q.first + (s1 - k0 > last - first + 1 ? 0 : first) < own.last) mask = kByIndex;
    }
#pragma unroll 1
    for (int base = 0; base < TR; base += 8 * NT) {
      float c[NT][4], dp[NT][4];
      product_rows<D, NT>(c, x0, T.y0, base, g, t);
      product_rows<D, NT>(dp, x1, T.y1, base, g, t);
      scores_by_mask<D, NT, true, kOwnKeys, kCap, kBias>(a, o, T, k0, base, t, mask, c, dp);
      constexpr float kOne[2] = {1.f, 1.f};
      product_cols<D, NT>(acc0, kOne, dp, T.y0, base, g, t);
      if constexpr (kOwnKeys) product_cols<D, NT>(acc1, kOne, c, T.y1, base, g, t);
    }
    __syncthreads();
    tile = nxt;
    stage ^= 1;
  }
  const int64_t at = (int64_t)unit * n_own * D, all = (int64_t)a.units * n_own * D;
  float* out0;
  float* out1 = nullptr;
  if constexpr (kOwnKeys) {
    out0 = (splits > 1 ? a.part_kv + (int64_t)sp * 2 * all : a.dk) + at;
    out1 = (splits > 1 ? a.part_kv + ((int64_t)sp * 2 + 1) * all : a.dv) + at;
  } else {
    out0 = (splits > 1 ? a.part + (int64_t)sp * all : a.dq) + at;
  }
  uint32_t bad = bad_rows<D>(acc0);
  if constexpr (kOwnKeys) bad |= bad_rows<D>(acc1);
  store_rows<D>(out0, r0, n_own, acc0, a.scale, a.scale, (bad >> g) & 1u, (bad >> (g + 8)) & 1u, g, t);
  if constexpr (kOwnKeys)
    store_rows<D>(out1, r0, n_own, acc1, 1.f, 1.f, (bad >> g) & 1u, (bad >> (g + 8)) & 1u, g, t);
  for (; bad; bad &= bad - 1) {
    const int r = r0 + __ffs(bad) - 1;
    if (r >= n_own) break;
    float o0[2], o1[2];
    slow_row_bwd<D, kOwnKeys>(args, unit, r, tile0 * TR, min(tile1 * TR, n_str), o0, o1);
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int c = lane + 32 * h;
      if (c >= D) continue;
      out0[(int64_t)r * D + c] = o0[h];
      if (kOwnKeys) out1[(int64_t)r * D + c] = o1[h];
    }
  }
}

// The blocks that make dk and dv come first: they have four products a pair, those of dq three.
template <int D, bool kCap, bool kBias>
__global__ void __launch_bounds__(kMaxWarps * 32) k_attn_bwd(const __grid_constant__ AttnArgs args, int blocks_kv) {
  __shared__ Tile<D> tiles[2];
  const AttnArgs& a = args;
  grid_begin();
  if (!a.delta && blockIdx.x == 0 && threadIdx.x == 0) *a.status = kDevOk;
  const int b = blockIdx.x;
  if (b < blocks_kv * a.splits_kv) backward_block<D, true, kCap, kBias>(args, a, tiles, b / a.splits_kv, b % a.splits_kv);
  else {
    const int c = b - blocks_kv * a.splits_kv;
    backward_block<D, false, kCap, kBias>(args, a, tiles, c / a.splits, c % a.splits);
  }
}

template <int D, bool kCap, bool kBias>
cudaError_t fwd_of(const AttnArgs& a, cudaStream_t st) {
  const int per = 16 * a.warps;
  const dim3 grid((unsigned)(a.units * ((a.rows + per - 1) / per)), (unsigned)a.splits);
  cudaError_t e = launch(k_attn_fwd<D, kCap, kBias>, grid, dim3(32 * a.warps), 0, st, a);
  if (e == cudaSuccess && a.splits > 1)
    e = attn_join<D>(a, st);
  return e;
}

template <int D, bool kCap, bool kBias>
cudaError_t bwd_of(const AttnArgs& a, cudaStream_t st) {
  const int per = 16 * a.warps;
  const int64_t blocks_q = (int64_t)a.units * ((a.rows + per - 1) / per);
  const int64_t blocks_kv = (int64_t)a.units * ((a.Gk + per - 1) / per);
  const int64_t nrows = (int64_t)a.units * a.rows;
  cudaError_t e = cudaSuccess;
  if (a.delta) e = launch(k_attn_delta<D>, dim3((unsigned)((nrows + 31) / 32)), dim3(256), 0, st, a);
  if (e != cudaSuccess) return e;
  e = launch(k_attn_bwd<D, kCap, kBias>, dim3((unsigned)(blocks_q * a.splits + blocks_kv * a.splits_kv)), dim3(32 * a.warps), 0, st,
             a, (int)blocks_kv);
  if (e != cudaSuccess || (a.splits == 1 && a.splits_kv == 1)) return e;
  const int64_t nq = nrows * D, nk = (int64_t)a.units * a.Gk * D;
  const int64_t n = (a.splits > 1 ? nq : 0) + (a.splits_kv > 1 ? 2 * nk : 0);
  return launch(k_attn_sum, dim3((unsigned)((n / 4 + 255) / 256)), dim3(256), 0, st, a, nq, nk);
}

template <int D, typename F>
cudaError_t by_features(const AttnArgs& a, F f) {
  if (a.cap > 0.f) return a.slopes ? f(std::true_type(), std::true_type()) : f(std::true_type(), std::false_type());
  return a.slopes ? f(std::false_type(), std::true_type()) : f(std::false_type(), std::false_type());
}

}  // namespace

template <int D>
cudaError_t attn_mma_fwd(const AttnArgs& a, cudaStream_t st) {
  return by_features<D>(a, [&](auto cap, auto bias) { return fwd_of<D, decltype(cap)::value, decltype(bias)::value>(a, st); });
}
template <int D>
cudaError_t attn_mma_bwd(const AttnArgs& a, cudaStream_t st) {
  return by_features<D>(a, [&](auto cap, auto bias) { return bwd_of<D, decltype(cap)::value, decltype(bias)::value>(a, st); });
}

}  // namespace fs
