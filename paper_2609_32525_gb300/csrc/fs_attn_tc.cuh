// Self-attention of the slice tokens on tcgen05: the same results as fs_attn_mma.cuh's kernels, for
// calls with enough rows to fill tiles of 128.
//
// A block owns 128 rows (queries; for dk and dv keys) and streams the other side in tiles.  Own
// rows lie in TMEM as the first operand, split into tf32 parts; the streamed side comes as
// images that one preparation kernel lays out per call, rows in panels of 32 channels and their
// transposes, both parts, in the 128-byte swizzle, so that plain bulk copies bring them and
// every operand is K-major.  (d = 16 has images of 32 channels, half of them zeros that its
// scores' products leave out: products 16 wide take as long as 32.)  Per tile
//
//   S = X0 Y0^T (and dP = X1 Y1^T)   first operand TMEM, 3 products of parts, into TMEM
//   weights (and score gradients)    a warpgroup, one own row per thread, registers
//   parts of them back into TMEM     in place of S and dP
//   acc = P Y^T (and dS Y^T)         first operand TMEM
//
// and each thread adds its row of acc to fp32 registers: the tensor core cuts its accumulator
// towards zero at every step, and one tile is as long as a chain may get (within it the small
// products come first).
//
// Two pairs of warpgroups take alternate tiles, each pair with its own TMEM buffers and its own
// issuing warp, so that one's products run under the other's exponentials; the warpgroups of a
// pair share a tile's columns.  In the forward up to d = 32 each of them is a stream of its own, with
// its maximum, sum and products, so that they need not agree on a maximum.  (With one warpgroup per
// pair the kernels waited on latency: 21% of the tensor rate, 24% of the issue slots.)  First
// operands in TMEM are what lets products 32 columns wide run at the tensor rate: from shared
// memory the 128 own rows would be read again for each of them, 4 KB against 1 KB of the tile's.
//
// d = 64: the own rows' parts take 128 columns of TMEM a tensor and an accumulator 64.  So a pair's
// warpgroups share the forward's accumulator and exchange their rows' maxima, and dk and dv, for
// which TMEM would hold one pair only, are made by blocks of their own: one more product a pair,
// and every kind of block has its two pairs.
//
// Warps: 0 loads, 1 and 2 issue, 4 to 19 are the four warpgroups.
#pragma once

#include "fs_attn.cuh"
#include "fs_attn_tc.h"
#include "fs_tc_ptx.cuh"

#include <algorithm>

namespace fs {
namespace {

using namespace tc;

constexpr int kThreads = 640, kOwn = 128;
constexpr int kListMost = kAttnTcTiles;  // tiles of one block's range
constexpr size_t kMostSmem = 232448;

enum Mode { kFwd, kDq, kDkv, kDk, kDv };  // dk and dv together up to d = 32
__host__ __device__ constexpr bool own_is_keys(Mode m) { return m == kDkv || m == kDk || m == kDv; }
__host__ __device__ constexpr bool has_dp(Mode m) { return m == kDq || m == kDkv || m == kDk; }
constexpr int width_of(int D) { return D < 32 ? 32 : D; }  // channels of an image

// ---- images ------------------------------------------------------------------------------------

// Row image: panels of 32 channels, rows of 128 bytes; column image: per 32 rows a block of a row
// of 128 bytes for each channel.  Both 128-byte swizzled, 4 KB per 32 rows and channels.
__device__ __forceinline__ uint32_t image_at(int row, int col4) {  // 16-byte piece col4 of a row
  return (uint32_t)(row * 128 + ((col4 ^ (row & 7)) << 4));
}

template <int D>
__global__ void __launch_bounds__(256) k_attn_prep(const __grid_constant__ AttnTcArgs args) {
  __shared__ float tile[32][33];
  __shared__ float dot[32];
  const int64_t zero = grid_begin();
  const AttnArgs& a = args.a;
  const int job = blockIdx.y, tid = threadIdx.x + (int)zero;
  const bool of_q = job >= 2;  // jobs: k, v, q, dout
  if (job == 0 && blockIdx.x == 0 && tid == 0) *a.status = kDevOk;
  const int n = of_q ? a.rows : a.Gk, pad = of_q ? args.rows_pad : args.k_pad, atoms = pad / 32;
  const int unit = blockIdx.x / atoms, atom = blockIdx.x - unit * atoms;
  if (unit >= a.units) return;
  const float* src = (job == 0 ? a.k : job == 1 ? a.v : job == 2 ? a.q : a.dout) + (int64_t)unit * n * D;
  const int b = unit / a.Hkv, tokens = of_q ? a.Gq : a.Gk;
  const int* docs = of_q ? (a.doc_q ? a.doc_q + (int64_t)b * a.Gq : nullptr)
                         : (a.doc_k ? a.doc_k + (int64_t)b * a.Gk : nullptr);
  const int r = tid >> 3, c4 = tid & 7, row = atom * 32 + r;
  bool ok = row < n;
  if (ok && docs) ok = docs[row % tokens] >= 0;  // tokens that nothing sees are zeros
  constexpr int W = width_of(D);
  uint8_t* rows_hi = args.row_img[job];
  uint8_t* cols_hi = args.col_img[job];
  const size_t lo_off = (size_t)a.units * pad * (4 * W);
  float s = 0.f;  // D = dout . out
#pragma unroll
  for (int p = 0; p < W / 32; p++) {
    const int c = 32 * p + 4 * c4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (ok && c < D) v = *reinterpret_cast<const float4*>(src + (int64_t)row * D + c);
    if (rows_hi) {
      const Split s0 = split(v.x), s1 = split(v.y), s2 = split(v.z), s3 = split(v.w);
      const size_t at = ((size_t)(unit * (W / 32) + p) * pad + atom * 32) * 128 + image_at(r, c4);
      *reinterpret_cast<uint4*>(rows_hi + at) = make_uint4(s0.hi, s1.hi, s2.hi, s3.hi);
      *reinterpret_cast<uint4*>(rows_hi + lo_off + at) = make_uint4(s0.lo, s1.lo, s2.lo, s3.lo);
    }
    if (cols_hi) {
      if (p > 0) __syncthreads();
      tile[r][4 * c4] = v.x; tile[r][4 * c4 + 1] = v.y; tile[r][4 * c4 + 2] = v.z; tile[r][4 * c4 + 3] = v.w;
      __syncthreads();
      const Split s0 = split(tile[4 * c4][r]), s1 = split(tile[4 * c4 + 1][r]), s2 = split(tile[4 * c4 + 2][r]),
                  s3 = split(tile[4 * c4 + 3][r]);
      // channel 32 p + r, rows 4 c4 ..
      const size_t at = ((size_t)unit * pad + atom * 32) * (4 * W) + p * 4096 + image_at(r, c4);
      *reinterpret_cast<uint4*>(cols_hi + at) = make_uint4(s0.hi, s1.hi, s2.hi, s3.hi);
      *reinterpret_cast<uint4*>(cols_hi + lo_off + at) = make_uint4(s0.lo, s1.lo, s2.lo, s3.lo);
    }
    if (job == 3 && ok && c < D) {
      const float4 o = *reinterpret_cast<const float4*>(a.out + ((int64_t)unit * n + row) * D + c);
      s += v.x * o.x + v.y * o.y + v.z * o.z + v.w * o.w;
    }
  }
  if (job == 3) {
#pragma unroll
    for (int m = 4; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
    if (c4 == 0) dot[r] = s;
    __syncthreads();
  }
  if (tid >= 32 || (job != 0 && job != 3) || (job == 0 && unit % a.Hkv != 0)) return;
  const int mine = atom * 32 + tid, tok = mine % tokens;
  const bool in = mine < n;
  const int doc = docs && in ? max(docs[tok], -1) : -1;  // any negative number: not in use
  int lo = doc >= 0 ? doc : INT_MAX, hi = doc;
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) {
    lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, m));
    hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, m));
  }
  if (job == 0) {
    const int64_t at = (int64_t)b * pad + mine;
    if (a.slopes) args.k_pos[at] = !in ? 0.f : a.pos_k ? a.pos_k[(int64_t)b * a.Gk + tok] : (float)tok;
    if (docs) {
      args.k_doc[at] = doc;
      if (tid == 0) args.k_range[(int64_t)b * atoms + atom] = make_int2(lo, hi);
    }
    return;
  }
  const int64_t at = (int64_t)unit * pad + mine, all = (int64_t)a.units * pad;
  const int first = a.Gk - a.Gq, h = (unit % a.Hkv) * (a.H / a.Hkv) + (in ? mine / a.Gq : 0);
  args.q_info[at] = in ? -lse2_of(a.lse[(int64_t)unit * n + mine]) : -INFINITY;  // weight 0 past the last row
  args.q_info[all + at] = in ? -dot[tid] : 0.f;
  if (in) a.delta[(int64_t)unit * n + mine] = dot[tid];
  if (a.slopes) {
    args.q_info[2 * all + at] = in ? a.slopes[h] * kLog2e : 0.f;
    args.q_info[3 * all + at] = !in ? 0.f : a.pos_q ? a.pos_q[(int64_t)b * a.Gq + tok] : (float)(first + tok);
  }
  if (docs) {
    args.q_tok[at] = doc;
    if (tid == 0) args.q_range[(int64_t)unit * atoms + atom] = make_int2(lo, hi);
  }
  if (a.causal || docs) args.q_tok[all + at] = first + tok;
}

// ---- tensor-core pieces -------------------------------------------------------------------------

constexpr uint32_t kHiWord = sdesc_hi(1024, kSw128);
constexpr uint32_t idesc_tf32(int N) {
  return (1u << 4) | (2u << 7) | (2u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(kOwn >> 4) << 24);
}
// D (+)= A B^T with A in TMEM (tf32), one lane of a converged warp issues.
__device__ __forceinline__ void mma_tf32(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, e;\n .reg .b64 b;\n mov.b64 b, {%2, %3};\n"
      " setp.ne.b32 p, %5, 0;\n elect.sync _|e, 0xffffffff;\n"
      " @e tcgen05.mma.cta_group::1.kind::tf32 [%0], [%1], b, %4, p;\n}\n" ::"r"(d),
      "r"(a), "r"(b_lo), "n"(kHiWord), "r"(idesc), "r"(accumulate)
      : "memory");
}
// d = X Y^T over D channels: X's parts in TMEM, Y's N rows in shared memory, panel by panel.
template <int N, int D>
__device__ __forceinline__ void issue_rows(uint32_t d, uint32_t x_hi, uint32_t x_lo, uint32_t y_hi, uint32_t y_lo) {
  constexpr uint32_t id = idesc_tf32(N);
#pragma unroll
  for (int k = 0; k < D / 8; k++) {
    const uint32_t at = (k >> 2) * (N * 8) + (k & 3) * 2;
    mma_tf32(d, x_lo + 8 * k, y_hi + at, id, k > 0);
    mma_tf32(d, x_hi + 8 * k, y_lo + at, id, 1);
  }
#pragma unroll
  for (int k = 0; k < D / 8; k++) mma_tf32(d, x_hi + 8 * k, y_hi + (k >> 2) * (N * 8) + (k & 3) * 2, id, 1);
}
// d = X Y_hi^T's large products, d + 32 = the small ones, for 32 streamed rows.
template <int D>
__device__ __forceinline__ void issue_rows_split(uint32_t d, uint32_t x_hi, uint32_t x_lo, uint32_t y) {
#pragma unroll
  for (int k = 0; k < D / 8; k++) mma_tf32(d, x_hi + 8 * k, y + 2 * k, idesc_tf32(64), k > 0);
#pragma unroll
  for (int k = 0; k < D / 8; k++) mma_tf32(d + 32, x_lo + 8 * k, y + 2 * k, idesc_tf32(32), 1);
}
// d = P Y over TN streamed rows, W channels: P's parts in TMEM, Y's column image in shared memory.
template <int TN, int W>
__device__ __forceinline__ void issue_cols(uint32_t d, uint32_t p_hi, uint32_t p_lo, uint32_t y_hi, uint32_t y_lo) {
  constexpr uint32_t id = idesc_tf32(W);
#pragma unroll
  for (int k = 0; k < TN / 8; k++) {
    const uint32_t at = (k >> 2) * (W * 8) + (k & 3) * 2;
    mma_tf32(d, p_lo + 8 * k, y_hi + at, id, k > 0);
    mma_tf32(d, p_hi + 8 * k, y_lo + at, id, 1);
  }
#pragma unroll
  for (int k = 0; k < TN / 8; k++) mma_tf32(d, p_hi + 8 * k, y_hi + (k >> 2) * (W * 8) + (k & 3) * 2, id, 1);
}

// Columns of a pair's TMEM: S, dP (written over by parts of the weights and score gradients),
// low parts, accumulators; the own rows' parts before both pairs.  For dk and dv the products of S
// and dP are in two chains, x_hi (y_hi, y_lo) with both parts of the tile as one operand of 64
// rows, and x_lo y_hi: 8 products where one chain takes 12 of the same length (a product 32
// columns wide takes as long as one of 64).  Their low halves lie where low parts go later.  (d = 64
// has no room for the second chain; its tiles with two score products are 32 rows, so that both
// pairs fit: 128 columns each.)
template <Mode M, int D>
struct Map {
  static constexpr int W = width_of(D);
  static constexpr bool WIDE = D == 64;
  static constexpr int TN = M == kDkv || (WIDE && has_dp(M)) ? 32 : 64;
  static constexpr int ROWS = has_dp(M) ? 2 : 1, COLS = M == kDkv ? 2 : 1;  // images of a stage
  static constexpr uint32_t IMG = TN * 4 * W;                              // bytes of one part
  static constexpr uint32_t INFO = (ROWS + COLS) * 2 * IMG, STAGE = INFO + (M == kDv ? 2048 : 1024);
  static constexpr int ST = WIDE ? (TN == 64 ? 3 : 4) : M == kFwd ? 6 : 4;
  static constexpr uint32_t X0 = 0, X1 = 2 * W, PAIR = WIDE && !has_dp(M) ? 128 : 4 * W;
  static constexpr uint32_t PAIR_COLS = WIDE && has_dp(M) ? 128 : 192;
  static constexpr uint32_t S = 0, DP = TN == 32 && WIDE ? 32 : 64, PLO = M == kDkv ? 32 : 64, DSLO = 96;
  static constexpr uint32_t ACC0 = TN == 32 && WIDE ? 64 : 128, ACC1 = 160;
  // A thread's share of its row's results: the forward's stream (all channels, half of the
  // keys), half of dq's channels, or dk (half 0) or dv (half 1); d = 64: half of the channels.
  static constexpr int NA = M == kDq && !WIDE ? 16 : 32;
  static constexpr bool SHARED = M == kFwd && WIDE;  // the pair's warpgroups share a maximum
  static constexpr size_t SMEM = (size_t)ST * STAGE + 1024 + kListMost * 4 + 512 + (SHARED ? 2048 : 0);
  static_assert(SMEM <= kMostSmem && PAIR + 2 * PAIR_COLS <= 512, "");
};

__device__ __forceinline__ uint64_t both(float x) { return pack2(__float_as_uint(x), __float_as_uint(x)); }
// Parts of N values into N columns each.  (A high part that is cut instead of rounded is an
// operation less, but leaves a low part that loses twice as much to tf32: dq's error grew from
// 7e-7 to 1e-6, at no gain in time.)
template <int N>
__device__ __forceinline__ void store_parts(uint32_t hi_at, uint32_t lo_at, const uint32_t (&p)[N]) {
#pragma unroll
  for (int j = 0; j < N; j += 16) {
    uint32_t h[16], l[16];
#pragma unroll
    for (int i = 0; i < 16; i++) h[i] = tf32_hi(__uint_as_float(p[j + i]));
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const uint64_t lo = fma2(pack2(h[i], h[i + 1]), both(-1.f), pack2(p[j + i], p[j + i + 1]));
      l[i] = (uint32_t)lo;
      l[i + 1] = (uint32_t)(lo >> 32);
    }
    tmem_st16(hi_at + j, h);
    tmem_st16(lo_at + j, l);
  }
}

// What a thread knows of its own row, and which streamed rows it may see: keys below `limit`
// (own queries), or queries from `limit` on (own keys).  The statistic and D are negated.
struct Row {
  int limit, doc;
  float pos, slope2, nlse2, ndelta;
};

// Of a stage's streamed rows, by column.
template <Mode M, int TN>
struct Info {
  const float *nlse2, *ndelta, *slope2, *pos;
  const int *doc, *index;
  __device__ __forceinline__ explicit Info(const uint8_t* p) {
    const float* f = reinterpret_cast<const float*>(p);
    if (own_is_keys(M)) {
      nlse2 = f; ndelta = f + TN; slope2 = f + 2 * TN; pos = f + 3 * TN;
      doc = reinterpret_cast<const int*>(f + 4 * TN);
      index = reinterpret_cast<const int*>(f + 5 * TN);
    } else {
      nlse2 = ndelta = slope2 = nullptr;
      index = nullptr;
      pos = f;
      doc = reinterpret_cast<const int*>(f + TN);
    }
  }
};

// What a tile's scores need, so that each tile runs code without the rest: per pair, each test
// of a feature at run time cost as much as the feature (a forward with a bias at 1024 tokens
// took 57 us with the tests inside).
enum Masks { kSeesAll, kByIndex, kByIndexAndDoc };

// Four neighbouring columns' entries of an info array.
template <typename T>
__device__ __forceinline__ void four(T (&v)[4], const T* p) {
  const float4 f = *reinterpret_cast<const float4*>(p);
  memcpy(v, &f, sizeof(f));
}

// The factor that takes the forward's scores, as columns() leaves them, to base-2 units.
template <bool kCap, bool kBias>
__device__ __forceinline__ float score_unit(const AttnArgs& a) {
  return kCap || kBias || !(a.scale > 0.f) ? 1.f : a.scale * kLog2e;
}

// N columns from j0 on of a tile at k0, as the bits of fp32.  Forward: the products in s become
// scores in score_unit()s.  Backward: s becomes the weights, and dP in d the score gradients
// without their factor `scale`, which the sums get at the end (dv's blocks have no dP).
template <Mode M, int TN, int N, bool kCap, bool kBias, int kMask>
__device__ __forceinline__ void columns(const AttnArgs& a, const Row& o, const Info<M, TN>& f, int k0, int j0,
                                        uint32_t (&s)[N], uint32_t (&d)[N]) {
  const float f2 = kCap ? a.scale / a.cap : a.scale * kLog2e, cap2 = a.cap * kLog2e;
  const bool unit = M == kFwd && !kCap && !kBias && a.scale > 0.f;
#pragma unroll
  for (int q = 0; q < N; q += 4) {
    float nlse2[4], ndelta[4], slope2[4], pos[4];
    int doc[4], index[4];
    if (own_is_keys(M)) {
      four(nlse2, f.nlse2 + j0 + q);
      if (has_dp(M)) four(ndelta, f.ndelta + j0 + q);
      if (kBias) four(slope2, f.slope2 + j0 + q);
      if (kMask) four(index, f.index + j0 + q);
    }
    if (kBias) four(pos, f.pos + j0 + q);
    if (kMask == kByIndexAndDoc) four(doc, f.doc + j0 + q);
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      const int j = q + e;
      uint64_t x = pack2(s[j], s[j + 1]), keep = 0;  // keep: 1 - (c / cap)^2
      if (kCap) {
        const uint64_t y = mul2(x, both(f2));
        const float t0 = tanhf(lo_f(y)), t1 = tanhf(hi_f(y));
        const uint64_t t = pack2(__float_as_uint(t0), __float_as_uint(t1));
        x = mul2(t, both(cap2));
        keep = fma2(mul2(t, both(-1.f)), t, both(1.f));
      }
      uint64_t shift = 0;  // minus the bias, minus the statistic
      if (M != kFwd) {
        shift = own_is_keys(M) ? pack2(__float_as_uint(nlse2[e]), __float_as_uint(nlse2[e + 1])) : both(o.nlse2);
      }
      if (kBias) {
        const float b0 = -(own_is_keys(M) ? slope2[e] : o.slope2) * fabsf(o.pos - pos[e]);
        const float b1 = -(own_is_keys(M) ? slope2[e + 1] : o.slope2) * fabsf(o.pos - pos[e + 1]);
        const uint64_t b = pack2(__float_as_uint(b0), __float_as_uint(b1));
        shift = M == kFwd ? b : add2(shift, b);
      }
      if (kCap) {
        if (M != kFwd || kBias) x = add2(x, shift);
      } else if (M != kFwd || kBias) {
        x = fma2(x, both(f2), shift);
      } else if (!unit) {
        x = mul2(x, both(f2));
      }
      bool ok0 = true, ok1 = true;
      if (kMask) {
        ok0 = own_is_keys(M) ? index[e] >= o.limit : k0 + j0 + j < o.limit;
        ok1 = own_is_keys(M) ? index[e + 1] >= o.limit : k0 + j0 + j + 1 < o.limit;
      }
      if (kMask == kByIndexAndDoc) {
        ok0 = ok0 && doc[e] == o.doc;
        ok1 = ok1 && doc[e + 1] == o.doc;
      }
      if (M == kFwd) {
        s[j] = ok0 ? (uint32_t)x : 0xff800000u;  // -infinity
        s[j + 1] = ok1 ? (uint32_t)(x >> 32) : 0xff800000u;
      } else {
        const uint32_t p0 = __float_as_uint(ex2(lo_f(x))), p1 = __float_as_uint(ex2(hi_f(x)));
        if (has_dp(M)) {
          const uint64_t nd = own_is_keys(M) ? pack2(__float_as_uint(ndelta[e]), __float_as_uint(ndelta[e + 1])) : both(o.ndelta);
          uint64_t w = pack2(p0, p1);
          if (kCap) w = mul2(w, keep);
          const uint64_t g = mul2(w, add2(pack2(d[j], d[j + 1]), nd));
          d[j] = ok0 ? (uint32_t)g : 0u;
          d[j + 1] = ok1 ? (uint32_t)(g >> 32) : 0u;
        }
        s[j] = ok0 ? p0 : 0u;
        s[j + 1] = ok1 ? p1 : 0u;
      }
    }
  }
}
// Cap and bias are the kernel's (with all variants in one kernel a backward took a quarter longer,
// by spilled registers and instruction cache), masks a tile's.
template <Mode M, int TN, int N, bool kCap, bool kBias>
__device__ __forceinline__ void columns_by_mask(const AttnArgs& a, const Row& o, const Info<M, TN>& f, int k0, int j0,
                                                int mask, uint32_t (&s)[N], uint32_t (&d)[N]) {
  if (mask == kSeesAll) columns<M, TN, N, kCap, kBias, kSeesAll>(a, o, f, k0, j0, s, d);
  else if (mask == kByIndex) columns<M, TN, N, kCap, kBias, kByIndex>(a, o, f, k0, j0, s, d);
  else columns<M, TN, N, kCap, kBias, kByIndexAndDoc>(a, o, f, k0, j0, s, d);
}
// ---- a block --------------------------------------------------------------------------------------

template <Mode M, int D, bool kCap, bool kBias>
__device__ __forceinline__ void block_of(const AttnTcArgs& args, int block, int sp, uint8_t* smem) {
  using C = Map<M, D>;
  constexpr int TN = C::TN, ST = C::ST, W = C::W, NA = C::NA;
  // The call's pointers stay in the constant bank: a copy with the wait's zero added to them would
  // hold some thirty registers through the loops.  All data is read behind the wait, which is a
  // barrier to the compiler, and none of it is declared constant.
  const AttnArgs& a = args.a;
  int* list = reinterpret_cast<int*>(smem + (size_t)ST * C::STAGE);
  uint64_t* bars = reinterpret_cast<uint64_t*>(list + kListMost);
  uint64_t *full = bars, *empty = full + ST, *x_ready = empty + ST, *s_full = x_ready + 1, *p_ready = s_full + 2,
           *done = p_ready + 2, *drain = done + 2, *top_ready = drain + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(top_ready + 2);
  int* count = reinterpret_cast<int*>(tmem_slot + 1);
  Abort* ab = reinterpret_cast<Abort*>(count + 1);
  float* tops = reinterpret_cast<float*>(list + kListMost) + 128;  // [4][128], where shared
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < ST; s++) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    mbar_init(x_ready, 16);
    for (int w = 0; w < 2; w++) {
      mbar_init(&s_full[w], 1);
      mbar_init(&p_ready[w], 8);
      mbar_init(&done[w], 1);
      mbar_init(&drain[w], 1);
      mbar_init(&top_ready[w], 8);
    }
    ab->flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_trigger();
  grid_wait();
  uint32_t* status = a.status;

  constexpr bool own_keys = own_is_keys(M);
  const int n_own = own_keys ? a.Gk : a.rows, n_str = own_keys ? a.rows : a.Gk;
  const int pad = own_keys ? args.rows_pad : args.k_pad;
  const int splits = own_keys ? a.splits_kv : a.splits;
  const int blocks = (n_own + kOwn - 1) / kOwn;
  const int unit = block / blocks, r_blk = (block - unit * blocks) * kOwn;
  const Unit u = unit_of(a, unit, D);
  const Side& own_s = own_keys ? u.k : u.q;
  const int ntiles = (n_str + TN - 1) / TN;
  const int tile0 = (int)((int64_t)ntiles * sp / splits), tile1 = (int)((int64_t)ntiles * (sp + 1) / splits);
  const Own own = own_range(a, own_s, r_blk, r_blk + kOwn);

  // The tiles of this block's range that may hold a visible pair, in order.
  if (warp == 0) {
    int n = 0;
    for (int t0 = tile0; t0 < tile1; t0 += 32) {
      const int tile = t0 + lane, s0 = tile * TN, s1 = min(s0 + TN, n_str);
      bool see = tile < tile1;
      if (see && a.causal) {
        if (!own_keys) {
          see = s0 <= own.last || s0 < u.prefix;
        } else {
          const int f = u.q.token(s0), l = u.q.token(s1 - 1);
          const int last = u.q.first + (s1 - s0 > l - f + 1 ? a.Gq - 1 : l);
          see = own.first <= last || own.first < u.prefix;
        }
      }
      if (see && a.doc_q) {
        bool any = false;
        for (int i = s0 / 32; i * 32 < s1; i++) {
          const int2 r = own_keys ? args.q_range[(int64_t)unit * (pad / 32) + i]
                                  : args.k_range[(int64_t)u.b * (pad / 32) + i];
          any |= r.x <= own.doc_hi && r.y >= own.doc_lo;
        }
        see = any;
      }
      const uint32_t m = __ballot_sync(0xffffffffu, see);
      if (see) list[n + __popc(m & ((1u << lane) - 1u))] = tile;
      n += __popc(m);
    }
    if (lane == 0) *count = n;
  }
  __syncthreads();
  const int n = *count;

  const int wg = (warp - 4) >> 2, pr = wg >> 1, half = wg & 1, wq = warp & 3, own_row = r_blk + wq * 32 + lane;

  if (warp == 0) {
    if (lane == 0) {
      const uint8_t *row0, *row1 = nullptr, *col0, *col1 = nullptr;
      const size_t at = (size_t)unit * pad * (4 * W), lo_off = (size_t)a.units * pad * (4 * W);
      row0 = args.row_img[own_keys ? 2 : 0] + at;
      if (has_dp(M)) row1 = args.row_img[own_keys ? 3 : 1] + at;
      col0 = args.col_img[M == kFwd ? 1 : M == kDq ? 0 : M == kDv ? 3 : 2] + at;
      if (M == kDkv) col1 = args.col_img[3] + at;
      const int64_t all = (int64_t)a.units * pad, qat = (int64_t)unit * pad, kat = (int64_t)u.b * pad;
      const bool index = a.causal || a.doc_q;
      uint32_t bytes = (C::ROWS + C::COLS) * 2 * C::IMG;
      if (own_keys) bytes += TN * 4 * ((has_dp(M) ? 2 : 1) + (a.slopes ? 2 : 0) + (a.doc_q ? 1 : 0) + (index ? 1 : 0));
      else bytes += TN * 4 * ((a.slopes ? 1 : 0) + (a.doc_q ? 1 : 0));
      int i = 0;
      for (; i < n; i++) {
        const int s = i % ST;
        if (i >= ST && !mbar_wait(&empty[s], (uint32_t)((i / ST - 1) & 1), ab, status)) break;
        uint8_t* st = smem + (size_t)s * C::STAGE;
        const int64_t r0 = (int64_t)list[i] * TN;
        uint64_t* bar = &full[s];
        mbar_expect_tx(bar, bytes);
        auto rows = [&](int k, const uint8_t* src) {
          constexpr uint32_t kPanel = TN * 128;
#pragma unroll
          for (int p = 0; p < W / 32; p++) {
            const size_t from = ((size_t)p * pad + r0) * 128;
            bulk_load(st + (2 * k) * C::IMG + p * kPanel, src + from, kPanel, bar);
            bulk_load(st + (2 * k + 1) * C::IMG + p * kPanel, src + lo_off + from, kPanel, bar);
          }
        };
        auto cols = [&](int k, const uint8_t* src) {
          bulk_load(st + (2 * k) * C::IMG, src + r0 * (4 * W), C::IMG, bar);
          bulk_load(st + (2 * k + 1) * C::IMG, src + lo_off + r0 * (4 * W), C::IMG, bar);
        };
        rows(0, row0);
        if (has_dp(M)) rows(1, row1);
        cols(C::ROWS, col0);
        if (M == kDkv) cols(C::ROWS + 1, col1);
        uint8_t* info = st + C::INFO;
        auto part = [&](int k, const void* src) { bulk_load(info + k * TN * 4, src, TN * 4, bar); };
        if (own_keys) {
          part(0, args.q_info + qat + r0);
          if (has_dp(M)) part(1, args.q_info + all + qat + r0);
          if (a.slopes) {
            part(2, args.q_info + 2 * all + qat + r0);
            part(3, args.q_info + 3 * all + qat + r0);
          }
          if (a.doc_q) part(4, args.q_tok + qat + r0);
          if (index) part(5, args.q_tok + all + qat + r0);
        } else {
          if (a.slopes) part(0, args.k_pos + kat + r0);
          if (a.doc_q) part(1, args.k_doc + kat + r0);
        }
      }
      for (int j = (i > ST ? i - ST : 0); j < i; j++)  // no copy is left in flight
        mbar_drain(&full[j % ST], (uint32_t)((j / ST) & 1));
    }
  } else if (warp == 1 || warp == 2) {
    const int w = warp - 1;
    const uint32_t t0 = tmem + C::PAIR + (uint32_t)w * C::PAIR_COLS, x0 = tmem + C::X0, x1 = tmem + C::X1;
    bool ok = mbar_wait_w(x_ready, 0, ab, status);
    if (ok && w < n) ok = mbar_wait_w(&full[w % ST], 0, ab, status);
    tc_fence_after();
    for (int i = w, k = 0; ok && i < n; i += 2, k++) {
      const int s = i % ST;
      const uint32_t st = sdesc_lo(smem_u32(smem + (size_t)s * C::STAGE), 16);
      constexpr uint32_t kImg = C::IMG / 16;
      // the products of the pair's last tile have read what S now overwrites
      if (k > 0 && !(ok = mbar_wait_w(&done[w], (uint32_t)((k - 1) & 1), ab, status))) break;
      tc_fence_after();
      if (M == kDkv) {
        issue_rows_split<D>(t0 + C::S, x0, x0 + W, st);
        issue_rows_split<D>(t0 + C::DP, x1, x1 + W, st + 2 * kImg);
      } else {
        issue_rows<TN, D>(t0 + C::S, x0, x0 + W, st, st + kImg);
        if (has_dp(M)) issue_rows<TN, D>(t0 + C::DP, x1, x1 + W, st + 2 * kImg, st + 3 * kImg);
      }
      mma_commit_w(&s_full[w]);
      // the pair's next tile, waited for while the warpgroups work on this one
      if (i + 2 < n && !(ok = mbar_wait_w(&full[(i + 2) % ST], (uint32_t)(((i + 2) / ST) & 1), ab, status))) break;
      if (!(ok = mbar_wait_w(&p_ready[w], (uint32_t)(k & 1), ab, status))) break;
      tc_fence_after();
      const uint32_t c0 = st + C::ROWS * 2 * kImg;
      if constexpr (M == kFwd && !C::SHARED) {  // 32 keys each
        issue_cols<32, W>(t0 + C::ACC0, t0 + C::S, t0 + C::PLO, c0, c0 + kImg);
        issue_cols<32, W>(t0 + C::ACC1, t0 + C::S + 32, t0 + C::PLO + 32, c0 + 256, c0 + kImg + 256);
      }
      if constexpr (C::SHARED || M == kDv) issue_cols<TN, W>(t0 + C::ACC0, t0 + C::S, t0 + C::PLO, c0, c0 + kImg);
      if constexpr (M == kDq || M == kDk) issue_cols<TN, W>(t0 + C::ACC0, t0 + C::S, t0 + C::DP, c0, c0 + kImg);
      if constexpr (M == kDkv) {
        issue_cols<TN, W>(t0 + C::ACC0, t0 + C::DP, t0 + C::DSLO, c0, c0 + kImg);
        issue_cols<TN, W>(t0 + C::ACC1, t0 + C::S, t0 + C::PLO, c0 + 2 * kImg, c0 + 3 * kImg);
      }
      mma_commit_w(&empty[s]);
      mma_commit_w(&done[w]);
    }
    mma_commit_w(&drain[w]);
    mbar_drain_w(&drain[w], 0);
  } else if (warp >= 4) {
    const uint32_t lanes = (uint32_t)(wq * 32) << 16;
    // own rows' parts into TMEM: warpgroup 0 the first operand of S, warpgroup 1 that of dP
    if (wg == 0 || (wg == 1 && has_dp(M))) {
      const float* src = wg == 0 ? own_s.x0 : own_s.x1;
      const uint32_t at = tmem + lanes + (wg == 0 ? C::X0 : C::X1);
      constexpr int kAtOnce = D < 32 ? D : 32;
#pragma unroll 1
      for (int c = 0; c < D; c += kAtOnce) {
        uint32_t x[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; i += 4) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (own_row < n_own) v = *reinterpret_cast<const uint4*>(src + (int64_t)own_row * D + c + i);
          x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
        }
        store_parts(at + c, at + W + c, x);
      }
      tmem_wait_st();
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(x_ready);
    Row o;
    {
      const int r = min(own_row, n_own - 1), tok = own_s.token(r);
      const int index = own_s.first + tok;
      if (own_keys) o.limit = a.causal && index >= u.prefix ? index : INT_MIN;
      else o.limit = a.causal ? min(a.Gk, max(index + 1, u.prefix)) : a.Gk;
      // no streamed row has the document of an own row without one
      o.doc = own_s.doc ? (own_s.doc[tok] >= 0 ? own_s.doc[tok] : INT_MIN) : 0;
      o.pos = a.slopes ? own_s.place(tok) : 0.f;
      o.slope2 = !own_keys && a.slopes ? a.slopes[u.kvh * (a.H / a.Hkv) + r / a.Gq] * kLog2e : 0.f;
      o.nlse2 = M == kDq ? -lse2_of(a.lse[(int64_t)unit * a.rows + r]) : 0.f;
      o.ndelta = M == kDq ? -a.delta[(int64_t)unit * a.rows + r] : 0.f;
    }
    const uint32_t t0 = tmem + lanes + C::PAIR + (uint32_t)pr * C::PAIR_COLS;
    const uint32_t acc_at = t0 + C::ACC0 + (uint32_t)half * NA;
    float acc[NA];
#pragma unroll
    for (int c = 0; c < NA; c++) acc[c] = 0.f;
    float top = -INFINITY, sum = 0.f;
    float keep = 1.f;  // from the accumulators' base to that of the products not yet added
    auto flush = [&]() {
      uint32_t v[NA];
      if constexpr (NA == 32) tmem_ld32(acc_at, v);
      else tmem_ld16(acc_at, v);
      tmem_wait_ld(v);
#pragma unroll
      for (int c = 0; c < NA; c++)
        acc[c] = M == kFwd ? fmaf(acc[c], keep, __uint_as_float(v[c])) : acc[c] + __uint_as_float(v[c]);
    };
    // the first key that some own query does not see
    const int seen_by_all = a.causal ? min(a.Gk, max(own.first + 1, u.prefix)) : a.Gk;
    bool ok = true;
    for (int i = pr, k = 0; i < n; i += 2, k++) {
      if (k > 0) {  // the last tile's products, added while this one's scores are formed
        if (!(ok = mbar_wait_w(&done[pr], (uint32_t)((k - 1) & 1), ab, status))) break;
        tc_fence_after();
        flush();
      }
      if (!(ok = mbar_wait_w(&s_full[pr], (uint32_t)(k & 1), ab, status))) break;
      tc_fence_after();
      const Info<M, TN> f(smem + (size_t)(i % ST) * C::STAGE + C::INFO);
      const int k0 = list[i] * TN;
      int mask = kSeesAll;
      if (a.doc_q) {
        mask = kByIndexAndDoc;
      } else if (!own_keys) {
        if (k0 + TN > seen_by_all) mask = kByIndex;
      } else if (a.causal && own.last >= u.prefix) {  // some query of the tile may be before some own key
        const int s1 = min(k0 + TN, n_str), l = u.q.token(s1 - 1), t1 = u.q.token(k0);
        if (u.q.first + (s1 - k0 > l - t1 + 1 ? 0 : t1) < own.last) mask = kByIndex;
      }
      if constexpr (M == kFwd) {
        const int j0 = 32 * half;
        // Twice over the columns, 16 at a time, for the maximum and for the weights: all 32 scores
        // beside the accumulators would spill, and a spilled accumulator is a load from the
        // second-level cache (1000 clocks a tile).  Capped or biased scores go back in between.
        const float unit2 = score_unit<kCap, kBias>(a);
        float m = top;
#pragma unroll 1
        for (int h = 0; h < 32; h += 16) {
          uint32_t s[16];
          tmem_ld16(t0 + C::S + j0 + h, s);
          tmem_wait_ld(s);
          columns_by_mask<M, TN, 16, kCap, kBias>(a, o, f, k0, j0 + h, mask, s, s);
          float x = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
#pragma unroll
          for (int j = 2; j < 16; j += 2) x = max3(x, __uint_as_float(s[j]), __uint_as_float(s[j + 1]));
          m = fmaxf(m, x * unit2);
          if (kCap || kBias) tmem_st16(t0 + C::S + j0 + h, s);
        }
        if (kCap || kBias) tmem_wait_st();
        if constexpr (C::SHARED) {  // the other half's maximum; it is read before the next one is written
          tops[(2 * pr + half) * kOwn + wq * 32 + lane] = m;
          __syncwarp();
          if (lane == 0) mbar_arrive(&top_ready[pr]);
          if (!(ok = mbar_wait_w(&top_ready[pr], (uint32_t)(k & 1), ab, status))) break;
          m = fmaxf(m, tops[(2 * pr + (half ^ 1)) * kOwn + wq * 32 + lane]);
        }
        const float base = m == -INFINITY ? 0.f : m;
        keep = ex2(top - base);
        top = m;
        uint64_t part = 0;
#pragma unroll 1
        for (int h = 0; h < 32; h += 16) {
          uint32_t s[16];
          tmem_ld16(t0 + C::S + j0 + h, s);
          tmem_wait_ld(s);
          if (!(kCap || kBias)) columns_by_mask<M, TN, 16, kCap, kBias>(a, o, f, k0, j0 + h, mask, s, s);
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            const uint64_t x = fma2(pack2(s[j], s[j + 1]), both(unit2), both(-base));
            s[j] = __float_as_uint(ex2(lo_f(x)));
            s[j + 1] = __float_as_uint(ex2(hi_f(x)));
            part = add2(part, pack2(s[j], s[j + 1]));
          }
          store_parts(t0 + C::S + j0 + h, t0 + C::PLO + j0 + h, s);
        }
        sum = sum * keep + (lo_f(part) + hi_f(part));
      } else {
#pragma unroll 1
        for (int h = half * (TN / 2); h < (half + 1) * (TN / 2); h += 16) {
          uint32_t s[16], d[16];
          tmem_ld16(t0 + C::S + h, s);
          if (has_dp(M)) tmem_ld16(t0 + C::DP + h, d);
          if constexpr (M == kDkv) {
            uint32_t sl[16], dl[16];
            tmem_ld16(t0 + C::PLO + h, sl);
            tmem_ld16(t0 + C::DSLO + h, dl);
            tmem_wait_ld(s);
            tmem_wait_ld(d);
            tmem_wait_ld(sl);
            tmem_wait_ld(dl);
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
              const uint64_t x = add2(pack2(s[j], s[j + 1]), pack2(sl[j], sl[j + 1]));
              const uint64_t y = add2(pack2(d[j], d[j + 1]), pack2(dl[j], dl[j + 1]));
              s[j] = (uint32_t)x, s[j + 1] = (uint32_t)(x >> 32);
              d[j] = (uint32_t)y, d[j + 1] = (uint32_t)(y >> 32);
            }
          } else {
            tmem_wait_ld(s);
            if (has_dp(M)) tmem_wait_ld(d);
          }
          columns_by_mask<M, TN, 16, kCap, kBias>(a, o, f, k0, h, mask, s, d);
          if constexpr (M == kDkv) {
            store_parts(t0 + C::DP + h, t0 + C::DSLO + h, d);
            store_parts(t0 + C::S + h, t0 + C::PLO + h, s);
          } else if constexpr (M == kDv) {
            store_parts(t0 + C::S + h, t0 + C::PLO + h, s);
          } else {
            store_parts(t0 + C::S + h, t0 + C::DP + h, d);
          }
        }
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_ready[pr]);
    }
    const int mine = (n - pr + 1) / 2;  // tiles of this pair
    if (ok && mine > 0 && mbar_wait_w(&done[pr], (uint32_t)((mine - 1) & 1), ab, status)) {
      tc_fence_after();
      flush();
    }
    // The pairs' shares (in the forward all streams' rows) through shared memory, in place of the
    // stages, which nothing reads any more once every warpgroup is here.
    constexpr int kRowWords = 36, kFrom = M == kFwd && !C::SHARED ? 1 : 2;  // warpgroups from kFrom on hand over
    float* merge = reinterpret_cast<float*>(smem) + (size_t)(wq * 32 + lane) * kRowWords;
    named_barrier(1, 512);
    {
      float* to = merge + (size_t)wg * kOwn * kRowWords;
      if (wg >= kFrom) {
#pragma unroll
        for (int c = 0; c < NA; c += 4)
          *reinterpret_cast<float4*>(to + c) = make_float4(acc[c], acc[c + 1], acc[c + 2], acc[c + 3]);
      }
      if (M == kFwd) {
        to[32] = top;
        to[33] = sum;
      }
    }
    named_barrier(1, 512);
    if (wg < kFrom) {
      if constexpr (M == kFwd) {
        float m = top;
#pragma unroll
        for (int g = 0; g < 4; g++) m = fmaxf(m, merge[g * kOwn * kRowWords + 32]);
        const float base = m == -INFINITY ? 0.f : m;
        const float f0 = exp2_fast(top - base);
#pragma unroll
        for (int c = 0; c < 32; c++) acc[c] *= f0;
        sum = 0.f;
        for (int g = 0; g < 4; g++) {
          const float* other = merge + (size_t)g * kOwn * kRowWords;
          const float f = exp2_fast(other[32] - base);
          sum += other[33] * f;
          if (C::SHARED ? g != half + 2 : g == 0) continue;  // shared: the other pair's same channels
#pragma unroll
          for (int c = 0; c < 32; c++) acc[c] += other[c] * f;
        }
        top = m;
      } else {
        const float* other = merge + (size_t)(wg + 2) * kOwn * kRowWords;
#pragma unroll
        for (int c = 0; c < NA; c++) acc[c] += other[c];
      }
      constexpr bool kSpread = C::WIDE || M == kDq;  // a thread's channels start at NA * half
      bool bad = false;
#pragma unroll
      for (int c = 0; c < NA; c++) bad |= !(fabsf(acc[c]) < INFINITY);
      bad = bad && own_row < n_own;
      const int64_t all = (int64_t)a.units * n_own, at = (int64_t)unit * n_own;
      const int first = kSpread ? NA * half : 0;
      const bool dv = M == kDv || (M == kDkv && half);
      float *out, *stat = nullptr;
      if (M == kFwd) {
        out = a.splits > 1 ? a.part + ((int64_t)sp * all + at) * D : a.out + at * D;
        if (a.splits > 1) stat = a.part + (int64_t)a.splits * all * D + ((int64_t)sp * all + at) * 2;
      } else if (M == kDq) {
        out = splits > 1 ? a.part + ((int64_t)sp * all + at) * D : a.dq + at * D;
      } else {
        out = splits > 1 ? a.part_kv + (((int64_t)sp * 2 + (dv ? 1 : 0)) * all + at) * D : (dv ? a.dv : a.dk) + at * D;
      }
      if (own_row < n_own && !bad) {
        const float w = M == kFwd ? (stat ? 1.f : sum == 0.f ? 0.f : 1.f / sum) : dv ? 1.f : a.scale;
#pragma unroll
        for (int c = 0; c < NA; c += 4)
          if (D >= 32 || first + c < D)
            *reinterpret_cast<float4*>(out + (int64_t)own_row * D + first + c) =
                make_float4(acc[c] * w, acc[c + 1] * w, acc[c + 2] * w, acc[c + 3] * w);
        if (M == kFwd && (!C::SHARED || half == 0)) {
          if (stat) {
            stat[2 * own_row] = top;
            stat[2 * own_row + 1] = sum;
          } else {
            a.lse[at + own_row] = (top + log2f(sum)) * kLn2;
          }
        }
      }
      uint32_t rows = __ballot_sync(0xffffffffu, bad);
      for (; rows; rows &= rows - 1) {
        const int r = r_blk + wq * 32 + __ffs(rows) - 1, s0 = tile0 * TN, s1 = min(tile1 * TN, n_str);
        float o0[2], o1[2], m, l;
        if (M == kFwd) slow_row<D>(args.a, unit, r, s0, s1, &m, &l, o0);
        else slow_row_bwd<D, own_keys>(args.a, unit, r, s0, s1, o0, o1);
        const float w = M == kFwd && !stat ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
        const int c = lane + (C::WIDE ? first : 0);  // this half's channels
        const float x = C::WIDE && half ? (dv ? o1[1] : o0[1]) : (dv ? o1[0] : o0[0]);
        if (c < D && c >= first && c < first + NA) out[(int64_t)r * D + c] = x * w;
        if (M == kFwd && lane == 0 && (!C::SHARED || half == 0)) {
          if (stat) {
            stat[2 * r] = m;
            stat[2 * r + 1] = l;
          } else {
            a.lse[at + r] = (m + log2f(l)) * kLn2;
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

// (by an offset: through an integer the pointer would lose its address space)
__device__ __forceinline__ uint8_t* stages_of(uint8_t* raw) { return raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u); }

// Blocks in the order of their work under a prefix mask: late queries see most keys.
template <int D, bool kCap, bool kBias>
__global__ void __launch_bounds__(kThreads, 1) k_attn_fwd_tc(const __grid_constant__ AttnTcArgs args) {
  extern __shared__ __align__(1024) uint8_t raw[];
  block_of<kFwd, D, kCap, kBias>(args, (int)(gridDim.x - 1 - blockIdx.x), blockIdx.y, stages_of(raw));
}
// dk and dv first: they have four products a pair, dq three.  d = 64: dk, dq, and last dv, which
// has two.
template <int D, bool kCap, bool kBias>
__global__ void __launch_bounds__(kThreads, 1) k_attn_bwd_tc(const __grid_constant__ AttnTcArgs args, int blocks_kv,
                                                             int blocks_q) {
  extern __shared__ __align__(1024) uint8_t raw[];
  const int b = blockIdx.x, nkv = blocks_kv * args.a.splits_kv, nq = blocks_q * args.a.splits;
  if (b < nkv) {
    block_of<D == 64 ? kDk : kDkv, D, kCap, kBias>(args, b / args.a.splits_kv, b % args.a.splits_kv, stages_of(raw));
  } else if (D < 64 || b < nkv + nq) {
    const int c = b - nkv;
    block_of<kDq, D, kCap, kBias>(args, blocks_q - 1 - c / args.a.splits, c % args.a.splits, stages_of(raw));
  } else if constexpr (D == 64) {
    const int c = b - nkv - nq;
    block_of<kDv, D, kCap, kBias>(args, c / args.a.splits_kv, c % args.a.splits_kv, stages_of(raw));
  }
}

template <int D>
constexpr size_t bwd_smem() {
  if constexpr (D == 64) return std::max({Map<kDq, D>::SMEM, Map<kDk, D>::SMEM, Map<kDv, D>::SMEM});
  else return std::max(Map<kDq, D>::SMEM, Map<kDkv, D>::SMEM);
}

}  // namespace

template <int D>
cudaError_t attn_tc(const AttnTcArgs& t, bool backward, cudaStream_t st) {
  const AttnArgs& a = t.a;
  const int atoms = std::max(t.k_pad, backward ? t.rows_pad : 0) / 32;
  cudaError_t e = launch(k_attn_prep<D>, dim3((unsigned)(a.units * atoms), backward ? 4 : 2), dim3(256), 0, st, t);
  if (e != cudaSuccess) return e;
  const int64_t blocks_q = (int64_t)a.units * ((a.rows + kOwn - 1) / kOwn);
  const int64_t blocks_kv = (int64_t)a.units * ((a.Gk + kOwn - 1) / kOwn);
  const int64_t nrows = (int64_t)a.units * a.rows;
  const bool cap = a.cap > 0.f, bias = a.slopes != nullptr;
  if (!backward) {
    constexpr size_t smem = Map<kFwd, D>::SMEM;
    const auto kernel = cap ? (bias ? k_attn_fwd_tc<D, true, true> : k_attn_fwd_tc<D, true, false>)
                            : (bias ? k_attn_fwd_tc<D, false, true> : k_attn_fwd_tc<D, false, false>);
    e = allow_smem<smem>(kernel);
    if (e == cudaSuccess)
      e = launch(kernel, dim3((unsigned)blocks_q, (unsigned)a.splits), dim3(kThreads), smem, st, t);
    if (e == cudaSuccess && a.splits > 1)
      e = attn_join<D>(a, st);
    return e;
  }
  constexpr size_t smem = bwd_smem<D>();
  const auto kernel = cap ? (bias ? k_attn_bwd_tc<D, true, true> : k_attn_bwd_tc<D, true, false>)
                          : (bias ? k_attn_bwd_tc<D, false, true> : k_attn_bwd_tc<D, false, false>);
  e = allow_smem<smem>(kernel);
  const int64_t kinds = D == 64 ? 2 : 1;  // dk and dv apart
  if (e == cudaSuccess)
    e = launch(kernel, dim3((unsigned)(kinds * blocks_kv * a.splits_kv + blocks_q * a.splits)), dim3(kThreads), smem, st,
               t, (int)blocks_kv, (int)blocks_q);
  if (e != cudaSuccess || (a.splits == 1 && a.splits_kv == 1)) return e;
  const int64_t nq = nrows * D, nk = (int64_t)a.units * a.Gk * D;
  const int64_t n = (a.splits > 1 ? nq : 0) + (a.splits_kv > 1 ? 2 * nk : 0);
  return launch(k_attn_sum, dim3((unsigned)((n / 4 + 255) / 256)), dim3(256), 0, st, a, nq, nk);
}

}  // namespace fs
