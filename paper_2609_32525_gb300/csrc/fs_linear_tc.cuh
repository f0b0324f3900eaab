// Linear maps on tcgen05 (internal): what the bf16 and the fp32 products share.
//
// D[m, n] = sum_k A[m, k] B[n, k].  Two CTAs of a cluster share a tile of 256 x (64 to 256) values of D:
// each holds 128 of A's rows and half of B's, so that an operand byte is loaded once for 256 rows of the other
// one, and the leader issues products of 256 x n x 16 for both (cta_group::2).  Pairs are persistent and walk
// over units (tile, part of the sum); while a unit's epilogue runs, the next one's products go to the other
// half of TMEM.  An epilogue warp owns 32 rows of some columns; a residual or pre-activation comes by TMA
// into the 32 x 128 byte box that the result leaves from, so all traffic with HBM is in whole 128-byte lines.
// Results whose pitch TMA cannot address leave by plain stores.
//
// The tensor core cuts its accumulator towards zero at every step.  bf16 results do not see that; fp32
// results (dW, split sums, fp32 rows) are taken out of TMEM every few hundred terms and added up in
// registers.  dbias, the sum of g over its rows, is a product with ones.
#pragma once

#include "fs_internal.h"
#include "fs_launch.h"
#include "fs_linear_end.cuh"
#include "fs_tc_pair.cuh"

#include <algorithm>
#include <cudaTypedefs.h>
#include <mutex>
#include <type_traits>

namespace fs {
namespace {

using namespace tc;

constexpr int kMaxStages = 12;
constexpr uint32_t kABytes = 128 * 128;          // 128 rows (or 64 terms x 128) of 64 values
constexpr uint32_t kBox = 32 * 128;              // an epilogue warp's box
constexpr uint32_t kOnes = 1024;
constexpr size_t kSmem = 231424;                 // with the barriers below the limit of a block
// dbias' accumulators, of 32 columns; fp32 rows' small parts have one of their own, kSumSmall columns on.  (All parts in one,
// 48 cuts to hi's step in 256 terms: 6.8e-7 of the norm for 131,072 rows of N(0, 1), 1.2e-7 in two.)
constexpr uint32_t kSumCol = 256, kSumSmall = 32;
// Epilogue warpgroups and boxes of a warp; what the boxes leave for the stages.
template <int kGroups, int kPer>
struct Block {
  static constexpr int kThreads = 64 + 128 * kGroups;
  static constexpr uint32_t kBoxes = kGroups * 4 * kPer * kBox, kStageRoom = kSmem - 1024 - kOnes - kBoxes;
};

enum { kEndFwd = 0, kEndDx = 1, kEndRaw = 2 };

struct TcArgs {
  CUtensorMap a, b, y, pre, res;
  LinearEnd e;
  int64_t M, K, per;
  int N, ldy, n_tiles, tiles, units, bn, splits, stages, seg;  // ldy: pitch of y; seg: blocks of 64 terms taken out at a time
  int step_n, step_m;                                   // from a pair's unit to its next one
  uint32_t stage_bytes, idesc, idesc_sum, a_step, b_step;  // steps: 16 terms on in a stage, in 16-byte units
  int a_mn, b_mn;
  int load_res, load_pre, store_pre, plain;             // plain: y, res and pre by plain accesses
  int pre_at_rows;                                      // fp32: pre by lanes in place (a box serves one tensor)
  const char* ahead;                                    // null, or A to prefetch to L2 a tile ahead, in whole rows
  int sums;                                             // dbias is wanted
  float* part_sums;                                     // split: [splits][M]
  uint32_t* status;
  int reset;
  uint32_t none;                                        // 0
};

// The units of a pair, number `pair` and every pairs-th one after it; stepped, not divided, since an epilogue
// warp's few hundred instructions a chunk run one after another.  Where sums are split a pair has one unit, so that no
// step leaves its part.
struct Unit {
  int m, n;
  int left;  // units from this one on, 0 or less: none
  int64_t first;
  __device__ __forceinline__ Unit(const TcArgs& g, int u) : left(g.units - u) {
    const int split = u / g.tiles;
    first = split * g.per;
    const int t = u - split * g.tiles;
    m = t / g.n_tiles;
    n = t - m * g.n_tiles;
  }
  __device__ __forceinline__ void next(const TcArgs& g, int pairs) {
    left -= pairs;
    n += g.step_n;
    m += g.step_m;
    if (n >= g.n_tiles) n -= g.n_tiles, m++;
  }
  // Its part of the sum, and the part's first term.
  __device__ __forceinline__ int split(const TcArgs& g) const { return g.splits > 1 ? (int)(first / g.per) : 0; }
  __device__ __forceinline__ int64_t k0() const { return first; }
  __device__ __forceinline__ int blocks(const TcArgs& g) const {
    const int64_t k = g.K - first < g.per ? g.K - first : g.per;
    return (int)((k + 63) >> 6);
  }
};

// Which half of TMEM a segment's products go to.  A unit with dbias, its pair's only one, uses the first half for all
// and columns of the second one for the sums; the others take turns.
struct Halves {
  uint32_t uses0 = 0, uses1 = 0;
  int turn = 0;
  __device__ __forceinline__ int pick(bool sums) {
    if (sums) return 0;
    turn ^= 1;
    return turn;
  }
  __device__ __forceinline__ uint32_t uses(int half) const { return half ? uses1 : uses0; }
  __device__ __forceinline__ void use(int half) {
    uses0 += half ^ 1;
    uses1 += half;
  }
};

__device__ __forceinline__ uint4 ld_box(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

// 16 neighbouring values of a row in a box, from piece piece0 on: piece j of 16 bytes of row r lies
// at (j ^ r % 8) * 16, TMA's 128-byte swizzle.  line: the box's address + 128 r.
template <typename T>
struct Line {
  static constexpr int kPieces = sizeof(T);
  __device__ __forceinline__ static uint32_t at(uint32_t line, int piece) {
    return line + (((uint32_t)piece ^ ((line >> 7) & 7)) << 4);
  }
  __device__ __forceinline__ static void load(uint32_t line, int piece0, float (&v)[16]) {
#pragma unroll
    for (int j = 0; j < kPieces; j++) {
      const uint4 w = ld_box(at(line, piece0 + j));
      const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; i++) {
        if constexpr (sizeof(T) == 2)
          v[8 * j + 2 * i] = __uint_as_float(x[i] << 16), v[8 * j + 2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
        else
          v[4 * j + i] = __uint_as_float(x[i]);
      }
    }
  }
  __device__ __forceinline__ static void store(uint32_t line, int piece0, const float (&v)[16]) {
#pragma unroll
    for (int j = 0; j < kPieces; j++) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; i++)
        x[i] = sizeof(T) == 2 ? pack_bf16(v[8 * j + 2 * i], v[8 * j + 2 * i + 1]) : __float_as_uint(v[4 * j + i]);
      st_shared_v4(at(line, piece0 + j), x[0], x[1], x[2], x[3]);
    }
  }
};

// 16 fp32 values of a row in memory, n of which are there; plain: at any address.
template <bool kStore>
__device__ __forceinline__ void rows16(float* p, int n, bool plain, float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 16; i += 4) {
    if (!plain) {  // four columns are all there or none
      if (i < n) {
        float4* q = reinterpret_cast<float4*>(p + i);
        if (kStore) *q = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        else v[i] = q->x, v[i + 1] = q->y, v[i + 2] = q->z, v[i + 3] = q->w;
      } else if (!kStore) {
        v[i] = v[i + 1] = v[i + 2] = v[i + 3] = 0.f;
      }
    } else {
#pragma unroll
      for (int j = i; j < i + 4; j++) {
        if (kStore && j < n) p[j] = v[j];
        if (!kStore) v[j] = j < n ? p[j] : 0.f;
      }
    }
  }
}

// What the end of a map does: dropout (counters of 32 or of 64 bits) and a residual.
enum { kNoDrop = 0, kDrop32 = 1, kDrop64 = 2 };

// The end of a map on 16 neighbouring columns of a row, step by step for all of them, so that the
// chains of 16 values (4 counters) are under way at once.  quad: the first one's counter.
template <int END, typename T, int DROP, bool kRes, typename Q>
__device__ __forceinline__ void end16(const TcArgs& g, const act::DropKey& key, int64_t row, Q quad, int col, int piece0,
                                      uint32_t yline, uint32_t pline, float (&v)[16]) {
  constexpr bool kFast = sizeof(T) == 2;
  if constexpr (END == kEndFwd) {
    if (g.e.bias) {
      if ((g.N & 3) == 0) {  // (four columns past the last ones get biases that nobody looks at)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 b = *reinterpret_cast<const float4*>(g.e.bias + min(col + i, g.N - 4));
          v[i] += b.x, v[i + 1] += b.y, v[i + 2] += b.z, v[i + 3] += b.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; i++) v[i] += g.e.bias[min(col + i, g.N - 1)];
      }
    }
    if (g.store_pre) Line<T>::store(pline, piece0, v);
    if constexpr (!kFast) {
      if (g.pre_at_rows && row < g.M) rows16<true>(static_cast<float*>(g.e.pre_out) + row * g.N + col, g.N - col, g.plain, v);
    }
    act::apply<kFast>(g.e.act, v);
  }
  if constexpr (END == kEndDx) {
    if (g.load_pre || (!kFast && g.pre_at_rows)) {
      float u[16];
      if (g.load_pre) {
        Line<T>::load(pline, piece0, u);
      } else if constexpr (!kFast) {
        float* pre = const_cast<float*>(static_cast<const float*>(g.e.pre_in)) + row * g.N + col;
        rows16<false>(pre, row < g.M ? g.N - col : 0, g.plain, u);
      }
      act::slope<kFast>(g.e.act, u, v);
#pragma unroll
      for (int i = 0; i < 16; i++) v[i] = u[i];
    }
  }
  if constexpr (DROP != kNoDrop || kRes) {
    float r[16];
    if constexpr (kRes) {
      Line<T>::load(yline, piece0, r);
    } else {
#pragma unroll
      for (int i = 0; i < 16; i++) r[i] = 0.f;
    }
    if constexpr (DROP != kNoDrop) {
      act::keep_by<16>({g.e.rng, g.e.threshold, g.e.scale}, key, quad, v, r);
    } else {
#pragma unroll
      for (int i = 0; i < 16; i++) r[i] += v[i];
    }
    Line<T>::store(yline, piece0, r);
  } else {
    Line<T>::store(yline, piece0, v);
  }
}
// f(v, i) fills the i-th 16 of n * 16 values.
template <int END, typename T, int DROP, bool kRes, int n, typename Q, typename F>
__device__ __forceinline__ void end_loop(const TcArgs& g, const act::DropKey& key, int64_t row, Q quad, int col,
                                         uint32_t yline, uint32_t pline, F&& f) {
#pragma unroll 1
  for (int i = 0; i < n; i++) {
    float v[16];
    f(v, i);
    end16<END, T, DROP, kRes>(g, key, row, (Q)(quad + 4 * i), col + 16 * i, Line<T>::kPieces * i, yline, pline, v);
  }
}
template <int END, typename T, int n, typename F>
__device__ __forceinline__ void end_chunk(const TcArgs& g, const act::DropKey& key, int64_t row, int col, uint32_t yline,
                                          uint32_t pline, F&& f) {
  if (END != kEndRaw && g.e.rng) {
    const uint64_t quad = (uint64_t)row * (uint64_t)((g.N + 3) >> 2) + (uint64_t)(col >> 2);
    // one branch for a warp
    if (__all_sync(0xffffffffu, ((quad + 4 * n) >> 32) == 0)) {
      const uint32_t q = (uint32_t)quad;
      if (g.load_res) end_loop<END, T, END != kEndRaw ? kDrop32 : 0, true, n>(g, key, row, q, col, yline, pline, f);
      else end_loop<END, T, END != kEndRaw ? kDrop32 : 0, false, n>(g, key, row, q, col, yline, pline, f);
    } else {
      if (g.load_res) end_loop<END, T, END != kEndRaw ? kDrop64 : 0, true, n>(g, key, row, quad, col, yline, pline, f);
      else end_loop<END, T, END != kEndRaw ? kDrop64 : 0, false, n>(g, key, row, quad, col, yline, pline, f);
    }
  } else {
    if (g.load_res) end_loop<END, T, kNoDrop, true, n>(g, key, row, 0u, col, yline, pline, f);
    else end_loop<END, T, kNoDrop, false, n>(g, key, row, 0u, col, yline, pline, f);
  }
}

template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, int have) {
  if constexpr (kBytes == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(have) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(src), "r"(have), "n"(kBytes) : "memory");
}
// A box between shared memory and rows that TMA cannot address, by a warp.  Rows of bf16 with an even pitch are rows
// of half as many words; with an odd one they go value by value.  kWords: neighbouring words of an access (two
// where the pitch in words is even).
template <int kWords>
__device__ __forceinline__ void box_in(const uint32_t* rows, int64_t ld, int64_t M, int N, int64_t row0, int col0, uint32_t box) {
  constexpr int kLanes = 32 / kWords;
  const int lane = threadIdx.x & 31, c = lane % kLanes * kWords, first = lane / kLanes;
  const int n_rows = col0 + c < N ? (int)min(M - row0, (int64_t)32) : 0;
  const uint32_t* p = rows + (row0 + first) * ld + col0 + c;
#pragma unroll 4
  for (int r = first; r < 32; r += kWords) {
    copy_async<4 * kWords>(box + r * 128 + (((c >> 2) ^ (r & 7)) << 4) + (c & 3) * 4, r < n_rows ? p : rows, r < n_rows ? 4 * kWords : 0);
    p += kWords * ld;
  }
}
// (eight accesses at a time: more would take registers from the paths that have no use for this one)
template <int kWords>
__device__ __forceinline__ void box_out(uint32_t* rows, int64_t ld, int64_t M, int N, int64_t row0, int col0, uint32_t box) {
  constexpr int kLanes = 32 / kWords;
  const int lane = threadIdx.x & 31, c = lane % kLanes * kWords, first = lane / kLanes;
  const int n_rows = col0 + c < N ? (int)min(M - row0, (int64_t)32) : 0;
  uint32_t* p = rows + (row0 + first) * ld + col0 + c;
#pragma unroll 1
  for (int r0 = first; r0 < 32; r0 += 8 * kWords) {
    uint2 w[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const int r = r0 + i * kWords;
      const uint32_t at = box + r * 128 + (((c >> 2) ^ (r & 7)) << 4) + (c & 3) * 4;
      if constexpr (kWords == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[i].x), "=r"(w[i].y) : "r"(at) : "memory");
      else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[i].x) : "r"(at) : "memory");
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
      if (r0 + i * kWords < n_rows) {
        if constexpr (kWords == 2) *reinterpret_cast<uint2*>(p) = w[i];
        else *p = w[i].x;
      }
      p += kWords * ld;
    }
  }
}
__device__ __forceinline__ void box_of_bf16(unsigned short* rows, int64_t ld, int64_t M, int N, int64_t row0, int col0, uint32_t box,
                                            bool load) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int j = 0; j < 8; j++) {  // 32 columns of 8 rows
    const int c = lane + 32 * (j & 1), r0 = 8 * (j >> 1), n_rows = col0 + c < N ? (int)min(M - row0 - r0, (int64_t)8) : 0;
    unsigned short *p = rows + (row0 + r0) * ld + col0 + c, w[8];
    if (load) {
#pragma unroll
      for (int r = 0; r < 8; r++) w[r] = r < n_rows ? p[r * ld] : (unsigned short)0;
    }
#pragma unroll
    for (int r = 0; r < 8; r++) {
      const uint32_t q = box + (r0 + r) * 128 + (((c >> 3) ^ r) << 4) + (c & 7) * 2;
      if (load) asm volatile("st.shared.u16 [%0], %1;" ::"r"(q), "h"(w[r]) : "memory");
      else asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w[r]) : "r"(q) : "memory");
    }
    if (!load) {
#pragma unroll
      for (int r = 0; r < 8; r++)
        if (r < n_rows) p[r * ld] = w[r];
    }
  }
}
// Columns of T; loads are under way until copies_wait.
template <typename T>
__device__ __forceinline__ void box_by_lanes(T* rows, int64_t ld, int64_t M, int N, int64_t row0, int col0, uint32_t box, bool load) {
  if (sizeof(T) == 2 && (ld & 1)) {
    box_of_bf16(reinterpret_cast<unsigned short*>(rows), ld, M, N, row0, col0, box, load);
    return;
  }
  constexpr int kPer = 4 / sizeof(T);
  uint32_t* w = reinterpret_cast<uint32_t*>(rows);
  ld /= kPer, N /= kPer, col0 /= kPer;
  if ((ld & 1) == 0) {
    if (load) box_in<2>(w, ld, M, N, row0, col0, box);
    else box_out<2>(w, ld, M, N, row0, col0, box);
  } else {
    if (load) box_in<1>(w, ld, M, N, row0, col0, box);
    else box_out<1>(w, ld, M, N, row0, col0, box);
  }
}
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncwarp();
}

// An epilogue warp's boxes.  A box is filled by loads that were issued one chunk earlier (two boxes
// take turns), or both serve one chunk where it has two inputs or two results.
template <int END, typename T, int kPer>
struct Boxes {
  const TcArgs& g;
  uint32_t base;       // shared address of the warp's two boxes
  uint64_t* bar;       // two barriers
  uint32_t phases = 0; // one bit a barrier
  int turn = 0;
  const bool both;     // both boxes serve one chunk
  const bool serial;   // a chunk's loads start after the one before has left
  const int loads;
  static constexpr int kCols = 128 / sizeof(T);
  __device__ __forceinline__ Boxes(const TcArgs& g_, uint32_t base_, uint64_t* bar_)
      : g(g_),
        base(base_),
        bar(bar_),
        both(kPer == 2 && (g_.store_pre || (g_.load_res && g_.load_pre))),
        serial(kPer == 1 || both),
        loads(g_.load_res + g_.load_pre) {}

  // Where y and the residual, and the pre-activations lie for the next chunk processed.
  __device__ __forceinline__ uint32_t ybox() const { return base + (serial ? 0 : turn * kBox); }
  __device__ __forceinline__ uint32_t pbox() const { return both ? base + kBox : ybox(); }

  // Starts the loads of a chunk, `ahead` chunks after the next one processed; its box's last store
  // has to be read out first.
  __device__ __forceinline__ void start(int ahead, int64_t row, int col) {
    if (!loads) return;
    if (g.plain) {
      const uint32_t to = base + (serial ? 0 : (turn + ahead) & 1) * kBox;
      auto one = [&](const void* from, uint32_t box) {
        box_by_lanes<T>(const_cast<T*>(static_cast<const T*>(from)), g.ldy, g.M, g.N, row, col, box, true);
      };
      if (g.load_res) one(g.e.res, to);
      if (g.load_pre) one(g.e.pre_in, both ? to + kBox : to);
      __syncwarp();
      return;
    }
    if ((threadIdx.x & 31) == 0) {
      bulk_wait_read<0>();
      const int b = serial ? 0 : (turn + ahead) & 1;
      mbar_expect_tx(&bar[b], loads * kBox);
      const uint32_t box = base + b * kBox;
      if (g.load_res) tma_load(box, &g.res, col, (int)row, &bar[b]);
      if (g.load_pre) tma_load(both ? box + kBox : box, &g.pre, col, (int)row, &bar[b]);
    }
    __syncwarp();
  }
  // Before the chunk's box is read and written.
  __device__ __forceinline__ bool ready(int64_t row, int col, Abort* ab, uint32_t* status) {
    if (g.plain) {
      if (loads) copies_wait();
      return true;
    }
    if (loads) {
      const int b = serial ? 0 : turn;
      const bool ok = mbar_wait_w(&bar[b], (phases >> b) & 1u, ab, status);
      phases ^= 1u << b;
      return ok;
    }
    if ((threadIdx.x & 31) == 0) {
      if (serial) bulk_wait_read<0>();
      else bulk_wait_read<1>();
    }
    __syncwarp();
    return true;
  }
  // After it was written.
  __device__ __forceinline__ void send(int64_t row, int col, int split) {
    if (g.plain) {
      __syncwarp();
      T* y = static_cast<T*>(g.e.y) + (int64_t)split * g.M * g.ldy;
      box_by_lanes<T>(y, g.ldy, g.M, g.N, row, col, ybox(), false);
      if (g.store_pre) box_by_lanes<T>(static_cast<T*>(g.e.pre_out), g.ldy, g.M, g.N, row, col, pbox(), false);
      __syncwarp();
    } else {
      fence_proxy_async_smem();
      __syncwarp();
      if ((threadIdx.x & 31) == 0) {
        if (row < g.M && col < g.N) {
          tma_store(&g.y, col, (int)row, split, ybox());
          if (g.store_pre) tma_store(&g.pre, col, (int)row, 0, pbox());
        }
        bulk_commit();
      }
    }
    turn ^= 1;
  }
};


// ---- epilogues -----------------------------------------------------------------------------------

// An epilogue warp's place: TMEM lanes, rows and barriers.
struct Place {
  const TcArgs& g;
  uint32_t lanes, free0;  // TMEM address of its lanes; the leader's first acc_empty
  uint64_t* acc_full;
  int rank, wg, sub, lane, pair, pairs;
  Abort* ab;
  uint32_t* status;
  __device__ __forceinline__ int64_t row(const Unit& w) const { return (int64_t)w.m * 256 + rank * 128 + sub * 32; }
  __device__ __forceinline__ bool wait(Halves& h, int half) const {
    const bool ok = mbar_wait_w(&acc_full[half], h.uses(half) & 1u, ab, status);
    h.use(half);
    tc_fence_after();
    return ok;
  }
  __device__ __forceinline__ void release(int half) const {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive_leader(free0 + 8 * half);
  }
};

// bf16 rows: the pair's tiles are one sequence of chunks of 64 columns, which the warpgroups take in turn.
template <int END, typename T, int kGroups, int kPer>
__device__ __forceinline__ void row_epilogue(const Place& at, Boxes<END, T, kPer>& box, const act::DropKey& key) {
  const TcArgs& g = at.g;
  const int chunks = g.bn >> 6;
  auto place = [&](Unit& w, int& c) {  // from a chunk number past the unit's to the unit that it is in
    while (c >= chunks) c -= chunks, w.next(g, at.pairs);
  };
  int c = at.wg, nc = at.wg;
  Unit nw(g, at.pair);  // (nw, nc): the chunk whose loads start next
  place(nw, nc);
  auto start_next = [&](int ahead) {
    if (nw.left > 0) box.start(ahead, at.row(nw), nw.n * g.bn + nc * 64);
    nc += kGroups;
    place(nw, nc);
  };
  Halves h;
  bool ok = true;
  if (box.loads) start_next(0);
  for (Unit w(g, at.pair); w.left > 0 && ok; w.next(g, at.pairs)) {
    const int64_t row0 = at.row(w);
    const int half = h.pick(false);
    ok = at.wait(h, half);
    if (!ok) break;
    if (c >= chunks) at.release(half);
    for (; c < chunks && ok; c += kGroups) {
      const int col = w.n * g.bn + c * 64;
      if (box.loads && !box.serial) start_next(1);
      ok = box.ready(row0, col, at.ab, at.status);
      if (!ok) break;
      const uint32_t from = at.lanes + half * 256 + c * 64;
      end_chunk<END, T, 4>(g, key, row0 + at.lane, col, box.ybox() + at.lane * 128, box.pbox() + at.lane * 128,
                           [&](float(&v)[16], int i) {
                             uint32_t r[16];
                             tmem_ld16(from + 16 * i, r);
                             tmem_wait_ld(r);
                             if (i == 3 && c + kGroups >= chunks) at.release(half);
#pragma unroll
                             for (int j = 0; j < 16; j++) v[j] = __uint_as_float(r[j]);
                           });
      box.send(row0, col, 0);  // (split sums are fp32)
      if (box.loads && box.serial) start_next(1);
    }
    c -= chunks;
  }
}

// fp32 results: two warpgroups take half of a tile's columns each and add its segments up in registers; the last
// segment's sums go back to TMEM, from where the end is a loop.  PARTS == 3: the small products' accumulator lies
// 128 columns on.
template <int END, int PARTS, int kPer>
__device__ __forceinline__ void sum_epilogue(const Place& at, Boxes<END, float, kPer>& box, const act::DropKey& key) {
  const TcArgs& g = at.g;
  constexpr int kMost = PARTS == 1 ? 8 : 4;  // pieces of 16 columns
  const int cols = g.bn >> 1, first = at.wg * cols;
  Halves h;
  bool ok = true;
  // small: where the small parts' accumulator lies from there, 0 where it has been added
  auto piece = [&](uint32_t t, uint32_t small, float(&v)[16]) {
    uint32_t r[16];
    tmem_ld16(t, r);
    if (PARTS == 3 && small) {
      uint32_t s[16];
      tmem_ld16(t + small, s);
      tmem_wait_ld(s);
      tmem_wait_ld(r);
#pragma unroll
      for (int j = 0; j < 16; j++) v[j] = __uint_as_float(r[j]) + __uint_as_float(s[j]);
    } else {
      tmem_wait_ld(r);
#pragma unroll
      for (int j = 0; j < 16; j++) v[j] = __uint_as_float(r[j]);
    }
  };
  for (Unit w(g, at.pair); w.left > 0 && ok; w.next(g, at.pairs)) {
    const int64_t row0 = at.row(w);
    const int col = w.n * g.bn + first, blocks = w.blocks(g), part = w.split(g);
    const bool sums = g.sums && w.n == 0, many = blocks > g.seg;
    float acc[kMost][16], sum = 0.f;
    box.start(0, row0, col);
    int half = 0;
    uint32_t t = 0;
    for (int kb = 0; kb < blocks && ok; kb += g.seg) {
      half = h.pick(sums);
      ok = at.wait(h, half);
      if (!ok) break;
      t = at.lanes + half * 256 + first;
      const bool last = kb + g.seg >= blocks;
      if (many) {
#pragma unroll
        for (int i = 0; i < kMost; i++) {
          if (16 * i >= cols) continue;
          float v[16];
          piece(t + 16 * i, 128, v);
#pragma unroll
          for (int j = 0; j < 16; j++) acc[i][j] = kb == 0 ? v[j] : acc[i][j] + v[j];
          if (last) {
            uint32_t r[16];
#pragma unroll
            for (int j = 0; j < 16; j++) r[j] = __float_as_uint(acc[i][j]);
            tmem_st16(t + 16 * i, r);
          }
        }
      }
      if (END == kEndRaw && sums && at.wg == 0) {
        float v[16];
        piece(at.lanes + kSumCol, kSumSmall, v);
        sum += v[0];
      }
      if (!last) at.release(half);
    }
    if (!ok) break;
    if (many) tmem_wait_st();
    if (END == kEndRaw && sums && at.wg == 0 && row0 + at.lane < g.M) {
      if (g.splits > 1) g.part_sums[(int64_t)part * g.M + row0 + at.lane] = sum;
      else lin::end_sum(g.e, row0 + at.lane, sum);
    }
#pragma unroll 1
    for (int i = 0; 32 * i < cols; i++) {
      const bool more = 32 * (i + 1) < cols;
      if (!box.serial && more) box.start(1, row0, col + (i + 1) * 32);
      ok = box.ready(row0, col + i * 32, at.ab, at.status);
      if (!ok) break;
      end_chunk<END, float, 2>(g, key, row0 + at.lane, col + i * 32, box.ybox() + at.lane * 128, box.pbox() + at.lane * 128,
                               [&](float(&v)[16], int p) {
                                 piece(t + 32 * i + 16 * p, many ? 0 : 128, v);
                                 if (p == 1 && !more) at.release(half);
                               });
      box.send(row0, col + i * 32, part);
      if (box.serial && more) box.start(1, row0, col + (i + 1) * 32);
    }
  }
}

// ---- the products' issue -----------------------------------------------------------------------

// Waits until a half of TMEM is free for a segment.  By the leader's issuing warp.
struct Issuer {
  Halves h;
  __device__ __forceinline__ bool take(int half, uint64_t* acc_empty, Abort* ab, uint32_t* status) {
    const bool ok = mbar_wait_w(&acc_empty[half], (h.uses(half) & 1u) ^ 1u, ab, status);
    h.use(half);
    tc_fence_after();
    return ok;
  }
};

// A block's last steps.  A CTA that gave up may have copies on their way that count on barriers whose phase never
// ends (the other CTA's part is missing): they land in microseconds, and a hundred times that is waited for them.
__device__ __forceinline__ void leave(Abort* ab, uint32_t tmem, bool dealloc) {
  __syncwarp();
  if (ab->flag) {
    const uint64_t t0 = globaltimer();
    for (uint32_t i = 0; i < 1000000u && globaltimer() - t0 < 2000000ull; i++) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  pair_sync();
  tc_fence_after();
  if (dealloc) tmem_dealloc_pair(tmem, 512);
}

// ---- host side ---------------------------------------------------------------------------------

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  });
  return fn;
}

// [planes][rows][ld] of which cols columns are looked at; boxes of 128 bytes x box_rows.
bool make_map(CUtensorMap* map, const void* p, int size, int64_t cols, int64_t rows, int64_t planes, int64_t ld,
              int box_rows) {
  const auto fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)(ld * size), (cuuint64_t)(ld * rows * size)};
  cuuint32_t box[3] = {(cuuint32_t)(128 / size), (cuuint32_t)box_rows, 1}, estr[3] = {1, 1, 1};
  return fn(map, size == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<void*>(p),
            dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// dbias as a product with ones takes the second half of TMEM, so that the unit that does it does nothing else
// meanwhile.  Where a tile's columns are a small part of dW the other units would wait for that one: then two
// kernels add g up (dW of 32,768 rows, 1024 x 4096: 328 us with the product, 205 without, 229 with the kernels).
// Up to two tiles of columns are at most 64 tiles (8192 rows of dW): one unit a pair, on all but small parts of a device.
inline bool sums_apart(const TcArgs& g) { return g.n_tiles > 2 || g.units > num_sms() / 2; }
// After the product: dbias by the kernels, and the join of split sums.
inline cudaError_t finish(const TcArgs& g, const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch,
                          int ld, cudaStream_t st) {
  LinearEnd end = e;
  if (p.op == kLinDw && e.sums && sums_apart(g)) {
    float* part = reinterpret_cast<float*>(static_cast<char*>(scratch) + align_up(plan.part, 256));
    const cudaError_t err = linear_sums(p, ld, part, e, st);
    if (err != cudaSuccess) return err;
    end.sums = nullptr;
  }
  if (plan.splits == 1) return cudaSuccess;
  return linear_join(p, plan.splits, static_cast<const float*>(scratch), g.part_sums, end, st);
}

// What both kinds of product need from their problem.  false: no tensor map, or a plan that is not for this device.
inline bool fill_args(TcArgs& g, const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch) {
  const bool f32 = p.dtype == FS_F32, split = plan.splits > 1, dw = p.op == kLinDw;
  g.e = e;
  g.M = p.M, g.N = p.N, g.K = p.K, g.per = plan.per, g.splits = plan.splits;
  g.a_mn = dw, g.b_mn = p.op != kLinFwd;
  g.bn = linear_tile_n(p.N, g.b_mn, f32);
  g.n_tiles = (p.N + g.bn - 1) / g.bn;
  g.tiles = (int)((p.M + 255) / 256) * g.n_tiles;
  g.units = g.tiles * plan.splits;
  if (split && g.units > num_sms() / 2) return false;  // Unit::next does not step from part to part
  const int pairs = std::min(g.units, num_sms() / 2);
  g.step_n = pairs % g.n_tiles, g.step_m = pairs / g.n_tiles;
  g.idesc = idesc_bf16(256, g.bn, g.a_mn, g.b_mn);
  g.idesc_sum = idesc_bf16(256, 32, g.a_mn, false);
  g.a_step = g.a_mn ? 128 : 2, g.b_step = g.b_mn ? 128 : 2;
  g.status = p.status, g.reset = p.reset;
  const int size = split || dw || f32 ? 4 : 2;
  float* part = static_cast<float*>(scratch);
  g.ldy = p.N;
  if (split) {
    g.ldy = (p.N + 3) & ~3;
    g.e.y = part;
    g.part_sums = part + (int64_t)plan.splits * p.M * g.ldy;
  } else {
    g.load_res = dw ? e.accumulate != 0 : e.res != nullptr;
    if (dw) g.e.res = e.y;
    g.load_pre = p.op == kLinDx && e.act != FS_ACT_NONE;
    g.store_pre = e.pre_out != nullptr;
  }
  if (f32 && !dw && !split && (g.store_pre || (g.load_pre && g.load_res))) {
    g.pre_at_rows = 1;
    g.load_pre = g.store_pre = 0;
  }
  g.sums = dw && e.sums && !sums_apart(g);
  // Segments: where results are fp32, 256 terms of three parts; 512 of one, 1024 where dbias keeps the products
  // waiting while a segment is taken out (bwd of 1,048,576 x 256 x 256 444 -> 430 us; by norm, terms of random sign are off
  // by 9.9e-7 then, 4.9e-7 in segments of 512).
  g.seg = split || dw || f32 ? (f32 ? 4 : g.sums ? 16 : 8) : 1 << 30;
  g.plain = g.ldy * size % 16 != 0;
  if (g.plain) return true;
  bool ok = make_map(&g.y, g.e.y, size, g.ldy, p.M, plan.splits, g.ldy, 32);
  if (g.load_res) ok = ok && make_map(&g.res, g.e.res, size, g.ldy, p.M, 1, g.ldy, 32);
  if (g.load_pre) ok = ok && make_map(&g.pre, e.pre_in, size, g.ldy, p.M, 1, g.ldy, 32);
  if (g.store_pre) ok = ok && make_map(&g.pre, e.pre_out, size, g.ldy, p.M, 1, g.ldy, 32);
  return ok;
}

}  // namespace
}  // namespace fs
