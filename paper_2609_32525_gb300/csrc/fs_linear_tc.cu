// Linear maps on tcgen05: D[m, n] = sum_k A[m, k] B[n, k] in bf16 products with fp32 accumulation,
// and all that follows the product.
//
// Work.  Two CTAs of a cluster share a tile of 256 x (64 to 256) values of D: each holds 128 of
// A's rows and half of B's, so that an operand byte is loaded once for 256 rows of the other one,
// and the leader issues products of 256 x n x 16 for both (cta_group::2).  Pairs are persistent and
// walk over units (tile, part of the sum); while a unit's epilogue runs, the next one's products
// go to the other half of TMEM.
//   warp 0       TMA loads of A and B, 64 terms at a time, into a ring of 128-byte-swizzled stages
//   warp 1       TMEM, products (leader)
//   warps 2 on   epilogue: 32 rows each, columns shared between two or three warpgroups; a residual or
//                pre-activation comes by TMA into the 32 x 128 byte box that the result leaves
//                from, so all traffic with HBM is in whole 128-byte lines
// x and W lie with their terms next to each other (K-major), W in dx and both operands of dW with
// their rows or columns of D next to each other (MN-major): the descriptors say so, nothing is
// transposed.
//
// Precision.  The tensor core cuts its accumulator towards zero at every step.  bf16 results do
// not see that; fp32 results (dW, split sums, fp32 rows) are taken out of TMEM every few hundred
// terms and added up in registers.  fp32 operands come as three bf16 parts (k_linear_pack: hi, mid, lo
// leave out less than 2^-26 of a value) and six products of parts; the five small ones have an
// accumulator of their own.  dbias, the sum of g over its rows, is a product with ones.
//
// Rows whose pitch TMA cannot address (a multiple of 16 bytes) are copied to one that it can
// (k_linear_pack), and results of such a pitch leave by plain stores.
#include "fs_internal.h"
#include "fs_launch.h"
#include "fs_linear_end.cuh"
#include "fs_tc_pair.cuh"

#include <algorithm>
#include <cudaTypedefs.h>
#include <mutex>

namespace fs {
namespace {

using namespace tc;

constexpr int kMaxStages = 12;
constexpr uint32_t kABytes = 128 * 128;          // 128 rows (or 64 terms x 128) of 64 values
constexpr uint32_t kBox = 32 * 128;              // an epilogue warp's box
constexpr uint32_t kOnes = 1024;
constexpr size_t kSmem = 231424;                 // with the barriers below the limit of a block
constexpr uint32_t kSumCol = 256;                // dbias' accumulator
// Epilogue warpgroups and boxes of a warp; what the boxes leave for the stages.
template <int kGroups, int kPer>
struct Block {
  static constexpr int kThreads = 64 + 128 * kGroups;
  static constexpr uint32_t kBoxes = kGroups * 4 * kPer * kBox, kStageRoom = kSmem - 1024 - kOnes - kBoxes;
};
// Where sums are short the epilogue is the work: five warpgroups with one box each.  Where they are long, or a
// chunk has two inputs or results, three with two boxes.  (1,048,576 x 256 x 256 with dropout and residual:
// 361 us against 404 with three groups; 32,768 x 1024 x 4096 173 us with three against 183 with five.)
constexpr int kManyGroups = 5, kShortK = 512;

enum { kEndFwd = 0, kEndDx = 1, kEndRaw = 2 };

struct TcArgs {
  CUtensorMap a, b, y, pre, res;
  LinearEnd e;
  int64_t M, K, per;
  int N, ldy, n_tiles, m_tiles, tiles, units, bn, splits, stages, seg;  // ldy: pitch of y; seg: blocks of 64 terms taken out at a time
  int step_n, step_m, step_split;                       // from a pair's unit to its next one
  uint32_t stage_bytes, idesc, idesc_sum, a_step, b_step;  // steps: 16 terms on in a stage, in 16-byte units
  int a_mn, b_mn;
  int load_res, load_pre, store_pre, plain;             // plain: y, res and pre by plain accesses
  const char* ahead;                                    // null, or A to prefetch to L2 a tile ahead, in whole rows
  int sums;                                             // dbias is wanted
  float* part_sums;                                     // split: [splits][M]
  uint32_t* status;
  int reset;
};

// The units of a pair, number `pair` and every pairs-th one after it; stepped, not divided, since an epilogue
// warp's few hundred instructions a chunk run one after another.
struct Unit {
  int m, n, split;
  int left;  // units from this one on, 0 or less: none
  __device__ __forceinline__ Unit(const TcArgs& g, int u) : left(g.units - u) {
    split = u / g.tiles;
    const int t = u - split * g.tiles;
    m = t / g.n_tiles;
    n = t - m * g.n_tiles;
  }
  __device__ __forceinline__ void next(const TcArgs& g, int pairs) {
    left -= pairs;
    n += g.step_n;
    m += g.step_m;
    split += g.step_split;
    if (n >= g.n_tiles) n -= g.n_tiles, m++;
    if (m >= g.m_tiles) m -= g.m_tiles, split++;
  }
  __device__ __forceinline__ int64_t k0(const TcArgs& g) const { return split * g.per; }
  __device__ __forceinline__ int blocks(const TcArgs& g) const {
    const int64_t k = g.K - k0(g) < g.per ? g.K - k0(g) : g.per;
    return (int)((k + 63) >> 6);
  }
};

// Which half of TMEM a segment's products go to.  Units with dbias use the first half for all and
// columns of the second one for the sums; the others take turns.
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

// What the end of a map does: dropout (counters of 32 or of 64 bits) and a residual.
enum { kNoDrop = 0, kDrop32 = 1, kDrop64 = 2 };

// The end of a map on 16 neighbouring columns of a row, step by step for all of them, so that the
// chains of 16 values (4 counters) are under way at once.  quad: the first one's counter.
template <int END, typename T, int DROP, bool kRes, typename Q>
__device__ __forceinline__ void end16(const TcArgs& g, const act::DropKey& key, Q quad, int col, int piece0, uint32_t yline,
                                      uint32_t pline, float (&v)[16]) {
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
    act::apply<kFast>(g.e.act, v);
  }
  if constexpr (END == kEndDx) {
    if (g.load_pre) {
      float u[16];
      Line<T>::load(pline, piece0, u);
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
__device__ __forceinline__ void end_loop(const TcArgs& g, const act::DropKey& key, Q quad, int col, uint32_t yline,
                                         uint32_t pline, F&& f) {
  // (results that are in registers already need constant indexes)
#pragma unroll(sizeof(T) == 2 ? 1 : n)
  for (int i = 0; i < n; i++) {
    float v[16];
    f(v, i);
    end16<END, T, DROP, kRes>(g, key, (Q)(quad + 4 * i), col + 16 * i, Line<T>::kPieces * i, yline, pline, v);
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
      if (g.load_res) end_loop<END, T, END != kEndRaw ? kDrop32 : 0, true, n>(g, key, q, col, yline, pline, f);
      else end_loop<END, T, END != kEndRaw ? kDrop32 : 0, false, n>(g, key, q, col, yline, pline, f);
    } else {
      if (g.load_res) end_loop<END, T, END != kEndRaw ? kDrop64 : 0, true, n>(g, key, quad, col, yline, pline, f);
      else end_loop<END, T, END != kEndRaw ? kDrop64 : 0, false, n>(g, key, quad, col, yline, pline, f);
    }
  } else {
    if (g.load_res) end_loop<END, T, kNoDrop, true, n>(g, key, 0u, col, yline, pline, f);
    else end_loop<END, T, kNoDrop, false, n>(g, key, 0u, col, yline, pline, f);
  }
}

// A box between shared memory and rows that TMA cannot address, by a warp.
template <typename T>
__device__ __forceinline__ void box_by_lanes(T* rows, int64_t ld, int64_t M, int N, int64_t row0, int col0, uint32_t box,
                                             bool load) {
  constexpr int kCols = 128 / sizeof(T), kV = 16 / sizeof(T);
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int c = lane; c < kCols; c += 32) {
    if (col0 + c >= N) continue;
#pragma unroll 8
    for (int r = 0; r < 32; r++) {
      if (row0 + r >= M) continue;
      T* p = rows + (row0 + r) * ld + col0 + c;
      const uint32_t at = box + r * 128 + (((c / kV) ^ (r & 7)) << 4) + (c % kV) * (int)sizeof(T);
      if constexpr (sizeof(T) == 2) {
        unsigned short w;
        if (load) {
          w = *reinterpret_cast<const unsigned short*>(p);
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"(w) : "memory");
        } else {
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(at) : "memory");
          *reinterpret_cast<unsigned short*>(p) = w;
        }
      } else {
        float w;
        if (load) {
          w = *reinterpret_cast<const float*>(p);
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(w) : "memory");
        } else {
          asm volatile("ld.shared.f32 %0, [%1];" : "=f"(w) : "r"(at) : "memory");
          *reinterpret_cast<float*>(p) = w;
        }
      }
    }
  }
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
    if (!loads || g.plain) return;
    if ((threadIdx.x & 31) == 0) {
      bulk_wait_read<0>();
      const int b = serial ? 0 : (turn + ahead) & 1;
      mbar_expect_tx(&bar[b], loads * kBox);
      const uint32_t box = base + b * kBox;
      if (g.load_res) load(box, &g.res, col, (int)row, &bar[b]);
      if (g.load_pre) load(both ? box + kBox : box, &g.pre, col, (int)row, &bar[b]);
    }
    __syncwarp();
  }
  __device__ __forceinline__ void load(uint32_t box, const CUtensorMap* map, int c0, int c1, uint64_t* full) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(box),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(0), "r"(smem_u32(full))
        : "memory");
  }
  // Before the chunk's box is read and written.
  __device__ __forceinline__ bool ready(int64_t row, int col, Abort* ab, uint32_t* status) {
    if (g.plain) {
      const LinearEnd& e = g.e;
      if (g.load_res) box_by_lanes<T>(const_cast<T*>(static_cast<const T*>(e.res)), g.ldy, g.M, g.N, row, col, ybox(), true);
      if (g.load_pre) box_by_lanes<T>(const_cast<T*>(static_cast<const T*>(e.pre_in)), g.ldy, g.M, g.N, row, col, pbox(), true);
      __syncwarp();
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

template <int END, typename T, int PARTS, int kGroups, int kPer>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Block<kGroups, kPer>::kThreads, 1) k_linear_tc(const __grid_constant__ TcArgs g) {
  constexpr bool kFlush = sizeof(T) == 4;  // fp32 results
  using B = Block<kGroups, kPer>;
  extern __shared__ __align__(1024) uint8_t raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], drain, in_full[4 * kGroups][2];
  __shared__ uint32_t tmem_slot;
  __shared__ Abort abort_;
  uint8_t* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  const uint32_t stage0 = smem_u32(smem), boxes = stage0 + B::kStageRoom, ones = boxes + B::kBoxes;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  Abort* ab = &abort_;

  if (tid == 0) {
    abort_.flag = 0;
    for (int i = 0; i < kMaxStages; i++) mbar_init(&full[i], 1), mbar_init(&empty[i], 1);
    for (int i = 0; i < 2; i++) mbar_init(&acc_full[i], 1), mbar_init(&acc_empty[i], 8 * kGroups);
    for (int i = 0; i < 8 * kGroups; i++) mbar_init(&in_full[i >> 1][i & 1], 1);
    mbar_init(&drain, 1);
    fence_mbar_init();
  }
  if (tid < (int)kOnes / 16) st_shared_v4(ones + tid * 16, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
  fence_proxy_async_smem();
  if (warp == 1) tmem_alloc_pair(&tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  pair_sync();
  tc_fence_after();
  grid_trigger();
  const int64_t zero = grid_wait();
  const uint32_t tmem = tmem_slot;
  uint32_t* status = g.status + zero;
  if (g.reset && blockIdx.x == 0 && tid == 0) *status = 0;

  if (warp == 0) {
    if (lane == 0) {
      prefetch_tmap(&g.a);
      prefetch_tmap(&g.b);
      RingOf ring(g.stages);
      const uint32_t bar0 = leader_addr(&full[0]);
      const int bhalf = g.bn >> 1;
      uint32_t issued = 0;
      bool ok = true;
      for (Unit w(g, pair); w.left > 0 && ok; w.next(g, pairs)) {
        const int m = w.m * 256 + (int)rank * 128, n = w.n * g.bn + (int)rank * bhalf, blocks = w.blocks(g);
        const int64_t k0 = w.k0(g);
        Unit nw = w;
        nw.next(g, pairs);
        if (g.ahead && nw.left > 0) {
          // A's rows lie next to each other: they come from HBM in one piece, not in the 128-byte columns that the
          // stages take.
          const int64_t row = (int64_t)nw.m * 256 + rank * 128, rows = g.M - row < 128 ? g.M - row : 128;
          if (rows > 0) bulk_prefetch(g.ahead + zero + row * g.K * 2, (uint32_t)(rows * g.K * 2));
        }
        for (int s = 0; s < blocks * PARTS; s++) {
          const int kb = s / PARTS, part = s - kb * PARTS;
          if (!mbar_wait(&empty[ring.i], ring.pass ^ 1u, ab, status)) {
            ok = false;
            break;
          }
          if (rank == 0) mbar_expect_tx(&full[ring.i], 2 * g.stage_bytes);
          const uint32_t bar = bar0 + 8 * ring.i, a = stage0 + ring.i * g.stage_bytes, b = a + kABytes;
          const int k = (int)(k0 + (int64_t)kb * 64);
          if (g.a_mn) {
            tma_load_pair(a, &g.a, m, k, part, bar);
            tma_load_pair(a + 8192, &g.a, m + 64, k, part, bar);
          } else {
            tma_load_pair(a, &g.a, k, m, part, bar);
          }
          if (g.b_mn) {
            for (int j = 0; j < bhalf; j += 64) tma_load_pair(b + j * 128, &g.b, n + j, k, part, bar);
          } else {
            tma_load_pair(b, &g.b, k, n, part, bar);
          }
          ring.next();
          issued++;
        }
      }
      // The stages' last products are behind this CTA too before its barriers go: the leader's commits
      // arrive at them.
      for (uint32_t j = issued > (uint32_t)g.stages ? issued - g.stages : 0; ok && j < issued; j++)
        mbar_drain(&empty[j % g.stages], (j / g.stages) & 1u);
    }
  } else if (warp == 1) {
    if (rank == 0) {
      RingOf ring(g.stages);
      Halves h;
      bool ok = true, last_sums = false;
      const uint32_t a_lo0 = sdesc_lo(stage0, g.a_mn ? 8192 : 16), b_lo0 = sdesc_lo(stage0 + kABytes, g.b_mn ? 8192 : 16);
      const uint32_t ones_lo = sdesc_lo(ones, 128), stage_step = g.stage_bytes >> 4;
      for (Unit w(g, pair); w.left > 0 && ok; w.next(g, pairs)) {
        const bool sums = g.sums && w.n == 0;
        const int blocks = w.blocks(g);
        for (int kb = 0; kb < blocks && ok; kb += g.seg) {
          const int half = h.pick(sums), end = min(kb + g.seg, blocks);
          ok = mbar_wait_pair_w(&acc_empty[half], (h.uses(half) & 1u) ^ 1u, ab, status);
          // Into or out of a unit with sums, the other half has to be read out as well.
          if (ok && sums != last_sums && h.uses(half ^ 1))
            ok = mbar_wait_pair_w(&acc_empty[half ^ 1], (h.uses(half ^ 1) - 1) & 1u, ab, status);
          if (!ok) break;
          last_sums = sums;
          h.use(half);
          tc_fence_after();
          const uint32_t d = tmem + half * 256, d_small = d + 128;
          for (int b = kb; b < end && ok; b++) {
            if constexpr (PARTS == 1) {
              ok = mbar_wait_w(&full[ring.i], ring.pass, ab, status);
              if (!ok) break;
              tc_fence_after();
              const uint32_t a_lo = a_lo0 + ring.i * stage_step, b_lo = b_lo0 + ring.i * stage_step;
#pragma unroll
              for (int k = 0; k < 4; k++) {
                mma_pair_w<kHi128, kHi128>(d, a_lo + k * g.a_step, b_lo + k * g.b_step, g.idesc, b > kb || k);
                if (sums) mma_pair_w<kHi128, kHi32>(tmem + kSumCol, a_lo + k * g.a_step, ones_lo, g.idesc_sum, b > kb || k);
              }
              mma_commit_pair_w(&empty[ring.i]);
              ring.next();
            } else {
              uint32_t a_lo[3], b_lo[3];
              int slot[3];
#pragma unroll
              for (int p = 0; p < 3; p++) {
                ok = ok && mbar_wait_w(&full[ring.i], ring.pass, ab, status);
                if (!ok) break;
                tc_fence_after();
                slot[p] = ring.i;
                a_lo[p] = a_lo0 + ring.i * stage_step, b_lo[p] = b_lo0 + ring.i * stage_step;
                ring.next();
#pragma unroll
                for (int k = 0; k < 4; k++) {
                  const uint32_t more = b > kb || k;
                  auto mul = [&](uint32_t to, int i, int j, uint32_t add) {
                    mma_pair_w<kHi128, kHi128>(to, a_lo[i] + k * g.a_step, b_lo[j] + k * g.b_step, g.idesc, add);
                  };
                  if (p == 0) mul(d, 0, 0, more);
                  if (p == 1) mul(d_small, 0, 1, more), mul(d_small, 1, 0, 1), mul(d_small, 1, 1, 1);
                  if (p == 2) mul(d_small, 0, 2, 1), mul(d_small, 2, 0, 1);
                  if (sums)
                    mma_pair_w<kHi128, kHi32>(tmem + kSumCol, a_lo[p] + k * g.a_step, ones_lo, g.idesc_sum, more || p);
                }
              }
              if (!ok) break;
#pragma unroll
              for (int p = 0; p < 3; p++) mma_commit_pair_w(&empty[slot[p]]);
            }
          }
          mma_commit_pair_w(&acc_full[half]);
        }
      }
      // No product is left under way.
      mma_commit_leader_w(&drain);
      mbar_drain_w(&drain, 0);
    }
  } else {
    const int e = warp - 2, wg = e >> 2, sub = warp & 3;
    const uint32_t lanes = tmem + ((uint32_t)(sub * 32) << 16), free0 = leader_addr(&acc_empty[0]);
    Boxes<END, T, kPer> box(g, boxes + e * kPer * kBox, in_full[e]);
    const act::DropKey key = lin::drop_key(g.e);
    Halves h;
    bool ok = true;
    auto row_of = [&](const Unit& w) { return (int64_t)w.m * 256 + rank * 128 + sub * 32; };
    auto release = [&](int half) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_leader(free0 + 8 * half);
    };
    if constexpr (!kFlush) {
      // The pair's tiles as one sequence of chunks of 64 columns, which the warpgroups take in turn.
      const int chunks = g.bn >> 6;
      auto place = [&](Unit& w, int& c) {  // from a chunk number past the unit's to the unit that it is in
        while (c >= chunks) c -= chunks, w.next(g, pairs);
      };
      int c = wg, nc = wg;
      Unit nw(g, pair);  // (nw, nc): the chunk whose loads start next
      place(nw, nc);
      auto start_next = [&](int ahead) {
        if (nw.left > 0) box.start(ahead, row_of(nw), nw.n * g.bn + nc * 64);
        nc += kGroups;
        place(nw, nc);
      };
      if (box.loads) start_next(0);
      for (Unit w(g, pair); w.left > 0 && ok; w.next(g, pairs)) {
        const int64_t row0 = row_of(w);
        const int half = h.pick(false);
        ok = mbar_wait_w(&acc_full[half], h.uses(half) & 1u, ab, status);
        if (!ok) break;
        h.use(half);
        tc_fence_after();
        if (c >= chunks) release(half);
        for (; c < chunks && ok; c += kGroups) {
          const int col = w.n * g.bn + c * 64;
          if (box.loads && !box.serial) start_next(1);
          ok = box.ready(row0, col, ab, status);
          if (!ok) break;
          const uint32_t from = lanes + half * 256 + c * 64;
          end_chunk<END, T, 4>(g, key, row0 + lane, col, box.ybox() + lane * 128, box.pbox() + lane * 128,
                               [&](float(&v)[16], int i) {
                                 uint32_t r[16];
                                 tmem_ld16(from + 16 * i, r);
                                 tmem_wait_ld(r);
                                 if (i == 3 && c + kGroups >= chunks) release(half);
#pragma unroll
                                 for (int j = 0; j < 16; j++) v[j] = __uint_as_float(r[j]);
                               });
          box.send(row0, col, w.split);
          if (box.loads && box.serial) start_next(1);
        }
        c -= chunks;
      }
    } else {
      // The warpgroups take half of a tile's columns each and add its segments up in registers.
      constexpr int kMost = PARTS == 1 ? 4 : 2;
      const int chunks = g.bn >> 6, first = wg * (g.bn >> 1);
      for (Unit w(g, pair); w.left > 0 && ok; w.next(g, pairs)) {
        const int64_t row0 = row_of(w);
        const int col = w.n * g.bn + first, blocks = w.blocks(g);
        const bool sums = g.sums && w.n == 0;
        float acc[kMost][32], sum = 0.f;
        box.start(0, row0, col);
        for (int kb = 0; kb < blocks && ok; kb += g.seg) {
          const int half = h.pick(sums);
          ok = mbar_wait_w(&acc_full[half], h.uses(half) & 1u, ab, status);
          if (!ok) break;
          h.use(half);
          tc_fence_after();
          const uint32_t t = lanes + half * 256 + first;
#pragma unroll
          for (int i = 0; i < kMost; i++) {
            if (i >= chunks) continue;
            uint32_t r[32];
            tmem_ld32(t + i * 32, r);
            if constexpr (PARTS == 3) {
              uint32_t s[32];
              tmem_ld32(t + 128 + i * 32, s);
              tmem_wait_ld2(r, s);
#pragma unroll
              for (int j = 0; j < 32; j++) r[j] = __float_as_uint(__uint_as_float(r[j]) + __uint_as_float(s[j]));
            } else {
              tmem_wait_ld(r);
            }
            if (kb == 0) {
#pragma unroll
              for (int j = 0; j < 32; j++) acc[i][j] = __uint_as_float(r[j]);
            } else {
#pragma unroll
              for (int j = 0; j < 32; j++) acc[i][j] += __uint_as_float(r[j]);
            }
          }
          if (END == kEndRaw && sums && wg == 0) {
            uint32_t r[16];
            tmem_ld16(lanes + kSumCol, r);
            tmem_wait_ld(r);
            sum += __uint_as_float(r[0]);
          }
          release(half);
        }
        if (!ok) break;
        if (END == kEndRaw && sums && wg == 0 && row0 + lane < g.M) {
          if (g.splits > 1) g.part_sums[(int64_t)w.split * g.M + row0 + lane] = sum;
          else lin::end_sum(g.e, row0 + lane, sum);
        }
#pragma unroll
        for (int i = 0; i < kMost; i++) {
          if (i >= chunks || !ok) continue;
          if (!box.serial && i + 1 < chunks) box.start(1, row0, col + (i + 1) * 32);
          ok = box.ready(row0, col + i * 32, ab, status);
          if (!ok) continue;
          end_chunk<END, T, 2>(g, key, row0 + lane, col + i * 32, box.ybox() + lane * 128, box.pbox() + lane * 128,
                               [&](float(&v)[16], int h) {
#pragma unroll
                                 for (int j = 0; j < 16; j++) v[j] = acc[i][16 * h + j];
                               });
          box.send(row0, col + i * 32, w.split);
          if (box.serial && i + 1 < chunks) box.start(1, row0, col + (i + 1) * 32);
        }
      }
    }
    if (lane == 0) bulk_wait_all();  // the results are written before the next kernel's wait ends
  }
  // A CTA that gave up may have copies on their way that count on barriers whose phase never ends (the other
  // CTA's part is missing): they land in microseconds, and a hundred times that is waited for them.
  __syncwarp();
  if (ab->flag) {
    const uint64_t t0 = globaltimer();
    for (uint32_t i = 0; i < 1000000u && globaltimer() - t0 < 2000000ull; i++) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  pair_sync();
  tc_fence_after();
  if (warp == 1) tmem_dealloc_pair(tmem, 512);
}

// ---- operands that TMA can address -----------------------------------------------------------
//
// fp32 rows as three bf16 parts, and bf16 rows of an odd pitch as they are, with a pitch of whole 16
// bytes: 8 columns a thread.  Rounding to nearest leaves at most 2^-9 of a value to the next part, so hi, mid and lo
// leave 2^-27; a value that would round to infinity is cut instead,
// and an infinity has no further parts.
struct PackJob {
  const void* src;
  __nv_bfloat16* dst;
  int64_t rows, threads;
  int C, ld;  // ld: the pitch of dst, C rounded up to 8; its last columns are 0
};
struct PackArgs {
  PackJob job[3];
  int jobs;
  uint32_t* status;
};

__device__ __forceinline__ void parts_of(float x, unsigned short (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 3; i++) {
    __nv_bfloat16 b = __float2bfloat16_rn(x);
    if (i == 0 && fabsf(__bfloat162float(b)) == INFINITY) b = __float2bfloat16_rz(x);
    p[i] = __bfloat16_as_ushort(b);
    x = fabsf(x) == INFINITY ? 0.f : x - __bfloat162float(b);
  }
}

template <typename T>
__global__ void __launch_bounds__(256) k_linear_pack(PackArgs a) {
  const int64_t zero = grid_begin();
  if (blockIdx.x == 0 && threadIdx.x == 0) a.status[zero] = 0;
  int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  int n = 0;
  while (n < a.jobs && i >= a.job[n].threads) i -= a.job[n++].threads;
  if (n == a.jobs) return;
  const PackJob& j = a.job[n];
  const int pieces = j.ld >> 3;
  const int64_t row = i / pieces;
  if (row >= j.rows) return;
  const int col = (int)(i - row * pieces) * 8, left = j.C - col;
  const T* src = static_cast<const T*>(j.src) + row * j.C + col;
  T v[8];
  if (sizeof(T) == 4 && (j.C & 3) == 0 && left >= 8) {
    reinterpret_cast<float4*>(v)[0] = reinterpret_cast<const float4*>(src)[0];
    reinterpret_cast<float4*>(v)[1] = reinterpret_cast<const float4*>(src)[1];
  } else {
#pragma unroll
    for (int k = 0; k < 8; k++) v[k] = k < left ? src[k] : T(0.f);
  }
  __nv_bfloat16* dst = j.dst + row * j.ld + col;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(v);
  } else {
    unsigned short p[8][3];
#pragma unroll
    for (int k = 0; k < 8; k++) parts_of(v[k], p[k]);
#pragma unroll
    for (int q = 0; q < 3; q++) {
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; k++) w[k] = (uint32_t)p[2 * k][q] | ((uint32_t)p[2 * k + 1][q] << 16);
      *reinterpret_cast<uint4*>(dst + q * j.rows * j.ld) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
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

template <int END, typename T, int PARTS, int kGroups, int kPer>
cudaError_t run(TcArgs& g, cudaStream_t st) {
  using B = Block<kGroups, kPer>;
  const auto k_tc = k_linear_tc<END, T, PARTS, kGroups, kPer>;
  g.stages = std::min<int>(kMaxStages, (int)(B::kStageRoom / g.stage_bytes));
  cudaError_t e = allow_smem<kSmem>(k_tc);
  if (e != cudaSuccess) return e;
  const int pairs = std::min(g.units, num_sms() / 2);
  return launch(k_tc, dim3((unsigned)(2 * pairs)), dim3(B::kThreads), kSmem, st, g);
}

}  // namespace

int linear_tile_n(int N, bool b_mn, bool f32) {
  const int most = f32 ? 128 : 256, tiles = (N + most - 1) / most, step = b_mn ? 128 : 64;
  return ((N + tiles - 1) / tiles + step - 1) / step * step;
}

cudaError_t linear_pack(const LinearPack* packs, int n, int dtype, uint32_t* status, cudaStream_t st) {
  PackArgs a{};
  a.status = status;
  int64_t threads = 0;
  for (int i = 0; i < n; i++) {
    PackJob& j = a.job[a.jobs++];
    j.src = packs[i].src;
    j.dst = static_cast<__nv_bfloat16*>(packs[i].dst);
    j.rows = packs[i].rows;
    j.C = packs[i].C;
    j.ld = linear_pitch(j.C);
    j.threads = (j.rows * (j.ld >> 3) + 255) / 256 * 256;
    threads += j.threads;
  }
  const dim3 grid((unsigned)(threads / 256));
  return dtype == FS_BF16 ? launch(k_linear_pack<__nv_bfloat16>, grid, dim3(256), 0, st, a)
                          : launch(k_linear_pack<float>, grid, dim3(256), 0, st, a);
}

cudaError_t linear_tc(const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch, cudaStream_t st) {
  const bool f32 = p.dtype == FS_F32, split = plan.splits > 1, dw = p.op == kLinDw;
  const int parts = f32 ? 3 : 1;
  TcArgs g{};
  g.e = e;
  g.M = p.M, g.N = p.N, g.K = p.K, g.per = plan.per, g.splits = plan.splits;
  g.a_mn = dw, g.b_mn = p.op != kLinFwd;
  g.bn = linear_tile_n(p.N, g.b_mn, f32);
  g.n_tiles = (p.N + g.bn - 1) / g.bn;
  g.m_tiles = (int)((p.M + 255) / 256);
  g.tiles = g.m_tiles * g.n_tiles;
  g.units = g.tiles * plan.splits;
  const int pairs = std::min(g.units, num_sms() / 2);
  g.step_n = pairs % g.n_tiles, g.step_m = pairs / g.n_tiles % g.m_tiles, g.step_split = pairs / g.tiles;
  g.stage_bytes = kABytes + (uint32_t)g.bn / 2 * 128;
  const bool raw = split || dw;
  // Segments: where results are fp32, 256 terms of three parts, 512 of one.
  g.seg = split || dw || f32 ? (f32 ? 4 : 8) : 1 << 30;
  g.idesc = idesc_bf16(256, g.bn, g.a_mn, g.b_mn);
  g.idesc_sum = idesc_bf16(256, 32, g.a_mn, false);
  g.a_step = g.a_mn ? 128 : 2, g.b_step = g.b_mn ? 128 : 2;
  g.status = p.status, g.reset = p.reset;
  const int lda = linear_pitch((int)(g.a_mn ? p.M : p.K)), ldb = linear_pitch((int)(g.b_mn ? p.N : p.K));
  bool ok = g.a_mn ? make_map(&g.a, p.a, 2, p.M, p.K, parts, lda, 64) : make_map(&g.a, p.a, 2, p.K, p.M, parts, lda, 128);
  ok = ok && (g.b_mn ? make_map(&g.b, p.b, 2, p.N, p.K, parts, ldb, 64) : make_map(&g.b, p.b, 2, p.K, p.N, parts, ldb, g.bn / 2));
  const int size = raw || f32 ? 4 : 2;
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
  g.sums = dw && e.sums;
  if (g.n_tiles == 1 && !split && !dw && !f32 && p.K % 8 == 0) g.ahead = static_cast<const char*>(p.a);
  g.plain = g.ldy * size % 16 != 0;
  if (!g.plain) {
    ok = ok && make_map(&g.y, g.e.y, size, g.ldy, p.M, plan.splits, g.ldy, 32);
    if (g.load_res) ok = ok && make_map(&g.res, g.e.res, size, g.ldy, p.M, 1, g.ldy, 32);
    if (g.load_pre) ok = ok && make_map(&g.pre, e.pre_in, size, g.ldy, p.M, 1, g.ldy, 32);
    if (g.store_pre) ok = ok && make_map(&g.pre, e.pre_out, size, g.ldy, p.M, 1, g.ldy, 32);
  }
  if (!ok) return cudaErrorInvalidValue;
  cudaError_t err;
  using B = __nv_bfloat16;
  const bool few = g.store_pre || (g.load_res && g.load_pre) || p.K > kShortK;
  if (raw) err = f32 ? run<kEndRaw, float, 3, 2, 2>(g, st) : run<kEndRaw, float, 1, 2, 2>(g, st);
  else if (p.op == kLinFwd)
    err = f32    ? run<kEndFwd, float, 3, 2, 2>(g, st)
          : few  ? run<kEndFwd, B, 1, 3, 2>(g, st)
                 : run<kEndFwd, B, 1, kManyGroups, 1>(g, st);
  else
    err = f32    ? run<kEndDx, float, 3, 2, 2>(g, st)
          : few  ? run<kEndDx, B, 1, 3, 2>(g, st)
                 : run<kEndDx, B, 1, kManyGroups, 1>(g, st);
  if (err != cudaSuccess || !split) return err;
  return linear_join(p, plan.splits, part, g.part_sums, e, st);
}

}  // namespace fs
