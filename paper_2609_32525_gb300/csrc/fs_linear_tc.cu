// Linear maps of bf16 rows on tcgen05 (see fs_linear_tc.cuh).
//   warp 0       TMA loads of A and B, 64 terms at a time, into a ring of 128-byte-swizzled stages
//   warp 1       TMEM, products (leader)
//   warps 2 on   epilogue
// x and W lie with their terms next to each other (K-major), W in dx and both operands of dW with
// their rows or columns of D next to each other (MN-major): the descriptors say so, nothing is
// transposed.  Rows whose pitch TMA cannot address (a multiple of 16 bytes) are copied to one that
// it can first (k_linear_pack).
#include "fs_linear_tc.cuh"

namespace fs {
namespace {

// Where sums are short the epilogue is the work: five warpgroups with one box each.  Where they are long, or a
// chunk has two inputs or results, three with two boxes.  (1,048,576 x 256 x 256 with dropout and residual:
// 353 us; with four groups 384, with six 359, with three and their two boxes 383 before the others had a box fewer.
// 32,768 x 1024 x 4096: 173 us with three against 183 with five.)
constexpr int kManyGroups = 5, kShortK = 512;

// T: float for dW and split sums.
template <int END, typename T, int kGroups, int kPer>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Block<kGroups, kPer>::kThreads, 1)
    k_linear_bf16(const __grid_constant__ TcArgs g) {
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
        const int64_t k0 = w.k0();
        Unit nw = w;
        nw.next(g, pairs);
        if (g.ahead && nw.left > 0) {
          // A's rows lie next to each other: they come from HBM in one piece, not in the 128-byte columns that the
          // stages take.
          const int64_t row = (int64_t)nw.m * 256 + rank * 128, rows = g.M - row < 128 ? g.M - row : 128;
          if (rows > 0) bulk_prefetch(g.ahead + zero + row * g.K * 2, (uint32_t)(rows * g.K * 2));
        }
        for (int kb = 0; kb < blocks; kb++) {
          if (!mbar_wait(&empty[ring.i], ring.pass ^ 1u, ab, status)) {
            ok = false;
            break;
          }
          if (rank == 0) mbar_expect_tx(&full[ring.i], 2 * g.stage_bytes);
          const uint32_t bar = bar0 + 8 * ring.i, a = stage0 + ring.i * g.stage_bytes, b = a + kABytes;
          const int k = (int)(k0 + (int64_t)kb * 64);
          if (g.a_mn) {
            tma_load_pair(a, &g.a, m, k, 0, bar);
            tma_load_pair(a + 8192, &g.a, m + 64, k, 0, bar);
          } else {
            tma_load_pair(a, &g.a, k, m, 0, bar);
          }
          if (g.b_mn) {
            for (int j = 0; j < bhalf; j += 64) tma_load_pair(b + j * 128, &g.b, n + j, k, 0, bar);
          } else {
            tma_load_pair(b, &g.b, k, n, 0, bar);
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
      Issuer issue;
      bool ok = true;
      const uint32_t a_lo0 = sdesc_lo(stage0, g.a_mn ? 8192 : 16), b_lo0 = sdesc_lo(stage0 + kABytes, g.b_mn ? 8192 : 16);
      const uint32_t ones_lo = sdesc_lo(ones, 128), stage_step = g.stage_bytes >> 4;
      for (Unit w(g, pair); w.left > 0 && ok; w.next(g, pairs)) {
        const bool sums = g.sums && w.n == 0;
        const int blocks = w.blocks(g);
        for (int kb = 0; kb < blocks && ok; kb += g.seg) {
          const int half = issue.h.pick(sums), end = min(kb + g.seg, blocks);
          ok = issue.take(half, acc_empty, ab, status);
          const uint32_t d = tmem + half * 256;
          for (int b = kb; b < end && ok; b++) {
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
          }
          if (ok) mma_commit_pair_w(&acc_full[half]);
        }
      }
      // No product is left under way.
      mma_commit_leader_w(&drain);
      mbar_drain_w(&drain, 0);
    }
  } else {
    const int e = warp - 2, sub = warp & 3;
    Boxes<END, T, kPer> box(g, boxes + e * kPer * kBox, in_full[e]);
    const act::DropKey key = lin::drop_key(g.e);
    const Place at{g, tmem + ((uint32_t)(sub * 32) << 16), leader_addr(&acc_empty[0]), acc_full, (int)rank, e >> 2, sub, lane,
                   pair, pairs, ab, status};
    if constexpr (sizeof(T) == 2) row_epilogue<END, T, kGroups, kPer>(at, box, key);
    else sum_epilogue<END, 1, kPer>(at, box, key);
    if (lane == 0) bulk_wait_all();  // the results are written before the next kernel's wait ends
  }
  leave(ab, tmem, warp == 1);
}

// ---- rows that TMA can address -----------------------------------------------------------------
//
// bf16 rows of an odd pitch with a pitch of whole 16 bytes: 8 columns a thread.
struct PackJob {
  const __nv_bfloat16* src;
  __nv_bfloat16* dst;
  int64_t rows, threads;
  int C, ld;  // ld: the pitch of dst, C rounded up to 8; its last columns are 0
};
struct PackArgs {
  PackJob job[3];
  int jobs;
  uint32_t* status;
};

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
  const unsigned short* src = reinterpret_cast<const unsigned short*>(j.src) + row * j.C + col;
  uint32_t v[8];
#pragma unroll
  for (int k = 0; k < 8; k++) v[k] = k < left ? src[k] : 0;
  *reinterpret_cast<uint4*>(j.dst + row * j.ld + col) =
      make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

template <int END, typename T, int kGroups, int kPer>
cudaError_t run(TcArgs& g, cudaStream_t st) {
  using B = Block<kGroups, kPer>;
  const auto k_tc = k_linear_bf16<END, T, kGroups, kPer>;
  g.stages = std::min<int>(kMaxStages, (int)(B::kStageRoom / g.stage_bytes));
  cudaError_t e = allow_smem<kSmem>(k_tc);
  if (e != cudaSuccess) return e;
  const int pairs = std::min(g.units, num_sms() / 2);
  return launch(k_tc, dim3((unsigned)(2 * pairs)), dim3(B::kThreads), kSmem, st, g);
}

}  // namespace

int linear_tile_n(int N, bool b_mn, bool f32) {
  if (f32) return 128;
  const int tiles = (N + 255) / 256, step = b_mn ? 128 : 64;
  return ((N + tiles - 1) / tiles + step - 1) / step * step;
}

cudaError_t linear_pack(const LinearPack* packs, int n, uint32_t* status, cudaStream_t st) {
  PackArgs a{};
  a.status = status;
  int64_t threads = 0;
  for (int i = 0; i < n; i++) {
    PackJob& j = a.job[a.jobs++];
    j.src = static_cast<const __nv_bfloat16*>(packs[i].src);
    j.dst = static_cast<__nv_bfloat16*>(packs[i].dst);
    j.rows = packs[i].rows;
    j.C = packs[i].C;
    j.ld = linear_pitch(j.C);
    j.threads = (j.rows * (j.ld >> 3) + 255) / 256 * 256;
    threads += j.threads;
  }
  return launch(k_linear_pack, dim3((unsigned)(threads / 256)), dim3(256), 0, st, a);
}

cudaError_t linear_tc(const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch, cudaStream_t st) {
  if (p.dtype == FS_F32) return linear_tc_f32(p, plan, e, scratch, st);
  TcArgs g{};
  const bool split = plan.splits > 1, raw = split || p.op == kLinDw;
  bool ok = fill_args(g, p, plan, e, scratch);
  g.stage_bytes = kABytes + (uint32_t)g.bn / 2 * 128;
  const int lda = linear_pitch((int)(g.a_mn ? p.M : p.K)), ldb = linear_pitch((int)(g.b_mn ? p.N : p.K));
  ok = ok && (g.a_mn ? make_map(&g.a, p.a, 2, p.M, p.K, 1, lda, 64) : make_map(&g.a, p.a, 2, p.K, p.M, 1, lda, 128));
  ok = ok && (g.b_mn ? make_map(&g.b, p.b, 2, p.N, p.K, 1, ldb, 64) : make_map(&g.b, p.b, 2, p.K, p.N, 1, ldb, g.bn / 2));
  if (!ok) return cudaErrorInvalidValue;
  // (a tile of long rows would be more than L2 keeps)
  if (g.n_tiles == 1 && !raw && p.K % 8 == 0 && p.K <= kShortK) g.ahead = static_cast<const char*>(p.a);
  using B = __nv_bfloat16;
  const bool few = g.store_pre || (g.load_res && g.load_pre) || p.K > kShortK;
  const cudaError_t err = raw                ? run<kEndRaw, float, 2, 2>(g, st)
                          : p.op == kLinFwd ? (few ? run<kEndFwd, B, 3, 2>(g, st) : run<kEndFwd, B, kManyGroups, 1>(g, st))
                                            : (few ? run<kEndDx, B, 3, 2>(g, st) : run<kEndDx, B, kManyGroups, 1>(g, st));
  return err != cudaSuccess ? err : finish(g, p, plan, e, scratch, lda, st);
}

}  // namespace fs
