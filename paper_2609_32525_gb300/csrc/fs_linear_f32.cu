// Linear maps of fp32 rows on tcgen05 (see fs_linear_tc.cuh): each operand value as three bf16 parts and
// six products of parts.
//
// hi is x cut to 8 bits (so that nothing overflows), mid and lo what is left, rounded: they leave out 2^-25 of
// x.  hi hi goes to one accumulator, hi mid, mid hi, mid mid, hi lo and lo hi to another, so that the small
// products are not cut to the large ones' steps; the others are below 2^-23 of a product.  Six bf16 products give
// fp32's accuracy at a sixth of the bf16 rate, four times what fp32 multiply-adds reach.
//
//   warp 0         TMEM, products (leader)
//   warp 1         TMA copies of 64 terms of A and B, a block ahead
//   warps 4..15    loaders: split a block, into the stage's six images.  Where TMA cannot address a pitch they
//                  copy too, 16, 8 or 4 bytes at a time.
//   warps 16..23   epilogue
// An earlier form wrote the parts to memory first (a kernel of its own, 6 bytes written and read for 4):
// 131,072 x 256 x 256 forward 155 us, here 120, 2.2 TB/s of what it cannot do without.  What bounds it: 2.0 us a block
// of 64 terms in the loaders, whose products take 0.8, and behind an activation the epilogue, 2000 clocks for
// a SILU of 32 x 16 values and more for the derivative of a GELU.
#include "fs_linear_tc.cuh"

namespace fs {
namespace {

constexpr int kLoaders = 12, kFirstLoader = 4, kFirstEpilogue = 16, kThreadsF32 = 768;
// Pieces of a loader in a block; image rows that all loaders take at a time.
constexpr int kPieces = 1536 / (kLoaders * 32), kLines = kLoaders * 4;
constexpr uint32_t kPartA = kABytes, kPartB = kABytes / 2, kStageF32 = 3 * (kPartA + kPartB);
constexpr int kStagesF32 = 2;
constexpr uint32_t kBoxesF32 = 8 * kBox;
// A block's values as they come: [piece][half][loader] of 16 bytes.
constexpr uint32_t kRaw = kPieces * 2 * kLoaders * 32 * 16;
constexpr size_t kSmemF32 = 1024 + kStagesF32 * kStageF32 + kBoxesF32 + kRaw + kOnes;
static_assert(kSmemF32 + 1024 <= 232448);

// A matrix in memory.
struct Source {
  const float* p;
  int64_t rows;
  int cols, ld, vec;  // vec: floats of an aligned copy (4, 2 or 1)
};
// 8 columns of a row, n of which are there (the others are 0): to `to` and, the second half, to `to + half`.  p has
// to be an address of the matrix where n is 0, too.
__device__ __forceinline__ void copy8(const float* p, int n, int vec, uint32_t to, uint32_t half) {
  auto have = [&](int i, int size) { return min(max(n - i, 0), size) * 4; };
  if (vec == 4) {
    copy_async<16>(to, p, have(0, 4));
    copy_async<16>(to + half, n > 4 ? p + 4 : p, have(4, 4));
  } else if (vec == 2) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) copy_async<8>(to + (i >> 2) * half + (i & 3) * 4, n > i ? p + i : p, have(i, 2));
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) copy_async<4>(to + (i >> 2) * half + (i & 3) * 4, n > i ? p + i : p, have(i, 1));
  }
}

// The three parts of 8 values, 16 bytes each.  kInfinite: some value of the warp is.  An infinity has the parts (+-1, 0, +-inf):
// it then meets the other operand's hi alone, which has that value's sign and is 0 only where the value is, and sums are
// infinite or NaN as in fp32.  (As hi it would meet mid and lo, too, which are 0 or of either sign: NaN.)  The 1 is for an
// infinity in both operands.
template <bool kInfinite>
__device__ __forceinline__ void split8(const float (&v)[8], uint4 (&p)[3]) {
  uint32_t w[3][4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const uint32_t x0 = __float_as_uint(v[2 * i]), x1 = __float_as_uint(v[2 * i + 1]);
    const float r0 = v[2 * i] - __uint_as_float(x0 & 0xFFFF0000u), r1 = v[2 * i + 1] - __uint_as_float(x1 & 0xFFFF0000u);
    const uint32_t mid = pack_bf16(r0, r1);
    w[0][i] = __byte_perm(x0, x1, 0x7632);
    w[1][i] = mid;
    w[2][i] = pack_bf16(r0 - __uint_as_float(mid << 16), r1 - __uint_as_float(mid & 0xFFFF0000u));
  }
  if (kInfinite) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const uint32_t half = i & 1 ? 0xFFFF0000u : 0x0000FFFFu, x = __byte_perm(__float_as_uint(v[i]), 0, 0x3232) & half;
      if (fabsf(v[i]) != INFINITY) continue;
      w[0][i >> 1] ^= 0x40004000u & half;  // 0x7F80 to 0x3F80, which is 1
      w[1][i >> 1] &= ~half;
      w[2][i >> 1] = (w[2][i >> 1] & ~half) | x;
    }
  }
#pragma unroll
  for (int i = 0; i < 3; i++) p[i] = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
}

// The lanes with an infinity among their values.  The vote takes every value, so that all of them have come from
// shared memory when it is over: only then may the next copies go there.  What releases the memory has to use the
// vote's result, in a way that no compiler can leave out (& g.none): nothing else keeps the compiler, or the load
// unit, from releasing it earlier.
__device__ __forceinline__ uint32_t lanes_with_infinity(const float (&v)[kPieces][8]) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < kPieces; i++)
#pragma unroll
    for (int j = 0; j < 8; j += 2) top = max3(top, fabsf(v[i][j]), fabsf(v[i][j + 1]));
  return __ballot_sync(0xffffffffu, top == INFINITY);
}

// kTma: both operands have a pitch of whole 16 bytes.
template <int END, bool kTma>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreadsF32, 1)
    k_linear_f32(const __grid_constant__ TcArgs g, Source a, Source b) {
  extern __shared__ __align__(1024) uint8_t raw[];
  __shared__ uint64_t full[kStagesF32], empty[kStagesF32], acc_full[2], acc_empty[2], drain, in_full[8][2], raw_full, raw_empty;
  __shared__ uint32_t tmem_slot;
  __shared__ Abort abort_;
  uint8_t* smem = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  const uint32_t stage0 = smem_u32(smem), boxes = stage0 + kStagesF32 * kStageF32, raws = boxes + kBoxesF32, ones = raws + kRaw;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  Abort* ab = &abort_;

  if (tid == 0) {
    abort_.flag = 0;
    for (int i = 0; i < kStagesF32; i++) mbar_init(&full[i], 2 * kLoaders), mbar_init(&empty[i], 1);
    for (int i = 0; i < 2; i++) mbar_init(&acc_full[i], 1), mbar_init(&acc_empty[i], 16);
    for (int i = 0; i < 16; i++) mbar_init(&in_full[i >> 1][i & 1], 1);
    mbar_init(&drain, 1);
    mbar_init(&raw_full, 1);
    mbar_init(&raw_empty, kLoaders);
    fence_mbar_init();
  }
  if (tid < (int)kOnes / 16) st_shared_v4(ones + tid * 16, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
  fence_proxy_async_smem();
  if (warp == 0) tmem_alloc_pair(&tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  pair_sync();
  tc_fence_after();
  grid_trigger();
  const int64_t zero = grid_wait(a.p, b.p);
  const uint32_t tmem = tmem_slot;
  uint32_t* status = g.status + zero;
  if (g.reset && blockIdx.x == 0 && tid == 0) *status = 0;

  // (registers: 768 x 80 = 61,440 at launch; 128 x 40 + 384 x 64 + 256 x 120 = 60,416 from here on)
  if (warp >= kFirstLoader && warp < kFirstEpilogue) {
    set_registers<false, 64>();
    // 1536 pieces of 8 values a block, 4 a thread: piece i is image row t / 8 + 48 i, A's 128 and then B's 64, and
    // columns 8 (t % 8) on.  An image row of a K-major operand is a row of D's, of an MN-major one a term (64 terms
    // for each 64 rows of D).  A thread copies its own pieces to slots that it alone reads, a block ahead.
    const int t = tid - 32 * kFirstLoader, line = t >> 3, piece = t & 7;
    const uint32_t full0 = leader_addr(&full[0]), slot0 = raws + t * 16, half_step = kLoaders * 32 * 16;
    Ring<kStagesF32> ring;
    auto fetch = [&](const Unit& w, int kb, uint32_t after) {
      if (w.left <= 0) return;
      const int64_t k = w.k0() + (int64_t)kb * 64, m = (int64_t)w.m * 256 + rank * 128;
      const int n = w.n * 128 + (int)rank * 64, col = 8 * piece;
      // the first piece's row and column, and where rows and columns end from there
      const int64_t row_a = g.a_mn ? k : m, row_b = g.b_mn ? k : n;
      const int col_a = (int)(g.a_mn ? m : k) + col, col_b = (int)(g.b_mn ? n : k) + col;
      const int rows_a = (int)min(a.rows - row_a, (int64_t)192), rows_b = (int)min(b.rows - row_b, (int64_t)192);
      const float *from_a = a.p + row_a * a.ld + col_a, *from_b = b.p + row_b * b.ld + col_b;
#pragma unroll
      for (int i = 0; i < kPieces; i++) {
        const int r = line + kLines * i;
        const bool of_a = r < 128;
        int row = of_a ? r : r - 128, cols = of_a ? a.cols - col_a : b.cols - col_b;
        const float* from = of_a ? from_a : from_b;
        if (of_a && g.a_mn && r >= 64) row -= 64, from += 64, cols -= 64;
        const int have = row < (of_a ? rows_a : rows_b) ? min(max(cols, 0), 8) : 0;
        from = have ? from + (int64_t)row * (of_a ? a.ld : b.ld) : (of_a ? a.p : b.p);
        copy8(from, have, of_a ? a.vec : b.vec, slot0 + after + i * 2 * half_step, half_step);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    Unit w(g, pair);  // the block whose copies start next
    int kb = 0, left = 0;
    for (Unit x = w; x.left > 0; x.next(g, pairs)) left += x.blocks(g);
    if (!kTma) fetch(w, kb, 0);
    const uint32_t none = g.none;
    uint32_t stored = 0;
    bool ok = true;
    for (; left > 0; left--) {
      float v[kPieces][8];
      uint32_t infinite;
      if (kTma) {
        ok = mbar_wait_w(&raw_full, stored & 1u, ab, status);
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < kPieces; i++) {
          // boxes of 32 columns: of a K-major operand A's two of 128 rows and B's two of 64, of an MN-major one A's
          // four and B's two of 64 terms
          const int r = line + kLines * i, q = r < 128 ? r : r - 128;
          const bool of_a = r < 128, by_64 = !of_a || g.a_mn;
          const uint32_t row = by_64 ? (uint32_t)(((q >> 6) * 2 + (piece >> 2)) * 64 + (q & 63)) : (uint32_t)((piece >> 2) * 128 + q);
          const uint32_t at = raws + (of_a ? 0 : 2 * kPartA) + row * 128;
#pragma unroll
          for (int h = 0; h < 2; h++) {
            const uint4 x = ld_box(at + (((uint32_t)((piece & 3) * 2 + h) ^ (q & 7)) << 4));
            v[i][4 * h] = __uint_as_float(x.x), v[i][4 * h + 1] = __uint_as_float(x.y);
            v[i][4 * h + 2] = __uint_as_float(x.z), v[i][4 * h + 3] = __uint_as_float(x.w);
          }
        }
        infinite = lanes_with_infinity(v);
        if (lane == 0) mbar_arrive(&raw_empty + (infinite & none));
      } else {
        if (w.left > 0 && ++kb >= w.blocks(g)) kb = 0, w.next(g, pairs);
        asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
        for (int i = 0; i < 2 * kPieces; i++) {
          const uint4 x = ld_box(slot0 + i * half_step);
          v[i >> 1][4 * (i & 1)] = __uint_as_float(x.x), v[i >> 1][4 * (i & 1) + 1] = __uint_as_float(x.y);
          v[i >> 1][4 * (i & 1) + 2] = __uint_as_float(x.z), v[i >> 1][4 * (i & 1) + 3] = __uint_as_float(x.w);
        }
        infinite = lanes_with_infinity(v);
        fetch(w, kb, infinite & none);
      }
      ok = mbar_wait_w(&empty[ring.i], ring.pass ^ 1u, ab, status);
      if (!ok) break;
      const uint32_t stage = stage0 + ring.i * kStageF32;
      auto store = [&](auto is_infinite) {
#pragma unroll
        for (int i = 0; i < kPieces; i++) {
          const int r = line + kLines * i;
          uint4 p[3];
          split8<decltype(is_infinite)::value>(v[i], p);
          const bool of_a = r < 128;
          const uint32_t at = stage + (of_a ? r : r - 128 + 3 * 128) * 128 + ((uint32_t)(piece ^ (r & 7)) << 4);
          const uint32_t step = of_a ? kPartA : kPartB;
#pragma unroll
          for (int q = 0; q < 3; q++) st_shared_v4(at + q * step, p[q].x, p[q].y, p[q].z, p[q].w);
        }
      };
      if (infinite) store(std::true_type{});
      else store(std::false_type{});
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive_leader(full0 + 8 * ring.i);
      ring.next();
      stored++;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    // The leader's commits arrive at this CTA's barriers: not before the last of them do they go.
    for (uint32_t j = stored > kStagesF32 ? stored - kStagesF32 : 0; ok && j < stored; j++)
      mbar_drain_w(&empty[j % kStagesF32], (j / kStagesF32) & 1u);
  } else if (warp < kFirstLoader) {
    set_registers<false, 40>();
    if (kTma && warp == 1 && lane == 0) {
      prefetch_tmap(&g.a);
      prefetch_tmap(&g.b);
      // A block goes to shared memory when the one before has been read from there.  (Asking for it in L2 some blocks
      // earlier made the forward of 131,072 x 256 x 256 6% slower: the copy engine works twice.)
      uint32_t issued = 0;
      bool ok = true;
      for (Unit w(g, pair); w.left > 0 && ok; w.next(g, pairs)) {
        const int blocks = w.blocks(g), m = w.m * 256 + (int)rank * 128, n = w.n * 128 + (int)rank * 64;
        for (int kb = 0; kb < blocks; kb++) {
          const int k = (int)(w.k0() + (int64_t)kb * 64);
          ok = mbar_wait(&raw_empty, (issued & 1u) ^ 1u, ab, status);
          if (!ok) break;
          mbar_expect_tx(&raw_full, kRaw);
#pragma unroll
          for (int j = 0; j < 4; j++) {
            if (g.a_mn) tma_load(raws + j * 8192, &g.a, m + 32 * j, k, &raw_full);
            else if (j < 2) tma_load(raws + j * kPartA, &g.a, k + 32 * j, m, &raw_full);
          }
#pragma unroll
          for (int j = 0; j < 2; j++) {
            if (g.b_mn) tma_load(raws + 2 * kPartA + j * 8192, &g.b, n + 32 * j, k, &raw_full);
            else tma_load(raws + 2 * kPartA + j * 8192, &g.b, k + 32 * j, n, &raw_full);
          }
          issued++;
        }
      }
      if (issued) mbar_drain(&raw_full, (issued - 1) & 1u);  // no copy is left in flight
    }
    if (warp == 0 && rank == 0) {
      Ring<kStagesF32> ring;
      Issuer issue;
      bool ok = true;
      const uint32_t a_lo0 = sdesc_lo(stage0, g.a_mn ? 8192 : 16), b_lo0 = sdesc_lo(stage0 + 3 * kPartA, 16);
      const uint32_t ones_lo = sdesc_lo(ones, 128);
      for (Unit w(g, pair); w.left > 0 && ok; w.next(g, pairs)) {
        const bool sums = g.sums && w.n == 0;
        const int blocks = w.blocks(g);
        for (int kb = 0; kb < blocks && ok; kb += g.seg) {
          const int half = issue.h.pick(sums), end = min(kb + g.seg, blocks);
          ok = issue.take(half, acc_empty, ab, status);
          const uint32_t d = tmem + half * 256;
          for (int blk = kb; blk < end && ok; blk++) {
            ok = mbar_wait_w(&full[ring.i], ring.pass, ab, status);
            if (!ok) break;
            tc_fence_after();
            const uint32_t a_lo = a_lo0 + ring.i * (kStageF32 >> 4), b_lo = b_lo0 + ring.i * (kStageF32 >> 4);
#pragma unroll
            for (int k = 0; k < 4; k++) {
              const uint32_t more = blk > kb || k;
              auto mul = [&](uint32_t to, int i, int j, uint32_t add) {
                mma_pair_w<kHi128, kHi128>(to, a_lo + i * (kPartA >> 4) + k * g.a_step, b_lo + j * (kPartB >> 4) + k * g.b_step,
                                           g.idesc, add);
              };
              mul(d + 128, 0, 2, more);
              mul(d + 128, 2, 0, 1);
              mul(d + 128, 1, 1, 1);
              mul(d + 128, 0, 1, 1);
              mul(d + 128, 1, 0, 1);
              mul(d, 0, 0, more);
              if (sums)
#pragma unroll
                for (int i = 2; i >= 0; i--)  // lo and mid apart from hi, as the products
                  mma_pair_w<kHi128, kHi32>(tmem + kSumCol + (i ? kSumSmall : 0), a_lo + i * (kPartA >> 4) + k * g.a_step, ones_lo,
                                            g.idesc_sum, more || i == 1);
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
    set_registers<true, 120>();
    const int e = warp - kFirstEpilogue, sub = warp & 3;
    Boxes<END, float, 1> box(g, boxes + e * kBox, in_full[e]);
    const act::DropKey key = lin::drop_key(g.e);
    const Place at{g, tmem + ((uint32_t)(sub * 32) << 16), leader_addr(&acc_empty[0]), acc_full, (int)rank, e >> 2, sub, lane,
                   pair, pairs, ab, status};
    sum_epilogue<END, 3, 1>(at, box, key);
    if (lane == 0) bulk_wait_all();  // the results are written before the next kernel's wait ends
  }
  leave(ab, tmem, warp == 0);
}

template <int END, bool kTma>
cudaError_t run(const TcArgs& g, const Source& a, const Source& b, cudaStream_t st) {
  const auto k_tc = k_linear_f32<END, kTma>;
  cudaError_t e = allow_smem<kSmemF32>(k_tc);
  if (e != cudaSuccess) return e;
  const int pairs = std::min(g.units, num_sms() / 2);
  return launch(k_tc, dim3((unsigned)(2 * pairs)), dim3(kThreadsF32), kSmemF32, st, g, a, b);
}

}  // namespace

cudaError_t linear_tc_f32(const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch, cudaStream_t st) {
  TcArgs g{};
  if (!fill_args(g, p, plan, e, scratch)) return cudaErrorInvalidValue;
  auto source = [](const void* q, int64_t rows, int cols) {
    return Source{static_cast<const float*>(q), rows, cols, cols, cols % 4 == 0 ? 4 : cols % 2 == 0 ? 2 : 1};
  };
  const Source a = g.a_mn ? source(p.a, p.K, (int)p.M) : source(p.a, p.M, (int)p.K);
  const Source b = g.b_mn ? source(p.b, p.K, p.N) : source(p.b, p.N, (int)p.K);
  const bool split = plan.splits > 1, raw = split || p.op == kLinDw, tma = a.vec == 4 && b.vec == 4;
  if (tma && (!make_map(&g.a, a.p, 4, a.cols, a.rows, 1, a.ld, g.a_mn ? 64 : 128) ||
              !make_map(&g.b, b.p, 4, b.cols, b.rows, 1, b.ld, 64)))
    return cudaErrorInvalidValue;
  const cudaError_t err = raw                ? (tma ? run<kEndRaw, true>(g, a, b, st) : run<kEndRaw, false>(g, a, b, st))
                          : p.op == kLinFwd ? (tma ? run<kEndFwd, true>(g, a, b, st) : run<kEndFwd, false>(g, a, b, st))
                                            : (tma ? run<kEndDx, true>(g, a, b, st) : run<kEndDx, false>(g, a, b, st));
  return err != cudaSuccess ? err : finish(g, p, plan, e, scratch, a.ld, st);
}

}  // namespace fs
