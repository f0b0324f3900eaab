// Linear maps in fp32 multiply-adds, for sizes that fill no tensor-core tiles and for rows past TMA's coordinates, and the
// fixed-order join of products whose sums were split.
//
// A block owns 64 x 64 values of D and runs over the sum in steps of 16, which it stages in shared
// memory two deep; a thread owns 4 x 4 values, so that four neighbouring channels, which share a
// dropout counter, are in one thread.  Sums are added up over 128 terms at a time and these added
// in turn: a chain of 8192 terms then rounds like one of 128 and one of 64.
#include "fs_launch.h"
#include "fs_linear_end.cuh"

#include <algorithm>

namespace fs {
namespace {

constexpr int kT = 64, kK = 16, kPitch = kT + 4;

struct SimtArgs {
  const void *a, *b;
  int64_t M, K, per;
  int N, splits, ld;
  float *part, *part_sums;
  uint32_t* status;  // to clear, or null
  LinearEnd e;
};

struct Tiles {
  float a[2][kK][kPitch], b[2][kK][kPitch];
};

// block: of the grid of D's tiles (rows, columns) and the sum's parts.
template <typename T, int OP>
__device__ __forceinline__ void simt_block(const SimtArgs& a, int64_t zero, Tiles& tiles, uint3 block) {
  auto &As = tiles.a, &Bs = tiles.b;
  const T* A = static_cast<const T*>(a.a) + zero;
  const T* B = static_cast<const T*>(a.b) + zero;
  const int t = threadIdx.x, tx = t & 15, ty = t >> 4;
  if (a.status && t == 0 && (block.x | block.y | block.z) == 0) *a.status = 0;
  const int64_t m0 = (int64_t)block.x * kT;
  const int n0 = block.y * kT;
  const int64_t k0 = (int64_t)block.z * a.per, k1 = k0 + a.per < a.K ? k0 + a.per : a.K;
  // A: x and g have their channels (k) next to each other, g transposed its m; B: W has its k next
  // to each other in the forward product, its n in dx, and x transposed its n.
  constexpr bool kAk = OP != kLinDw, kBk = OP == kLinFwd;
  const int64_t lda = kAk ? a.K : a.M, ldb = kBk ? a.K : a.N;
  float ra[4], rb[4];
  auto fetch = [&](int64_t k) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int kk = kAk ? t & 15 : (t >> 6) + 4 * i, m = kAk ? (t >> 4) + 16 * i : t & 63;
      const bool in = k + kk < k1 && m0 + m < a.M;
      ra[i] = in ? (float)(kAk ? A[(m0 + m) * lda + k + kk] : A[(k + kk) * lda + m0 + m]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int kk = kBk ? t & 15 : (t >> 6) + 4 * i, n = kBk ? (t >> 4) + 16 * i : t & 63;
      const bool in = k + kk < k1 && n0 + n < a.N;
      rb[i] = in ? (float)(kBk ? B[(int64_t)(n0 + n) * ldb + k + kk] : B[(k + kk) * ldb + n0 + n]) : 0.f;
    }
  };
  auto put = [&](int s) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      As[s][kAk ? t & 15 : (t >> 6) + 4 * i][kAk ? (t >> 4) + 16 * i : t & 63] = ra[i];
      Bs[s][kBk ? t & 15 : (t >> 6) + 4 * i][kBk ? (t >> 4) + 16 * i : t & 63] = rb[i];
    }
  };
  float acc[4][4] = {}, sub[4][4] = {}, sum[4] = {}, sub_sum[4] = {};
  fetch(k0);
  put(0);
  int s = 0, step = 0;
  for (int64_t k = k0; k < k1; k += kK) {
    __syncthreads();
    if (k + kK < k1) fetch(k + kK);
#pragma unroll
    for (int kk = 0; kk < kK; kk++) {
      const float4 x = *reinterpret_cast<const float4*>(&As[s][kk][ty * 4]);
      const float4 y = *reinterpret_cast<const float4*>(&Bs[s][kk][tx * 4]);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; i++) {
#pragma unroll
        for (int j = 0; j < 4; j++) sub[i][j] = fmaf(xs[i], ys[j], sub[i][j]);
        if (OP == kLinDw) sub_sum[i] += xs[i];
      }
    }
    s ^= 1;
    if (k + kK < k1) put(s);
    if ((++step & 7) == 0 || k + kK >= k1) {
#pragma unroll
      for (int i = 0; i < 4; i++) {
#pragma unroll
        for (int j = 0; j < 4; j++) acc[i][j] += sub[i][j], sub[i][j] = 0.f;
        sum[i] += sub_sum[i], sub_sum[i] = 0.f;
      }
    }
  }
  const int col = n0 + tx * 4;
  const act::DropKey key = lin::drop_key(a.e);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int64_t m = m0 + ty * 4 + i;
    if (m >= a.M) break;
    if (OP == kLinDw && a.e.sums && block.y == 0 && tx == 0) {
      if (a.splits > 1) a.part_sums[(int64_t)block.z * a.M + m] = sum[i];
      else lin::end_sum(a.e, m, sum[i]);
    }
    if (col >= a.N) continue;
    if (a.splits > 1)
      *reinterpret_cast<float4*>(a.part + ((int64_t)block.z * a.M + m) * a.ld + col) =
          make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    else
      lin::end4<T, OP>(a.e, key, m, col, a.N, acc[i]);
  }
}

template <typename T, int OP>
__global__ void __launch_bounds__(256) k_linear_simt(SimtArgs a) {
  __shared__ __align__(16) Tiles tiles;
  const int64_t zero = grid_begin();
  simt_block<T, OP>(a, zero, tiles, blockIdx);
}
// dx and dW in one launch: small backward calls are mostly launches.
template <typename T>
__global__ void __launch_bounds__(256) k_linear_simt_bwd(SimtArgs x, SimtArgs w, dim3 grid_x, dim3 grid_w) {
  __shared__ __align__(16) Tiles tiles;
  const int64_t zero = grid_begin();
  const unsigned nx = grid_x.x * grid_x.y * grid_x.z;
  unsigned b = blockIdx.x;
  const dim3 g = b < nx ? grid_x : grid_w;
  if (b >= nx) b -= nx;
  const uint3 block = make_uint3(b % g.x, b / g.x % g.y, b / (g.x * g.y));
  if (blockIdx.x < nx) simt_block<T, kLinDx>(x, zero, tiles, block);
  else simt_block<T, kLinDw>(w, zero, tiles, block);
}

// Few rows through the forward: what counts is W, which is read once for four rows.  A warp owns four columns (a
// dropout counter) and has the loads of 32 x 16 bytes of each on their way at a time; its lanes' sums are added by
// shuffles.
// One row, 1024 -> 4096 channels, bf16 with GELU: 7 us, 31 with the tiles above; eight rows 11, 12 on the tensor cores.  From
// five rows on W is read twice, and terms past a few thousand wait for one another: 4096 -> 4096, four rows 17 us against
// 17, eight 32 against 19.
template <typename T, bool kVec>
__global__ void __launch_bounds__(128) k_linear_few(SimtArgs a) {
  const int64_t zero = grid_begin();
  constexpr int kV = kVec ? 16 / (int)sizeof(T) : 1;
  const T* x = static_cast<const T*>(a.a) + zero;
  const T* W = static_cast<const T*>(a.b) + zero;
  if (a.status && threadIdx.x == 0 && blockIdx.x == 0) *a.status = 0;
  const int lane = threadIdx.x & 31, col = (blockIdx.x * 4 + (threadIdx.x >> 5)) * 4, K = (int)a.K, M = (int)a.M;
  const act::DropKey key = lin::drop_key(a.e);
  if (col >= a.N) return;
  auto load = [&](const T* p, float(&v)[kV]) {
    if constexpr (!kVec) {
      v[0] = (float)p[0];
    } else {
      const uint4 w = *reinterpret_cast<const uint4*>(p);
      const T* t = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int i = 0; i < kV; i++) v[i] = (float)t[i];
    }
  };
  for (int r0 = 0; r0 < M; r0 += 4) {
    float acc[4][4][2] = {};
#pragma unroll 4
    for (int k = lane * kV; k < K; k += 32 * kV) {
      float w[4][kV], v[kV];
#pragma unroll
      for (int j = 0; j < 4; j++) load(W + (int64_t)min(col + j, a.N - 1) * K + k, w[j]);
#pragma unroll
      for (int r = 0; r < 4; r++) {
        if (r0 + r >= M) break;
        load(x + (int64_t)(r0 + r) * K + k, v);
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int i = 0; i < kV; i++) acc[r][j][i & 1] = fmaf(v[i], w[j][i], acc[r][j][i & 1]);
      }
    }
    float mine[4] = {};
#pragma unroll
    for (int r = 0; r < 4; r++)
#pragma unroll
      for (int j = 0; j < 4; j++) {
        float s = acc[r][j][0] + acc[r][j][1];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == r) mine[j] = s;
      }
    if (lane < 4 && r0 + lane < M) lin::end4<T, kLinFwd>(a.e, key, r0 + lane, col, a.N, mine);
  }
}

// 32 quads of columns a block; eight threads share a quad's parts (thread y takes parts y, y + 8, ...),
// and their sums are added in order.  What counts is how many loads are on their way.
template <typename T, int OP>
__global__ void __launch_bounds__(256) k_linear_join(int64_t M, int N, int ld, int splits, const float* __restrict__ part,
                                                      const float* __restrict__ part_sums, LinearEnd e) {
  __shared__ float4 sm[8][33];
  grid_begin(part, part_sums);
  const int64_t quads = M * (ld >> 2), i = (int64_t)blockIdx.x * 32 + threadIdx.x;
  const bool tail = i >= quads;  // dbias
  const int64_t m4 = (i - quads) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (!tail) {
#pragma unroll 4
    for (int p = threadIdx.y; p < splits; p += 8) {
      const float4 v = reinterpret_cast<const float4*>(part)[(int64_t)p * quads + i];
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
  } else if (OP == kLinDw && e.sums && m4 < M) {
    float v[4];
    for (int p = threadIdx.y; p < splits; p += 8) {
      act::load4(part_sums + (int64_t)p * M + m4, (int)(M - m4 < 4 ? M - m4 : 4), (M & 3) == 0, v);
      s.x += v[0], s.y += v[1], s.z += v[2], s.w += v[3];
    }
  }
  sm[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y != 0) return;
  const act::DropKey key = lin::drop_key(e);
#pragma unroll
  for (int y = 1; y < 8; y++) {
    const float4 v = sm[y][threadIdx.x];
    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
  }
  float v[4] = {s.x, s.y, s.z, s.w};
  if (tail) {
    if (OP == kLinDw && e.sums)
#pragma unroll
      for (int j = 0; j < 4; j++)
        if (m4 + j < M) lin::end_sum(e, m4 + j, v[j]);
    return;
  }
  const int64_t row = i / (ld >> 2);
  lin::end4<T, OP>(e, key, row, (int)(i - row * (ld >> 2)) * 4, N, v);
}

// The sums of g's columns over ranges of rows, 16 bytes of columns a thread and 8 rows a block at a time, and
// their sum in order.  A thread adds up eight rows in pairs and these sums in turn, the parts go to eight chains: of a
// million rows a value is rounded some 150 times, not 1200 (of N(0, 1) 2.4e-7 of the norm, 5.8e-7 in one chain each).
template <typename T, int kV>
__global__ void __launch_bounds__(256) k_linear_sums(const T* g, int64_t rows, int C, int ld, float* part) {
  __shared__ float sm[8][32 * kV];
  grid_begin(g, part);
  const int c = (blockIdx.x * 32 + threadIdx.x) * kV;
  const int64_t per = ((rows + gridDim.y - 1) / gridDim.y + 7) & ~(int64_t)7, r0 = blockIdx.y * per;
  const int64_t r1 = min(r0 + per, rows);
  float s[kV] = {};
  if (c < C) {
    for (int64_t r = r0 + threadIdx.y; r < r1; r += 64) {
      struct alignas(sizeof(T) * kV) {
        T v[kV];
      } w[8];
#pragma unroll
      for (int j = 0; j < 8; j++) {
        if constexpr (kV == 1) w[j].v[0] = r + 8 * j < r1 ? g[(r + 8 * j) * ld + c] : T(0.f);
        else *reinterpret_cast<uint4*>(&w[j]) = r + 8 * j < r1 ? *reinterpret_cast<const uint4*>(g + (r + 8 * j) * ld + c) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < kV; i++) {
        auto two = [&](int j) { return (float)w[j].v[i] + (float)w[j + 1].v[i]; };
        s[i] += (two(0) + two(2)) + (two(4) + two(6));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kV; i++) sm[threadIdx.y][threadIdx.x * kV + i] = s[i];
  __syncthreads();
  for (int i = threadIdx.y * 32 + threadIdx.x; i < 32 * kV; i += 256) {
    float t = 0.f;
#pragma unroll
    for (int y = 0; y < 8; y++) t += sm[y][i];
    if (blockIdx.x * 32 * kV + i < C) part[(int64_t)blockIdx.y * C + blockIdx.x * 32 * kV + i] = t;
  }
}
// parts: a multiple of 8.
__global__ void __launch_bounds__(128) k_linear_sums_join(const float* part, int C, int parts, LinearEnd e) {
  grid_begin(part);
  const int c = blockIdx.x * 128 + threadIdx.x;
  if (c >= C) return;
  float s[8] = {};
  for (int p = 0; p < parts; p += 8)
#pragma unroll
    for (int i = 0; i < 8; i++) s[i] += part[(int64_t)(p + i) * C + c];
  lin::end_sum(e, c, ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
}
static_assert(kLinearSumParts % 8 == 0);
template <typename T, int kV>
cudaError_t run_sums(const LinearProblem& p, int ld, float* part, const LinearEnd& e, cudaStream_t st) {
  const int C = (int)p.M;
  cudaError_t err = launch(k_linear_sums<T, kV>, dim3((unsigned)((C + 32 * kV - 1) / (32 * kV)), kLinearSumParts), dim3(32, 8), 0,
                           st, static_cast<const T*>(p.a), p.K, C, ld, part);
  if (err != cudaSuccess) return err;
  return launch(k_linear_sums_join, dim3((unsigned)((C + 127) / 128)), dim3(128), 0, st, part, C, kLinearSumParts, e);
}

SimtArgs simt_args(const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch) {
  SimtArgs a{};
  a.a = p.a; a.b = p.b; a.M = p.M; a.N = p.N; a.K = p.K; a.per = plan.per; a.splits = plan.splits;
  a.ld = (p.N + 3) & ~3;
  a.part = static_cast<float*>(scratch);
  a.part_sums = a.part + (int64_t)plan.splits * p.M * a.ld;
  a.status = p.reset ? p.status : nullptr;
  a.e = e;
  return a;
}
dim3 simt_grid(const SimtArgs& a) {
  return dim3((unsigned)((a.M + kT - 1) / kT), (unsigned)((a.N + kT - 1) / kT), (unsigned)a.splits);
}

template <typename T, int OP>
cudaError_t run_simt(const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch, cudaStream_t st) {
  const SimtArgs a = simt_args(p, plan, e, scratch);
  if (OP == kLinFwd && plan.few) {
    const bool vec = p.K % (16 / (int)sizeof(T)) == 0;
    return launch(vec ? k_linear_few<T, true> : k_linear_few<T, false>, dim3((unsigned)((p.N + 15) / 16)), dim3(128), 0, st, a);
  }
  cudaError_t err = launch(k_linear_simt<T, OP>, simt_grid(a), dim3(256), 0, st, a);
  if (err == cudaSuccess && plan.splits > 1) err = linear_join(p, plan.splits, a.part, a.part_sums, e, st);
  return err;
}

template <typename T, int OP>
cudaError_t run_join(const LinearProblem& p, int splits, const float* part, const float* sums, const LinearEnd& e,
                     cudaStream_t st) {
  const int ld = (p.N + 3) & ~3;
  const int64_t jobs = p.M * (ld >> 2) + (OP == kLinDw && e.sums ? (p.M + 3) / 4 : 0);
  return launch(k_linear_join<T, OP>, dim3((unsigned)((jobs + 31) / 32)), dim3(32, 8), 0, st, p.M, p.N, ld, splits, part,
                sums, e);
}

}  // namespace

cudaError_t linear_simt(const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch,
                        cudaStream_t st) {
  using B = __nv_bfloat16;
  const bool b = p.dtype == FS_BF16;
  if (p.op == kLinFwd) return b ? run_simt<B, kLinFwd>(p, plan, e, scratch, st) : run_simt<float, kLinFwd>(p, plan, e, scratch, st);
  if (p.op == kLinDx) return b ? run_simt<B, kLinDx>(p, plan, e, scratch, st) : run_simt<float, kLinDx>(p, plan, e, scratch, st);
  return b ? run_simt<B, kLinDw>(p, plan, e, scratch, st) : run_simt<float, kLinDw>(p, plan, e, scratch, st);
}

cudaError_t linear_simt_bwd(const LinearProblem& px, const LinearPlan& lx, const LinearEnd& ex, void* sx, const LinearProblem& pw,
                            const LinearPlan& lw, const LinearEnd& ew, void* sw, cudaStream_t st) {
  const SimtArgs x = simt_args(px, lx, ex, sx), w = simt_args(pw, lw, ew, sw);
  const dim3 gx = simt_grid(x), gw = simt_grid(w);
  const dim3 grid(gx.x * gx.y * gx.z + gw.x * gw.y * gw.z);
  cudaError_t err = px.dtype == FS_BF16 ? launch(k_linear_simt_bwd<__nv_bfloat16>, grid, dim3(256), 0, st, x, w, gx, gw)
                                        : launch(k_linear_simt_bwd<float>, grid, dim3(256), 0, st, x, w, gx, gw);
  if (err == cudaSuccess && lx.splits > 1) err = linear_join(px, lx.splits, x.part, x.part_sums, ex, st);
  if (err == cudaSuccess && lw.splits > 1) err = linear_join(pw, lw.splits, w.part, w.part_sums, ew, st);
  return err;
}

cudaError_t linear_sums(const LinearProblem& p, int ld, float* part, const LinearEnd& e, cudaStream_t st) {
  if (p.dtype == FS_BF16) return run_sums<__nv_bfloat16, 8>(p, ld, part, e, st);
  return ld % 4 == 0 ? run_sums<float, 4>(p, ld, part, e, st) : run_sums<float, 1>(p, ld, part, e, st);
}

cudaError_t linear_join(const LinearProblem& p, int splits, const float* part, const float* sums, const LinearEnd& e,
                        cudaStream_t st) {
  using B = __nv_bfloat16;
  const bool b = p.dtype == FS_BF16;
  if (p.op == kLinFwd) return b ? run_join<B, kLinFwd>(p, splits, part, sums, e, st) : run_join<float, kLinFwd>(p, splits, part, sums, e, st);
  if (p.op == kLinDx) return b ? run_join<B, kLinDx>(p, splits, part, sums, e, st) : run_join<float, kLinDx>(p, splits, part, sums, e, st);
  return run_join<float, kLinDw>(p, splits, part, sums, e, st);  // D is fp32
}

}  // namespace fs
