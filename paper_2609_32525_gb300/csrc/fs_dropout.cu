// Dropout of rows with an activation and a residual, forward and backward.  Each value is read and
// written once (a mask is computed, not stored).  1,048,576 x 256 bf16 with a residual: 253 us, 94% of this
// card's copy rate; without the residual 223 us, which is the generator: 18 products of 32 x 32 bits for
// four values at 32 a clock and SM are 129 us of it, beside its xors, comparisons and selections at 64 as many (2.5
// instructions a clock and SM, the logic pipe 58% busy, most stalls for a pipe).  Blocks walk
// over the rows, 16 an SM (8 for ragged rows), more than are resident: 8 take 10 us longer there, 32 up to 1 us for 60,033 rows.
#include "fs_act.cuh"
#include "fs_internal.h"
#include "fs_launch.h"
#include "fs_linear.h"

#include <algorithm>

namespace fs {
namespace {

// What is read beside x: nothing, a residual, or the pre-activations of a backward.
enum { kPlain = 0, kRes = 1, kSlope = 2 };

// n values, quad after quad: v becomes the result; other: what is read beside x.  ACT: the activation, or kAnyAct.
constexpr int kAnyAct = -1;
template <typename T, int MODE, int ACT, int n, typename Q>
__device__ __forceinline__ void drop(const DropArgs& a, const act::DropKey& key, Q quad, float (&other)[n], float (&v)[n]) {
  constexpr bool kFast = sizeof(T) == 2;
  if (MODE == kSlope) {
    if constexpr (ACT == kAnyAct) act::slope<kFast>(a.act, other, v);
    else act::slope<kFast, ACT>(other, v);
#pragma unroll
    for (int i = 0; i < n; i++) v[i] = other[i];
  } else {
    if constexpr (ACT == kAnyAct) act::apply<kFast>(a.act, v);
    else act::apply<kFast, ACT>(v);
  }
  if (a.rng) {
    float r[n];
#pragma unroll
    for (int i = 0; i < n; i++) r[i] = MODE == kRes ? other[i] : 0.f;
    act::keep_by<n>({a.rng, a.threshold, a.scale}, key, quad, v, r);
#pragma unroll
    for (int i = 0; i < n; i++) v[i] = r[i];
  } else if (MODE == kRes) {
#pragma unroll
    for (int i = 0; i < n; i++) v[i] += other[i];
  }
}

// Rows of a multiple of four channels: the quads lie one after another, so rows do not matter.
// A thread takes 16 bytes of each tensor at a time, the next ones on their way while it works.
// Q: uint32_t where the quads' numbers fit.  A kernel an activation: behind one branch the loop of each has the registers
// of all.  bf16: at most 48 registers (five blocks an SM; 264 us above with the compiler's choice, 253 with this one);
// fp32 is left to the compiler (323 us for 1,048,576 x 256, 409 with the bound).
template <typename T, int MODE, int ACT, typename Q>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 5 : 0) k_dropout(DropArgs a) {
  const int64_t zero = grid_begin();
  constexpr int kV = 16 / sizeof(T);  // values of a piece
  const int64_t values = a.rows * a.C, step = (int64_t)gridDim.x * 256 * kV;
  const T *x = static_cast<const T*>(a.x) + zero, *beside = static_cast<const T*>(MODE == kRes ? a.res : a.pre);
  T* y = static_cast<T*>(a.y);
  act::DropKey key{};
  if (a.rng) key = act::drop_key(a.rng + zero);
  int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * kV;
  int4 w = make_int4(0, 0, 0, 0), u = w;
  auto load = [&](int64_t p) {
    if (p + kV <= values) {
      w = *reinterpret_cast<const int4*>(x + p);
      if (MODE != kPlain) u = *reinterpret_cast<const int4*>(beside + p);
    } else if (p < values) {  // a last quad of bf16
      *reinterpret_cast<int2*>(&w) = *reinterpret_cast<const int2*>(x + p);
      if (MODE != kPlain) *reinterpret_cast<int2*>(&u) = *reinterpret_cast<const int2*>(beside + p);
    }
  };
  load(at);
  for (; at < values; at += step) {
    float v[kV], f[kV] = {};
#pragma unroll
    for (int h = 0; h < kV; h += 4) {
      act::load4(reinterpret_cast<const T*>(&w) + h, 4, true, *reinterpret_cast<float(*)[4]>(v + h));
      if (MODE != kPlain) act::load4(reinterpret_cast<const T*>(&u) + h, 4, true, *reinterpret_cast<float(*)[4]>(f + h));
    }
    load(at + step);
    drop<T, MODE, ACT, kV>(a, key, (Q)(at >> 2), f, v);
    int4 out;
#pragma unroll
    for (int h = 0; h < kV; h += 4)
      act::store4(reinterpret_cast<T*>(&out) + h, 4, true, *reinterpret_cast<const float(*)[4]>(v + h));
    if (at + kV <= values) *reinterpret_cast<int4*>(y + at) = out;
    else *reinterpret_cast<int2*>(y + at) = *reinterpret_cast<const int2*>(&out);
  }
}

// Any number of channels: a row's last quad may be a part of one, and rows begin anywhere.
template <typename T, int MODE, typename Q>
__global__ void __launch_bounds__(256) k_dropout_ragged(DropArgs a) {
  const int64_t zero = grid_begin();
  const int per_row = (a.C + 3) >> 2;
  const int64_t quads = a.rows * per_row, step = (int64_t)gridDim.x * 256;
  const T *x = static_cast<const T*>(a.x) + zero, *beside = static_cast<const T*>(MODE == kRes ? a.res : a.pre);
  T* y = static_cast<T*>(a.y);
  act::DropKey key{};
  if (a.rng) key = act::drop_key(a.rng + zero);
  int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  int64_t row = q / per_row;
  int col = (int)(q - row * per_row);
  const int64_t rows_on = step / per_row;
  const int cols_on = (int)(step - rows_on * per_row);
  float nv[4], nf[4] = {};
  auto load = [&]() {
    const int n = a.C - 4 * col;
    const int64_t at = row * a.C + 4 * col;
    act::load4(x + at, n, false, nv);
    if (MODE != kPlain) act::load4(beside + at, n, false, nf);
  };
  if (q < quads) load();
  for (; q < quads; q += step) {
    const int n = a.C - 4 * col;
    const int64_t at = row * a.C + 4 * col;
    float v[4], f[4];
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = nv[i], f[i] = nf[i];
    row += rows_on, col += cols_on;
    if (col >= per_row) col -= per_row, row++;
    if (q + step < quads) load();
    drop<T, MODE, kAnyAct, 4>(a, key, (Q)q, f, v);
    act::store4(y + at, n, false, v);
  }
}

template <typename T, int MODE, int ACT>
cudaError_t run_flat(const DropArgs& a, bool low, dim3 grid, cudaStream_t st) {
  return launch(low ? k_dropout<T, MODE, ACT, uint32_t> : k_dropout<T, MODE, ACT, uint64_t>, grid, dim3(256), 0, st, a);
}
template <typename T, int MODE>
cudaError_t run(const DropArgs& a, cudaStream_t st) {
  const bool flat = (a.C & 3) == 0;
  const int64_t quads = a.rows * ((a.C + 3) >> 2), pieces = flat ? (quads * 4 * (int64_t)sizeof(T) + 15) / 16 : quads;
  const bool low = quads + 8 < (1LL << 32);
  const dim3 grid((unsigned)std::min<int64_t>((pieces + 255) / 256, (int64_t)num_sms() * (flat ? 16 : 8)));
  if (!flat) return launch(low ? k_dropout_ragged<T, MODE, uint32_t> : k_dropout_ragged<T, MODE, uint64_t>, grid, dim3(256), 0, st, a);
  if (a.act == FS_ACT_GELU) return run_flat<T, MODE, FS_ACT_GELU>(a, low, grid, st);
  if (a.act == FS_ACT_SILU) return run_flat<T, MODE, FS_ACT_SILU>(a, low, grid, st);
  if (a.act == FS_ACT_RELU) return run_flat<T, MODE, FS_ACT_RELU>(a, low, grid, st);
  if constexpr (MODE != kSlope) return run_flat<T, MODE, FS_ACT_NONE>(a, low, grid, st);
  else return cudaErrorInvalidValue;  // (a backward without an activation reads nothing beside x)
}
template <typename T>
cudaError_t by_mode(const DropArgs& a, cudaStream_t st) {
  if (a.backward && a.act != FS_ACT_NONE) return run<T, kSlope>(a, st);
  return a.res ? run<T, kRes>(a, st) : run<T, kPlain>(a, st);
}

}  // namespace

cudaError_t dropout(const DropArgs& a, cudaStream_t st) {
  return a.dtype == FS_BF16 ? by_mode<__nv_bfloat16>(a, st) : by_mode<float>(a, st);
}

}  // namespace fs
