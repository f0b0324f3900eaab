// Dropout of rows with an activation and a residual, forward and backward.  Bound by memory: each
// value is read and written once (a mask is computed, not stored), and the generator's 40
// instructions for four values stay below the time of their bytes (1,048,576 x 256 bf16 with a
// residual: the rows alone take 237 us at this card's copy rate).
#include "fs_act.cuh"
#include "fs_internal.h"
#include "fs_launch.h"
#include "fs_linear.h"

#include <algorithm>

namespace fs {
namespace {

// n values, quad after quad.
template <typename T, int n>
__device__ __forceinline__ void drop(const DropArgs& a, const act::DropKey& key, uint64_t quad, float (&pre)[n],
                                     float (&res)[n], float (&v)[n]) {
  constexpr bool kFast = sizeof(T) == 2;
  if (a.backward) {
    act::slope<kFast>(a.act, pre, v);
#pragma unroll
    for (int i = 0; i < n; i++) v[i] = pre[i];
  } else {
    act::apply<kFast>(a.act, v);
  }
  if (a.rng) {
    act::keep<n>({a.rng, a.threshold, a.scale}, key, quad, v, res);
#pragma unroll
    for (int i = 0; i < n; i++) v[i] = res[i];
  } else {
#pragma unroll
    for (int i = 0; i < n; i++) v[i] += res[i];
  }
}

// Rows of a multiple of four channels: the quads lie one after another, so rows do not matter.
// A thread takes kP pieces of 16 bytes of each tensor at a time, a block's width apart, loaded
// before the first is worked on.
template <typename T, int kP>
__global__ void __launch_bounds__(256) k_dropout(DropArgs a) {
  const int64_t zero = grid_begin();
  constexpr int kV = 16 / sizeof(T);  // values of a piece
  const int64_t values = a.rows * a.C, step = (int64_t)gridDim.x * 256 * kP * kV;
  const T *x = static_cast<const T*>(a.x) + zero, *res = static_cast<const T*>(a.res), *pre = static_cast<const T*>(a.pre);
  T* y = static_cast<T*>(a.y);
  act::DropKey key{};
  if (a.rng) key = act::drop_key(a.rng + zero);
  const bool slope = a.backward && a.act != FS_ACT_NONE;
  for (int64_t first = ((int64_t)blockIdx.x * 256 * kP + threadIdx.x) * kV; first < values; first += step) {
    int4 w[kP], r[kP], u[kP];
#pragma unroll
    for (int p = 0; p < kP; p++) {
      const int64_t at = first + p * 256 * kV;
      w[p] = r[p] = u[p] = make_int4(0, 0, 0, 0);
      if (at + kV <= values) {
        w[p] = *reinterpret_cast<const int4*>(x + at);
        if (a.res) r[p] = *reinterpret_cast<const int4*>(res + at);
        if (slope) u[p] = *reinterpret_cast<const int4*>(pre + at);
      } else if (at < values) {  // a last quad of bf16
        *reinterpret_cast<int2*>(&w[p]) = *reinterpret_cast<const int2*>(x + at);
        if (a.res) *reinterpret_cast<int2*>(&r[p]) = *reinterpret_cast<const int2*>(res + at);
        if (slope) *reinterpret_cast<int2*>(&u[p]) = *reinterpret_cast<const int2*>(pre + at);
      }
    }
#pragma unroll
    for (int p = 0; p < kP; p++) {
      const int64_t at = first + p * 256 * kV;
      float v[kV], f[kV], g[kV];
#pragma unroll
      for (int h = 0; h < kV; h += 4) {
        act::load4(reinterpret_cast<const T*>(&w[p]) + h, 4, true, *reinterpret_cast<float(*)[4]>(v + h));
        act::load4(reinterpret_cast<const T*>(&u[p]) + h, 4, true, *reinterpret_cast<float(*)[4]>(f + h));
        act::load4(reinterpret_cast<const T*>(&r[p]) + h, 4, true, *reinterpret_cast<float(*)[4]>(g + h));
      }
      drop<T, kV>(a, key, (uint64_t)at >> 2, f, g, v);
      int4 out;
#pragma unroll
      for (int h = 0; h < kV; h += 4)
        act::store4(reinterpret_cast<T*>(&out) + h, 4, true, *reinterpret_cast<const float(*)[4]>(v + h));
      if (at + kV <= values) *reinterpret_cast<int4*>(y + at) = out;
      else if (at < values) *reinterpret_cast<int2*>(y + at) = *reinterpret_cast<const int2*>(&out);
    }
  }
}

// Any number of channels: a row's last quad may be a part of one, and rows begin anywhere.
template <typename T>
__global__ void __launch_bounds__(256) k_dropout_ragged(DropArgs a) {
  const int64_t zero = grid_begin();
  const int per_row = (a.C + 3) >> 2;
  const int64_t quads = a.rows * per_row, step = (int64_t)gridDim.x * 256;
  const T *x = static_cast<const T*>(a.x) + zero, *res = static_cast<const T*>(a.res), *pre = static_cast<const T*>(a.pre);
  T* y = static_cast<T*>(a.y);
  act::DropKey key{};
  if (a.rng) key = act::drop_key(a.rng + zero);
  const bool slope = a.backward && a.act != FS_ACT_NONE;
  int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
  int64_t row = q / per_row;
  int col = (int)(q - row * per_row);
  const int64_t rows_on = step / per_row;
  const int cols_on = (int)(step - rows_on * per_row);
  for (; q < quads; q += step) {
    const int n = a.C - 4 * col;
    const int64_t at = row * a.C + 4 * col;
    float v[4], f[4] = {}, g[4] = {};
    act::load4(x + at, n, false, v);
    if (slope) act::load4(pre + at, n, false, f);
    if (a.res) act::load4(res + at, n, false, g);
    drop<T, 4>(a, key, (uint64_t)q, f, g, v);
    act::store4(y + at, n, false, v);
    row += rows_on, col += cols_on;
    if (col >= per_row) col -= per_row, row++;
  }
}

template <typename T>
cudaError_t run(const DropArgs& a, cudaStream_t st) {
  const bool flat = (a.C & 3) == 0;
  const int64_t pieces = flat ? (a.rows * a.C * (int64_t)sizeof(T) + 15) / 16 : a.rows * ((a.C + 3) >> 2);
  // Two pieces a thread where that still fills the device.
  const int64_t most = (int64_t)num_sms() * 8;
  const bool two = flat && pieces >= most * 512;
  const int64_t blocks = std::min<int64_t>((pieces + (two ? 511 : 255)) / (two ? 512 : 256), most);
  return launch(!flat ? k_dropout_ragged<T> : two ? k_dropout<T, 2> : k_dropout<T, 1>, dim3((unsigned)blocks), dim3(256), 0,
                st, a);
}

}  // namespace

cudaError_t dropout(const DropArgs& a, cudaStream_t st) {
  return a.dtype == FS_BF16 ? run<__nv_bfloat16>(a, st) : run<float>(a, st);
}

}  // namespace fs
