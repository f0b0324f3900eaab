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

template <typename T>
__device__ __forceinline__ void drop4(const DropArgs& a, const act::DropKey& key, uint64_t quad, const float (&pre)[4],
                                      const float (&res)[4], float (&v)[4]) {
  constexpr bool kFast = sizeof(T) == 2;
  if (a.backward) act::slope4<kFast>(a.act, pre, v);
  else act::apply4<kFast>(a.act, v);
  if (a.rng) act::keep4({a.rng, a.threshold, a.scale}, key, quad, v);
  if (a.res)
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] += res[i];
}

// Rows of a multiple of four channels: the quads lie one after another, so rows do not matter.
// A thread takes 16 bytes of each tensor at a time.
template <typename T>
__global__ void __launch_bounds__(256) k_dropout(DropArgs a) {
  const int64_t zero = grid_begin();
  constexpr int kQ = 16 / (4 * sizeof(T));  // quads in 16 bytes
  const int64_t quads = a.rows * (a.C >> 2), step = (int64_t)gridDim.x * 256 * kQ;
  const T *x = static_cast<const T*>(a.x) + zero, *res = static_cast<const T*>(a.res), *pre = static_cast<const T*>(a.pre);
  T* y = static_cast<T*>(a.y);
  act::DropKey key{0, 0};
  if (a.rng) key = {a.rng[zero], a.rng[1 + zero]};
  const bool slope = a.backward && a.act != FS_ACT_NONE;
  for (int64_t q = ((int64_t)blockIdx.x * 256 + threadIdx.x) * kQ; q < quads; q += step) {
    if (kQ == 2 && q + 2 <= quads) {
      const int4 w = *reinterpret_cast<const int4*>(x + 4 * q);
      int4 r = make_int4(0, 0, 0, 0), u = r, out;
      if (a.res) r = *reinterpret_cast<const int4*>(res + 4 * q);
      if (slope) u = *reinterpret_cast<const int4*>(pre + 4 * q);
#pragma unroll
      for (int h = 0; h < 2; h++) {
        float v[4], f[4], g[4];
        act::load4(reinterpret_cast<const T*>(&w) + 4 * h, 4, true, v);
        act::load4(reinterpret_cast<const T*>(&u) + 4 * h, 4, true, f);
        act::load4(reinterpret_cast<const T*>(&r) + 4 * h, 4, true, g);
        drop4<T>(a, key, (uint64_t)(q + h), f, g, v);
        act::store4(reinterpret_cast<T*>(&out) + 4 * h, 4, true, v);
      }
      *reinterpret_cast<int4*>(y + 4 * q) = out;
    } else {
      float v[4], f[4] = {}, g[4] = {};
      act::load4(x + 4 * q, 4, true, v);
      if (slope) act::load4(pre + 4 * q, 4, true, f);
      if (a.res) act::load4(res + 4 * q, 4, true, g);
      drop4<T>(a, key, (uint64_t)q, f, g, v);
      act::store4(y + 4 * q, 4, true, v);
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
  act::DropKey key{0, 0};
  if (a.rng) key = {a.rng[zero], a.rng[1 + zero]};
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
    drop4<T>(a, key, (uint64_t)q, f, g, v);
    act::store4(y + at, n, false, v);
    row += rows_on, col += cols_on;
    if (col >= per_row) col -= per_row, row++;
  }
}

template <typename T>
cudaError_t run(const DropArgs& a, cudaStream_t st) {
  const bool flat = (a.C & 3) == 0;
  const int64_t threads = flat ? (a.rows * (a.C >> 2) * 4 * (int64_t)sizeof(T) + 15) / 16 : a.rows * ((a.C + 3) >> 2);
  const int64_t blocks = std::min<int64_t>((threads + 255) / 256, (int64_t)num_sms() * 8);
  return launch(flat ? k_dropout<T> : k_dropout_ragged<T>, dim3((unsigned)blocks), dim3(256), 0, st, a);
}

}  // namespace

cudaError_t dropout(const DropArgs& a, cudaStream_t st) {
  return a.dtype == FS_BF16 ? run<__nv_bfloat16>(a, st) : run<float>(a, st);
}

}  // namespace fs
