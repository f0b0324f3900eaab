// The end of a linear map on four neighbouring columns of D (internal), shared by every kernel that
// forms or joins D.
#pragma once

#include "fs_act.cuh"
#include "fs_linear.h"

namespace fs {
namespace lin {

template <typename T>
constexpr bool kFastAct = sizeof(T) == 2;

// (by a whole warp)
__device__ __forceinline__ act::DropKey drop_key(const LinearEnd& e) {
  act::DropKey k{};
  if (e.rng) k = act::drop_key(e.rng);
  return k;
}

// v = D[row, col .. col + 3] of N columns; N % 4 == 0 or the columns past N are left out.
template <typename T, int OP>
__device__ __forceinline__ void end4(const LinearEnd& e, const act::DropKey& key, int64_t row, int col, int N,
                                     float (&v)[4]) {
  const int n = N - col;
  const bool whole = (N & 3) == 0;
  const int64_t at = row * N + col;
  if constexpr (OP == kLinDw) {
    float* y = static_cast<float*>(e.y) + at;
    if (e.accumulate) {
      float old[4];
      act::load4(y, n, whole, old);
#pragma unroll
      for (int i = 0; i < 4; i++) v[i] += old[i];
    }
    act::store4(y, n, whole, v);
    return;
  }
  if constexpr (OP == kLinFwd) {
    if (e.bias) {
      float b[4];
      act::load4(e.bias + col, n, whole, b);
#pragma unroll
      for (int i = 0; i < 4; i++) v[i] += b[i];
    }
    if (e.pre_out) act::store4(static_cast<T*>(e.pre_out) + at, n, whole, v);
    act::apply<kFastAct<T>>(e.act, v);
  } else if (e.act != FS_ACT_NONE) {
    float u[4];
    act::load4(static_cast<const T*>(e.pre_in) + at, n, whole, u);
    act::slope<kFastAct<T>>(e.act, u, v);
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = u[i];
  }
  float r[4] = {};
  if (e.res) act::load4(static_cast<const T*>(e.res) + at, n, whole, r);
  if (e.rng) {
    const uint64_t quads = (uint64_t)((N + 3) >> 2);
    act::keep<4>({e.rng, e.threshold, e.scale}, key, (uint64_t)row * quads + (uint64_t)(col >> 2), v, r);
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = r[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] += r[i];
  }
  act::store4(static_cast<T*>(e.y) + at, n, whole, v);
}

// The sum of A over k (dbias): one value.
__device__ __forceinline__ void end_sum(const LinearEnd& e, int64_t m, float v) {
  e.sums[m] = e.accumulate ? e.sums[m] + v : v;
}

}  // namespace lin
}  // namespace fs
