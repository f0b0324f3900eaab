// Row kernels: layer norm over the channels of a row and the 8-bit checkpoint of a row
// (internal declarations; fs_rows.cuh has the kernels, one translation unit per dtype).
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

namespace fs {

struct RowsArgs {
  // forward: v = x + res (rounded to the dtype, written to sum), y = norm(v); backward: x is v,
  // y is dv
  const void *x, *res;
  void *sum, *y;
  const float *gamma, *beta;
  float *mean, *rstd;
  int8_t* q8;
  uint8_t* e8;
  // backward
  const void *dy, *dres;
  float *dgamma, *dbeta, *part;
  uint32_t* status;
  int64_t rows;
  int C;
  float eps;
  int accumulate;
};

constexpr int kCkptBlock = 32;  // channels that share a scale
constexpr int kRowsMaxC = 8192;

// Most blocks of the backward's main pass: rows of partial sums [blocks][2 C] in the workspace.
template <typename T>
int64_t norm_bwd_blocks(int64_t rows, int C);

template <typename T>
cudaError_t norm_fwd(const RowsArgs& a, cudaStream_t st);
template <typename T>
cudaError_t norm_bwd(const RowsArgs& a, int64_t* blocks, cudaStream_t st);  // *blocks: those that it used
template <typename T>
cudaError_t ckpt_pack(const RowsArgs& a, cudaStream_t st);
template <typename T>
cudaError_t ckpt_unpack(const RowsArgs& a, cudaStream_t st);

}  // namespace fs
