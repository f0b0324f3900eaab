// Linear maps of rows and dropout (internal): what the entry points hand to the kernels.
#pragma once

#include <cuda_runtime.h>
#include <cstddef>
#include <cstdint>

#include "flashslice.h"

namespace fs {

constexpr int kLinearMaxC = 8192;
constexpr int kLinearFew = 8;   // rows of a forward that a kernel of its own can take

// The three products of a linear map, each D[m, n] = sum_k A[m, k] B[n, k]:
//   forward  D = u  [rows, Cout], A = x, B = W
//   dx       D = dx [rows, Cin],  A = g, B = W transposed
//   dW       D = dW [Cout, Cin],  A = g transposed, B = x transposed; and the sums of A over k
enum LinearOp { kLinFwd = 0, kLinDx = 1, kLinDw = 2 };

// What happens to D.
struct LinearEnd {
  const float* bias;     // forward
  int act;               // fs_act
  const uint64_t* rng;   // null: no dropout
  uint32_t threshold;
  float scale;
  const void* pre_in;    // dx: the pre-activations behind x
  const void* res;
  void* y;               // the rows' type; dW: fp32
  void* pre_out;         // forward
  float* sums;           // dW: dbias, may be null
  int accumulate;        // dW
};

struct LinearProblem {
  int op, dtype;
  int64_t M;             // rows of D
  int N;                 // columns of D
  int64_t K;             // terms of a sum
  const void *a, *b;     // x and W, g and W, g and x, as the caller has them
  uint32_t* status;      // the call's status word, cleared by its first kernel (reset)
  bool reset;
};

// How a product runs; a function of its sizes and the device alone.
struct LinearPlan {
  int path;         // 0: fp32 multiply-adds, 1: tcgen05
  int few;          // path 0: by the kernel for few rows
  int splits;       // parts of the sum, added in order by k_linear_join
  int64_t per;      // terms of a part
  size_t part;      // bytes of scratch for parts
  size_t total;     // bytes of scratch
};
LinearPlan linear_plan(int op, int dtype, int64_t M, int N, int64_t K);

cudaError_t linear_simt(const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch,
                        cudaStream_t st);
// dx and dW, both by fp32 multiply-adds, in one launch (and their joins).  Fewer than 2^31 blocks together.
cudaError_t linear_simt_bwd(const LinearProblem& px, const LinearPlan& lx, const LinearEnd& ex, void* sx, const LinearProblem& pw,
                            const LinearPlan& lw, const LinearEnd& ew, void* sw, cudaStream_t st);
// bf16 operands with a pitch of whole 16 bytes (linear_pack), fp32 ones as they are.
cudaError_t linear_tc(const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch, cudaStream_t st);
cudaError_t linear_tc_f32(const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, void* scratch, cudaStream_t st);
// Columns of D in one of its tiles (fp32 operands take half the columns for two accumulators).
int linear_tile_n(int N, bool b_mn, bool f32);
inline int linear_pitch(int C) { return (C + 7) & ~7; }
inline bool linear_packed(int dtype, int C) { return dtype == FS_BF16 && (C & 7) != 0; }
inline size_t linear_pack_bytes(int64_t rows, int C) { return (size_t)rows * linear_pitch(C) * 2; }
struct LinearPack {
  const void* src;
  void* dst;
  int64_t rows;
  int C;
};
// Up to three tensors in one launch, which also clears the status word.
cudaError_t linear_pack(const LinearPack* packs, int n, uint32_t* status, cudaStream_t st);
// dbias alone: the sums of a (rows of pitch ld, a multiple of 16 bytes in bf16) over its K rows; part
// [kLinearSumParts][M].
constexpr int kLinearSumParts = 128;
cudaError_t linear_sums(const LinearProblem& p, int ld, float* part, const LinearEnd& e, cudaStream_t st);
// Adds up the parts of a product and ends it: part [splits][M][ld], ld the columns rounded up to a
// multiple of 4; sums [splits][M] behind it for dW.
cudaError_t linear_join(const LinearProblem& p, int splits, const float* part, const float* sums, const LinearEnd& e,
                        cudaStream_t st);

// y = res + keep(act(x)) (forward), y = keep(x) act'(pre) (backward) over rows of C channels.
struct DropArgs {
  const void *x, *res, *pre;
  void* y;
  const uint64_t* rng;
  uint32_t threshold;
  float scale;
  int act, dtype, backward;
  int64_t rows;
  int C;
};
cudaError_t dropout(const DropArgs& a, cudaStream_t st);

}  // namespace fs
