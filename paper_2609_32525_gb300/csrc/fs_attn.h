// Attention of the slice tokens (internal declarations).
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

namespace fs {

// One call, in the kernels' terms.  The heads that share a key head form a unit (b, kv head);
// their query rows lie one after another in memory, so a unit has rows = (H / Hkv) Gq rows and
// row r is query r % Gq of the unit's head r / Gq.
struct AttnArgs {
  const float *q, *k, *v;        // [units, rows, d], [units, Gk, d]
  const float *slopes;           // [H] or null
  const float *pos_q, *pos_k;    // [B, Gq], [B, Gk] or null
  const int *doc_q, *doc_k;      // [B, Gq], [B, Gk] or null
  const int *prefix;             // [B] or null (0)
  float *out, *lse;              // forward: written; backward: read
  const float *dout;
  float *dq, *dk, *dv;
  float *delta;                  // [units, rows]; null: made where they are used
  float *part;                   // partial results of the splits
  float *part_kv;
  uint32_t *status;
  int B, H, Hkv, Gq, Gk, rows, units;
  int causal;                    // the prefix mask
  int warps;                     // per block: 16 rows each
  int splits, splits_kv;         // of the keys (forward, dq), of the rows (dk, dv)
  float scale, cap;
};

// How a call is run on the current device: on tcgen05 (fs_attn_tc.cuh) or with warps' own
// products (fs_attn_mma.cuh), there with so many warps per block; splits of the keys, and of the
// query rows for dk and dv.
struct AttnPlan {
  bool tc;
  bool delta;  // backward: D by a kernel of its own
  int warps, splits, splits_kv;
};
AttnPlan attn_plan(int64_t units, int64_t rows, int64_t Gk, int d, bool backward);

template <int D>
cudaError_t attn_mma_fwd(const AttnArgs& a, cudaStream_t st);
template <int D>
cudaError_t attn_mma_bwd(const AttnArgs& a, cudaStream_t st);

cudaError_t attn_fwd(const AttnArgs& a, int d, cudaStream_t st);
cudaError_t attn_bwd(const AttnArgs& a, int d, cudaStream_t st);

}  // namespace fs
