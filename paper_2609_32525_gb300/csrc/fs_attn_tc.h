// Token attention on tcgen05 (internal declarations).
#pragma once

#include "fs_attn.h"

namespace fs {

constexpr int kAttnTcTiles = 1024;  // most tiles of a block's range

// What the tensor-core kernels need beside the call: images of k, v, q, dout (null where unused;
// the low parts lie behind all units' high ones), rows padded to whole tiles of 64.
struct AttnTcArgs {
  AttnArgs a;
  uint8_t *row_img[4], *col_img[4];
  float* k_pos;    // [B, k_pad]
  int* k_doc;      // [B, k_pad]
  int2* k_range;   // [B, k_pad / 32]: lowest and highest document of 32 keys
  float* q_info;   // [4][units, rows_pad]: lse, D, slope (base 2), position
  int* q_tok;      // [2][units, rows_pad]: document, index
  int2* q_range;   // [units, rows_pad / 32]
  int rows_pad, k_pad;
};

template <int D>
cudaError_t attn_tc(const AttnTcArgs& t, bool backward, cudaStream_t st);

}  // namespace fs
