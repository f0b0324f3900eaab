// Token attention: how a call is run, and the dispatch of the warps' kernels (fs_attn_mma.cuh).
#include "fs_attn.h"
#include "fs_attn_tc.h"
#include "fs_internal.h"

#include <algorithm>

namespace fs {

AttnPlan attn_plan(int64_t units, int64_t rows, int64_t Gk, int d, bool backward) {
  AttnPlan p{};
  p.splits_kv = 1;
  const int64_t sms = num_sms();
  // tcgen05 where a tile of 128 rows is full and there are pairs enough to pay for the images and
  // for a block's start; at d = 16, whose warps work least, on more keys a block, too.  Both sides
  // in us (tcgen05 / warps), heads x tokens:
  //   forward   d = 16  8 x 384 10.6 / 9.9, 8 x 512 11.9 / 12.4, 8 x 1024 18.3 / 29.2,
  //                     128 x 256 19.6 / 15.6, 32 x 512 14.8 / 25.9
  //             d = 32  8 x 256 11.3 / 9.5, 8 x 384 12.3 / 11.4, 8 x 512 12.5 / 14.9,
  //                     32 x 256 13.4 / 15.0, 32 x 512 16.0 / 35.2, 128 x 128 9.7 / 11.6
  //             d = 64  4 x 512 16.2 / 13.1, 4 x 768 16.4 / 19.3, 4 x 2048 36 / 94, 64 x 128 13.2 / 13.5
  //   backward  d = 16  8 x 256 13.7 / 10.4, 8 x 384 14.2 / 16.2, 128 x 128 19.5 / 15.4, 8 x 2048 93 / 173
  //             d = 32  8 x 256 15.9 / 13.3, 8 x 384 17.6 / 18.8, 8 x 512 20.6 / 28.8, 32 x 128 13.9 / 12.8
  //             d = 64  4 x 256 19.9 / 15.4, 4 x 384 21.6 / 22.7, 4 x 512 24.6 / 33.7, 4 x 2048 123 / 397,
  //                     4 x 128 rows against 1024 keys 32 / 23
  const int64_t keys = d == 16 ? (backward ? 256 : 384) : 128;
  const int64_t pairs = !backward ? 1500000 : d == 64 ? 700000 : 1100000;
  p.tc = rows >= 128 && Gk >= keys && units * rows * Gk >= pairs;
  if (p.tc) {
    // One block of 128 rows per SM at a time: the split whose waves of blocks cost least, a
    // block's time being its tiles and about two more; ranges of two tiles at least, and no
    // more tiles than a block lists.  n splits the longer side; the other one is split into ranges
    // of the same length, so that few keys against the rows of many heads stay whole.  (One count
    // for both left most dq blocks without a tile, each with a share of dq to write and to add: us,
    // one count / two, backward at d = 32 of 8 heads that share their keys, 1024 queries x 256 keys
    // 122 / 25, 2048 x 2048 520 / 110, 8192 x 128 888 / 89.)
    const int64_t kt = (Gk + 63) / 64, rt = (rows + 63) / 64, tiles = backward ? std::max(kt, rt) : kt;
    const int64_t blocks_q = units * ((rows + 127) / 128);
    const int64_t blocks_kv = backward ? units * ((Gk + 127) / 128) * (d == 64 ? 2 : 1) : 0;
    const int64_t least = (tiles * 2 + kAttnTcTiles - 1) / kAttnTcTiles;
    double best = 1e300;
    for (int64_t n = least; n <= std::max<int64_t>(least, std::min<int64_t>(tiles / 2, 32)); n++) {
      const int64_t of_keys = (n * kt + tiles - 1) / tiles, of_rows = (n * rt + tiles - 1) / tiles;
      const int64_t blocks = blocks_q * of_keys + blocks_kv * of_rows;
      const double t = (double)((blocks + sms - 1) / sms) * ((double)((tiles + n - 1) / n) + 2.0);
      if (t < 0.97 * best) {
        best = t;
        p.splits = (int)of_keys;
        if (backward) p.splits_kv = (int)of_rows;
      }
    }
    p.delta = true;
    return p;
  }
  // Blocks take 16 rows a warp, up to 64.  Where they would leave SMs without two warps for
  // each of the four schedulers, the streamed side is split, down to single tiles.
  const int64_t most = backward ? std::max(rows, Gk) : rows;
  p.warps = most <= 16 ? 1 : most <= 32 ? 2 : 4;
  const int64_t per = 16 * p.warps, tile = d == 64 ? 32 : 64;
  const int64_t want = sms * 8 / p.warps / (backward ? 2 : 1);
  auto split = [&](int64_t own, int64_t streamed) {
    const int64_t blocks = units * ((own + per - 1) / per), tiles = (streamed + tile - 1) / tile;
    // The forward takes two tiles in turn: what a join costs is more than the second tile (us, whole
    // / split, 8 heads x 128 tokens: d = 16 5.9 / 8.4, d = 32 7.1 / 8.3; three tiles 8.5 / 7.4 in a
    // graph).  The backward's tiles are longer: 8 x 128, d = 32 13.8 / 12.2.
    if (!backward && tiles <= 2) return 1;
    return (int)std::max<int64_t>(1, std::min(want / blocks, tiles));
  };
  p.splits = split(rows, Gk);
  if (backward) {
    p.splits_kv = split(Gk, rows);
    // D = dout . out by a kernel of its own where blocks that own keys meet more than two tiles of
    // queries; else they make it on the way, which saves a launch of three.  Both sides in us
    // (on the way / own kernel): 8 heads x 64 tokens, d = 32 8.0 / 8.6, 128 x 64 10.7 / 11.9,
    // 12 x 100, d = 64 13.7 / 14.3; above the rule 4 x 512, d = 64 35.8 / 33.7, 16 x 1024 337 / 324.
    // A single warp has too few lanes for it: 8 x 16 9.4 / 8.7.
    p.delta = p.warps == 1 || (rows + tile - 1) / tile > 2 * p.splits_kv;
  }
  return p;
}

cudaError_t attn_fwd(const AttnArgs& a, int d, cudaStream_t st) {
  return d == 16 ? attn_mma_fwd<16>(a, st) : d == 32 ? attn_mma_fwd<32>(a, st) : attn_mma_fwd<64>(a, st);
}
cudaError_t attn_bwd(const AttnArgs& a, int d, cudaStream_t st) {
  return d == 16 ? attn_mma_bwd<16>(a, st) : d == 32 ? attn_mma_bwd<32>(a, st) : attn_mma_bwd<64>(a, st);
}

}  // namespace fs
