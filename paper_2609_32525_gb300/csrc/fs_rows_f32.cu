#include "fs_rows.cuh"

namespace fs {
template cudaError_t norm_fwd<float>(const RowsArgs&, cudaStream_t);
template cudaError_t norm_bwd<float>(const RowsArgs&, int64_t*, cudaStream_t);
template cudaError_t ckpt_pack<float>(const RowsArgs&, cudaStream_t);
template cudaError_t ckpt_unpack<float>(const RowsArgs&, cudaStream_t);
template int64_t norm_bwd_blocks<float>(int64_t, int);
}  // namespace fs
