#include "fs_rows.cuh"

namespace fs {
template cudaError_t norm_fwd<__nv_bfloat16>(const RowsArgs&, cudaStream_t);
template cudaError_t norm_bwd<__nv_bfloat16>(const RowsArgs&, int64_t*, cudaStream_t);
template cudaError_t ckpt_pack<__nv_bfloat16>(const RowsArgs&, cudaStream_t);
template cudaError_t ckpt_unpack<__nv_bfloat16>(const RowsArgs&, cudaStream_t);
template int64_t norm_bwd_blocks<__nv_bfloat16>(int64_t, int);
}  // namespace fs
