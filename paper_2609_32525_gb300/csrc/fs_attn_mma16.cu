#include "fs_attn_mma.cuh"

namespace fs {
template cudaError_t attn_mma_fwd<16>(const AttnArgs&, cudaStream_t);
template cudaError_t attn_mma_bwd<16>(const AttnArgs&, cudaStream_t);
}  // namespace fs
