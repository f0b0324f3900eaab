#include "fs_attn_tc.cuh"

namespace fs {
template cudaError_t attn_tc<32>(const AttnTcArgs&, bool, cudaStream_t);
}  // namespace fs
