// The norms between two blocks in bf16, the residual stream in fp32.
#include "la_block_norm_kernels.cuh"

namespace la {

cudaError_t launch_block_norm_mixed(const BlockNormArgs& a, bool backward, cudaStream_t stream) { return by_alignment<__nv_bfloat16, float>(a, backward, stream); }

}  // namespace la
