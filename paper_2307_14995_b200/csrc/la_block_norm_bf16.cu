// The norms between two blocks in bf16, the residual stream in bf16.
#include "la_block_norm_kernels.cuh"

namespace la {

cudaError_t launch_block_norm_bf16(const BlockNormArgs& a, bool backward, cudaStream_t stream) { return by_alignment<__nv_bfloat16, __nv_bfloat16>(a, backward, stream); }

}  // namespace la
