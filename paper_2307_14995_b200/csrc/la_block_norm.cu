// The norms between two blocks with the residual stream in fp32 (one file for each of its types: each has some fifty kernels).
#include "la_block_norm_kernels.cuh"

namespace la {

cudaError_t launch_block_norm_f32(const BlockNormArgs& a, bool backward, cudaStream_t stream) { return by_alignment<float, float>(a, backward, stream); }

cudaError_t launch_block_norm(const BlockNormArgs& a, bool backward, int dt, int res_dt, cudaStream_t stream) {
  if (dt == DT_F32 && res_dt == DT_F32) return launch_block_norm_f32(a, backward, stream);
  if (dt == DT_BF16 && res_dt == DT_F32) return launch_block_norm_mixed(a, backward, stream);
  if (dt == DT_BF16 && res_dt == DT_BF16) return launch_block_norm_bf16(a, backward, stream);
  return cudaErrorInvalidValue;
}

}  // namespace la
