// What stands between two blocks: declarations (formulas: la_block_norm_kernels.cuh).
#pragma once
#include "la_common.cuh"

namespace la {

enum { GATE_PLAIN = 0, GATE_SIGMOID = 1, GATE_SILU = 2 };
constexpr int BLOCK_NORM_MAX_D = 16384;

struct BlockNormArgs {
  const void *x, *y, *u;                 // [rows, D]; x residual dtype; u or NULL
  const float *w_post, *s, *w_pre;       // [D], or NULL = ones
  void *h, *n;                           // forward; h residual dtype; either may be NULL
  const void *dh, *dn;                   // backward; either may be NULL = zeros
  void *dx, *dy, *du;
  float *dw_post, *ds, *dw_pre;          // or NULL
  float* parts;                          // [nparts][3][D]
  int nparts;
  long long rows;
  int D, gate, post_norm;
  float eps;
};
cudaError_t launch_block_norm_f32(const BlockNormArgs& a, bool backward, cudaStream_t stream);
cudaError_t launch_block_norm_mixed(const BlockNormArgs& a, bool backward, cudaStream_t stream);  // bf16, residual stream in fp32
cudaError_t launch_block_norm_bf16(const BlockNormArgs& a, bool backward, cudaStream_t stream);
cudaError_t launch_block_norm(const BlockNormArgs& a, bool backward, int dt, int res_dt, cudaStream_t stream);

}  // namespace la
