// The gated delta rule: shared declarations of its kernels.
//
// Per value head, S [D, D] fp32, a_t = exp(g_t), q and k of key head h / (H / Hk):
//   S_t = a_t (S_{t-1} - beta_t k_t (k_t^T S_{t-1})) + beta_t k_t v_t^T,      o_t = scale S_t^T q_t.
// Chunk form, C tokens from the state S, G_i = g_0 + .. + g_i, D_ij = exp(G_i - G_j), n_ij = (k_i . k_j) D_ij for i > j:
//   That = (I + n diag(beta))^-1 (unit lower triangular),   Uhat = That V,   What = That diag(e^G) K,
//   Y = Uhat - What S,   V' = diag(beta) Y,
//   O = scale (diag(e^G) Q S + ((Q K^T) (.) D) V'),   S' = e^G_end S + K^T diag(e^(G_end - G)) V'.
// Adjoint for E' = dL/dS':
//   dV' = scale ((Q K^T) (.) D)^T dO + diag(e^(G_end - G)) K E',   dR = That^T diag(beta) dV' = dV,
//   E = e^G_end E' + scale Q^T diag(e^G) dO - K^T diag(e^G) dR   (= ... - What^T diag(beta) dV'),
//   F = scale (dO V'^T) (.) D (i >= j),   Hh = (dR Y^T) (.) D (i > j),   H = Hh diag(beta),
//   dQ = scale diag(e^G) dO S^T + F K,
//   dK = F^T Q + diag(e^(G_end - G)) V' E'^T - diag(e^G) dR S^T - H^T K - H K,
//   dbeta_j = dV'_j . Y_j - sum_{i > j} (k_i . k_j) Hh_ij,
//   dg_s = sum_{j < s <= i} Z_ij + sum_{i >= s} a_i + sum_{j < s} b_j + e^G_end <S, E'>,   Z_ij = F_ij (q_i . k_j) - H_ij (k_i . k_j),
//   a_i = e^G_i (scale q_i . S do_i - k_i . S dR_i),   b_j = e^(G_end - G_j) k_j . E' v'_j,
// the derivatives by the logarithms of D_ij, e^G_i, e^(G_end - G_j) and e^G_end, summed over those that contain g_s.  (As differences of
// q . dq and k . dk, which need no Z, they would be the small rest of large terms where a head forgets fast.)
// Y instead of V' and That instead of the inverse of I + diag(beta) n keep every formula free of a division by beta, which may be 0,
// and every decay is exp of a difference G_i - G_j, i >= j, or of a sum: nothing is divided by a decay either, which may be 0 too.
#pragma once
#include "la_common.cuh"

namespace la {

struct DeltaArgs {
  const void *q, *k, *v;      // q, k: Hk heads; v, d_o: H heads
  const float *g, *beta;      // one value per (token, value head)
  const void* d_o;
  void* o;
  void *dq, *dk, *dv;
  float *dg, *dbeta;
  const float *kv_in, *grad_kv_out;
  float *kv_out, *grad_kv_in;
  void *ws, *ws_bwd;          // records of the chunks (see the kernels)
  float scale;
  int B, H, Hk, N, D, nchunk;
  long long sB, sH, sT;       // element offset of row (b, h, t) of v, o, d_o, dv: b sB + h sH + t sT
  long long sBk, sHk, sTk;    // the same of q, k, dq, dk
  long long gB, gH, gT;       // the same of g, beta, dg, dbeta
};

// A decay of e^-1000 is zero in fp32 and in double alike; clamped there, -inf (forget everything) has differences.  NaN passes.
__device__ __forceinline__ double clamped_log_decay(float g) { return g < -1000.f ? -1000.0 : (double)g; }

// CUDA-core kernels (fp32 and bf16 inputs), chunks of 64 tokens.
constexpr int DELTA_SIMT_CHUNK = 64;
size_t delta_simt_chunk_bytes(int D, bool bwd);  // workspace of one chunk of one head
cudaError_t launch_delta_simt_fwd(const DeltaArgs& a, int in_dt, int out_dt, cudaStream_t stream);
// have_fwd: a.ws holds what the forward pass left there
cudaError_t launch_delta_simt_bwd(const DeltaArgs& a, bool have_fwd, int in_dt, int out_dt, cudaStream_t stream);

// Tensor-core kernels (bf16 inputs), chunks of 128 tokens.
constexpr int DELTA_TC_CHUNK = 128;
size_t delta_tc_chunk_bytes(int D, bool bwd);
cudaError_t launch_delta_tc_fwd(const DeltaArgs& a, int out_dt, cudaStream_t stream);
cudaError_t launch_delta_tc_bwd(const DeltaArgs& a, bool have_fwd, int out_dt, cudaStream_t stream);

// a.N >= 1 consecutive tokens on a state that is updated in place (a.kv_out).
cudaError_t launch_delta_steps(const DeltaArgs& a, int in_dt, int out_dt, cudaStream_t stream);

}  // namespace la
