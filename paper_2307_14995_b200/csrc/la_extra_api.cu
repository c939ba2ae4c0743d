// C-ABI entry points of the gated delta rule and of the norms between two blocks (declared in include/la.h): argument checks,
// workspace sizes and launches.
#include <cmath>
#include <initializer_list>

#include "../../include/la.h"
#include "la_block_norm.cuh"
#include "la_check.cuh"
#include "la_delta.cuh"

namespace la {
namespace {

bool any_unaligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!aligned16(p)) return true;
  return false;
}

la_status check_delta(const la_delta_shape* s) {
  if (!s) return LA_ERR_INVALID_ARG;
  if (s->B < 1 || s->H < 1 || s->Hk < 1 || s->N < 1 || s->d < 1 || s->e < 1) return LA_ERR_INVALID_ARG;
  if (s->H % s->Hk != 0) return LA_ERR_INVALID_ARG;
  if (s->in_dtype != LA_BF16 && s->in_dtype != LA_F32) return LA_ERR_INVALID_ARG;
  if (s->out_dtype != LA_BF16 && s->out_dtype != LA_F32) return LA_ERR_INVALID_ARG;
  if (s->path < LA_PATH_AUTO || s->path > LA_PATH_TENSOR) return LA_ERR_INVALID_ARG;
  if (s->layout != LA_LAYOUT_BHND && s->layout != LA_LAYOUT_BNHD) return LA_ERR_INVALID_ARG;
  if (!std::isfinite(s->scale)) return LA_ERR_INVALID_ARG;
  if (!(s->d == s->e && (s->d == 64 || s->d == 128))) return LA_ERR_UNSUPPORTED;
  if (s->in_dtype == LA_F32 && s->out_dtype != LA_F32) return LA_ERR_UNSUPPORTED;
  // grids have a row per (batch, head); token indices are 32 bits, element offsets 64
  if ((long long)s->B * s->H > 65535 || s->N >= (1 << 30) || (double)s->B * s->H * s->N * s->d >= 2147483648.0 * 64.0) return LA_ERR_UNSUPPORTED;
  return LA_OK;
}

la_status delta_path(const la_delta_shape* s, bool* tensor) {
  const bool could = s->in_dtype == LA_BF16 && tc_supported();
  if (s->path == LA_PATH_TENSOR && !could) return LA_ERR_UNSUPPORTED;
  *tensor = could && s->path != LA_PATH_SIMT;
  return LA_OK;
}

size_t delta_bytes(const la_delta_shape* s, bool tensor, bool bwd) {
  const int chunk = tensor ? DELTA_TC_CHUNK : DELTA_SIMT_CHUNK;
  return (size_t)s->B * s->H * ((s->N + chunk - 1) / chunk) * (tensor ? delta_tc_chunk_bytes(s->d, bwd) : delta_simt_chunk_bytes(s->d, bwd));
}

DeltaArgs delta_args(const la_delta_shape* s, bool tensor) {
  DeltaArgs a{};
  a.B = s->B; a.H = s->H; a.Hk = s->Hk; a.N = s->N; a.D = s->d;
  const int chunk = tensor ? DELTA_TC_CHUNK : DELTA_SIMT_CHUNK;
  a.nchunk = (s->N + chunk - 1) / chunk;
  a.scale = s->scale;
  const long long N = s->N, D = s->d, H = s->H, Hk = s->Hk;
  a.sB = N * H * D;
  a.sBk = N * Hk * D;
  a.gB = N * H;
  if (s->layout == LA_LAYOUT_BNHD) {
    a.sH = a.sHk = D; a.sT = H * D; a.sTk = Hk * D; a.gH = 1; a.gT = H;
  } else {
    a.sH = a.sHk = N * D; a.sT = a.sTk = D; a.gH = N; a.gT = 1;
  }
  return a;
}

la_status check_norm(const la_block_norm_shape* s) {
  if (!s) return LA_ERR_INVALID_ARG;
  if (s->rows < 1 || s->D < 1) return LA_ERR_INVALID_ARG;
  if (s->dtype != LA_BF16 && s->dtype != LA_F32) return LA_ERR_INVALID_ARG;
  if (s->res_dtype != LA_BF16 && s->res_dtype != LA_F32) return LA_ERR_INVALID_ARG;
  if (s->gate < LA_GATE_PLAIN || s->gate > LA_GATE_SILU || (s->post_norm != 0 && s->post_norm != 1)) return LA_ERR_INVALID_ARG;
  if (!(std::isfinite(s->eps) && s->eps >= 0.f)) return LA_ERR_INVALID_ARG;
  if (s->D > BLOCK_NORM_MAX_D || (double)s->rows * s->D >= 2147483648.0 * 1024.0) return LA_ERR_UNSUPPORTED;
  if (s->dtype == LA_F32 && s->res_dtype != LA_F32) return LA_ERR_UNSUPPORTED;
  return LA_OK;
}
// Thread blocks of the backward pass, each of which leaves a part of the sums over tokens: as many as run at once; of few, a multiple of eight.
int norm_parts(const la_block_norm_shape* s) {
  const long long most = s->D > 4096 && s->D <= 8192 ? 148 * 2 : 148;
  const long long rows = (s->rows + 7) / 8 * 8;
  return (int)(rows < most ? rows : most);
}
BlockNormArgs norm_args(const la_block_norm_shape* s, const void* x, const void* y, const void* u, const float* w_post, const float* sc,
                        const float* w_pre) {
  BlockNormArgs a{};
  a.x = x; a.y = y; a.u = u;
  a.w_post = w_post; a.s = sc; a.w_pre = w_pre;
  a.rows = s->rows; a.D = s->D; a.gate = s->gate; a.post_norm = s->post_norm; a.eps = s->eps;
  return a;
}

}  // namespace
}  // namespace la

using namespace la;

extern "C" {

size_t la_delta_workspace_bytes(int op, const la_delta_shape* shape) {
  bool tensor;
  if (op != LA_OP_FWD && op != LA_OP_BWD && op != LA_OP_DECODE) return (size_t)-1;
  if (check_delta(shape) != LA_OK || delta_path(shape, &tensor) != LA_OK) return (size_t)-1;
  if (op == LA_OP_DECODE) return 0;
  return delta_bytes(shape, tensor, false) + (op == LA_OP_BWD ? delta_bytes(shape, tensor, true) : 0);
}

la_status la_delta_fwd(const la_delta_shape* shape, const void* q, const void* k, const void* v, const float* g, const float* beta,
                       void* o, const float* kv_in, float* kv_out, void* workspace, size_t workspace_bytes, void* stream) {
  la_status st = check_delta(shape);
  if (st != LA_OK) return st;
  if (!q || !k || !v || !g || !beta || !o) return LA_ERR_INVALID_ARG;
  if (any_unaligned({q, k, v, g, beta, o, kv_in, kv_out})) return LA_ERR_INVALID_ARG;
  bool tensor;
  if ((st = delta_path(shape, &tensor)) != LA_OK) return st;
  if (!workspace || workspace_bytes < delta_bytes(shape, tensor, false)) return LA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return LA_ERR_INVALID_ARG;
  if ((st = check_device()) != LA_OK) return st;
  DeltaArgs a = delta_args(shape, tensor);
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.o = o;
  a.kv_in = kv_in; a.kv_out = kv_out;
  a.ws = workspace;
  const cudaStream_t cs = static_cast<cudaStream_t>(stream);
  LA_TRY_CUDA(tensor ? launch_delta_tc_fwd(a, (int)shape->out_dtype, cs) : launch_delta_simt_fwd(a, (int)shape->in_dtype, (int)shape->out_dtype, cs));
  return LA_OK;
}

la_status la_delta_bwd(const la_delta_shape* shape, const void* q, const void* k, const void* v, const float* g, const float* beta,
                       const void* d_o, void* dq, void* dk, void* dv, float* dg, float* dbeta, const float* kv_in,
                       const float* grad_kv_out, float* grad_kv_in, const void* fwd_workspace, void* workspace,
                       size_t workspace_bytes, void* stream) {
  la_status st = check_delta(shape);
  if (st != LA_OK) return st;
  if (!q || !k || !v || !g || !beta || !d_o || !dq || !dk || !dv || !dg || !dbeta) return LA_ERR_INVALID_ARG;
  if (any_unaligned({q, k, v, g, beta, d_o, dq, dk, dv, dg, dbeta, kv_in, grad_kv_out, grad_kv_in})) return LA_ERR_INVALID_ARG;
  bool tensor;
  if ((st = delta_path(shape, &tensor)) != LA_OK) return st;
  const size_t bwd = delta_bytes(shape, tensor, true), need = bwd + (fwd_workspace ? 0 : delta_bytes(shape, tensor, false));
  if (!workspace || workspace_bytes < need) return LA_ERR_WORKSPACE;
  if ((reinterpret_cast<uintptr_t>(workspace) | reinterpret_cast<uintptr_t>(fwd_workspace)) & 255u) return LA_ERR_INVALID_ARG;
  if (fwd_workspace) {
    const uintptr_t w = reinterpret_cast<uintptr_t>(workspace), f = reinterpret_cast<uintptr_t>(fwd_workspace);
    if (f < w + bwd && w < f + delta_bytes(shape, tensor, false)) return LA_ERR_INVALID_ARG;
  }
  if ((st = check_device()) != LA_OK) return st;
  DeltaArgs a = delta_args(shape, tensor);
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.d_o = d_o;
  a.dq = dq; a.dk = dk; a.dv = dv; a.dg = dg; a.dbeta = dbeta;
  a.kv_in = kv_in; a.grad_kv_out = grad_kv_out; a.grad_kv_in = grad_kv_in;
  a.ws_bwd = workspace;
  a.ws = fwd_workspace ? const_cast<void*>(fwd_workspace) : static_cast<char*>(workspace) + bwd;
  const cudaStream_t cs = static_cast<cudaStream_t>(stream);
  const bool have = fwd_workspace != nullptr;
  LA_TRY_CUDA(tensor ? launch_delta_tc_bwd(a, have, (int)shape->out_dtype, cs)
                     : launch_delta_simt_bwd(a, have, (int)shape->in_dtype, (int)shape->out_dtype, cs));
  return LA_OK;
}

la_status la_delta_steps(const la_delta_shape* shape, const void* q, const void* k, const void* v, const float* g, const float* beta,
                         float* kv, void* o, void* stream) {
  la_status st = check_delta(shape);
  if (st != LA_OK) return st;
  if (!q || !k || !v || !g || !beta || !kv || !o) return LA_ERR_INVALID_ARG;
  if (any_unaligned({q, k, v, g, beta, kv, o})) return LA_ERR_INVALID_ARG;
  if ((st = check_device()) != LA_OK) return st;
  DeltaArgs a = delta_args(shape, false);
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.o = o;
  a.kv_out = kv;
  LA_TRY_CUDA(launch_delta_steps(a, (int)shape->in_dtype, (int)shape->out_dtype, static_cast<cudaStream_t>(stream)));
  return LA_OK;
}

size_t la_block_norm_workspace_bytes(const la_block_norm_shape* shape) {
  if (check_norm(shape) != LA_OK) return (size_t)-1;
  return (size_t)norm_parts(shape) * 3 * shape->D * sizeof(float);
}

la_status la_block_norm_fwd(const la_block_norm_shape* shape, const void* x, const void* y, const void* u, const float* w_post,
                            const float* s, const float* w_pre, void* h, void* n, void* stream) {
  la_status st = check_norm(shape);
  if (st != LA_OK) return st;
  if (!x || !y || (!h && !n)) return LA_ERR_INVALID_ARG;
  if (any_unaligned({x, y, u, w_post, s, w_pre, h, n})) return LA_ERR_INVALID_ARG;
  if ((st = check_device()) != LA_OK) return st;
  BlockNormArgs a = norm_args(shape, x, y, u, w_post, s, w_pre);
  a.h = h;
  a.n = n;
  LA_TRY_CUDA(launch_block_norm(a, false, (int)shape->dtype, (int)shape->res_dtype, static_cast<cudaStream_t>(stream)));
  return LA_OK;
}

la_status la_block_norm_bwd(const la_block_norm_shape* shape, const void* x, const void* y, const void* u, const float* w_post,
                            const float* s, const float* w_pre, const void* dh, const void* dn, void* dx, void* dy, void* du,
                            float* dw_post, float* ds, float* dw_pre, void* workspace, size_t workspace_bytes, void* stream) {
  la_status st = check_norm(shape);
  if (st != LA_OK) return st;
  if (!x || !y || (!dh && !dn) || !dx || !dy || (u != nullptr) != (du != nullptr)) return LA_ERR_INVALID_ARG;
  if (any_unaligned({x, y, u, w_post, s, w_pre, dh, dn, dx, dy, du, dw_post, ds, dw_pre})) return LA_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < la_block_norm_workspace_bytes(shape)) return LA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return LA_ERR_INVALID_ARG;
  if ((st = check_device()) != LA_OK) return st;
  BlockNormArgs a = norm_args(shape, x, y, u, w_post, s, w_pre);
  a.dh = dh; a.dn = dn; a.dx = dx; a.dy = dy; a.du = du;
  a.dw_post = dw_post; a.ds = ds; a.dw_pre = dw_pre;
  a.parts = static_cast<float*>(workspace);
  a.nparts = norm_parts(shape);
  LA_TRY_CUDA(launch_block_norm(a, true, (int)shape->dtype, (int)shape->res_dtype, static_cast<cudaStream_t>(stream)));
  return LA_OK;
}

}  // extern "C"
