// Recurrent form of the gated delta rule for all (batch, value head) pairs, state [BH, D, D] fp32 updated in place:
//   S <- a S,   r = v - S^T k,   S <- S + beta k r^T,   o = scale S^T q        (a = exp(g)).
// The state is read once, kept in registers over the T >= 1 tokens of the call and written once, as in the plain decode kernel: the
// step moves 8 D^2 bytes of state against 7 D^2 flops, so HBM bounds it where there are many states, and where there are few the
// round trips do.  A column of S needs two sums over its rows, S^T k before the update and S^T q after it.  The second is
//   S_new^T q = a S^T q + beta (q . k) r,
// so both are taken of the state as it is, in one pass with one barrier to a token.  No atomics, the order of every sum is fixed: N
// calls with one token give the bits of one call with N.  64 x 32 states, d = 128: 44 us, 6.2 TB/s (94 % of the copy bandwidth); 32 states 3.4 us
// of the device, 6.2 to 6.6 called one after the other.
#include "la_delta.cuh"

namespace la {
namespace {

constexpr int THREADS = 256;
constexpr int CHUNK = 8;  // tokens whose inputs are on chip at a time, one warp each for q . k

template <typename TI, typename TO, int D>
__global__ void __launch_bounds__(THREADS) delta_steps_kernel(const DeltaArgs a) {
  constexpr int LPR = D / 4;          // threads to a row of the state, four columns each
  constexpr int RPP = THREADS / LPR;  // rows at a time
  constexpr int PASSES = D / RPP;
  __shared__ alignas(16) float sq[CHUNK][D], sk[CHUNK][D], sv[CHUNK][D];
  __shared__ float qk[CHUNK], decay[CHUNK], beta[CHUNK];
  __shared__ float4 red[2][2][RPP][LPR];
  grid_dep_wait();
  grid_dep_launch();
  const int bh = blockIdx.x, b = bh / a.H, h = bh % a.H, hk = h / (a.H / a.Hk);
  const int tid = threadIdx.x, col4 = tid % LPR, row0 = tid / LPR;
  float4* const state = reinterpret_cast<float4*>(a.kv_out + (size_t)bh * D * D);
  const long long row = b * a.sB + h * a.sH, krow = b * a.sBk + hk * a.sHk, gate = b * a.gB + h * a.gH;

  float4 s[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) s[p] = ld_f4_streaming(&state[(size_t)(row0 + p * RPP) * LPR + col4]);

  for (int t = 0; t < a.N; ++t) {
    const int u = t % CHUNK;
    if (u == 0) {
      if (t > 0) __syncthreads();  // the chunk before has been read
      const int n = min(CHUNK, a.N - t);
      for (int x = tid; x < n * LPR; x += THREADS) {
        const int tok = x / LPR, c = x % LPR * 4;
        const long long kat = krow + (t + tok) * a.sTk + c;
        float w[4];
        Vec4<TI>::load(static_cast<const TI*>(a.q) + kat, w);
        *reinterpret_cast<float4*>(&sq[tok][c]) = make_float4(w[0], w[1], w[2], w[3]);
        Vec4<TI>::load(static_cast<const TI*>(a.k) + kat, w);
        *reinterpret_cast<float4*>(&sk[tok][c]) = make_float4(w[0], w[1], w[2], w[3]);
        Vec4<TI>::load(static_cast<const TI*>(a.v) + row + (t + tok) * a.sT + c, w);
        *reinterpret_cast<float4*>(&sv[tok][c]) = make_float4(w[0], w[1], w[2], w[3]);
      }
      if (tid < n) {
        decay[tid] = expf(a.g[gate + (t + tid) * a.gT]);
        beta[tid] = a.beta[gate + (t + tid) * a.gT];
      }
      __syncthreads();
      if (tid / 32 < n) {  // (read behind the token's barrier)
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x = fmaf(sq[tid / 32][tid % 32 + 32 * i], sk[tid / 32][tid % 32 + 32 * i], x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (tid % 32 == 0) qk[tid / 32] = x;
      }
    }
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;  // S^T k and S^T q of this thread's rows
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const float ki = sk[u][row0 + p * RPP], qi = sq[u][row0 + p * RPP];
      x.x = fmaf(s[p].x, ki, x.x); x.y = fmaf(s[p].y, ki, x.y); x.z = fmaf(s[p].z, ki, x.z); x.w = fmaf(s[p].w, ki, x.w);
      y.x = fmaf(s[p].x, qi, y.x); y.y = fmaf(s[p].y, qi, y.y); y.z = fmaf(s[p].z, qi, y.z); y.w = fmaf(s[p].w, qi, y.w);
    }
    red[t & 1][0][row0][col4] = x;
    red[t & 1][1][row0][col4] = y;
    __syncthreads();
    x = red[t & 1][0][0][col4];
#pragma unroll
    for (int r = 1; r < RPP; ++r) {
      const float4 z = red[t & 1][0][r][col4];
      x.x += z.x; x.y += z.y; x.z += z.z; x.w += z.w;
    }
    const float dec = decay[u], bt = beta[u];
    const float4 v = *reinterpret_cast<const float4*>(&sv[u][4 * col4]);
    float4 r;  // beta (v - a S^T k)
    r.x = bt * fmaf(-dec, x.x, v.x); r.y = bt * fmaf(-dec, x.y, v.y); r.z = bt * fmaf(-dec, x.z, v.z); r.w = bt * fmaf(-dec, x.w, v.w);
    if (row0 == t % RPP) {
      y = red[t & 1][1][0][col4];
#pragma unroll
      for (int i = 1; i < RPP; ++i) {
        const float4 z = red[t & 1][1][i][col4];
        y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
      }
      const float c = qk[u];
      const float w[4] = {a.scale * fmaf(dec, y.x, c * r.x), a.scale * fmaf(dec, y.y, c * r.y), a.scale * fmaf(dec, y.z, c * r.z),
                          a.scale * fmaf(dec, y.w, c * r.w)};
      Vec4<TO>::store(static_cast<TO*>(a.o) + row + t * a.sT + 4 * col4, w);
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const float ki = sk[u][row0 + p * RPP];
      s[p].x = fmaf(ki, r.x, dec * s[p].x);
      s[p].y = fmaf(ki, r.y, dec * s[p].y);
      s[p].z = fmaf(ki, r.z, dec * s[p].z);
      s[p].w = fmaf(ki, r.w, dec * s[p].w);
    }
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) __stcs(&state[(size_t)(row0 + p * RPP) * LPR + col4], s[p]);
}

template <typename TI, typename TO, int D>
cudaError_t launch_t(const DeltaArgs& a, cudaStream_t stream) {
  KernelTimer timer(K_DECODE, stream);
  const cudaError_t err = launch_early(delta_steps_kernel<TI, TO, D>, dim3((unsigned)(a.B * a.H)), dim3(THREADS), 0, stream, 1, a);
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}

}  // namespace

cudaError_t launch_delta_steps(const DeltaArgs& a, int in_dt, int out_dt, cudaStream_t stream) {
  if (a.D == 64) {
    if (in_dt == DT_F32 && out_dt == DT_F32) return launch_t<float, float, 64>(a, stream);
    if (in_dt == DT_BF16 && out_dt == DT_F32) return launch_t<__nv_bfloat16, float, 64>(a, stream);
    if (in_dt == DT_BF16 && out_dt == DT_BF16) return launch_t<__nv_bfloat16, __nv_bfloat16, 64>(a, stream);
  } else if (a.D == 128) {
    if (in_dt == DT_F32 && out_dt == DT_F32) return launch_t<float, float, 128>(a, stream);
    if (in_dt == DT_BF16 && out_dt == DT_F32) return launch_t<__nv_bfloat16, float, 128>(a, stream);
    if (in_dt == DT_BF16 && out_dt == DT_BF16) return launch_t<__nv_bfloat16, __nv_bfloat16, 128>(a, stream);
  }
  return cudaErrorInvalidValue;
}

}  // namespace la
