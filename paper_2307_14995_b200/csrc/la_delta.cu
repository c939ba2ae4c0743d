// The gated delta rule on the CUDA cores (formulas: la_delta.cuh): fp32 inputs, and bf16 inputs where the caller asks for this path.
// Everything between input and output is fp32, chunk sums of log decays are double.
//
// Chunks of 64 tokens.  What depends on a chunk's own tokens alone (That, Uhat, What) is made for all chunks at once, then one walk
// over the chunks carries the state, a thread block per 32 value columns of a head (the columns of S do not meet), then the
// outputs are made for all chunks at once; backward the same with the adjoint.  The workspace keeps, per head and chunk,
//   What [64, D], Y [64, D] (Uhat until the walk), That [64, 64], S [D, D] (entering)          forward
//   dV' [64, D] (its part from the scores until the walk), E' [D, D] (leaving)                  backward
// The walk's two products per chunk and the passes over S and E' bound it; it is the path for checks and small models.
#include "la_delta.cuh"

namespace la {
namespace {

constexpr int C = DELTA_SIMT_CHUNK, THREADS = 256, SLICE = 32;

template <int D>
struct Record {
  static constexpr size_t W = 0, Y = W + C * D, T = Y + C * D, S = T + C * C, FWD = S + D * D;  // in floats
  static constexpr size_t L = 0, E = L + C * D, BWD = E + D * D;
};

// acc[i][j] += sum_k a(row, k) b(k, col) for row = ty + 16 i, col = tx + 16 j
template <int M, int N, typename FA, typename FB>
__device__ __forceinline__ void product(float (&acc)[M / 16][N / 16], int K, FA a, FB b) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll 4
  for (int k = 0; k < K; ++k) {
    float x[M / 16], y[N / 16];
#pragma unroll
    for (int i = 0; i < M / 16; ++i) x[i] = a(ty + 16 * i, k);
#pragma unroll
    for (int j = 0; j < N / 16; ++j) y[j] = b(k, tx + 16 * j);
#pragma unroll
    for (int i = 0; i < M / 16; ++i)
#pragma unroll
      for (int j = 0; j < N / 16; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
  }
}
template <int M, int N>
__device__ __forceinline__ void clear(float (&acc)[M][N]) {
#pragma unroll
  for (int i = 0; i < M; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) acc[i][j] = 0.f;
}
// f(row, col, value) over the elements that this thread holds
template <int M, int N, typename F>
__device__ __forceinline__ void each(const float (&acc)[M][N], F f) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < M; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) f(ty + 16 * i, tx + 16 * j, acc[i][j]);
}

struct Place {
  int b, h, hk, c, n;                // chunk c has n tokens
  long long row, krow, gate;         // element offsets of its first token
  size_t rec;                        // index of its records
};
__device__ __forceinline__ Place place(const DeltaArgs& a, int bh, int c) {
  Place p;
  p.b = bh / a.H;
  p.h = bh % a.H;
  p.hk = p.h / (a.H / a.Hk);
  p.c = c;
  p.n = min(C, a.N - c * C);
  p.row = p.b * a.sB + p.h * a.sH + (long long)c * C * a.sT;
  p.krow = p.b * a.sBk + p.hk * a.sHk + (long long)c * C * a.sTk;
  p.gate = p.b * a.gB + p.h * a.gH + (long long)c * C * a.gT;
  p.rec = (size_t)bh * a.nchunk + c;
  return p;
}

// rows [n of C][D] of a token tensor to shared memory, zero behind the last one
template <int D, typename T>
__device__ __forceinline__ void load_rows(float (*dst)[D + 1], const T* src, long long stride, int n) {
#pragma unroll 8
  for (int i = threadIdx.x; i < C * D; i += THREADS) {
    const int t = i / D, x = i % D;
    dst[t][x] = t < n ? to_f32(src[t * stride + x]) : 0.f;
  }
}

// sums of the log decays up to each token, and beta; tokens behind the last one forget nothing and write nothing
struct Gates {
  double sum[C];
  float beta[C], since[C], until[C];  // since: decay from the state entering to the token; until: from the token to the chunk's end
  float all;
};
__device__ __forceinline__ void load_gates(Gates& s, const DeltaArgs& a, const Place& p) {
  const int t = threadIdx.x;
  if (t < C) {
    s.sum[t] = t < p.n ? clamped_log_decay(a.g[p.gate + t * a.gT]) : 0.0;
    s.beta[t] = t < p.n ? a.beta[p.gate + t * a.gT] : 0.f;
  }
  __syncthreads();
  double x = 0.0, end = 0.0;
  if (t < C)
    for (int i = 0; i < C; ++i) {
      end += s.sum[i];
      if (i == t) x = end;
    }
  __syncthreads();
  if (t < C) {
    s.sum[t] = x;
    s.since[t] = expf((float)x);
    s.until[t] = expf((float)(end - x));
    if (t == 0) s.all = expf((float)end);
  }
  __syncthreads();
}
__device__ __forceinline__ float decay(const Gates& s, int i, int j) { return expf((float)(s.sum[i] - s.sum[j])); }

// ---- That, Uhat, What -----------------------------------------------------------------------------------------------------------
template <typename TI, int D>
__global__ void __launch_bounds__(THREADS) delta_prepare_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  auto x = reinterpret_cast<float(*)[D + 1]>(smem);              // k, then v
  auto n = reinterpret_cast<float(*)[C + 1]>(smem + C * (D + 1));  // n diag(beta)
  auto t = n + C;
  __shared__ Gates gates;
  grid_dep_wait();
  grid_dep_launch();
  const Place p = place(a, blockIdx.y, blockIdx.x);
  float* rec = static_cast<float*>(a.ws) + p.rec * Record<D>::FWD;
  load_rows<D>(x, static_cast<const TI*>(a.k) + p.krow, a.sTk, p.n);
  load_gates(gates, a, p);
  {
    float acc[4][4];
    clear(acc);
    product<C, C>(acc, D, [&](int i, int k) { return x[i][k]; }, [&](int k, int j) { return x[j][k]; });
    each(acc, [&](int i, int j, float v) { n[i][j] = i > j ? v * decay(gates, i, j) * gates.beta[j] : 0.f; });
  }
  __syncthreads();
  // column j of the inverse by forward substitution, four threads to a column
  const int j = threadIdx.x >> 2, part = threadIdx.x & 3;
  for (int i = 0; i < C; ++i) {
    float v = 0.f;
    for (int m = j + part; m < i; m += 4) v = fmaf(n[i][m], t[m][j], v);
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    v += __shfl_xor_sync(0xffffffffu, v, 2);
    if (part == 0) t[i][j] = i < j ? 0.f : (i == j ? 1.f : 0.f) - v;
    __syncwarp();
  }
  __syncthreads();
#pragma unroll 8
  for (int i = threadIdx.x; i < C * C; i += THREADS) rec[Record<D>::T + i] = t[i / C][i % C];
  float acc[4][D / 16];
  clear(acc);
  product<C, D>(acc, C, [&](int i, int k) { return t[i][k] * gates.since[k]; }, [&](int k, int c) { return x[k][c]; });
  each(acc, [&](int i, int c, float v) { rec[Record<D>::W + i * D + c] = v; });
  __syncthreads();
  load_rows<D>(x, static_cast<const TI*>(a.v) + p.row, a.sT, p.n);
  __syncthreads();
  clear(acc);
  product<C, D>(acc, C, [&](int i, int k) { return t[i][k]; }, [&](int k, int c) { return x[k][c]; });
  each(acc, [&](int i, int c, float v) { rec[Record<D>::Y + i * D + c] = v; });
}

// ---- the walk: S entering every chunk, Y -------------------------------------------------------------------------------------------
template <typename TI, int D>
__global__ void __launch_bounds__(THREADS) delta_walk_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  auto k = reinterpret_cast<float(*)[D + 1]>(smem);
  auto w = k + C;
  auto s = reinterpret_cast<float(*)[SLICE + 1]>(smem + 2 * C * (D + 1));
  auto y = s + D;
  __shared__ Gates gates;
  grid_dep_wait();
  grid_dep_launch();
  const int bh = blockIdx.y, e0 = blockIdx.x * SLICE;
#pragma unroll 8
  for (int i = threadIdx.x; i < D * SLICE; i += THREADS)
    s[i / SLICE][i % SLICE] = a.kv_in ? a.kv_in[((size_t)bh * D + i / SLICE) * D + e0 + i % SLICE] : 0.f;
  for (int c = 0; c < a.nchunk; ++c) {
    const Place p = place(a, bh, c);
    float* rec = static_cast<float*>(a.ws) + p.rec * Record<D>::FWD;
    __syncthreads();
    load_rows<D>(k, static_cast<const TI*>(a.k) + p.krow, a.sTk, p.n);
    load_rows<D>(w, rec + Record<D>::W, D, C);
    load_gates(gates, a, p);
#pragma unroll 8
    for (int i = threadIdx.x; i < D * SLICE; i += THREADS) rec[Record<D>::S + (i / SLICE) * D + e0 + i % SLICE] = s[i / SLICE][i % SLICE];
    float acc[4][2];
    clear(acc);
    product<C, SLICE>(acc, D, [&](int i, int x) { return w[i][x]; }, [&](int x, int e) { return s[x][e]; });
    each(acc, [&](int i, int e, float v) {
      float* at = rec + Record<D>::Y + i * D + e0 + e;
      const float got = *at - v;
      *at = got;
      y[i][e] = got * (gates.beta[i] * gates.until[i]);
    });
    __syncthreads();
    float next[D / 16][2];
    clear(next);
    product<D, SLICE>(next, C, [&](int x, int i) { return k[i][x]; }, [&](int i, int e) { return y[i][e]; });
    each(next, [&](int x, int e, float v) { s[x][e] = fmaf(gates.all, s[x][e], v); });
  }
  __syncthreads();
  if (a.kv_out)
#pragma unroll 8
    for (int i = threadIdx.x; i < D * SLICE; i += THREADS)
      a.kv_out[((size_t)bh * D + i / SLICE) * D + e0 + i % SLICE] = s[i / SLICE][i % SLICE];
}

// ---- O ------------------------------------------------------------------------------------------------------------------------------
template <typename TI, typename TO, int D>
__global__ void __launch_bounds__(THREADS) delta_output_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  auto q = reinterpret_cast<float(*)[D + 1]>(smem);
  auto k = q + C;
  auto f = reinterpret_cast<float(*)[C + 1]>(smem + 2 * C * (D + 1));
  __shared__ Gates gates;
  grid_dep_wait();
  grid_dep_launch();
  const Place p = place(a, blockIdx.y, blockIdx.x);
  const float* rec = static_cast<const float*>(a.ws) + p.rec * Record<D>::FWD;
  load_rows<D>(q, static_cast<const TI*>(a.q) + p.krow, a.sTk, p.n);
  load_rows<D>(k, static_cast<const TI*>(a.k) + p.krow, a.sTk, p.n);
  load_gates(gates, a, p);
  {
    float acc[4][4];
    clear(acc);
    product<C, C>(acc, D, [&](int i, int x) { return q[i][x]; }, [&](int x, int j) { return k[j][x]; });
    each(acc, [&](int i, int j, float v) { f[i][j] = i >= j ? v * decay(gates, i, j) * gates.beta[j] : 0.f; });
  }
  __syncthreads();
  float acc[4][D / 16];
  clear(acc);
  product<C, D>(acc, D, [&](int i, int x) { return q[i][x]; }, [&](int x, int e) { return rec[Record<D>::S + x * D + e]; });
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < D / 16; ++j) acc[i][j] *= gates.since[(threadIdx.x >> 4) + 16 * i];
  product<C, D>(acc, C, [&](int i, int x) { return f[i][x]; }, [&](int x, int e) { return rec[Record<D>::Y + x * D + e]; });
  TO* o = static_cast<TO*>(a.o) + p.row;
  each(acc, [&](int i, int e, float v) {
    if (i < p.n) o[i * a.sT + e] = from_f32<TO>(a.scale * v);
  });
}

// ---- backward: the scores' part of dV' ----------------------------------------------------------------------------------------------
template <typename TI, int D>
__global__ void __launch_bounds__(THREADS) delta_scores_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  auto q = reinterpret_cast<float(*)[D + 1]>(smem);
  auto k = q + C;
  auto f = reinterpret_cast<float(*)[C + 1]>(smem + 2 * C * (D + 1));
  __shared__ Gates gates;
  grid_dep_wait();
  grid_dep_launch();
  const Place p = place(a, blockIdx.y, blockIdx.x);
  float* rec = static_cast<float*>(a.ws_bwd) + p.rec * Record<D>::BWD;
  load_rows<D>(q, static_cast<const TI*>(a.q) + p.krow, a.sTk, p.n);
  load_rows<D>(k, static_cast<const TI*>(a.k) + p.krow, a.sTk, p.n);
  load_gates(gates, a, p);
  {
    float acc[4][4];
    clear(acc);
    product<C, C>(acc, D, [&](int i, int x) { return q[i][x]; }, [&](int x, int j) { return k[j][x]; });
    each(acc, [&](int i, int j, float v) { f[i][j] = i >= j ? v * decay(gates, i, j) : 0.f; });
  }
  __syncthreads();
  load_rows<D>(q, static_cast<const TI*>(a.d_o) + p.row, a.sT, p.n);
  __syncthreads();
  float acc[4][D / 16];
  clear(acc);
  product<C, D>(acc, C, [&](int j, int t) { return f[t][j]; }, [&](int t, int e) { return q[t][e]; });
  each(acc, [&](int j, int e, float v) { rec[Record<D>::L + j * D + e] = a.scale * v; });
}

// ---- backward: the walk, E' leaving every chunk, dV' ----------------------------------------------------------------------------------
template <typename TI, int D>
__global__ void __launch_bounds__(THREADS) delta_walk_back_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  auto k = reinterpret_cast<float(*)[D + 1]>(smem);
  auto w = k + C;
  auto q = w + C;
  auto s = reinterpret_cast<float(*)[SLICE + 1]>(smem + 3 * C * (D + 1));
  auto y = s + D;
  auto d_o = y + C;
  __shared__ Gates gates;
  grid_dep_wait();
  grid_dep_launch();
  const int bh = blockIdx.y, e0 = blockIdx.x * SLICE;
#pragma unroll 8
  for (int i = threadIdx.x; i < D * SLICE; i += THREADS)
    s[i / SLICE][i % SLICE] = a.grad_kv_out ? a.grad_kv_out[((size_t)bh * D + i / SLICE) * D + e0 + i % SLICE] : 0.f;
  for (int c = a.nchunk - 1; c >= 0; --c) {
    const Place p = place(a, bh, c);
    const float* fwd = static_cast<const float*>(a.ws) + p.rec * Record<D>::FWD;
    float* rec = static_cast<float*>(a.ws_bwd) + p.rec * Record<D>::BWD;
    __syncthreads();
    load_rows<D>(k, static_cast<const TI*>(a.k) + p.krow, a.sTk, p.n);
    load_rows<D>(q, static_cast<const TI*>(a.q) + p.krow, a.sTk, p.n);
    load_rows<D>(w, fwd + Record<D>::W, D, C);
    load_gates(gates, a, p);
    const TI* const in = static_cast<const TI*>(a.d_o) + p.row + e0;
#pragma unroll 8
    for (int i = threadIdx.x; i < C * SLICE; i += THREADS) {
      const int t = i / SLICE;
      d_o[t][i % SLICE] = t < p.n ? to_f32(in[t * a.sT + i % SLICE]) * (a.scale * gates.since[t]) : 0.f;
    }
#pragma unroll 8
    for (int i = threadIdx.x; i < D * SLICE; i += THREADS) rec[Record<D>::E + (i / SLICE) * D + e0 + i % SLICE] = s[i / SLICE][i % SLICE];
    float acc[4][2];
    clear(acc);
    product<C, SLICE>(acc, D, [&](int i, int x) { return k[i][x]; }, [&](int x, int e) { return s[x][e]; });
    each(acc, [&](int i, int e, float v) {
      float* at = rec + Record<D>::L + i * D + e0 + e;
      const float got = fmaf(gates.until[i], v, *at);
      *at = got;
      y[i][e] = -got * gates.beta[i];
    });
    __syncthreads();
    float next[D / 16][2];
    clear(next);
    product<D, SLICE>(next, C, [&](int x, int i) { return q[i][x]; }, [&](int i, int e) { return d_o[i][e]; });
    product<D, SLICE>(next, C, [&](int x, int i) { return w[i][x]; }, [&](int i, int e) { return y[i][e]; });
    each(next, [&](int x, int e, float v) { s[x][e] = fmaf(gates.all, s[x][e], v); });
  }
  __syncthreads();
  if (a.grad_kv_in)
#pragma unroll 8
    for (int i = threadIdx.x; i < D * SLICE; i += THREADS)
      a.grad_kv_in[((size_t)bh * D + i / SLICE) * D + e0 + i % SLICE] = s[i / SLICE][i % SLICE];
}

// ---- backward: gradients.  A thread block per key head and chunk takes the value heads of the group in order. --------------------------
template <typename TI, typename TO, int D>
__global__ void __launch_bounds__(THREADS) delta_grad_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  auto y = reinterpret_cast<float(*)[D + 1]>(smem);
  auto d_o = y + C;  // that of dV' before
  auto dr = d_o + C;
  auto f = reinterpret_cast<float(*)[C + 1]>(smem + 3 * C * (D + 1));
  auto h = f + C;
  auto z = h + C;
  float* const st = smem + 3 * C * (D + 1) + 3 * C * (C + 1);  // [D][D + 1]: S, then E'
  __shared__ Gates gates;
  __shared__ float row_a[C], row_b[C];
  __shared__ float part[THREADS / 32];
  grid_dep_wait();
  grid_dep_launch();
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, G = a.H / a.Hk;
  const int b = blockIdx.y / a.Hk, hk = blockIdx.y % a.Hk;
  float sum_q[4][D / 16], sum_k[4][D / 16];
  clear(sum_q);
  clear(sum_k);
  Place p;
  for (int gh = 0; gh < G; ++gh) {
    p = place(a, b * a.H + hk * G + gh, blockIdx.x);
    const float* fwd = static_cast<const float*>(a.ws) + p.rec * Record<D>::FWD;
    const float* rec = static_cast<const float*>(a.ws_bwd) + p.rec * Record<D>::BWD;
    const TI* const kk = static_cast<const TI*>(a.k) + p.krow;
    const TI* const qq = static_cast<const TI*>(a.q) + p.krow;
    auto key = [&](int t, int x) { return t < p.n ? to_f32(kk[t * a.sTk + x]) : 0.f; };
    auto query = [&](int t, int x) { return t < p.n ? to_f32(qq[t * a.sTk + x]) : 0.f; };
    __syncthreads();
    load_gates(gates, a, p);
    load_rows<D>(y, fwd + Record<D>::Y, D, C);
    load_rows<D>(d_o, rec + Record<D>::L, D, C);
#pragma unroll 8
    for (int i = tid; i < C * C; i += THREADS) h[i / C][i % C] = fwd[Record<D>::T + i];
    __syncthreads();
    // dR = That^T diag(beta) dV', and dV' . Y
    {
      float acc[4][D / 16];
      clear(acc);
      product<C, D>(acc, C, [&](int j, int i) { return h[i][j] * gates.beta[i]; }, [&](int i, int e) { return d_o[i][e]; });
      TO* dv = static_cast<TO*>(a.dv) + p.row;
      each(acc, [&](int j, int e, float v) {
        dr[j][e] = v;
        if (j < p.n) dv[j * a.sT + e] = from_f32<TO>(v);
      });
    }
    float dbeta = 0.f;
    {
      const int t = tid >> 2;
      for (int e = tid & 3; e < D; e += 4) dbeta = fmaf(d_o[t][e], y[t][e], dbeta);
    }
    __syncthreads();
    load_rows<D>(d_o, static_cast<const TI*>(a.d_o) + p.row, a.sT, p.n);
#pragma unroll 8
    for (int i = tid; i < D * D; i += THREADS) st[(i / D) * (D + 1) + i % D] = fwd[Record<D>::S + i];
    __syncthreads();
    // Hh, with the products of the keys for dbeta; F
    {
      float hh[4][4], n[4][4];
      clear(hh);
      clear(n);
      product<C, C>(hh, D, [&](int i, int e) { return dr[i][e]; }, [&](int e, int j) { return y[j][e]; });
      product<C, C>(n, D, [&](int i, int x) { return key(i, x); }, [&](int x, int j) { return key(j, x); });
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = ty + 16 * i, c = tx + 16 * j;
          const float v = r > c ? hh[i][j] * decay(gates, r, c) : 0.f;
          h[r][c] = v;
          f[r][c] = z[r][c] = r > c ? n[i][j] * v : 0.f;
        }
    }
    __syncthreads();
    {
      const int j = tid >> 2;
      for (int i = tid & 3; i < C; i += 4) dbeta -= f[i][j];
      dbeta += __shfl_xor_sync(0xffffffffu, dbeta, 1);
      dbeta += __shfl_xor_sync(0xffffffffu, dbeta, 2);
      if ((tid & 3) == 0 && j < p.n) a.dbeta[p.gate + j * a.gT] = dbeta;
    }
    __syncthreads();
    {
      float acc[4][4], qk[4][4];
      clear(acc);
      clear(qk);
      product<C, C>(acc, D, [&](int i, int e) { return d_o[i][e]; }, [&](int e, int j) { return y[j][e]; });
      product<C, C>(qk, D, [&](int i, int x) { return query(i, x); }, [&](int x, int j) { return key(j, x); });
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = ty + 16 * i, c = tx + 16 * j;
          const float v = r >= c ? a.scale * acc[i][j] * decay(gates, r, c) * gates.beta[c] : 0.f;
          f[r][c] = v;
          h[r][c] *= gates.beta[c];
          z[r][c] = fmaf(v, qk[i][j], -gates.beta[c] * z[r][c]);
        }
    }
    __syncthreads();
    // scales the rows of acc, and sums up the products of each with the same row of x over the sixteen threads that share it
    auto scaled_dots = [&](float(&acc)[4][D / 16], const float* with, float times, auto x, float(&dot)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dot[i] = 0.f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          acc[i][j] *= times * with[ty + 16 * i];
          dot[i] = fmaf(acc[i][j], x(ty + 16 * i, tx + 16 * j), dot[i]);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) dot[i] += __shfl_xor_sync(0xffffffffu, dot[i], o);
      }
    };
    float acc[4][D / 16], dot_q[4], dot[4];
    // dQ
    clear(acc);
    product<C, D>(acc, D, [&](int i, int e) { return d_o[i][e]; }, [&](int e, int x) { return st[x * (D + 1) + e]; });
    scaled_dots(acc, gates.since, a.scale, query, dot_q);
    product<C, D>(acc, C, [&](int i, int j) { return f[i][j]; }, [&](int j, int x) { return key(j, x); });
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < D / 16; ++j) sum_q[i][j] += acc[i][j];
    // dK: what the keys read
    clear(acc);
    product<C, D>(acc, D, [&](int i, int e) { return dr[i][e]; }, [&](int e, int x) { return st[x * (D + 1) + e]; });
    scaled_dots(acc, gates.since, 1.f, key, dot);
    if (tx == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) row_a[ty + 16 * i] = dot_q[i] - dot[i];
    product<C, D>(acc, C, [&](int i, int j) { return h[i][j]; }, [&](int j, int x) { return key(j, x); });
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < D / 16; ++j) sum_k[i][j] -= acc[i][j];
    float whole = 0.f;
#pragma unroll 8
    for (int i = tid; i < D * D; i += THREADS) whole = fmaf(st[(i / D) * (D + 1) + i % D], rec[Record<D>::E + i], whole);
    whole *= gates.all;
    __syncthreads();
#pragma unroll 8
    for (int i = tid; i < D * D; i += THREADS) st[(i / D) * (D + 1) + i % D] = rec[Record<D>::E + i];
    if (tid < C) {  // Z's sums along its rows: of the columns before s
      float x = 0.f;
      for (int s = 0; s < C; ++s) {
        const float next = x + z[tid][s];
        z[tid][s] = x;
        x = next;
      }
    }
    __syncthreads();
    // dK: what the keys write
    clear(acc);
    product<C, D>(acc, D, [&](int i, int e) { return y[i][e] * gates.beta[i]; }, [&](int e, int x) { return st[x * (D + 1) + e]; });
    scaled_dots(acc, gates.until, 1.f, key, dot);
    if (tx == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) row_b[ty + 16 * i] = dot[i];
    product<C, D>(acc, C, [&](int j, int t) { return f[t][j]; }, [&](int t, int x) { return query(t, x); });
    product<C, D>(acc, C, [&](int j, int t) { return -h[t][j]; }, [&](int t, int x) { return key(t, x); });
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < D / 16; ++j) sum_k[i][j] += acc[i][j];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) whole += __shfl_xor_sync(0xffffffffu, whole, o);
    if ((tid & 31) == 0) part[tid >> 5] = whole;
    __syncthreads();
    if (tid < p.n) {
      float x = 0.f;
      for (int i = 0; i < THREADS / 32; ++i) x += part[i];
      for (int j = 0; j < tid; ++j) x += row_b[j];
      for (int i = p.n - 1; i >= tid; --i) x += z[i][tid] + row_a[i];
      a.dg[p.gate + tid * a.gT] = x;
    }
  }
  TO* const dq = static_cast<TO*>(a.dq) + p.krow;
  TO* const dk = static_cast<TO*>(a.dk) + p.krow;
  each(sum_q, [&](int i, int x, float v) {
    if (i < p.n) dq[i * a.sTk + x] = from_f32<TO>(v);
  });
  each(sum_k, [&](int i, int x, float v) {
    if (i < p.n) dk[i * a.sTk + x] = from_f32<TO>(v);
  });
}

template <typename K>
cudaError_t start(K kern, int kind, dim3 grid, size_t floats, const DeltaArgs& a, cudaStream_t stream) {
  const size_t smem = floats * sizeof(float);
  cudaError_t err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (err != cudaSuccess) return err;
  KernelTimer timer(kind, stream);
  err = launch_early(kern, grid, dim3(THREADS), smem, stream, 1, a);
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}

template <typename TI, int D>
cudaError_t states(const DeltaArgs& a, cudaStream_t stream) {
  const dim3 chunks(a.nchunk, a.B * a.H), slices(D / SLICE, a.B * a.H);
  const cudaError_t err = start(delta_prepare_kernel<TI, D>, K_PREPASS, chunks, C * (D + 1) + 2 * C * (C + 1), a, stream);
  if (err != cudaSuccess) return err;
  return start(delta_walk_kernel<TI, D>, K_SCAN, slices, 2 * C * (D + 1) + (D + C) * (SLICE + 1), a, stream);
}
template <typename TI, typename TO, int D>
cudaError_t fwd_t(const DeltaArgs& a, cudaStream_t stream) {
  const cudaError_t err = states<TI, D>(a, stream);
  if (err != cudaSuccess) return err;
  return start(delta_output_kernel<TI, TO, D>, K_WALK, dim3(a.nchunk, a.B * a.H), 2 * C * (D + 1) + C * (C + 1), a, stream);
}
template <typename TI, typename TO, int D>
cudaError_t bwd_t(const DeltaArgs& a, bool have_fwd, cudaStream_t stream) {
  cudaError_t err = have_fwd ? cudaSuccess : states<TI, D>(a, stream);
  if (err != cudaSuccess) return err;
  const dim3 chunks(a.nchunk, a.B * a.H), slices(D / SLICE, a.B * a.H);
  err = start(delta_scores_kernel<TI, D>, K_PREPASS, chunks, 2 * C * (D + 1) + C * (C + 1), a, stream);
  if (err != cudaSuccess) return err;
  err = start(delta_walk_back_kernel<TI, D>, K_SCAN, slices, 3 * C * (D + 1) + (D + 2 * C) * (SLICE + 1), a, stream);
  if (err != cudaSuccess) return err;
  return start(delta_grad_kernel<TI, TO, D>, K_WALK_PAIR, dim3(a.nchunk, a.B * a.Hk), 3 * C * (D + 1) + 3 * C * (C + 1) + D * (D + 1), a, stream);
}

}  // namespace

size_t delta_simt_chunk_bytes(int D, bool bwd) {
  return sizeof(float) * (D == 64 ? (bwd ? Record<64>::BWD : Record<64>::FWD) : (bwd ? Record<128>::BWD : Record<128>::FWD));
}

#define LA_DELTA_TYPES(CALL)                                                                                                        \
  if (a.D == 64) {                                                                                                                  \
    if (in_dt == DT_F32 && out_dt == DT_F32) return CALL(float, float, 64);                                                         \
    if (in_dt == DT_BF16 && out_dt == DT_F32) return CALL(__nv_bfloat16, float, 64);                                                \
    if (in_dt == DT_BF16 && out_dt == DT_BF16) return CALL(__nv_bfloat16, __nv_bfloat16, 64);                                       \
  } else if (a.D == 128) {                                                                                                          \
    if (in_dt == DT_F32 && out_dt == DT_F32) return CALL(float, float, 128);                                                        \
    if (in_dt == DT_BF16 && out_dt == DT_F32) return CALL(__nv_bfloat16, float, 128);                                               \
    if (in_dt == DT_BF16 && out_dt == DT_BF16) return CALL(__nv_bfloat16, __nv_bfloat16, 128);                                      \
  }                                                                                                                                 \
  return cudaErrorInvalidValue;

cudaError_t launch_delta_simt_fwd(const DeltaArgs& a, int in_dt, int out_dt, cudaStream_t stream) {
#define CALL(I, O, D) fwd_t<I, O, D>(a, stream)
  LA_DELTA_TYPES(CALL)
#undef CALL
}
cudaError_t launch_delta_simt_bwd(const DeltaArgs& a, bool have_fwd, int in_dt, int out_dt, cudaStream_t stream) {
#define CALL(I, O, D) bwd_t<I, O, D>(a, have_fwd, stream)
  LA_DELTA_TYPES(CALL)
#undef CALL
}

}  // namespace la
