// The gated delta rule on the CUDA cores (formulas: la_delta.cuh): fp32 inputs, and bf16 inputs where the caller asks for this path.
// Everything between input and output is fp32, chunk sums of log decays are double.
//
// Chunks of 64 tokens.  What depends on a chunk's own tokens alone (That, Uhat, What) is made for all chunks at once, then one walk
// over the chunks carries the state, a thread block per 32 value columns of a head (the columns of S do not meet), then the
// outputs are made for all chunks at once; backward the same with the adjoint.  The workspace keeps, per head and chunk,
//   What [64, D], Y [64, D] (Uhat until the walk), That [64, 64], S [D, D] (entering)          forward
//   dV' [64, D] (its part from the scores until the walk), E' [D, D] (leaving)                  backward
// Products read four values of consecutive k at a time, since with one at a time shared memory has eight words to give for sixteen
// multiplications.  1 x 2 heads x 256 tokens, d = 64, forward and backward, us: 131, of which the two walks 45 and the gradients 39 (one value at a
// time, rows fetched when their turn comes and the inverse row by row 214): eight thread blocks, whose latency bounds it.  It
// is the path for checks and small models.
#include "la_delta.cuh"

namespace la {
namespace {

constexpr int C = DELTA_SIMT_CHUNK, THREADS = 256, SLICE = 32, PC = C + 4;  // PC, PD: pitch of rows of C and of D values

template <int D>
struct Record {
  static constexpr size_t W = 0, Y = W + C * D, T = Y + C * D, S = T + C * C, FWD = S + D * D;  // in floats
  static constexpr size_t L = 0, E = L + C * D, BWD = E + D * D;
};

// Operands of a product, four values of consecutive k at a time: rows along which k runs (one access, so their pitch is a multiple of
// 16 bytes; that of four more than a multiple of 32 values keeps the rows of a warp in different banks), rows of one k each, and values
// of a function; all of them times a value per row or per k.
struct Along {
  const float* p;
  int pitch;
  __device__ __forceinline__ void four(int r, int k, float (&x)[4]) const {
    const float4 v = *reinterpret_cast<const float4*>(p + r * pitch + k);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  }
};
struct Across {
  const float* p;
  int pitch;
  __device__ __forceinline__ void four(int r, int k, float (&x)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = p[(k + i) * pitch + r];
  }
};
template <typename F>
struct Of {
  F f;  // f(k, row)
  __device__ __forceinline__ void four(int r, int k, float (&x)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = f(k + i, r);
  }
};
template <typename F>
__device__ __forceinline__ Of<F> of(F f) { return {f}; }
template <typename A, bool ROW>
struct Times {
  A a;
  const float* by;
  __device__ __forceinline__ void four(int r, int k, float (&x)[4]) const {
    a.four(r, k, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= by[ROW ? r : k + i];
  }
};
template <typename A>
__device__ __forceinline__ Times<A, false> times_k(A a, const float* by) { return {a, by}; }
template <typename A>
__device__ __forceinline__ Times<A, true> times_row(A a, const float* by) { return {a, by}; }

// acc[i][j] += sum_k a(row, k) b(col, k) for row = ty + 16 i, col = tx + 16 j
template <int M, int N, typename A, typename B>
__device__ __forceinline__ void product(float (&acc)[M / 16][N / 16], int K, A a, B b) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll 2
  for (int k = 0; k < K; k += 4) {
    float x[M / 16][4], y[N / 16][4];
#pragma unroll
    for (int i = 0; i < M / 16; ++i) a.four(ty + 16 * i, k, x[i]);
#pragma unroll
    for (int j = 0; j < N / 16; ++j) b.four(tx + 16 * j, k, y[j]);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int i = 0; i < M / 16; ++i)
#pragma unroll
        for (int j = 0; j < N / 16; ++j) acc[i][j] = fmaf(x[i][kk], y[j][kk], acc[i][j]);
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

// Rows [n of C][D] of a token tensor, zero behind the last one, on their way to shared memory; in registers while a product runs.
template <int D, int PITCH = D + 4>
struct Rows {
  float x[C * D / THREADS];
  template <typename T>
  __device__ __forceinline__ void fetch(const T* src, long long stride, int n) {
#pragma unroll
    for (int i = 0; i < C * D / THREADS; ++i) {
      const int at = i * THREADS + threadIdx.x, t = at / D;
      x[i] = t < n ? to_f32(src[t * stride + at % D]) : 0.f;
    }
  }
  __device__ __forceinline__ void put(float* dst) const {
#pragma unroll
    for (int i = 0; i < C * D / THREADS; ++i) {
      const int at = i * THREADS + threadIdx.x;
      dst[at / D * PITCH + at % D] = x[i];
    }
  }
};
template <int D, typename T>
__device__ __forceinline__ void load_rows(float* dst, const T* src, long long stride, int n) {
  Rows<D> rows;
  rows.fetch(src, stride, n);
  rows.put(dst);
}

// sums of the log decays up to each token, and beta; tokens behind the last one forget nothing and write nothing
struct Gates {
  double sum[C];
  float beta[C], since[C], until[C];  // since: decay from the state entering to the token; until: from the token to the chunk's end
  float all;
};
struct Gate {
  float g, beta;
};
__device__ __forceinline__ Gate fetch_gate(const DeltaArgs& a, const Place& p) {
  const int t = threadIdx.x;
  if (t >= p.n) return {0.f, 0.f};
  return {a.g[p.gate + t * a.gT], a.beta[p.gate + t * a.gT]};
}
__device__ __forceinline__ void make_gates(Gates& s, const Gate& own) {
  const int t = threadIdx.x;
  double x = clamped_log_decay(own.g);
  if (t < C) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, x, o);
      if ((t & 31) >= o) x += y;
    }
    s.sum[t] = x;
    s.beta[t] = own.beta;
  }
  __syncthreads();
  const double half = s.sum[C / 2 - 1], end = half + s.sum[C - 1];
  __syncthreads();
  if (t < C) {
    if (t >= C / 2) x += half;
    s.sum[t] = x;
    s.since[t] = expf((float)x);
    s.until[t] = expf((float)(end - x));
    if (t == 0) s.all = expf((float)end);
  }
  __syncthreads();
}
__device__ __forceinline__ void load_gates(Gates& s, const DeltaArgs& a, const Place& p) { make_gates(s, fetch_gate(a, p)); }
__device__ __forceinline__ float decay(const Gates& s, int i, int j) { return expf((float)(s.sum[i] - s.sum[j])); }

// ---- That, Uhat, What -----------------------------------------------------------------------------------------------------------
template <typename TI, int D>
__global__ void __launch_bounds__(THREADS) delta_prepare_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  constexpr int PD = D + 4;
  float* const x = smem;           // k, then v
  float* const n = x + C * PD;     // n diag(beta)
  float* const t = n + C * PC;
  __shared__ Gates gates;
  grid_dep_wait();
  grid_dep_launch();
  const Place p = place(a, blockIdx.y, blockIdx.x);
  float* rec = static_cast<float*>(a.ws) + p.rec * Record<D>::FWD;
  const int tid = threadIdx.x, lane = tid & 31;
  const Gate own = fetch_gate(a, p);
  load_rows<D>(x, static_cast<const TI*>(a.k) + p.krow, a.sTk, p.n);
  make_gates(gates, own);
  {
    float acc[4][4];
    clear(acc);
    product<C, C>(acc, D, Along{x, PD}, Along{x, PD});
    each(acc, [&](int i, int j, float v) { n[i * PC + j] = i > j ? v * decay(gates, i, j) * gates.beta[j] : 0.f; });
  }
  Rows<D> v;  // on their way until the keys are no longer needed
  v.fetch(static_cast<const TI*>(a.v) + p.row, a.sT, p.n);
  __syncthreads();
  // the inverse: blocks of 32 on the diagonal by forward substitution, a warp each, a column to a lane; the one below is -T22 (n21 T11),
  // made by way of the one above, which is zero
  if (tid < 64) {
    const int at = tid >> 5 << 5;
    float y[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      float s[4] = {i == lane ? 1.f : 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int m = 0; m < i; m += 4) {
        const float4 w = *reinterpret_cast<const float4*>(n + (at + i) * PC + at + m);
        s[0] = fmaf(-w.x, y[m], s[0]);
        if (m + 1 < i) s[1] = fmaf(-w.y, y[m + 1], s[1]);
        if (m + 2 < i) s[2] = fmaf(-w.z, y[m + 2], s[2]);
        if (m + 3 < i) s[3] = fmaf(-w.w, y[m + 3], s[3]);
      }
      y[i] = (s[0] + s[1]) + (s[2] + s[3]);
      t[(at + i) * PC + at + lane] = y[i];
    }
  }
  __syncthreads();
  {
    const int r = tid >> 3, c = (tid & 7) * 4;
    auto block = [&](const float* left, const float* right, float sign, float* to) {  // [32, 32], four columns of a row to a thread
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
      for (int m = 0; m < 32; ++m) {
        const float l = left[r * PC + m];
        const float4 w = *reinterpret_cast<const float4*>(right + m * PC + c);
        s[0] = fmaf(l, w.x, s[0]);
        s[1] = fmaf(l, w.y, s[1]);
        s[2] = fmaf(l, w.z, s[2]);
        s[3] = fmaf(l, w.w, s[3]);
      }
      *reinterpret_cast<float4*>(to + r * PC + c) = make_float4(sign * s[0], sign * s[1], sign * s[2], sign * s[3]);
    };
    block(n + 32 * PC, t, 1.f, t + 32);
    __syncthreads();
    block(t + 32 * PC + 32, t + 32, -1.f, t + 32 * PC);
    __syncthreads();
    *reinterpret_cast<float4*>(t + r * PC + 32 + c) = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __syncthreads();
#pragma unroll 8
  for (int i = tid; i < C * C; i += THREADS) rec[Record<D>::T + i] = t[i / C * PC + i % C];
  float acc[4][D / 16];
  clear(acc);
  product<C, D>(acc, C, times_k(Along{t, PC}, gates.since), Across{x, PD});
  each(acc, [&](int i, int c, float w) { rec[Record<D>::W + i * D + c] = w; });
  __syncthreads();
  v.put(x);
  __syncthreads();
  clear(acc);
  product<C, D>(acc, C, Along{t, PC}, Across{x, PD});
  each(acc, [&](int i, int c, float u) { rec[Record<D>::Y + i * D + c] = u; });
}

// ---- the walk: S entering every chunk, Y -------------------------------------------------------------------------------------------
template <typename TI, int D>
__global__ void __launch_bounds__(THREADS) delta_walk_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  constexpr int PD = D + 4, PS = SLICE + 1;
  float* const k = smem;
  float* const w = k + C * PD;
  float* const s = w + C * PD;
  float* const y = s + D * PS;
  __shared__ Gates gates;
  grid_dep_wait();
  grid_dep_launch();
  const int bh = blockIdx.y, e0 = blockIdx.x * SLICE, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll 8
  for (int i = threadIdx.x; i < D * SLICE; i += THREADS)
    s[i / SLICE * PS + i % SLICE] = a.kv_in ? a.kv_in[((size_t)bh * D + i / SLICE) * D + e0 + i % SLICE] : 0.f;
  // a chunk's inputs come while the one before is worked on
  Rows<D> keys, whats;
  float uhat[4][2];
  Gate gate;
  auto record = [&](int c) { return static_cast<float*>(a.ws) + ((size_t)bh * a.nchunk + c) * Record<D>::FWD; };
  auto fetch = [&](int c) {
    const Place p = place(a, bh, c);
    gate = fetch_gate(a, p);
    keys.fetch(static_cast<const TI*>(a.k) + p.krow, a.sTk, p.n);
    whats.fetch(record(c) + Record<D>::W, D, C);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) uhat[i][j] = record(c)[Record<D>::Y + (ty + 16 * i) * D + e0 + tx + 16 * j];
  };
  fetch(0);
  for (int c = 0; c < a.nchunk; ++c) {
    float* const rec = record(c);
    float acc[4][2];
    __syncthreads();
    keys.put(k);
    whats.put(w);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = -uhat[i][j];
    make_gates(gates, gate);
    if (c + 1 < a.nchunk) fetch(c + 1);
#pragma unroll 8
    for (int i = threadIdx.x; i < D * SLICE; i += THREADS) rec[Record<D>::S + (i / SLICE) * D + e0 + i % SLICE] = s[i / SLICE * PS + i % SLICE];
    product<C, SLICE>(acc, D, Along{w, PD}, Across{s, PS});
    each(acc, [&](int i, int e, float v) {
      rec[Record<D>::Y + i * D + e0 + e] = -v;
      y[i * PS + e] = -v * (gates.beta[i] * gates.until[i]);
    });
    __syncthreads();
    float next[D / 16][2];
    clear(next);
    product<D, SLICE>(next, C, Across{k, PD}, Across{y, PS});
    each(next, [&](int x, int e, float v) { s[x * PS + e] = fmaf(gates.all, s[x * PS + e], v); });
  }
  __syncthreads();
  if (a.kv_out)
#pragma unroll 8
    for (int i = threadIdx.x; i < D * SLICE; i += THREADS)
      a.kv_out[((size_t)bh * D + i / SLICE) * D + e0 + i % SLICE] = s[i / SLICE * PS + i % SLICE];
}

// ---- O ------------------------------------------------------------------------------------------------------------------------------
template <typename TI, typename TO, int D>
__global__ void __launch_bounds__(THREADS) delta_output_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  constexpr int PD = D + 4;
  float* const q = smem;
  float* const k = q + C * PD;
  float* const f = k + C * PD;
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
    product<C, C>(acc, D, Along{q, PD}, Along{k, PD});
    each(acc, [&](int i, int j, float v) { f[i * PC + j] = i >= j ? v * decay(gates, i, j) * gates.beta[j] : 0.f; });
  }
  __syncthreads();
  float acc[4][D / 16];
  clear(acc);
  product<C, D>(acc, D, Along{q, PD}, Across{rec + Record<D>::S, D});
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < D / 16; ++j) acc[i][j] *= gates.since[(threadIdx.x >> 4) + 16 * i];
  product<C, D>(acc, C, Along{f, PC}, Across{rec + Record<D>::Y, D});
  TO* o = static_cast<TO*>(a.o) + p.row;
  each(acc, [&](int i, int e, float v) {
    if (i < p.n) o[i * a.sT + e] = from_f32<TO>(a.scale * v);
  });
}

// ---- backward: the scores' part of dV' ----------------------------------------------------------------------------------------------
template <typename TI, int D>
__global__ void __launch_bounds__(THREADS) delta_scores_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  constexpr int PD = D + 4;
  float* const q = smem;
  float* const k = q + C * PD;
  float* const f = k + C * PD;
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
    product<C, C>(acc, D, Along{q, PD}, Along{k, PD});
    each(acc, [&](int i, int j, float v) { f[i * PC + j] = i >= j ? v * decay(gates, i, j) : 0.f; });
  }
  __syncthreads();
  load_rows<D>(q, static_cast<const TI*>(a.d_o) + p.row, a.sT, p.n);
  __syncthreads();
  float acc[4][D / 16];
  clear(acc);
  product<C, D>(acc, C, Across{f, PC}, Across{q, PD});
  each(acc, [&](int j, int e, float v) { rec[Record<D>::L + j * D + e] = a.scale * v; });
}

// ---- backward: the walk, E' leaving every chunk, dV' ----------------------------------------------------------------------------------
template <typename TI, int D>
__global__ void __launch_bounds__(THREADS) delta_walk_back_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  constexpr int PD = D + 4, PS = SLICE + 1;
  float* const k = smem;
  float* const w = k + C * PD;
  float* const q = w + C * PD;
  float* const s = q + C * PD;
  float* const y = s + D * PS;
  float* const d_o = y + C * PS;
  __shared__ Gates gates;
  grid_dep_wait();
  grid_dep_launch();
  const int bh = blockIdx.y, e0 = blockIdx.x * SLICE, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll 8
  for (int i = threadIdx.x; i < D * SLICE; i += THREADS)
    s[i / SLICE * PS + i % SLICE] = a.grad_kv_out ? a.grad_kv_out[((size_t)bh * D + i / SLICE) * D + e0 + i % SLICE] : 0.f;
  Rows<D> keys, queries, whats;
  Rows<SLICE, PS> outs;
  float scores[4][2];
  Gate gate;
  auto record = [&](int c) { return static_cast<float*>(a.ws_bwd) + ((size_t)bh * a.nchunk + c) * Record<D>::BWD; };
  auto fetch = [&](int c) {
    const Place p = place(a, bh, c);
    gate = fetch_gate(a, p);
    keys.fetch(static_cast<const TI*>(a.k) + p.krow, a.sTk, p.n);
    queries.fetch(static_cast<const TI*>(a.q) + p.krow, a.sTk, p.n);
    whats.fetch(static_cast<const float*>(a.ws) + p.rec * Record<D>::FWD + Record<D>::W, D, C);
    outs.fetch(static_cast<const TI*>(a.d_o) + p.row + e0, a.sT, p.n);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) scores[i][j] = record(c)[Record<D>::L + (ty + 16 * i) * D + e0 + tx + 16 * j];
  };
  fetch(a.nchunk - 1);
  for (int c = a.nchunk - 1; c >= 0; --c) {
    float* const rec = record(c);
    float from_scores[4][2];
    __syncthreads();
    keys.put(k);
    queries.put(q);
    whats.put(w);
    outs.put(d_o);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) from_scores[i][j] = scores[i][j];
    make_gates(gates, gate);
    if (c) fetch(c - 1);
#pragma unroll 8
    for (int i = threadIdx.x; i < D * SLICE; i += THREADS) rec[Record<D>::E + (i / SLICE) * D + e0 + i % SLICE] = s[i / SLICE * PS + i % SLICE];
    float acc[4][2];
    clear(acc);
    product<C, SLICE>(acc, D, Along{k, PD}, Across{s, PS});
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = ty + 16 * i, e = tx + 16 * j;
        const float got = fmaf(gates.until[r], acc[i][j], from_scores[i][j]);
        rec[Record<D>::L + r * D + e0 + e] = got;
        y[r * PS + e] = -got * gates.beta[r];
        d_o[r * PS + e] *= a.scale * gates.since[r];
      }
    __syncthreads();
    float next[D / 16][2];
    clear(next);
    product<D, SLICE>(next, C, Across{q, PD}, Across{d_o, PS});
    product<D, SLICE>(next, C, Across{w, PD}, Across{y, PS});
    each(next, [&](int x, int e, float v) { s[x * PS + e] = fmaf(gates.all, s[x * PS + e], v); });
  }
  __syncthreads();
  if (a.grad_kv_in)
#pragma unroll 8
    for (int i = threadIdx.x; i < D * SLICE; i += THREADS)
      a.grad_kv_in[((size_t)bh * D + i / SLICE) * D + e0 + i % SLICE] = s[i / SLICE * PS + i % SLICE];
}

// ---- backward: gradients.  A thread block per key head and chunk takes the value heads of the group in order. --------------------------
template <typename TI, typename TO, int D>
__global__ void __launch_bounds__(THREADS) delta_grad_kernel(const DeltaArgs a) {
  extern __shared__ float smem[];
  constexpr int PD = D + 4;
  constexpr bool KEPT = D == 64;  // keys and queries stay in shared memory (D = 128: in the state's place, until it comes)
  float* const y = smem;
  float* const d_o = y + C * PD;  // that of dV' before
  float* const dr = d_o + C * PD;
  float* const f = dr + C * PD;
  float* const h = f + C * PC;  // That, then -H
  float* const z = h + C * PC;
  float* const st = z + C * PC;  // [D][PD]: S, then E'
  float* const ks = KEPT ? st + D * PD : st;
  float* const qs = ks + C * PD;
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
    auto key = [&](int t, int x) { return KEPT ? ks[t * PD + x] : t < p.n ? to_f32(kk[t * a.sTk + x]) : 0.f; };
    auto query = [&](int t, int x) { return KEPT ? qs[t * PD + x] : t < p.n ? to_f32(qq[t * a.sTk + x]) : 0.f; };
    auto load_state = [&](const float* from) {
#pragma unroll 16
      for (int i = tid; i < D * D; i += THREADS) st[i / D * PD + i % D] = from[i];
    };
    __syncthreads();
    {
      const Gate own = fetch_gate(a, p);
      Rows<D> r0, r1;
      r0.fetch(fwd + Record<D>::Y, D, C);
      r1.fetch(rec + Record<D>::L, D, C);
      r0.put(y);
      r1.put(d_o);
#pragma unroll
      for (int i = tid; i < C * C; i += THREADS) h[i / C * PC + i % C] = fwd[Record<D>::T + i];
      if (!KEPT || gh == 0) {
        r0.fetch(kk, a.sTk, p.n);
        r1.fetch(qq, a.sTk, p.n);
        r0.put(ks);
        r1.put(qs);
      }
      make_gates(gates, own);
    }
    Rows<D> outs;
    outs.fetch(static_cast<const TI*>(a.d_o) + p.row, a.sT, p.n);
    // dR = That^T diag(beta) dV', and dV' . Y
    {
      float acc[4][D / 16];
      clear(acc);
      product<C, D>(acc, C, times_k(Across{h, PC}, gates.beta), Across{d_o, PD});
      TO* dv = static_cast<TO*>(a.dv) + p.row;
      each(acc, [&](int j, int e, float v) {
        dr[j * PD + e] = v;
        if (j < p.n) dv[j * a.sT + e] = from_f32<TO>(v);
      });
    }
    float dbeta = 0.f;
    {
      const int t = tid >> 2;
      for (int e = tid & 3; e < D; e += 4) dbeta = fmaf(d_o[t * PD + e], y[t * PD + e], dbeta);
    }
    __syncthreads();
    outs.put(d_o);
    if (KEPT) load_state(fwd + Record<D>::S);
    // Hh, with the products of the keys for dbeta; F
    {
      float hh[4][4], n[4][4];
      clear(hh);
      clear(n);
      product<C, C>(hh, D, Along{dr, PD}, Along{y, PD});
      product<C, C>(n, D, Along{ks, PD}, Along{ks, PD});
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = ty + 16 * i, c = tx + 16 * j;
          const float v = r > c ? hh[i][j] * decay(gates, r, c) : 0.f;
          h[r * PC + c] = -v;
          f[r * PC + c] = z[r * PC + c] = r > c ? n[i][j] * v : 0.f;
        }
    }
    __syncthreads();
    {
      const int j = tid >> 2;
      for (int i = tid & 3; i < C; i += 4) dbeta -= f[i * PC + j];
      dbeta += __shfl_xor_sync(0xffffffffu, dbeta, 1);
      dbeta += __shfl_xor_sync(0xffffffffu, dbeta, 2);
      if ((tid & 3) == 0 && j < p.n) a.dbeta[p.gate + j * a.gT] = dbeta;
    }
    __syncthreads();
    {
      float acc[4][4], qk[4][4];
      clear(acc);
      clear(qk);
      product<C, C>(acc, D, Along{d_o, PD}, Along{y, PD});
      product<C, C>(qk, D, Along{qs, PD}, Along{ks, PD});
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int r = ty + 16 * i, c = tx + 16 * j;
          const float v = r >= c ? a.scale * acc[i][j] * decay(gates, r, c) * gates.beta[c] : 0.f;
          f[r * PC + c] = v;
          h[r * PC + c] *= gates.beta[c];
          z[r * PC + c] = fmaf(v, qk[i][j], -gates.beta[c] * z[r * PC + c]);
        }
    }
    __syncthreads();
    if (!KEPT) {
      load_state(fwd + Record<D>::S);
      __syncthreads();
    }
    for (int r = tid >> 5; r < C; r += THREADS / 32) {  // Z's sums along its rows: of the columns before s
      const int lane = tid & 31;
      const float2 v = *reinterpret_cast<const float2*>(z + r * PC + 2 * lane);
      float x = v.x + v.y;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const float before = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += before;
      }
      x = __shfl_up_sync(0xffffffffu, x, 1);
      if (lane == 0) x = 0.f;
      *reinterpret_cast<float2*>(z + r * PC + 2 * lane) = make_float2(x, x + v.x);
    }
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
    product<C, D>(acc, D, Along{d_o, PD}, Along{st, PD});
    scaled_dots(acc, gates.since, a.scale, query, dot_q);
    product<C, D>(acc, C, Along{f, PC}, of(key));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < D / 16; ++j) sum_q[i][j] += acc[i][j];
    // dK: what the keys read
    clear(acc);
    product<C, D>(acc, D, Along{dr, PD}, Along{st, PD});
    scaled_dots(acc, gates.since, -1.f, key, dot);
    if (tx == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) row_a[ty + 16 * i] = dot_q[i] + dot[i];
    product<C, D>(acc, C, Along{h, PC}, of(key));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < D / 16; ++j) sum_k[i][j] += acc[i][j];
    float whole = 0.f;
    __syncthreads();
#pragma unroll 16
    for (int i = tid; i < D * D; i += THREADS) {  // each thread the elements that it put there: <S, E'>, and E' in S's place
      float* const at = st + i / D * PD + i % D;
      const float e = rec[Record<D>::E + i];
      whole = fmaf(*at, e, whole);
      *at = e;
    }
    whole *= gates.all;
    __syncthreads();
    // dK: what the keys write
    clear(acc);
    product<C, D>(acc, D, times_row(Along{y, PD}, gates.beta), Along{st, PD});
    scaled_dots(acc, gates.until, 1.f, key, dot);
    if (tx == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) row_b[ty + 16 * i] = dot[i];
    product<C, D>(acc, C, Across{f, PC}, of(query));
    product<C, D>(acc, C, Across{h, PC}, of(key));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < D / 16; ++j) sum_k[i][j] += acc[i][j];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) whole += __shfl_xor_sync(0xffffffffu, whole, o);
    if ((tid & 31) == 0) part[tid >> 5] = whole;
    __syncthreads();
    {  // four threads to a token
      const int t = tid >> 2;
      float x = 0.f;
      for (int j = tid & 3; j < t; j += 4) x += row_b[j];
      for (int i = t + (tid & 3); i < p.n; i += 4) x += z[i * PC + t] + row_a[i];
      x += __shfl_xor_sync(0xffffffffu, x, 1);
      x += __shfl_xor_sync(0xffffffffu, x, 2);
      for (int i = 0; i < THREADS / 32; ++i) x += part[i];
      if ((tid & 3) == 0 && t < p.n) a.dg[p.gate + t * a.gT] = x;
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
  const cudaError_t err = start(delta_prepare_kernel<TI, D>, K_PREPASS, chunks, C * (D + 4) + 2 * C * PC, a, stream);
  if (err != cudaSuccess) return err;
  return start(delta_walk_kernel<TI, D>, K_SCAN, slices, 2 * C * (D + 4) + (D + C) * (SLICE + 1), a, stream);
}
template <typename TI, typename TO, int D>
cudaError_t fwd_t(const DeltaArgs& a, cudaStream_t stream) {
  const cudaError_t err = states<TI, D>(a, stream);
  if (err != cudaSuccess) return err;
  return start(delta_output_kernel<TI, TO, D>, K_WALK, dim3(a.nchunk, a.B * a.H), 2 * C * (D + 4) + C * PC, a, stream);
}
template <typename TI, typename TO, int D>
cudaError_t bwd_t(const DeltaArgs& a, bool have_fwd, cudaStream_t stream) {
  cudaError_t err = have_fwd ? cudaSuccess : states<TI, D>(a, stream);
  if (err != cudaSuccess) return err;
  const dim3 chunks(a.nchunk, a.B * a.H), slices(D / SLICE, a.B * a.H);
  err = start(delta_scores_kernel<TI, D>, K_PREPASS, chunks, 2 * C * (D + 4) + C * PC, a, stream);
  if (err != cudaSuccess) return err;
  err = start(delta_walk_back_kernel<TI, D>, K_SCAN, slices, 3 * C * (D + 4) + (D + 2 * C) * (SLICE + 1), a, stream);
  if (err != cudaSuccess) return err;
  return start(delta_grad_kernel<TI, TO, D>, K_WALK_PAIR, dim3(a.nchunk, a.B * a.Hk),
               3 * C * (D + 4) + 3 * C * PC + D * (D + 4) + (D == 64 ? 2 * C * (D + 4) : 0), a, stream);
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
