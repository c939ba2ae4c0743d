// What stands between two blocks of a model, one pass over each token's row of D features:
//   z = y r_y (.) w_post (.) act(u),   h = x + s (.) z,   n = h r_h (.) w_pre,   r_a = 1 / sqrt(mean(a^2) + eps)   (0 for a zero row
// without eps), and the gradients of <h, dh> + <n, dn>, from x, y and u again:
//   H = dh + r_h (w_pre dn - n^ mean(w_pre dn n^)),  n^ = h r_h;     dx = H,   ds = sum H z,   dw_pre = sum dn n^,
//   du = s H y^ w_post act'(u),  y^ = y r_y;     p = s H act(u) w_post,   dw_post = sum s H act(u) y^,   dy = r_y (p - y^ mean(p y^)).
//
// HBM bounds both: every input is read once and every output written once, a row stays in registers from the one to the other.  LANES
// threads share a row (a warp up to 512 features, else a part of a thread block or all of it), each with NV groups of eight
// features, 16 bytes of bf16 at a time; rows whose width is no multiple of eight are not aligned and take the same features one by
// one.  The sums over tokens (ds, dw) stay in registers over the rows that a thread block takes, leave it as one part [3][D] in the
// workspace, and a second kernel adds the parts up in order: no atomics, the same bits every time.
#include "la_block_norm.cuh"

namespace la {
namespace {

constexpr int THREADS = 256;

// eight consecutive features
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  float a[4], b[4];
  if constexpr (sizeof(T) == 2) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  } else {
    Vec4<T>::load(p, a);
    Vec4<T>::load(p + 4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    const float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[4], x[5], x[6], x[7]};
    Vec4<T>::store(p, a);
    Vec4<T>::store(p + 4, b);
  }
}

// Group v of the thread `lane` of a row: features (v LANES + lane) 8 .. + 7, or, one by one, (8 v + i) LANES + lane.
template <int LANES, bool VEC>
struct Cols {
  int lane, D;
  template <typename T>
  __device__ __forceinline__ void load(const T* row, int v, float (&x)[8], float other = 0.f) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = other;
    if (VEC) {
      const int at = (v * LANES + lane) * 8;
      if (row && at < D) load8(row + at, x);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = (8 * v + i) * LANES + lane;
        if (row && at < D) x[i] = to_f32(row[at]);
      }
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, int v, const float (&x)[8]) const {
    if (VEC) {
      const int at = (v * LANES + lane) * 8;
      if (at < D) store8(row + at, x);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = (8 * v + i) * LANES + lane;
        if (at < D) row[at] = from_f32<T>(x[i]);
      }
    }
  }
};

// Sum over the LANES threads of a row, the same in each; `slot` alternates between calls, so one barrier is enough.
template <int LANES, int ROWS>
struct RowSum {
  float part[2][ROWS][LANES <= 32 ? 1 : LANES / 32];
  __device__ __forceinline__ float operator()(float x, int slot, int row) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (LANES <= 32) return x;
    if ((threadIdx.x & 31) == 0) part[slot][row][(threadIdx.x / 32) % (LANES / 32)] = x;
    __syncthreads();
    x = part[slot][row][0];
#pragma unroll
    for (int i = 1; i < LANES / 32; ++i) x += part[slot][row][i];
    return x;
  }
};

__device__ __forceinline__ float inverse_rms(float sum, float inv_d, float eps) {
  const float m = fmaf(sum, inv_d, eps);
  return m == 0.f ? 0.f : rsqrtf(m);
}
// act(u) and its derivative
__device__ __forceinline__ float act(int kind, float u, float& slope) {
  if (kind == GATE_PLAIN) {
    slope = 1.f;
    return u;
  }
  const float s = 1.f / (1.f + expf(-u));
  if (kind == GATE_SIGMOID) {
    slope = s * (1.f - s);
    return s;
  }
  slope = fmaf(u * s, 1.f - s, s);
  return u * s;
}

template <typename T, typename TR, int LANES, int NV, bool VEC>
__global__ void __launch_bounds__(LANES > THREADS ? LANES : THREADS) block_norm_fwd_kernel(const BlockNormArgs a) {
  constexpr int ROWS = (LANES > THREADS ? LANES : THREADS) / LANES;
  __shared__ RowSum<LANES, ROWS> sum;
  grid_dep_wait();
  grid_dep_launch();
  const int sub = threadIdx.x / LANES;
  const Cols<LANES, VEC> cols{(int)threadIdx.x % LANES, a.D};
  const float inv_d = 1.f / (float)a.D;
  const long long groups = (a.rows + ROWS - 1) / ROWS;
  for (long long group = blockIdx.x; group < groups; group += gridDim.x) {
    const long long row = group * ROWS + sub;
    const bool mine = row < a.rows;  // (the others keep the barriers company)
    const long long at = mine ? row * a.D : 0;
    float y[NV][8], x[NV][8];
    float ss = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      cols.load(static_cast<const T*>(a.y) + at, v, y[v]);
      cols.load(static_cast<const TR*>(a.x) + at, v, x[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(y[v][i], y[v][i], ss);
    }
    float ry = 1.f;
    if (a.post_norm) ry = inverse_rms(sum(ss, 0, sub), inv_d, a.eps);
    ss = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float w[8], u[8], s[8];
      cols.load(a.w_post, v, w, 1.f);
      cols.load(a.s, v, s, 1.f);
      cols.load(a.u ? static_cast<const T*>(a.u) + at : nullptr, v, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float z = y[v][i] * ry * w[i], slope;
        if (a.u) z *= act(a.gate, u[i], slope);
        x[v][i] = fmaf(s[i], z, x[v][i]);
        ss = fmaf(x[v][i], x[v][i], ss);
      }
      if (mine && a.h) cols.store(static_cast<TR*>(a.h) + at, v, x[v]);
    }
    if (!a.n) continue;
    const float rh = inverse_rms(sum(ss, 1, sub), inv_d, a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float w[8];
      cols.load(a.w_pre, v, w, 1.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] *= x[v][i] * rh;
      if (mine) cols.store(static_cast<T*>(a.n) + at, v, w);
    }
  }
}

template <typename T, typename TR, int LANES, int NV, bool VEC>
__global__ void __launch_bounds__(LANES > THREADS ? LANES : THREADS) block_norm_bwd_kernel(const BlockNormArgs a) {
  constexpr int ROWS = (LANES > THREADS ? LANES : THREADS) / LANES;
  __shared__ RowSum<LANES, ROWS> sum;
  grid_dep_wait();
  grid_dep_launch();
  const int sub = threadIdx.x / LANES;
  const Cols<LANES, VEC> cols{(int)threadIdx.x % LANES, a.D};
  const float inv_d = 1.f / (float)a.D;
  const long long groups = (a.rows + ROWS - 1) / ROWS;
  float g_post[NV][8], g_s[NV][8], g_pre[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) g_post[v][i] = g_s[v][i] = g_pre[v][i] = 0.f;
  for (long long group = blockIdx.x; group < groups; group += gridDim.x) {
    const long long row = group * ROWS + sub;
    const bool mine = row < a.rows;
    const long long at = mine ? row * a.D : 0;
    float y[NV][8], h[NV][8], u[NV][8], dn[NV][8];
    float ss = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      cols.load(static_cast<const T*>(a.y) + at, v, y[v]);
      cols.load(static_cast<const TR*>(a.x) + at, v, h[v]);
      cols.load(a.u ? static_cast<const T*>(a.u) + at : nullptr, v, u[v]);
      cols.load(a.dn && mine ? static_cast<const T*>(a.dn) + at : nullptr, v, dn[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(y[v][i], y[v][i], ss);
    }
    float ry = 1.f;
    if (a.post_norm) ry = inverse_rms(sum(ss, 0, sub), inv_d, a.eps);
    ss = 0.f;
    float dot = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float w[8], s[8], wp[8];
      cols.load(a.w_post, v, w, 1.f);
      cols.load(a.s, v, s, 1.f);
      cols.load(a.w_pre, v, wp, 1.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float z = y[v][i] * ry * w[i], slope;
        if (a.u) z *= act(a.gate, u[v][i], slope);
        h[v][i] = fmaf(s[i], z, h[v][i]);
        ss = fmaf(h[v][i], h[v][i], ss);
        dot = fmaf(dn[v][i] * wp[i], h[v][i], dot);
      }
    }
    float rh = 0.f, along = 0.f;
    if (a.dn) {
      rh = inverse_rms(sum(ss, 1, sub), inv_d, a.eps);
      along = sum(dot, 0, sub) * rh * inv_d;  // mean(w_pre dn n^)
    }
    float py = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float w[8], s[8], wp[8], dh[8], du[8];
      cols.load(a.w_post, v, w, 1.f);
      cols.load(a.s, v, s, 1.f);
      cols.load(a.w_pre, v, wp, 1.f);
      cols.load(a.dh && mine ? static_cast<const TR*>(a.dh) + at : nullptr, v, dh);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float nh = h[v][i] * rh, yh = y[v][i] * ry;
        float H = dh[i];
        if (a.dn) {
          H = fmaf(rh, dn[v][i] * wp[i] - nh * along, H);
          g_pre[v][i] = fmaf(dn[v][i], nh, g_pre[v][i]);
        }
        dh[i] = H;
        float gate = 1.f, slope = 0.f;
        if (a.u) gate = act(a.gate, u[v][i], slope);
        if (mine) {
          g_s[v][i] = fmaf(H, yh * w[i] * gate, g_s[v][i]);
          g_post[v][i] = fmaf(H * s[i], yh * gate, g_post[v][i]);
        }
        du[i] = H * s[i] * yh * w[i] * slope;
        h[v][i] = H * s[i] * gate * w[i];  // p
        py = fmaf(h[v][i], yh, py);
      }
      if (mine) cols.store(static_cast<TR*>(a.dx) + at, v, dh);
      if (mine && a.u) cols.store(static_cast<T*>(a.du) + at, v, du);
    }
    if (a.post_norm) py = sum(py, 1, sub) * inv_d;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (a.post_norm) {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[v][i] = ry * (h[v][i] - y[v][i] * ry * py);
      }
      if (mine) cols.store(static_cast<T*>(a.dy) + at, v, h[v]);
    }
    __syncthreads();  // (the row's sums have two slots and are used twice)
  }
  // the thread block's part; where it has several rows at a time, their threads add up in order
  float* const part = a.parts + (size_t)blockIdx.x * 3 * a.D;
  for (int r = 0; r < ROWS; ++r) {
    if (sub == r) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = VEC ? (v * LANES + cols.lane) * 8 + i : (8 * v + i) * LANES + cols.lane;
          if (c >= a.D) continue;
          part[c] = g_post[v][i] + (r > 0 ? part[c] : 0.f);
          part[a.D + c] = g_s[v][i] + (r > 0 ? part[a.D + c] : 0.f);
          part[2 * a.D + c] = g_pre[v][i] + (r > 0 ? part[2 * a.D + c] : 0.f);
        }
    }
    __syncthreads();
  }
}

// Adds up the parts: 32 features to a thread block, the parts shared by its eight warps.
__global__ void __launch_bounds__(THREADS) block_norm_sum_kernel(const float* parts, int nparts, int D, float* dw_post, float* ds, float* dw_pre) {
  __shared__ float red[THREADS / 32][32];
  grid_dep_wait();
  grid_dep_launch();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x / 32;
  float x = 0.f;
  if (c < 3 * D) {
#pragma unroll 8
    for (int p = w; p < nparts; p += THREADS / 32) x += parts[(size_t)p * 3 * D + c];
  }
  red[w][threadIdx.x & 31] = x;
  __syncthreads();
  if (w == 0 && c < 3 * D) {
#pragma unroll
    for (int i = 1; i < THREADS / 32; ++i) x += red[i][threadIdx.x];
    float* const to = c < D ? dw_post : c < 2 * D ? ds : dw_pre;
    if (to) to[c % D] = x;
  }
}

template <typename T, typename TR, int LANES, int NV, bool VEC>
cudaError_t run(const BlockNormArgs& a, bool backward, cudaStream_t stream) {
  constexpr int BLOCK = LANES > THREADS ? LANES : THREADS, ROWS = BLOCK / LANES;
  const long long groups = (a.rows + ROWS - 1) / ROWS;
  KernelTimer timer(K_GATE, stream);
  cudaError_t err;
  if (backward) {
    err = launch_early(block_norm_bwd_kernel<T, TR, LANES, NV, VEC>, dim3((unsigned)(groups < a.nparts ? groups : a.nparts)), dim3(BLOCK), 0, stream, 1, a);
  } else {
    const long long cap = 148LL * 64;  // a few waves, then each thread block takes further rows
    err = launch_early(block_norm_fwd_kernel<T, TR, LANES, NV, VEC>, dim3((unsigned)(groups < cap ? groups : cap)), dim3(BLOCK), 0, stream, 1, a);
  }
  count_launch();
  if (err == cudaSuccess) err = cudaGetLastError();
  if (err != cudaSuccess || !backward) return err;
  const int n = (int)(groups < a.nparts ? groups : a.nparts);
  err = launch_early(block_norm_sum_kernel, dim3((unsigned)((3 * a.D + 31) / 32)), dim3(THREADS), 0, stream, 1, (const float*)a.parts, n, a.D,
                     a.dw_post, a.ds, a.dw_pre);
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}

template <typename T, typename TR, bool VEC>
cudaError_t by_width(const BlockNormArgs& a, bool backward, cudaStream_t stream) {
  if (a.D <= 256) return run<T, TR, 32, 1, VEC>(a, backward, stream);
  if (a.D <= 512) return run<T, TR, 32, 2, VEC>(a, backward, stream);
  if (a.D <= 1024) return run<T, TR, 128, 1, VEC>(a, backward, stream);
  if (a.D <= 2048) return run<T, TR, 128, 2, VEC>(a, backward, stream);
  if (a.D <= 4096) return run<T, TR, 256, 2, VEC>(a, backward, stream);
  if (a.D <= 8192) return run<T, TR, 512, 2, VEC>(a, backward, stream);
  if (a.D <= BLOCK_NORM_MAX_D) return run<T, TR, 1024, 2, VEC>(a, backward, stream);
  return cudaErrorInvalidValue;
}
template <typename T, typename TR>
cudaError_t by_alignment(const BlockNormArgs& a, bool backward, cudaStream_t stream) {
  return a.D % 8 == 0 ? by_width<T, TR, true>(a, backward, stream) : by_width<T, TR, false>(a, backward, stream);
}

}  // namespace

cudaError_t launch_block_norm(const BlockNormArgs& a, bool backward, int dt, int res_dt, cudaStream_t stream) {
  if (dt == DT_F32 && res_dt == DT_F32) return by_alignment<float, float>(a, backward, stream);
  if (dt == DT_BF16 && res_dt == DT_F32) return by_alignment<__nv_bfloat16, float>(a, backward, stream);
  if (dt == DT_BF16 && res_dt == DT_BF16) return by_alignment<__nv_bfloat16, __nv_bfloat16>(a, backward, stream);
  return cudaErrorInvalidValue;
}

}  // namespace la
