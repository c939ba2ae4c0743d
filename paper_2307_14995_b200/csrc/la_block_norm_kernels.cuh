// What stands between two blocks of a model, one pass over each token's row of D features:
//   z = y r_y (.) w_post (.) act(u),   h = x + s (.) z,   n = h r_h (.) w_pre,   r_a = 1 / sqrt(mean(a^2) + eps)   (0 for a zero row
// without eps), and the gradients of <h, dh> + <n, dn>, from x, y and u again:
//   H = dh + r_h (w_pre dn - n^ mean(w_pre dn n^)),  n^ = h r_h;     dx = H,   ds = sum H z,   dw_pre = sum dn n^,
//   du = s H y^ w_post act'(u),  y^ = y r_y;     p = s H act(u) w_post,   dw_post = sum s H act(u) y^,   dy = r_y (p - y^ mean(p y^)).
//
// HBM bounds both: every input is read once and every output written once.  LANES threads share a row (a warp up to 512 features,
// else a part of a thread block or all of it), each with NV groups of eight features.  Two forms: the kernels right below, a row's loads
// when its turn comes, and a ring of rows on their way (further down, "many rows").  The sums over tokens (ds, dw) stay on chip over the rows
// that a thread block takes, leave it as one part [3][D] in the workspace, and a second kernel adds the parts up in order: no
// atomics, the same bits every time.
//
// Forward, the ring takes rows from 4 MB of residual stream on, us without / with it (bf16, gate): 4096 features 148 rows 4.5 / 5.3, 296
// 5.7 / 5.4, 2400 30.5 / 22.6; 1024 features 296 rows 3.0 / 4.7, 2400 8.8 / 9.2, 4800 16.1 / 14.3.  Rows that are not aligned it takes in any
// number, since the other form loads them value by value: 1003 features one row 4.6 / 4.9, 296 4.9 / 5.8, 301 features 3001 rows 12.3 / 8.7, 5001
// features one row 7.9 / 6.1, 296 15.8 / 12.3.  Backward always, where it fits into
// shared memory (up to 8192 features; fp32 with a gate up to 5608, 5601 where that is no multiple of eight): 4096 features one row 16 / 10, 296 rows 39 / 15, 4800 rows 343 / 83.
#pragma once
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

// Sum over the LANES threads of a row, the same in each.  One barrier is enough where a thread block's calls alternate between the two
// slots: one is written again behind the other's barrier, where all have read it.  Where they do not, a barrier has to stand between two
// calls with the same slot.  (A slot that every call turns over: 4096 x 16384 in fp32 forward 311 us, with the two named 300.)
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
  const bool alternate = a.post_norm && a.n;  // (else a row has one sum)
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
    if (!alternate) __syncthreads();
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

// For rows that the ring does not take.  A row's values and the sums over tokens do not fit in the registers together: the sums are in
// shared memory [3][D], and what a row has is read again (from L2) where it is used.  4096 x 16384 in bf16: 860 us, all in registers 1775.
template <typename T, typename TR, int LANES, int NV, bool VEC>
__global__ void __launch_bounds__(LANES) block_norm_bwd_kernel(const BlockNormArgs a) {
  extern __shared__ float sums[];
  __shared__ RowSum<LANES, 1> sum;
  grid_dep_wait();
  grid_dep_launch();
  const Cols<LANES, VEC> cols{(int)threadIdx.x, a.D};
  const float inv_d = 1.f / (float)a.D;
  float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int k = 0; k < 3; ++k) cols.store(sums + k * a.D, v, zero);  // (everyone's own)
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const long long at = row * a.D;
    float y[NV][8], h[NV][8], u[8], dn[8];
    auto get_y = [&](int v) { cols.load(static_cast<const T*>(a.y) + at, v, y[v]); };
    auto get_u = [&](int v) { cols.load(a.u ? static_cast<const T*>(a.u) + at : nullptr, v, u); };
    auto get_dn = [&](int v) { cols.load(a.dn ? static_cast<const T*>(a.dn) + at : nullptr, v, dn); };
    float ry = 1.f;
    if (a.post_norm) {
      float ss = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        get_y(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(y[v][i], y[v][i], ss);
      }
      ry = inverse_rms(sum(ss, 0, 0), inv_d, a.eps);
    }
    float ss = 0.f, dot = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float w[8], s[8], wp[8];
      get_y(v);
      cols.load(static_cast<const TR*>(a.x) + at, v, h[v]);
      get_u(v);
      get_dn(v);
      cols.load(a.w_post, v, w, 1.f);
      cols.load(a.s, v, s, 1.f);
      cols.load(a.w_pre, v, wp, 1.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float z = y[v][i] * ry * w[i], slope;
        if (a.u) z *= act(a.gate, u[i], slope);
        h[v][i] = fmaf(s[i], z, h[v][i]);
        ss = fmaf(h[v][i], h[v][i], ss);
        dot = fmaf(dn[i] * wp[i], h[v][i], dot);
      }
    }
    float rh = 0.f, along = 0.f;
    if (a.dn) {
      rh = inverse_rms(sum(ss, 1, 0), inv_d, a.eps);
      along = sum(dot, 0, 0) * rh * inv_d;  // mean(w_pre dn n^)
    }
    float py = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float w[8], s[8], wp[8], dh[8], du[8], to_post[8], to_s[8], to_pre[8];
      get_y(v);
      get_u(v);
      get_dn(v);
      cols.load(sums, v, to_post);
      cols.load(sums + a.D, v, to_s);
      cols.load(sums + 2 * a.D, v, to_pre);
      cols.load(a.w_post, v, w, 1.f);
      cols.load(a.s, v, s, 1.f);
      cols.load(a.w_pre, v, wp, 1.f);
      cols.load(a.dh ? static_cast<const TR*>(a.dh) + at : nullptr, v, dh);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float nh = h[v][i] * rh, yh = y[v][i] * ry;
        float H = dh[i];
        if (a.dn) {
          H = fmaf(rh, dn[i] * wp[i] - nh * along, H);
          to_pre[i] = fmaf(dn[i], nh, to_pre[i]);
        }
        dh[i] = H;
        float gate = 1.f, slope = 0.f;
        if (a.u) gate = act(a.gate, u[i], slope);
        to_s[i] = fmaf(H, yh * w[i] * gate, to_s[i]);
        to_post[i] = fmaf(H * s[i], yh * gate, to_post[i]);
        du[i] = H * s[i] * yh * w[i] * slope;
        h[v][i] = H * s[i] * gate * w[i];  // p
        py = fmaf(h[v][i], yh, py);
      }
      cols.store(sums, v, to_post);
      cols.store(sums + a.D, v, to_s);
      cols.store(sums + 2 * a.D, v, to_pre);
      cols.store(static_cast<TR*>(a.dx) + at, v, dh);
      if (a.u) cols.store(static_cast<T*>(a.du) + at, v, du);
    }
    if (a.post_norm) py = sum(py, 1, 0) * inv_d;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (a.post_norm) {
        get_y(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[v][i] = ry * (h[v][i] - y[v][i] * ry * py);
      }
      cols.store(static_cast<T*>(a.dy) + at, v, h[v]);
    }
    __syncthreads();  // (a row's sums are slots 0 1 0 1, some of them left out)
  }
  // the thread block's part
  float* const part = a.parts + (size_t)blockIdx.x * 3 * a.D;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      cols.load(sums + k * a.D, v, zero);
      cols.store(part + k * a.D, v, zero);
    }
}

// ---- many rows -----------------------------------------------------------------------------------------------------------------------------
// The same with the rows of a thread block's next turns on their way while it works on one: every thread copies what it will read
// itself into a ring of S stages in shared memory (cp.async), so that nobody waits for anybody but in the row sums.  One thread block
// of 512 threads to an SM, 512 / LANES rows at a time, each row's threads with a barrier of their own; sums over tokens in registers to
// the end.  Forward and backward, us (at the copy bandwidth): 65536 x 4096 in bf16 447 and 914 (409 and 654), without the ring 739 and 4146;
// 16384 x 4096 in fp32 209 and 338 (204 and 327); 16384 x 2048 in bf16 with the residual stream in fp32 86 and 134 (72 and 112).  What
// is left backward is the meeting of a row's threads, with one row of 4096 features at a time; instructions are issued in 61 % of the clocks.
//
// Rows whose width is no multiple of eight begin anywhere in 16 bytes.  They move from the 16-byte boundary before them, and what a unit
// has of the rows beside is left out; all rows of a thread block begin at the same place (the grid is a multiple of eight, and a block
// takes rows that are a grid apart), so that a thread's features are the same in all.  us, and with pairs of features (4 bytes of bf16) that
// need an even beginning alone: 16384 x 1003 in fp32 71 and 118 (91 and 159), in bf16 63 and 113 (73 and 123); 16384 x 5001 in bf16 344 and 818 (490
// and 1367).  A row's first and last units, whose values go one by one, are what aligned rows do not have (16384 x 1000 in bf16: 44 and 79).
constexpr int RING = 512;
template <int BYTES>
__device__ __forceinline__ void copy(uint32_t to, const void* from) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
template <int BYTES>
__device__ __forceinline__ void copy_part(uint32_t to, const void* from, int bytes) {  // the rest are zeros
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
constexpr int STAGES = 5;  // at most
__device__ __forceinline__ void copies_wait(int n) {  // all but the last n stages
  switch (n) {
    case 0: copies_wait<0>(); break;
    case 1: copies_wait<1>(); break;
    case 2: copies_wait<2>(); break;
    case 3: copies_wait<3>(); break;
    default: copies_wait<4>();
  }
}

// One tensor's place in a stage, and this thread's features of a row: unit u has features (u LANES + lane) F - shift .. + F - 1.  F is
// eight where all tensors are bf16 and four where one is fp32, 16 bytes of the wider type: neighbours' pieces touch, so that every
// sector is asked for once.  Four too for gradients of unaligned rows in bf16, whose ends are shorter then (with eight 117 and 900 for the 112
// and 809 above; forward, 16384 x 2999, eight take 175 and four 194).  (With eight of fp32, two pieces of a thread side by side, 16384 x 4096 took 361 and 627.)
template <int LANES, int NV, int FEATURES, bool ALIGNED>
struct RingRow {
  static constexpr int F = FEATURES, U = 8 * NV / F;
  template <bool BWD>
  static constexpr bool kept() { return NV == 1 && (!BWD || F == 8); }  // the weights' place
  int lane, D, shift;
  long long total;  // features of the tensor
  __device__ __forceinline__ int feature(int u) const { return (u * LANES + lane) * F - shift; }
  __device__ __forceinline__ bool whole(int f) const { return ALIGNED ? f < D : f >= 0 && f + F <= D; }
  template <typename T>
  static constexpr int bytes() { return RING * 8 * NV * (int)sizeof(T); }
  // stage memory: unit u of thread t at piece u RING + t
  template <typename T>
  __device__ __forceinline__ void fetch(uint32_t to, const T* base, long long row) const {
    constexpr int PIECE = F * (int)sizeof(T);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int f = feature(u);
      const uint32_t dst = to + (uint32_t)(u * RING + threadIdx.x) * PIECE;
      const T* const at = base + row * D + f;
      if (f < D) {
        const long long left = total - (row * D + f);  // (only the tensor's last piece is cut short)
        if (ALIGNED || left >= F) copy<PIECE>(dst, at);
        else copy_part<PIECE>(dst, at, (int)left * (int)sizeof(T));
      }
    }
  }
  template <typename T>
  __device__ __forceinline__ void get(const unsigned char* from, int u, float (&x)[F]) const {
    const unsigned char* const src = from + (u * RING + threadIdx.x) * F * (int)sizeof(T);
    if constexpr (sizeof(T) == 4) {
      const float4 v = *reinterpret_cast<const float4*>(src);
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
      uint32_t w[F / 2];
      if constexpr (F == 4) *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(src);
      else *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(src);
#pragma unroll
      for (int i = 0; i < F / 2; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    if (!ALIGNED) {
      const int f = feature(u);
      if (!whole(f)) {
#pragma unroll
        for (int i = 0; i < F; ++i) x[i] = f + i >= 0 && f + i < D ? x[i] : 0.f;
      }
    }
  }
  template <typename T>
  __device__ __forceinline__ void put(T* base, long long row, int u, const float (&x)[F]) const {
    T* const at = base + row * D;
    const int f = feature(u);
    if (whole(f)) {
      if constexpr (F == 4) Vec4<T>::store(at + f, x);
      else store8(at + f, x);
    } else if (!ALIGNED) {
#pragma unroll
      for (int i = 0; i < F; ++i)
        if (f + i >= 0 && f + i < D) at[f + i] = from_f32<T>(x[i]);
    }
  }
  // Weights in shared memory begin where the units do, `length` of them; units of eight: the first four of every eight, then the
  // others, so that neighbours read without conflicts (weight_at: where position p is).
  static __host__ __device__ __forceinline__ int length(int D) { return (D + (ALIGNED ? 7 : 14)) / 8 * 8; }
  static __device__ __forceinline__ int weight_at(int p, int D) { return F == 8 ? (p & 4 ? length(D) / 2 : 0) + (p >> 3) * 4 + (p & 3) : p; }
  __device__ __forceinline__ void weights(const float* w, int u, float (&x)[F]) const {
    const int p = feature(u) < D ? (u * LANES + lane) * F : 0;
    const float4 a = *reinterpret_cast<const float4*>(w + (F == 8 ? p / 2 : p));
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    if constexpr (F == 8) {
      const float4 b = *reinterpret_cast<const float4*>(w + length(D) / 2 + p / 2);
      x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
  }
};

// Sums of values over a row's threads: over each warp's lanes, then every warp adds up the warps' sums the same way.
template <int LANES>
struct RowSums {
  static constexpr int W = LANES / 32;
  float part[2][8][20];  // slot, value, warp; the pitch keeps the lanes of several() apart
  __device__ __forceinline__ void meet() const { asm volatile("bar.sync %0, %1;" ::"r"(1 + (int)threadIdx.x / LANES), "n"(LANES) : "memory"); }
  __device__ __forceinline__ float one(float x, int& slot) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (W <= 1) return x;
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, first = warp / W * W;
    if (lane == 0) part[slot][0][warp] = x;
    meet();
    x = part[slot][0][first + lane % W];
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    slot ^= 1;  // (written again behind the next sum's barrier)
    return x;
  }
  // eight at once, by halves: four lanes end up with one value's sum
  __device__ __forceinline__ void several(float (&x)[8], int& slot) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, first = warp / W * W;
#pragma unroll
    for (int o = 16, n = 4; o >= 4; o >>= 1, n >>= 1)
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float keep = lane & o ? x[n + i] : x[i], give = lane & o ? x[i] : x[n + i];
        x[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
      }
    float v = x[0];
    v += __shfl_xor_sync(0xffffffffu, v, 2);
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    if (W > 1) {
      if ((lane & 3) == 0) part[slot][lane >> 2][warp] = v;
      meet();
      v = 0.f;
#pragma unroll
      for (int w = 0; w < W; w += 4)
        if (w + (lane & 3) < W) v += part[slot][lane >> 2][first + w + (lane & 3)];
      v += __shfl_xor_sync(0xffffffffu, v, 2);
      v += __shfl_xor_sync(0xffffffffu, v, 1);
      slot ^= 1;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __shfl_sync(0xffffffffu, v, 4 * i);
  }
};

template <int F>
__device__ __forceinline__ uint64_t pair(const float (&x)[F], int i) { return f2_pack(x[i], x[i + 1]); }
template <int F>
__device__ __forceinline__ void unpair(uint64_t v, float (&x)[F], int i) { f2_unpack(v, x[i], x[i + 1]); }
__device__ __forceinline__ float pair_sum(uint64_t v) {
  float a, b;
  f2_unpack(v, a, b);
  return a + b;
}

// 1 / (1 + exp(-u)) of two values.  The exponential and the reciprocal are good to an ulp or two (5.4e-7 of the result with the roundings
// around them), but the exponent -u log2(e) is a rounded product, whose error is multiplied by |u|: |u| 7.3e-8 of a small result more, 2^-20
// at u = -20, 2^-18 at u = -80.  Where u is bf16, given to 2^-9 of itself, that stays.  EXACT, where u is fp32: the exponent is t + r, the product
// rounded down and the rest, r = (what the product lost) - u (log2(e)'s own rest), and 2^(t + r) = 2^t + 2^t r ln 2 (|r| < 2^-15).  Beyond |u| = 104
// the result is 0 or 1, and r stays finite; the product is rounded down so that r >= 0 where 2^t is infinite and the sum stays so.
// 65536 x 4096 in bf16, forward and backward: 1461 us, EXACT 1511.
template <bool EXACT>
__device__ __forceinline__ uint64_t sigmoid2(uint64_t u) {
  constexpr float LOG2E = 1.44269502f, REST = 1.92596299e-8f, LN2 = 0.693147181f;
  float a, b;
  uint64_t t, r = 0;
  if (EXACT) {
    f2_unpack(u, a, b);
    asm("min.NaN.xorsign.abs.f32 %0, %0, %1;" : "+f"(a) : "f"(104.f));  // the sign of u
    asm("min.NaN.xorsign.abs.f32 %0, %0, %1;" : "+f"(b) : "f"(104.f));
    u = f2_pack(a, b);
    t = f2_mul_down(u, f2_pack(-LOG2E, -LOG2E));
    const uint64_t lost = f2_fma(u, f2_pack(LOG2E, LOG2E), t);                                   // (its negative)
    r = f2_fma(u, f2_pack(-REST * LN2, -REST * LN2), f2_mul(lost, f2_pack(-LN2, -LN2)));  // times ln 2
  } else {
    t = f2_mul(u, f2_pack(-LOG2E, -LOG2E));
  }
  f2_unpack(t, a, b);
  asm("ex2.approx.f32 %0, %0;" : "+f"(a));
  asm("ex2.approx.f32 %0, %0;" : "+f"(b));
  uint64_t e = f2_pack(a, b);
  if (EXACT) e = f2_fma(e, r, e);
  f2_unpack(f2_add(e, f2_pack(1.f, 1.f)), a, b);
  asm("rcp.approx.f32 %0, %0;" : "+f"(a));
  asm("rcp.approx.f32 %0, %0;" : "+f"(b));
  return f2_pack(a, b);
}
// g becomes act(g), slope act'(g); one branch for all of a unit's features
template <bool SLOPE, bool EXACT, int F>
__device__ __forceinline__ void gate_values(int kind, float (&g)[F], float (&slope)[F]) {
  const uint64_t one = f2_pack(1.f, 1.f), minus = f2_pack(-1.f, -1.f);
  if (kind == GATE_SILU) {
#pragma unroll
    for (int i = 0; i < F; i += 2) {
      const uint64_t s = sigmoid2<EXACT>(pair(g, i)), v = f2_mul(pair(g, i), s);
      unpair(v, g, i);
      if (SLOPE) unpair(f2_fma(v, f2_fma(s, minus, one), s), slope, i);
    }
  } else if (kind == GATE_SIGMOID) {
#pragma unroll
    for (int i = 0; i < F; i += 2) {
      const uint64_t s = sigmoid2<EXACT>(pair(g, i));
      unpair(s, g, i);
      if (SLOPE) unpair(f2_mul(s, f2_fma(s, minus, one)), slope, i);
    }
  } else if (SLOPE) {
#pragma unroll
    for (int i = 0; i < F; ++i) slope[i] = 1.f;
  }
}

template <typename T, typename TR, int LANES, int NV, bool VEC, bool BWD>
__global__ void __launch_bounds__(RING, 1) block_norm_ring_kernel(const BlockNormArgs a, const int S) {
  using Row = RingRow<LANES, NV, sizeof(TR) == 4 || (BWD && !VEC) ? 4 : 8, VEC>;  // (see RingRow)
  constexpr int F = Row::F, U = Row::U, ROWS = RING / LANES;
  constexpr int BT = Row::template bytes<T>(), BR = Row::template bytes<TR>();
  extern __shared__ __align__(16) unsigned char ring[];
  __shared__ RowSums<LANES> sums;
  grid_dep_wait();
  grid_dep_launch();
  // the stages: y, x, u and backward dn, dh; behind them the weights
  const int stage_bytes = BT + BR + (a.u ? BT : 0) + (BWD ? BT + BR : 0);
  const int at_x = BT, at_u = BT + BR, at_dn = at_u + (a.u ? BT : 0), at_dh = at_dn + BT;
  float* const w_post = reinterpret_cast<float*>(ring + S * stage_bytes);
  const int wd = Row::length(a.D);
  float *const w_s = w_post + wd, *const w_pre = w_s + wd;
  for (int i = threadIdx.x; i < S * stage_bytes / 16; i += RING) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0u, 0u, 0u, 0u);  // units past the end stay zeros
  __syncthreads();
  const int sub = threadIdx.x / LANES;
  const long long first = VEC ? (long long)blockIdx.x * ROWS + sub : (long long)gridDim.x * sub + blockIdx.x, step = (long long)gridDim.x * ROWS;
  const Row my{(int)threadIdx.x % LANES, a.D, VEC ? 0 : (int)(blockIdx.x * (unsigned)a.D % F), a.rows * a.D};
  const float inv_d = 1.f / (float)a.D;
  const uint32_t ring_at = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  auto fetch = [&](long long row, int s) {
    if (row < a.rows) {
      const uint32_t to = ring_at + s * stage_bytes;
      my.fetch(to, static_cast<const T*>(a.y), row);
      my.fetch(to + at_x, static_cast<const TR*>(a.x), row);
      if (a.u) my.fetch(to + at_u, static_cast<const T*>(a.u), row);
      if (BWD && a.dn) my.fetch(to + at_dn, static_cast<const T*>(a.dn), row);
      if (BWD && a.dh) my.fetch(to + at_dh, static_cast<const TR*>(a.dh), row);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // With eight features to a thread what is read stays in registers, with sixteen it is read again where it is used.  The weights stay
  // there too where they leave enough: forward, and backward where units are of eight.
  constexpr bool KEEP = NV == 1, KEPT = Row::template kept<BWD>();
  float g_post[BWD ? U : 1][F], g_s[BWD ? U : 1][F], g_pre[BWD ? U : 1][F];
#pragma unroll
  for (int u = 0; u < (BWD ? U : 1); ++u)
#pragma unroll
    for (int i = 0; i < F; ++i) g_post[u][i] = g_s[u][i] = g_pre[u][i] = 0.f;
  for (int s = 0; s < S; ++s) fetch(first + s * step, s);
  float k_post[KEPT ? U : 1][F], k_s[KEPT ? U : 1][F], k_pre[KEPT ? U : 1][F];
  if constexpr (KEPT) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < F; ++i) {
        const int f = my.feature(u) + i;
        const bool in = f >= 0 && f < a.D;
        k_post[u][i] = in && a.w_post ? a.w_post[f] : 1.f;
        k_s[u][i] = in && a.s ? a.s[f] : 1.f;
        k_pre[u][i] = in && a.w_pre ? a.w_pre[f] : 1.f;
      }
  } else {
    for (int p = threadIdx.x; p < wd; p += RING) {
      const int at = Row::weight_at(p, a.D), i = p - my.shift;
      const bool in = i >= 0 && i < a.D;
      w_post[at] = in && a.w_post ? a.w_post[i] : 1.f;
      w_s[at] = in && a.s ? a.s[i] : 1.f;
      w_pre[at] = in && a.w_pre ? a.w_pre[i] : 1.f;
    }
    __syncthreads();
  }
  auto weights = [&](const float(&kept)[KEPT ? U : 1][F], const float* at, int u, float (&x)[F]) {
    if constexpr (KEPT) {
#pragma unroll
      for (int i = 0; i < F; ++i) x[i] = kept[u][i];
    } else {
      my.weights(at, u, x);
    }
  };
  int s = 0, slot = 0;
  float y[U][F], g[U][F], slope[U][F], h[U][F];
  auto get_y = [&](const unsigned char* in, int u) { my.template get<T>(in, u, y[u]); };
  auto get_gate = [&](const unsigned char* in, int u) {
    if (a.u) {
      my.template get<T>(in + at_u, u, g[u]);
      gate_values<BWD, sizeof(T) == 4>(a.gate, g[u], slope[u]);
    } else {
#pragma unroll
      for (int i = 0; i < F; ++i) g[u][i] = 1.f, slope[u][i] = 0.f;
    }
  };
  auto square_of_y = [&](const unsigned char* in) {
    uint64_t sum = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[F];
      my.template get<T>(in, u, v);
#pragma unroll
      for (int i = 0; i < F; i += 2) sum = f2_fma(pair(v, i), pair(v, i), sum);
    }
    return pair_sum(sum);
  };
  float ry = 1.f;
  const bool ahead = S > 2;  // two rows may be waited for
  for (long long row = first; row < a.rows; row += step) {
    const unsigned char* const in = ring + s * stage_bytes;
    const int after = s + 1 == S ? 0 : s + 1;
    if constexpr (!BWD) {
      copies_wait(S - 1);
      if (a.post_norm) ry = inverse_rms(sums.one(square_of_y(in), slot), inv_d, a.eps);
      uint64_t sum_h = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[F], w[F], sc[F];
        get_y(in, u);
        my.template get<TR>(in + at_x, u, x);
        get_gate(in, u);
        weights(k_post, w_post, u, w);
        weights(k_s, w_s, u, sc);
        const uint64_t ry2 = f2_pack(ry, ry);
#pragma unroll
        for (int i = 0; i < F; i += 2) {
          const uint64_t z = f2_mul(f2_mul(f2_mul(pair(y[u], i), ry2), pair(w, i)), pair(g[u], i));
          const uint64_t v = f2_fma(pair(sc, i), z, pair(x, i));
          unpair(v, h[u], i);
          sum_h = f2_fma(v, v, sum_h);
        }
        if (a.h) my.put(static_cast<TR*>(a.h), row, u, h[u]);
      }
      fetch(row + S * step, s);
      if (a.n) {
        const float rh = inverse_rms(sums.one(pair_sum(sum_h), slot), inv_d, a.eps);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float w[F];
          weights(k_pre, w_pre, u, w);
#pragma unroll
          for (int i = 0; i < F; ++i) w[i] *= h[u][i] * rh;
          my.put(static_cast<T*>(a.n), row, u, w);
        }
      }
    } else {
      // One meeting of a row's threads: c = s z (so h = x + c), and sum p y^ = sum H c is taken apart,
      //   sum H c = sum dh c + r_h (sum w_pre dn c - mean(w_pre dn n^) r_h sum h c),
      // whose terms are no larger than those of H itself; the square of the next row's y is summed up with them.  (With a
      // meeting for each sum that depends on another, three a row: 1005 us for 65536 x 4096 in bf16.)
      if (a.post_norm && (row == first || !ahead)) {
        copies_wait(S - 1);
        ry = inverse_rms(sums.one(square_of_y(in), slot), inv_d, a.eps);
      }
      copies_wait(ahead ? S - 2 : S - 1);
      uint64_t sum[5] = {0, 0, 0, 0, 0};  // h h, w_pre dn h, dh c, w_pre dn c, h c: two at a time
      const uint64_t ry2 = f2_pack(ry, ry);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[F], w[F], sc[F], wp[F], dn[F], dh[F];
        get_y(in, u);
        my.template get<TR>(in + at_x, u, x);
        get_gate(in, u);
        my.template get<T>(in + at_dn, u, dn);
        my.template get<TR>(in + at_dh, u, dh);
        weights(k_post, w_post, u, w);
        weights(k_s, w_s, u, sc);
        weights(k_pre, w_pre, u, wp);
#pragma unroll
        for (int i = 0; i < F; i += 2) {
          const uint64_t c = f2_mul(pair(sc, i), f2_mul(f2_mul(f2_mul(pair(y[u], i), ry2), pair(w, i)), pair(g[u], i)));
          const uint64_t v = f2_add(c, pair(x, i)), n = f2_mul(pair(dn, i), pair(wp, i));
          unpair(v, h[u], i);
          sum[0] = f2_fma(v, v, sum[0]);
          sum[1] = f2_fma(n, v, sum[1]);
          sum[2] = f2_fma(pair(dh, i), c, sum[2]);
          sum[3] = f2_fma(n, c, sum[3]);
          sum[4] = f2_fma(v, c, sum[4]);
        }
      }
      float all[8];
#pragma unroll
      for (int i = 0; i < 5; ++i) all[i] = pair_sum(sum[i]);
      all[5] = a.post_norm && ahead ? square_of_y(ring + after * stage_bytes) : 0.f;  // (behind the last row: whatever, not used)
      all[6] = all[7] = 0.f;
      sums.several(all, slot);
      float rh = 0.f, along = 0.f;
      if (a.dn) {
        rh = inverse_rms(all[0], inv_d, a.eps);
        along = all[1] * rh * inv_d;  // mean(w_pre dn n^)
      }
      const float py = fmaf(rh, all[3] - along * rh * all[4], all[2]), along_y = a.post_norm ? py * inv_d * ry : 0.f;
      const uint64_t rh2 = f2_pack(rh, rh), along2 = f2_pack(-along, -along), along_y2 = f2_pack(-along_y, -along_y);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float w[F], sc[F], dn[F], dh[F], dy[F];
        if (!KEEP) {
          get_y(in, u);
          get_gate(in, u);
        }
        my.template get<T>(in + at_dn, u, dn);
        my.template get<TR>(in + at_dh, u, dh);
        weights(k_pre, w_pre, u, w);
#pragma unroll
        for (int i = 0; i < F; i += 2) {
          const uint64_t nh = f2_mul(pair(h[u], i), rh2), n = pair(dn, i);
          unpair(f2_fma(rh2, f2_fma(nh, along2, f2_mul(n, pair(w, i))), pair(dh, i)), dh, i);  // H
          unpair(f2_fma(n, nh, pair(g_pre[u], i)), g_pre[u], i);
        }
        my.put(static_cast<TR*>(a.dx), row, u, dh);
        weights(k_post, w_post, u, w);
        weights(k_s, w_s, u, sc);
#pragma unroll
        for (int i = 0; i < F; i += 2) {
          const uint64_t yh = f2_mul(pair(y[u], i), ry2), H = pair(dh, i), Hg = f2_mul(H, pair(g[u], i)), ws = pair(w, i), yw = f2_mul(yh, ws);
          const uint64_t Hsg = f2_mul(Hg, pair(sc, i)), p = f2_mul(Hsg, ws);
          unpair(f2_fma(Hg, yw, pair(g_s[u], i)), g_s[u], i);
          unpair(f2_fma(Hsg, yh, pair(g_post[u], i)), g_post[u], i);
          if (a.u) unpair(f2_mul(f2_mul(f2_mul(H, pair(sc, i)), yw), pair(slope[u], i)), slope[u], i);  // du
          unpair(f2_mul(ry2, f2_fma(pair(y[u], i), along_y2, p)), dy, i);
        }
        if (a.u) my.put(static_cast<T*>(a.du), row, u, slope[u]);
        my.put(static_cast<T*>(a.dy), row, u, dy);
      }
      fetch(row + S * step, s);
      ry = a.post_norm ? inverse_rms(all[5], inv_d, a.eps) : 1.f;
    }
    s = after;
  }
  if (!BWD) return;
  // the thread block's part: its rows' threads add up in order
  copies_wait<0>();
  __syncthreads();
  float* const mine = reinterpret_cast<float*>(ring) + (size_t)sub * 3 * a.D;
  float* const part = a.parts + (size_t)blockIdx.x * 3 * a.D;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < F; ++i) {
      const int f = my.feature(u) + i;
      if (f < 0 || f >= a.D) continue;
      mine[f] = g_post[BWD ? u : 0][i];
      mine[a.D + f] = g_s[BWD ? u : 0][i];
      mine[2 * a.D + f] = g_pre[BWD ? u : 0][i];
    }
  __syncthreads();
  for (int c = threadIdx.x; c < 3 * a.D; c += RING) {
    float x = reinterpret_cast<const float*>(ring)[c];
    for (int r = 1; r < ROWS; ++r) x += reinterpret_cast<const float*>(ring)[(size_t)r * 3 * a.D + c];
    part[c] = x;
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

cudaError_t sum_parts(const BlockNormArgs& a, int n, cudaStream_t stream);

template <typename T, typename TR, int LANES, int NV, bool VEC>
cudaError_t run_fwd(const BlockNormArgs& a, cudaStream_t stream) {
  constexpr int BLOCK = LANES > THREADS ? LANES : THREADS, ROWS = BLOCK / LANES;
  const long long groups = (a.rows + ROWS - 1) / ROWS, cap = 148LL * 64;  // a few waves, then each thread block takes further rows
  KernelTimer timer(K_GATE, stream);
  const cudaError_t err = launch_early(block_norm_fwd_kernel<T, TR, LANES, NV, VEC>, dim3((unsigned)(groups < cap ? groups : cap)), dim3(BLOCK), 0, stream, 1, a);
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}
template <typename T, typename TR, int LANES, int NV, bool VEC>
cudaError_t run_bwd(const BlockNormArgs& a, cudaStream_t stream) {
  const int smem = 3 * a.D * 4, grid = (int)(a.rows < a.nparts ? a.rows : a.nparts);
  cudaError_t err = cudaFuncSetAttribute(block_norm_bwd_kernel<T, TR, LANES, NV, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (err != cudaSuccess) return err;
  {
    KernelTimer timer(K_GATE, stream);
    err = launch_early(block_norm_bwd_kernel<T, TR, LANES, NV, VEC>, dim3((unsigned)grid), dim3(LANES), smem, stream, 1, a);
    count_launch();
    if (err == cudaSuccess) err = cudaGetLastError();
  }
  return err != cudaSuccess ? err : sum_parts(a, grid, stream);
}

cudaError_t sum_parts(const BlockNormArgs& a, int n, cudaStream_t stream) {
  KernelTimer timer(K_GATE, stream);
  const cudaError_t err = launch_early(block_norm_sum_kernel, dim3((unsigned)((3 * a.D + 31) / 32)), dim3(THREADS), 0, stream, 1,
                                       (const float*)a.parts, n, a.D, a.dw_post, a.ds, a.dw_pre);
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}

template <typename T, typename TR, int LANES, int NV, bool VEC, bool BWD>
cudaError_t run_ring(const BlockNormArgs& a, cudaStream_t stream) {
  using Row = RingRow<LANES, NV, sizeof(TR) == 4 || (BWD && !VEC) ? 4 : 8, VEC>;
  constexpr int ROWS = RING / LANES, BT = Row::template bytes<T>(), BR = Row::template bytes<TR>();
  const int stage = BT + BR + (a.u ? BT : 0) + (BWD ? BT + BR : 0), weights = Row::template kept<BWD>() ? 0 : 3 * Row::length(a.D) * 4;
  constexpr int most = 227 * 1024 - (int)sizeof(RowSums<LANES>);
  int stages = STAGES;
  while (stages > 1 && stages * stage + weights > most) --stages;
  int smem = stages * stage + weights;
  if (BWD && smem < ROWS * 3 * a.D * 4) smem = ROWS * 3 * a.D * 4;
  if (smem > most) return cudaErrorNotSupported;
  auto kern = block_norm_ring_kernel<T, TR, LANES, NV, VEC, BWD>;
  cudaError_t err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (err != cudaSuccess) return err;
  long long grid = (a.rows + ROWS - 1) / ROWS;
  if (!VEC) grid = grid < 144 ? (grid + 7) / 8 * 8 : 144;  // a multiple of eight: see above
  else if (grid > 148) grid = 148;
  if (BWD && grid > a.nparts) return cudaErrorInvalidValue;
  {
    KernelTimer timer(K_GATE, stream);
    err = launch_early(kern, dim3((unsigned)grid), dim3(RING), smem, stream, 1, a, stages);
    count_launch();
    if (err == cudaSuccess) err = cudaGetLastError();
  }
  return err != cudaSuccess || !BWD ? err : sum_parts(a, (int)grid, stream);
}

// Backward eight features to a thread as far as 512 threads go: with sixteen its sums over tokens leave too few registers.
template <typename T, typename TR, bool VEC, bool BWD>
cudaError_t ring_by_width(const BlockNormArgs& a, cudaStream_t stream) {
  const int d = a.D + (VEC ? 0 : 7);  // that many may have to fit
  if (d <= 256) return run_ring<T, TR, 32, 1, VEC, BWD>(a, stream);
  if (d <= 512) return run_ring<T, TR, BWD ? 64 : 32, BWD ? 1 : 2, VEC, BWD>(a, stream);
  if (d <= 1024) return run_ring<T, TR, 128, 1, VEC, BWD>(a, stream);
  if (d <= 2048) return run_ring<T, TR, BWD ? 256 : 128, BWD ? 1 : 2, VEC, BWD>(a, stream);
  if (d <= 4096) return run_ring<T, TR, BWD ? 512 : 256, BWD ? 1 : 2, VEC, BWD>(a, stream);
  if (d > 8192) return cudaErrorNotSupported;
  return run_ring<T, TR, 512, 2, VEC, BWD>(a, stream);
}

template <typename T, typename TR, bool VEC>
cudaError_t by_width(const BlockNormArgs& a, bool backward, cudaStream_t stream) {
  if (a.D > BLOCK_NORM_MAX_D) return cudaErrorInvalidValue;
  if (backward) {
    const cudaError_t err = a.D <= 8192 ? ring_by_width<T, TR, VEC, true>(a, stream) : cudaErrorNotSupported;
    if (err != cudaErrorNotSupported) return err;
    return a.D <= 8192 ? run_bwd<T, TR, 512, 2, VEC>(a, stream) : run_bwd<T, TR, 1024, 2, VEC>(a, stream);
  }
  if (a.D <= 8192 && (!VEC || a.rows * a.D * (long long)sizeof(TR) >= 4 << 20)) {
    const cudaError_t err = ring_by_width<T, TR, VEC, false>(a, stream);
    if (err != cudaErrorNotSupported) return err;
  }
  if constexpr (VEC) {
    if (a.D <= 256) return run_fwd<T, TR, 32, 1, VEC>(a, stream);
    if (a.D <= 512) return run_fwd<T, TR, 32, 2, VEC>(a, stream);
    if (a.D <= 1024) return run_fwd<T, TR, 128, 1, VEC>(a, stream);
    if (a.D <= 2048) return run_fwd<T, TR, 128, 2, VEC>(a, stream);
    if (a.D <= 4096) return run_fwd<T, TR, 256, 2, VEC>(a, stream);
  }
  if (a.D <= 8192) return run_fwd<T, TR, 512, 2, VEC>(a, stream);
  return run_fwd<T, TR, 1024, 2, VEC>(a, stream);
}
template <typename T, typename TR>
cudaError_t by_alignment(const BlockNormArgs& a, bool backward, cudaStream_t stream) {
  return a.D % 8 == 0 ? by_width<T, TR, true>(a, backward, stream) : by_width<T, TR, false>(a, backward, stream);
}

}  // namespace

}  // namespace la
