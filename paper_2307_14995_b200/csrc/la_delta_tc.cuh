// Tensor-core kernels of the gated delta rule (included by la_tc.cu, inside its anonymous namespace, after the helpers and the walk, whose
// arithmetic on pairs they share).  bf16 inputs, D = 128 or 64, chunks of 128 tokens.  Formulas: la_delta.cuh, in this order:
//
//   prepare   per chunk, from its own tokens: That by its transpose U = That^T (upper triangular, lanes are rows of U),
//             X = scale ((Q K^T) (.) D) diag(beta) That,   J^T = K^T diag(beta e^(G_end - G)) That  [d, tokens],
//             M = J^T diag(e^G) K,   N = J^T V.   Then the chunk as a whole is the affine map
//                 S' = e^G_end S - M S + N,     and its outputs are   O = scale diag(e^G) Q S + X (V - diag(e^G) K S),
//   chain     the map over all chunks, one after the other, a thread block per slice of value columns: one product a chunk,
//   output    O, per chunk.
//   Backward:   E = e^G_end E' - M^T E' + (scale Q^T diag(e^G) dO - K^T diag(e^G) Z),   Z = X^T dO: the same chain, in reverse,
//   adjoint   Z and that sum, per chunk,
//   values    Y = That (V - diag(e^G) K S) and dR = Z + U diag(beta e^(G_end - G)) K E', per chunk,
//   gradients the rest, per chunk.
//
// Why: what is sequential is one product of [D, D] and [D, columns] per 128 tokens, with the operand already in the layout that the tensor
// cores read (records below), and everything else has a thread block per chunk.  A walk that formed V' from What S, then S' from
// V', would be two dependent products with two conversions between them.
//
// As in the walk, operands formed on chip from fp32 values are two bf16 terms hi + lo, off by 2^-16 of a value at most and by 2.7e-6 of
// it on the root of the mean square: in a result that passes six of them 6e-6 (measured, relative 2-norm: outputs, states and gradients up
// to 8e-6 in a head, dg up to 4e-5 where the products of state and gradient that it sums up nearly cancel).  Products of two such operands leave
// out lo x lo, except where it comes with the columns of an operand [hi | lo].  Sums are fp32, in an order that depends on the shape
// alone: the products of lo terms first, so that fewer additions meet a large sum, whose rounding is towards zero.
//
// Operands in shared memory and in the workspace are images: rows of 128 bytes (64 elements) in the 128-byte swizzle, panel after panel of
// 64 columns, all panels of hi and then those of lo; one image serves K-major and MN-major.  They move by untiled bulk copies.  States are
// slices of 32 value columns, a panel each: [hi | lo] of the 32 columns, which is the operand of the chain's thread block that made them.
//
// Every kernel waits for its predecessor before it does anything (its tensor memory included), and every wait inside is bounded: X_WAIT
// makes the outcome the same for all threads of the block, which then drain what is in flight, free tensor memory and return.

// Workspace records of one chunk of one head, in bytes.
template <int D>
struct XRec {
  static constexpr size_t STATE = (size_t)D * D * 4;  // an image of a state or a state in fp32
  static constexpr size_t ALL = 0, END = 8;            // e^G_end, and its logarithm as two terms
  static constexpr size_t GATES = 256;                 // XGateTable
  static constexpr size_t U = GATES + 2560, X = U + 65536, M = X + 65536, N = M + STATE, S = N + STATE, FWD = S + STATE;
  static constexpr size_t TOK = (size_t)128 * D * 4;  // an image or fp32 values of all tokens
  static constexpr size_t Z = 0, DR = Z + TOK, Y = DR + TOK, B = Y + TOK, E = B + STATE, BWD = E + STATE;
};

struct XMaps {
  CUtensorMap q, k, v, d_o;    // boxes of 64 features x 128 tokens
  CUtensorMap o, dq, dk, dv;   // results: boxes of 128 bytes x 128 tokens; tokens behind the last one are not written
};

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src),
               "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void bulk_store(void* dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void prefetch(const void* src, uint32_t bytes) {  // to L2
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_store_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// The images of U (upper triangular) and X (lower) have 64 x 64 zeros: the half of a panel, of both terms, which neither moves nor is
// kept; whoever loads one clears it in shared memory.
constexpr uint32_t TRIANGLE = 49152;  // bytes that move
template <bool UPPER>
__device__ __forceinline__ void load_triangle(unsigned char* dst, const unsigned char* src, uint64_t* bar) {
#pragma unroll
  for (uint32_t term = 0; term < 65536; term += 32768) {
    bulk_load(dst + term + (UPPER ? 0 : 24576), src + term + (UPPER ? 0 : 24576), 8192, bar);
    bulk_load(dst + term + (UPPER ? 16384 : 0), src + term + (UPPER ? 16384 : 0), 16384, bar);
  }
}
template <bool UPPER>
__device__ __forceinline__ void store_triangle(unsigned char* dst, const unsigned char* src) {
#pragma unroll
  for (uint32_t term = 0; term < 65536; term += 32768) {
    bulk_store(dst + term + (UPPER ? 0 : 24576), src + term + (UPPER ? 0 : 24576), 8192);
    bulk_store(dst + term + (UPPER ? 16384 : 0), src + term + (UPPER ? 16384 : 0), 16384);
  }
}
template <bool UPPER>
__device__ __forceinline__ void prefetch_triangle(const unsigned char* src) {
#pragma unroll
  for (uint32_t term = 0; term < 65536; term += 32768) {
    prefetch(src + term + (UPPER ? 0 : 24576), 8192);
    prefetch(src + term + (UPPER ? 16384 : 0), 16384);
  }
}
template <bool UPPER>
__device__ __forceinline__ void clear_triangle(unsigned char* image, int tid, int threads) {
  for (int i = tid; i < 1024; i += threads)
    reinterpret_cast<uint4*>(image + (i >> 9) * 32768 + (UPPER ? 8192 : 16384))[i & 511] = make_uint4(0u, 0u, 0u, 0u);
}

// Byte offset of columns 8 c .. 8 c + 7 of row r in an image whose panels have `rows` rows.
__device__ __forceinline__ uint32_t image_at(int r, int c, int rows) { return (uint32_t)((c >> 3) * rows * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4)); }

// Eight values as packed hi and lo terms.
__device__ __forceinline__ void split8(const float* x, uint4& h, uint4& l) {
  split2(f2_pack(x[0], x[1]), h.x, l.x);
  split2(f2_pack(x[2], x[3]), h.y, l.y);
  split2(f2_pack(x[4], x[5]), h.z, l.z);
  split2(f2_pack(x[6], x[7]), h.w, l.w);
}
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ void join8(const uint4& h, const uint4& l, float* x) {
  x[0] = bf_lo(h.x) + bf_lo(l.x); x[1] = bf_hi(h.x) + bf_hi(l.x);
  x[2] = bf_lo(h.y) + bf_lo(l.y); x[3] = bf_hi(h.y) + bf_hi(l.y);
  x[4] = bf_lo(h.z) + bf_lo(l.z); x[5] = bf_hi(h.z) + bf_hi(l.z);
  x[6] = bf_lo(h.w) + bf_lo(l.w); x[7] = bf_hi(h.w) + bf_hi(l.w);
}
// 16 accumulator columns of this thread's lane (a wait has to follow), or 32
__device__ __forceinline__ void load_acc16(uint32_t taddr, float (&x)[16]) { tmem_ld_x16(taddr, *reinterpret_cast<uint32_t(*)[16]>(&x)); }
__device__ __forceinline__ void load_acc(uint32_t taddr, float (&x)[32]) {
  tmem_ld_x32(taddr, *reinterpret_cast<uint32_t(*)[32]>(&x));
  tmem_ld_wait();
}
// 32 values as an A operand: 16 columns of hi terms, 16 of lo terms
__device__ __forceinline__ void store_operand(uint32_t hi, uint32_t lo, const float (&x)[32]) {
  uint32_t h[16], l[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) split2(f2_pack(x[2 * i], x[2 * i + 1]), h[i], l[i]);
  tmem_st_x16(hi, h);
  tmem_st_x16(lo, l);
}

// Decay sums of a chunk in units of log2, as two fp32 terms each: their differences keep the accuracy of the small ones among large.
// A decay from token j to token i of another block of 32 is the product of the one from j to its block's last token (or to the first of
// i's) and the rest, one factor per row and block and one per column, both at most 1 and made once; inside a block of 32 it is an
// exponential of its own.
struct alignas(16) XGateTable {
  float2 sum[128];
  float to_last[128];     // decay from j to the last token of its block of 32
  float beta[128];
  float from_first[128];  // decay from the first token of i's block of 32 to i
};
static_assert(sizeof(XGateTable) == 2560, "as the workspace has it");
__device__ __forceinline__ float decay2(const float2& a, const float2& b) { return ex2_approx((a.x - b.x) + (a.y - b.y)); }
__device__ __forceinline__ float2 two_terms(double x) {
  const float h = (float)x;
  return make_float2(h, (float)(x - (double)h));
}
// Threads 0 .. 127 make a chunk's table, in shared memory and in its record, from where the other kernels take it; every thread of
// the block calls, a barrier has to follow.  part: four doubles.  end: the whole chunk's sum.
__device__ __forceinline__ void make_gates(XGateTable& s, double* part, unsigned char* rec, size_t table, float g, float beta, int tid, float2& end) {
  double x = 0.0;
  if (tid < 128) {
    x = clamped_log_decay(g) * 1.4426950408889634;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, x, o);
      if ((tid & 31) >= o) x += y;
    }
    if ((tid & 31) == 31) part[tid >> 5] = x;
  }
  __syncthreads();
  end = two_terms(((part[0] + part[1]) + part[2]) + part[3]);
  if (tid < 128) {
    for (int w = 0; w < (tid >> 5); ++w) x += part[w];
    const float2 own = two_terms(x);
    const float2 last = make_float2(__shfl_sync(0xffffffffu, own.x, 31), __shfl_sync(0xffffffffu, own.y, 31));
    const float2 first = make_float2(__shfl_sync(0xffffffffu, own.x, 0), __shfl_sync(0xffffffffu, own.y, 0));
    const float to_last = decay2(last, own), from_first = decay2(own, first);
    s.sum[tid] = own;
    s.beta[tid] = beta;
    s.to_last[tid] = to_last;
    s.from_first[tid] = from_first;
    XGateTable& kept = *reinterpret_cast<XGateTable*>(rec + table);
    kept.sum[tid] = own;
    kept.beta[tid] = beta;
    kept.to_last[tid] = to_last;
    kept.from_first[tid] = from_first;
    if (tid == 0) {
      *reinterpret_cast<float*>(rec) = ex2_approx(end.x + end.y);
      *reinterpret_cast<float2*>(rec + 8) = end;
    }
  }
}

struct XPlace {
  int b, h, hk, n;
  long long row, gate;
  size_t rec;
};
__device__ __forceinline__ XPlace x_place(const DeltaArgs& a, int bh, int c) {
  XPlace p;
  p.b = bh / a.H;
  p.h = bh % a.H;
  p.hk = p.h / (a.H / a.Hk);
  p.n = min(128, a.N - c * 128);
  p.row = p.b * a.sB + p.h * a.sH + (long long)c * 128 * a.sT;
  p.gate = p.b * a.gB + p.h * a.gH + (long long)c * 128 * a.gT;
  p.rec = (size_t)bh * a.nchunk + c;
  return p;
}

// The thread block `ahead` places after this one: what it will load is fetched to L2 while this one computes, so that HBM is busy all the
// time and not only while blocks begin.  (false: there is none)
__device__ __forceinline__ bool later_block(unsigned ahead, unsigned& x, unsigned& y) {
  const unsigned n = blockIdx.x + ahead;
  x = n % gridDim.x;
  y = blockIdx.y + n / gridDim.x;
  return y < gridDim.y;
}

// One warp looks, the others stand at the block's barrier: sixteen that look take issue slots of the thread block beside them (half
// of the prepare kernel's instructions were such looks; its time did not change, since the slots were not what it waited for).  Then each
// sees the completed phase for itself.
#define X_WAIT(bar, par, code)                                                \
  do {                                                                        \
    bool ok_ = true;                                                          \
    if (threadIdx.x < 32) {                                                   \
      ok_ = wait_or_abort(&(bar), (par), &sm.abort);                          \
      if (!ok_ && !sm.abort) atomicCAS(&g_tc_status, 0u, (unsigned)(code));   \
      if (!ok_) sm.abort = 1;                                                 \
    }                                                                         \
    if (!__syncthreads_and(ok_)) return false;                                \
    if (threadIdx.x >= 32) (void)mbar_try_wait(&(bar), (par));                \
    tc_fence_after_sync();                                                    \
  } while (0)

// Operands written to shared memory (or tensor memory) are handed to the tensor cores: fences and a barrier.
#define X_HAND_OVER()            \
  do {                           \
    fence_proxy_async_smem();    \
    tmem_st_wait();              \
    tc_fence_before_sync();      \
    __syncthreads();             \
    tc_fence_after_sync();       \
  } while (0)

// Announces `bytes` of loads on barrier i (one thread).
template <typename SM>
__device__ __forceinline__ uint64_t* expect(SM& sm, int i, uint32_t bytes) {
  ++sm.armed[i];
  mbar_arrive_expect_tx(&sm.bars[i], bytes);
  return &sm.bars[i];
}

// Products are issued by warp 0, and in the gradient kernel by this one too.
constexpr int X_ISSUER = 12;

// Start and end that all kernels below share.  body() returns false when a wait gave up.
template <int COLS, typename SM, typename F>
__device__ __forceinline__ void x_run(SM& sm, int nbars, F body) {
  const int tid = threadIdx.x, warp = tid >> 5;
  grid_dep_wait();
  if (tid == 0) {
    for (int i = 0; i < nbars; ++i) {
      mbar_init(&sm.bars[i], 1);
      sm.armed[i] = 0;
    }
    sm.abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_slot, COLS);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  grid_dep_launch();
  const uint32_t tmem = sm.tmem_slot;
  const bool ok = body(tmem);
  if (!ok) {  // products and copies that are still under way end before the block does; those of a warp are told by its own commit
    for (int w = 0, par = 0; w < (int)(blockDim.x >> 5); w += X_ISSUER, par ^= 1) {
      if (warp == w) {
        umma_commit_if(&sm.bars[nbars - 1], elect_one());
        drain_wait(&sm.bars[nbars - 1], par);
      }
      __syncthreads();
    }
    if (tid == 32)
      for (int i = 0; i < nbars - 1; ++i)
        if (sm.armed[i]) drain_wait(&sm.bars[i], (sm.armed[i] - 1) & 1);
  }
  if (tid == 0) bulk_store_done();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, COLS);
}

constexpr uint32_t XHI = UMMA_DESC_HI_SBO1024;
__device__ __forceinline__ uint32_t kmaj(const void* p) { return umma_desc_lo(smem_u32(p), 16); }
__device__ __forceinline__ uint32_t mnmaj(const void* p, uint32_t panel = 16384) { return umma_desc_lo(smem_u32(p), panel); }

// ---- prepare ---------------------------------------------------------------------------------------------------------------------------
// One thread block of 512 threads per chunk; 101 KB of shared memory and 256 columns of tensor memory, so that two share an SM and one's
// products run beside the other's conversions.  Thread (q, lane) of quarter w has row q * 32 + lane of every accumulator and of every
// image, columns w * 32 .. + 31: one block of 32 tokens.
//
// The inverse U of the upper triangular I + (n diag(beta))^T: columns of the four diagonal blocks of 32 by back substitution in fp32 (a
// warp each), then U12 = -U11 A12 U22 on the tensor cores for the two blocks of 64 at once, then for the whole.  (On the CUDA cores the
// step from 16 to 64 took 11000 clocks with two thread blocks to an SM.)  Powers of the triangle would need no order of rows, but grow far beyond the inverse where keys are
// alike.
//
// What it costs is the latency of its dependent steps, of which nine wait for a product, and the instructions between them, most of
// which are executed once and fetched for it.  2048 chunks, D = 128, us: decays made by every kernel for itself and all of them
// exponentials, 256 threads, 525; factors made once, 255; with 512 threads 228, of which the tensor cores work for a fifth
// and an instruction is issued in two clocks of five; 217 since U and X move without their zeros (0.6 GB in 0.2 ms: HBM is not it).
enum { XP_LOAD = 0, XP_V, XP_MMA, XP_DRAIN, XP_BARS };
template <int D>
struct alignas(1024) XPrepSmem {
  unsigned char k[32768];  // (D = 64: the keys twice)
  unsigned char x[65536];  // q; blocks of A and U in fp32; images of U and X; v; image of M
  XGateTable gates;
  float until[128];        // beta e^(G_end - G)
  float since[128];        // e^G
  float last_beta[128];    // gates.to_last times beta
  double part[4];
  uint64_t bars[XP_BARS];
  int armed[XP_BARS];
  uint32_t tmem_slot;
  int abort;
};

// element (i, m) of a 32 x 32 fp32 block whose 16-byte groups are permuted by row, so that a thread per row stores without conflicts
__device__ __forceinline__ int block_at(int i, int m) { return i * 32 + ((((m >> 2) ^ i) & 7) << 2) + (m & 3); }

template <int D>
__global__ void __launch_bounds__(512, 2)
x_prepare_kernel(const __grid_constant__ XMaps maps, const __grid_constant__ DeltaArgs a) {
  extern __shared__ unsigned char smem_raw[];
  using Rec = XRec<D>;
  XPrepSmem<D>& sm = *reinterpret_cast<XPrepSmem<D>*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3, w4 = warp >> 2, row = q * 32 + lane, c0 = w4 * 32;
  x_run<256>(sm, XP_BARS, [&](const uint32_t tmem) -> bool {
    const XPlace p = x_place(a, blockIdx.y, blockIdx.x);
    unsigned char* const rec = static_cast<unsigned char*>(a.ws) + p.rec * Rec::FWD;
    const uint32_t R = tmem, P = tmem + 128, mine = (uint32_t)(q * 32) << 16;
    constexpr int PANELS = D / 64;
    float g_own = 0.f, beta_own = 0.f;
    if (tid < p.n) {
      g_own = ld_f1(a.g + p.gate + tid * a.gT);
      beta_own = ld_f1(a.beta + p.gate + tid * a.gT);
    }
    if (tid == 0) {
      uint64_t* const bar = expect(sm, XP_LOAD, (2 + PANELS) * 16384);
      for (int x = 0; x < 2; ++x) tma_load_4d(sm.k + x * 16384, &maps.k, bar, D == 128 ? x * 64 : 0, blockIdx.x * 128, p.hk, p.b);
      for (int x = 0; x < PANELS; ++x) tma_load_4d(sm.x + x * 16384, &maps.q, bar, x * 64, blockIdx.x * 128, p.hk, p.b);
      for (int x = 0; x < PANELS; ++x) tma_prefetch_4d(&maps.v, x * 64, blockIdx.x * 128, p.h, p.b);
    }
    float2 end;
    make_gates(sm.gates, sm.part, rec, Rec::GATES, g_own, beta_own, tid, end);
    if (tid < 128) {
      const float2 s = sm.gates.sum[tid];
      sm.since[tid] = ex2_approx(s.x + s.y);
      sm.until[tid] = beta_own * decay2(end, s);
      sm.last_beta[tid] = beta_own * sm.gates.to_last[tid];
    }
    constexpr uint32_t ID_KK = umma_idesc_bf16(128, 128, false, false);
    constexpr uint32_t ID_KN64 = umma_idesc_bf16(128, 64, false, true), ID_KN32 = umma_idesc_bf16(128, 32, false, true);
    constexpr uint32_t ID_KN = umma_idesc_bf16(128, 128, false, true);
    constexpr uint32_t ID_NK = umma_idesc_bf16(128, 128, true, false);
    constexpr int NK = D / 16;
    __syncwarp();
    const uint32_t go = warp == 0 ? elect_one() : 0;
    int par = 0;
    X_WAIT(sm.bars[XP_LOAD], 0, 50);
    if (warp == 0) {
      umma_group_ss<NK, true, true>(R, kmaj(sm.k), kmaj(sm.k), XHI, ID_KK, 0, go);
      umma_group_ss<NK, true, true>(P, kmaj(sm.x), kmaj(sm.k), XHI, ID_KK, 0, go);
      umma_commit_if(&sm.bars[XP_MMA], go);
    }
    X_WAIT(sm.bars[XP_MMA], par, 51);
    par ^= 1;

    // A = (n diag(beta))^T: row j, columns i > j.  Shared memory by turns: blocks of 32 on A's and on U's diagonal, U's blocks beside them,
    // and a B operand of two times 32 rows.
    float* const fa = reinterpret_cast<float*>(sm.x);
    float* const fu = reinterpret_cast<float*>(sm.x + 16384);
    float* const fu12 = reinterpret_cast<float*>(sm.x + 32768);
    unsigned char* const pair = sm.x + 40960;
    const float2 own = sm.gates.sum[row];
    const float bt = sm.gates.beta[row];
    // A's columns of this thread where they are of a later block of 32: one factor for the row, one for each column
    auto later_columns = [&](uint32_t(&h)[16], uint32_t(&l)[16]) {
      float x[32];
      load_acc(R + mine + c0, x);
      const float f = bt * decay2(sm.gates.sum[c0], own);
      const uint64_t ff = f2_pack(f, f);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float2 d = *reinterpret_cast<const float2*>(&sm.gates.from_first[c0 + 2 * i]);
        split2(f2_mul(f2_mul(f2_pack(d.x, d.y), ff), f2_pack(x[2 * i], x[2 * i + 1])), h[i], l[i]);
      }
    };
    {
      uint32_t h[16], l[16];
      const bool corner = q < 2 && w4 >= 2;
      if (w4 == q) {
        float x[32];
        load_acc(R + mine + c0, x);
#pragma unroll
        for (int c = 0; c < 32; ++c) x[c] = c > lane ? x[c] * (decay2(sm.gates.sum[c0 + c], own) * bt) : 0.f;
#pragma unroll
        for (int c = 0; c < 32; c += 4)
          *reinterpret_cast<float4*>(fa + q * 1024 + block_at(lane, c)) = make_float4(x[c], x[c + 1], x[c + 2], x[c + 3]);
      } else if (corner) {
        later_columns(h, l);
      }
      tc_fence_before_sync();
      __syncthreads();  // (the scores are read)
      tc_fence_after_sync();
      if (corner) {  // the corner of 64 x 64, an A operand of lanes 0 .. 63
        tmem_st_x16(R + mine + 64 + (w4 - 2) * 16, h);
        tmem_st_x16(R + mine + 96 + (w4 - 2) * 16, l);
      }
    }
    {  // P = scale ((Q K^T) (.) D) diag(beta), row i, columns m <= i, as an A operand in place of its scores
      uint32_t h[16], l[16];
      if (w4 < q) {
        float x[32];
        load_acc(P + mine + c0, x);
        const float f = a.scale * decay2(own, sm.gates.sum[c0 + 31]);
        const uint64_t ff = f2_pack(f, f);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float2 d = *reinterpret_cast<const float2*>(&sm.last_beta[c0 + 2 * i]);
          split2(f2_mul(f2_mul(f2_pack(d.x, d.y), ff), f2_pack(x[2 * i], x[2 * i + 1])), h[i], l[i]);
        }
      } else if (w4 == q) {
        float x[32];
        load_acc(P + mine + c0, x);
#pragma unroll
        for (int c = 0; c < 32; ++c) x[c] = c <= lane ? x[c] * (decay2(own, sm.gates.sum[c0 + c]) * (a.scale * sm.gates.beta[c0 + c])) : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) split2(f2_pack(x[2 * i], x[2 * i + 1]), h[i], l[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) h[i] = l[i] = 0u;
      }
      // The corner of 32 x 32 of the blocks of 64, lanes 0 .. 31 and 64 .. 95, lies for a while where P is zero in those rows
      const bool small = (q == 0 && w4 == 1) || (q == 2 && w4 == 3);
      tc_fence_before_sync();
      __syncthreads();
      tc_fence_after_sync();
      if (!(w4 == 3 && (q & 1) == 0)) {
        tmem_st_x16(P + mine + w4 * 16, h);
        tmem_st_x16(P + mine + 64 + w4 * 16, l);
      }
      if (small) {
        later_columns(h, l);
        tmem_st_x16(P + mine + 48, h);
        tmem_st_x16(P + mine + 112, l);
      }
    }
    if (warp < 4) {  // blocks of 32, one to a warp: column `lane` of the inverse, from the diagonal upwards
      const float* const blk = fa + warp * 1024;
      float* const to = fu + warp * 1024;
      float x[32];
#pragma unroll
      for (int i = 31; i >= 0; --i) {
        float v[4] = {i == lane ? 1.f : 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int m4 = (i + 1) / 4 * 4; m4 < 32; m4 += 4) {
          const float4 w = *reinterpret_cast<const float4*>(blk + block_at(i, m4));
          if (m4 + 0 > i) v[0] = fmaf(-w.x, x[m4 + 0], v[0]);
          if (m4 + 1 > i) v[1] = fmaf(-w.y, x[m4 + 1], v[1]);
          if (m4 + 2 > i) v[2] = fmaf(-w.z, x[m4 + 2], v[2]);
          if (m4 + 3 > i) v[3] = fmaf(-w.w, x[m4 + 3], v[3]);
        }
        x[i] = (v[0] + v[1]) + (v[2] + v[3]);
        to[block_at(i, lane)] = x[i];
      }
    }
    __syncthreads();
    // blocks of 64: the corner is -U11 (A12 U22), both at once: lanes 0 .. 31 and 64 .. 95 of one A operand, a B operand for each
    auto put_pair = [&](int b, int r, int c, const float (&x)[8]) {
      uint4 h, l;
      split8(x, h, l);
      const uint32_t at = b * 4096 + image_at(r, c, 32);
      *reinterpret_cast<uint4*>(pair + at) = h;
      *reinterpret_cast<uint4*>(pair + 8192 + at) = l;
    };
    auto row8 = [&](const float* blk, int r, int c, float (&x)[8]) {
      const float4 w0 = *reinterpret_cast<const float4*>(blk + block_at(r, 8 * c)), w1 = *reinterpret_cast<const float4*>(blk + block_at(r, 8 * c + 4));
      x[0] = w0.x; x[1] = w0.y; x[2] = w0.z; x[3] = w0.w; x[4] = w1.x; x[5] = w1.y; x[6] = w1.z; x[7] = w1.w;
    };
    auto pair_product = [&]() {  // to columns 0 .. 31 and 32 .. 63 of R
      if (warp == 0) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          umma_group_tsd2(R + 32 * b, P + 112, mnmaj(pair + b * 4096), XHI, ID_KN32, 0, go);
          umma_group_tsd2(R + 32 * b, P + 48, mnmaj(pair + 8192 + b * 4096), XHI, ID_KN32, 1, go);
          umma_group_tsd2(R + 32 * b, P + 48, mnmaj(pair + b * 4096), XHI, ID_KN32, 1, go);
        }
        umma_commit_if(&sm.bars[XP_MMA], go);
      }
    };
    if (tid < 256) {
      float x[8];
      row8(fu + ((tid >> 7) * 2 + 1) * 1024, (tid >> 2) & 31, tid & 3, x);
      put_pair(tid >> 7, (tid >> 2) & 31, tid & 3, x);
    }
    X_HAND_OVER();
    pair_product();
    X_WAIT(sm.bars[XP_MMA], par, 59);
    par ^= 1;
    const bool upper = (q & 1) == 0;
    float y8[8];
    if (upper) {
      float x[8];
      uint4 h, l;
      tmem_ld_x8(R + mine + 16 * q + w4 * 8, *reinterpret_cast<uint32_t(*)[8]>(&y8));
      tmem_ld_wait();
      put_pair(q >> 1, lane, w4, y8);
      row8(fu + q * 1024, lane, w4, x);
      split8(x, h, l);
      tmem_st_x4(P + mine + 48 + w4 * 4, h);
      tmem_st_x4(P + mine + 112 + w4 * 4, l);
    }
    X_HAND_OVER();
    pair_product();
    X_WAIT(sm.bars[XP_MMA], par, 60);
    par ^= 1;
    if (upper) {
      tmem_ld_x8(R + mine + 16 * q + w4 * 8, *reinterpret_cast<uint32_t(*)[8]>(&y8));
      tmem_ld_wait();
      float* const to = fu12 + (q >> 1) * 1024;
      *reinterpret_cast<float4*>(to + block_at(lane, 8 * w4)) = make_float4(-y8[0], -y8[1], -y8[2], -y8[3]);
      *reinterpret_cast<float4*>(to + block_at(lane, 8 * w4 + 4)) = make_float4(-y8[4], -y8[5], -y8[6], -y8[7]);
      tmem_st_x4(P + mine + 48 + w4 * 4, make_uint4(0u, 0u, 0u, 0u));
      tmem_st_x4(P + mine + 112 + w4 * 4, make_uint4(0u, 0u, 0u, 0u));
    }
    __syncthreads();
    // a row of a 64 x 64 operand in A's place (rows are those of the product's K), eight values at a time
    auto put_square = [&](int c, const float (&x)[8]) {
      uint4 h, l;
      split8(x, h, l);
      const uint32_t at = image_at(row & 63, c, 64);
      *reinterpret_cast<uint4*>(sm.x + at) = h;
      *reinterpret_cast<uint4*>(sm.x + 8192 + at) = l;
    };
    auto square_product = [&](uint32_t hi, uint32_t lo) {  // to columns 0 .. 63 of R
      if (warp == 0) {
        umma_group_tsd4<false>(R, lo, mnmaj(sm.x), XHI, ID_KN64, 0, go);
        umma_group_tsd4<false>(R, hi, mnmaj(sm.x + 8192), XHI, ID_KN64, 1, go);
        umma_group_tsd4<false>(R, hi, mnmaj(sm.x), XHI, ID_KN64, 1, go);
        umma_commit_if(&sm.bars[XP_MMA], go);
      }
    };
    auto block8 = [&](int blk, int c, float (&x)[8]) {  // columns 8 c .. of row `row & 63` of a diagonal block of 64 of U
      if (c >= 4) {
        row8(upper ? fu12 + blk * 1024 : fu + (2 * blk + 1) * 1024, lane, c - 4, x);
      } else if (upper) {
        row8(fu + 2 * blk * 1024, lane, c, x);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
      }
    };
    if (q >= 2) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x[8];
        block8(1, w4 * 2 + c, x);
        put_square(w4 * 2 + c, x);
      }
    }
    X_HAND_OVER();
    square_product(R + 64, R + 96);  // A12 U22 (lanes 64 .. 127: whatever)
    X_WAIT(sm.bars[XP_MMA], par, 52);
    par ^= 1;
    if (q < 2) {
      float y[16];
      load_acc16(R + mine + w4 * 16, y);
      tmem_ld_wait();
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x[8];
        uint4 h, l;
        put_square(w4 * 2 + c, *reinterpret_cast<const float(*)[8]>(&y[8 * c]));
        block8(0, w4 * 2 + c, x);
        split8(x, h, l);
        tmem_st_x4(R + mine + 64 + (w4 * 2 + c) * 4, h);
        tmem_st_x4(R + mine + 96 + (w4 * 2 + c) * 4, l);
      }
    }
    X_HAND_OVER();
    square_product(R + 64, R + 96);  // U11 (A12 U22)
    X_WAIT(sm.bars[XP_MMA], par, 53);
    par ^= 1;
    auto put_image = [&](const uint4 (&h)[4], const uint4 (&l)[4], int r, int c, int rows, uint32_t lo) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t at = image_at(r, c + k, rows);
        *reinterpret_cast<uint4*>(sm.x + at) = h[k];
        *reinterpret_cast<uint4*>(sm.x + lo + at) = l[k];
      }
    };
    uint4 h[4], l[4];
    auto terms = [&](const float (&x)[32]) {
#pragma unroll
      for (int k = 0; k < 4; ++k) split8(&x[8 * k], h[k], l[k]);
    };
    // the image of U, over all of its blocks once they have been read
    if (q < 2 && w4 >= 2) {
      float x[32];
      load_acc(R + mine + (w4 - 2) * 32, x);
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i] = -x[i];
      terms(x);
    } else if (q >= 2 && w4 < 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) h[k] = l[k] = make_uint4(0u, 0u, 0u, 0u);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float x[8];
        block8(q >> 1, (w4 & 1) * 4 + k, x);
        split8(x, h[k], l[k]);
      }
    }
    __syncthreads();
    put_image(h, l, row, w4 * 4, 128, 32768);
    X_HAND_OVER();
    if (tid == 0) {
      store_triangle<true>(rec + Rec::U, sm.x);
      tma_store_commit();
    }
    if (warp == 0) {  // X = P That: That [m][j] is U [j][m]
      umma_group_tsd<true>(R, P + 64, kmaj(sm.x), XHI, ID_KK, 0, go);
      umma_group_tsd<true>(R, P, kmaj(sm.x + 32768), XHI, ID_KK, 1, go);
      umma_group_tsd<true>(R, P, kmaj(sm.x), XHI, ID_KK, 1, go);
      umma_commit_if(&sm.bars[XP_MMA], go);
      if (tid == 0) tma_store_wait_read();
      __syncwarp();
    }
    // U's columns times beta e^(G_end - G)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t *const hw = &h[k].x, *const lw = &l[k].x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 u = *reinterpret_cast<const float2*>(&sm.until[c0 + 8 * k + 2 * i]);
        split2(f2_mul(f2_add(f2_pack(bf_lo(hw[i]), bf_hi(hw[i])), f2_pack(bf_lo(lw[i]), bf_hi(lw[i]))), f2_pack(u.x, u.y)), hw[i], lw[i]);
      }
    }
    X_WAIT(sm.bars[XP_MMA], par, 54);
    par ^= 1;
    put_image(h, l, row, w4 * 4, 128, 32768);
    X_HAND_OVER();
    if (warp == 0) {  // J^T [d, j] = K^T U'^T
      umma_group_ss<8, false, true>(P, mnmaj(sm.k), kmaj(sm.x + 32768), XHI, ID_NK, 0, go);
      umma_group_ss<8, false, true>(P, mnmaj(sm.k), kmaj(sm.x), XHI, ID_NK, 1, go);
      umma_commit_if(&sm.bars[XP_MMA], go);
    }
    {  // X leaves as an image
      float x[32];
      load_acc(R + mine + c0, x);
      terms(x);
    }
    X_WAIT(sm.bars[XP_MMA], par, 55);
    par ^= 1;
    put_image(h, l, row, w4 * 4, 128, 32768);
    X_HAND_OVER();
    if (tid == 0) {
      store_triangle<false>(rec + Rec::X, sm.x);
      tma_store_commit();
    }
    {  // J^T as an A operand in X's place; D = 64: lanes 64 .. 127 have J^T once more, for M, times e^G
      float x[32];
      load_acc(P + mine + c0, x);
      if (D == 64 && q >= 2) {
#pragma unroll
        for (int c = 0; c < 32; ++c) x[c] *= sm.since[c0 + c];
      }
      store_operand(R + mine + w4 * 16, R + mine + 64 + w4 * 16, x);
    }
    if (tid == 0) {  // (D = 64: [V | K])
      tma_store_wait_read();
      uint64_t* const bar = expect(sm, XP_V, 32768);
      tma_load_4d(sm.x, &maps.v, bar, 0, blockIdx.x * 128, p.h, p.b);
      if (D == 128) tma_load_4d(sm.x + 16384, &maps.v, bar, 64, blockIdx.x * 128, p.h, p.b);
      else tma_load_4d(sm.x + 16384, &maps.k, bar, 0, blockIdx.x * 128, p.hk, p.b);
    }
    X_HAND_OVER();
    X_WAIT(sm.bars[XP_V], 0, 56);
    if (warp == 0) {  // N = J^T V
      umma_group_tsd<false>(P, R + 64, mnmaj(sm.x), XHI, ID_KN, 0, go);
      umma_group_tsd<false>(P, R, mnmaj(sm.x), XHI, ID_KN, 1, go);
      umma_commit_if(&sm.bars[XP_MMA], go);
    }
    X_WAIT(sm.bars[XP_MMA], par, 57);
    par ^= 1;
    float* const n_to = reinterpret_cast<float*>(rec + Rec::N) + row;  // column by column: a warp stores 128 consecutive bytes
    float x[32];
    if (D == 128) {  // N is stored while M is made of J^T diag(e^G)
      tmem_ld_x32(P + mine + c0, *reinterpret_cast<uint32_t(*)[32]>(&x));
#pragma unroll
      for (int pc = 0; pc < 2; ++pc) {
        uint32_t jh[8], jl[8];
        tmem_ld_x8(R + mine + w4 * 16 + pc * 8, jh);
        tmem_ld_x8(R + mine + 64 + w4 * 16 + pc * 8, jl);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 s = *reinterpret_cast<const float2*>(&sm.since[c0 + pc * 16 + 2 * i]);
          split2(f2_mul(f2_add(f2_pack(bf_lo(jh[i]), bf_hi(jh[i])), f2_pack(bf_lo(jl[i]), bf_hi(jl[i]))), f2_pack(s.x, s.y)), jh[i], jl[i]);
        }
        tmem_st_x8(R + mine + w4 * 16 + pc * 8, jh);
        tmem_st_x8(R + mine + 64 + w4 * 16 + pc * 8, jl);
      }
      X_HAND_OVER();
      if (warp == 0) {
        umma_group_tsd<false>(P, R + 64, mnmaj(sm.k), XHI, ID_KN, 0, go);
        umma_group_tsd<false>(P, R, mnmaj(sm.k), XHI, ID_KN, 1, go);
        umma_commit_if(&sm.bars[XP_MMA], go);
      }
#pragma unroll
      for (int c = 0; c < 32; ++c) n_to[(c0 + c) * D] = x[c];
      X_WAIT(sm.bars[XP_MMA], par, 58);
    } else if (q < 2 && w4 < 2) {
      load_acc(P + mine + c0, x);
#pragma unroll
      for (int c = 0; c < 32; ++c) n_to[(c0 + c) * D] = x[c];
    }
    if (D == 128 || (q >= 2 && w4 >= 2)) {
      load_acc(P + mine + c0, x);
      terms(x);
      put_image(h, l, row & (D - 1), (w4 * 4) & (D / 8 - 1), D, D * D * 2);
    }
    X_HAND_OVER();
    if (tid == 0) {
      bulk_store(rec + Rec::M, sm.x, D * D * 4);
      tma_store_commit();
    }
    return true;
  });
}

// ---- chain -----------------------------------------------------------------------------------------------------------------------------
// S' = e^G_end S - M S + N over the chunks (REV: E = e^G_end E' - M^T E' + B from the last to the first), NE value columns of one head
// per thread block, the state in registers in fp32; the state that enters each chunk (REV: the gradient of the one that leaves it) goes
// to the workspace as an image.  A step is one product, a conversion and two barriers; the images of M come three steps ahead.
// Both terms of the state are columns of one B operand, [hi | lo], so that hi of M meets both in one pass: with NE = 32 an
// instruction takes as long as its A operand comes from shared memory, whatever its columns.  Of a step's 2540 clocks the products take
// 1600: M passes through shared memory twice, 64 KB in and 64 KB out to the tensor cores; half the columns for M's lo terms, state images
// stored from registers instead of by a bulk copy or one warp alone looking for the products' end change nothing.  2048 chunks in 32 heads: 122 us.
// D = 64: both terms of M are rows of one A operand; the rows of lo pass through shared memory to the threads of those of hi.
constexpr int XC_STAGES = 3;
enum { XC_LOAD0 = 0, XC_MMA = XC_STAGES, XC_DRAIN, XC_BARS };
template <int D, int NE>
struct alignas(1024) XChainSmem {
  unsigned char m[XC_STAGES][D * D * 4];
  unsigned char b[2 * NE * D * 2];
  float other[D == 64 ? 64 : 1][NE + 1];
  uint64_t bars[XC_BARS];
  int armed[XC_BARS];
  uint32_t tmem_slot;
  int abort;
};
struct XChainArgs {
  const unsigned char* fwd;  // records with M and e^G_end
  const unsigned char* add;  // N or B of chunk 0 of head 0
  unsigned char* image;      // where the images of the states go
  size_t fwd_stride, add_stride, image_stride;
  const float* in;           // [BH, D, D] or NULL
  float* out;
  int nchunk;
};

template <int D, int NE, bool REV>
__global__ void __launch_bounds__(256)
x_chain_kernel(const __grid_constant__ XChainArgs a) {
  extern __shared__ unsigned char smem_raw[];
  using Rec = XRec<D>;
  using Sm = XChainSmem<D, NE>;
  Sm& sm = *reinterpret_cast<Sm*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  constexpr int V = NE / 2;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3, half = warp >> 2, row = q * 32 + lane;
  constexpr uint32_t COLS = 2 * NE < 32 ? 32 : 2 * NE;
  x_run<COLS>(sm, XC_BARS, [&](const uint32_t tmem) -> bool {
    const int bh = blockIdx.y, e0 = blockIdx.x * NE;
    const uint32_t mine = (uint32_t)(q * 32) << 16;
    const bool owner = D == 128 || q < 2;
    const int first = REV ? a.nchunk - 1 : 0, step = REV ? -1 : 1;
    auto index = [&](int i) { return (size_t)bh * a.nchunk + (size_t)(first + step * i); };
    auto load_m = [&](int i) {
      const int s = i % XC_STAGES;
      bulk_load(sm.m[s], a.fwd + index(i) * a.fwd_stride + Rec::M, D * D * 4, expect(sm, XC_LOAD0 + s, D * D * 4));
    };
    if (tid == 0)
      for (int i = 0; i < XC_STAGES && i < a.nchunk; ++i) load_m(i);
    __syncwarp();
    const uint32_t go = warp == 0 ? elect_one() : 0;
    constexpr uint32_t ID2 = umma_idesc_bf16(128, 2 * NE, REV, true);
    float s[V], add[V], all = 0.f;
    if (owner) {
      const size_t at = ((size_t)bh * D + row) * D + e0 + half * V;
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const float4 w = a.in ? ld_f4(reinterpret_cast<const float4*>(a.in + at + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
        s[i] = w.x; s[i + 1] = w.y; s[i + 2] = w.z; s[i + 3] = w.w;
      }
    }
    auto fetch = [&](int i, float (&to)[V], float& f) {  // of step i
      const float* const from = reinterpret_cast<const float*>(a.add + index(i) * a.add_stride) + (size_t)(e0 + half * V) * D + row;
#pragma unroll
      for (int x = 0; x < V; ++x) to[x] = ld_f1(from + x * D);
      f = ld_f1(reinterpret_cast<const float*>(a.fwd + index(i) * a.fwd_stride + Rec::ALL));
    };
    if (owner) fetch(0, add, all);
    int par = 0;
    for (int i = 0; i < a.nchunk; ++i) {
      if (owner) {
#pragma unroll
        for (int c = 0; c < V / 8; ++c) {
          uint4 h, l;
          split8(&s[8 * c], h, l);
          const int col = (half * V / 32) * 8 + half * V % 32 / 8 + c;  // 16-byte group, the lo terms four further
          *reinterpret_cast<uint4*>(sm.b + image_at(row, col, D)) = h;
          *reinterpret_cast<uint4*>(sm.b + image_at(row, col + 4, D)) = l;
        }
      }
      X_HAND_OVER();
      if (tid == 0) {
        bulk_store(a.image + index(i) * a.image_stride + (size_t)e0 * D * 4, sm.b, NE * D * 4);
        tma_store_commit();
      }
      if (warp == 0) {
        const int st = i % XC_STAGES;
        const bool ok = wait_or_abort(&sm.bars[XC_LOAD0 + st], (i / XC_STAGES) & 1, &sm.abort);
        if (__all_sync(0xffffffffu, ok)) {
          tc_fence_after_sync();
          const unsigned char* const m = sm.m[st];
          const uint32_t b = mnmaj(sm.b, D * 128);
          if (D == 128) {
            umma_group_ss<8, !REV, false>(tmem, REV ? mnmaj(m + 32768) : kmaj(m + 32768), b, XHI, ID2, 0, go);
            umma_group_ss<8, !REV, false>(tmem, REV ? mnmaj(m) : kmaj(m), b, XHI, ID2, 1, go);
          } else {
            umma_group_ss<4, !REV, false>(tmem, REV ? mnmaj(m, 8192) : kmaj(m), b, XHI, ID2, 0, go);
          }
          umma_commit_if(&sm.bars[XC_MMA], go);
        } else {
          if (!ok && !sm.abort) atomicCAS(&g_tc_status, 0u, 62u);
          sm.abort = 1;
        }
      }
      float next[V], next_all = 0.f;
      if (owner && i + 1 < a.nchunk) fetch(i + 1, next, next_all);
      if (tid == 0) tma_store_wait_read();  // (the barrier of X_WAIT lets the next operand be written)
      __syncwarp();
      X_WAIT(sm.bars[XC_MMA], par, 61);
      par ^= 1;
      if (tid == 0 && i + XC_STAGES < a.nchunk) load_m(i + XC_STAGES);
      __syncwarp();
      uint32_t d0[V], d1[V];
      if (V == 16) {
        tmem_ld_x16(tmem + mine + half * V, *reinterpret_cast<uint32_t(*)[16]>(d0));
        tmem_ld_x16(tmem + mine + 32 + half * V, *reinterpret_cast<uint32_t(*)[16]>(d1));
      } else {
        tmem_ld_x32(tmem + mine + half * 64, *reinterpret_cast<uint32_t(*)[32]>(d0));
        tmem_ld_x32(tmem + mine + half * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(d1));
      }
      tmem_ld_wait();
      if constexpr (D == 64) {
        if (!owner)
#pragma unroll
          for (int x = 0; x < V; ++x) sm.other[row - 64][half * V + x] = __uint_as_float(d0[x]) + __uint_as_float(d1[x]);
        __syncthreads();
      }
      if (owner) {
#pragma unroll
        for (int x = 0; x < V; ++x) {
          float m = __uint_as_float(d0[x]) + __uint_as_float(d1[x]);
          if constexpr (D == 64) m += sm.other[row][half * V + x];
          s[x] = fmaf(all, s[x], add[x]) - m;
          add[x] = next[x];
        }
        all = next_all;
      }
    }
    if (owner && a.out) {
      const size_t at = ((size_t)bh * D + row) * D + e0 + half * V;
#pragma unroll
      for (int x = 0; x < V; x += 4) *reinterpret_cast<float4*>(a.out + at + x) = make_float4(s[x], s[x + 1], s[x + 2], s[x + 3]);
    }
    return true;
  });
}

// ---- output ----------------------------------------------------------------------------------------------------------------------------
// O = scale diag(e^G) Q S + X (V - diag(e^G) K S): 64 value columns of a chunk per thread block, two thread blocks to an SM.  Both terms of
// the state, and then of the bracket, are one B operand of 128 columns [hi | lo]; the halves of the results are added up on the way
// out of tensor memory.  Bound by its three dependent groups of products; the loads of the thread block 296 places on come to L2 meanwhile.
// 2048 chunks: 103 us, 0.5 GB (43 % of HBM's rate).
enum { XO_LOAD = 0, XO_X, XO_MMA, XO_DRAIN, XO_BARS };
template <int D>
struct alignas(1024) XOutSmem {
  unsigned char qk[65536];  // q, k; then X
  unsigned char s[32768];   // [hi | lo] of the state's columns, then of the bracket
  XGateTable gates;
  uint64_t bars[XO_BARS];
  int armed[XO_BARS];
  uint32_t tmem_slot;
  int abort;
};

// 8 N values of a token's row as they are (or zeros), and what to do with each
template <int N>
__device__ __forceinline__ void load_raw32(const __nv_bfloat16* p, bool in, uint4 (&w)[N]) {
#pragma unroll
  for (int c = 0; c < N; ++c) {
    w[c] = make_uint4(0u, 0u, 0u, 0u);
    if (in) w[c] = *reinterpret_cast<const uint4*>(p + 8 * c);
  }
}
template <int N, typename F>
__device__ __forceinline__ void each32(const uint4 (&w)[N], F f) {
#pragma unroll
  for (int c = 0; c < N; ++c) {
    f(8 * c, bf_lo(w[c].x)); f(8 * c + 1, bf_hi(w[c].x)); f(8 * c + 2, bf_lo(w[c].y)); f(8 * c + 3, bf_hi(w[c].y));
    f(8 * c + 4, bf_lo(w[c].z)); f(8 * c + 5, bf_hi(w[c].z)); f(8 * c + 6, bf_lo(w[c].w)); f(8 * c + 7, bf_hi(w[c].w));
  }
}
// 32 values of a row of a result, columns c0 .. + 31, to a tile of 128-byte rows in the swizzle (panels of 64 bf16 or 32 fp32 columns): a
// thread that stored its row itself would touch as many lines as there are lanes with every instruction.
template <typename T>
__device__ __forceinline__ void put_row32(unsigned char* tile, int row, int c0, const float (&x)[32]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x[8 * c + 2 * i], x[8 * c + 2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
      }
      *reinterpret_cast<uint4*>(tile + image_at(row, c0 / 8 + c, 128)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
#pragma unroll
    for (int c = 0; c < 8; ++c)
      *reinterpret_cast<float4*>(tile + image_at(row, c0 / 4 + c, 128)) = make_float4(x[4 * c], x[4 * c + 1], x[4 * c + 2], x[4 * c + 3]);
  }
}
// One thread: the tile's `cols` columns to columns x0 .. of the result.
template <typename T>
__device__ __forceinline__ void store_tile(const CUtensorMap* map, const unsigned char* tile, int x0, int cols, int token, int head, int batch) {
  constexpr int PER = 128 / (int)sizeof(T);
  for (int x = 0; x < cols; x += PER) tma_store_4d(map, tile + x / PER * 16384, x0 + x, token, head, batch);
}
// The sum of the two halves [hi | lo], 64 columns each, of a product: columns c0 .. c0 + 31
__device__ __forceinline__ void load_both(uint32_t taddr, float (&x)[32]) {
  float y[32];
  load_acc(taddr, x);
  load_acc(taddr + 64, y);
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] += y[i];
}

// The same of a product with a state's slices [hi | lo], 32 columns each: the 32 of slice s
__device__ __forceinline__ void load_slice(uint32_t taddr, int s, float (&x)[32]) {
  float y[32];
  load_acc(taddr + 64 * s, x);
  load_acc(taddr + 64 * s + 32, y);
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] += y[i];
}

template <int D, typename TO>
__global__ void __launch_bounds__(256, 2)
x_output_kernel(const __grid_constant__ XMaps maps, const __grid_constant__ DeltaArgs a) {
  extern __shared__ unsigned char smem_raw[];
  using Rec = XRec<D>;
  XOutSmem<D>& sm = *reinterpret_cast<XOutSmem<D>*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3, half = warp >> 2, row = q * 32 + lane;
  x_run<256>(sm, XO_BARS, [&](const uint32_t tmem) -> bool {
    constexpr int PANELS = D / 64, NK = D / 16;
    const int c = blockIdx.x / PANELS, eh = blockIdx.x % PANELS;
    const XPlace p = x_place(a, blockIdx.y, c);
    const unsigned char* const rec = static_cast<const unsigned char*>(a.ws) + p.rec * Rec::FWD;
    const uint32_t mine = (uint32_t)(q * 32) << 16;
    if (tid == 0) {
      uint64_t* const bar = expect(sm, XO_LOAD, 2 * PANELS * 16384 + 2 * D * 128 + 2560);
      bulk_load(&sm.gates, rec + Rec::GATES, 2560, bar);
      for (int x = 0; x < PANELS; ++x) tma_load_4d(sm.qk + x * 16384, &maps.q, bar, x * 64, c * 128, p.hk, p.b);
      for (int x = 0; x < PANELS; ++x) tma_load_4d(sm.qk + 32768 + x * 16384, &maps.k, bar, x * 64, c * 128, p.hk, p.b);
      bulk_load(sm.s, rec + Rec::S + eh * 2 * D * 128, 2 * D * 128, bar);
      prefetch_triangle<false>(rec + Rec::X);
      unsigned nx, ny;
      if (later_block(296, nx, ny) && nx % PANELS == 0) {
        const XPlace o = x_place(a, ny, nx / PANELS);
        for (int x = 0; x < PANELS; ++x) {
          tma_prefetch_4d(&maps.q, x * 64, nx / PANELS * 128, o.hk, o.b);
          tma_prefetch_4d(&maps.k, x * 64, nx / PANELS * 128, o.hk, o.b);
          tma_prefetch_4d(&maps.v, x * 64, nx / PANELS * 128, o.h, o.b);
        }
        prefetch(static_cast<const unsigned char*>(a.ws) + o.rec * Rec::FWD + Rec::S, Rec::STATE);
      }
    }
    uint4 raw[4];
    load_raw32(static_cast<const __nv_bfloat16*>(a.v) + p.row + row * a.sT + eh * 64 + half * 32, row < p.n, raw);
    __syncwarp();
    const uint32_t go = warp == 0 ? elect_one() : 0;
    constexpr uint32_t ID2 = umma_idesc_bf16(128, 128, false, true);
    X_WAIT(sm.bars[XO_LOAD], 0, 70);
    const float since = ex2_approx(sm.gates.sum[row].x + sm.gates.sum[row].y);
    if (warp == 0) {
      umma_group_ss<NK, true, false>(tmem, kmaj(sm.qk + 32768), mnmaj(sm.s, D * 128), XHI, ID2, 0, go);
      umma_group_ss<NK, true, false>(tmem + 128, kmaj(sm.qk), mnmaj(sm.s, D * 128), XHI, ID2, 0, go);
      umma_commit_if(&sm.bars[XO_MMA], go);
    }
    X_WAIT(sm.bars[XO_MMA], 0, 71);
    if (tid == 0) load_triangle<false>(sm.qk, rec + Rec::X, expect(sm, XO_X, TRIANGLE));
    clear_triangle<false>(sm.qk, tid, 256);
    {
      float x[32];
      load_slice(tmem + mine, half, x);
      each32(raw, [&](int i, float v) { x[i] = fmaf(-since, x[i], v); });
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint4 h, l;
        split8(&x[8 * i], h, l);
        const uint32_t at = image_at(row, half * 4 + i, 128);
        *reinterpret_cast<uint4*>(sm.s + at) = h;
        *reinterpret_cast<uint4*>(sm.s + 16384 + at) = l;
      }
    }
    X_HAND_OVER();
    X_WAIT(sm.bars[XO_X], 0, 72);
    if (warp == 0) {
      umma_group_ss<8, true, false>(tmem, kmaj(sm.qk + 32768), mnmaj(sm.s), XHI, ID2, 0, go);
      umma_group_ss<8, true, false>(tmem, kmaj(sm.qk), mnmaj(sm.s), XHI, ID2, 1, go);
      umma_commit_if(&sm.bars[XO_MMA], go);
    }
    float v[32];
    load_slice(tmem + 128 + mine, half, v);
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] *= a.scale * since;
    X_WAIT(sm.bars[XO_MMA], 1, 73);
    float x[32];
    load_both(tmem + mine + half * 32, x);
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] += v[i];
    put_row32<TO>(sm.qk, row, half * 32, x);
    X_HAND_OVER();
    if (tid == 0) {
      store_tile<TO>(&maps.o, sm.qk, eh * 64, 64, c * 128, p.h, p.b);
      tma_store_commit();
    }
    return true;
  });
}

// ---- adjoint ---------------------------------------------------------------------------------------------------------------------------
// Z = X^T dO, and B = scale Q^T diag(e^G) dO - K^T diag(e^G) Z for the chain in reverse: 64 value columns of a chunk per thread block.
// D = 64: [Q | K] are the rows of one A operand and [dO' | Z'] the columns of one B operand, of whose product two quarters are wanted.
// 2048 chunks: 130 us, 0.5 GB; fetching ahead to L2, as the kernels around it do, made this one slower (and the prepare kernel).
enum { XA_LOAD = 0, XA_QK, XA_MMA, XA_DRAIN, XA_BARS };
template <int D>
struct alignas(1024) XAdjSmem {
  unsigned char x[65536];   // X; then q, k (D = 64: and the lo terms of the B operand)
  unsigned char t[32768];   // dO in the second half; the B operand [hi | lo] (D = 64: its hi terms)
  XGateTable gates;
  uint64_t bars[XA_BARS];
  int armed[XA_BARS];
  uint32_t tmem_slot;
  int abort;
};

template <int D>
__global__ void __launch_bounds__(256, 2)
x_adjoint_kernel(const __grid_constant__ XMaps maps, const __grid_constant__ DeltaArgs a) {
  extern __shared__ unsigned char smem_raw[];
  using Rec = XRec<D>;
  XAdjSmem<D>& sm = *reinterpret_cast<XAdjSmem<D>*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3, half = warp >> 2, row = q * 32 + lane;
  x_run<256>(sm, XA_BARS, [&](const uint32_t tmem) -> bool {
    constexpr int PANELS = D / 64;
    const int c = blockIdx.x / PANELS, eh = blockIdx.x % PANELS;
    const XPlace p = x_place(a, blockIdx.y, c);
    const unsigned char* const fwd = static_cast<const unsigned char*>(a.ws) + p.rec * Rec::FWD;
    unsigned char* const bwd = static_cast<unsigned char*>(a.ws_bwd) + p.rec * Rec::BWD;
    const uint32_t mine = (uint32_t)(q * 32) << 16, R = tmem + 128;
    if (tid == 0) {
      uint64_t* const bar = expect(sm, XA_LOAD, TRIANGLE + 16384 + 2560);
      bulk_load(&sm.gates, fwd + Rec::GATES, 2560, bar);
      load_triangle<false>(sm.x, fwd + Rec::X, bar);
      tma_load_4d(sm.t + 16384, &maps.d_o, bar, eh * 64, c * 128, p.h, p.b);
    }
    __syncwarp();
    const uint32_t go = warp == 0 ? elect_one() : 0;
    constexpr uint32_t ID1 = umma_idesc_bf16(128, 64, true, true), ID2 = umma_idesc_bf16(128, 128, true, true);
    clear_triangle<false>(sm.x, tid, 256);
    fence_proxy_async_smem();
    X_WAIT(sm.bars[XA_LOAD], 0, 80);
    const float since = ex2_approx(sm.gates.sum[row].x + sm.gates.sum[row].y);
    if (warp == 0) {
      umma_group_ss<8, false, false>(tmem, mnmaj(sm.x + 32768), mnmaj(sm.t + 16384), XHI, ID1, 0, go);
      umma_group_ss<8, false, false>(tmem, mnmaj(sm.x), mnmaj(sm.t + 16384), XHI, ID1, 1, go);
      umma_commit_if(&sm.bars[XA_MMA], go);
    }
    uint4 raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = *reinterpret_cast<const uint4*>(sm.t + 16384 + image_at(row, half * 4 + i, 128));
    X_WAIT(sm.bars[XA_MMA], 0, 81);
    if (tid == 0) {
      uint64_t* const bar = expect(sm, XA_QK, 2 * PANELS * 16384);
      for (int x = 0; x < PANELS; ++x) tma_load_4d(sm.x + x * 16384, &maps.q, bar, x * 64, c * 128, p.hk, p.b);
      for (int x = 0; x < PANELS; ++x) tma_load_4d(sm.x + (PANELS + x) * 16384, &maps.k, bar, x * 64, c * 128, p.hk, p.b);
    }
    float z[32];
    load_acc(tmem + mine + half * 32, z);
    {
      float* const to = reinterpret_cast<float*>(bwd + Rec::Z) + (size_t)(eh * 64 + half * 32) * 128 + row;
#pragma unroll
      for (int i = 0; i < 32; ++i) to[i * 128] = z[i];
    }
    unsigned char* const lo_terms = D == 128 ? sm.t + 16384 : sm.x + 32768;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
      float x[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[2 * k] = bf_lo(w[k]) * (a.scale * since), x[2 * k + 1] = bf_hi(w[k]) * (a.scale * since);
      uint4 h, l;
      split8(x, h, l);
      const uint32_t at = image_at(row, half * 4 + i, 128);
      *reinterpret_cast<uint4*>(sm.t + at) = h;
      *reinterpret_cast<uint4*>(lo_terms + at) = l;
    }
    auto put_z = [&](unsigned char* hi, unsigned char* lo) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint4 h, l;
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = -since * z[8 * i + k];
        split8(x, h, l);
        const uint32_t at = image_at(row, half * 4 + i, 128);
        *reinterpret_cast<uint4*>(hi + at) = h;
        *reinterpret_cast<uint4*>(lo + at) = l;
      }
    };
    if (D == 64) put_z(sm.t + 16384, sm.x + 49152);
    X_HAND_OVER();
    X_WAIT(sm.bars[XA_QK], 0, 82);
    if (warp == 0) {
      umma_group_ss<8, false, false>(R, mnmaj(sm.x), mnmaj(sm.t), XHI, ID2, 0, go);
      if (D == 64) umma_group_ss<8, false, false>(R, mnmaj(sm.x), mnmaj(sm.x + 32768), XHI, ID2, 1, go);
      umma_commit_if(&sm.bars[XA_MMA], go);
    }
    X_WAIT(sm.bars[XA_MMA], 1, 83);
    float* const to = reinterpret_cast<float*>(bwd + Rec::B) + (eh * 64 + half * 32) * D + (row & (D - 1));
    float x[32];
    if constexpr (D == 128) {
      put_z(sm.t, sm.t + 16384);
      X_HAND_OVER();
      if (warp == 0) {
        umma_group_ss<8, false, false>(R, mnmaj(sm.x + 32768), mnmaj(sm.t), XHI, ID2, 1, go);
        umma_commit_if(&sm.bars[XA_MMA], go);
      }
      X_WAIT(sm.bars[XA_MMA], 0, 84);
      load_both(R + mine + half * 32, x);
#pragma unroll
      for (int i = 0; i < 32; ++i) to[i * D] = x[i];
    } else {
      float(*const other)[65] = reinterpret_cast<float(*)[65]>(sm.t);
      load_acc(R + mine + (q >= 2 ? 64 : 0) + half * 32, x);
      if (q >= 2)
#pragma unroll
        for (int i = 0; i < 32; ++i) other[half * 32 + i][row - 64] = x[i];
      __syncthreads();
      if (q < 2)
#pragma unroll
        for (int i = 0; i < 32; ++i) to[i * D] = x[i] + other[half * 32 + i][row];
    }
    return true;
  });
}

// ---- values ----------------------------------------------------------------------------------------------------------------------------
// Y = That (V - diag(e^G) K S) (even thread blocks) and dR = Z + U diag(beta e^(G_end - G)) K E' (odd ones), as images; dR is dV.  Side
// by side, the two read the same K and U.  Two dependent products behind loads of 160 KB: 2048 chunks 205 us, 1 GB (45 % of HBM's rate).
enum { XV_LOAD = 0, XV_U, XV_MMA, XV_DRAIN, XV_BARS };
template <int D>
struct alignas(1024) XValSmem {
  unsigned char u[65536];  // k; then U
  unsigned char s[32768];  // [hi | lo] of the state's columns, of the bracket, of the result
  XGateTable gates;
  uint64_t bars[XV_BARS];
  int armed[XV_BARS];
  uint32_t tmem_slot;
  int abort;
};

template <int D, typename TO>
__global__ void __launch_bounds__(256, 2)
x_values_kernel(const __grid_constant__ XMaps maps, const __grid_constant__ DeltaArgs a) {
  extern __shared__ unsigned char smem_raw[];
  using Rec = XRec<D>;
  XValSmem<D>& sm = *reinterpret_cast<XValSmem<D>*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3, half = warp >> 2, row = q * 32 + lane;
  x_run<128>(sm, XV_BARS, [&](const uint32_t tmem) -> bool {
    constexpr int PANELS = D / 64, NK = D / 16;
    const bool grad = blockIdx.x & 1;
    const int c = (blockIdx.x >> 1) / PANELS, eh = (blockIdx.x >> 1) % PANELS;
    const XPlace p = x_place(a, blockIdx.y, c);
    const unsigned char* const fwd = static_cast<const unsigned char*>(a.ws) + p.rec * Rec::FWD;
    unsigned char* const bwd = static_cast<unsigned char*>(a.ws_bwd) + p.rec * Rec::BWD;
    const uint32_t mine = (uint32_t)(q * 32) << 16;
    if (tid == 0) {
      uint64_t* const bar = expect(sm, XV_LOAD, PANELS * 16384 + 2 * D * 128 + 2560);
      bulk_load(&sm.gates, fwd + Rec::GATES, 2560, bar);
      for (int x = 0; x < PANELS; ++x) tma_load_4d(sm.u + x * 16384, &maps.k, bar, x * 64, c * 128, p.hk, p.b);
      const unsigned char* const state = grad ? bwd + Rec::E : fwd + Rec::S;
      bulk_load(sm.s, state + eh * 2 * D * 128, 2 * D * 128, bar);
      unsigned nx, ny;
      if (later_block(296, nx, ny) && nx % (2 * PANELS) == 0) {
        const XPlace o = x_place(a, ny, nx / (2 * PANELS));
        for (int x = 0; x < PANELS; ++x) {
          tma_prefetch_4d(&maps.k, x * 64, nx / (2 * PANELS) * 128, o.hk, o.b);
          tma_prefetch_4d(&maps.v, x * 64, nx / (2 * PANELS) * 128, o.h, o.b);
        }
        const unsigned char* const of = static_cast<const unsigned char*>(a.ws) + o.rec * Rec::FWD;
        const unsigned char* const ob = static_cast<const unsigned char*>(a.ws_bwd) + o.rec * Rec::BWD;
        prefetch(of + Rec::S, Rec::STATE);
        prefetch_triangle<true>(of + Rec::U);
        prefetch(ob + Rec::E, Rec::STATE);
        prefetch(ob + Rec::Z, Rec::TOK);
      }
    }
    const float2 end = *reinterpret_cast<const float2*>(fwd + Rec::END);
    float add[32];
    if (grad) {
      const float* const z = reinterpret_cast<const float*>(bwd + Rec::Z) + (size_t)(eh * 64 + half * 32) * 128 + row;
#pragma unroll
      for (int i = 0; i < 32; ++i) add[i] = ld_f1(z + i * 128);
    } else {
      uint4 raw[4];
      load_raw32(static_cast<const __nv_bfloat16*>(a.v) + p.row + row * a.sT + eh * 64 + half * 32, row < p.n, raw);
      each32(raw, [&](int i, float v) { add[i] = v; });
    }
    __syncwarp();
    const uint32_t go = warp == 0 ? elect_one() : 0;
    constexpr uint32_t ID2 = umma_idesc_bf16(128, 128, false, true), ID2T = umma_idesc_bf16(128, 128, true, true);
    X_WAIT(sm.bars[XV_LOAD], 0, 90);
    const float2 own = sm.gates.sum[row];
    const float times = grad ? sm.gates.beta[row] * decay2(end, own) : -ex2_approx(own.x + own.y);
    if (warp == 0) {
      umma_group_ss<NK, true, false>(tmem, kmaj(sm.u), mnmaj(sm.s, D * 128), XHI, ID2, 0, go);
      umma_commit_if(&sm.bars[XV_MMA], go);
    }
    X_WAIT(sm.bars[XV_MMA], 0, 91);
    if (tid == 0) load_triangle<true>(sm.u, fwd + Rec::U, expect(sm, XV_U, TRIANGLE));
    clear_triangle<true>(sm.u, tid, 256);
    float x[32];
    auto put = [&]() {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint4 h, l;
        split8(&x[8 * i], h, l);
        const uint32_t at = image_at(row, half * 4 + i, 128);
        *reinterpret_cast<uint4*>(sm.s + at) = h;
        *reinterpret_cast<uint4*>(sm.s + 16384 + at) = l;
      }
    };
    load_slice(tmem + mine, half, x);
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = grad ? times * x[i] : fmaf(times, x[i], add[i]);
    put();
    X_HAND_OVER();
    X_WAIT(sm.bars[XV_U], 0, 92);
    if (warp == 0) {
      if (grad) {
        umma_group_ss<8, true, false>(tmem, kmaj(sm.u + 32768), mnmaj(sm.s), XHI, ID2, 0, go);
        umma_group_ss<8, true, false>(tmem, kmaj(sm.u), mnmaj(sm.s), XHI, ID2, 1, go);
      } else {
        umma_group_ss<8, false, false>(tmem, mnmaj(sm.u + 32768), mnmaj(sm.s), XHI, ID2T, 0, go);
        umma_group_ss<8, false, false>(tmem, mnmaj(sm.u), mnmaj(sm.s), XHI, ID2T, 1, go);
      }
      umma_commit_if(&sm.bars[XV_MMA], go);
    }
    X_WAIT(sm.bars[XV_MMA], 1, 93);
    load_both(tmem + mine + half * 32, x);
    if (grad) {
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i] += add[i];
      put_row32<TO>(sm.u, row, half * 32, x);
    }
    put();
    X_HAND_OVER();
    if (tid == 0) {
      if (grad) store_tile<TO>(&maps.dv, sm.u, eh * 64, 64, c * 128, p.h, p.b);
      unsigned char* const to = bwd + (grad ? Rec::DR : Rec::Y) + eh * 16384;
      bulk_store(to, sm.s, 16384);
      bulk_store(to + PANELS * 16384, sm.s + 16384, 16384);
      tma_store_commit();
    }
    return true;
  });
}

// ---- gradients ---------------------------------------------------------------------------------------------------------------------------
// dQ, dK, dg and dbeta of a chunk of a key head: one thread block of 512 threads, which takes the value heads of the group one after
// the other.  Thread (q, lane) of quarter w has row q * 32 + lane, columns w * 32 .. + 31 of every accumulator.
//   1  dO S^T, dR S^T, then Y E'^T                          what the states have of dQ and dK, scaled by rows; a_i, b_j, <S, E'>
//   2  Q K^T, dO Y^T, then K K^T, dR Y^T                    scores: F and -H as images; Z's sums (dg, dbeta)
//   3  dQ += F K,   dK += F^T Q - H^T K - H K               one image of each for both orientations
// Sums over columns of a chunk's [128, 128] matrix go by butterflies over the lanes (16 values, 16 shuffles); sums over s run by scans.
// 224 KB of operands come first, E' takes the place of S, q and k that of E', F and -H those of Y and dR, so that there is one thread
// block to an SM.  The order is what keeps its threads within 128 registers: with the scores first F and -H (64 registers) waited for
// the rest to be made, and what was spilled for them went to L2, since there is no L1 beside 227 KB of shared memory (480 us for 2048
// chunks; 308 now).  The tensor cores work for a quarter of it; the rest are the scores' exponentials and sums between the products, with
// no second thread block to fill them.
enum { XG_LOAD = 0, XG_E, XG_QK, XG_MMA, XG_DRAIN, XG_BARS };
template <int D>
struct alignas(1024) XGradSmem {
  unsigned char a[65536];  // S; E'; q, k
  unsigned char o[32768];  // dO; sums
  unsigned char y[65536];  // Y; F
  unsigned char s[65536];  // dR; -H
  float2 sum[128];         // the head of the gate table
  float to_last[128];
  uint64_t bars[XG_BARS];
  int armed[XG_BARS];
  uint32_t tmem_slot;
  int abort;
};
struct alignas(16) XSums {
  float beta[128], col[4][128], pre[128], rows[4][128], total[4][4];
  float a[4][128], b[4][128], a_sum[4], b_sum[4], part[16];
};

// Over the 32 lanes, sums of each of 16 values per lane: lane l returns that of value l / 2.
__device__ __forceinline__ float lane_sums16(const float (&v)[16], int lane) {
  float t[8], r[4], u[2];
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    const bool up = (lane & 16) != 0;
    t[x] = (up ? v[8 + x] : v[x]) + __shfl_xor_sync(0xffffffffu, up ? v[x] : v[8 + x], 16);
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const bool up = (lane & 8) != 0;
    r[x] = (up ? t[4 + x] : t[x]) + __shfl_xor_sync(0xffffffffu, up ? t[x] : t[4 + x], 8);
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const bool up = (lane & 4) != 0;
    u[x] = (up ? r[2 + x] : r[x]) + __shfl_xor_sync(0xffffffffu, up ? r[x] : r[2 + x], 4);
  }
  const bool up = (lane & 2) != 0;
  const float w = (up ? u[1] : u[0]) + __shfl_xor_sync(0xffffffffu, up ? u[0] : u[1], 2);
  return w + __shfl_xor_sync(0xffffffffu, w, 1);
}
// Sum over the lanes from this one on, or up to and without it
__device__ __forceinline__ float suffix_sum(float x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const float y = __shfl_down_sync(0xffffffffu, x, o);
    if (lane + o < 32) x += y;
  }
  return x;
}
__device__ __forceinline__ float prefix_sum_before(float x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const float y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  const float y = __shfl_up_sync(0xffffffffu, x, 1);
  return lane == 0 ? 0.f : y;
}
// D[tokens, features] (+)= A[tokens, e] S[features, e]^T over the e columns of a state's slices: A K-major panels of 64 columns, terms: 0 for the
// state's hi terms, 4 (16-byte groups) for the lo terms
template <int D>
__device__ __forceinline__ void state_product(uint32_t d, uint32_t a, uint32_t b, uint32_t terms, uint32_t idesc, uint32_t acc, uint32_t go) {
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
    umma_ss(d, a + umma_kstep<true>(k), b + (k >> 1) * (D * 8) + (k & 1) * 2 + terms, XHI, idesc, k > 0 || acc, go);
}

template <int D, typename TO>
__global__ void __launch_bounds__(512, 1)
x_gradient_kernel(const __grid_constant__ XMaps maps, const __grid_constant__ DeltaArgs a) {
  extern __shared__ unsigned char smem_raw[];
  using Rec = XRec<D>;
  XGradSmem<D>& sm = *reinterpret_cast<XGradSmem<D>*>(smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  XSums& sums = *reinterpret_cast<XSums*>(sm.o);
  static_assert(sizeof(XSums) <= 16384, "sums");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3, w4 = warp >> 2, row = q * 32 + lane, c0 = w4 * 32;
  x_run<512>(sm, XG_BARS, [&](const uint32_t tmem) -> bool {
    constexpr int PANELS = D / 64, NK = D / 16, TOK = 128 * D * 2;  // bytes of 128 rows of bf16, and half of their image
    constexpr uint32_t ID_SC = umma_idesc_bf16(128, 128, false, false), ID_ST = umma_idesc_bf16(128, D, false, false);
    constexpr uint32_t ID_N = umma_idesc_bf16(128, D, false, true), ID_T = umma_idesc_bf16(128, D, true, true);
    const int c = blockIdx.x, b = blockIdx.y / a.Hk, hk = blockIdx.y % a.Hk, G = a.H / a.Hk;
    const uint32_t mine = (uint32_t)(q * 32) << 16, T0 = tmem, T1 = tmem + 128, T2 = tmem + 256, T3 = tmem + 384;
    __syncwarp();
    const uint32_t go = warp == 0 ? elect_one() : 0;
    const bool feat = c0 < D;  // has columns of features
    int mma = 0, second = 0;   // parities
    unsigned char* const first = static_cast<unsigned char*>(a.ws_bwd) + ((size_t)(b * a.H + hk * G) * a.nchunk + c) * Rec::BWD;
    auto load_qk = [&](uint64_t* bar) {
      for (int x = 0; x < PANELS; ++x) tma_load_4d(sm.a + x * 16384, &maps.q, bar, x * 64, c * 128, hk, b);
      for (int x = 0; x < PANELS; ++x) tma_load_4d(sm.a + TOK + x * 16384, &maps.k, bar, x * 64, c * 128, hk, b);
    };
    for (int gh = 0; gh < G; ++gh, second ^= 1) {
      const XPlace p = x_place(a, b * a.H + hk * G + gh, c);
      const unsigned char* const fwd = static_cast<const unsigned char*>(a.ws) + p.rec * Rec::FWD;
      const unsigned char* const bwd = static_cast<const unsigned char*>(a.ws_bwd) + p.rec * Rec::BWD;
      if (tid == 0) {
        uint64_t* const bar = expect(sm, XG_LOAD, 5 * TOK + D * D * 4 + 1536);
        bulk_load(sm.a, fwd + Rec::S, D * D * 4, bar);
        for (int x = 0; x < PANELS; ++x) tma_load_4d(sm.o + x * 16384, &maps.d_o, bar, x * 64, c * 128, p.h, p.b);
        bulk_load(sm.s, bwd + Rec::DR, 2 * TOK, bar);
        bulk_load(sm.y, bwd + Rec::Y, 2 * TOK, bar);
        bulk_load(sm.sum, fwd + Rec::GATES, 1536, bar);
      }
      const XGateTable& gates = *reinterpret_cast<const XGateTable*>(fwd + Rec::GATES);
      const float2 end = *reinterpret_cast<const float2*>(fwd + Rec::END);
      const float beta_row = gates.beta[row], beta_tid = tid < 128 ? gates.beta[tid] : 0.f;
      X_WAIT(sm.bars[XG_LOAD], second, 101);
      // ---- what the states have ----
      if (warp == 0) {
        state_product<D>(T0, kmaj(sm.o), kmaj(sm.a), 4, ID_ST, 0, go);
        state_product<D>(T0, kmaj(sm.o), kmaj(sm.a), 0, ID_ST, 1, go);
        state_product<D>(T1, kmaj(sm.s + TOK), kmaj(sm.a), 0, ID_ST, 0, go);
        state_product<D>(T1, kmaj(sm.s), kmaj(sm.a), 4, ID_ST, 1, go);
        state_product<D>(T1, kmaj(sm.s), kmaj(sm.a), 0, ID_ST, 1, go);
        umma_commit_if(&sm.bars[XG_MMA], go);
      }
      if (tid == 0) {
        prefetch(bwd + Rec::E, Rec::STATE);
        for (int x = 0; x < PANELS; ++x) tma_prefetch_4d(&maps.q, x * 64, c * 128, hk, b);
        for (int x = 0; x < PANELS; ++x) tma_prefetch_4d(&maps.k, x * 64, c * 128, hk, b);
        unsigned nx, ny;
        if (gh + 1 == G && later_block(148, nx, ny)) {
          const XPlace o = x_place(a, ny / a.Hk * a.H + ny % a.Hk * G, nx);
          const unsigned char* const ob = static_cast<const unsigned char*>(a.ws_bwd) + o.rec * Rec::BWD;
          prefetch(static_cast<const unsigned char*>(a.ws) + o.rec * Rec::FWD + Rec::S, Rec::STATE);
          prefetch(ob + Rec::DR, Rec::TOK);
          prefetch(ob + Rec::Y, Rec::TOK);
          for (int x = 0; x < PANELS; ++x) tma_prefetch_4d(&maps.d_o, x * 64, nx * 128, o.h, o.b);
        }
      }
      __syncwarp();
      const float2 own = sm.sum[row];
      const float since = ex2_approx(own.x + own.y), until = decay2(end, own);
      constexpr int IT = D * D / 8 / 512;
      auto part_at = [&](int n) {  // eight columns of a row (hi terms; the lo terms are four groups further)
        const int i = tid + n * 512, r = i / 4 % D;
        return (uint32_t)(i / (4 * D) * D * 128 + r * 128 + (((i & 3) ^ (r & 7)) << 4));
      };
      uint4 sh[IT], sl[IT];  // this thread's part of S for <S, E'>
#pragma unroll
      for (int n = 0; n < IT; ++n) {
        sh[n] = *reinterpret_cast<const uint4*>(sm.a + part_at(n));
        sl[n] = *reinterpret_cast<const uint4*>(sm.a + (part_at(n) ^ 64));
      }
      X_WAIT(sm.bars[XG_MMA], mma, 102);
      mma ^= 1;
      if (tid == 0) bulk_load(sm.a, bwd + Rec::E, D * D * 4, expect(sm, XG_E, D * D * 4));
      X_WAIT(sm.bars[XG_E], second, 103);
      if (warp == 0) {
        state_product<D>(T2, kmaj(sm.y + TOK), kmaj(sm.a), 0, ID_ST, 0, go);
        state_product<D>(T2, kmaj(sm.y), kmaj(sm.a), 4, ID_ST, 1, go);
        state_product<D>(T2, kmaj(sm.y), kmaj(sm.a), 0, ID_ST, 1, go);
        umma_commit_if(&sm.bars[XG_MMA], go);
      }
      float whole = 0.f;
#pragma unroll
      for (int n = 0; n < IT; ++n) {
        float x[8], y[8];
        join8(sh[n], sl[n], x);
        join8(*reinterpret_cast<const uint4*>(sm.a + part_at(n)), *reinterpret_cast<const uint4*>(sm.a + (part_at(n) ^ 64)), y);
#pragma unroll
        for (int i = 0; i < 8; ++i) whole = fmaf(x[i], y[i], whole);
      }
      whole *= ex2_approx(end.x + end.y);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) whole += __shfl_xor_sync(0xffffffffu, whole, o);
      X_WAIT(sm.bars[XG_MMA], mma, 104);
      mma ^= 1;
      if (tid == 0) load_qk(expect(sm, XG_QK, 2 * TOK));
      X_WAIT(sm.bars[XG_QK], second, 105);
      float dot_a = 0.f, dot_b = 0.f;
      if (feat)
#pragma unroll
        for (int pc = 0; pc < 2; ++pc) {
          float x[16], y[16];
          uint4 kr[2], qr[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t at = image_at(row, w4 * 4 + pc * 2 + k, 128);
            qr[k] = *reinterpret_cast<const uint4*>(sm.a + at);
            kr[k] = *reinterpret_cast<const uint4*>(sm.a + TOK + at);
          }
          load_acc16(T0 + mine + c0 + pc * 16, x);
          tmem_ld_wait();
          each32(qr, [&](int i, float w) {
            x[i] *= a.scale * since;
            dot_a = fmaf(x[i], w, dot_a);
          });
          tmem_st_x16(T0 + mine + c0 + pc * 16, *reinterpret_cast<uint32_t(*)[16]>(&x));
          load_acc16(T1 + mine + c0 + pc * 16, x);
          load_acc16(T2 + mine + c0 + pc * 16, y);
          tmem_ld_wait();
          each32(kr, [&](int i, float w) {
            x[i] *= -since;
            dot_a = fmaf(x[i], w, dot_a);
            y[i] *= until;
            dot_b = fmaf(y[i], w, dot_b);
            x[i] = fmaf(beta_row, y[i], x[i]);
          });
          tmem_st_x16(T1 + mine + c0 + pc * 16, *reinterpret_cast<uint32_t(*)[16]>(&x));
        }
      X_HAND_OVER();
      // ---- scores ----
      if (warp == 0) {
        umma_group_ss<NK, true, true>(T2, kmaj(sm.a), kmaj(sm.a + TOK), XHI, ID_SC, 0, go);
        umma_group_ss<NK, true, true>(T3, kmaj(sm.o), kmaj(sm.y + TOK), XHI, ID_SC, 0, go);
        umma_group_ss<NK, true, true>(T3, kmaj(sm.o), kmaj(sm.y), XHI, ID_SC, 1, go);
        umma_commit_if(&sm.bars[XG_MMA], go);
      }
      X_WAIT(sm.bars[XG_MMA], mma, 106);
      mma ^= 1;
      // F, and Z without beta_j; then -H and the rest of Z (two values to an instruction where they are of another block of 32)
      uint64_t z[16];
      const float to_block = w4 < q ? decay2(own, sm.sum[c0 + 31]) : 0.f;
      if (tid < 128) sums.beta[tid] = beta_tid;  // (dO is read)
      __syncthreads();
      auto scores = [&](int pc, float times, float sign, bool diagonal, uint4(&hi)[2], uint4(&lo)[2]) {  // columns 16 pc .. + 15
        float u[16], f[16];
        load_acc16(T2 + mine + c0 + pc * 16, u);
        load_acc16(T3 + mine + c0 + pc * 16, f);
        tmem_ld_wait();
        if (w4 < q) {
          const uint64_t all = f2_pack(times * to_block, times * to_block);
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float2 d = *reinterpret_cast<const float2*>(&sm.to_last[c0 + pc * 16 + i]);
            const uint64_t v = f2_mul(f2_mul(f2_pack(d.x, d.y), all), f2_pack(f[i], f[i + 1]));
            f2_unpack(v, f[i], f[i + 1]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int n = pc * 16 + i;
            f[i] = n < lane || (diagonal && n == lane) ? f[i] * (times * decay2(own, sm.sum[c0 + n])) : 0.f;
          }
        }
        const uint64_t s2 = f2_pack(sign, sign);
        uint32_t h[8], l[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 bt = *reinterpret_cast<const float2*>(&sums.beta[c0 + pc * 16 + 2 * i]);
          const uint64_t v = f2_mul(f2_pack(f[2 * i], f[2 * i + 1]), s2);
          z[pc * 8 + i] = f2_fma(v, f2_pack(u[2 * i], u[2 * i + 1]), z[pc * 8 + i]);
          split2(f2_mul(v, f2_pack(bt.x, bt.y)), h[i], l[i]);
        }
        hi[0] = make_uint4(h[0], h[1], h[2], h[3]);
        hi[1] = make_uint4(h[4], h[5], h[6], h[7]);
        lo[0] = make_uint4(l[0], l[1], l[2], l[3]);
        lo[1] = make_uint4(l[4], l[5], l[6], l[7]);
      };
      auto put = [&](unsigned char* image, int c, const uint4& h, const uint4& l) {
        const uint32_t at = image_at(row, w4 * 4 + c, 128);
        *reinterpret_cast<uint4*>(image + at) = h;
        *reinterpret_cast<uint4*>(image + 32768 + at) = l;
      };
#pragma unroll
      for (int i = 0; i < 16; ++i) z[i] = 0;
      uint4 fh[4], fl[4];
#pragma unroll
      for (int pc = 0; pc < 2; ++pc) {
        fh[2 * pc] = fh[2 * pc + 1] = fl[2 * pc] = fl[2 * pc + 1] = make_uint4(0u, 0u, 0u, 0u);
        if (w4 <= q) scores(pc, a.scale, 1.f, true, *reinterpret_cast<uint4(*)[2]>(&fh[2 * pc]), *reinterpret_cast<uint4(*)[2]>(&fl[2 * pc]));
      }
      tc_fence_before_sync();
      __syncthreads();
      tc_fence_after_sync();
      if (warp == 0) {
        umma_group_ss<NK, true, true>(T2, kmaj(sm.a + TOK), kmaj(sm.a + TOK), XHI, ID_SC, 0, go);
        umma_group_ss<NK, true, true>(T3, kmaj(sm.s + TOK), kmaj(sm.y), XHI, ID_SC, 0, go);
        umma_group_ss<NK, true, true>(T3, kmaj(sm.s), kmaj(sm.y + TOK), XHI, ID_SC, 1, go);
        umma_group_ss<NK, true, true>(T3, kmaj(sm.s), kmaj(sm.y), XHI, ID_SC, 1, go);
        umma_commit_if(&sm.bars[XG_MMA], go);
      }
      X_WAIT(sm.bars[XG_MMA], mma, 107);
      mma ^= 1;
      // (Y and dR are read) F and -H as images
#pragma unroll
      for (int k = 0; k < 4; ++k) put(sm.y, k, fh[k], fl[k]);
#pragma unroll
      for (int pc = 0; pc < 2; ++pc) {
        uint4 h[2], l[2];
        h[0] = h[1] = l[0] = l[1] = make_uint4(0u, 0u, 0u, 0u);
        if (w4 <= q) scores(pc, 1.f, -1.f, false, h, l);
        put(sm.s, 2 * pc, h[0], l[0]);
        put(sm.s, 2 * pc + 1, h[1], l[1]);
      }
      // The last products are issued by a warp whose scores are above the diagonal, so that it has no part in Z: an issuing warp waits as long
      // as its products run, here 4100 clocks, and the others sum up Z meanwhile, at a barrier of their own.
      sums.a[w4][row] = dot_a;
      sums.b[w4][row] = dot_b;
      if (lane == 0) sums.part[warp] = whole;
      if (warp == X_ISSUER) {
        sums.rows[w4][row] = 0.f;
        sums.col[q][c0 + lane] = 0.f;
        if (lane == 0) sums.total[w4][q] = 0.f;
      }
      X_HAND_OVER();
      if (warp == X_ISSUER) {
        const uint32_t go = elect_one();
        const unsigned char *const qt = sm.a, *const kt = sm.a + TOK;
#pragma unroll
        for (int term = 1; term >= 0; --term) {
          umma_group_ss<8, true, false>(T0, kmaj(sm.y + term * 32768), mnmaj(kt), XHI, ID_N, 1, go);
          umma_group_ss<8, false, false>(T1, mnmaj(sm.y + term * 32768), mnmaj(qt), XHI, ID_T, 1, go);
          umma_group_ss<8, false, false>(T1, mnmaj(sm.s + term * 32768), mnmaj(kt), XHI, ID_T, 1, go);
          umma_group_ss<8, true, false>(T1, kmaj(sm.s + term * 32768), mnmaj(kt), XHI, ID_N, 1, go);
        }
        umma_commit_if(&sm.bars[XG_MMA], go);
      } else {
        // ---- dg, dbeta meanwhile, in dO's place.  For s in block b of 32: of Z's rows i >= s and columns j < s those of row blocks after b
        // and column blocks before b as sums of whole blocks, the others of one or the other as scans of rows' or columns' sums, and those
        // of block b in both as the sums over rows i >= s of what a row has before s.
        float row_sum = 0.f;
#pragma unroll
        for (int pc = 0; pc < 2; ++pc) {
          float v[16], u[16];
#pragma unroll
          for (int i = 0; i < 8; ++i) f2_unpack(z[pc * 8 + i], v[2 * i], v[2 * i + 1]);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            u[i] = lane >= pc * 16 + i ? row_sum : 0.f;
            row_sum = fmaf(sums.beta[c0 + pc * 16 + i], v[i], row_sum);
          }
          if (w4 == q) {
            const float pre = lane_sums16(u, lane);
            if ((lane & 1) == 0) sums.pre[c0 + pc * 16 + (lane >> 1)] = pre;
          }
          const float col = w4 <= q ? lane_sums16(v, lane) : 0.f;
          if ((lane & 1) == 0) sums.col[q][c0 + pc * 16 + (lane >> 1)] = col;
        }
        sums.rows[w4][row] = row_sum;
        asm volatile("bar.sync 1, 480;" ::: "memory");
        float ai = 0.f, bi = 0.f, dbeta = 0.f, dg = 0.f;
        if (tid < 128) {  // token tid, in block `warp`
          ai = (sums.a[0][tid] + sums.a[1][tid]) + (sums.a[2][tid] + sums.a[3][tid]);
          bi = (sums.b[0][tid] + sums.b[1][tid]) + (sums.b[2][tid] + sums.b[3][tid]);
          dbeta = bi;
          bi *= beta_tid;
          float left = 0.f, below = 0.f;  // of row tid the column blocks before its own, of column tid the row blocks after it
          for (int w = 0; w < warp; ++w) left += sums.rows[w][tid];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float col = sums.col[x][tid];
            dbeta += col;
            if (x > warp) below += col;
          }
          below *= beta_tid;
          ai = suffix_sum(ai, lane);
          const float b_before = prefix_sum_before(bi, lane);
          dg = sums.pre[tid] + suffix_sum(left, lane) + prefix_sum_before(below, lane);
          if (lane == 0) sums.a_sum[warp] = ai;
          if (lane == 31) sums.b_sum[warp] = b_before + bi;
          bi = b_before;
        }
        {  // sums of whole blocks
          const float x = suffix_sum(row_sum, lane);
          if (lane == 0) sums.total[w4][q] = x;
        }
        asm volatile("bar.sync 1, 480;" ::: "memory");
        if (tid < p.n && tid < 128) {
          float w = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) w += sums.part[i];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (i > warp) {
              ai += sums.a_sum[i];
              for (int k = 0; k < warp; ++k) dg += sums.total[k][i];
            }
            if (i < warp) bi += sums.b_sum[i];
          }
          a.dg[p.gate + tid * a.gT] = w + ((dg + ai) + bi);
          a.dbeta[p.gate + tid * a.gT] = dbeta;
        }
      }
      X_WAIT(sm.bars[XG_MMA], mma, 111);
      mma ^= 1;
      // ---- dQ, dK; of a group of heads the sum so far is kept where Y and dR of its first head were ----
      if (feat)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          float x[32];
          load_acc((which ? T1 : T0) + mine + c0, x);
          float* const kept = reinterpret_cast<float*>(first + (which ? Rec::Y : Rec::DR)) + (size_t)c0 * 128 + row;
          if (gh > 0)
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] += kept[i * 128];
          if (gh + 1 < G) {
#pragma unroll
            for (int i = 0; i < 32; ++i) kept[i * 128] = x[i];
          } else {
            put_row32<TO>(which ? sm.s : sm.y, row, c0, x);
          }
        }
      X_HAND_OVER();
      if (tid == 0 && gh + 1 == G) {
        store_tile<TO>(&maps.dq, sm.y, 0, D, c * 128, hk, b);
        store_tile<TO>(&maps.dk, sm.s, 0, D, c * 128, hk, b);
        tma_store_commit();
      }
    }
    return true;
  });
}

// ---- launches ----------------------------------------------------------------------------------------------------------------------------
bool make_token_map(CUtensorMap* m, const void* ptr, const DeltaArgs& a, bool shared, bool f32 = false) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return false;
  const cuuint64_t esz = f32 ? 4 : 2;
  cuuint64_t dims[4] = {(cuuint64_t)a.D, (cuuint64_t)a.N, (cuuint64_t)(shared ? a.Hk : a.H), (cuuint64_t)a.B};
  cuuint64_t strides[3] = {(cuuint64_t)(shared ? a.sTk : a.sT) * esz, (cuuint64_t)(shared ? a.sHk : a.sH) * esz, (cuuint64_t)(shared ? a.sBk : a.sB) * esz};
  cuuint32_t box[4] = {(cuuint32_t)(128 / esz), 128, 1, 1}, es[4] = {1, 1, 1, 1};
  return enc(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename SM, typename K, typename... A>
cudaError_t x_launch(K kern, int kind, dim3 grid, int threads, cudaStream_t stream, const A&... args) {
  constexpr size_t smem = sizeof(SM) + 1024;
  static_assert(smem <= 232448, "shared memory of a thread block");
  cudaError_t err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (err != cudaSuccess) return err;
  KernelTimer timer(kind, stream);
  err = launch_early(kern, grid, dim3((unsigned)threads), smem, stream, 1, args...);
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}

// Thread blocks with 32 value columns each as long as they all run at once (one to an SM), else with 64: 32 heads of 128 features, 64
// chunks each, 125 us with 32 columns and 173 with 64.
template <int D, bool REV>
cudaError_t x_chain(const DeltaArgs& d, cudaStream_t stream) {
  using Rec = XRec<D>;
  XChainArgs a{};
  a.fwd = static_cast<const unsigned char*>(d.ws);
  a.fwd_stride = Rec::FWD;
  unsigned char* const bwd = static_cast<unsigned char*>(d.ws_bwd);
  a.add = REV ? bwd + Rec::B : a.fwd + Rec::N;
  a.image = REV ? bwd + Rec::E : static_cast<unsigned char*>(d.ws) + Rec::S;
  a.add_stride = a.image_stride = REV ? Rec::BWD : Rec::FWD;
  a.in = REV ? d.grad_kv_out : d.kv_in;
  a.out = REV ? d.grad_kv_in : d.kv_out;
  a.nchunk = d.nchunk;
  const int heads = d.B * d.H;
  if (heads * (D / 32) <= 148)
    return x_launch<XChainSmem<D, 32>>(x_chain_kernel<D, 32, REV>, K_SCAN, dim3(D / 32, heads), 256, stream, a);
  return x_launch<XChainSmem<D, 64>>(x_chain_kernel<D, 64, REV>, K_SCAN, dim3(D / 64, heads), 256, stream, a);
}

template <int D>
cudaError_t x_states(const XMaps& m, const DeltaArgs& a, cudaStream_t stream) {
  const cudaError_t err = x_launch<XPrepSmem<D>>(x_prepare_kernel<D>, K_PREPASS, dim3(a.nchunk, a.B * a.H), 512, stream, m, a);
  return err != cudaSuccess ? err : x_chain<D, false>(a, stream);
}

template <int D, typename TO>
cudaError_t x_fwd(const DeltaArgs& a, cudaStream_t stream) {
  XMaps m{};
  if (!make_token_map(&m.q, a.q, a, true) || !make_token_map(&m.k, a.k, a, true) || !make_token_map(&m.v, a.v, a, false) ||
      !make_token_map(&m.o, a.o, a, false, sizeof(TO) == 4))
    return cudaErrorInvalidValue;
  const cudaError_t err = x_states<D>(m, a, stream);
  if (err != cudaSuccess) return err;
  return x_launch<XOutSmem<D>>(x_output_kernel<D, TO>, K_WALK, dim3(a.nchunk * (D / 64), a.B * a.H), 256, stream, m, a);
}

template <int D, typename TO>
cudaError_t x_bwd(const DeltaArgs& a, bool have_fwd, cudaStream_t stream) {
  XMaps m{};
  constexpr bool F32 = sizeof(TO) == 4;
  if (!make_token_map(&m.q, a.q, a, true) || !make_token_map(&m.k, a.k, a, true) || !make_token_map(&m.v, a.v, a, false) ||
      !make_token_map(&m.d_o, a.d_o, a, false) || !make_token_map(&m.dq, a.dq, a, true, F32) || !make_token_map(&m.dk, a.dk, a, true, F32) ||
      !make_token_map(&m.dv, a.dv, a, false, F32))
    return cudaErrorInvalidValue;
  cudaError_t err = have_fwd ? cudaSuccess : x_states<D>(m, a, stream);
  if (err == cudaSuccess)
    err = x_launch<XAdjSmem<D>>(x_adjoint_kernel<D>, K_PREPASS, dim3(a.nchunk * (D / 64), a.B * a.H), 256, stream, m, a);
  if (err == cudaSuccess) err = x_chain<D, true>(a, stream);
  if (err == cudaSuccess)
    err = x_launch<XValSmem<D>>(x_values_kernel<D, TO>, K_WALK, dim3(a.nchunk * (D / 64) * 2, a.B * a.H), 256, stream, m, a);
  if (err == cudaSuccess) err = x_launch<XGradSmem<D>>(x_gradient_kernel<D, TO>, K_WALK_PAIR, dim3(a.nchunk, a.B * a.Hk), 512, stream, m, a);
  return err;
}

#undef X_WAIT
#undef X_HAND_OVER
