// Blocks of the history: their mean keys, and the choice of the blocks that a block of queries attends to.
//
//   m_{h,b} = 1 / n_b sum_{t in b} k_{h,t}                     n_b tokens of block b
//   s_{h,i,b} = (sum_{t in query block i} q_{h,t}) . m_{h,b}   and the top_k blocks b of the largest s
//
// The choice is that of 64-bit scores, but 64-bit arithmetic runs at a sixtieth of the 32-bit rate here.  So all scores
// are taken in 32 bits, with a bound E on their error, and only the candidates that lie within 2 E of the top_k-th
// largest 32-bit score T are scored again in 64 bits: a score above T + 2 E is among the top_k whatever the roundings
// were, one below T - 2 E is not, because the top_k-th largest of the true scores lies within E of T.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "pdl.cuh"
#include "ptx.cuh"
#include "rows.cuh"

namespace ispa {

namespace {

// ------------------------------------------------------------ mean keys
constexpr int M_THREADS = 128;

// Sixteen e4m3 codes as fp32.
__device__ __forceinline__ void add16(const uint4& w, float* s) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t h2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(static_cast<uint16_t>(u[i >> 1] >> (16 * (i & 1)))));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h2));
    s[2 * i] += f.x;
    s[2 * i + 1] += f.y;
  }
}

// A block of the grid: block blockIdx.x of the frames' blocks, head blockIdx.y.  A row's LPR lanes take 16 bytes each,
// eight rows apart on their way at once.  HBM bounds it: the 455 MB of 57 frames of 1560 tokens x 40 heads in 8 bits,
// blocks of 128, in 78 us, 6.0 TB/s with the means' 15 MB (89 % of the copy rate; issue slots 74 %).
template <bool E4M3, int D>
__global__ void __launch_bounds__(M_THREADS) means_kernel(const __grid_constant__ MeansParams p) {
  constexpr int VALS = E4M3 ? 16 : 8, LPR = D / VALS, ROWS = M_THREADS / LPR;
  __shared__ float part[M_THREADS / 32][D];
  const int h = blockIdx.y;
  const int64_t frame = p.first_frame + blockIdx.x / p.nb;
  const int b = blockIdx.x % p.nb;
  const int slot = static_cast<int>(frame < p.n_sink ? frame : p.n_sink + (frame - p.n_sink) % (p.capacity - p.n_sink));
  const int n = min(p.block, p.P - b * p.block);
  const int lane = threadIdx.x % LPR;
  pdl_wait();
  pdl_trigger();
  const uint4* from = static_cast<const uint4*>(p.k) +
                      ((static_cast<int64_t>(h) * p.capacity + slot) * p.P + static_cast<int64_t>(b) * p.block) * LPR +
                      lane;
  float s[VALS];
#pragma unroll
  for (int e = 0; e < VALS; ++e) s[e] = 0.f;
  for (int r0 = threadIdx.x / LPR; r0 < n; r0 += 8 * ROWS) {
    uint4 w[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      w[u] = r0 + u * ROWS < n ? __ldg(from + static_cast<int64_t>(r0 + u * ROWS) * LPR) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if constexpr (E4M3) {
        add16(w[u], s);
      } else {
        float f[8];
        unpack8(w[u], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += f[e];
      }
    }
  }
#pragma unroll
  for (int o = LPR; o < 32; o *= 2)
#pragma unroll
    for (int e = 0; e < VALS; ++e) s[e] += __shfl_xor_sync(0xffffffffu, s[e], o);
  const int warp = threadIdx.x / 32;
  if (threadIdx.x % 32 < LPR) {
#pragma unroll
    for (int e = 0; e < VALS; ++e) part[warp][lane * VALS + e] = s[e];
  }
  __syncthreads();
  const int c = threadIdx.x;
  if (c < D) {
    float v = part[0][c];
#pragma unroll
    for (int i = 1; i < M_THREADS / 32; ++i) v += part[i][c];
    v = __fdiv_rn(v, static_cast<float>(n));
    if (E4M3) v *= __ldg(p.k_scale + h);
    p.means[((static_cast<int64_t>(h) * p.capacity + slot) * p.nb + b) * D + c] = v;
  }
}

// ------------------------------------------------------------ selection
// Three kernels: sums of the queries, 32-bit scores, the choice.  4680 queries x 12 heads over 1250 candidates: 21 us
// where reading once takes 3.3; the launches' latency bounds it (each a launch's own 2 us and a chain of loads, passes
// and barriers; issue slots 50 to 60 %).  Few candidates or one query block: one kernel, one query 7.6 us
// (select_kernel); one query block and few heads: two, the sum in the scoring one.
// Workspace: per head and query block the sum of the queries (hi, and lo with the rest); room for 64-bit scores, the
// 32-bit scores, the sum's norm, and a bound on what hi + lo is off by; per head and tile of candidates the largest
// norm of a mean.  hi and lo are multiples of 256 bytes, so that hi's rows can be read by 16 bytes and what follows
// lies on its 8 and 4.
struct SelectWs {
  float* hi;          // [H][n_qt][d]
  float* lo;
  double* exact;      // [H][n_qt][n_cand]
  float* score;       // [H][n_qt][n_cand]
  float* norm;        // [H][n_qt]
  float* lost;        // [H][n_qt]
  float* largest;     // [H][tiles]
};
__host__ __device__ __forceinline__ SelectWs ws_of(void* ws, int64_t H, int64_t n_qt, int64_t d, int64_t n_cand) {
  SelectWs w;
  w.hi = static_cast<float*>(ws);
  w.lo = w.hi + H * n_qt * d;
  w.exact = reinterpret_cast<double*>(w.lo + H * n_qt * d);
  w.score = reinterpret_cast<float*>(w.exact + H * n_qt * n_cand);
  w.norm = w.score + H * n_qt * n_cand;
  w.lost = w.norm + H * n_qt;
  w.largest = w.lost + H * n_qt;
  return w;
}

// Block number of a candidate.  The runs behind the last one end at INT32_MAX.
__device__ __forceinline__ int id_of(const SelectParams& p, int cand) {
  int shift = p.run_shift[ISPA_MAX_RANGES - 1];
#pragma unroll
  for (int r = ISPA_MAX_RANGES - 2; r >= 0; --r)
    if (cand < p.run_end[r]) shift = p.run_shift[r];
  return cand + shift;
}

// hi + lo = the sum of hi and x, hi rounded to nearest (Knuth's TwoSum); lo collects.
__device__ __forceinline__ void two_sum(float& hi, float& lo, float x) {
  const float s = __fadd_rn(hi, x), t = __fsub_rn(s, hi);
  lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(s, t)), __fsub_rn(x, t)));
  hi = s;
}

// The same of 2^-7 x, whose products are exact, two at a time.
__device__ __forceinline__ void two_sum_7(float2& hi, float2& lo, float2 x) {
  const float2 c = make_float2(0.0078125f, 0.0078125f), minus = make_float2(-1.f, -1.f);
  const float2 s = fma2(c, x, hi), t = fma2(minus, s, hi);   // t: -2^-7 x, as far as s has it
  lo = add2(lo, add2(fma2(minus, add2(s, t), hi), fma2(c, x, t)));
  hi = s;
}

// Of two bf16 values each the larger magnitude; its sign has no meaning.
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Sum of a query block's queries of one head, by THREADS threads: rows over the threads, then over the block.  Of 2^-7
// of the queries, exact for every bf16 value, so that the sum of finite ones stays finite; the order of the scores is
// the same.  Feature c's sum (hi, lo) to thread c < D, hi the rounded sum of both whatever cancelled on the way; a
// barrier has passed since the last use of `part` by others.
//
// TwoSum is exact, so hi + lo is off by the roundings of lo alone.  With Y the largest |2^-7 q| and steps of 2^-24 Y:
// the k-th sum of a thread's N rows is at most k Y, and its lo takes a residue of k steps; the block's k-th sum is at
// most N k Y, and its lo takes a residue of N k steps and then a thread's lo of N (N + 1) / 2.  So the lo's stay below
// (N k (k + 1) + N (N + 1) k) / 2 steps, and both additions round to 2^-24 of that: over k <= ROWS, with the threads'
// own, 2^-33.4 Y for N = 8 and 2^-32.1 Y for N = 4.  lost_of: 2^-32 sqrt(D) Y for all features, twice, for the
// roundings of 64-bit scores (below 2^-37 sqrt(D) Y |m|).
template <int D>
__device__ __forceinline__ float lost_of(float y) {
  return (D == 128 ? 11.5f : 8.f) * 4.6566129e-10f * y;
}
template <int D, int THREADS>
struct QSum {
  static constexpr int LPR = D / 8, ROWS = THREADS / LPR;
  static constexpr int N = kSelectQueries / ROWS;   // rows of a thread, all on their way at once
  static_assert(ROWS >= 16 && ROWS <= 32, "lost_of's partial sums");
  float2 part[ROWS][LPR * 9];   // a lane's eight 9 apart: 16 lanes to as many pairs of banks
  float top[THREADS / 32];      // the largest magnitude that a warp read (NaN aside, with which the sum is NaN)
  __device__ __forceinline__ float2 of(const SelectParams& p, int h, int qt) {
    const int lane = threadIdx.x % LPR, r0 = threadIdx.x / LPR;
    const int n = min(kSelectQueries, p.n_q - qt * kSelectQueries);
    const int64_t row = static_cast<int64_t>(p.H) * LPR;
    const uint4* from = reinterpret_cast<const uint4*>(p.q) + (static_cast<int64_t>(qt) * kSelectQueries) * row +
                        h * LPR + lane;
    uint4 w[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int r = r0 + u * ROWS;
      w[u] = r < n ? __ldg(from + r * row) : make_uint4(0, 0, 0, 0);
    }
    float2 hi[4], lo[4] = {};
    uint32_t most = 0;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      float f[8];
      unpack8(w[u], f);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 x = make_float2(f[2 * e], f[2 * e + 1]);
        if (u == 0) hi[e] = make_float2(0.0078125f * x.x, 0.0078125f * x.y);
        else two_sum_7(hi[e], lo[e], x);
      }
      most = larger2(larger2(most, w[u].x), larger2(w[u].y, larger2(w[u].z, w[u].w)));
    }
    const float own = fmaxf(fabsf(__uint_as_float(most << 16)), fabsf(__uint_as_float(most & 0xffff0000u)));
    const float of_warp = warp_max(own);
    if ((threadIdx.x & 31) == 0) top[threadIdx.x / 32] = of_warp;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      part[r0][lane * 9 + 2 * e] = make_float2(hi[e].x, lo[e].x);
      part[r0][lane * 9 + 2 * e + 1] = make_float2(hi[e].y, lo[e].y);
    }
    __syncthreads();
    float a = 0.f, b = 0.f;
    if (threadIdx.x < D) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        if (r >= n) break;
        const float2 v = part[r][threadIdx.x + threadIdx.x / 8];
        two_sum(a, b, v.x);
        b += v.y;
      }
    }
    float rest = 0.f;
    if (fabsf(a) < INFINITY) two_sum(a, rest, b);
    return make_float2(a, rest);
  }
};
// A norm for the bound from a sum of at most 128 squares: what those lose below fp32's normal range, 2^-150 each and as
// much in their additions, is at most 2^-142, and the root of a sum at most the sum of the roots.
__device__ __forceinline__ float norm_of(float squares) { return sqrtf(squares) + 4.2351647e-22f; }   // 2^-71

// The sum to the workspace, with its norm and lost_of; all threads of the block.
template <int D, int THREADS>
__device__ __forceinline__ void keep_sum(const SelectWs& ws, int64_t list, float2 v, const QSum<D, THREADS>& sum,
                                         float (*red)[32]) {
  if (threadIdx.x < D) {
    ws.hi[list * D + threadIdx.x] = v.x;
    ws.lo[list * D + threadIdx.x] = v.y;
  }
  const float s = block_reduce<SumOp>(threadIdx.x < D ? v.x * v.x : 0.f, THREADS / 32, red, 0);
  if (threadIdx.x == 0) {
    ws.norm[list] = norm_of(s);
    float y = sum.top[0];
#pragma unroll
    for (int i = 1; i < THREADS / 32; ++i) y = fmaxf(y, sum.top[i]);
    ws.lost[list] = lost_of<D>(0.0078125f * y);
  }
}

// Registers of three blocks an SM, so that a row's eight words are all on their way: 37 query blocks of 12 heads over
// 1250 candidates 21.0 us in all, of 40 heads over 650 32.5; of four 22.1 and 33.8.
constexpr int Q_THREADS = 256;
template <int D>
__global__ void __launch_bounds__(Q_THREADS, 3) qsum_kernel(const __grid_constant__ SelectParams p) {
  __shared__ QSum<D, Q_THREADS> sum;
  __shared__ float red[2][32];
  const int qt = blockIdx.x, h = blockIdx.y;
  pdl_wait();
  pdl_trigger();
  const float2 v = sum.of(p, h, qt);
  keep_sum(ws_of(p.ws, p.H, p.n_qt, D, p.n_cand), static_cast<int64_t>(h) * p.n_qt + qt, v, sum, red);
}

// 32-bit scores: a tile of 64 candidates x 8 J query blocks of one head in shared memory, 2 x J a thread.  A warp's
// lanes read 16 candidates' words and two query blocks' at a time, with J = 5 in 9 cycles of shared memory for 10 of
// products; J = 3 for 17 to 24 query blocks, where 5 takes 1 us more for 12 heads x 1250.  OWN: one query block, whose
// sum every block of the grid takes for itself.  BLOCKS: that an SM is to hold; with the registers of two (122 where
// three leave 80) the rows are read further ahead.  In all, 37 query blocks of 12 heads x 1250, a grid of 240 blocks:
// 21.2 us with two, 24.0 with three, 24.1 without a bound; of 40 heads x 650, 440 blocks: 32.8, 32.5 and 32.7; 74 query
// blocks of 40 heads 61.2, 60.0 and 60.4.
constexpr int S_CAND = 64, S_THREADS = 256;
template <int D, int J>
constexpr int kScoreSmem = (S_CAND + 8 * J) * (D + 4) * 4;
__device__ __forceinline__ void copy16(uint32_t dst, const float4* src, bool here) {   // else zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(here ? 16 : 0) : "memory");
}
template <int D, int J, bool OWN, int BLOCKS>
__global__ void __launch_bounds__(S_THREADS, BLOCKS) score_kernel(const __grid_constant__ SelectParams p) {
  static_assert(!OWN || J == 1, "one query block");
  constexpr int LD = D + 4, QT = 8 * J, VPR = D / 4;   // rows 4 banks apart; a row's float4
  extern __shared__ float4 tile[];
  float* const m = reinterpret_cast<float*>(tile);   // [S_CAND][LD]
  float* const q = m + S_CAND * LD;                  // [QT][LD]
  __shared__ float red[2][32];
  const int c0 = blockIdx.x * S_CAND, h = blockIdx.y;
  const SelectWs ws = ws_of(p.ws, p.H, p.n_qt, D, p.n_cand);
  // Behind qsum_kernel this starts when all its blocks have the kernels before behind them, so the means can be read
  // while it works.
  if constexpr (OWN) pdl_wait();
  const uint32_t m_at = smem_u32(m), q_at = smem_u32(q);
  const float4* const means = reinterpret_cast<const float4*>(p.means) + h * p.ids * VPR;
  {
    constexpr int ROWS = S_THREADS / VPR, N = S_CAND / ROWS;   // rows at a time; one lane looks up one number
    const int r0 = threadIdx.x / VPR, c = threadIdx.x % VPR, lane = threadIdx.x & 31;
    const int id = id_of(p, min(c0 + r0 + lane % N * ROWS, p.n_cand - 1));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = r0 + i * ROWS;
      const bool here = c0 + r < p.n_cand;
      const int64_t row = __shfl_sync(0xffffffffu, id, lane / VPR * VPR + i);
      copy16(m_at + (r * LD + 4 * c) * 4, means + (here ? row * VPR + c : 0), here);
    }
  }
  if constexpr (!OWN) pdl_wait();
  pdl_trigger();
  if constexpr (OWN) {
    __shared__ QSum<D, S_THREADS> sum;
    const float2 v = sum.of(p, h, 0);
    if (threadIdx.x < D) q[threadIdx.x] = v.x;
#pragma unroll
    for (int i = threadIdx.x; i < 7 * D; i += S_THREADS) q[(1 + i / D) * LD + i % D] = 0.f;
    if (blockIdx.x == 0) keep_sum(ws, h, v, sum, red);
  }
  // candidates tc + 32 i, query blocks tq + 8 j: a warp has 16 of the one and two of the other
  const int tc = threadIdx.x % 16 + 16 * (threadIdx.x / 128), tq = threadIdx.x / 16 % 8;
  for (int q0 = blockIdx.z * QT; q0 < p.n_qt; q0 += gridDim.z * QT) {
    const int rows = min(QT, p.n_qt - q0);
    if constexpr (!OWN) {
      const float4* from = reinterpret_cast<const float4*>(ws.hi + (static_cast<int64_t>(h) * p.n_qt + q0) * D);
      if (q0 > static_cast<int>(blockIdx.z) * QT) __syncthreads();
#pragma unroll
      for (int i = threadIdx.x; i < QT * VPR; i += S_THREADS) {
        const bool here = i < rows * VPR;
        copy16(q_at + (i / VPR * LD + 4 * (i % VPR)) * 4, from + (here ? i : 0), here);
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    float2 acc[2][J] = {};
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
      float4 a[2], b[J];
#pragma unroll
      for (int i = 0; i < 2; ++i) a[i] = *reinterpret_cast<const float4*>(m + (tc + 32 * i) * LD + c);
#pragma unroll
      for (int j = 0; j < J; ++j) b[j] = *reinterpret_cast<const float4*>(q + (tq + 8 * j) * LD + c);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j)
          acc[i][j] = fma2(make_float2(a[i].z, a[i].w), make_float2(b[j].z, b[j].w),
                           fma2(make_float2(a[i].x, a[i].y), make_float2(b[j].x, b[j].y), acc[i][j]));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (c0 + tc + 32 * i < p.n_cand && tq + 8 * j < rows)
          ws.score[(static_cast<int64_t>(h) * p.n_qt + q0 + tq + 8 * j) * p.n_cand + c0 + tc + 32 * i] =
              acc[i][j].x + acc[i][j].y;
  }
  if (blockIdx.z > 0) return;
  // the largest of the tile's norms: four threads a mean
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    const float4 v = *reinterpret_cast<const float4*>(m + threadIdx.x / 4 * LD + 4 * (4 * c + threadIdx.x % 4));
    s = fmaf(v.x, v.x, fmaf(v.y, v.y, fmaf(v.z, v.z, fmaf(v.w, v.w, s))));
  }
  s = block_reduce<MaxOp>(group_reduce<SumOp>(s, 4), S_THREADS / 32, red, 1);
  if (threadIdx.x == 0) ws.largest[h * gridDim.x + blockIdx.x] = norm_of(s);
}

// Keys whose order as integers is that of the scores; both zeros alike, NaN below all.
__device__ __forceinline__ uint32_t order_key(float f) {
  if (f != f) return 0;
  const uint32_t u = __float_as_uint(f + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t order_key(double f) {
  if (f != f) return 0;
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(f + 0.0));
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ float score_of(uint32_t key) {   // of any key but NaN's
  return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key);
}
__device__ __forceinline__ double score_of(uint64_t key) {
  return __longlong_as_double(static_cast<long long>(key >> 63 ? key & ~(uint64_t{1} << 63) : ~key));
}

constexpr int kFew = 64;   // candidates that are ranked one against one

template <int W>
struct PickShared {
  int4 hist[2][64];           // 256 counts, of the highest digit first; used in turn
  uint32_t list[kFew];
  uint32_t lo[W], hi[W];
  float norms[W];
  uint64_t counts[2][W];
  int few[kFew];
  uint64_t few_key[3][kFew], few_least;   // of the score, and of where scores near it begin and end
  int n_list, n_few, few_ties, few_close;
  int wide[258];
  double sum[128];            // of the queries, in 64 bits
};

// Two counts in a word: their sum over the warps before this one, and over all.
template <int W>
__device__ __forceinline__ uint64_t warps_before(uint64_t* of, uint64_t v, uint64_t& all) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  uint64_t s = 0;
  all = v;
  if constexpr (W > 1) {
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) of[warp] = v;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const uint64_t x = of[w];
      if (w < warp) s += x;
      all += x;
    }
  }
  return s;
}

// Of 256 counts, of the highest digit first: the digit where they add up to k, how many lie above it, how many at it.
// Every warp by itself.
__device__ __forceinline__ int digit_of(const int4* hist, int k, int& above, int& at) {
  const int lane = threadIdx.x & 31;
  const int4 x = hist[2 * lane], y = hist[2 * lane + 1];
  const int v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  int sum = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) sum += v[j];
  int before = sum;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const int u = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += u;
  }
  const int from = __ffs(__ballot_sync(0xffffffffu, before >= k)) - 1;
  before -= sum;
  int digit = 0, n = 0, b = before;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (b < k) digit = 8 * lane + j, before = b, n = v[j];
    b += v[j];
  }
  above = __shfl_sync(0xffffffffu, before, from);
  at = __shfl_sync(0xffffffffu, n, from);
  return 255 - __shfl_sync(0xffffffffu, digit, from);
}

// The k-th largest (1 <= k <= how many count) of the 64-bit keys key(i), i < n, among those with live(i), and how many
// of those equal to it are among the k largest.  Digit by digit from the top.
template <int THREADS, typename Get, typename Live>
__device__ uint64_t kth_largest(int n, int k, Get&& key, Live&& live, int* hist, int& ties) {
  uint64_t known = 0;
#pragma unroll 1
  for (int shift = 56; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += THREADS) hist[i] = 0;
    __syncthreads();
    const uint64_t above = shift == 56 ? 0 : ~uint64_t{0} << (shift + 8);
    for (int i = threadIdx.x; i < n; i += THREADS) {
      if (!live(i)) continue;
      const uint64_t x = key(i);
      if ((x & above) == known) atomicAdd(hist + (x >> shift & 255), 1);
    }
    __syncthreads();
    if (threadIdx.x < 32) {   // the digit where the count from the top reaches k; hist[256..257] carry it out
      int sum = 0, mine[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += mine[j] = hist[255 - (8 * threadIdx.x + j)];
      int before = sum;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const int v = __shfl_up_sync(0xffffffffu, before, o);
        if (static_cast<int>(threadIdx.x) >= o) before += v;
      }
      before -= sum;
      if (before < k && before + sum >= k) {
        int j = 0;
        while (before + mine[j] < k) before += mine[j++];
        hist[256] = 255 - (8 * threadIdx.x + j);
        hist[257] = before;
      }
    }
    __syncthreads();
    known |= static_cast<uint64_t>(hist[256]) << shift;
    k -= hist[257];
  }
  __syncthreads();
  ties = k;
  return known;
}

// The sum that QSum takes, a feature a thread, as three floats, whose sum has all 53 bits of a double.  Not inlined and
// short: almost no list needs it, and what it takes (20 us where a list does) is less than its registers and code would
// cost the others.
template <int D, int THREADS>
__device__ __noinline__ void sum_again(const SelectParams& p, int h, int qt, double* sum) {
  const int n = min(kSelectQueries, p.n_q - qt * kSelectQueries);
  const int64_t row = static_cast<int64_t>(p.H) * D;
  for (int c = threadIdx.x; c < D; c += THREADS) {
    const __nv_bfloat16* from = p.q + static_cast<int64_t>(qt) * kSelectQueries * row + h * D + c;
    float hi = 0.f, mid = 0.f, lo = 0.f;
#pragma unroll 4
    for (int r = 0; r < n; ++r) {
      float x = 0.f, y = 0.f;
      two_sum(hi, x, 0.0078125f * __bfloat162float(from[r * row]));
      two_sum(mid, y, x);
      lo += y;
    }
    sum[c] = fabsf(hi) < INFINITY ? static_cast<double>(hi) + (static_cast<double>(mid) + static_cast<double>(lo)) : hi;
  }
}

// One block of W warps a list.  Warp w takes the candidates from w 32 steps on, a step of 32 neighbours at a time.
// PER: the steps, with their keys in registers; 0: any number, read again for each pass.  Latency bounds it (the passes
// over the keys, with a barrier each): 1250 candidates in two warps 3 us longer than in eight.
template <int W>
__device__ __forceinline__ void pick_begin(PickShared<W>& sh) {   // a barrier follows before pick
#pragma unroll
  for (int i = threadIdx.x; i < 128; i += 32 * W) sh.hist[i / 64][i % 64] = make_int4(0, 0, 0, 0);
  if (threadIdx.x == 0) sh.n_list = sh.n_few = 0;
}
template <int D, int W, int PER>
__device__ __forceinline__ void pick(const SelectParams& p, PickShared<W>& sh, int h, int64_t list, const float* norms,
                                     int n_norms) {
  constexpr int THREADS = 32 * W;
  const int n = p.n_cand, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  int32_t* const out = p.blocks + list * p.top_k;
  const SelectWs ws = ws_of(p.ws, p.H, p.n_qt, D, n);
  const float* score = ws.score + list * n;
  double* exact = ws.exact + list * n;
  const int steps = PER ? PER : (n + THREADS - 1) / THREADS, first = warp * 32 * steps + lane;
  float f[PER ? PER : 1];
  if constexpr (PER != 0) {
#pragma unroll
    for (int j = 0; j < PER; ++j) f[j] = first + 32 * j < n ? __ldcg(score + first + 32 * j) : 0.f;
  }
  const float q_norm = __ldcg(ws.norm + list), lost = __ldcg(ws.lost + list);
  float m_norm = 0.f;
  for (int i = threadIdx.x; i < n_norms; i += THREADS) m_norm = max_nan(m_norm, __ldcg(norms + i));
  uint32_t keys[PER ? PER : 1];
  if constexpr (PER != 0) {
#pragma unroll
    for (int j = 0; j < PER; ++j) keys[j] = order_key(f[j]);
  }
  const auto each = [&](auto&& f) {   // f(candidate, key, there is one), all lanes alike
    if constexpr (PER != 0) {
#pragma unroll
      for (int j = 0; j < PER; ++j) f(first + 32 * j, keys[j], first + 32 * j < n);
    } else {
#pragma unroll 1
      for (int j = 0; j < steps; j += 8) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int i = first + 32 * (j + u);
          x[u] = j + u < steps && i < n ? __ldcg(score + i) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int i = first + 32 * (j + u);
          f(i, order_key(x[u]), j + u < steps && i < n);
        }
      }
    }
  };
  // T, the top_k-th largest 32-bit score, by counts.
  uint32_t lo = 0xffffffffu, hi = 0;
  each([&](int, uint32_t x, bool here) {
    if (here) lo = min(lo, x), hi = max(hi, x);
  });
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  m_norm = warp_max(m_norm);
  if (W > 1 && lane == 0) sh.lo[warp] = lo, sh.hi[warp] = hi, sh.norms[warp] = m_norm;
  __syncthreads();
  if constexpr (W > 1) {
#pragma unroll
    for (int w = 0; w < W; ++w) {
      lo = min(lo, sh.lo[w]);
      hi = max(hi, sh.hi[w]);
      m_norm = max_nan(m_norm, sh.norms[w]);
    }
  }
  int bits = 32 - __clz(lo ^ hi);                       // of the keys, not known yet
  uint32_t known = bits == 32 ? 0 : hi >> bits << bits;
  int k = p.top_k, left = n;                            // wanted and there among those that it can be
  // 256 steps of one size from the smallest to the largest: mostly few candidates are in the one that T is in.  (The
  // keys' digits, which differ little in front, made their lanes wait for one another's counts.)
  const float base = score_of(lo), scale = 256.f / (score_of(hi) - base);
  const auto step_of = [&](uint32_t x) {                // never smaller for a larger key
    return max(0, min(255, static_cast<int>((score_of(x) - base) * scale)));
  };
  int step = -1;                                        // that T is in, if it is known so
  if (left > kFew && bits > 0 && lo && fabsf(base) < INFINITY && score_of(hi) < INFINITY) {
    each([&](int, uint32_t x, bool here) {
      if (here) atomicAdd(reinterpret_cast<int*>(sh.hist[0]) + (255 - step_of(x)), 1);
    });
    __syncthreads();
    int above, at;
    const int s = digit_of(sh.hist[0], k, above, at);
    if (at <= kFew) {
      step = s;
      k -= above;
      left = at;
    } else {
      __syncthreads();
#pragma unroll
      for (int i = threadIdx.x; i < 64; i += THREADS) sh.hist[0][i] = make_int4(0, 0, 0, 0);
      __syncthreads();
    }
  }
  // Else its key digit by digit, from the highest of the bits that the keys do not share, until few have the digits
  // found so far.
  const auto among = [&](uint32_t x) { return bits == 32 || x - known < 1u << bits; };
  for (int turn = 0; bits > 0 && left > kFew; ++turn) {
    int4* const hist = sh.hist[turn & 1];
    const int shift = max(0, bits - 8);
    each([&](int, uint32_t x, bool here) {
      if (here && among(x)) atomicAdd(reinterpret_cast<int*>(hist) + (255 - ((x - known) >> shift)), 1);
    });
    __syncthreads();
    int above;
    known |= static_cast<uint32_t>(digit_of(hist, k, above, left)) << shift;
    k -= above;
    bits = shift;
    if (turn > 0 && bits > 0 && left > kFew) {          // the other counts, which all have read
#pragma unroll
      for (int i = threadIdx.x; i < 64; i += THREADS) sh.hist[(turn & 1) ^ 1][i] = make_int4(0, 0, 0, 0);
      __syncthreads();
    }
  }
  // Those are ranked one against one.
  uint32_t t_key = known;
  if (bits > 0) {
    if (step >= 0) {
      each([&](int, uint32_t x, bool here) {
        if (here && step_of(x) == step) sh.list[atomicAdd(&sh.n_list, 1)] = x;
      });
    } else {
      each([&](int, uint32_t x, bool here) {
        if (here && among(x)) sh.list[atomicAdd(&sh.n_list, 1)] = x;
      });
    }
    __syncthreads();
    // every warp by itself: of a lane's two, one that less than k are above of and k or more at or above
    const uint32_t a = lane < left ? sh.list[lane] : 0, b = lane + 32 < left ? sh.list[lane + 32] : 0;
    int a_above = 0, a_at = 0, b_above = 0, b_at = 0;
    for (int i = 0; i < left; ++i) {
      const uint32_t x = sh.list[i];
      a_above += x > a;
      a_at += x >= a;
      b_above += x > b;
      b_at += x >= b;
    }
    const bool a_is = lane < left && a_above < k && a_at >= k, b_is = lane + 32 < left && b_above < k && b_at >= k;
    const uint32_t found = __ballot_sync(0xffffffffu, a_is || b_is);
    t_key = __shfl_sync(0xffffffffu, a_is ? a : b, __ffs(found) - 1);
  }
  // The bound: a product's sum in 32 bits over d terms is off by at most (d + 1) 2^-24 |q| |m| (Cauchy-Schwarz; q's
  // rounding to 32 bits among it), besides what the sum of the queries has lost and what underflows, 2^-150 a product;
  // the other 23 steps are for the roundings of |q|, |m| and of T +- 2 E.
  const float E = ((D + 24) * 5.9604645e-8f * q_norm + lost) * m_norm + 1.1754944e-38f;
  const float T = t_key ? score_of(t_key) : INFINITY;
  // without a finite bound everything is scored again
  const bool bounded = E < INFINITY && fabsf(T) < INFINITY;
  const float low = T - 2.f * E - 2.5e-7f * fabsf(T), high = T + 2.f * E + 2.5e-7f * fabsf(T);
  const uint32_t low_key = bounded ? order_key(low) : 0, high_key = bounded ? order_key(high) : 0xffffffffu;
  // sure: key above high_key; open: from low_key to high_key
  uint32_t n_sure = 0, n_in = 0;
  each([&](int, uint32_t x, bool here) {
    n_sure += here && x > high_key;
    n_in += here && x >= low_key;
  });
  uint64_t all;
  const uint64_t before = warps_before<W>(sh.counts[0], static_cast<uint64_t>(n_sure) << 32 | n_in, all);
  const int need = p.top_k - static_cast<int>(all >> 32);   // of the open ones
  const int n_open = static_cast<int>(all) - static_cast<int>(all >> 32);
  const uint32_t lower_lanes = (1u << lane) - 1u;
  int at = static_cast<int>(before);
  if (need >= n_open) {   // all of them
    each([&](int i, uint32_t x, bool here) {
      const bool in = here && x >= low_key;
      const uint32_t mask = __ballot_sync(0xffffffffu, in);
      if (in) out[at + __popc(mask & lower_lanes)] = id_of(p, i);
      at += __popc(mask);
    });
    return;
  }
  // 64-bit scores, a warp a candidate, every one's terms in the same order.  First of hi + lo: where another score lies
  // so near the last one taken that what the sum has lost could turn them round, then of the queries' sum in 64 bits
  // (at once where no bound holds or many are open).
  uint64_t least;   // open candidates are taken above this key, `ties` of those at it
  int ties;
  double q[D / 32];
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    const int64_t c = list * D + lane + 32 * j;
    q[j] = static_cast<double>(ws.hi[c]) + static_cast<double>(ws.lo[c]);
  }
  const auto score64 = [&](int cand) {
    const float* m = p.means + (h * p.ids + id_of(p, cand)) * D + lane;
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) s = fma(q[j], static_cast<double>(__ldg(m + 32 * j)), s);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
  };
  const double apart = 2.0 * static_cast<double>(lost) * m_norm;
  if (n_open <= kFew) {
    each([&](int i, uint32_t x, bool here) {
      if (here && x >= low_key && x <= high_key) sh.few[atomicAdd(&sh.n_few, 1)] = i;
    });
  }
#pragma unroll 1
  for (bool in64 = !bounded || n_open > kFew;; in64 = true) {
    if (in64) sum_again<D, THREADS>(p, h, static_cast<int>(list - static_cast<int64_t>(h) * p.n_qt), sh.sum);
    __syncthreads();
    if (in64) {
#pragma unroll
      for (int j = 0; j < D / 32; ++j) q[j] = sh.sum[lane + 32 * j];
    }
    if (n_open > kFew) {
      const auto open = [&](int i) {
        const uint32_t x = order_key(__ldcg(score + i));
        return x >= low_key && x <= high_key;
      };
      for (int i = warp; i < n; i += W)
        if (open(i)) {
          const double s = score64(i);
          if (lane == 0) exact[i] = s;
        }
      __syncthreads();
      least = kth_largest<THREADS>(n, need, [&](int i) { return order_key(exact[i]); }, open, sh.wide, ties);
      break;
    }
    for (int i = warp; i < n_open; i += W) {
      const double s = score64(sh.few[i]);
      if (lane < 3) sh.few_key[lane][i] = order_key(s + (lane == 0 ? 0.0 : lane == 1 ? -apart : apart));
      if (lane == 0) exact[sh.few[i]] = s;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n_open; i += THREADS) {   // those that less than `need` are above of, and so on
      const uint64_t x = sh.few_key[0][i], from = sh.few_key[1][i], to = sh.few_key[2][i];
      int ahead = 0, equal = 0, near = 0;
      for (int j = 0; j < n_open; ++j) {
        const uint64_t y = sh.few_key[0][j];
        ahead += y > x;
        equal += y == x;
        near += y >= from && y <= to;
      }
      if (ahead < need && ahead + equal >= need) {   // equal ones write the same
        sh.few_least = x;
        sh.few_ties = need - ahead;
        sh.few_close = near > 1;
      }
    }
    __syncthreads();
    least = sh.few_least;
    ties = sh.few_ties;
    if (in64 || !sh.few_close) break;   // the next turn's first barrier is behind these reads
  }
  // In the order of their numbers: the sure ones, the open ones above `least` and the first `ties` of those at it.
  const auto key64 = [&](int i, uint32_t x, bool here) {   // 0: not in question (a NaN's, too, where `least` is more)
    return !here || x < low_key ? 0 : x > high_key ? ~uint64_t{0} : order_key(exact[i]);
  };
  const auto asked = [&](uint32_t x, bool here) { return here && x >= low_key; };
  uint32_t n_above = 0, n_tied = 0;
  each([&](int i, uint32_t x, bool here) {
    const uint64_t e = key64(i, x, here);
    n_above += asked(x, here) && e > least;
    n_tied += asked(x, here) && e == least;
  });
  const uint64_t ahead = warps_before<W>(sh.counts[1], static_cast<uint64_t>(n_tied) << 32 | n_above, all);
  int tied = static_cast<int>(ahead >> 32);   // ties before this step
  at = static_cast<int>(ahead) + min(tied, ties);
  each([&](int i, uint32_t x, bool here) {
    const uint64_t e = key64(i, x, here);
    const bool tie = asked(x, here) && e == least;
    const uint32_t tie_mask = __ballot_sync(0xffffffffu, tie);
    const bool in = asked(x, here) && (e > least || (tie && tied + __popc(tie_mask & lower_lanes) < ties));
    const uint32_t mask = __ballot_sync(0xffffffffu, in);
    if (in) out[at + __popc(mask & lower_lanes)] = id_of(p, i);
    at += __popc(mask);
    tied += __popc(tie_mask);
  });
}

template <int D, int W, int PER>
__global__ void __launch_bounds__(32 * W) pick_kernel(const __grid_constant__ SelectParams p) {
  __shared__ PickShared<W> sh;
  const int h = blockIdx.y, n = p.n_cand;
  const int64_t list = static_cast<int64_t>(h) * p.n_qt + blockIdx.x;
  pick_begin(sh);
  pdl_wait();
  pdl_trigger();
  if (n <= p.top_k) {   // everything there is
    int32_t* const out = p.blocks + list * p.top_k;
    for (int i = threadIdx.x; i < p.top_k; i += 32 * W) out[i] = i < n ? id_of(p, i) : -1;
    return;
  }
  const int tiles = (n + S_CAND - 1) / S_CAND;
  pick<D, W, PER>(p, sh, h, list, ws_of(p.ws, p.H, p.n_qt, D, n).largest + h * tiles, tiles);
}

// All in one launch, for few candidates or one query block: a cluster a list, every CTA with the queries' sum and its
// share of the candidates, a warp eight means at a time and as many on their way; then the first CTA chooses.  Latency
// bounds it (sum, means, the cluster's barrier, the choice's passes).  1250 candidates of 12 heads: one query 7.6 us
// where two launches take 9.8, 128 queries 8.2 (10.7); one query of 40 heads 10.2 (18.1).  Block numbers looked up by
// every lane instead of one took 1.4 us more.
constexpr int O_WARPS = 8, O_THREADS = 32 * O_WARPS, O_BATCH = 8;
template <int D, int PER>
__global__ void __launch_bounds__(O_THREADS) select_kernel(const __grid_constant__ SelectParams p) {
  constexpr int V = D / 32;   // features of a lane
  using Vec = std::conditional_t<V == 4, float4, float2>;
  __shared__ PickShared<O_WARPS> sh;
  __shared__ QSum<D, O_THREADS> sum;
  __shared__ __align__(16) float q_sum[D];
  __shared__ float red[2][32];
  const int rank = static_cast<int>(cluster_ctarank()), c = static_cast<int>(gridDim.x);
  const int h = blockIdx.y / p.n_qt, qt = blockIdx.y % p.n_qt;
  const int64_t list = blockIdx.y;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, n = p.n_cand;
  pick_begin(sh);
  pdl_wait();
  pdl_trigger();
  const SelectWs ws = ws_of(p.ws, p.H, p.n_qt, D, n);
  float* const norms = reinterpret_cast<float*>(ws.exact + list * n);   // [c], read before exact is written
  const Vec* const means = reinterpret_cast<const Vec*>(p.means) + h * p.ids * 32 + lane;
  const int step = c * O_WARPS * O_BATCH;
  Vec here[O_BATCH], next[O_BATCH];   // two batches on their way
  const auto load = [&](Vec (&m)[O_BATCH], int c0) {
    const int id = id_of(p, min(c0 + lane % O_BATCH, n - 1));
#pragma unroll
    for (int i = 0; i < O_BATCH; ++i) {
      const int64_t row = __shfl_sync(0xffffffffu, id, i);
      m[i] = c0 + i < n ? __ldg(means + row * 32) : Vec{};
    }
  };
  int c0 = (rank * O_WARPS + warp) * O_BATCH;
  load(here, c0);
  load(next, c0 + step);
  const float2 v = sum.of(p, h, qt);
  if (threadIdx.x < D) q_sum[threadIdx.x] = v.x;
  if (rank == 0) keep_sum(ws, list, v, sum, red);
  __syncthreads();
  const Vec qv = reinterpret_cast<const Vec*>(q_sum)[lane];
  float largest = 0.f;
  const auto batch = [&](Vec (&m)[O_BATCH]) {
    float s[2 * O_BATCH];   // products, then squares
#pragma unroll
    for (int i = 0; i < O_BATCH; ++i) {
      if constexpr (V == 4) {
        s[i] = fmaf(m[i].x, qv.x, fmaf(m[i].y, qv.y, fmaf(m[i].z, qv.z, m[i].w * qv.w)));
        s[O_BATCH + i] = fmaf(m[i].x, m[i].x, fmaf(m[i].y, m[i].y, fmaf(m[i].z, m[i].z, m[i].w * m[i].w)));
      } else {
        s[i] = fmaf(m[i].x, qv.x, m[i].y * qv.y);
        s[O_BATCH + i] = fmaf(m[i].x, m[i].x, m[i].y * m[i].y);
      }
    }
    load(m, c0 + 2 * step);
    // each lane sends half of its sums on at every step and keeps the others: lanes 2 i and 2 i + 1 end with sum i
#pragma unroll
    for (int half = O_BATCH; half > 0; half /= 2) {
      const bool up = lane & (2 * half);
#pragma unroll
      for (int i = 0; i < half; ++i) {
        const float give = up ? s[i] : s[i + half], keep = up ? s[i + half] : s[i];
        s[i] = keep + __shfl_xor_sync(0xffffffffu, give, 2 * half);
      }
    }
    s[0] += __shfl_xor_sync(0xffffffffu, s[0], 1);
    const int i = lane / 2;
    if (i < O_BATCH) {
      if (lane % 2 == 0 && c0 + i < n) ws.score[list * n + c0 + i] = s[0];
    } else {
      largest = max_nan(largest, s[0]);
    }
    c0 += step;
  };
#pragma unroll 1
  while (c0 < n) {
    batch(here);
    if (c0 < n) batch(next);
  }
  largest = block_reduce<MaxOp>(largest, O_WARPS, red, 1);
  if (threadIdx.x == 0) norms[rank] = norm_of(largest);
  cluster_sync();   // the scores are there
  if (rank == 0) pick<D, O_WARPS, PER>(p, sh, h, list, norms, c);
}

int sm_count() {
  int dev = 0, sms = 152;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}

template <int D>
cudaError_t select_d(const SelectParams& p, cudaStream_t s) {
  const int n = p.n_cand;
  // One launch where an SM's share of the means is small; us in one launch, in three in brackets.  128 features: 1024
  // queries of 12 heads, shares of 125, 400 and 700, 8.4 (11.6), 12.9 (12.0), 15.5 (12.8); 4680 queries of 12 heads,
  // 438, 511 and 949, 15.9 (18.0), 16.0 (18.2), 22.6 (18.6); 512 of 3 heads, 300 and 603, 14.5 (14.2), 16.1 (13.7);
  // 300 of 40, 450 and 650, 13.8 (15.5), 15.8 (16.9).  64 features: 1024 queries of 12 heads, 200, 325 and 500, 7.0
  // (8.0), 8.9 (8.3), 13.4 (11.4); 4680 of 12, 175 and 350, 10.7 (14.0), 8.4 (10.7).  One query block, which all of
  // the scoring kernel's blocks would add up, but for few heads too: one query over 4825 candidates of 12 heads 15.6
  // (two launches 21.1), of 7 14.7 (17.0), of 3 14.6 (12.6), of one 14.4 (10.1).
  const int sms = sm_count(), wanted = (n + O_WARPS * O_BATCH - 1) / (O_WARPS * O_BATCH);
  const int64_t items = static_cast<int64_t>(p.H) * p.n_qt;
  const int c = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({8, sms / items, wanted})));
  const int64_t share = std::max<int64_t>(n / c, n * items / sms);   // n >= 2: it keeps the grid's y below 65536
  if (n > p.top_k && (share <= (D == 128 ? 450 : 200) || (p.n_qt == 1 && 3 * items * c >= sms))) {
    const auto one = [&](auto kernel) {
      const dim3 grid(static_cast<unsigned>(c), static_cast<unsigned>(items));
      return launch_pdl_cluster(kernel, grid, dim3(O_THREADS), 0, c, s, p);
    };
    return n <= 256 ? one(select_kernel<D, 1>) : n <= 1280 ? one(select_kernel<D, 5>)
         : n <= 2560 ? one(select_kernel<D, 10>) : n <= 5120 ? one(select_kernel<D, 20>)
         : one(select_kernel<D, 0>);
  }
  const dim3 lists(static_cast<unsigned>(p.n_qt), static_cast<unsigned>(p.H));
  if (p.n_cand > p.top_k) {
    const int64_t tiles = (n + S_CAND - 1) / S_CAND;
    // Query blocks by groups of 8 J: one after the other in a block of the grid, or side by side where that leaves the
    // blocks that the SMs hold: 1250 candidates of 4 heads, 9344 queries 20.2 us in all, else 24.5; of 2 heads, 18720
    // queries 19.6, else 35.0; of 12 heads the same both ways.
    const auto score = [&](auto j, auto own) {
      constexpr int J = decltype(j)::value;
      const int64_t groups = (p.n_qt + 8 * J - 1) / (8 * J);
      const int64_t z = std::max<int64_t>(1, std::min<int64_t>(groups, 4 * sms / (tiles * p.H)));
      const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(p.H), static_cast<unsigned>(z));
      const auto with = [&](auto kernel) {
        const cudaError_t e = set_smem_limit_once(reinterpret_cast<const void*>(kernel), kScoreSmem<D, J>);
        return e != cudaSuccess ? e : launch_pdl(kernel, grid, dim3(S_THREADS), kScoreSmem<D, J>, s, p);
      };
      if constexpr (J >= 3)
        if (tiles * p.H * z <= 2 * sms) return with(score_kernel<D, J, false, 2>);
      return with(score_kernel<D, J, decltype(own)::value, 3>);
    };
    cudaError_t e = p.n_qt == 1 ? cudaSuccess : launch_pdl(qsum_kernel<D>, lists, dim3(Q_THREADS), 0, s, p);
    if (e != cudaSuccess) return e;
    using std::integral_constant;
    e = p.n_qt == 1    ? score(integral_constant<int, 1>(), std::true_type())
        : p.n_qt <= 8  ? score(integral_constant<int, 1>(), std::false_type())
        : p.n_qt <= 16 ? score(integral_constant<int, 2>(), std::false_type())
        : p.n_qt <= 24 ? score(integral_constant<int, 3>(), std::false_type())
        : p.n_qt <= 32 ? score(integral_constant<int, 4>(), std::false_type())
                       : score(integral_constant<int, 5>(), std::false_type());
    if (e != cudaSuccess) return e;
  }
  const auto pick = [&](auto kernel, int warps) { return launch_pdl(kernel, lists, dim3(32 * warps), 0, s, p); };
  return n <= 128    ? pick(pick_kernel<D, 1, 4>, 1)
         : n <= 768  ? pick(pick_kernel<D, 4, 6>, 4)
         : n <= 1280 ? pick(pick_kernel<D, 8, 5>, 8)
         : n <= 2560 ? pick(pick_kernel<D, 8, 10>, 8)
         : n <= 5120 ? pick(pick_kernel<D, 8, 20>, 8)
                     : pick(pick_kernel<D, 8, 0>, 8);
}

}  // namespace

cudaError_t launch_key_means(const MeansParams& p, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>(p.units), static_cast<unsigned>(p.H));
  if (p.k_scale) return launch_pdl(means_kernel<true, 128>, grid, dim3(M_THREADS), 0, s, p);
  if (p.d == 128) return launch_pdl(means_kernel<false, 128>, grid, dim3(M_THREADS), 0, s, p);
  return launch_pdl(means_kernel<false, 64>, grid, dim3(M_THREADS), 0, s, p);
}

size_t select_ws_bytes(int64_t H, int64_t n_qt, int64_t d, int64_t ids) {
  if (static_cast<double>(H) * n_qt * (ids + d) > 1e17) return 0;   // far past any memory, and no overflow below
  return static_cast<size_t>(H) * (n_qt * ids * 12 + n_qt * d * 8 + n_qt * 8 + (ids + S_CAND - 1) / S_CAND * 4);
}

cudaError_t launch_select(const SelectParams& p, cudaStream_t s) {
  return p.d == 128 ? select_d<128>(p, s) : select_d<64>(p, s);
}

}  // namespace ispa
