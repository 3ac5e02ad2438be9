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

// A block of the grid: block blockIdx.x of the frames' blocks, head blockIdx.y.  A row's LPR lanes take 16 bytes each.
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
                      ((static_cast<int64_t>(h) * p.capacity + slot) * p.P + static_cast<int64_t>(b) * p.block) * LPR + lane;
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
// Workspace: per head and query block the sum of the queries as two floats a feature, then per head, query block and
// candidate the 32-bit score, per head and candidate the mean's norm, and room for 64-bit scores.
struct SelectWs {
  float2* qsum;    // [H][n_qt][d]
  double* exact;   // [H][n_qt][n_cand]
  float* score;    // [H][n_qt][n_cand]
  float* norm;     // [H][n_cand]
};
__host__ __device__ __forceinline__ SelectWs ws_of(void* ws, int64_t H, int64_t n_qt, int64_t d, int64_t n_cand) {
  SelectWs w;
  w.qsum = static_cast<float2*>(ws);
  w.exact = reinterpret_cast<double*>(w.qsum + H * n_qt * d);
  w.score = reinterpret_cast<float*>(w.exact + H * n_qt * n_cand);
  w.norm = w.score + H * n_qt * n_cand;
  return w;
}

__device__ __forceinline__ int id_of(const SelectParams& p, int cand) {
  int r = 0;
  while (r + 1 < p.n_runs && cand >= p.run_end[r]) ++r;
  return cand + p.run_shift[r];
}

// hi + lo = the sum of a and b, hi rounded to nearest (Knuth's TwoSum); lo collects.
__device__ __forceinline__ void two_sum(float& hi, float& lo, float x) {
  const float s = __fadd_rn(hi, x), t = __fsub_rn(s, hi);
  lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(s, t)), __fsub_rn(x, t)));
  hi = s;
}

// Sum of a query block's queries of one head: rows over the threads, then over the block.  Of 2^-7 of the queries, exact
// for every bf16 value, so that the sum of finite ones stays finite; the order of the scores is the same.
template <int D>
__global__ void __launch_bounds__(256) qsum_kernel(const __grid_constant__ SelectParams p) {
  constexpr int LPR = D / 8, ROWS = 256 / LPR;
  __shared__ float2 part[ROWS][D];
  const int qt = blockIdx.x, h = blockIdx.y, lane = threadIdx.x % LPR, r0 = threadIdx.x / LPR;
  const int n = min(kSelectQueries, p.n_q - qt * kSelectQueries);
  pdl_wait();
  pdl_trigger();
  const int64_t row = static_cast<int64_t>(p.H) * LPR;
  const uint4* from = reinterpret_cast<const uint4*>(p.q) + (static_cast<int64_t>(qt) * kSelectQueries) * row +
                      h * LPR + lane;
  float hi[8] = {}, lo[8] = {};
  uint4 w[kSelectQueries / ROWS];
#pragma unroll
  for (int u = 0; u < kSelectQueries / ROWS; ++u)
    w[u] = r0 + u * ROWS < n ? __ldg(from + (r0 + u * ROWS) * row) : make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int u = 0; u < kSelectQueries / ROWS; ++u) {
    float f[8];
    unpack8(w[u], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) two_sum(hi[e], lo[e], 0.0078125f * f[e]);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) part[r0][lane * 8 + e] = make_float2(hi[e], lo[e]);
  __syncthreads();
  const int c = threadIdx.x;
  if (c < D) {
    float a = part[0][c].x, b = part[0][c].y;
    for (int r = 1; r < ROWS; ++r) {
      two_sum(a, b, part[r][c].x);
      b += part[r][c].y;
    }
    const SelectWs ws = ws_of(p.ws, p.H, p.n_qt, D, p.n_cand);
    ws.qsum[(static_cast<int64_t>(h) * p.n_qt + qt) * D + c] = make_float2(a, fabsf(a) < INFINITY ? b : 0.f);
  }
}

// 32-bit scores: a tile of 64 candidates x 32 query blocks of one head, 2 x 4 a thread.
constexpr int S_CAND = 64, S_QT = 32;
template <int D>
__global__ void __launch_bounds__(256) score_kernel(const __grid_constant__ SelectParams p) {
  extern __shared__ float4 sm4[];
  float* const m = reinterpret_cast<float*>(sm4);   // [S_CAND][D + 4]
  float* const q = m + S_CAND * (D + 4);            // [S_QT][D + 4]
  const int c0 = blockIdx.x * S_CAND, h = blockIdx.y;
  const SelectWs ws = ws_of(p.ws, p.H, p.n_qt, D, p.n_cand);
  pdl_wait();
  pdl_trigger();
  for (int i = threadIdx.x; i < S_CAND * (D / 4); i += 256) {
    const int r = i / (D / 4), c = i % (D / 4);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c0 + r < p.n_cand)
      v = __ldg(reinterpret_cast<const float4*>(p.means + (h * p.ids + id_of(p, c0 + r)) * D) + c);
    *reinterpret_cast<float4*>(m + r * (D + 4) + 4 * c) = v;
  }
  const int tc = threadIdx.x % 16, tq = threadIdx.x / 16;   // candidates tc + 16 i, query blocks tq + 16 j
  for (int q0 = 0; q0 < p.n_qt; q0 += S_QT) {
    __syncthreads();
    for (int i = threadIdx.x; i < S_QT * D; i += 256) {
      const int r = i / D, c = i % D;
      q[r * (D + 4) + c] = q0 + r < p.n_qt ? ws.qsum[(static_cast<int64_t>(h) * p.n_qt + q0 + r) * D + c].x : 0.f;
    }
    __syncthreads();
    float acc[4][2] = {};
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
      float4 a[4], b[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(m + (tc + 16 * i) * (D + 4) + c);
#pragma unroll
      for (int j = 0; j < 2; ++j) b[j] = *reinterpret_cast<const float4*>(q + (tq + 16 * j) * (D + 4) + c);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[i][j] = fmaf(a[i].w, b[j].w, fmaf(a[i].z, b[j].z, fmaf(a[i].y, b[j].y, fmaf(a[i].x, b[j].x, acc[i][j]))));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (c0 + tc + 16 * i < p.n_cand && q0 + tq + 16 * j < p.n_qt)
          ws.score[(static_cast<int64_t>(h) * p.n_qt + q0 + tq + 16 * j) * p.n_cand + c0 + tc + 16 * i] = acc[i][j];
  }
  if (threadIdx.x < S_CAND && c0 + threadIdx.x < p.n_cand) {
    float s = 0.f;
    for (int c = 0; c < D; ++c) {
      const float v = m[threadIdx.x * (D + 4) + c];
      s = fmaf(v, v, s);
    }
    ws.norm[static_cast<int64_t>(h) * p.n_cand + c0 + threadIdx.x] = sqrtf(s);
  }
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
__device__ __forceinline__ float score_of(uint32_t key) {   // of the last key but NaN's: finite or infinite
  return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key);
}

constexpr int P_THREADS = 256, P_WARPS = P_THREADS / 32;
constexpr int kFew = 64;   // candidates that are ranked one against one

// The k-th largest (1 <= k <= how many count) of the keys key(i), i < n, among those with live(i), and how many of
// those equal to it are among the k largest.  Digit by digit from the top.
template <typename Key, typename Get, typename Live>
__device__ Key kth_largest(int n, int k, Get&& key, Live&& live, int* hist, int& ties) {
  Key known = 0;
#pragma unroll 1
  for (int shift = 8 * sizeof(Key) - 8; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += P_THREADS) hist[i] = 0;
    __syncthreads();
    const Key above = shift == 8 * static_cast<int>(sizeof(Key)) - 8 ? Key{0} : ~Key{0} << (shift + 8);
    for (int i = threadIdx.x; i < n; i += P_THREADS) {
      if (!live(i)) continue;
      const Key x = key(i);
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
    known |= static_cast<Key>(hist[256]) << shift;
    k -= hist[257];
  }
  __syncthreads();
  ties = k;
  return known;
}

// One block a list.
template <int D>
__global__ void __launch_bounds__(P_THREADS) pick_kernel(const __grid_constant__ SelectParams p) {
  __shared__ int hist[258];
  __shared__ float red[2][32];
  __shared__ int counts[2][P_WARPS + 2];
  __shared__ int few[kFew];
  __shared__ uint64_t few_key[kFew], few_least;
  __shared__ int n_few, above_window;
  const int qt = blockIdx.x, h = blockIdx.y, n = p.n_cand, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int64_t list = static_cast<int64_t>(h) * p.n_qt + qt;
  int32_t* const out = p.blocks + list * p.top_k;
  pdl_wait();
  pdl_trigger();
  if (n <= p.top_k) {   // everything there is
    for (int i = threadIdx.x; i < p.top_k; i += P_THREADS) out[i] = i < n ? id_of(p, i) : -1;
    return;
  }
  const SelectWs ws = ws_of(p.ws, p.H, p.n_qt, D, n);
  const float* score = ws.score + list * n;
  const float2* qs = ws.qsum + list * D;
  double* exact = ws.exact + list * n;

  // The bound: a product's sum in 32 bits over d terms is off by at most (d + 2) 2^-24 |q| |m| (Cauchy-Schwarz; q's
  // rounding to 32 bits among it); the rest covers the roundings of |q|, |m| and of T +- 2 E themselves, 2^-126
  // products that underflow.
  float mm = 0.f, qq = 0.f;
  for (int i = threadIdx.x; i < n; i += P_THREADS) mm = max_nan(mm, ws.norm[static_cast<int64_t>(h) * n + i]);
  if (threadIdx.x < D) qq = qs[threadIdx.x].x * qs[threadIdx.x].x;
  mm = block_reduce<MaxOp>(mm, P_WARPS, red, 0);
  qq = block_reduce<SumOp>(qq, P_WARPS, red, 1);
  const float E = (D + 24) * 5.9604645e-8f * sqrtf(qq) * mm + 1.1754944e-38f;

  int ties;
  const auto key = [&](int i) { return order_key(score[i]); };
  const uint32_t t_key = kth_largest<uint32_t>(n, p.top_k, key, [](int) { return true; }, hist, ties);
  const float T = score_of(t_key);
  // without a finite bound everything is scored again
  const bool bounded = E < INFINITY && fabsf(T) < INFINITY;
  const float low = T - 2.f * E - 1e-6f * fabsf(T) * 0.25f, high = T + 2.f * E + 1e-6f * fabsf(T) * 0.25f;
  const auto sure = [&](int i) { return bounded && score[i] > high; };
  const auto open = [&](int i) { return !bounded || (score[i] >= low && score[i] <= high); };
  if (threadIdx.x == 0) n_few = above_window = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += P_THREADS) {
    if (sure(i)) atomicAdd(&above_window, 1);
    else if (open(i)) {
      const int at = atomicAdd(&n_few, 1);
      if (at < kFew) few[at] = i;
    }
  }
  __syncthreads();
  const int need = p.top_k - above_window, n_open = n_few;   // of the open ones
  uint64_t least = 0;   // open candidates are taken above this key, `ties` of those at it
  ties = n_open;
  if (need < n_open) {
    // 64-bit scores, a warp a candidate, every one's terms in the same order
    double q[D / 32];
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      const float2 v = qs[lane + 32 * j];
      q[j] = static_cast<double>(v.x) + static_cast<double>(v.y);
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
    if (n_open <= kFew) {
      for (int i = warp; i < n_open; i += P_WARPS) {
        const double s = score64(few[i]);
        if (lane == 0) few_key[i] = order_key(s), exact[few[i]] = s;
      }
      __syncthreads();
      if (threadIdx.x < n_open) {   // the one with `need - 1` ahead of it is the last one taken
        int ahead = 0, equal = 0;
        for (int j = 0; j < n_open; ++j) {
          ahead += few_key[j] > few_key[threadIdx.x];
          equal += few_key[j] == few_key[threadIdx.x];
        }
        if (ahead < need && ahead + equal >= need) {
          few_least = few_key[threadIdx.x];   // equal ones write the same
          hist[0] = need - ahead;
        }
      }
      __syncthreads();
      least = few_least;
      ties = hist[0];
    } else {
      for (int i = warp; i < n; i += P_WARPS)
        if (open(i)) {
          const double s = score64(i);
          if (lane == 0) exact[i] = s;
        }
      __syncthreads();
      least = kth_largest<uint64_t>(n, need, [&](int i) { return order_key(exact[i]); }, open, hist, ties);
    }
  }
  // In the order of their numbers: the sure ones, the open ones above `least` and the first `ties` of those at it.
  const bool all_open = need >= n_open;
  int done = 0, tied = 0;   // written, and ties met so far
  for (int i0 = 0; i0 < n; i0 += P_THREADS) {
    const int i = i0 + threadIdx.x;
    bool in = false, tie = false;
    if (i < n) {
      if (sure(i)) in = true;
      else if (open(i)) {
        if (all_open) in = true;
        else {
          const uint64_t x = order_key(exact[i]);
          in = x > least;
          tie = x == least;
        }
      }
    }
    const uint32_t tie_mask = __ballot_sync(0xffffffffu, tie);
    if (lane == 0) counts[0][warp] = __popc(tie_mask);
    __syncthreads();
    int rank = tied + __popc(tie_mask & ((1u << lane) - 1u));
    for (int w = 0; w < P_WARPS; ++w) {
      if (w < warp) rank += counts[0][w];
      tied += counts[0][w];
    }
    in = in || (tie && rank < ties);
    const uint32_t mask = __ballot_sync(0xffffffffu, in);
    if (lane == 0) counts[1][warp] = __popc(mask);
    __syncthreads();
    int at = done + __popc(mask & ((1u << lane) - 1u));
    for (int w = 0; w < P_WARPS; ++w) {
      if (w < warp) at += counts[1][w];
      done += counts[1][w];
    }
    if (in) out[at] = id_of(p, i);
  }
}

template <int D>
cudaError_t select_d(const SelectParams& p, cudaStream_t s) {
  const dim3 lists(static_cast<unsigned>(p.n_qt), static_cast<unsigned>(p.H));
  if (p.n_cand > p.top_k) {
    cudaError_t e = launch_pdl(qsum_kernel<D>, lists, dim3(256), 0, s, p);
    if (e != cudaSuccess) return e;
    constexpr int smem = (S_CAND + S_QT) * (D + 4) * 4;
    e = set_smem_limit_once(reinterpret_cast<const void*>(score_kernel<D>), smem);
    if (e != cudaSuccess) return e;
    e = launch_pdl(score_kernel<D>, dim3(static_cast<unsigned>((p.n_cand + S_CAND - 1) / S_CAND),
                                         static_cast<unsigned>(p.H)),
                   dim3(256), smem, s, p);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(pick_kernel<D>, lists, dim3(P_THREADS), 0, s, p);
}

}  // namespace

cudaError_t launch_key_means(const MeansParams& p, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>(p.units), static_cast<unsigned>(p.H));
  if (p.k_scale) return launch_pdl(means_kernel<true, 128>, grid, dim3(M_THREADS), 0, s, p);
  if (p.d == 128) return launch_pdl(means_kernel<false, 128>, grid, dim3(M_THREADS), 0, s, p);
  return launch_pdl(means_kernel<false, 64>, grid, dim3(M_THREADS), 0, s, p);
}

size_t select_ws_bytes(int64_t H, int64_t n_qt, int64_t d, int64_t ids) {
  return static_cast<size_t>(H) * (n_qt * d * 8 + n_qt * ids * 12 + ids * 4);
}

cudaError_t launch_select(const SelectParams& p, cudaStream_t s) {
  return p.d == 128 ? select_d<128>(p, s) : select_d<64>(p, s);
}

}  // namespace ispa
