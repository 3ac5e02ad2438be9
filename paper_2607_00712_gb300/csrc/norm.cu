// The norms on both sides of a transformer block, with the block's gate, the residual scale and the next block's
// modulation (a DiT's adaptive norms), one pass over the rows:
//
//   x <- x_scale x + y_scale gate_g post(y)            (residual part, RES)
//   h  = pre(x) (1 + scale_g) + shift_g                -> bf16, or 8-bit codes with a scale per row
//
//   rms(v)   = v / sqrt(mean(v^2) + eps) w + b
//   layer(v) = (v - mean v) / sqrt(mean((v - mean v)^2) + eps) w + b
//
// g = row / rows_per_group picks the row of the modulation vectors (one per latent frame, say).
//
// Memory bounds it: x, y and the results cross HBM once.  A row lives in registers from its load to its store, eight
// values a thread, so the second pass of the variance and the maximum of the codes cost no traffic.  Everything between
// load and store is fp32; x is rounded to its own type first and h is taken from the rounded value, the one that the
// next reader of x sees.
//
//   stream_kernel   many rows: teams of warps go through a run of rows that bulk copies bring into shared memory, the
//                   factors of the columns (weights, gate, modulation) kept there per group of rows
//   norm_kernel     few rows, very long ones, or vectors that change every few rows: a block a row
//
// Gate, residual and two RMS norms of 4680 x 5120 bf16: 37.1 us, 76 % of the measured copy rate.  With a block a row 59
// us (the vectors, fp32, were 2.5 times the rows' own bytes through L1); with the factors in registers and the next
// row's loads too, 48 (one team of 640 threads an SM: nothing to do while it reduces); with one vector of eight a
// thread and everything in shared memory, 59 (the reductions' instructions); loads into registers instead of bulk
// copies, 53.  Layer norms take 44.6: the mean, then the squares, are two reductions in a row.  Norm of 4680 x 1536
// bf16: 9.4 us, of which 4 are launch, factors and the last rows' way out (each further row at 84 % of the copy rate);
// with a warp a row, the vectors from L1, 10.7.  One row of 1536 2.4 us.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "forms.h"
#include "internal.h"
#include "pdl.cuh"
#include "rows.cuh"

namespace ispa {

namespace {

struct Reducer {
  float (*red)[32];
  int warps, slot = 0;
  template <typename Op>
  __device__ __forceinline__ float all(float v) {
    v = block_reduce<Op>(v, warps, red, slot);
    slot ^= 1;
    return v;
  }
};

// The norm of a row that the threads hold as V vectors of eight, in place.
template <int V>
__device__ __forceinline__ void norm_row(float (&v)[V][8], const ispa_norm& n, int nv, int dim, int t, int step,
                                         Reducer& r) {
  if (n.kind == ISPA_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i)   // vectors past the row hold zeros
#pragma unroll
      for (int e = 0; e < 8; ++e) s += v[i][e];
    const float mean = r.template all<SumOp>(s) / static_cast<float>(dim);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (t + i * step < nv)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] -= mean;
  }
  float rstd = 1.f;
  if (n.kind != ISPA_NORM_NONE) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(v[i][e], v[i][e], s);
    rstd = __frsqrt_rn(r.template all<SumOp>(s) / static_cast<float>(dim) + n.eps);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = t + i * step;
    if (c < nv) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] *= rstd;
      if (n.weight) {
        load8(n.weight + 8 * c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] *= w[e];
      }
      if (n.bias) {
        load8(n.bias + 8 * c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] += w[e];
      }
    }
  }
}

// One row a block, V vectors of eight values a thread.
template <int V, bool XF32, bool RES>
__global__ void __launch_bounds__(512) norm_kernel(const __grid_constant__ NormParams p) {
  __shared__ float red[2][32];
  pdl_wait();
  pdl_trigger();
  const int64_t row = blockIdx.x;
  const int t = threadIdx.x, step = blockDim.x, nv = p.dim / 8;
  Reducer r{red, step >> 5};
  const int64_t base = row * p.dim;
  const int64_t mod = p.gate || p.scale || p.shift ? row / p.rows_per_group * p.mod_stride : 0;

  float x[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = t + i * step;
    if (c < nv) {
      if constexpr (XF32) {
        const float4* s = reinterpret_cast<const float4*>(static_cast<const float*>(p.x) + base + 8 * c);
        const float4 a = s[0], b = s[1];
        x[i][0] = a.x, x[i][1] = a.y, x[i][2] = a.z, x[i][3] = a.w;
        x[i][4] = b.x, x[i][5] = b.y, x[i][6] = b.z, x[i][7] = b.w;
      } else {
        unpack8(*reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.x) + base + 8 * c), x[i]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
    }
  }

  if constexpr (RES) {
    float y[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = t + i * step;
      unpack8(c < nv ? *reinterpret_cast<const uint4*>(p.y + base + 8 * c) : make_uint4(0, 0, 0, 0), y[i]);
    }
    norm_row<V>(y, p.post, nv, p.dim, t, step, r);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = t + i * step;
      if (c < nv) {
        float g[8];
        if (p.gate) {
          load8(p.gate + mod + 8 * c, g);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[i][e] *= g[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = fmaf(p.y_scale, y[i][e], p.x_scale * x[i][e]);
        if constexpr (XF32) {
          float4* s = reinterpret_cast<float4*>(static_cast<float*>(p.x_out) + base + 8 * c);
          s[0] = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
          s[1] = make_float4(x[i][4], x[i][5], x[i][6], x[i][7]);
        } else {
          const uint4 w = pack8(x[i]);
          *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.x_out) + base + 8 * c) = w;
          unpack8(w, x[i]);   // the next norm reads x as it is stored
        }
      }
    }
    if (!p.out) return;   // uniform over the grid
  }

  norm_row<V>(x, p.pre, nv, p.dim, t, step, r);
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = t + i * step;
    if (c < nv) {
      float m[8];
      if (p.scale) {
        load8(p.scale + mod + 8 * c, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] *= 1.f + m[e];
      }
      if (p.shift) {
        load8(p.shift + mod + 8 * c, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] += m[e];
      }
      if (p.format == ISPA_ROWS_BF16) {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + base + 8 * c) = pack8(x[i]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max_nan(amax, fabsf(x[i][e]));
      }
    }
  }
  if (p.format == ISPA_ROWS_BF16) return;
  amax = r.template all<MaxOp>(amax);
  const float top = p.format == ISPA_ROWS_E4M3 ? 448.f : 127.f;
  const float inv = code_factor(amax, top);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = t + i * step;
    if (c < nv) {
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.out) + base + 8 * c) =
          p.format == ISPA_ROWS_E4M3 ? make_uint2(pack_e4m3x4(x[i], inv), pack_e4m3x4(x[i] + 4, inv))
                                     : make_uint2(pack_i8x4(x[i], inv), pack_i8x4(x[i] + 4, inv));
    }
  }
  if (t == 0) p.out_scale[row] = code_scale(amax, top);
}

// ------------------------------------------------------------ many rows
constexpr uint64_t S_DRAIN_NS = 200ull * 1000 * 1000;

// Vector c of a row: two runs of four values.  With an fp32 stream they are half a row apart, so that a warp reads and
// writes whole lines; with a bf16 stream they are neighbours, one 16-byte word.
template <bool XF32>
struct Cols {
  int c0, c1;
  __device__ __forceinline__ Cols(int c, int dim) : c0(XF32 ? 4 * c : 8 * c), c1(XF32 ? dim / 2 + 4 * c : 8 * c + 4) {}
  __device__ __forceinline__ void f32(const float* p, float* f) const {
    const float4 a = *reinterpret_cast<const float4*>(p + c0), b = *reinterpret_cast<const float4*>(p + c1);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  }
  __device__ __forceinline__ void put_f32(float* p, const float* f) const {
    *reinterpret_cast<float4*>(p + c0) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + c1) = make_float4(f[4], f[5], f[6], f[7]);
  }
  __device__ __forceinline__ void bf16(const __nv_bfloat16* p, float* f) const {
    if constexpr (XF32) {
      const uint2 a = *reinterpret_cast<const uint2*>(p + c0), b = *reinterpret_cast<const uint2*>(p + c1);
      unpack8(make_uint4(a.x, a.y, b.x, b.y), f);
    } else {
      unpack8(*reinterpret_cast<const uint4*>(p + c0), f);
    }
  }
  __device__ __forceinline__ void put_bf16(__nv_bfloat16* p, const uint4& w) const {
    if constexpr (XF32) {
      *reinterpret_cast<uint2*>(p + c0) = make_uint2(w.x, w.y);
      *reinterpret_cast<uint2*>(p + c1) = make_uint2(w.z, w.w);
    } else {
      *reinterpret_cast<uint4*>(p + c0) = w;
    }
  }
  __device__ __forceinline__ void put_codes(uint8_t* p, uint32_t a, uint32_t b) const {
    if constexpr (XF32) {
      *reinterpret_cast<uint32_t*>(p + c0) = a;
      *reinterpret_cast<uint32_t*>(p + c1) = b;
    } else {
      *reinterpret_cast<uint2*>(p + c0) = make_uint2(a, b);
    }
  }
};

// -mean / root and 1 / root of the team's row, whose values past the row are zeros.  A warp takes its own values' mean
// and squares about that mean; the warps' are joined by n_w (m_w - m)^2 (Chan, Golub, LeVeque 1983), which needs one
// barrier where the plain two passes need two, and loses as little.  vectors: this thread's of the row; inv_own, other:
// 1 / values of this warp, and values of warp lane % TEAM_WARPS.
template <int V>
__device__ __forceinline__ float2 team_norm(const float (&v)[V][8], const ispa_norm& n, float inv_dim, int vectors,
                                            float inv_own, float other, Team& tm) {
  if (n.kind == ISPA_NORM_NONE) return make_float2(0.f, 1.f);
  float m = 0.f, q = 0.f;
  if (n.kind == ISPA_NORM_RMS) {
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) q = fmaf(v[i][e], v[i][e], q);
    q = warp_reduce<SumOp>(q);
    if (tm.warps > 1) q = group_reduce<SumOp>(tm.gather(make_float2(0.f, q)).y, TEAM_WARPS);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) m += v[i][e];
    m = warp_reduce<SumOp>(m) * inv_own;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < vectors)
#pragma unroll
        for (int e = 0; e < 8; ++e) q = fmaf(v[i][e] - m, v[i][e] - m, q);
    q = warp_reduce<SumOp>(q);
    if (tm.warps > 1) {
      const float2 a = tm.gather(make_float2(m, q));
      m = group_reduce<SumOp>(a.x * other, TEAM_WARPS) * inv_dim;
      q = group_reduce<SumOp>(fmaf((a.x - m) * other, a.x - m, a.y), TEAM_WARPS);
    }
  }
  const float rstd = rsqrtf(fmaf(q, inv_dim, n.eps));   // off by 2^-22.9 at most, a tenth of what the sums may be
  return make_float2(-m * rstd, rstd);   // v rstd - m rstd
}

// Block (32 * warps of a team, teams), one an SM; block b takes rows [b, b + 1) * rows_per_block, its teams in turn.
// Rows come through shared memory by bulk copies, a team's next row while it works on one: registers would hold a third
// as much.  A team's thread takes up to V vectors of the row.  The columns' factors stand in shared memory too, per
// group of rows, for all teams.
template <int V, bool XF32, bool RES>
__global__ void __launch_bounds__(s_threads(V, RES), 1)
    stream_kernel(const __grid_constant__ NormParams p, int rows_per_block) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int abort_word;
  const int t = threadIdx.x, step = blockDim.x, teams = blockDim.y, dim = p.dim, nv = dim / 8, lane = t & 31;
  const bool modulated = p.gate || p.scale || p.shift, next_norm = !RES || p.out;
  const int arrays = !RES ? 2 : p.post.bias ? 4 : 3;
  // [A, B, (G, (H))][half][vector], the teams' rows [2][x, (y)], their barriers and their reductions
  float4* factors = reinterpret_cast<float4*>(smem);
  const int x_bytes = dim * (XF32 ? 4 : 2), row_bytes = x_bytes + (RES ? 2 * dim : 0);
  uint8_t* const rows = smem + 32 * arrays * nv + 2 * row_bytes * threadIdx.y;
  uint64_t* const bars = reinterpret_cast<uint64_t*>(smem + 32 * arrays * nv + 2 * row_bytes * teams);
  const uint32_t full = smem_u32(bars + 2 * threadIdx.y);
  Team tm{reinterpret_cast<float2*>(bars + 2 * teams) + threadIdx.y * 2 * TEAM_WARPS, step >> 5,
          1 + static_cast<int>(threadIdx.y), 0};
  const int vectors = t < nv ? (nv - t + step - 1) / step : 0;   // of this thread
  const float inv_dim = 1.f / static_cast<float>(dim);
  float own = 0.f, other = 0.f;   // values of this warp, and of the warp that this lane joins
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int left = nv - i * step, w = lane & (TEAM_WARPS - 1);
    own += 8.f * static_cast<float>(max(0, min(32, left - (t & ~31))));
    if (w < tm.warps) other += 8.f * static_cast<float>(max(0, min(32, left - 32 * w)));
  }
  const float inv_own = 1.f / own;
  auto put = [&](int array, int c, const float* f) {
    factors[(2 * array) * nv + c] = make_float4(f[0], f[1], f[2], f[3]);
    factors[(2 * array + 1) * nv + c] = make_float4(f[4], f[5], f[6], f[7]);
  };
  auto get = [&](int array, int c, float* f) {
    const float4 a = factors[(2 * array) * nv + c], b = factors[(2 * array + 1) * nv + c];
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  };
  if (t == 0) {
    mbar_init(full, 1);
    mbar_init(full + 8, 1);
    abort_word = 0;
    fence_mbar_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const WaitCtx wc{&abort_word, p.status, p.wait_limit_ns};

  int first = blockIdx.x * rows_per_block;   // rows are fewer than 2^31
  const int last = min(static_cast<int64_t>(first) + rows_per_block, p.rows);
  auto fetch = [&](int row, int stage) {
    mbar_arrive_expect_tx(full + 8 * stage, row_bytes);
    const uint32_t dst = smem_u32(rows) + stage * row_bytes;
    bulk_load(dst, static_cast<const uint8_t*>(p.x) + static_cast<int64_t>(row) * x_bytes, x_bytes, full + 8 * stage);
    if constexpr (RES) bulk_load(dst + x_bytes, p.y + static_cast<int64_t>(row) * dim, 2 * dim, full + 8 * stage);
  };
  int row = first + threadIdx.y;
  const int per = static_cast<int>(min(p.rows_per_group, p.rows));
  uint32_t turn = 0, issued = 0;   // rows that this team has begun, and (thread 0) that it has sent for
  bool ok = true;
  if (t == 0 && row < last) fetch(row, issued++ & 1);
  while (first < last) {
    const int group = modulated ? first / per : 0;
    const int64_t group_end = static_cast<int64_t>(group + 1) * per;
    const int end = modulated && group_end < last ? static_cast<int>(group_end) : last;
    // h = (x rstd - mean rstd) A + B and x = x_scale x + (y rstd - mean rstd) G + H, per column
    __syncthreads();
    for (int c = threadIdx.y * step + t; c < nv; c += step * teams) {
      const Cols<XF32> cols(c, dim);
      const int64_t at = static_cast<int64_t>(group) * p.mod_stride;
      float u[8], v[8], f[8], g[8];   // all loads on their way before the first is used
      if (next_norm) {
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = 1.f, v[e] = 0.f, f[e] = 0.f, g[e] = 0.f;
        if (p.pre.weight) cols.f32(p.pre.weight, u);
        if (p.scale) cols.f32(p.scale + at, f);
        if (p.shift) cols.f32(p.shift + at, g);
        if (p.pre.bias) cols.f32(p.pre.bias, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] *= 1.f + f[e], v[e] = fmaf(v[e], 1.f + f[e], g[e]);
        put(0, c, u);
        put(1, c, v);
      }
      if constexpr (RES) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = 1.f, u[e] = 1.f, v[e] = 0.f;
        if (p.post.weight) cols.f32(p.post.weight, u);
        if (p.gate) cols.f32(p.gate + at, f);
        if (p.post.bias) cols.f32(p.post.bias, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= p.y_scale, u[e] *= f[e], v[e] *= f[e];
        put(2, c, u);
        if (p.post.bias) put(3, c, v);
      }
    }
    __syncthreads();

    for (; row < end; row += teams, ++turn) {   // stays below 2^31: see the launch
      const int stage = turn & 1;
      if (t == 0 && ok && last - row > teams) fetch(row + teams, issued++ & 1);   // all have read the last row there
      ok &= mbar_wait(full + 8 * stage, (turn >> 1) & 1, wc, 51, row);   // a row that never comes: recorded
      const uint8_t* src = rows + stage * row_bytes;
      const int64_t base = static_cast<int64_t>(row) * dim;
      float x[V][8], f[8];
      auto load_x = [&](int i) {
        const Cols<XF32> cols(t + i * step, dim);
        if constexpr (XF32) cols.f32(reinterpret_cast<const float*>(src), x[i]);
        else cols.bf16(reinterpret_cast<const __nv_bfloat16*>(src), x[i]);
      };
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!RES && i < vectors) {
          load_x(i);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
        }
      }
      if constexpr (RES) {
        const __nv_bfloat16* ys = reinterpret_cast<const __nv_bfloat16*>(src + x_bytes);
        float y[V][8];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          if (i < vectors) {
            Cols<XF32>(t + i * step, dim).bf16(ys, y[i]);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[i][e] = 0.f;
          }
        }
        const float2 n = team_norm<V>(y, p.post, inv_dim, vectors, inv_own, other, tm);
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i < vectors) {
            const Cols<XF32> cols(t + i * step, dim);
            load_x(i);
            get(2, t + i * step, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = fmaf(fmaf(y[i][e], n.y, n.x), f[e], p.x_scale * x[i][e]);
            if (p.post.bias) {
              get(3, t + i * step, f);
#pragma unroll
              for (int e = 0; e < 8; ++e) x[i][e] += f[e];
            }
            if constexpr (XF32) {
              cols.put_f32(static_cast<float*>(p.x_out) + base, x[i]);
            } else {
              const uint4 w = pack8(x[i]);
              cols.put_bf16(static_cast<__nv_bfloat16*>(p.x_out) + base, w);
              unpack8(w, x[i]);   // the next norm reads x as it is stored
            }
          }
      }
      if (next_norm) {   // uniform over the grid
        const float2 n = team_norm<V>(x, p.pre, inv_dim, vectors, inv_own, other, tm);
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (i < vectors) {
            float b[8];
            get(0, t + i * step, f);
            get(1, t + i * step, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = fmaf(fmaf(x[i][e], n.y, n.x), f[e], b[e]);
            if (p.format == ISPA_ROWS_BF16) {
              Cols<XF32>(t + i * step, dim).put_bf16(static_cast<__nv_bfloat16*>(p.out) + base, pack8(x[i]));
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) amax = max_nan(amax, fabsf(x[i][e]));
            }
          }
        if (p.format != ISPA_ROWS_BF16) {
          amax = warp_max(amax);
          if (tm.warps > 1) amax = warp_max(tm.gather(make_float2(amax, 0.f)).x);
          const bool e4m3 = p.format == ISPA_ROWS_E4M3;
          const float top = e4m3 ? 448.f : 127.f, inv = code_factor(amax, top);
          const auto put = [&](auto&& pack) {
#pragma unroll
            for (int i = 0; i < V; ++i)
              if (i < vectors)
                Cols<XF32>(t + i * step, dim)
                    .put_codes(static_cast<uint8_t*>(p.out) + base, pack(x[i]), pack(x[i] + 4));
          };
          if (e4m3) put([&](const float* h) { return pack_e4m3x4(h, inv); });
          else put([&](const float* h) { return pack_i8x4(h, inv); });
          if (t == 0) p.out_scale[row] = code_scale(amax, top);
        }
      }
      tm.sync();   // the row's stage is free
    }
    first = end;
  }
  if (t == 0 && !ok)   // after a timeout: nothing in flight when the block leaves
    for (uint32_t i = issued < 2 ? 0 : issued - 2; i < issued; ++i)
      mbar_wait_drain(full + 8 * (i & 1), (i >> 1) & 1, S_DRAIN_NS);
}

template <bool XF32, bool RES>
cudaError_t launch_typed(const NormParams& p, int sms, cudaStream_t s) {
  const NormForm f = norm_form(p.rows, p.dim, XF32, RES, p.post.bias != nullptr, p.gate || p.scale || p.shift,
                               p.rows_per_group, sms);
  if (f.stream) {
    const auto go = [&](auto kernel) {
      const cudaError_t e = set_smem_limit_once(reinterpret_cast<const void*>(kernel), S_SMEM);
      if (e != cudaSuccess) return e;
      return launch_pdl(kernel, dim3(static_cast<unsigned>((p.rows + f.rows - 1) / f.rows)),
                        dim3(32 * f.warps, f.teams), f.smem, s, p, static_cast<int>(f.rows));
    };
    return f.vectors == 1   ? go(stream_kernel<1, XF32, RES>)
           : f.vectors == 2 ? go(stream_kernel<2, XF32, RES>)
           : f.vectors == 3 ? go(stream_kernel<3, XF32, RES>)
                            : go(stream_kernel<4, XF32, RES>);
  }
  const auto go = [&](auto kernel) {
    return launch_pdl(kernel, dim3(static_cast<unsigned>(p.rows)), dim3(32 * f.warps), 0, s, p);
  };
  return f.vectors == 1   ? go(norm_kernel<1, XF32, RES>)
         : f.vectors == 2 ? go(norm_kernel<2, XF32, RES>)
         : f.vectors == 4 ? go(norm_kernel<4, XF32, RES>)
                          : go(norm_kernel<8, XF32, RES>);
}

}  // namespace

cudaError_t launch_norm(const NormParams& p, bool x_fp32, bool residual, cudaStream_t s) {
  int dev = 0, sms = 152;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return x_fp32 ? (residual ? launch_typed<true, true>(p, sms, s) : launch_typed<true, false>(p, sms, s))
                : (residual ? launch_typed<false, true>(p, sms, s) : launch_typed<false, false>(p, sms, s));
}

}  // namespace ispa
