// Rotary positions of a chunk's queries and keys, with the RMS norm that stands in front of them in many models:
//
//   n_{t,h} = x_{t,h} / sqrt(mean(x^2) + eps) w      mean over the head, or over all heads of the token
//   (u, v) <- f (u cos a - v sin a, u sin a + v cos a),   a = 2 pi frac(pos_axis(i)(t) steps_i)
//
// for the pairs i of each head: features (2i, 2i + 1), or (i, i + pairs); features past 2 pairs only take the norm.
//
// Angles: steps_i is the pair's turns per position as a 64-bit fraction of a turn, so pos * steps_i modulo 2^64 is the
// position's fraction of a turn with no rounding however far the position is; its upper 32 bits (2^-32 of a turn,
// 1.5e-9 rad) go to fp32.  The reduced angle lies in [-pi, pi), where __sinf and __cosf are off by at most 2^-21.19:
// 2^-12 of a bf16 rounding step of the largest value, against a dozen more instructions a pair for sincosf.
//
// Memory bounds it: each value crosses HBM once in and once out.  Block: one or more warps a token; a thread takes eight
// neighbouring features of one head (16 bytes) per step, and because a warp's lanes are dealt to heads in groups of a
// power of two, a lane meets the same features of every head: its sines and cosines are computed once a token and
// stay in registers.  Partners of the second layout come from a neighbouring lane by a shuffle.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "pdl.cuh"
#include "rows.cuh"

namespace ispa {

namespace {

// The upper 32 bits of the 64-bit product's lower half: the position's fraction of a turn in units of 2^-32.
__device__ __forceinline__ uint32_t turn_fraction(int64_t pos, uint64_t step) {
  return static_cast<uint32_t>((static_cast<uint64_t>(pos) * step) >> 32);
}

// V: vectors a thread holds at once.  Block (32 * warps of a token, tokens of a block): one of the two is 1 warp / 1
// token.  blockIdx.y: which of the rows (queries or keys).
template <int V, bool HALF, bool MULTI>
__global__ void __launch_bounds__(MULTI ? 512 : 256) rope_kernel(const __grid_constant__ RopeParams p) {
  __shared__ float red[2][32];
  pdl_wait();
  pdl_trigger();
  const int64_t tok = MULTI ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y;
  if (tok >= p.n) return;   // a whole warp; blocks of one token have none
  const RopeRowsParams& o = p.rows[blockIdx.y];
  const int lph = p.lanes_per_head, d = p.head_dim;
  const int c = threadIdx.x & (lph - 1);           // this lane's vector of every head it meets
  const bool live = 8 * c < d;
  const int heads_step = blockDim.x / lph;         // heads the block takes per step
  const int head0 = threadIdx.x / lph;
  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(o.x) + tok * o.x_stride + 8 * c;
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(o.out) + tok * o.out_stride + 8 * c;

  uint4 raw[V];
  auto load = [&](int h) {
    return live && h < o.heads ? *reinterpret_cast<const uint4*>(x + static_cast<int64_t>(h) * d)
                               : make_uint4(0, 0, 0, 0);
  };
#pragma unroll
  for (int i = 0; i < V; ++i) raw[i] = load(head0 + i * heads_step);

  // sines and cosines of this lane's features: pair i of the layout
  constexpr int NP = HALF ? 8 : 4;
  float cs[NP], sn[NP];
  uint32_t turned = 0;   // features (pairs) past the rotated ones pass as they are, infinities too
  const int pairs = p.pairs;
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    int i = HALF ? 8 * c + j : 4 * c + j;
    bool second = false;
    if (HALF && i >= pairs) {
      i -= pairs;
      second = true;
    }
    cs[j] = 1.f;
    sn[j] = 0.f;
    if (i < pairs) {
      const int axis = i < p.axis_end[0] ? 0 : i < p.axis_end[1] ? 1 : 2;
      const int64_t pos = static_cast<int64_t>(p.pos[axis * p.n + tok]) + (axis == 0 ? p.pos0 : 0);
      const float a = static_cast<float>(static_cast<int32_t>(turn_fraction(pos, p.steps[i]))) *
                      1.46291807926715968105e-9f;   // 2 pi / 2^32
      cs[j] = p.factor * __cosf(a);
      sn[j] = p.factor * __sinf(a);
      if (second) sn[j] = -sn[j];   // out = cos own - sin partner in the first half, + in the second
      turned |= 1u << j;
    }
  }

  float rstd = 1.f;
  if (o.norm == ISPA_QK_NORM_TOKEN) {
    float s = 0.f, f[8];
    auto add = [&](const uint4& w) {
      unpack8(w, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(f[e], f[e], s);
    };
#pragma unroll
    for (int i = 0; i < V; ++i) add(raw[i]);
    for (int h = head0 + V * heads_step; h < o.heads; h += heads_step) add(load(h));
    s = MULTI ? block_reduce<SumOp>(s, blockDim.x >> 5, red, 0) : warp_reduce<SumOp>(s);
    rstd = __frsqrt_rn(s / static_cast<float>(o.heads * d) + o.eps);
  }
  float w[8];
  if (o.norm == ISPA_QK_NORM_HEAD && o.weight && live) load8(o.weight + 8 * c, w);

  auto finish = [&](const uint4& v, int h) {
    float f[8];
    unpack8(v, f);
    if (o.norm == ISPA_QK_NORM_HEAD) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(f[e], f[e], s);
      s = group_reduce<SumOp>(s, lph);
      const float r = __frsqrt_rn(s / static_cast<float>(d) + o.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = o.weight ? f[e] * r * w[e] : f[e] * r;
    } else if (o.norm == ISPA_QK_NORM_TOKEN) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= rstd;
      if (o.weight && live && h < o.heads) {
        float wt[8];
        load8(o.weight + static_cast<int64_t>(h) * d + 8 * c, wt);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= wt[e];
      }
    }
    float g[8];
    if constexpr (HALF) {
      // feature 8 c + e's partner is `pairs` (a multiple of 8) features on, or back in the second half
      const int lane = threadIdx.x & 31;
      const int from = 8 * c < pairs ? lane + (pairs >> 3) : 8 * c < 2 * pairs ? lane - (pairs >> 3) : lane;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float q = __shfl_sync(0xffffffffu, f[e], from);
        g[e] = turned >> e & 1 ? fmaf(cs[e], f[e], -sn[e] * q) : f[e];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool t = turned >> j & 1;
        g[2 * j] = t ? fmaf(cs[j], f[2 * j], -sn[j] * f[2 * j + 1]) : f[2 * j];
        g[2 * j + 1] = t ? fmaf(sn[j], f[2 * j], cs[j] * f[2 * j + 1]) : f[2 * j + 1];
      }
    }
    if (live && h < o.heads) *reinterpret_cast<uint4*>(out + static_cast<int64_t>(h) * d) = pack8(g);
  };
  // Every lane of a warp goes round alike (the shuffles need all of them): the step counts from the block's first head.
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i * heads_step < o.heads) finish(raw[i], head0 + i * heads_step);
  for (int h = V * heads_step; h < o.heads; h += V * heads_step) {
#pragma unroll
    for (int i = 0; i < V; ++i) raw[i] = load(h + head0 + i * heads_step);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (h + i * heads_step < o.heads) finish(raw[i], h + head0 + i * heads_step);
  }
}

template <bool HALF>
cudaError_t launch_layout(const RopeParams& p, int n_ops, int sms, cudaStream_t s) {
  int heads = p.rows[0].heads;
  if (n_ops > 1 && p.rows[1].heads > heads) heads = p.rows[1].heads;
  const int steps = (heads * p.lanes_per_head + 31) / 32;   // vectors a lane of one warp would take
  const auto go = [&](auto kernel, int warps, int toks) {
    const int64_t blocks = (p.n + toks - 1) / toks;
    return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks), n_ops), dim3(32 * warps, toks), 0, s, p);
  };
  if (p.n > 4 * sms && steps <= 8) {
    if (steps <= 4) return go(rope_kernel<4, HALF, false>, 1, 8);
    return go(steps <= 6 ? rope_kernel<6, HALF, false> : rope_kernel<8, HALF, false>, 1, 8);
  }
  if (steps <= 16) return go(rope_kernel<1, HALF, true>, steps, 1);
  if (steps <= 32) return go(rope_kernel<2, HALF, true>, (steps + 1) / 2, 1);
  return go(rope_kernel<4, HALF, true>, steps <= 64 ? (steps + 3) / 4 : 16, 1);
}

}  // namespace

cudaError_t launch_rope(const RopeParams& p, int n_ops, bool half, cudaStream_t s) {
  int dev = 0, sms = 152;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return half ? launch_layout<true>(p, n_ops, sms, s) : launch_layout<false>(p, n_ops, sms, s);
}

bool rope_steps(const ispa_rope_frequencies& f, int32_t n_pairs, uint64_t* steps, float* factor) {
  constexpr double kTwoPi = 6.283185307179586476925286766559;
  const bool scaled = f.scaling != ISPA_ROPE_SCALE_NONE, parts = f.scaling == ISPA_ROPE_SCALE_PARTS;
  if (f.scaling < ISPA_ROPE_SCALE_NONE || f.scaling > ISPA_ROPE_SCALE_PARTS || !(f.base >= 1.0) || !isfinite(f.base) ||
      (scaled && (!(f.scale >= 1.0) || !isfinite(f.scale))) ||
      (parts && (!(f.trained_length > 0.0) || !isfinite(f.trained_length) || !(f.low >= 0.0) || !(f.low < f.high) ||
                 !isfinite(f.high))))
    return false;
  double base = f.base, divide = 1.0;
  if (f.scaling == ISPA_ROPE_SCALE_LINEAR || (f.scaling == ISPA_ROPE_SCALE_BASE && n_pairs == 1)) divide = f.scale;
  else if (f.scaling == ISPA_ROPE_SCALE_BASE) base *= pow(f.scale, static_cast<double>(n_pairs) / (n_pairs - 1));
  if (!isfinite(base)) return false;
  for (int32_t i = 0; i < n_pairs; ++i) {
    double w = pow(base, -static_cast<double>(i) / n_pairs) / divide;
    if (parts) {
      const double turns = f.trained_length * w / kTwoPi;
      const double keep = std::min(1.0, std::max(0.0, (turns - f.low) / (f.high - f.low)));
      w *= keep + (1.0 - keep) / f.scale;
    }
    steps[i] = static_cast<uint64_t>(rint(ldexp(w / kTwoPi, 64)));   // w <= 1: below 2^62
  }
  if (factor) *factor = parts ? static_cast<float>(0.1 * log(f.scale) + 1.0) : 1.f;
  return true;
}

}  // namespace ispa
