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
// Memory bounds it: each value crosses HBM once in and once out.  A block first makes the sines and cosines of its tokens
// (a warp that made them for itself spent more on them than on its heads: 3117 tokens of 24 and 8 heads of 128, half
// layout, 58 us), then a warp takes a row, the queries or keys of one token, held in registers between the norm's sum
// and the rotation; with few rows a block takes one.  A thread takes eight features of one head per step: eight
// neighbours, or four and the four that they turn with, so that no pair is spread over two lanes.  A warp's lanes are
// dealt to heads in groups of a power of two, so a lane meets the same features, angles and weights in every head.
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

// V: vectors a thread holds at once.  Block: 8 warps of a row each, or (MULTI) the warps of one row; row r is token
// r / n_rows, tensor r % n_rows.
template <int V, bool HALF, bool MULTI>
__global__ void __launch_bounds__(MULTI ? 512 : 256) rope_kernel(const __grid_constant__ RopeParams p) {
  __shared__ float2 table[MULTI ? 1 : 8][128];   // cosine and sine of the block's tokens' pairs
  __shared__ float red[2][32];
  const int tensors = p.n_rows, lane = threadIdx.x & 31;
  const int64_t n_rows = p.n * tensors, row0 = static_cast<int64_t>(blockIdx.x) * (MULTI ? 1 : 8);
  const int64_t tok0 = row0 / tensors;
  const int64_t row = row0 + (MULTI ? 0 : threadIdx.x >> 5), tok = row / tensors;
  const RopeRowsParams& o = p.rows[row - tok * tensors];
  const int lph = p.lanes_per_head, d = p.head_dim, pairs = p.pairs;
  const int c = lane & (lph - 1);                                     // this lane's vector of every head it meets
  const bool live = 8 * c < d && row < n_rows;
  const int heads_step = (MULTI ? blockDim.x : 32) / lph;             // heads a row's warps take per step
  const int head0 = (MULTI ? threadIdx.x : lane) / lph;
  // features at[0] .. + 3 and at[1] .. + 3 of a head, pairs 4 c .. 4 c + 3
  const int at0 = !HALF ? 8 * c : 4 * c < pairs ? 4 * c : 8 * c;
  const int at1 = HALF && 4 * c < pairs ? pairs + 4 * c : at0 + 4;
  const int turned = min(4, max(0, pairs - 4 * c));                   // of the lane's pairs; what follows them passes
  pdl_wait();
  pdl_trigger();

  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(o.x) + tok * o.x_stride;
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(o.out) + tok * o.out_stride;
  uint4 raw[V];
  auto load = [&](int h) {
    if (!live || h >= o.heads) return make_uint4(0, 0, 0, 0);
    const __nv_bfloat16* s = x + static_cast<int64_t>(h) * d;
    if constexpr (!HALF) return *reinterpret_cast<const uint4*>(s + at0);
    const uint2 a = *reinterpret_cast<const uint2*>(s + at0), b = *reinterpret_cast<const uint2*>(s + at1);
    return make_uint4(a.x, a.y, b.x, b.y);
  };
#pragma unroll
  for (int i = 0; i < V; ++i) raw[i] = load(head0 + i * heads_step);

  // the block's tokens: all its rows' (of the last block, those that there are)
  const int toks = MULTI ? 1 : static_cast<int>(min(p.n, (row0 + 7) / tensors + 1) - tok0);
  for (int i = threadIdx.x; i < toks * pairs; i += blockDim.x) {
    const int k = i / pairs, j = i - k * pairs;
    const int axis = j < p.axis_end[0] ? 0 : j < p.axis_end[1] ? 1 : 2;
    const int64_t pos = static_cast<int64_t>(p.pos[axis * p.n + tok0 + k]) + (axis == 0 ? p.pos0 : 0);
    const float a = static_cast<float>(static_cast<int32_t>(turn_fraction(pos, p.steps[j]))) *
                    1.46291807926715968105e-9f;   // 2 pi / 2^32
    table[k][j] = make_float2(p.factor * __cosf(a), p.factor * __sinf(a));
  }
  __syncthreads();
  if (row >= n_rows) return;   // whole warps, and no barrier follows where a block has several rows
  float2 cs[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) cs[j] = j < turned ? table[MULTI ? 0 : tok - tok0][4 * c + j] : make_float2(1.f, 0.f);

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
    rstd = rsqrtf(s / static_cast<float>(o.heads * d) + o.eps);   // off by 2^-22.9 at most
  }
  float w[8];
  auto weight = [&](const float* from) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(from + at0)), b = __ldg(reinterpret_cast<const float4*>(from + at1));
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  };
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = 1.f;
  if (o.norm == ISPA_QK_NORM_HEAD && o.weight && live) weight(o.weight);
  const float inv_d = 1.f / static_cast<float>(d);

  auto finish = [&](const uint4& v, int h) {
    float f[8];
    unpack8(v, f);
    if (o.norm == ISPA_QK_NORM_HEAD) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(f[e], f[e], s);
      const float r = rsqrtf(fmaf(group_reduce<SumOp>(s, lph), inv_d, o.eps));
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= r * w[e];
    } else if (o.norm == ISPA_QK_NORM_TOKEN) {
      if (o.weight && live && h < o.heads) weight(o.weight + static_cast<int64_t>(h) * d);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= rstd * w[e];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int a = HALF ? j : 2 * j, b = HALF ? 4 + j : 2 * j + 1;
      const float u = f[a], q = f[b];
      if (j < turned) {   // the others pass as they are, infinities too
        f[a] = fmaf(cs[j].x, u, -cs[j].y * q);
        f[b] = fmaf(cs[j].y, u, cs[j].x * q);
      }
    }
    if (live && h < o.heads) {
      __nv_bfloat16* to = out + static_cast<int64_t>(h) * d;
      const uint4 g = pack8(f);
      if constexpr (!HALF) {
        *reinterpret_cast<uint4*>(to + at0) = g;
      } else {
        *reinterpret_cast<uint2*>(to + at0) = make_uint2(g.x, g.y);
        *reinterpret_cast<uint2*>(to + at1) = make_uint2(g.z, g.w);
      }
    }
  };
  // Every lane of a warp goes round alike (the head's sum needs all of them): the step counts from the first head.
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
cudaError_t launch_layout(const RopeParams& p, int sms, cudaStream_t s) {
  int heads = p.rows[0].heads;
  if (p.n_rows > 1 && p.rows[1].heads > heads) heads = p.rows[1].heads;
  const int steps = (heads * p.lanes_per_head + 31) / 32;   // vectors a lane of one warp takes
  const int64_t rows = p.n * p.n_rows;
  const auto go = [&](auto kernel, int threads, int rows_per_block) {
    const int64_t blocks = (rows + rows_per_block - 1) / rows_per_block;
    return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks)), dim3(threads), 0, s, p);
  };
  if (rows > 8 * sms) {
    if (steps <= 2) return go(rope_kernel<2, HALF, false>, 256, 8);
    if (steps <= 6) return go(rope_kernel<6, HALF, false>, 256, 8);
    if (steps <= 12) return go(rope_kernel<12, HALF, false>, 256, 8);
    return go(rope_kernel<20, HALF, false>, 256, 8);
  }
  if (steps <= 16) return go(rope_kernel<1, HALF, true>, 32 * steps, 1);
  if (steps <= 32) return go(rope_kernel<2, HALF, true>, 32 * ((steps + 1) / 2), 1);
  return go(rope_kernel<4, HALF, true>, 32 * (steps <= 64 ? (steps + 3) / 4 : 16), 1);
}

}  // namespace

cudaError_t launch_rope(const RopeParams& p, bool half, cudaStream_t s) {
  int dev = 0, sms = 152;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return half ? launch_layout<true>(p, sms, s) : launch_layout<false>(p, sms, s);
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
