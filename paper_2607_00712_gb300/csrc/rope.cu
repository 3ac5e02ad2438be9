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
// 2^-12 of a bf16 rounding step of the largest value.
//
// Memory bounds it: each value crosses HBM once in and once out.
//
//   rope_stream_kernel   many tokens: a team of warps a token, queries and keys, with its angles made once
//   rope_kernel          few tokens, or rows too long for shared memory: a block for a token's queries or keys
//
// A thread takes eight features of one head per step: eight neighbours, or four and the four that they turn with, so
// that no pair is spread over two lanes.  A warp's lanes are dealt to heads in groups of a power of two, so a lane
// meets the same features, angles and weights in every head.
//
// Queries and keys of 4680 x 40 heads of 128, norm over the token: 39.0 us, 72 % of the measured copy rate (33.5
// without the norm); 12 heads 15.2 us, 13.4 with a norm per head, of which 6 are the start (angles, weights); one token
// 2.0 us.  Angles made by every warp for itself cost more than its heads: 69 us, and 58 for 3117 tokens of 24 and 8
// heads in the half layout (15.4 now); a warp a token with its row in registers 77 (164 registers, too few warps).
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "forms.h"
#include "internal.h"
#include "pdl.cuh"
#include "rows.cuh"

namespace ispa {

namespace {

// The upper 32 bits of the 64-bit product's lower half: the position's fraction of a turn in units of 2^-32.
__device__ __forceinline__ uint32_t turn_fraction(uint64_t pos, uint64_t step) {
  return static_cast<uint32_t>((pos * step) >> 32);
}

// What a lane does in every head it meets: features at0 .. + 3 and at1 .. + 3, pairs 4 c .. 4 c + 3, of which the first
// `turned` turn.
template <bool HALF>
struct Lane {
  int c, at0, at1, turned;
  bool live;
  __device__ __forceinline__ Lane(int lane, const RopeParams& p) {
    c = lane & (p.lanes_per_head - 1);
    live = 8 * c < p.head_dim;
    at0 = !HALF ? 8 * c : 4 * c < p.pairs ? 4 * c : 8 * c;
    at1 = HALF && 4 * c < p.pairs ? p.pairs + 4 * c : at0 + 4;
    turned = min(4, max(0, p.pairs - 4 * c));
  }
  __device__ __forceinline__ uint4 load(const __nv_bfloat16* head) const {
    if constexpr (!HALF) {
      return *reinterpret_cast<const uint4*>(head + at0);
    } else {
      const uint2 a = *reinterpret_cast<const uint2*>(head + at0), b = *reinterpret_cast<const uint2*>(head + at1);
      return make_uint4(a.x, a.y, b.x, b.y);
    }
  }
  __device__ __forceinline__ void store(__nv_bfloat16* head, const float* f) const {
    const uint4 g = pack8(f);
    if constexpr (!HALF) {
      *reinterpret_cast<uint4*>(head + at0) = g;
    } else {
      *reinterpret_cast<uint2*>(head + at0) = make_uint2(g.x, g.y);
      *reinterpret_cast<uint2*>(head + at1) = make_uint2(g.z, g.w);
    }
  }
  __device__ __forceinline__ void weight(const float* from, float* w) const {
    const float4 a = *reinterpret_cast<const float4*>(from + at0), b = *reinterpret_cast<const float4*>(from + at1);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  }
  __device__ __forceinline__ void turn(float* f, const float2* cs) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int a = HALF ? j : 2 * j, b = HALF ? 4 + j : 2 * j + 1;
      const float u = f[a], q = f[b];
      if (j < turned) {   // the others pass as they are, infinities too
        f[a] = fmaf(cs[j].x, u, -cs[j].y * q);
        f[b] = fmaf(cs[j].y, u, cs[j].x * q);
      }
    }
  }
};

// The kernels whose first tensor, the keys, goes into a ring, as codes or as bf16.
struct RopeCodesParams : RopeAppendParams {};
template <typename Params>
constexpr bool kRing = !std::is_same_v<Params, RopeParams>;
template <typename Params>
constexpr bool kCodes = std::is_same_v<Params, RopeCodesParams>;

// A token's place in the ring: row of head 0.
__device__ __forceinline__ int64_t ring_row(const RopeAppendParams& p, int tok) {
  const int f = quotient(tok, p.by_P);
  return static_cast<int64_t>(p.slot[f]) * p.P + (tok - f * p.P);
}
// Eight features of a head as codes of f * inv.
template <bool HALF>
__device__ __forceinline__ void store_codes(uint8_t* head, const Lane<HALF>& ln, const float* f, float inv) {
  const uint32_t a = pack_e4m3x4(f, inv), b = pack_e4m3x4(f + 4, inv);
  if constexpr (!HALF) {
    *reinterpret_cast<uint2*>(head + ln.at0) = make_uint2(a, b);
  } else {
    *reinterpret_cast<uint32_t*>(head + ln.at0) = a;
    *reinterpret_cast<uint32_t*>(head + ln.at1) = b;
  }
}
// Tokens first .. last - 1 of the values into the ring, by all threads of the block.
__device__ __forceinline__ void copy_values(const RopeAppendParams& p, int first, int last) {
  const int wph = p.head_dim / 8, shift = p.head_dim == 128 ? 4 : 3, words = p.rows[0].heads * wph;
  const int total = (last - first) * words;
  const uint4* from = reinterpret_cast<const uint4*>(p.v) + first * (p.v_stride / 8);
  uint4* to = reinterpret_cast<uint4*>(p.v_ring);
  for (int i0 = threadIdx.x; i0 < total; i0 += 4 * blockDim.x) {
    uint4 w[4];
    int64_t at[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + u * blockDim.x, tok = quotient(i, p.by_words), c = i - tok * words, h = c >> shift;
      at[u] = -1;
      if (i >= total) continue;
      w[u] = __ldcs(from + tok * (p.v_stride / 8) + c);
      at[u] = (h * p.ring_tok + ring_row(p, first + tok)) * wph + (c & (wph - 1));
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (at[u] >= 0) to[at[u]] = w[u];
  }
}

__device__ __forceinline__ float sum_squares(const uint4& w, float s) {
  float f[8];
  unpack8(w, f);
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(f[e], f[e], s);
  return s;
}

// Cosine and sine (times the factor) of a pair at position pos + pos0 of its axis; all of it modulo 2^64.
__device__ __forceinline__ float2 cos_sin(int32_t pos, int64_t pos0, uint64_t step, float factor) {
  const uint64_t at = static_cast<uint64_t>(static_cast<int64_t>(pos)) + static_cast<uint64_t>(pos0);
  const float a = static_cast<float>(static_cast<int32_t>(turn_fraction(at, step))) *
                  1.46291807926715968105e-9f;   // 2 pi / 2^32
  return make_float2(factor * __cosf(a), factor * __sinf(a));
}
__device__ __forceinline__ int axis_of(int pair, const RopeParams& p) {
  return pair < p.axis_end[0] ? 0 : pair < p.axis_end[1] ? 1 : 2;
}

// ------------------------------------------------------------ few rows
// A block a row (a token's queries or keys); V: vectors a thread holds at once.  blockIdx.y: which of the two.
template <int V, bool HALF, typename Params>
__global__ void __launch_bounds__(512) rope_kernel(const __grid_constant__ Params p) {
  __shared__ float2 table[128];
  __shared__ float red[2][32];
  const int64_t tok = blockIdx.x;
  const RopeRowsParams& o = p.rows[kRing<Params> ? min(static_cast<int>(blockIdx.y), p.n_rows - 1) : blockIdx.y];
  const int lph = p.lanes_per_head, d = p.head_dim;
  const Lane<HALF> ln(threadIdx.x, p);
  const int heads_step = blockDim.x / lph, head0 = threadIdx.x / lph;
  pdl_wait();
  pdl_trigger();

  int64_t row = 0;       // ring row of the keys
  bool keys = false;
  if constexpr (kRing<Params>) {
    row = ring_row(p, static_cast<int>(tok));
    keys = blockIdx.y == 0;
    if (static_cast<int>(blockIdx.y) == p.n_rows) {
      copy_values(p, static_cast<int>(tok), static_cast<int>(tok) + 1);
      return;
    }
  }
  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(o.x) + tok * o.x_stride;
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(o.out) + tok * o.out_stride;
  uint4 raw[V];
  auto load = [&](int h) {
    return ln.live && h < o.heads ? ln.load(x + static_cast<int64_t>(h) * d) : make_uint4(0, 0, 0, 0);
  };
#pragma unroll
  for (int i = 0; i < V; ++i) raw[i] = load(head0 + i * heads_step);
  for (int j = threadIdx.x; j < p.pairs; j += blockDim.x) {
    const int axis = axis_of(j, p);
    table[j] = cos_sin(p.pos[axis * p.n + tok], axis == 0 ? p.pos0 : 0, p.steps[j], p.factor);
  }
  float s = 0.f;
  if (o.norm == ISPA_QK_NORM_TOKEN) {
#pragma unroll
    for (int i = 0; i < V; ++i) s = sum_squares(raw[i], s);
    for (int h = head0 + V * heads_step; h < o.heads; h += heads_step) s = sum_squares(load(h), s);
  }
  s = block_reduce<SumOp>(s, blockDim.x >> 5, red, 0);   // the table is there too
  const float rstd = rsqrtf(s / static_cast<float>(o.heads * d) + o.eps);   // off by 2^-22.9 at most
  float2 cs[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) cs[j] = j < ln.turned ? table[4 * ln.c + j] : make_float2(1.f, 0.f);
  float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
  if (o.norm == ISPA_QK_NORM_HEAD && o.weight && ln.live) ln.weight(o.weight, w);

  auto finish = [&](const uint4& v, int h) {
    float f[8], r = rstd;
    unpack8(v, f);
    if (o.norm == ISPA_QK_NORM_HEAD)
      r = rsqrtf(group_reduce<SumOp>(sum_squares(v, 0.f), lph) / static_cast<float>(d) + o.eps);
    else if (o.norm == ISPA_QK_NORM_TOKEN && o.weight && ln.live && h < o.heads)
      ln.weight(o.weight + static_cast<int64_t>(h) * d, w);
    if (o.norm != ISPA_QK_NORM_NONE) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= r * w[e];
    }
    ln.turn(f, cs);
    if (ln.live && h < o.heads) {
      if (kRing<Params> && keys) {
        if constexpr (kRing<Params>) {
          const int64_t at = (static_cast<int64_t>(h) * p.ring_tok + row) * d;
          if constexpr (kCodes<Params>)
            store_codes(static_cast<uint8_t*>(p.k_ring) + at, ln, f, __fdiv_rn(1.f, __ldg(p.k_scale + h)));
          else
            ln.store(static_cast<__nv_bfloat16*>(p.k_ring) + at, f);
        }
      } else {
        ln.store(out + static_cast<int64_t>(h) * d, f);
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

// ------------------------------------------------------------ many tokens
constexpr uint64_t R_DRAIN_NS = 200ull * 1000 * 1000;

// Block (32 * warps of a team, teams), one an SM; block b takes tokens [b, b + 1) * per_block, its teams in turn.  A
// token's queries and keys come through shared memory by bulk copies, a team's next token while it works on one;
// weights of a norm over the token's heads stand there too, the eight of a lane in two planes, so that a warp reads
// whole lines.  NORM: of queries and keys alike.  FULL: every feature turns and a head's lanes are a power of two.
// STAGES: tokens of a team in shared memory, one where all of the block's tokens fit at once.
template <bool HALF, int NORM, bool FULL, int STAGES, typename Params>
__global__ void __launch_bounds__(1024, 1) rope_stream_kernel(const __grid_constant__ Params p, int per_block) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int abort_word;
  const int t = threadIdx.x, threads = blockDim.x, teams = blockDim.y, d = p.head_dim, lph = p.lanes_per_head;
  const Lane<HALF> ln(t, p);
  const bool live = FULL || ln.live;
  const int heads_step = threads / lph, head0 = t / lph, vecs = d / 8;
  // weights [queries, keys][plane][vectors of a row], the teams' tokens [2][queries, keys], tables, barriers,
  // reductions
  constexpr bool kWeights = NORM == ISPA_QK_NORM_TOKEN;
  const int n0 = p.rows[0].heads * d, n1 = p.n_rows > 1 ? p.rows[1].heads * d : 0, r_bytes = 2 * (n0 + n1);
  const int w_bytes = kWeights ? 4 * (n0 + n1) : 0;
  uint8_t* const rows = smem + w_bytes + STAGES * r_bytes * threadIdx.y;
  uint8_t* at = smem + w_bytes + STAGES * r_bytes * teams;
  const int table_bytes = (8 * p.pairs + 15) & ~15;   // a team's cosines and sines
  float2* const table = reinterpret_cast<float2*>(at + table_bytes * threadIdx.y);
  at += table_bytes * teams;
  const uint32_t full = smem_u32(at + 16 * threadIdx.y);
  at += 16 * teams;
  Team tm{reinterpret_cast<float2*>(at) + threadIdx.y * 2 * TEAM_WARPS, threads >> 5,
          1 + static_cast<int>(threadIdx.y), 0};
  if (t == 0) {
    mbar_init(full, 1);
    mbar_init(full + 8, 1);
    abort_word = 0;
    fence_mbar_init();
  }
  __syncthreads();
  if constexpr (kRing<Params>) {
    if (p.wait_first) pdl_wait();
  } else {
    pdl_wait();
  }
  pdl_trigger();
  const WaitCtx wc{&abort_word, p.status, p.wait_limit_ns};
  const int first = blockIdx.x * per_block;   // tokens are fewer than 2^30
  const int last = static_cast<int>(min(static_cast<int64_t>(first) + per_block, p.n));
  const auto stage_of = [&](uint32_t i) { return i & (STAGES - 1); };
  const auto parity_of = [&](uint32_t i) { return (i >> (STAGES - 1)) & 1; };
  auto fetch = [&](int tok, int stage) {
    mbar_arrive_expect_tx(full + 8 * stage, r_bytes);
    const uint32_t dst = smem_u32(rows) + stage * r_bytes;
    bulk_load(dst, static_cast<const __nv_bfloat16*>(p.rows[0].x) + tok * p.rows[0].x_stride, 2 * n0, full + 8 * stage);
    if (n1)
      bulk_load(dst + 2 * n0, static_cast<const __nv_bfloat16*>(p.rows[1].x) + tok * p.rows[1].x_stride, 2 * n1,
                full + 8 * stage);
  };
  int tok = first + threadIdx.y;
  uint32_t issued = 0;   // (thread 0) tokens that it has sent for
  bool ok = true;
  if (t == 0 && tok < last) fetch(tok, stage_of(issued++));
  // This thread's pairs t, t + threads, ...: their steps, and their position at the team's next token.
  uint64_t step[4];
  int pos[4];
  auto positions = [&](int k) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (t + j * threads < p.pairs && k < last) pos[j] = __ldg(p.pos + axis_of(t + j * threads, p) * p.n + k);
  };
#pragma unroll
  for (int j = 0; j < 4; ++j) step[j] = t + j * threads < p.pairs ? p.steps[t + j * threads] : 0;
  positions(tok);
  // codes: with 1 / scale of the key's head in its weights, and none behind the rotation
  auto copy_weights = [&](const float* from, float4* to, int n, bool codes) {
    for (int k = threadIdx.y * threads + t; k < n / 8; k += threads * teams) {   // vector k of a row
      const int c = k % vecs;
      const Lane<HALF> of(c, p);
      const float* w = from + (k - c) * 8;
      float4 a = from ? __ldg(reinterpret_cast<const float4*>(w + of.at0)) : make_float4(1.f, 1.f, 1.f, 1.f);
      float4 b = from ? __ldg(reinterpret_cast<const float4*>(w + of.at1)) : make_float4(1.f, 1.f, 1.f, 1.f);
      if constexpr (kCodes<Params>) {
        if (codes) {
          const float inv = __fdiv_rn(1.f, __ldg(p.k_scale + k / vecs));
          const auto by = [&](float v) {   // finite, so that a key of zero stays one
            v *= inv;
            return fabsf(v) == INFINITY ? copysignf(3.402823466e38f, v) : v;
          };
          a = make_float4(by(a.x), by(a.y), by(a.z), by(a.w));
          b = make_float4(by(b.x), by(b.y), by(b.z), by(b.w));
        }
      }
      to[k] = a;
      to[n / 8 + k] = b;
    }
  };
  if constexpr (kWeights) {
    copy_weights(p.rows[0].weight, reinterpret_cast<float4*>(smem), n0, true);
    if (n1) copy_weights(p.rows[1].weight, reinterpret_cast<float4*>(smem + 4 * n0), n1, false);
  }
  __syncthreads();
  const float inv_n0 = 1.f / static_cast<float>(n0), inv_n1 = n1 ? 1.f / static_cast<float>(n1) : 0.f;
  const float inv_d = 1.f / static_cast<float>(d);

  // the sum of a tensor's squares
  auto squares = [&](const uint8_t* src, int heads) {
    float q = 0.f;
    if (live) {
      const __nv_bfloat16* x = reinterpret_cast<const __nv_bfloat16*>(src) + head0 * d;
#pragma unroll 2
      for (int h = head0; h < heads; h += heads_step, x += heads_step * d) q = sum_squares(ln.load(x), q);
    }
    return warp_reduce<SumOp>(q);
  };
  // norm, rotation and way out of a tensor; cs: the pairs' cosines and sines, with 1 / root of a norm over the token in
  // them, r that factor for what passes
  auto finish = [&](const uint8_t* src, const RopeRowsParams& o, const float4* planes, int n, const float2* cs, float r,
                    bool first) {
    // keys (the first tensor) that go into the ring: head 0 of the token, and the step from one head to the next
    uint8_t* codes = nullptr;
    int64_t step_out = heads_step * d;
    const __nv_bfloat16* x = reinterpret_cast<const __nv_bfloat16*>(src) + head0 * d;
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(o.out) + tok * o.out_stride + head0 * d;
    if constexpr (kRing<Params>) {
      if (first) {
        const int64_t at = (head0 * p.ring_tok + ring_row(p, tok)) * d;
        step_out = heads_step * p.ring_tok * d;
        if constexpr (kCodes<Params>) codes = static_cast<uint8_t*>(p.k_ring) + at;
        else out = static_cast<__nv_bfloat16*>(p.k_ring) + at;
      }
    }
    const float4* wp = planes + head0 * vecs + ln.c;
    float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    if (NORM == ISPA_QK_NORM_HEAD && o.weight && live) ln.weight(o.weight, w);
    // every lane goes round alike: a head's sum needs all of them
    // Four heads of a lane side by side where each has a sum to wait for (3117 tokens of 24 and 8 heads 18.0 -> 16.9
    // us, 1560 of 160 and 40 44 -> 38); the others are slower so (4680 x 2 x 5120 39.7 -> 43).
    constexpr int kAhead = NORM == ISPA_QK_NORM_HEAD ? 4 : 2;
    int h = head0;
#pragma unroll kAhead
    for (int left = o.heads; left > 0; left -= heads_step) {
      const bool here = live && h < o.heads;
      float f[8];
      const uint4 raw = here ? ln.load(x) : make_uint4(0, 0, 0, 0);
      unpack8(raw, f);
      if constexpr (NORM == ISPA_QK_NORM_HEAD) {
        float q = sum_squares(raw, 0.f);
#pragma unroll
        for (int i = 16; i > 0; i >>= 1) {   // without a branch, so that the heads' shuffles run into one another
          const float other = __shfl_xor_sync(0xffffffffu, q, i);
          if (i < lph) q += other;
        }
        q = rsqrtf(fmaf(q, inv_d, o.eps));
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= q * w[e];
      }
      if constexpr (NORM == ISPA_QK_NORM_TOKEN) {
        if (here) {
          const float4 a = wp[0], b = wp[n / 8];
          f[0] *= a.x, f[1] *= a.y, f[2] *= a.z, f[3] *= a.w, f[4] *= b.x, f[5] *= b.y, f[6] *= b.z, f[7] *= b.w;
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int a = HALF ? j : 2 * j, b = HALF ? 4 + j : 2 * j + 1;
        const float u = f[a], v = f[b];
        if (FULL || j < ln.turned) {
          f[a] = fmaf(cs[j].x, u, -cs[j].y * v);
          f[b] = fmaf(cs[j].y, u, cs[j].x * v);
        } else if (NORM == ISPA_QK_NORM_TOKEN) {   // the others pass as they are, infinities too
          f[a] *= r;
          f[b] *= r;
        }
      }
      if (kCodes<Params> && first) {
        if constexpr (kCodes<Params>)
          if (here) store_codes(codes, ln, f, kWeights ? 1.f : __fdiv_rn(1.f, __ldg(p.k_scale + h)));
        codes += step_out;
      } else {
        if (here) ln.store(out, f);
        out += step_out;
      }
      h += heads_step;
      x += heads_step * d;
      wp += heads_step * vecs;
    }
  };

  uint32_t turn = 0;   // tokens that this team has begun
  for (; tok < last; tok += teams, ++turn) {
    const int stage = stage_of(turn);
    if (STAGES == 2 && t == 0 && ok && last - tok > teams)
      fetch(tok + teams, stage_of(issued++));   // all have read the last token there
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int pair = t + j * threads;
      if (pair < p.pairs) table[pair] = cos_sin(pos[j], axis_of(pair, p) == 0 ? p.pos0 : 0, step[j], p.factor);
    }
    positions(tok + teams);
    ok &= mbar_wait(full + 8 * stage, parity_of(turn), wc, 52, tok);   // a token that never comes: recorded
    const uint8_t* src = rows + stage * r_bytes;
    float2 s = make_float2(0.f, 0.f);
    if constexpr (NORM == ISPA_QK_NORM_TOKEN) {
      s.x = squares(src, p.rows[0].heads);
      if (n1) s.y = squares(src + 2 * n0, p.rows[1].heads);
    }
    if (NORM == ISPA_QK_NORM_TOKEN && tm.warps > 1) {   // also: the table is there
      const float2 all = tm.gather(s);
      s = make_float2(group_reduce<SumOp>(all.x, TEAM_WARPS), group_reduce<SumOp>(all.y, TEAM_WARPS));
    } else {
      tm.sync();
    }
    float2 cs[4], c1[4];
    float r0 = 1.f, r1 = 1.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) cs[j] = FULL || j < ln.turned ? table[4 * ln.c + j] : make_float2(1.f, 0.f);
    if constexpr (NORM == ISPA_QK_NORM_TOKEN) {
      r0 = rsqrtf(fmaf(s.x, inv_n0, p.rows[0].eps));   // off by 2^-22.9 at most
      r1 = rsqrtf(fmaf(s.y, inv_n1, p.rows[1].eps));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c1[j] = make_float2(cs[j].x * r0, cs[j].y * r0);
        if constexpr (!kRing<Params>) cs[j] = make_float2(cs[j].x * r1, cs[j].y * r1);
      }
      finish(src, p.rows[0], reinterpret_cast<const float4*>(smem), n0, c1, r0, true);
      if constexpr (kRing<Params>) {   // from the table once more: the first tensor needs the registers
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 v = FULL || j < ln.turned ? table[4 * ln.c + j] : make_float2(1.f, 0.f);
          cs[j] = make_float2(v.x * r1, v.y * r1);
        }
      }
      if (n1) finish(src + 2 * n0, p.rows[1], reinterpret_cast<const float4*>(smem + 4 * n0), n1, cs, r1, false);
    } else {
      finish(src, p.rows[0], nullptr, n0, cs, 1.f, true);
      if (n1) finish(src + 2 * n0, p.rows[1], nullptr, n1, cs, 1.f, false);
    }
    tm.sync();   // the token's stage and the table are free
    if (STAGES == 1 && t == 0 && ok && last - tok > teams) fetch(tok + teams, stage_of(issued++));
  }
  if (t == 0 && !ok)   // after a timeout: nothing in flight when the block leaves
    for (uint32_t i = issued < STAGES ? 0 : issued - STAGES; i < issued; ++i)
      mbar_wait_drain(full + 8 * stage_of(i), parity_of(i), R_DRAIN_NS);
  if constexpr (kRing<Params>)
    if (!p.wait_first) pdl_wait();   // the values' launch completes before this one does
}

// The values of many tokens, in a launch of their own in front of the keys', which starts as soon as this one's blocks
// have the kernel before behind them and runs beside it.  In the teams' loop the copies cost their registers: 4680
// tokens of 3 x 5120 with 8-bit keys 83 us against 50, of 3 x 1536 25.6 against 20.
__global__ void __launch_bounds__(256) values_kernel(const __grid_constant__ RopeAppendParams p, int per_block) {
  pdl_wait();
  pdl_trigger();
  const int first = blockIdx.x * per_block;
  copy_values(p, first, static_cast<int>(min(static_cast<int64_t>(first) + per_block, p.n)));
}

template <bool HALF, typename Params>
cudaError_t launch_layout(const Params& p, int sms, cudaStream_t s) {
  const int32_t heads[2] = {p.rows[0].heads, p.rows[1].heads}, norms[2] = {p.rows[0].norm, p.rows[1].norm};
  RopeForm f = rope_form(p.n, p.n_rows, heads, norms, p.head_dim, p.pairs, p.lanes_per_head, HALF, sms);
  if constexpr (kRing<Params>) {
    // Teams that have several tokens each make room for the values' block (see below): 4680 x 40 heads, norm per head,
    // 60 us with 25 warps and the values in front, 56 with 20 beside them; not without a norm (51 both ways), where
    // there is less to wait for.
    if (f.stream && p.v && norms[0] != ISPA_QK_NORM_NONE && f.tokens > f.teams && f.warps * f.teams > 24)
      f.teams = std::max(1, 24 / f.warps);
  }
  if (f.stream) {
    const auto go = [&](auto kernel) {
      cudaError_t e = set_smem_limit_once(reinterpret_cast<const void*>(kernel), R_SMEM);
      if (e != cudaSuccess) return e;
      Params q = p;
      if constexpr (kRing<Params>) {
        q.wait_first = p.v == nullptr;
        if (p.v) {
          // One block an SM where the keys' block leaves it room, so that both go on side by side: of a lane's 512
          // registers in a quarter of an SM, six warps with the keys' 64 and two with the 40 here (4680 x 40 heads, 20
          // warps, 50 us, 56 with eight blocks; with 25 warps 82 against 50), else as many as get through fastest.
          const bool beside = f.warps * f.teams <= 24;
          const int blocks = beside ? sms : 8 * sms, per = static_cast<int>((p.n + blocks - 1) / blocks);
          e = launch_pdl(values_kernel, dim3(static_cast<unsigned>((p.n + per - 1) / per)), dim3(256), 0, s, p, per);
          if (e != cudaSuccess) return e;
        }
      }
      return launch_pdl(kernel, dim3(static_cast<unsigned>((p.n + f.tokens - 1) / f.tokens)),
                        dim3(32 * f.warps, f.teams), f.smem, s, q, static_cast<int>(f.tokens));
    };
    const auto pick = [&](auto one, auto two) { return f.stages == 1 ? go(one) : go(two); };
    if (norms[0] == ISPA_QK_NORM_TOKEN)
      return f.full ? pick(rope_stream_kernel<HALF, ISPA_QK_NORM_TOKEN, true, 1, Params>,
                           rope_stream_kernel<HALF, ISPA_QK_NORM_TOKEN, true, 2, Params>)
                    : pick(rope_stream_kernel<HALF, ISPA_QK_NORM_TOKEN, false, 1, Params>,
                           rope_stream_kernel<HALF, ISPA_QK_NORM_TOKEN, false, 2, Params>);
    if (norms[0] == ISPA_QK_NORM_HEAD)
      return f.full ? pick(rope_stream_kernel<HALF, ISPA_QK_NORM_HEAD, true, 1, Params>,
                           rope_stream_kernel<HALF, ISPA_QK_NORM_HEAD, true, 2, Params>)
                    : pick(rope_stream_kernel<HALF, ISPA_QK_NORM_HEAD, false, 1, Params>,
                           rope_stream_kernel<HALF, ISPA_QK_NORM_HEAD, false, 2, Params>);
    return f.full ? pick(rope_stream_kernel<HALF, ISPA_QK_NORM_NONE, true, 1, Params>,
                         rope_stream_kernel<HALF, ISPA_QK_NORM_NONE, true, 2, Params>)
                  : pick(rope_stream_kernel<HALF, ISPA_QK_NORM_NONE, false, 1, Params>,
                         rope_stream_kernel<HALF, ISPA_QK_NORM_NONE, false, 2, Params>);
  }
  const auto go = [&](auto kernel) {
    int parts = p.n_rows;
    if constexpr (kRing<Params>) parts += p.v != nullptr;
    return launch_pdl(kernel, dim3(static_cast<unsigned>(p.n), parts), dim3(32 * f.warps), 0, s, p);
  };
  return f.vectors == 1   ? go(rope_kernel<1, HALF, Params>)
         : f.vectors == 2 ? go(rope_kernel<2, HALF, Params>)
                          : go(rope_kernel<4, HALF, Params>);
}

}  // namespace

cudaError_t launch_rope(const RopeParams& p, bool half, cudaStream_t s) {
  int dev = 0, sms = 152;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return half ? launch_layout<true>(p, sms, s) : launch_layout<false>(p, sms, s);
}

cudaError_t launch_rope_append(const RopeAppendParams& p, bool half, cudaStream_t s) {
  int dev = 0, sms = 152;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (p.k_scale) {
    const RopeCodesParams c{p};
    return half ? launch_layout<true>(c, sms, s) : launch_layout<false>(c, sms, s);
  }
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
