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
// Memory bounds it: x, y and the results cross HBM once, the modulation vectors stay in L1 and L2.  A row lives in
// registers from its load to its store, eight values (16 bytes of bf16) a thread and step, so the second pass of the
// variance and the maximum of the codes cost no traffic.  Everything between load and store is fp32; x is rounded to
// its own type first and h is taken from the rounded value, the one that the next reader of x sees.
#include <cuda_runtime.h>
#include <stdint.h>

#include "internal.h"
#include "pdl.cuh"
#include "rows.cuh"

namespace ispa {

namespace {

template <bool MULTI>
struct Reducer {
  float (*red)[32];
  int warps, slot = 0;
  template <typename Op>
  __device__ __forceinline__ float all(float v) {
    if constexpr (!MULTI) {
      return warp_reduce<Op>(v);
    } else {
      v = block_reduce<Op>(v, warps, red, slot);
      slot ^= 1;
      return v;
    }
  }
};

// The norm of a row that the threads hold as V vectors of eight, in place.
template <int V, bool MULTI>
__device__ __forceinline__ void norm_row(float (&v)[V][8], const ispa_norm& n, int nv, int dim, int t, int step,
                                         Reducer<MULTI>& r) {
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

__device__ __forceinline__ uint32_t pack_i8x4(const float* f) {
  uint32_t r = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) r |= (static_cast<uint32_t>(__float2int_rn(f[e])) & 0xFFu) << (8 * e);
  return r;
}

// MULTI: one row a block; else one row a warp.  Block (32 * warps of a row, rows of a block).
template <int V, bool MULTI, bool XF32, bool RES>
__global__ void __launch_bounds__(MULTI ? 512 : 256) norm_kernel(const __grid_constant__ NormParams p) {
  __shared__ float red[2][32];
  pdl_wait();
  pdl_trigger();
  const int64_t row = MULTI ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y;
  if (row >= p.rows) return;   // a whole warp; blocks of one row have none
  const int t = threadIdx.x, step = blockDim.x, nv = p.dim / 8;
  Reducer<MULTI> r{red, step >> 5};
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
    norm_row<V, MULTI>(y, p.post, nv, p.dim, t, step, r);
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

  norm_row<V, MULTI>(x, p.pre, nv, p.dim, t, step, r);
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
  const float inv = amax == 0.f ? 1.f : __fdiv_rn(top, amax);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = t + i * step;
    if (c < nv) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = __fmul_rn(x[i][e], inv);
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.out) + base + 8 * c) =
          p.format == ISPA_ROWS_E4M3
              ? make_uint2(pack_e4m3x4(x[i][0], x[i][1], x[i][2], x[i][3]),
                           pack_e4m3x4(x[i][4], x[i][5], x[i][6], x[i][7]))
              : make_uint2(pack_i8x4(x[i]), pack_i8x4(x[i] + 4));
    }
  }
  if (t == 0) p.out_scale[row] = amax == 0.f ? 1.f : __fdiv_rn(amax, top);
}

template <bool XF32, bool RES>
cudaError_t launch_typed(const NormParams& p, int sms, cudaStream_t s) {
  const int nv = p.dim / 8;
  const auto go = [&](auto kernel, int warps, int rows) {
    const int64_t blocks = (p.rows + rows - 1) / rows;
    return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks)), dim3(32 * warps, rows), 0, s, p);
  };
  if (p.rows > 4 * sms && nv <= 256) {
    if (nv <= 64) return go(norm_kernel<2, false, XF32, RES>, 1, 8);
    if (nv <= 128) return go(norm_kernel<4, false, XF32, RES>, 1, 8);
    if (nv <= 192) return go(norm_kernel<6, false, XF32, RES>, 1, 8);
    return go(norm_kernel<8, false, XF32, RES>, 1, 8);
  }
  const int warps = (nv + 31) / 32;
  if (warps <= 16) return go(norm_kernel<1, true, XF32, RES>, warps, 1);
  if (warps <= 32) return go(norm_kernel<2, true, XF32, RES>, (warps + 1) / 2, 1);
  if (warps <= 64) return go(norm_kernel<4, true, XF32, RES>, (warps + 3) / 4, 1);
  return go(norm_kernel<8, true, XF32, RES>, (warps + 7) / 8, 1);
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
