// Pieces shared by the kernels that work row by row (norm.cu, rope.cu): rows as vectors of eight
// values a thread, in fp32 once loaded, and sums over a warp or over the warps of a block.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "forms.h"
#include "ptx.cuh"

namespace ispa {

// Eight bf16 values (one 16-byte word) as fp32, and back (round to nearest even).
__device__ __forceinline__ void unpack8(const uint4& w, float* f) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = __uint_as_float(u[e] << 16);
    f[2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                    pack_bf16x2(f[6], f[7]));
}
// Two fp32 operations an instruction, each rounded to nearest.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return r;
}
// Eight consecutive fp32 values of a read-only array (16-byte aligned).
__device__ __forceinline__ void load8(const float* __restrict__ p, float* f) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}

// The larger of two values; NaN if one of them is NaN, so that a row that holds one cannot pass for a finite row.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Below this largest magnitude a group counts as all zeros: the quotient 448 / amax (127 / amax) would be infinite and
// amax / 448 lose bits of its mantissa.  Not for NaN.
constexpr float kTinyGroup = 6.0185310762101e-36f;   // 2^-117
__device__ __forceinline__ float code_factor(float amax, float top) {
  return amax < kTinyGroup ? 1.f : __fdiv_rn(top, amax);
}
__device__ __forceinline__ float code_scale(float amax, float top) {
  return amax < kTinyGroup ? 1.f : __fdiv_rn(amax, top);
}

// Four values of magnitude 127 at most, each rounded to the nearest even integer, as bytes.  Added to 1.5 * 2^23, whose
// unit is one, a value leaves its integer in the low bits: an addition each and three byte permutes, where conversions
// run at an eighth of that rate (int8 codes of 4680 x 5120 bf16 values 17.7 -> 14.7 us).
constexpr float kToInteger = 12582912.f;
__device__ __forceinline__ uint32_t low_bytes(float a, float b, float c, float d) {
  return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040),
                     __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t pack_i8x4(const float* f) {
  return low_bytes(__fadd_rn(f[0], kToInteger), __fadd_rn(f[1], kToInteger), __fadd_rn(f[2], kToInteger),
                   __fadd_rn(f[3], kToInteger));
}
// Of h * inv, rounded once.
__device__ __forceinline__ uint32_t pack_i8x4(const float* h, float inv) {
  return low_bytes(fmaf(h[0], inv, kToInteger), fmaf(h[1], inv, kToInteger), fmaf(h[2], inv, kToInteger),
                   fmaf(h[3], inv, kToInteger));
}
__device__ __forceinline__ uint32_t pack_e4m3x4(const float* h, float inv) {
  return pack_e4m3x4(__fmul_rn(h[0], inv), __fmul_rn(h[1], inv), __fmul_rn(h[2], inv), __fmul_rn(h[3], inv));
}

// The e4m3 quantisers keep every group whose quotient 448 / amax fp32 holds; up to 448 * 2^-128 it does not, and the
// zeros of such a group would become NaN.
constexpr float kTinyE4M3Group = 1.316553672920962e-36f;   // 7 * 2^-122

struct SumOp {
  static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct MaxOp {
  static __device__ __forceinline__ float of(float a, float b) { return max_nan(a, b); }
};

// Op over the lanes of a group of `lanes` (a power of two) neighbouring lanes; every lane gets it.
template <typename Op>
__device__ __forceinline__ float group_reduce(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v = Op::of(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
template <typename Op>
__device__ __forceinline__ float warp_reduce(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = Op::of(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
// The largest of a warp's values, none of them negative: their order is their bits', NaN above all (one instruction,
// where the shuffles of the sums take ten).
__device__ __forceinline__ float warp_max(float v) {
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
}
// Op over the block's `warps` warps (at most 32); every thread gets it.  `slot` (0 or 1) alternates from one call of
// a kernel to the next, so that one barrier a call is enough: a slot is written again only after the barrier of the
// call in between, which every thread reaches after its reads.
template <typename Op>
__device__ __forceinline__ float block_reduce(float v, int warps, float (*red)[32], int slot) {
  v = warp_reduce<Op>(v);
  if ((threadIdx.x & 31) == 0) red[slot][threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[slot][0];
  for (int i = 1; i < warps; ++i) v = Op::of(v, red[slot][i]);
  return v;
}

// A team of `warps` warps with its own named barrier and its own part of shared memory.
struct Team {
  float2* red;   // [2][TEAM_WARPS]
  int warps, barrier, slot;
  __device__ __forceinline__ void sync() const {
    if (warps > 1) asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(32 * warps) : "memory");
    else __syncwarp();
  }
  // Every warp's `v` to the lanes i with i % TEAM_WARPS = its number, zeros where there is no such warp.
  __device__ __forceinline__ float2 gather(float2 v) {
    float2* r = red + slot * TEAM_WARPS;
    slot ^= 1;   // written again after the barrier of the call in between
    const int i = threadIdx.x & (TEAM_WARPS - 1);
    if ((threadIdx.x & 31) == 0) r[threadIdx.x >> 5] = v;
    sync();
    return i < warps ? r[i] : make_float2(0.f, 0.f);
  }
};

}  // namespace ispa
