// Projection in 8-bit integers (W8A8, Sec. 4): out[t][n] = bf16(float(sum_k a[t][k] w[n][k]) a_scale[t] w_scale[n] +
// bias[n]) with the sum an exact 32-bit integer.
//
//   gemm_i8_kernel   many tokens: tensor cores
//   gemv_i8_kernel   few tokens: dp4a, bound by the weights' way from HBM
//
// The tensor cores of sm_103a have no integer form (tcgen05 kind::i8 does not exist there), and mma.sync's integer
// rate is a fraction of theirs.  But codes are exact in fp16, their products are integers up to 2^14, and the sum of
// 1024 of them stays within 2^24, where every integer is exact in the fp32 accumulator.  So codes go through
// kind::f16, and every 1024 of the contraction the accumulator is read back and added up in int32: the result is the
// integer sum, bit for bit, whatever the tile shape.  Against fp8 digits (two e4m3 digits a code, three or four
// products at twice the rate) this is the cheapest exact form: one product at the fp16 rate.
//
// GEMM: persistent CTAs over 128 x 128 tiles, pairs over 256 x 192 or 256 x 128 tiles (cta_group::2), or clusters that
// share a tile's contraction, whichever gives the shortest estimated run.  Per block of 64 codes: warp 0 has TMA bring
// the bytes as they are; four of twelve converter warps turn them into fp16 (byte u = code + 128 beside 0x64 is the
// fp16 number 1024 + u, less 1152 the code: a permute and a subtraction for two codes), activations into TMEM, weights
// into shared memory in the 128-byte swizzle that the UMMAs read; warp 1 issues the UMMAs; eight warps read the
// accumulators back, two sets in TMEM in turn.  Their int32 sums take up to 96 registers a thread, so the warpgroups
// share the registers out anew (setmaxnreg).  Every wait is bounded.
//
// 4680 x 5120 -> 5120 150.8 us, 1627 TFLOP/s, with operands and result in L2, 162 from and to HBM; 4680 x 1536 -> 4608
// 47.0 us; 61 x 5120 -> 640 9.1 us; one token of 1536 x 1536 1.9 us.  What bounds a long contraction is no single unit:
// a block of 192 columns takes 0.25 us where its UMMAs take 0.19, a team 0.47 us for a block (there are three), and the
// ring of four stages, from one block's conversion to the end of its UMMAs, 0.7 us; half of A's conversion left out
// gave 134 us, three quarters of the UMMAs 143.  On the way: one team of eight converter warps 405 us, four teams of
// two 218; the hand-over without an unrestricted release of cluster scope a block 168; A in TMEM, so that shared memory
// moves a third less, 225 in pairs of 192 with one lane in the TMA and UMMA roles; whole warps in these roles 159;
// twelve converter warps 157; sums of two runs in fp32 155; running stage counters 150.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "forms.h"
#include "internal.h"
#include "pdl.cuh"
#include "ptx.cuh"

namespace ispa {

namespace {

// ------------------------------------------------------------ few tokens
// out[t][n] of the sum (as fp32, rounded to nearest): the documented fp32 steps.
__device__ __forceinline__ float scaled(float s, float sa, float sw, float b) {
  return __fadd_rn(__fmul_rn(__fmul_rn(s, sa), sw), b);
}

// One warp: NC output channels and up to TT tokens.  Lane l takes the 16-byte words l, l + 32, ... of the rows.
// Block 8 warps; grid (ceil(Dout / (8 * NC)), ceil(T / TT)).
template <int TT, int NC>
__global__ void __launch_bounds__(256)
    gemv_i8_kernel(const int8_t* __restrict__ a, const float* __restrict__ a_scale, const int8_t* __restrict__ w,
                   const float* __restrict__ w_scale, const float* __restrict__ bias, int T, int D, int Dout,
                   __nv_bfloat16* __restrict__ out) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int n0 = (blockIdx.x * 8 + (threadIdx.x >> 5)) * NC, t0 = blockIdx.y * TT;
  if (n0 >= Dout) return;
  const int words = D / 16;
  int32_t acc[TT][NC] = {};
  for (int i = lane; i < words; i += 32) {
    int4 wv[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
      wv[c] = n0 + c < Dout ? __ldg(reinterpret_cast<const int4*>(w + static_cast<int64_t>(n0 + c) * D) + i)
                            : make_int4(0, 0, 0, 0);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int4 av = t0 + t < T ? __ldg(reinterpret_cast<const int4*>(a + static_cast<int64_t>(t0 + t) * D) + i)
                                 : make_int4(0, 0, 0, 0);
#pragma unroll
      for (int c = 0; c < NC; ++c)
        acc[t][c] = __dp4a(av.x, wv[c].x, __dp4a(av.y, wv[c].y, __dp4a(av.z, wv[c].z,
                                                                       __dp4a(av.w, wv[c].w, acc[t][c]))));
    }
  }
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      int32_t s = __reduce_add_sync(0xffffffffu, acc[t][c]);
      if (lane == (t * NC + c) % 32 && t0 + t < T && n0 + c < Dout)
        out[static_cast<int64_t>(t0 + t) * Dout + n0 + c] =
            __float2bfloat16_rn(scaled(__int2float_rn(s), a_scale[t0 + t], w_scale[n0 + c], bias ? bias[n0 + c] : 0.f));
    }
}

// ------------------------------------------------------------ many tokens
constexpr int I_EXACT = 1024 / IK;      // blocks whose sums the fp32 accumulator holds exactly
constexpr int I_CONV = 12, I_EPI = 8;   // converter and read-back warps
constexpr int I_TEAMS = I_CONV / 4;     // four converter warps, one per TMEM lane quarter, share a block
constexpr int I_THREADS = 32 * (4 + I_CONV + I_EPI);
constexpr int I_OUT_BLOCK = 32 * 64;
constexpr uint64_t I_DRAIN_NS = 200ull * 1000 * 1000;

template <int BN, bool PAIR>
struct ICfg {
  static constexpr int CTAS = PAIR ? 2 : 1;
  static constexpr int BR = BN / CTAS;              // this CTA's rows of B
  static constexpr int RAW = (IM + BR) * IK;        // bytes of a block as codes
  static constexpr int B16 = BR * 2 * IK;           // of its part of B as fp16
  // stages of fp16 (A in TMEM, B in shared memory) and of codes
  static constexpr int FST = 4, RST = BR == 128 ? 6 : 9;
  // A team waits for a stage of codes knowing that its own last block has landed, and for an fp16 stage knowing that
  // the UMMAs have read all blocks up to its own last one less FST.  Parities tell two uses of a stage apart, not
  // three: the stage's use before must be one that the team knows of.
  static_assert(RST % I_TEAMS == 0 && FST >= I_TEAMS, "parities stay unambiguous");
  static constexpr int A_COL = 512 - FST * IK / 2;  // TMEM columns of A's stages: two fp16 a column
  static_assert(2 * BN <= A_COL, "two accumulator sets and A fit in TMEM");
  static_assert(BN != 128 || PAIR || FST * B16 >= IM * BN * 4, "a split tile's sums fit into the fp16 stages");
  static constexpr int OFF_RAW = FST * B16;
  static constexpr int OFF_OUT = OFF_RAW + RST * RAW;
  static constexpr int OFF_SCALE = OFF_OUT + I_EPI * 2 * I_OUT_BLOCK;   // two blocks of 32 x 32 bf16 a read-back warp
  static constexpr int OFF_BAR = OFF_SCALE + I_EPI * BN * 4;           // w_scale and bias of a warp's BN / 2 columns
  static constexpr int N_BAR = 2 * RST + 2 * FST + 4 + 1;   // codes and fp16 full / empty, set full / empty, drain
  static constexpr int SMEM = OFF_BAR + N_BAR * 8 + 16;
  static_assert(SMEM > 116 * 1024 && SMEM <= 232448, "one CTA per SM");
  static_assert(B16 % 1024 == 0 && RAW % 512 == 0 && OFF_OUT % 512 == 0 && BR % 32 == 0, "shared memory layout");
  // fp16 operands (format 0), fp32 accumulator
  static constexpr uint32_t IDESC = (1u << 4) | (static_cast<uint32_t>(BN >> 3) << 17) |
                                    (static_cast<uint32_t>((IM * CTAS) >> 4) << 24);
  // Registers a thread after the split: the first four warps, converters, read-back warps (BN / 2 of theirs are sums).
  // Their sum over the warpgroups must not exceed what the kernel is launched with (checked at the launch).
  static constexpr int REGS_FIRST = 40, REGS_CONV = 56, REGS_EPI = 136;
  static constexpr int REGS_SUM = REGS_FIRST + I_CONV / 4 * REGS_CONV + I_EPI / 4 * REGS_EPI;
};

struct LinearParams {
  int32_t T, Dout, n_kb;
  int32_t n_mt, n_tiles;   // row tiles; all tiles (tile t: rows (t % n_mt), columns (t / n_mt))
  int32_t split;           // CTAs that share a tile's blocks (SPLIT)
  const float* a_scale;
  const float* w_scale;
  const float* bias;
  __nv_bfloat16* out;
  int* status;
  uint64_t wait_limit_ns;
};

// A converged warp's bounded wait (CLUSTER: for a barrier that the pair's other CTA arrives at too), the same answer in
// every lane; mbar_wait with the polling loop in line, because a kernel that shares its registers out anew cannot call
// functions.
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const WaitCtx& w, int site, int detail) {
  uint64_t t0 = 0;
  for (uint32_t i = 1;
       !__all_sync(0xffffffffu, CLUSTER ? mbar_try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity)); ++i) {
    if ((i & 63) == 0) {
      const uint64_t now = globaltimer_ns();
      if (t0 == 0) t0 = now;
      const bool late = now - t0 > w.limit_ns;
      if (late && (threadIdx.x & 31) == 0) {
        *w.abort = 1;
        record_error(w.status, DEVERR_TIMEOUT, site, bar, parity, detail);
      }
      if (__any_sync(0xffffffffu, late || *w.abort != 0)) return false;
    }
  }
  return true;
}

// mbar_wait_drain by a converged warp; the timer, hundreds of cycles a reading, only for what has not landed yet.
__device__ __forceinline__ void warp_drain(uint32_t bar, uint32_t parity, uint64_t limit_ns) {
  const bool done = __all_sync(0xffffffffu, mbar_test_wait(bar, parity));
  if (!done && (threadIdx.x & 31) == 0) mbar_wait_drain(bar, parity, limit_ns);
  __syncwarp();
}

// Four codes as four fp16 numbers.
__device__ __forceinline__ uint2 f16_of(uint32_t w) {
  const uint32_t u = w ^ 0x80808080u;   // code + 128
  uint32_t lo = __byte_perm(u, 0x64646464u, 0x4140), hi = __byte_perm(u, 0x64646464u, 0x4342);
  const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
  __half2 l = __hsub2(*reinterpret_cast<__half2*>(&lo), off), h = __hsub2(*reinterpret_cast<__half2*>(&hi), off);
  return make_uint2(*reinterpret_cast<uint32_t*>(&l), *reinterpret_cast<uint32_t*>(&h));
}

template <int BN, bool PAIR, bool SPLIT>
__global__ void __launch_bounds__(I_THREADS, 1)
    gemm_i8_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w,
                   const __grid_constant__ CUtensorMap tm_out, const __grid_constant__ LinearParams p) {
  using C = ICfg<BN, PAIR>;
  constexpr int RST = C::RST, FST = C::FST;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw;
  const uint32_t sbase = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::N_BAR);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const uint32_t rawf0 = smem_u32(bars), rawe0 = rawf0 + 8 * RST, f16f0 = rawe0 + 8 * RST, f16e0 = f16f0 + 8 * FST,
                 accf0 = f16e0 + 8 * FST, acce0 = accf0 + 16, drain_bar = acce0 + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR ? static_cast<int>(cluster_ctarank()) : 0;
  const int ctas = SPLIT ? p.split : C::CTAS, unit = blockIdx.x / ctas, units = gridDim.x / ctas;
  const int part = SPLIT ? static_cast<int>(cluster_ctarank()) : 0;
  const int kb0 = SPLIT ? p.n_kb * part / p.split : 0, kb1 = SPLIT ? p.n_kb * (part + 1) / p.split : p.n_kb;
  if (sbase & 1023u) {   // the same for every CTA of a launch
    if (threadIdx.x == 0) record_error(p.status, DEVERR_LAYOUT, 0, sbase, 0, 2);
    return;
  }
  // A pair's rank 0 issues the UMMAs: its fp16-full and set-empty barriers count both CTAs' warps.  Loads count on
  // their own CTA's barriers alone.  The fp16-empty, set-full and drain barriers are each CTA's own, arrived at by
  // commits that go to both.
  if (threadIdx.x == 0) {
    for (int i = 0; i < RST; ++i) {
      mbar_init(rawf0 + 8 * i, 1);
      mbar_init(rawe0 + 8 * i, 4);
    }
    for (int i = 0; i < FST; ++i) {
      mbar_init(f16f0 + 8 * i, 4 * C::CTAS);
      mbar_init(f16e0 + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(accf0 + 8 * i, 1);
      mbar_init(acce0 + 8 * i, I_EPI * C::CTAS);
    }
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if constexpr (PAIR) cluster_sync();   // both CTAs run and their barriers exist
  if (warp == 1) {
    if constexpr (PAIR) {
      tmem_alloc_pair(smem_u32(tmem_slot), 512);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(smem_u32(tmem_slot), 512);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();   // the codes and scales may come from the kernel before this one
  pdl_trigger();
  const WaitCtx wc{abort_flag, p.status, p.wait_limit_ns};

  if (warp < 4) {
    regs_dec<C::REGS_FIRST>();
    if (warp == 0) {
      // ---------------------------------------------------------- TMA producer
      const bool leader = elect_one();
      int g = 0;   // blocks issued over all tiles of this CTA
      uint32_t st = 0, ph = 1;
      bool ok = true;
      for (int t = unit; ok && t < p.n_tiles; t += units) {
        const int m0 = ((t % p.n_mt) * C::CTAS + rank) * IM, n0 = (t / p.n_mt) * BN + rank * C::BR;
        for (int kb = kb0; kb < kb1; ++kb, ++g) {
          if (!warp_wait(rawe0 + 8 * st, ph, wc, 41, g)) {
            ok = false;
            break;
          }
          const uint32_t dst = sbase + C::OFF_RAW + st * C::RAW, full = rawf0 + 8 * st;
          if (leader) {
            mbar_arrive_expect_tx(full, C::RAW);
            tma_load_2d(dst, &tm_a, full, kb * IK, m0);
            tma_load_2d(dst + IM * IK, &tm_w, full, kb * IK, n0);
          }
          __syncwarp();
          if (++st == RST) st = 0, ph ^= 1;
        }
      }
      for (int i = g > RST ? g - RST : 0; i < g; ++i)
        warp_drain(rawf0 + 8 * (i % RST), (i / RST) & 1, I_DRAIN_NS);
    } else if (warp == 1) {
      // ---------------------------------------------------------- UMMA issuer
      if (rank == 0) {
        const bool leader = elect_one();
        const uint64_t desc0 = sw128_desc(sbase, 16, 1024);   // + bytes / 16 inside the 256 KB window
        uint32_t st = 0, ph = 0;   // fp16 stage and its parity
        int i = 0;                 // accumulator sets filled
        bool ok = true;
        for (int t = unit; ok && t < p.n_tiles; t += units) {
          for (int c0 = kb0; ok && c0 < kb1; c0 += I_EXACT, ++i) {
            const int set = i & 1;
            if (!warp_wait<PAIR>(acce0 + 8 * set, ((i >> 1) & 1) ^ 1, wc, 44, i)) {
              ok = false;
              break;
            }
            const uint32_t acc = tmem + set * BN;
            uint32_t more = 0;
            for (int left = min(I_EXACT, kb1 - c0); left > 0; --left) {
              if (!warp_wait<PAIR>(f16f0 + 8 * st, ph, wc, 42, c0)) {
                ok = false;
                break;
              }
              tc_fence_after();
              const uint32_t ta = tmem + C::A_COL + st * (IK / 2);
              const uint64_t db = desc0 + st * (C::B16 / 16);
              if (leader) {
#pragma unroll
                for (int k = 0; k < IK / 16; ++k) {   // 16 fp16: 8 TMEM columns of A, 32 bytes inside B's swizzle row
                  if constexpr (PAIR) umma_ts_pair(acc, ta + 8 * k, db + 2 * k, C::IDESC, k ? 1u : more);
                  else umma_ts(acc, ta + 8 * k, db + 2 * k, C::IDESC, k ? 1u : more);
                }
                if constexpr (PAIR) tc_commit_pair(f16e0 + 8 * st);
                else tc_commit(f16e0 + 8 * st);
              }
              __syncwarp();
              more = 1;
              if (++st == FST) st = 0, ph ^= 1;
            }
            if (!ok) break;
            if (leader) {
              if constexpr (PAIR) tc_commit_pair(accf0 + 8 * set);
              else tc_commit(accf0 + 8 * set);
            }
            __syncwarp();
          }
        }
        if (leader) {
          if constexpr (PAIR) tc_commit_pair(drain_bar);
          else tc_commit(drain_bar);
        }
        __syncwarp();
      }
      warp_drain(drain_bar, 0, rank == 0 ? I_DRAIN_NS : p.wait_limit_ns + 2 * I_DRAIN_NS);
    }
    __syncwarp();
  } else if (warp < 4 + I_CONV) {
    // ------------------------------------------------------------ converters
    regs_dec<C::REGS_CONV>();
    // Each team its own blocks: the waits, the fence and the arrivals of one block hide behind the other teams' work.
    const int quarter = warp & 3;
    const int n = (unit < p.n_tiles ? (p.n_tiles - 1 - unit) / units + 1 : 0) * (kb1 - kb0);   // this CTA's blocks
    // A: a lane a row, 64 codes; the 64-byte swizzle puts 16-byte word c of row r at word c ^ (r / 2 mod 4), so that
    // eight rows' words lie in eight different bank groups.
    const int ra = quarter * 32 + lane, xa = (ra >> 1) & 3;
    // B: eight rows at a time, four lanes a row with 16 codes each: eight lanes read 128 bytes in a row and write, of
    // two neighbouring rows, the even (then the odd) 16-byte words, which the 128-byte swizzle puts into eight
    // different bank groups.
    const int rb = 8 * quarter + (lane >> 2), q = lane & 3;
    const uint32_t even = ((2 * q) ^ (rb & 7)) * 16, odd = ((2 * q + 1) ^ (rb & 7)) * 16;
    for (int g = (warp - 4) / 4; g < n; g += I_TEAMS) {
      const int rs = g % RST, fs = g % FST;
      if (!warp_wait(rawf0 + 8 * rs, (g / RST) & 1, wc, 45, g) ||
          !warp_wait(f16e0 + 8 * fs, ((g / FST) & 1) ^ 1, wc, 46, g))
        break;
      tc_fence_after();
      const uint8_t* src = smem + C::OFF_RAW + rs * C::RAW;
      const uint32_t ta = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + C::A_COL + fs * (IK / 2);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t x[16];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint4 v = *reinterpret_cast<const uint4*>(src + ra * IK + ((2 * h + c) ^ xa) * 16);
          const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint2 f = f16_of(u[e]);
            x[8 * c + 2 * e] = f.x;
            x[8 * c + 2 * e + 1] = f.y;
          }
        }
        tmem_st16(ta + 16 * h, x);
      }
      src += IM * IK + rb * IK + q * 16;
      uint8_t* dst = smem + fs * C::B16 + rb * 2 * IK;
      uint4 v[C::BR / 32];
#pragma unroll
      for (int j = 0; j < C::BR / 32; ++j) v[j] = *reinterpret_cast<const uint4*>(src + j * 32 * IK);
#pragma unroll
      for (int j = 0; j < C::BR / 32; ++j) {
        const uint2 x0 = f16_of(v[j].x), x1 = f16_of(v[j].y), x2 = f16_of(v[j].z), x3 = f16_of(v[j].w);
        uint8_t* row = dst + j * 32 * 2 * IK;
        *reinterpret_cast<uint4*>(row + even) = make_uint4(x0.x, x0.y, x1.x, x1.y);
        *reinterpret_cast<uint4*>(row + odd) = make_uint4(x2.x, x2.y, x3.x, x3.y);
      }
      fence_proxy_async_smem();   // each lane's own stores, before the UMMAs read them
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(rawe0 + 8 * rs);
        // The issuer stands in the other CTA: B's half needs a release of cluster scope, A's in TMEM the fence above.
        // Restricted to shared memory it costs 1 % (149.8 -> 150.8 us at 4680 x 5120 -> 5120), an unrestricted one a
        // quarter, and one warp that sends them all on waits 0.5 us for each (360 us).
        if (PAIR && rank == 1) mbar_arrive_cluster_smem(cluster_map(f16f0 + 8 * fs, 0));
        else mbar_arrive(f16f0 + 8 * fs);
      }
    }
  } else {
    // ------------------------------------------------------------ read-back
    regs_inc<C::REGS_EPI>();
    constexpr int HC = BN / 64;   // 32-column chunks of this warp's half
    const int quarter = warp & 3, half = (warp - 4 - I_CONV) >> 2;
    uint8_t* blocks = smem + C::OFF_OUT + (warp - 4 - I_CONV) * 2 * I_OUT_BLOCK;
    float* cols = reinterpret_cast<float*>(smem + C::OFF_SCALE) + (warp - 4 - I_CONV) * BN;   // scales, then biases
    // Up to two runs of 1024: their fp32 sum is the integer's rounding to fp32, so nothing is converted (the
    // conversions go 16 a clock and SM; 4680 x 1536 -> 4608 took 54 us with them).  A share of a split tile has to stay
    // exact: one run.
    const bool in_fp32 = kb1 - kb0 <= (SPLIT ? 1 : 2) * I_EXACT;
    int i = 0, stores = 0;   // sets read; blocks stored (they alternate on across tiles, wherever one ends)
    bool ok = true;
    for (int t = unit; ok && t < p.n_tiles; t += units) {
      const int m0 = ((t % p.n_mt) * C::CTAS + rank) * IM, n0 = (t / p.n_mt) * BN + half * (BN / 2);
      const int row = m0 + quarter * 32 + lane;
      // the scales are here before the sums are
      const float sa = row < p.T ? p.a_scale[row] : 0.f;
#pragma unroll
      for (int c = 0; c < HC; ++c) {
        const int n = n0 + 32 * c + lane;
        cols[32 * c + lane] = n < p.Dout ? p.w_scale[n] : 0.f;
        cols[BN / 2 + 32 * c + lane] = p.bias && n < p.Dout ? p.bias[n] : 0.f;
      }
      __syncwarp();
      int32_t sum[HC * 32];   // fp32 bits (in_fp32)
#pragma unroll
      for (int e = 0; e < HC * 32; ++e) sum[e] = 0;
      for (int c0 = kb0; c0 < kb1; c0 += I_EXACT, ++i) {
        const int set = i & 1;
        if (!warp_wait(accf0 + 8 * set, (i >> 1) & 1, wc, 43, i)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t taddr = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + set * BN + half * (BN / 2);
        if (in_fp32) {
#pragma unroll
          for (int c = 0; c < 2 * HC; ++c) {
            uint32_t v[16];
            tmem_ld16(taddr + 16 * c, v);
            tmem_wait_ld16(v);
#pragma unroll
            for (int e = 0; e < 16; ++e)
              sum[16 * c + e] = __float_as_int(__fadd_rn(__int_as_float(sum[16 * c + e]), __uint_as_float(v[e])));
          }
        } else {
#pragma unroll
          for (int c = 0; c < 2 * HC; ++c) {
            uint32_t v[16];
            tmem_ld16(taddr + 16 * c, v);
            tmem_wait_ld16(v);
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[16 * c + e] += __float2int_rn(__uint_as_float(v[e]));
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (PAIR) mbar_arrive_cluster(cluster_map(acce0 + 8 * set, 0));
          else mbar_arrive(acce0 + 8 * set);
        }
      }
      if (!ok) break;
      if constexpr (SPLIT) {
        // The partial sums, as integers, into the fp16 stages, which have been read: 16-byte word q of row r at
        // q ^ (r & 7).
        if (in_fp32) {
#pragma unroll
          for (int e = 0; e < HC * 32; ++e) sum[e] = __float2int_rn(__int_as_float(sum[e]));
        }
        int4* x = reinterpret_cast<int4*>(smem) + (quarter * 32 + lane) * (BN / 4);
#pragma unroll
        for (int q = 0; q < HC * 8; ++q)
          x[(half * (BN / 8) + q) ^ (lane & 7)] =
              make_int4(sum[4 * q], sum[4 * q + 1], sum[4 * q + 2], sum[4 * q + 3]);
        break;   // a split tile's CTA has no other
      }
      if (m0 + quarter * 32 >= p.T) continue;   // uniform over the warp; rows past T inside the block are clipped
      if (!in_fp32) {
#pragma unroll
        for (int e = 0; e < HC * 32; ++e) sum[e] = __float_as_int(__int2float_rn(sum[e]));
      }
#pragma unroll
      for (int c = 0; c < HC; ++c) {
        if (n0 + 32 * c >= p.Dout) break;       // uniform
        uint8_t* block = blocks + (stores++ & 1) * I_OUT_BLOCK;
        if (lane == 0) bulk_wait_read<1>();     // the store before last, this block's last, has read it
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t pk[4];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int o = 32 * c + 8 * q + 4 * e;
            const float4 sw = *reinterpret_cast<const float4*>(cols + o);
            const float4 bi = *reinterpret_cast<const float4*>(cols + BN / 2 + o);
            pk[2 * e] = pack_bf16x2(scaled(__int_as_float(sum[o]), sa, sw.x, bi.x),
                                    scaled(__int_as_float(sum[o + 1]), sa, sw.y, bi.y));
            pk[2 * e + 1] = pack_bf16x2(scaled(__int_as_float(sum[o + 2]), sa, sw.z, bi.z),
                                        scaled(__int_as_float(sum[o + 3]), sa, sw.w, bi.w));
          }
          // 64-byte swizzle: 16-byte word q of row r at word q ^ (r / 2 mod 4)
          *reinterpret_cast<uint4*>(block + lane * 64 + (q ^ ((lane >> 1) & 3)) * 16) =
              make_uint4(pk[0], pk[1], pk[2], pk[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          tma_store_2d(&tm_out, smem_u32(block), n0 + 32 * c, m0 + quarter * 32);
          bulk_commit_group();
        }
      }
    }
    if (lane == 0) bulk_wait_all();
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  if constexpr (SPLIT) {
    static_assert(!SPLIT || BN == 128, "a row is four columns a lane");
    cluster_sync();   // every CTA's partial sums are in its shared memory
    if (warp >= 4) {   // not the first four, whose registers are few
      const int m0 = unit % p.n_mt * IM, n0 = unit / p.n_mt * BN + 4 * lane;
      float sw[4], bi[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sw[e] = n0 + e < p.Dout ? p.w_scale[n0 + e] : 0.f;
        bi[e] = p.bias && n0 + e < p.Dout ? p.bias[n0 + e] : 0.f;
      }
      // one warp per row of this CTA's share; Dout is a multiple of 8, so a lane's four columns are all in or all out
      const int end = min(IM * (part + 1) / p.split, p.T - m0);
      for (int r = IM * part / p.split + warp - 4; r < end; r += I_CONV + I_EPI) {
        const uint32_t x = sbase + (r * (BN / 4) + (lane ^ (r & 7))) * 16;
        int4 o = make_int4(0, 0, 0, 0);
        for (int i = 0; i < p.split; ++i) {
          const float4 v = cluster_ld4(cluster_map(x, i));
          o.x += __float_as_int(v.x);
          o.y += __float_as_int(v.y);
          o.z += __float_as_int(v.z);
          o.w += __float_as_int(v.w);
        }
        const float sa = p.a_scale[m0 + r];
        if (n0 < p.Dout)
          *reinterpret_cast<uint2*>(p.out + static_cast<size_t>(m0 + r) * p.Dout + n0) =
              make_uint2(pack_bf16x2(scaled(__int2float_rn(o.x), sa, sw[0], bi[0]),
                                     scaled(__int2float_rn(o.y), sa, sw[1], bi[1])),
                         pack_bf16x2(scaled(__int2float_rn(o.z), sa, sw[2], bi[2]),
                                     scaled(__int2float_rn(o.w), sa, sw[3], bi[3])));
      }
    }
    cluster_sync();   // no CTA leaves while another still reads its shared memory
  }
  if constexpr (PAIR) cluster_sync();   // neither CTA's TMEM, barriers or shared memory is used by the other any more
  if (warp == 1) {
    tc_fence_after();
    if constexpr (PAIR) tmem_dealloc_pair(tmem, 512);
    else tmem_dealloc(tmem, 512);
  }
}

// The register split of gemm_i8_kernel fits into what its blocks are launched with; asked once per kernel (the code is
// the same on every device).
cudaError_t check_registers(const void* func, int sum, std::atomic<bool>& checked) {
  if (checked.load(std::memory_order_relaxed)) return cudaSuccess;
  cudaFuncAttributes attr;
  const cudaError_t e = cudaFuncGetAttributes(&attr, func);
  if (e != cudaSuccess) return e;
  if (attr.numRegs * (I_THREADS / 128) < sum) return cudaErrorInvalidConfiguration;
  checked.store(true, std::memory_order_relaxed);
  return cudaSuccess;
}

template <int BN, bool PAIR, bool SPLIT = false>
cudaError_t launch_gemm(int split, const int8_t* a_q, const float* a_scale, const int8_t* w_q, const float* w_scale,
                        const float* bias, int32_t T, int32_t D, int32_t Dout, __nv_bfloat16* out, int* status,
                        uint64_t wait_limit_ns, int sms, cudaStream_t s) {
  using C = ICfg<BN, PAIR>;
  const void* func = reinterpret_cast<const void*>(gemm_i8_kernel<BN, PAIR, SPLIT>);
  static std::atomic<bool> checked{false};
  cudaError_t e = check_registers(func, C::REGS_SUM, checked);
  if (e == cudaSuccess) e = set_smem_limit_once(func, C::SMEM);
  if (e != cudaSuccess) return e;
  CUtensorMap ta, tw, to;
  if (!encode_tmap_2d_u8_rows(&ta, a_q, D, T, D, IK, IM, true) ||
      !encode_tmap_2d_u8_rows(&tw, w_q, D, Dout, D, IK, C::BR, false) ||
      !encode_tmap_2d_sw64(&to, out, Dout, T, 2 * static_cast<uint64_t>(Dout), 32, 32))
    return cudaErrorInvalidValue;
  LinearParams p;
  p.T = T;
  p.Dout = Dout;
  p.n_kb = (D + IK - 1) / IK;   // past D the loads fill with zeros
  p.n_mt = (T + IM * C::CTAS - 1) / (IM * C::CTAS);
  p.n_tiles = p.n_mt * ((Dout + BN - 1) / BN);
  p.split = split;
  p.a_scale = a_scale;
  p.w_scale = w_scale;
  p.bias = bias;
  p.out = out;
  p.status = status;
  p.wait_limit_ns = wait_limit_ns;
  const int ctas = SPLIT ? split : C::CTAS, units = SPLIT ? p.n_tiles : std::min(p.n_tiles, sms / ctas);
  return launch_pdl_cluster(gemm_i8_kernel<BN, PAIR, SPLIT>, dim3(units * ctas), dim3(I_THREADS), C::SMEM, ctas, s, ta,
                            tw, to, p);
}

}  // namespace

cudaError_t launch_linear_i8(const int8_t* a_q, const float* a_scale, const int8_t* w_q, const float* w_scale,
                             const float* bias, int32_t T, int32_t D, int32_t Dout, void* out, int* status,
                             uint64_t wait_limit_ns, cudaStream_t s) {
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(out);
  int dev = 0, sms = 152;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const LinearForm g = linear_i8_form(T, D, Dout, sms);
  if (g.tokens) {
    const auto go = [&](auto kernel) {
      return launch_pdl(kernel, dim3((Dout + 8 * g.channels - 1) / (8 * g.channels), (T + g.tokens - 1) / g.tokens),
                        dim3(256), 0, s, a_q, a_scale, w_q, w_scale, bias, static_cast<int>(T), static_cast<int>(D),
                        static_cast<int>(Dout), o);
    };
    if (g.channels == 1)
      return g.tokens == 1   ? go(gemv_i8_kernel<1, 1>)
             : g.tokens == 2 ? go(gemv_i8_kernel<2, 1>)
             : g.tokens == 4 ? go(gemv_i8_kernel<4, 1>)
                             : go(gemv_i8_kernel<8, 1>);
    return g.tokens == 1   ? go(gemv_i8_kernel<1, 2>)
           : g.tokens == 2 ? go(gemv_i8_kernel<2, 2>)
           : g.tokens == 4 ? go(gemv_i8_kernel<4, 2>)
                           : go(gemv_i8_kernel<8, 2>);
  }
  if (g.split > 1)
    return launch_gemm<128, false, true>(g.split, a_q, a_scale, w_q, w_scale, bias, T, D, Dout, o, status,
                                         wait_limit_ns, sms, s);
  const auto run = !g.pair ? launch_gemm<128, false>
                   : g.bn == 192 ? launch_gemm<192, true> : launch_gemm<128, true>;
  return run(1, a_q, a_scale, w_q, w_scale, bias, T, D, Dout, o, status, wait_limit_ns, sms, s);
}

}  // namespace ispa
