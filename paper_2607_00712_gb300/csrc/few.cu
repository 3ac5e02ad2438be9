// Attention of one or two queries over the window, the chunk and listed blocks (the *_blocks entry points):
// out = sum_i exp(s_i - m) v_i / sum_i exp(s_i - m), s_i = scale q . k_i.
//
// A key is read for four products at most, so HBM, start and latency bound it, not the tensor cores: their tiles of 128
// queries and their start of 8 us are left out.  A cluster of up to eight CTAs a head.  A warp takes 16 neighbouring
// keys at a time, and has the next ones' K and V rows on their way to shared memory of its own (16 KB a warp, 192 KB an
// SM; the places of 32 units are looked up at once, one a lane).  The lanes of a K row halve the sums that they hold as
// they add them up, 8 shuffles for 16 scores of 128 features; one exponential a lane; the rows of V are added with the
// weights from their lanes.  Warps, then CTAs through shared memory of the cluster, merge (O, m, l) as Eq. 11-12 do.
// All of it in fp32, rounded once.
//
// One query, 12 heads, 5656 keys (34.8 MB, 5.0 us at the copy rate): 8.1 to 8.6 us a launch in a graph, 11.8 to 12.2
// with the tensor cores' kernel; 1024 keys 4.5 (12.4), 19112 keys 22.3 (25.2); two queries 9.7 to 10.2, 5.2, 23.3.  40
// heads x 15016 keys 49.0 (50.0; floor 45.3), in 8 bits 37.5 (41.8; 34).  40 heads x 73000 keys is the other way
// round, 221 against 209 (220 at the copy rate).  What bounds it: an SM takes 60 bytes a cycle in and as many out of
// its shared memory, and clusters of eight leave 56 SMs without work where there are 12 heads.  Steps: rows in
// registers, 32 keys at a time 11.4; asynchronous copies, 8 warps of three units 9.7; two products an instruction and
// 12 warps 9.0; whole units' copies without conditions 8.6.  Four queries were tried with eight warps alone, 15.2:
// from three on the other kernel's 11.8.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "internal.h"
#include "pdl.cuh"
#include "ptx.cuh"
#include "rows.cuh"

namespace ispa {

namespace {

constexpr int F_WARPS = 12, F_THREADS = 32 * F_WARPS;
constexpr int F_KEYS = 16;            // of a unit: of a warp at a time
constexpr int F_WARP_BYTES = 16384;   // of a warp's K and V rows on their way

struct FewParams : AttnParams {
  AttnLists lists;
  const uint8_t* q;          // [n_q][H][d], bf16 or codes
  const uint8_t* k_ring;     // [H][ring_tok][d]
  const uint8_t* k_cur;      // [n_q][H][d]
  const __nv_bfloat16* v_ring;
  const __nv_bfloat16* v_cur;
  int64_t ring_tok;
  int32_t units;             // of F_KEYS keys, of a head
  int32_t units_of_block;
  Divisor by_units;          // of a block
};

// Keys of a unit: rows `stride` apart, `n` of them (0: none).
struct Unit {
  int64_t row;
  int n;
  bool chunk;
};
__device__ __forceinline__ Unit unit_at(const FewParams& p, const int32_t* list, int u) {
  for (int s = 0; s < p.n_seg; ++s) {
    const AttnSeg& g = p.seg[s];
    if (g.src == 2) break;
    const int n = (g.count + F_KEYS - 1) / F_KEYS;
    if (u < n) return Unit{g.start + static_cast<int64_t>(u) * F_KEYS, min(F_KEYS, g.count - u * F_KEYS), g.src == 1};
    u -= n;
  }
  const int e = quotient(u, p.by_units), first = (u - e * p.units_of_block) * F_KEYS;
  const int id = e < p.lists.entries ? __ldg(list + e) : -1;
  if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(p.lists.n_ids)) return Unit{0, 0, false};
  const int frame = quotient(id, p.lists.by_nb), at = (id - frame * p.lists.nb) * p.lists.block;
  const int n = min(p.lists.block, p.lists.P - at) - first;
  return Unit{static_cast<int64_t>(frame) * p.lists.P + at + first, max(0, min(F_KEYS, n)), false};
}

// Sixteen bytes as fp32: eight bf16 values, or sixteen codes.
__device__ __forceinline__ void unpack(const uint4& w, float2 (&f)[4]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xFFFF0000u));
}
__device__ __forceinline__ void unpack(const uint4& w, float2 (&f)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t h2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(static_cast<uint16_t>(u[i >> 1] >> (16 * (i & 1)))));
    f[i] = __half22float2(*reinterpret_cast<const __half2*>(&h2));
  }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {   // zeros where not
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
template <int N>
__device__ __forceinline__ void copies_left() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A unit's rows in shared memory: K, then V, dense.  K rows have LK lanes of 16 bytes; a load of the warp takes
// 32 / LK keys, key (lane / LK) NK + i in load i.  V rows alike.
template <int D, bool QK8>
struct FewTile {
  static constexpr int KF = QK8 ? 16 : 8;   // features of a lane
  static constexpr int LK = D / KF, LV = D / 8;
  static constexpr int NK = LK / 2, NV = LV / 2;   // loads
  static_assert(32 / LK >= kFewQueries && 32 / LV >= kFewQueries, "the chunk's keys are one load");
  static constexpr int K_BYTES = F_KEYS * LK * 16, BYTES = K_BYTES + F_KEYS * LV * 16;
  static constexpr int STAGES = F_WARP_BYTES / BYTES;
};

// NQ: queries there is room for; n_q of them are there.
template <int D, bool QK8, int NQ>
__global__ void __launch_bounds__(F_THREADS, 1) few_kernel(const __grid_constant__ FewParams p) {
  using T = FewTile<D, QK8>;
  constexpr int KF = T::KF, LK = T::LK, LV = T::LV, NK = T::NK, NV = T::NV, STAGES = T::STAGES;
  extern __shared__ __align__(128) uint8_t smem[];
  const int rank = static_cast<int>(cluster_ctarank());
  int c;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(c));
  const int head = blockIdx.x / c, warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const int kl = lane % LK, kg = lane / LK, vl = lane % LV, vg = lane / LV, H = p.num_heads;
  uint8_t* const own = smem + warp * F_WARP_BYTES;
  const uint32_t own_at = smem_u32(own) + lane * 16;
  pdl_wait();
  pdl_trigger();
  const int32_t* list = p.lists.ids + static_cast<int64_t>(head) * p.lists.top_k;   // one query block
  const int first = rank * F_WARPS + warp, step = c * F_WARPS;
  const int rounds = first < p.units ? (p.units - first + step - 1) / step : 0;

  Unit mine = {};         // round 32 x + lane's, x = issued / 32
  uint64_t on_way = 0;    // (keys, chunk) of the units on their way, 6 bits each, the next one first
  auto issue = [&](int r, int slot) {
    uint64_t state = 0;
    if (r < rounds) {
      if (r % 32 == 0) mine = r + lane < rounds ? unit_at(p, list, first + (r + lane) * step) : Unit{0, 0, false};
      const int64_t at = __shfl_sync(0xffffffffu, mine.row, r % 32);
      const int n = __shfl_sync(0xffffffffu, mine.n, r % 32);
      const bool chunk = __shfl_sync(0xffffffffu, static_cast<int>(mine.chunk), r % 32);
      // rows of the ring lie [H][tokens], of the chunk [tokens][H]: those fit the first load
      const int64_t row = chunk ? at * H + head : head * p.ring_tok + at;
      const int stride = chunk ? H : 1;
      const uint4* k = reinterpret_cast<const uint4*>(chunk ? p.k_cur : p.k_ring) + (row + kg * stride) * LK + kl;
      const uint4* v = reinterpret_cast<const uint4*>(chunk ? p.v_cur : p.v_ring) + (row + vg * stride) * LV + vl;
      const uint32_t dst = own_at + slot * T::BYTES;
      if (n == F_KEYS) {
#pragma unroll
        for (int i = 0; i < NK; ++i) copy16(dst + i * 512, k + i * 32, true);
#pragma unroll
        for (int i = 0; i < NV; ++i) copy16(dst + T::K_BYTES + i * 512, v + i * 32, true);
      } else {
#pragma unroll
        for (int i = 0; i < NK; ++i) {
          const bool there = i * (32 / LK) + kg < n;
          copy16(dst + i * 512, there ? k + i * 32 : reinterpret_cast<const uint4*>(p.k_ring), there);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const bool there = i * (32 / LV) + vg < n;
          copy16(dst + T::K_BYTES + i * 512, there ? v + i * 32 : reinterpret_cast<const uint4*>(p.v_ring), there);
        }
      }
      state = static_cast<uint64_t>(n) | (chunk ? 32u : 0u);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    on_way = on_way >> 6 | state << (6 * (STAGES - 1));
  };
  // prologue: every slot
#pragma unroll 1
  for (int r = 0; r < STAGES; ++r) issue(r, r);

  // this lane's features of the queries
  float2 q[NQ][KF / 2];
  float ring_factor = p.scale_log2, chunk_factor = p.scale_log2;
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    uint4 w = make_uint4(0, 0, 0, 0);
    if (i < p.n_q) w = __ldg(reinterpret_cast<const uint4*>(p.q) + (static_cast<int64_t>(i) * H + head) * LK + kl);
    unpack(w, q[i]);
  }
  if constexpr (QK8) {
    const float qs = __ldg(p.q_scale + head);
    ring_factor *= qs * __ldg(p.kr_scale + head);
    chunk_factor *= qs * __ldg(p.kc_scale + head);
  }
  float2 o[NQ][4];
  float m[NQ], l[NQ];   // l: of this lane's keys
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[i][e] = make_float2(0.f, 0.f);
  }
  int slot = 0;
#pragma unroll 1
  for (int r = 0; r < rounds; ++r) {
    copies_left<STAGES - 1>();
    __syncwarp();   // every lane's copies are there
    const int n = static_cast<int>(on_way & 31);
    const float factor = on_way & 32 ? chunk_factor : ring_factor;
    const uint4* tile = reinterpret_cast<const uint4*>(own + slot * T::BYTES);
    // The products of a lane's features, for NK keys.  Of the row's LK lanes each sends half of its sums on at every
    // step and keeps the others, until one is left; the two lanes that then hold parts of the same key add them.  Lane
    // 2 x and 2 x + 1 end with key x.
    float s[NQ][NK];
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      float2 f[KF / 2];
      unpack(tile[(kg * NK + i) * LK + kl], f);
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        float2 a = make_float2(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < KF / 2; ++e) a = fma2(q[j][e], f[e], a);
        s[j][i] = a.x + a.y;
      }
    }
    float w[NQ];
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
#pragma unroll
      for (int half = NK / 2; half > 0; half /= 2) {
        const bool up = kl & (2 * half);
#pragma unroll
        for (int i = 0; i < half; ++i) {
          const float give = up ? s[j][i] : s[j][i + half], keep = up ? s[j][i + half] : s[j][i];
          s[j][i] = keep + __shfl_xor_sync(0xffffffffu, give, 2 * half);
        }
      }
      s[j][0] += __shfl_xor_sync(0xffffffffu, s[j][0], 1);
      const float score = lane / 2 < n ? s[j][0] * factor : -INFINITY;
      float top = fmaxf(m[j], score);
#pragma unroll
      for (int x = 2; x < 32; x *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      const float zero = top == -INFINITY ? 0.f : top;   // no key that counts yet
      w[j] = ex2_approx(score - zero);
      const float alpha = ex2_approx(m[j] - zero);
      l[j] = fmaf(l[j], alpha, w[j]);
      m[j] = top;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = fma2(o[j][e], make_float2(alpha, alpha), make_float2(0.f, 0.f));
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float2 f[4];
      unpack(tile[F_KEYS * LK + (vg * NV + i) * LV + vl], f);
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        const float x = __shfl_sync(0xffffffffu, w[j], 2 * (vg * NV + i));
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = fma2(make_float2(x, x), f[e], o[j][e]);
      }
    }
    __syncwarp();   // every lane has read the slot
    issue(r + STAGES, slot);
    slot = slot + 1 < STAGES ? slot + 1 : 0;
  }
  copies_left<0>();
  __syncthreads();   // the slots are free: the parts of the warps, and of the CTA, lie there
  float* const o_part = reinterpret_cast<float*>(smem);      // [F_WARPS][NQ][D]
  float* const o_cta = o_part + F_WARPS * NQ * D;            // [NQ][D]
  float* const m_part = o_cta + NQ * D;                      // [F_WARPS][NQ]
  float* const l_part = m_part + F_WARPS * NQ;
  float* const m_cta = l_part + F_WARPS * NQ;                // [NQ]
  float* const l_cta = m_cta + NQ;
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float a = e % 2 ? o[j][e / 2].y : o[j][e / 2].x;
#pragma unroll
      for (int x = LV; x < 32; x *= 2) a += __shfl_xor_sync(0xffffffffu, a, x);
      if (vg == 0) o_part[(warp * NQ + j) * D + 8 * vl + e] = a;
    }
#pragma unroll
    for (int x = 2; x < 32; x *= 2) l[j] += __shfl_xor_sync(0xffffffffu, l[j], x);
    if (lane == 0) {
      m_part[warp * NQ + j] = m[j];
      l_part[warp * NQ + j] = l[j];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < NQ * D; i += F_THREADS) {
    const int j = i / D;
    float top = -INFINITY, sum = 0.f, a = 0.f;
#pragma unroll
    for (int x = 0; x < F_WARPS; ++x) top = fmaxf(top, m_part[x * NQ + j]);
    const float zero = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int x = 0; x < F_WARPS; ++x) {
      const float f = ex2_approx(m_part[x * NQ + j] - zero);
      sum = fmaf(f, l_part[x * NQ + j], sum);
      a = fmaf(f, o_part[x * NQ * D + i], a);
    }
    o_cta[i] = a;
    if (i % D == 0) m_cta[j] = top, l_cta[j] = sum;
  }
  cluster_sync();
  if (rank == 0) {
    const uint32_t o_at = smem_u32(o_cta), m_at = smem_u32(m_cta), l_at = smem_u32(l_cta);
    for (int i = threadIdx.x; i < p.n_q * D; i += F_THREADS) {
      const int j = i / D, e = i % D;
      float ms[8], ls[8], os[8], top = -INFINITY, sum = 0.f, a = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const bool there = x < c;
        ms[x] = there ? cluster_ld1(cluster_map(m_at + 4 * j, x)) : -INFINITY;
        ls[x] = there ? cluster_ld1(cluster_map(l_at + 4 * j, x)) : 0.f;
        os[x] = there ? cluster_ld1(cluster_map(o_at + 4 * i, x)) : 0.f;
        top = fmaxf(top, ms[x]);
      }
      const float zero = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float f = ex2_approx(ms[x] - zero);
        sum = fmaf(f, ls[x], sum);
        a = fmaf(f, os[x], a);
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;   // 0: no key
      p.out[(static_cast<int64_t>(j) * H + head) * D + e] = __float2bfloat16_rn(a * inv);
      if (p.lse && e == 0) p.lse[static_cast<int64_t>(head) * p.n_q + j] = (top + __log2f(sum)) * 0.69314718055994531f;
    }
  }
  cluster_sync();   // no CTA leaves while another still reads its shared memory
}

template <int D, bool QK8, int NQ>
cudaError_t launch(const FewParams& p, int sms, cudaStream_t s) {
  static_assert(F_WARPS * F_WARP_BYTES >= 4 * (NQ * (F_WARPS + 1) * (D + 2)), "the parts fit the slots");
  constexpr int BYTES = F_WARPS * F_WARP_BYTES;
  auto kernel = few_kernel<D, QK8, NQ>;
  cudaError_t e = set_smem_limit_once(reinterpret_cast<const void*>(kernel), BYTES);
  if (e != cudaSuccess) return e;
  // as many CTAs as SMs, no more than eight a head and no more than have a unit for every warp
  const int most = std::max(1, std::min(8, sms / p.num_heads)), want = (p.units + F_WARPS - 1) / F_WARPS;
  const int c = std::max(1, std::min(most, want));
  return launch_pdl_cluster(kernel, dim3(static_cast<unsigned>(p.num_heads * c)), dim3(F_THREADS), BYTES, c, s, p);
}
template <int D, bool QK8>
cudaError_t launch_for(const FewParams& p, int sms, cudaStream_t s) {
  return p.n_q == 1 ? launch<D, QK8, 1>(p, sms, s) : launch<D, QK8, 2>(p, sms, s);
}

}  // namespace

cudaError_t launch_attention_few(int head_dim, const AttnParams& a, const AttnLists& lists, const void* q,
                                 const void* k_ring, const void* v_ring, const void* k_cur, const void* v_cur,
                                 int64_t ring_tok, cudaStream_t s) {
  FewParams p;
  static_cast<AttnParams&>(p) = a;
  p.lists = lists;
  p.q = static_cast<const uint8_t*>(q);
  p.k_ring = static_cast<const uint8_t*>(k_ring);
  p.k_cur = static_cast<const uint8_t*>(k_cur);
  p.v_ring = static_cast<const __nv_bfloat16*>(v_ring);
  p.v_cur = static_cast<const __nv_bfloat16*>(v_cur);
  p.ring_tok = ring_tok;
  p.units_of_block = (std::min(lists.block, lists.P) + F_KEYS - 1) / F_KEYS;
  p.by_units = divisor(p.units_of_block);
  int64_t units = static_cast<int64_t>(lists.entries) * p.units_of_block;
  for (int i = 0; i < a.n_seg; ++i)
    if (a.seg[i].src != 2) units += (a.seg[i].count + F_KEYS - 1) / F_KEYS;
  p.units = static_cast<int32_t>(units);   // below 2^31: as are the tiles' keys
  int dev = 0, sms = 152;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (a.q_scale) return launch_for<128, true>(p, sms, s);
  return head_dim == 128 ? launch_for<128, false>(p, sms, s) : launch_for<64, false>(p, sms, s);
}

}  // namespace ispa
