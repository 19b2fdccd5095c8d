// Device code that the decode attention kernels share: warp-private copies into shared memory, and the combination of
// split partials inside a thread-block cluster.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "ckv_common.cuh"

namespace ckv {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t src_bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, uint32_t src_bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a float of the shared memory of CTA `rank` of this cluster, at the offset `local_addr` has in this CTA's window
__device__ __forceinline__ float ld_cluster_f32(uint32_t local_addr, uint32_t rank) {
  uint32_t ra;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(local_addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(ra) : "memory");
  return v;
}


// Partials of one (sequence, KV head) over the NW warps of each of the CL CTAs of a cluster, kPartial floats per warp and
// query head: out[128] relative to 2^max, max (exp2 domain), sum.  `park` writes this warp's eight heads to the rows it is
// handed; after a cluster barrier every CTA combines its share of the output columns of every query head from all CTAs'
// rows and writes out [G, 128].  The rows take the place of whatever the CTA had in `smem`.
constexpr int kPartial = 132;

template <int CL, int NW, typename Park>
__device__ __forceinline__ void cluster_combine(unsigned char* smem, int warp, int lane, int G, __nv_bfloat16* out, Park park) {
  // ND output columns per combining CTA and step (a divisor of 32); with 10 CTAs the first 8 combine 16 columns each
  constexpr int D = 128, P = kPartial, NP = NW * CL;
  constexpr int ND = CL < 4 ? 32 : ((D % CL == 0 && 32 % (D / CL) == 0) ? D / CL : 16), NPG = 32 / ND, PER = NP / NPG;
  __syncthreads();  // every warp of the CTA is done with its ring: the partials take its place
  float* part = reinterpret_cast<float*>(smem);  // [warp][8 heads][P]
  float* scl = part + NW * 8 * P;               // [warp][NP] weights 2^(m_p - m)
  park(part + warp * 8 * P);
  cluster_sync_all();
  const uint32_t part_s = (uint32_t)__cvta_generic_to_shared(smem);
  const int d = lane % ND, pg = lane / ND;
  for (int head = warp; head < G && (int)blockIdx.x * ND < D; head += NW) {
    constexpr int NK = (NP + 31) / 32;
    static_assert(NP % NPG == 0, "the partials split evenly over the lane groups");
    float mp[NK], lp[NK], mm = -INFINITY;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const int pi = lane + 32 * k;  // partial of warp (pi % NW) of CTA (pi / NW)
      const uint32_t addr = part_s + (uint32_t)((((pi % NW) * 8 + head) * P + D) * 4);
      mp[k] = pi < NP ? ld_cluster_f32(addr, (uint32_t)(pi / NW)) : -INFINITY;
      lp[k] = pi < NP ? ld_cluster_f32(addr + 4u, (uint32_t)(pi / NW)) : 0.f;
      mm = fmaxf(mm, mp[k]);
    }
    mm = warp_max(mm);
    float ll = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const float f = mp[k] == -INFINITY ? 0.f : exp2f(mp[k] - mm);
      if (lane + 32 * k < NP) scl[warp * NP + lane + 32 * k] = f;
      ll = fmaf(f, lp[k], ll);
    }
    ll = warp_sum(ll);
    __syncwarp();
    for (int d0 = (int)blockIdx.x * ND; d0 < D; d0 += CL * ND) {  // this CTA's columns d0 .. d0 + ND - 1
      float acc = 0.f;
#pragma unroll 4
      for (int j = 0; j < PER; ++j) {
        const int pi = pg * PER + j;
        acc = fmaf(scl[warp * NP + pi], ld_cluster_f32(part_s + (uint32_t)((((pi % NW) * 8 + head) * P + d0 + d) * 4), (uint32_t)(pi / NW)),
                   acc);
      }
#pragma unroll
      for (int sft = ND; sft < 32; sft <<= 1) acc += __shfl_xor_sync(0xffffffffu, acc, sft);
      if (pg == 0) {
        const float inv = ll > 0.f ? 1.f / ll : 0.f;
        out[head * D + d0 + d] = __float2bfloat16_rn(acc * inv);
      }
    }
    __syncwarp();
  }
  cluster_sync_all();  // nobody leaves while its shared memory may still be read
}

}  // namespace ckv
