// Shared pieces of the projections (linear.cu, fp4_linear.cu): the activation, tensor memory among kernels that run beside one another, the
// order of tiles, and what the two CTAs of a pair say to one another.
#pragma once
#include "block.cuh"
#include "sm100.cuh"

namespace ssdi8 {

__device__ __forceinline__ float activate(float v, int act) {
  if (act == SSDI8_ACT_SILU) return v * rcp_approx(1.0f + ex2_approx(v * -1.44269504f));
  if (act == SSDI8_ACT_RELU2) return v < 0.f ? 0.f : v * v;   // (-inf is 0, a NaN stays one)
  return v;
}

namespace sm100 {

// Tensor memory for all warps but the loader's, by warp 2.  Behind the wait for the kernel before and ahead of the trigger for the next
// one: a kernel that held some while it waits, or that still had to ask for some when the next one may be scheduled beside it, could
// leave the two waiting for one another.
template <int GROUP>
__device__ __forceinline__ uint32_t allocated(uint32_t* slot, uint32_t columns, int warp, int threads) {
  if (warp == 2) {
    if (GROUP == 1) {
      tmem_alloc(slot, columns);
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(columns) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    pdl_launch_dependents();
  }
  tc_fence_before();
  named_bar_sync(2, threads - 32);
  tc_fence_after();
  return *slot;
}

// tile -> (row block, column block): GROUP row blocks at a time, so that the tiles in flight share rows of x and of w in L2
template <int GROUP>
__device__ __forceinline__ void tile_of(int tile, int mtiles, int ntiles, int* m, int* n) {
  const int per = GROUP * ntiles, group = tile / per, rest = tile % per;
  const int rows = min(GROUP, mtiles - group * GROUP);
  *m = group * GROUP + rest % rows;
  *n = rest / rows;
}

__device__ __forceinline__ uint32_t in_first(const void* p) {   // the same place in the pair's first CTA
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(p)));
  return a;
}
__device__ __forceinline__ void pair_load(void* dst, const CUtensorMap* tm, uint32_t bar, int x, int y) {   // bar: of the first CTA
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(smem_u32(dst)), "l"(tm), "r"(bar), "r"(x), "r"(y)
               : "memory");
}
__device__ __forceinline__ void pair_commit(uint64_t* bar) {   // arrives at this place in both CTAs
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(smem_u32(bar)), "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

}  // namespace sm100
}  // namespace ssdi8
