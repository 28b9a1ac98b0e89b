// Two CTAs on one tile: a cluster of two with cta_group::2 products, each CTA with half of the rows of either operand.
//
// Both CTAs load their halves; the copies of both count on a barrier of the first CTA (the leader), whose one warp issues the products of both, reading both CTAs' shared memory: an SM reads its own 128 rows
// of A and 128 of the 256 of B for a 128 x 256 tile, where a CTA by itself would read all 256, from L2 and from shared memory alike.
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace vardrop {

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// Barrier of the cluster: all threads of both CTAs.  Nothing bounds it, so every thread comes to it whatever its waits gave.
__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of the leader's copy of something in shared memory.
__device__ __forceinline__ uint32_t leaders(const void* p) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(p)));
    return a;
}
__device__ __forceinline__ void leader_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
// 2-D tiled load into this CTA's shared memory, counted on the leader's barrier.
__device__ __forceinline__ void pair_load_2d(uint32_t dst, const void* map, uint32_t bar, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
                 : "memory");
}
__device__ __forceinline__ void pair_tmem_alloc(uint32_t* dst_smem, uint32_t ncols) {     // one full warp of either CTA
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst_smem)), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_tmem_dealloc(uint32_t addr, uint32_t ncols) { asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(ncols) : "memory"); }
// The leader's products so far arrive on the barrier at this place in both CTAs when they have completed.
__device__ __forceinline__ void pair_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"(static_cast<uint16_t>(3)) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Instruction descriptor of a 256 x 256 tile, both operands bf16 or both fp16, fp32 accumulator.
__device__ __host__ constexpr uint32_t pair_idesc(bool fp16, int a_mn, int b_mn) {
    return (1u << 4) | (fp16 ? 0u : (1u << 7) | (1u << 10)) | (static_cast<uint32_t>(a_mn) << 15) | (static_cast<uint32_t>(b_mn) << 16) | ((256u >> 3) << 17) | ((256u >> 4) << 24);
}

}  // namespace vardrop
