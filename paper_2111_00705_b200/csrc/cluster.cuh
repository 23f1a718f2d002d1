// Shared memory of the other blocks of a cluster.
#pragma once
#include "common.cuh"

namespace cdadam {

// All threads of all blocks, converged: what was written before it is seen behind it.
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address that p has in block `rank`.
__device__ __forceinline__ uint32_t at_rank(const void *p, int rank)
{
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr(p)), "r"(rank));
    return at;
}
__device__ __forceinline__ int load_at(uint32_t at)
{
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ int4 load4_at(uint32_t at)
{
    int4 v;
    asm volatile("ld.shared::cluster.v4.s32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

}  // namespace cdadam
