// Clusters of CTAs, and bounded waits for barriers that another CTA of a cluster arrives on.
#pragma once

#include "rps_tma.cuh"

namespace rps_ops {

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive;\n\tbarrier.cluster.wait;" ::: "memory");
}

// Waits for the phase with the given parity; what the cluster did before it is then visible.  Gives up after limit_ns.
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity), "r"(rps::kSuspendHintNs)
        : "memory");
    return done != 0;
}

__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, uint64_t limit_ns)
{
    if (try_wait(bar, parity)) return true;
    const uint64_t start = rps::global_timer_ns();
#pragma unroll 1
    while (!try_wait(bar, parity))
        if (rps::global_timer_ns() - start > limit_ns) return false;
    return true;
}

}  // namespace rps_ops
