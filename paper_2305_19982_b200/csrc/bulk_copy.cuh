// Bulk copies into shared memory and the mbarriers that announce them (sm_90+ instructions), with
// bounded waits: a wait that runs out, or finds the CTA's give-up flag set, returns false.
#pragma once

#include <stdint.h>

#include "adama_internal.h"

namespace adama {

__device__ __forceinline__ uint32_t shared_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_init_fence() {
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_poll(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
constexpr unsigned long long kBulkWaitLimitNs = 2000000000ull;
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, volatile int *give_up) {
    if (barrier_poll(bar, parity)) return true;
    const unsigned long long t0 = now_ns();
    bool late = false;
    for (uint32_t spins = 1;; ++spins) {
        if (barrier_poll(bar, parity)) return true;
        if ((spins & 0x3f) == 0) {
            if (*give_up) return false;
            if (late) {  // and not in these looks either: it is not this thread that was held up
                *give_up = 1;
                return false;
            }
            late = now_ns() - t0 > kBulkWaitLimitNs;
        }
    }
}

// For one lane of every warp at its end: the warp whose wait ran out may be the last one of its CTA.
__device__ __forceinline__ void report_expired_wait(const volatile int *give_up, unsigned *status, unsigned site) {
    if (*give_up && atomicCAS(status, (unsigned)kDevOk, (unsigned)kDevTimeout) == (unsigned)kDevOk) status[1] = site;
}

// `bytes` (a multiple of 16) from global `src` to shared `dst`, both 16-byte aligned
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// 4 bytes from global to shared memory, any 4-byte alignment; this thread's earlier ones count as one
// arrival on the barrier once they have landed.
__device__ __forceinline__ void small_load(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void small_loads_arrive(uint32_t bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void small_loads_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// ---- clusters -------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
    cluster_arrive();
    cluster_wait();
}
// Three words into the shared memory of CTA `rank` of the cluster; ordered by the next cluster_sync.
__device__ __forceinline__ void store12(uint32_t dst, uint32_t rank, float a, float b, float c) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(dst), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0+4], %2;\n\tst.shared::cluster.f32 [%0+8], %3;"
                 ::"r"(r), "f"(a), "f"(b), "f"(c)
                 : "memory");
}
// 16 bytes into the shared memory of CTA `rank` of the cluster, announced on its barrier; dst and bar
// are this CTA's addresses of the same variables.
__device__ __forceinline__ void send16(uint32_t dst, uint32_t bar, uint32_t rank, float a, float b, float c, float d) {
    uint32_t rdst, rbar;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(rdst) : "r"(dst), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(rbar) : "r"(bar), "r"(rank));
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(
                     rdst),
                 "r"(__float_as_uint(a)), "r"(__float_as_uint(b)), "r"(__float_as_uint(c)), "r"(__float_as_uint(d)),
                 "r"(rbar)
                 : "memory");
}

}  // namespace adama
