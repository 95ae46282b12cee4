// Barriers in shared memory, bulk copies into it and writes to the other CTAs of a cluster, with waits that end.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace sr {

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint64_t* bar, uint32_t arrivals) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_address(bar)), "r"(arrivals) : "memory");
}
// Makes initialised barriers known to bulk copies and to the cluster; a cluster barrier follows.
__device__ __forceinline__ void barriers_ready() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void barrier_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_address(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(shared_address(bar)) : "memory");
}
// Writes 16 bytes to the same place in CTA `rank` of the cluster and counts them at its barrier `bar`; nothing is waited for.
__device__ __forceinline__ void store_at(void* to, unsigned long long lo, unsigned long long hi, uint64_t* bar, uint32_t rank) {
    asm volatile(
        "{\n\t.reg .b32 there, bar;\n\t"
        "mapa.shared::cluster.u32 there, %0, %4;\n\t"
        "mapa.shared::cluster.u32 bar, %3, %4;\n\t"
        "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [there], {%1, %2}, [bar];\n\t}" ::"r"(shared_address(to)), "l"(lo), "l"(hi), "r"(shared_address(bar)), "r"(rank)
        : "memory");
}
constexpr uint32_t kNap = 20000;          // ns that a test may sleep for: warps that ask again and again take issue slots from those that work
__device__ __forceinline__ bool barrier_test(uint64_t* bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(shared_address(bar)), "r"(parity), "r"(kNap) : "memory");
    return done != 0;
}
__device__ __forceinline__ unsigned long long nanoseconds() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
constexpr unsigned long long kWaitLimit = 1000000000ull;     // a second; a wait takes microseconds

// Waits for the phase with that parity.  After `limit` ns (looked at every millisecond or so), or where another thread of the CTA has given up, *gave_up is set and the
// wait ends all the same: whoever reads it says so in the results.
__device__ __noinline__ void barrier_wait_long(uint64_t* bar, uint32_t parity, volatile int* gave_up, unsigned long long limit) {
    const unsigned long long began = nanoseconds();
    for (;;) {
        for (int k = 0; k < 64; ++k)
            if (barrier_test(bar, parity)) return;
        if (*gave_up) return;
        if (nanoseconds() - began > limit) {
            *gave_up = 1;
            return;
        }
    }
}
__device__ __forceinline__ void barrier_wait(uint64_t* bar, uint32_t parity, volatile int* gave_up, unsigned long long limit = kWaitLimit) {
    if (!barrier_test(bar, parity)) barrier_wait_long(bar, parity, gave_up, limit);
}

// Copies `bytes` (a multiple of 16, both addresses on 16 bytes) from global into this CTA's shared memory and counts them at `bar`.
__device__ __forceinline__ void bulk_load(void* to, const void* from, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(shared_address(to)), "l"(from), "r"(bytes), "r"(shared_address(bar))
                 : "memory");
}

// Copies `bytes` (as above) from this CTA's shared memory to global; bulk_stores_done waits until the memory they come from has been
// read.
__device__ __forceinline__ void bulk_store(void* to, const void* from, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(shared_address(from)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_stores_done() {
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}
// What threads have written to shared memory is there for bulk copies; a barrier follows.
__device__ __forceinline__ void shared_written() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

}  // namespace sr
