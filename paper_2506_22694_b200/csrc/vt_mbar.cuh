// mbarriers in shared memory, what bounds the waits on them, and the election of the lane that issues copies.
#pragma once
#include "vt_common.cuh"

namespace vt {
namespace {

constexpr unsigned long long kWaitLimitNs = 2000000000ull;   // default bound of a device-side wait (Ctrl::wait_ns overrides)

// One lane of a converged warp.  The single-thread roles (copy producer, MMA issuer) are entered through this and
// not through `lane == 0`: behind elect.sync the compiler knows that one thread is active and hands tcgen05 and
// copy instructions their operands in uniform registers; behind a comparison it guards every one of them against
// a divergent warp (measured: 70-105 cycles to issue an MMA of M = 128, N = 16 instead of the 40 it takes).
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint64_t* b, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(count));
}
__device__ __forceinline__ void mbar_expect_tx(uint64_t* b, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
// By their addresses in shared memory (32 bits, where a warp keeps many of them) ...
__device__ __forceinline__ void bar_arrive(uint32_t b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(b) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t b, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
        : "=r"(ok) : "r"(b), "r"(parity) : "memory");
    return ok != 0;
}
// (non-blocking probe of a phase: try_wait may suspend the thread for a system-chosen time before it answers)
__device__ __forceinline__ bool bar_test(uint32_t b, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
        : "=r"(ok) : "r"(b), "r"(parity) : "memory");
    return ok != 0;
}
// ... and by pointers
__device__ __forceinline__ void mbar_arrive(uint64_t* b) { bar_arrive(smem_u32(b)); }
__device__ __forceinline__ bool mbar_try(uint64_t* b, uint32_t parity) { return bar_try(smem_u32(b), parity); }
__device__ __forceinline__ bool mbar_test(uint64_t* b, uint32_t parity) { return bar_test(smem_u32(b), parity); }

// The bound of a wait is kept with the SM's cycle counter (reading the nanosecond timer costs far more
// than a probe): two cycles per nanosecond, i.e. at least the time asked for at any SM clock up to
// 2 GHz.  It lives in shared memory and is looked at only once a wait has to spin.  Bounds under a
// millisecond spin on non-blocking probes only: try_wait may park the thread for a system-chosen time before
// it answers, which is what a long wait wants and a short bound cannot afford.
__device__ __forceinline__ long long bound_cycles(unsigned long long ns) {
    return (long long)(ns < (1ull << 61) ? 2 * ns : (1ull << 62));
}
constexpr long long kShortBoundCycles = 2000000;      // 1 ms
__device__ __forceinline__ unsigned long long global_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

}  // namespace
}  // namespace vt
