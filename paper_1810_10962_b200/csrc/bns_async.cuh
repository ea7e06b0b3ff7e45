// Barriers in shared memory with bounded waits, and 2^x: what the language-model kernels share.
#pragma once

#include "bns_elements.cuh"

namespace bns {

constexpr unsigned kPolls = 1u << 22;   // attempts before a wait gives up

// Bounded waits that ran out since the library was loaded.
__device__ unsigned g_lm_timeouts;

__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));   // 2 ulp, 2^-126 and below give 0
    return r;
}

__device__ __forceinline__ unsigned smem_address(const void* p) { return static_cast<unsigned>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void barrier_init(unsigned bar, unsigned arrivals) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void barrier_expect(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_try(unsigned bar, unsigned parity) {
    unsigned done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}
// False once this wait, or another one of the block, has run out.
__device__ __forceinline__ bool wait_bounded(unsigned bar, unsigned parity, volatile int* gave_up) {
    for (unsigned i = 0; i < kPolls; ++i) {
        if (barrier_try(bar, parity)) return true;
        if ((i & 255) == 255 && *gave_up) return false;
    }
    *gave_up = 1;
    atomicAdd(&g_lm_timeouts, 1u);
    return false;
}

}  // namespace bns
