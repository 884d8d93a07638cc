// Waits on an mbarrier that give up: a wait that runs out records a code in the device status word and raises the block's abort
// flag, which ends the waits of its other roles too.
#pragma once
#include "ptx_sm100.cuh"

namespace tdx {

constexpr long long kWaitLimitCycles = 4000000000LL;  // ~2 s at boost clock

enum : int { kTimeoutProducer = 1, kTimeoutMma = 2, kTimeoutEpilogue = 3 };

__device__ __forceinline__ bool wait_bounded_for(uint64_t* bar, uint32_t parity, volatile int* s_abort, int* g_status,
                                                 int code, long long limit_cycles) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    uint32_t spins = 0;
    for (;;) {
        if (ptx::mbar_try_wait(bar, parity)) return true;
        if ((++spins & 63u) == 0u) {
            if (*s_abort) return false;
            if (clock64() - t0 > limit_cycles) {
                *s_abort = 1;
                atomicCAS(g_status, 0, code);
                return false;
            }
        }
    }
}
__device__ __forceinline__ bool wait_bounded(uint64_t* bar, uint32_t parity, volatile int* s_abort, int* g_status,
                                             int code) {
    return wait_bounded_for(bar, parity, s_abort, g_status, code, kWaitLimitCycles);
}

// The same in few instructions, for kernels of many roles whose code is large beside the instruction caches.  The hardware may hold the
// thread for up to 20 us at a time, so that it does not take issue slots by polling; the limit is two turns of the clock's upper half, 2 to
// 5 s.
__device__ __forceinline__ bool wait_bounded_idle(uint64_t* bar, uint32_t parity, volatile int* s_abort, int* g_status, int code) {
    uint32_t ok, began, now;
    asm volatile("mov.u32 %0, %%clock_hi;" : "=r"(began));
    do {
        asm volatile(
            "{\n"
            ".reg .pred p;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
            "selp.u32 %0, 1, 0, p;\n"
            "}\n"
            : "=r"(ok)
            : "r"(ptx::smem_u32(bar)), "r"(parity), "r"(20000u)
            : "memory");
        if (ok) return true;
        asm volatile("mov.u32 %0, %%clock_hi;" : "=r"(now));
        if (now - began >= 2u) {
            *s_abort = 1;
            atomicCAS(g_status, 0, code);
        }
    } while (!*s_abort);
    return false;
}

}  // namespace tdx
