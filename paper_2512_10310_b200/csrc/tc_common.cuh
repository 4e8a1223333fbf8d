// What the kernels on the 5th-generation tensor cores share: instruction and matrix descriptors, bounded waits.
#pragma once

#include "common.cuh"
#include "ptx_sm100.cuh"

namespace evln {

constexpr long long kWaitLimitCycles = 2000000000LL;  // ~1 s at boost clocks

// --- descriptors --------------------------------------------------------------------------

// kind::f16 instruction descriptor: fp32 accumulate, bf16 A and B, M x N of the whole pair.
__device__ __forceinline__ constexpr uint32_t make_idesc(bool b_mn_major, int m, int n)
{
    return (1u << 4)                       // D format: f32
           | (1u << 7)                     // A format: bf16
           | (1u << 10)                    // B format: bf16
           | ((b_mn_major ? 1u : 0u) << 16)
           | ((uint32_t)(n >> 3) << 17)
           | ((uint32_t)(m >> 4) << 24);
}

// Shared-memory matrix descriptor, 128-byte swizzle, rows of 128 bytes, 8-row groups 1024 B apart.
__device__ __forceinline__ uint64_t make_sdesc(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)((lbo_bytes >> 4) & 0x3FFFu) << 16;
    d |= (uint64_t)((sbo_bytes >> 4) & 0x3FFFu) << 32;
    d |= (uint64_t)1 << 46;                // descriptor version of this architecture
    d |= (uint64_t)2 << 61;                // SWIZZLE_128B
    return d;
}

__device__ __forceinline__ bool wait_bounded(uint32_t bar, uint32_t parity, int code, int* status,
                                             volatile int* s_abort, long long limit_cycles = kWaitLimitCycles)
{
    if (ptx::mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    uint32_t spins = 0;
    while (!ptx::mbar_try_wait(bar, parity)) {
        if ((++spins & 0x3f) == 0) {
            if (*s_abort) return false;
            if (clock64() - t0 > limit_cycles) {
                *s_abort = 1;
                atomicCAS(status, 0, code);
                return false;
            }
        }
    }
    return true;
}

// One lane polls, the warp shares the outcome (fewer pollers on the barrier word).
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, int code, int* status,
                                          volatile int* s_abort, int lane)
{
    int r = 1;
    if (lane == 0) r = wait_bounded(bar, parity, code, status, s_abort) ? 1 : 0;
    return __shfl_sync(0xffffffffu, r, 0) != 0;
}

}  // namespace evln
