// roles.cuh -- what the warp roles of the attention and weight kernels share:
// short waits and the masking of scores.
#pragma once

#include "attn_core.cuh"

namespace rs {

// Keys whose bit is not set: -inf (whole warp; most chunks are open to all rows).
__device__ __forceinline__ void hide(uint32_t (&v)[32], uint32_t seen) {
    if (__all_sync(0xffffffffu, seen == 0xffffffffu)) return;
#pragma unroll
    for (int e = 0; e < 32; ++e)
        if (!((seen >> e) & 1u)) v[e] = 0xff800000u;
}

// A try that fails has waited for longer than this already (a test's limit).
constexpr long long kTryCycles = 1000;
__device__ __forceinline__ bool out_of_time(volatile int *abort, long long limit) {
    if (limit < kTryCycles) *abort = 1;
    return limit < kTryCycles;
}

// warp_wait with its usual case, a phase that is complete, on a short path.
__device__ __forceinline__ bool quick_wait(uint64_t *bar, uint32_t parity, volatile int *abort, long long limit) {
    if (__builtin_expect(__all_sync(0xffffffffu, sm100::mbar_try_wait(bar, parity)), 1)) return true;
    return !out_of_time(abort, limit) && warp_wait(bar, parity, abort, limit);
}

// Both barriers at once (they may be the same).
__device__ __forceinline__ bool quick_wait2(uint64_t *b1, uint32_t p1, uint64_t *b2, uint32_t p2, volatile int *abort,
                                            long long limit) {
    const bool r1 = sm100::mbar_try_wait(b1, p1), r2 = sm100::mbar_try_wait(b2, p2);
    if (__builtin_expect(__all_sync(0xffffffffu, r1 && r2), 1)) return true;
    return !out_of_time(abort, limit) && warp_wait(b1, p1, abort, limit) && warp_wait(b2, p2, abort, limit);
}

}  // namespace rs
