// Bounded waits of whole warps on mbarriers (gva_decode_mma.cuh has those of single threads).
#pragma once

#include "gva_decode_mma.cuh"

namespace gva {

// Bounded wait of a whole warp, straight-line where the phase is complete already, as it mostly is (with one lane waiting and the others
// behind a shuffle it took 100 cycles more).  Bounded like mbar_wait_bounded: kWaitLimitNs of wall time -- how long a poll takes that
// finds nothing is the hardware's choice (4 us measured), so a number of polls bounds nothing -- or until another warp of the block has given up.
__device__ __forceinline__ bool warp_gives_up(unsigned long long &t0, const volatile int *abort_flag) {
    const unsigned long long now = __shfl_sync(0xffffffffu, global_timer_ns(), 0);       // (one reading, so that all lanes leave together)
    if (t0 == 0) t0 = now;
    return now - t0 > kWaitLimitNs || (abort_flag && __any_sync(0xffffffffu, *abort_flag));
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const volatile int *abort_flag) {
    unsigned long long t0 = 0;
    for (uint32_t it = 0; !__all_sync(0xffffffffu, mbar_try_wait(bar, parity));)
        if (__builtin_expect((++it & 127u) == 0, 0) && warp_gives_up(t0, abort_flag)) return false;
    return true;
}
// Both of two phases: what they cost when complete overlaps.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, uint32_t bar2, uint32_t parity2, const volatile int *abort_flag) {
    unsigned long long t0 = 0;
    for (uint32_t it = 0;;) {
        const bool one = mbar_try_wait(bar, parity), two = mbar_try_wait(bar2, parity2);
        if (__all_sync(0xffffffffu, one && two)) return true;
        if (__builtin_expect((++it & 127u) == 0, 0) && warp_gives_up(t0, abort_flag)) return false;
    }
}

}  // namespace gva
