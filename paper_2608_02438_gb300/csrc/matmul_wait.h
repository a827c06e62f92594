// matmul_wait.h -- the bounded waits of the block-scaled 8-bit product's kernels.
// Besides mbar_try_wait and clock64 this is plain C++: the CPU tests compile it
// with stand-ins for the two.
#pragma once

#include <cstdint>

namespace xp {

// Bounded wait for a phase of `bar`.  It polls (a wait with a sleep hint wakes
// up later: an earlier form at 2048 x 38912 x 4096 took 739 us against 683) and bounds itself by
// the SM's cycle counter, read once in 64 polls: the global timer's latency
// would sit in every hand-off of a K block.  It gives up early where *abort is
// set, unless abort is NULL.  `since` (0 at the kernel's start) makes one limit of
// all the waits that name it: it counts from the first of them that had to wait.
constexpr long long MM_WAIT_CYCLES = 4000000000ll;       // about 2 s
__device__ __forceinline__ bool mm_wait(uint64_t *bar, uint32_t parity, volatile int *abort,
                                        long long cycles = MM_WAIT_CYCLES, volatile long long *since = nullptr)
{
    long long t0 = 0;
    for (uint32_t it = 1;; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 63u) == 0) {
            if (abort && *abort) return false;
            const long long t = clock64();
            if (t0 == 0) {
                t0 = t;
                if (since) {
                    if (*since == 0) *since = t;
                    t0 = *since;
                }
            }
            if (t - t0 > cycles) {
                if (abort) *abort = 1;
                return false;
            }
        }
    }
}

// Wait for the sums that the CTAs of the cluster send to this one.  They land in
// its shared memory, so it may not leave before they have, whatever became of its
// own work: this wait takes no notice of *abort, and outlasts the senders.  (Their
// waits share one limit, MM_WAIT_CYCLES, and end in their stores.)
__device__ __forceinline__ bool mm_wait_joined(uint64_t *bar, volatile int *abort)
{
    if (mm_wait(bar, 0, nullptr, 3 * MM_WAIT_CYCLES)) return true;
    *abort = 1;
    return false;
}

}  // namespace xp
