// Waits of the product kernels and what a kernel that gives one up has to see ended before its blocks leave: plain arithmetic and control flow, shared by
// the kernels and a host program that runs them against a simulated ring.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define TQ_WAIT_FN __host__ __device__ __forceinline__
#else
#define TQ_WAIT_FN inline
#endif

namespace tq {

// Polls until poll() holds, and gives up after `limit` polls in which progress() has not changed: a wait for a whole sum is as long as the sum, and goes on
// while its stages are filled.  Every 256 polls it looks at that, and whether another thread of the block has given up; a wait that ends at once reads neither.
template <class Poll, class Dead, class Progress>
TQ_WAIT_FN bool wait_with_progress(uint32_t limit, Poll poll, Dead dead, Progress progress) {
    uint32_t seen = 0, since = 0;
    for (uint32_t it = 1; since < limit; ++it, ++since) {
        if (poll()) return true;
        if (it % 256 == 0) {
            if (dead()) return false;
            const uint32_t now = progress();
            if (now != seen) { seen = now; since = 0; }
        }
    }
    return false;
}

// A ring of `stages`, filled `issued` times in turn: f(stage, parity) for each filling that may still be on its way, parity being that of its phase on the
// stage's barrier.  A stage is filled again only when its last filling has been read, so those before have landed.
template <class F>
TQ_WAIT_FN void for_outstanding(uint32_t issued, uint32_t stages, F f) {
    for (uint32_t j = issued > stages ? issued - stages : 0; j < issued; ++j) f(j % stages, (j / stages) & 1);
}

// The same for a pair of blocks, each of which fills its half of a stage while the bytes of both count on the first block's barrier; the first block's filling is
// also what expects them.  f(stage, parity, by): 3 where both have filled; 1 where only the first has: the second's bytes are expected but will not
// come; 2 where only the second has: its bytes come unexpected, and the phase has had no arrival.  Neither gets further ahead than the ring is long.
template <class F>
TQ_WAIT_FN void for_outstanding_of_pair(uint32_t issued0, uint32_t issued1, uint32_t stages, F f) {
    const uint32_t most = issued0 > issued1 ? issued0 : issued1;
    for (uint32_t j = most > stages ? most - stages : 0; j < most; ++j) f(j % stages, (j / stages) & 1, (j < issued0 ? 1u : 0u) | (j < issued1 ? 2u : 0u));
}

}  // namespace tq
