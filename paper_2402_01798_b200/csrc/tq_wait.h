// Waits of the product kernels: plain control flow, shared by the kernels and a host program that runs it.
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

}  // namespace tq
