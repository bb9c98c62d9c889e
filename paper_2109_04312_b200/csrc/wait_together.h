// A bounded wait of a whole warp (no CUDA in it, so that it can be tested without a GPU).
#pragma once
#include <cstdint>

namespace mate {

// Every lane calls it, and all of them get the same answer: true if what is waited for is there, false if nobody found it for `tries` tries or somebody
// else has given up meanwhile.  What follows needs all lanes (votes, tensor memory, barriers): one that had left by itself, because it saw the flag where
// the others saw the phase end, would be waited for without a bound.
template <typename W>
#ifdef __CUDACC__
__device__ __forceinline__
#else
inline
#endif
bool wait_together(const W &w, uint32_t tries) {
#pragma unroll 1
    for (uint32_t i = 0; i < tries; ++i) {
        if (w.all(w.there())) return true;
        if (w.any(w.given_up())) return false;
    }
    w.give_up();
    return false;
}

}  // namespace mate
