// Stable ranks of a tile of digits inside a CTA: the building block of the counting sorts (token ids of the embedding
// gradient, experts of the router).
#pragma once

#include "common.cuh"

namespace fp8dpa {

#if defined(__CUDACC__)

// Each warp ranks 32 consecutive digits per call, in lane order, on top of what it counted before: `counts` is the warp's
// own row of counters in shared memory.  Returns how many equal digits of this warp came before this lane's.  Lanes with
// digit < 0 take no part.  All 32 lanes call.
__device__ __forceinline__ int warp_stable_rank(int digit, int *counts, int lane)
{
    const uint32_t peers = __match_any_sync(0xffffffffu, digit);
    const int before = __popc(peers & ((1u << lane) - 1u));
    int base = 0;
    if (digit >= 0) base = counts[digit];
    __syncwarp();
    if (digit >= 0 && before == 0) counts[digit] = base + __popc(peers);
    __syncwarp();
    return base + before;
}

#endif  // __CUDACC__

}  // namespace fp8dpa
