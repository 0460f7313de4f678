// Stable ranks of a tile of digits inside a CTA: the building block of the counting sorts (token ids of the embedding
// gradient, experts of the router).
#pragma once

#include "common.cuh"

namespace fp8dpa {

#if defined(__CUDACC__)

// Each warp ranks 32 consecutive digits per call, in lane order, on top of what it counted before: `counts` is the warp's
// own row of counters in shared memory.  Returns how many equal digits of this warp came before this lane's.  Lanes with
// digit < 0 take no part; the others' digits have `bits` bits.  All 32 lanes call.  Cnt: int, or uint16_t where no count
// passes 65535.  The lanes with the same digit are found by one ballot per bit.
template <typename Cnt>
__device__ __forceinline__ int warp_stable_rank(int digit, int bits, Cnt *counts, int lane)
{
    uint32_t peers = __ballot_sync(0xffffffffu, digit >= 0);
    for (int b = 0; b < bits; ++b) {
        const bool one = (digit >> b) & 1;
        const uint32_t ones = __ballot_sync(0xffffffffu, one);
        peers &= one ? ones : ~ones;
    }
    const int before = __popc(peers & ((1u << lane) - 1u));
    int base = 0;
    if (digit >= 0) base = counts[digit];
    __syncwarp();
    if (digit >= 0 && before == 0) counts[digit] = (Cnt)(base + __popc(peers));
    __syncwarp();
    return base + before;
}

#endif  // __CUDACC__

}  // namespace fp8dpa
