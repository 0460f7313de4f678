// What the element-wise kernels share: the block maximum behind an amax output and the cast of eight BF16 values.
#pragma once

#include "common.cuh"

namespace fp8dpa {

#if defined(__CUDACC__)

__device__ __forceinline__ uint32_t absmax2e(uint32_t m, uint32_t w) { return __vmaxu2(m, w & 0x7FFF7FFFu); }

__device__ __forceinline__ void block_max_bf16_to(uint32_t m2, unsigned int *amax_bits)
{
    __shared__ uint32_t warp_max[32];
    uint32_t m = max(m2 & 0xFFFFu, m2 >> 16);
    m = __reduce_max_sync(0xffffffffu, m);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) warp_max[warp] = m;
    __syncthreads();
    if (warp == 0) {
        const int nwarps = (blockDim.x + 31) >> 5;
        m = lane < nwarps ? warp_max[lane] : 0u;
        m = __reduce_max_sync(0xffffffffu, m);
        if (lane == 0 && m != 0u) atomicMax(amax_bits, m << 16);
    }
}

// Eight BF16 values (four packed words) -> eight FP8 codes under `scale`: the codes fp8_cast gives for the same
// values (binary32 product, one rounding to FP8).  fmt: 0 = E4M3, 1 = E5M2.
__device__ __forceinline__ uint2 bf16x8_to_fp8x8(const uint32_t (&w)[4], float scale, int fmt)
{
    const float v0 = __fmul_rn(bf16_lo(w[0]), scale), v1 = __fmul_rn(bf16_hi(w[0]), scale);
    const float v2 = __fmul_rn(bf16_lo(w[1]), scale), v3 = __fmul_rn(bf16_hi(w[1]), scale);
    const float v4 = __fmul_rn(bf16_lo(w[2]), scale), v5 = __fmul_rn(bf16_hi(w[2]), scale);
    const float v6 = __fmul_rn(bf16_lo(w[3]), scale), v7 = __fmul_rn(bf16_hi(w[3]), scale);
    if (fmt == 0) return make_uint2(cvt_f32x4_to_fp8x4<0>(v0, v1, v2, v3), cvt_f32x4_to_fp8x4<0>(v4, v5, v6, v7));
    return make_uint2(cvt_f32x4_to_fp8x4<1>(v0, v1, v2, v3), cvt_f32x4_to_fp8x4<1>(v4, v5, v6, v7));
}

static __global__ void zero_word_kernel(unsigned int *word) { *word = 0u; }

// Launches a kernel that raises *amax with atomicMax at its end, behind what sets *amax to zero.  A memset has to end before
// the kernel starts; for large tensors a kernel of one thread does it instead and the main kernel, which waits for it only in
// front of the atomicMax (cudaGridDependencySynchronize), starts beside it.  The second launch costs the host 2.5 us more, so
// from 2^24 elements on, where the device is busy longer than the host (8192 x 4096: 43.4 -> 42.7 us for the layer norm
// with residual and codes, 27.6 -> 26.9 us for the embedding).
constexpr size_t AMAX_EARLY_ELEMENTS = (size_t)1 << 24;
template <typename... P, typename... A>
static int launch_behind_amax(void (*kernel)(P...), size_t elements, unsigned int *amax, unsigned grid, unsigned threads,
                              size_t smem, cudaStream_t st, A... args)
{
    if (amax && elements >= AMAX_EARLY_ELEMENTS) {
        zero_word_kernel<<<1, 1, 0, st>>>(amax);
        FP8_CUDA_CHECK(cudaGetLastError());
        return launch_early(kernel, grid, threads, smem, st, args...);
    }
    if (amax) FP8_CUDA_CHECK(cudaMemsetAsync(amax, 0, sizeof(float), st));
    kernel<<<grid, threads, smem, st>>>(args...);
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
}

#endif  // __CUDACC__

}  // namespace fp8dpa
