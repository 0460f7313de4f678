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

// A grid that is one cluster sets *amax to zero itself: its first thread at the start, before a cluster barrier that everybody
// passes in front of the atomicMax.  Both calls by all threads.
__device__ __forceinline__ bool amax_begin(unsigned int *amax)
{
    uint32_t ctas;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
    const bool alone = amax && ctas == gridDim.x;
    if (alone) {
        if (blockIdx.x == 0 && threadIdx.x == 0) *amax = 0u;
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    }
    return alone;
}
__device__ __forceinline__ void amax_end(uint32_t m2, unsigned int *amax, bool alone)
{
    cudaGridDependencySynchronize();
    if (alone) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    if (amax) block_max_bf16_to(m2, amax);
}

// Whether a cluster of 16 CTAs of up to 256 threads with `smem` bytes each finds room on the current device (clusters of more than
// 8 need not, on a partition of a GPU for instance).  The runtime is asked once per kernel, device and size of shared memory
// beyond what is known to fit.
template <auto Kernel>
static bool cluster_of_16_fits(int dev, size_t smem)
{
    static size_t fits[64] = {0}, fails[64] = {0};        // bytes + 1: the most that fit, the fewest that do not
    const bool known = dev >= 0 && dev < 64;
    if (known && smem < fits[dev]) return true;
    if (known && fails[dev] && smem + 1 >= fails[dev]) return false;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(16);
    c.blockDim = dim3(256);
    c.dynamicSmemBytes = smem;
    cudaLaunchAttribute a[1];
    a[0].id = cudaLaunchAttributeClusterDimension;
    a[0].val.clusterDim.x = 16;
    a[0].val.clusterDim.y = a[0].val.clusterDim.z = 1;
    c.attrs = a;
    c.numAttrs = 1;
    int clusters = 0;
    const bool ok = cudaFuncSetAttribute(Kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                    cudaOccupancyMaxActiveClusters(&clusters, Kernel, &c) == cudaSuccess && clusters > 0;
    if (!ok) cudaGetLastError();                          // a refusal is an answer, not an error of the call
    if (known) (ok ? fits : fails)[dev] = smem + 1;
    return ok;
}

// Launches a kernel that raises *amax between amax_begin and amax_end.  A grid of up to 16 CTAs is one cluster (see above), or
// up to 8 where a CTA may fill an SM or the device has no room for 16: a layer norm of 8 x 4096 takes 3.2 us in a graph and 7.9
// us of the host with its binding, 6.2 and 9.3 with a memset in front.  In front of other grids *amax is set to zero by a
// memset, which has to end before the kernel starts; for large tensors by a kernel of one thread, and the main kernel, which
// waits for it only in front of the atomicMax (cudaGridDependencySynchronize), starts beside it.  The second launch costs the
// host 2.5 us more, so from 2^24 elements on, where the device is busy longer than the host (8192 x 4096: 43.4 -> 42.7 us for
// the layer norm with residual and codes, 27.6 -> 26.9 us for the embedding).
constexpr size_t AMAX_EARLY_ELEMENTS = (size_t)1 << 24;
template <auto Kernel, typename P>
static int launch_behind_amax(size_t elements, unsigned int *amax, unsigned grid, unsigned threads, size_t smem, cudaStream_t st,
                              const P &p, int n)
{
    bool cluster = amax && grid > 1 && grid <= (threads <= 256 ? 16u : 8u);
    if (cluster && grid > 8) {
        int dev = -1;
        FP8_CUDA_CHECK(cudaGetDevice(&dev));
        cluster = cluster_of_16_fits<Kernel>(dev, smem);
    }
    if (cluster) {
        cudaLaunchConfig_t c = {};
        c.gridDim = dim3(grid);
        c.blockDim = dim3(threads);
        c.dynamicSmemBytes = smem;
        c.stream = st;
        cudaLaunchAttribute a[1];
        a[0].id = cudaLaunchAttributeClusterDimension;
        a[0].val.clusterDim.x = grid;
        a[0].val.clusterDim.y = a[0].val.clusterDim.z = 1;
        c.attrs = a;
        c.numAttrs = 1;
        FP8_CUDA_CHECK(cudaLaunchKernelEx(&c, Kernel, p, n));
        return FP8_OK;
    }
    if (amax && grid > 1 && elements >= AMAX_EARLY_ELEMENTS) {
        zero_word_kernel<<<1, 1, 0, st>>>(amax);
        FP8_CUDA_CHECK(cudaGetLastError());
        return launch_early(Kernel, grid, threads, smem, st, p, n);
    }
    if (amax && grid > 1) FP8_CUDA_CHECK(cudaMemsetAsync(amax, 0, sizeof(float), st));
    Kernel<<<grid, threads, smem, st>>>(p, n);
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
}

#endif  // __CUDACC__

}  // namespace fp8dpa
