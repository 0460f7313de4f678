// What the kernels share whose rows travel through a private ring in shared memory: asynchronous copies, packed FP32 pairs,
// sums over the threads of a row.
#pragma once

#include "common.cuh"

namespace fp8dpa {

#if defined(__CUDACC__)

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Rows travel through a private ring in shared memory: every thread copies what it alone reads, so it needs no barrier.
__device__ __forceinline__ uint4 ring_get(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void ring_put_zero(uint32_t at)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0u) : "memory");
}
__device__ __forceinline__ void ring_put(uint32_t at, uint64_t lo, uint64_t hi)
{
    asm volatile("st.shared.v2.b64 [%0], {%1, %2};" ::"r"(at), "l"(lo), "l"(hi) : "memory");
}
__device__ __forceinline__ void ring_get(uint32_t at, uint64_t &lo, uint64_t &hi)
{
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(lo), "=l"(hi) : "r"(at) : "memory");
}

// Eight BF16 values as four pairs for the packed FP32 instructions (two lanes each).
__device__ __forceinline__ void unpack4x2(const uint4 v, uint64_t (&f)[4])
{
    f[0] = pack_u32x2(v.x << 16, v.x & 0xFFFF0000u);
    f[1] = pack_u32x2(v.y << 16, v.y & 0xFFFF0000u);
    f[2] = pack_u32x2(v.z << 16, v.z & 0xFFFF0000u);
    f[3] = pack_u32x2(v.w << 16, v.w & 0xFFFF0000u);
}
__device__ __forceinline__ void load4x2(const float *p, uint64_t (&f)[4])
{
    const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
    f[0] = pack_f32x2(a.x, a.y);
    f[1] = pack_f32x2(a.z, a.w);
    f[2] = pack_f32x2(b.x, b.y);
    f[3] = pack_f32x2(b.z, b.w);
}
__device__ __forceinline__ uint64_t both(float v) { return pack_f32x2(v, v); }
__device__ __forceinline__ float add_halves(uint64_t v)
{
    float lo, hi;
    unpack_f32x2(v, lo, hi);
    return lo + hi;
}
__device__ __forceinline__ float4 quad(uint64_t a, uint64_t b)
{
    float4 v;
    unpack_f32x2(a, v.x, v.y);
    unpack_f32x2(b, v.z, v.w);
    return v;
}
__device__ __forceinline__ uint32_t round2(uint64_t v)
{
    float lo, hi;
    unpack_f32x2(v, lo, hi);
    return pack_bf16x2(lo, hi);
}

// max(m, |a|, |b|); NaN stays.  Rounding to BF16 keeps the order, so that an amax can be taken of the values before it and be
// rounded once: half the instructions of the maximum of the packed results.
__device__ __forceinline__ float absmax3(float m, float a, float b)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float absmax3(float m, uint64_t v)
{
    float lo, hi;
    unpack_f32x2(v, lo, hi);
    return absmax3(m, lo, hi);
}
// Eight BF16 values to eight FP8 codes under the scale in both halves of `scale2`: fp8_cast's (binary32 product, one rounding).
__device__ __forceinline__ uint2 codes8(const uint4 w, uint64_t scale2, int fmt)
{
    uint64_t f[4];
    float v[8];
    unpack4x2(w, f);
#pragma unroll
    for (int e = 0; e < 4; ++e) unpack_f32x2(mul_f32x2(f[e], scale2), v[2 * e], v[2 * e + 1]);
    if (fmt == 0) return make_uint2(cvt_f32x4_to_fp8x4<0>(v[0], v[1], v[2], v[3]), cvt_f32x4_to_fp8x4<0>(v[4], v[5], v[6], v[7]));
    return make_uint2(cvt_f32x4_to_fp8x4<1>(v[0], v[1], v[2], v[3]), cvt_f32x4_to_fp8x4<1>(v[4], v[5], v[6], v[7]));
}

// Sum over the threads that share a row: 2^lanes_log2 neighbouring lanes, or the whole CTA of up to WARPS warps through `red` (a
// buffer that this call alone uses until the next barrier; entries behind the CTA's warps are zero).
template <bool CTA, int WARPS>
__device__ __forceinline__ float row_sum(float v, int lanes_log2, float *red)
{
    switch (CTA ? 5 : lanes_log2) {
    case 5: v += __shfl_xor_sync(0xffffffffu, v, 16);
    case 4: v += __shfl_xor_sync(0xffffffffu, v, 8);
    case 3: v += __shfl_xor_sync(0xffffffffu, v, 4);
    case 2: v += __shfl_xor_sync(0xffffffffu, v, 2);
    case 1: v += __shfl_xor_sync(0xffffffffu, v, 1);
    }
    if (CTA) {
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; w += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(red + w);
            v += (q.x + q.y) + (q.z + q.w);
        }
    }
    return v;
}

// Who takes a row: 2^lanes_log2 lanes of a warp, a warp, or the CTA.
enum RowUnit { ROW_LANES, ROW_WARP, ROW_CTA };

// The rows of unit u of n: a contiguous share.
struct Rows {
    size_t begin, end;
};
__device__ __forceinline__ Rows rows_of(size_t u, size_t n, size_t T) { return {T * u / n, T * (u + 1) / n}; }

// Two vectors of D columns (each may be missing) from the CTAs' sums in `partial` [CTA][2][D]: 32 columns per CTA, a warp takes
// every 32nd of the sums, then the warps in order.  MAXIMA: the first CTA also leaves the largest of `maxima` [CTA] (bits of values
// that are not negative) in *amax.
template <bool MAXIMA>
static __global__ void __launch_bounds__(1024) column_sums_kernel(const float *__restrict__ partial, int parts, unsigned D,
                                                                  float *__restrict__ first, float *__restrict__ second,
                                                                  int accumulate, const unsigned int *__restrict__ maxima,
                                                                  unsigned int *__restrict__ amax)
{
    cudaGridDependencySynchronize();
    __shared__ float red[32][33];
    __shared__ unsigned int most;
    if (MAXIMA && blockIdx.x == 0) {
        if (threadIdx.x == 0) most = 0u;
        __syncthreads();
        unsigned int m = 0u;
        for (int c = threadIdx.x; c < parts; c += 1024) m = max(m, __ldcg(maxima + c));
        m = __reduce_max_sync(0xffffffffu, m);
        if ((threadIdx.x & 31) == 0) atomicMax(&most, m);
        __syncthreads();
        if (threadIdx.x == 0) *amax = most;
    }
    const unsigned j = blockIdx.x * 32 + (threadIdx.x & 31);      // over [2][D]
    const int r = threadIdx.x >> 5;
    float s = 0.0f;
    if (j < 2 * D && (j < D ? first : second)) {
#pragma unroll 8
        for (int c = r; c < parts; c += 32) s += __ldcg(partial + (size_t)c * 2 * D + j);
    }
    red[r][threadIdx.x & 31] = s;
    __syncthreads();
    s = red[threadIdx.x & 31][r];                                 // transposed: warp r adds the 32 sums of column r
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    const unsigned col = blockIdx.x * 32 + r;
    if ((threadIdx.x & 31) == 0 && col < 2 * D && (col < D ? first : second)) {
        float *o = col < D ? first + col : second + (col - D);
        *o = accumulate ? *o + s : s;
    }
}

#endif  // __CUDACC__

static inline int log2_at_least(unsigned n)
{
    int l = 0;
    while ((1u << l) < n) ++l;
    return l;
}

}  // namespace fp8dpa
