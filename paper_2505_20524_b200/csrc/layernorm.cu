// Layer norm: out = residual + gamma (x - mean) / sqrt(var + eps) + beta per token row, with the amax and the FP8 codes of
// the result for the next product, and its backward pass with the reduction of dgamma and dbeta.
#include <math.h>

#include "common.cuh"
#include "elementwise.cuh"

namespace fp8dpa {

// Rows per thread group in flight or in use.  Two rows ahead are enough: 8192 x 4096 takes the same time with 4, 5 and 6.
constexpr int LN_STAGES = 3;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A thread's private ring in shared memory: LN_STAGES rows of KG 16-byte groups of each of two tensors.  Every thread copies
// what it alone reads, so the ring needs no barrier.
template <int KG>
struct Ring {
    uint32_t base;
    __device__ __forceinline__ uint32_t slot(int stage, int tensor, int k) const
    {
        return base + (uint32_t)(((stage * 2 + tensor) * KG + k) * blockDim.x) * 16u;
    }
    __device__ __forceinline__ uint4 get(int stage, int tensor, int k) const
    {
        uint4 v;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(slot(stage, tensor, k)) : "memory");
        return v;
    }
};
template <int KG> static size_t ring_bytes(unsigned threads) { return (size_t)LN_STAGES * 2 * KG * 16 * threads; }

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

// Sums over the threads that share a row: a warp, or the whole CTA through `red` (a buffer that this call alone uses until
// the next barrier; 32 entries, those behind the CTA's warps zero).
template <bool WARP>
__device__ __forceinline__ float row_sum(float v, float *red)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if (!WARP) {
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.0f;
        for (unsigned w = 0; w < (blockDim.x >> 5); w += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(red + w);
            v += (q.x + q.y) + (q.z + q.w);
        }
    }
    return v;
}

// ---------------------------------------------------------------- forward
struct LnFwd {
    const uint16_t *x;
    const float *gamma, *beta;
    const uint16_t *residual;
    size_t T;
    unsigned n8;
    float eps;
    uint16_t *out;
    float *mean, *rstd;
    unsigned int *amax_bits;
    const float *q_scale;
    uint8_t *out8;
    int fmt;
};

// A row belongs to a warp (WARP) or to the CTA; its threads hold KG groups of eight columns each, gamma and beta of them in
// registers for all the rows they come by (every gridDim-th: neighbouring CTAs read neighbouring rows, 38.5 us against 41.8
// with a contiguous share each at 8192 x 4096 with residual and codes), and the row itself between the two sums (the mean, then the squared distances
// from it: no cancellation however far the mean lies from zero) and the result: one read of x.  Persistent; the next rows
// travel while one is worked on.
template <int KG, bool WARP, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) layernorm_fwd_kernel(const LnFwd p)
{
    extern __shared__ __align__(16) uint4 ring_mem[];
    __shared__ __align__(16) float red[2][32];
    const Ring<KG> ring{smem_u32(ring_mem + threadIdx.x)};
    const unsigned lane = WARP ? threadIdx.x & 31 : threadIdx.x, span = WARP ? 32 : blockDim.x;
    const unsigned groups = WARP ? blockDim.x >> 5 : 1;
    if (!WARP) {
        for (unsigned i = threadIdx.x; i < 64; i += blockDim.x) red[i >> 5][i & 31] = 0.0f;
        __syncthreads();
    }
    const size_t step = (size_t)gridDim.x * groups, t_first = (size_t)blockIdx.x * groups + (WARP ? threadIdx.x >> 5 : 0);
    const float qs = p.out8 ? __ldg(p.q_scale) : 1.0f;
    const float inv_d = 1.0f / (float)(p.n8 * 8);
    const uint4 *x = reinterpret_cast<const uint4 *>(p.x), *res = reinterpret_cast<const uint4 *>(p.residual);
    const auto fetch = [&](size_t t, int stage) {
        if (t < p.T) {
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                const unsigned i = k * span + lane;
                if (i >= p.n8) continue;
                cp_async16(ring.slot(stage, 0, k), x + t * p.n8 + i);
                if (res) cp_async16(ring.slot(stage, 1, k), res + t * p.n8 + i);
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < LN_STAGES - 1; ++s) fetch(t_first + s * step, s);
    uint64_t g[KG][4], b[KG][4];
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        const unsigned i = k * span + lane;
#pragma unroll
        for (int e = 0; e < 4; ++e) g[k][e] = b[k][e] = 0ull;
        if (i < p.n8) {
            load4x2(p.gamma + 8 * i, g[k]);
            load4x2(p.beta + 8 * i, b[k]);
        }
    }
    uint32_t m = 0;
    int stage = 0;
    for (size_t t = t_first; t < p.T; t += step) {
        cp_async_wait<LN_STAGES - 2>();
        fetch(t + (LN_STAGES - 1) * step, stage == 0 ? LN_STAGES - 1 : stage - 1);     // the stage of the row before this one
        uint64_t f[KG][4], s = 0ull;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const bool in = k * span + lane < p.n8;
            unpack4x2(in ? ring.get(stage, 0, k) : make_uint4(0u, 0u, 0u, 0u), f[k]);
            s = add_f32x2(s, add_f32x2(add_f32x2(f[k][0], f[k][1]), add_f32x2(f[k][2], f[k][3])));
        }
        const float mean = row_sum<WARP>(add_halves(s), red[0]) * inv_d;
        const uint64_t minus_mean = both(-mean);
        uint64_t ss = 0ull;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            if (k * span + lane >= p.n8) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[k][e] = add_f32x2(f[k][e], minus_mean);
                ss = fma_f32x2(f[k][e], f[k][e], ss);
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<WARP>(add_halves(ss), red[1]) * inv_d + p.eps);
        const uint64_t rstd2 = both(rstd);
        if (lane == 0) {
            if (p.mean) p.mean[t] = mean;
            if (p.rstd) p.rstd[t] = rstd;
        }
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const unsigned i = k * span + lane;
            if (i >= p.n8) continue;
            uint64_t r[4];
            if (res) unpack4x2(ring.get(stage, 1, k), r);
            uint32_t o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint64_t y = fma_f32x2(mul_f32x2(f[k][q], rstd2), g[k][q], b[k][q]);
                if (res) y = add_f32x2(y, r[q]);
                o[q] = round2(y);
                m = absmax2e(m, o[q]);
            }
            reinterpret_cast<uint4 *>(p.out)[t * p.n8 + i] = make_uint4(o[0], o[1], o[2], o[3]);
            if (p.out8) reinterpret_cast<uint2 *>(p.out8)[t * p.n8 + i] = bf16x8_to_fp8x8(o, qs, p.fmt);
        }
        stage = stage == LN_STAGES - 1 ? 0 : stage + 1;
    }
    cudaGridDependencySynchronize();
    if (p.amax_bits) block_max_bf16_to(m, p.amax_bits);
}

// ---------------------------------------------------------------- backward
// The rows of unit u of n: a contiguous share.
struct Rows {
    size_t begin, end;
};
__device__ __forceinline__ Rows rows_of(size_t u, size_t n, size_t T) { return {T * u / n, T * (u + 1) / n}; }

struct LnBwd {
    const uint16_t *dout, *x;
    const float *gamma, *mean, *rstd;
    size_t T;
    unsigned n8;
    uint16_t *dx;
    float *partial;
};

// With xh = (x - mean) rstd and g = gamma dout:  dx = rstd (g - mean(g) - xh mean(g xh)), dgamma = sum over rows of dout xh,
// dbeta = sum over rows of dout.  Persistent, rows and columns on threads as in the forward; a thread keeps its columns'
// dgamma and dbeta in registers over all its rows, and the CTA leaves them in `partial` [CTA][2][D] for
// layernorm_bwd_sum_kernel.  x and dout are read once, dx is written once.  A warp loads mean and rstd
// of 32 of its rows at a time: when all CTAs read those of neighbouring rows one by one, the few lines that hold them were
// what bound the kernel (8192 x 4096: 52.7 us).  KEEP: xh, g and gamma stay in registers between
// the sums and dx; for long rows (KG = 4) they are formed again from the ring.
template <int KG, bool WARP, bool KEEP, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) layernorm_bwd_kernel(const LnBwd p)
{
    cudaTriggerProgrammaticLaunchCompletion();
    extern __shared__ __align__(16) uint4 ring_mem[];
    __shared__ __align__(16) float2 red[2][32];
    const Ring<KG> ring{smem_u32(ring_mem + threadIdx.x)};
    const unsigned lane = WARP ? threadIdx.x & 31 : threadIdx.x, span = WARP ? 32 : blockDim.x;
    const unsigned groups = WARP ? blockDim.x >> 5 : 1, group = WARP ? threadIdx.x >> 5 : 0;
    const Rows rows = rows_of((size_t)blockIdx.x * groups + group, (size_t)gridDim.x * groups, p.T);
    const float inv_d = 1.0f / (float)(p.n8 * 8);
    if (!WARP) {
        for (unsigned i = threadIdx.x; i < 64; i += blockDim.x) red[i >> 5][i & 31] = make_float2(0.0f, 0.0f);
        __syncthreads();
    }
    const uint4 *x = reinterpret_cast<const uint4 *>(p.x), *dout = reinterpret_cast<const uint4 *>(p.dout);
    const auto fetch = [&](size_t t, int stage) {
        if (t < rows.end) {
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                const unsigned i = k * span + lane;
                if (i >= p.n8) continue;
                cp_async16(ring.slot(stage, 0, k), x + t * p.n8 + i);
                cp_async16(ring.slot(stage, 1, k), dout + t * p.n8 + i);
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < LN_STAGES - 1; ++s) fetch(rows.begin + s, s);
    constexpr int KK = KEEP ? KG : 1;
    uint64_t dg[KG][4], db[KG][4], gm[KK][4];
#pragma unroll
    for (int k = 0; k < KG; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) dg[k][e] = db[k][e] = 0ull;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
#pragma unroll
        for (int e = 0; e < 4; ++e) gm[k][e] = 0ull;
        if (KEEP && k * span + lane < p.n8) load4x2(p.gamma + 8 * (k * span + lane), gm[k]);
    }
    int stage = 0, flip = 0;
    float mu32 = 0.0f, rs32 = 0.0f, mu_ahead = 0.0f, rs_ahead = 0.0f;      // lane l: the statistics of row l of a batch of 32
    if (rows.begin + (threadIdx.x & 31) < rows.end) {
        mu_ahead = __ldg(p.mean + rows.begin + (threadIdx.x & 31));
        rs_ahead = __ldg(p.rstd + rows.begin + (threadIdx.x & 31));
    }
    for (size_t t = rows.begin; t < rows.end; ++t, flip ^= 1) {
        cp_async_wait<LN_STAGES - 2>();
        fetch(t + LN_STAGES - 1, stage == 0 ? LN_STAGES - 1 : stage - 1);
        const unsigned in_batch = (unsigned)(t - rows.begin) & 31u;
        if (in_batch == 0) {                     // the next 32 rows' statistics; the batch behind them is on its way
            mu32 = mu_ahead;
            rs32 = rs_ahead;
            const size_t ahead = t + 32 + (threadIdx.x & 31);
            if (ahead < rows.end) {
                mu_ahead = __ldg(p.mean + ahead);
                rs_ahead = __ldg(p.rstd + ahead);
            }
        }
        const float mu = __shfl_sync(0xffffffffu, mu32, in_batch), rs = __shfl_sync(0xffffffffu, rs32, in_batch);
        const uint64_t minus_mu = both(-mu), rs2 = both(rs);
        uint64_t xh[KK][4], ge[KK][4], a1 = 0ull, a2 = 0ull;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const unsigned i = k * span + lane;
            const int kk = KEEP ? k : 0;
            if (i >= p.n8) continue;
            uint64_t d[4];
            unpack4x2(ring.get(stage, 0, k), xh[kk]);
            unpack4x2(ring.get(stage, 1, k), d);
            if (!KEEP) load4x2(p.gamma + 8 * i, gm[0]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                xh[kk][e] = mul_f32x2(add_f32x2(xh[kk][e], minus_mu), rs2);
                ge[kk][e] = mul_f32x2(d[e], gm[kk][e]);
                dg[k][e] = fma_f32x2(d[e], xh[kk][e], dg[k][e]);
                db[k][e] = add_f32x2(db[k][e], d[e]);
                a1 = add_f32x2(a1, ge[kk][e]);
                a2 = fma_f32x2(ge[kk][e], xh[kk][e], a2);
            }
        }
        float s1 = add_halves(a1), s2 = add_halves(a2);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            s1 += __shfl_xor_sync(0xffffffffu, s1, off);
            s2 += __shfl_xor_sync(0xffffffffu, s2, off);
        }
        if (!WARP) {         // two buffers in turn: the next row's writes do not meet this row's reads
            if ((threadIdx.x & 31) == 0) red[flip][threadIdx.x >> 5] = make_float2(s1, s2);
            __syncthreads();
            s1 = s2 = 0.0f;
            for (unsigned w = 0; w < (blockDim.x >> 5); w += 2) {
                const float4 v = *reinterpret_cast<const float4 *>(&red[flip][w]);
                s1 += v.x + v.z;
                s2 += v.y + v.w;
            }
        }
        const uint64_t minus_m1 = both(-s1 * inv_d), minus_m2 = both(-s2 * inv_d);
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const unsigned i = k * span + lane;
            const int kk = KEEP ? k : 0;
            if (i >= p.n8) continue;
            if (!KEEP) {
                uint64_t d[4];
                unpack4x2(ring.get(stage, 0, k), xh[0]);
                unpack4x2(ring.get(stage, 1, k), d);
                load4x2(p.gamma + 8 * i, gm[0]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    xh[0][e] = mul_f32x2(add_f32x2(xh[0][e], minus_mu), rs2);
                    ge[0][e] = mul_f32x2(d[e], gm[0][e]);
                }
            }
            uint32_t o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                o[q] = round2(mul_f32x2(rs2, fma_f32x2(xh[kk][q], minus_m2, add_f32x2(ge[kk][q], minus_m1))));
            reinterpret_cast<uint4 *>(p.dx)[t * p.n8 + i] = make_uint4(o[0], o[1], o[2], o[3]);
        }
        stage = stage == LN_STAGES - 1 ? 0 : stage + 1;
    }
    const size_t D = (size_t)p.n8 * 8;
    float *mine = p.partial + (size_t)blockIdx.x * 2 * D;
    if (!WARP) {
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const unsigned i = k * span + lane;
            if (i >= p.n8) continue;
            float4 *a = reinterpret_cast<float4 *>(mine + 8 * i), *b = reinterpret_cast<float4 *>(mine + D + 8 * i);
            a[0] = quad(dg[k][0], dg[k][1]);
            a[1] = quad(dg[k][2], dg[k][3]);
            b[0] = quad(db[k][0], db[k][1]);
            b[1] = quad(db[k][2], db[k][3]);
        }
    } else {                 // the warps hold the same columns: add them in shared memory (the ring is free), warp by warp
        float4 *sum = reinterpret_cast<float4 *>(ring_mem);                               // [2][KG * 32][2]
        cp_async_wait<0>();
        __syncthreads();
        for (unsigned w = 0; w < groups; ++w) {
            if (group == w) {
#pragma unroll
                for (int k = 0; k < KG; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int at = (k * 32 + lane) * 2 + h;
                        float4 a = quad(dg[k][2 * h], dg[k][2 * h + 1]), b = quad(db[k][2 * h], db[k][2 * h + 1]);
                        if (w) {
                            const float4 u = sum[at], v = sum[KG * 64 + at];
                            a = make_float4(u.x + a.x, u.y + a.y, u.z + a.z, u.w + a.w);
                            b = make_float4(v.x + b.x, v.y + b.y, v.z + b.z, v.w + b.w);
                        }
                        sum[at] = a;
                        sum[KG * 64 + at] = b;
                    }
            }
            __syncthreads();
        }
        const float *sums = reinterpret_cast<const float *>(ring_mem);
        for (unsigned j = threadIdx.x; j < p.n8 * 8; j += blockDim.x) {
            mine[j] = sums[j];
            mine[D + j] = sums[KG * 256 + j];
        }
    }
}

// dgamma and dbeta from the CTAs' sums: 32 columns per CTA, a warp takes every 32nd of the sums, then the warps in order.
__global__ void __launch_bounds__(1024) layernorm_bwd_sum_kernel(const float *__restrict__ partial, int parts, unsigned D,
                                                                 float *__restrict__ dgamma, float *__restrict__ dbeta,
                                                                 int accumulate)
{
    cudaGridDependencySynchronize();
    __shared__ float red[32][33];
    const unsigned j = blockIdx.x * 32 + (threadIdx.x & 31);      // over [2][D]
    const int r = threadIdx.x >> 5;
    float s = 0.0f;
    if (j < 2 * D) {
#pragma unroll 8
        for (int c = r; c < parts; c += 32) s += __ldcg(partial + (size_t)c * 2 * D + j);
    }
    red[r][threadIdx.x & 31] = s;
    __syncthreads();
    s = red[threadIdx.x & 31][r];                                 // transposed: warp r adds the 32 sums of column r
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    const unsigned col = blockIdx.x * 32 + r;
    if ((threadIdx.x & 31) == 0 && col < 2 * D) {
        float *o = col < D ? dgamma + col : dbeta + (col - D);
        *o = accumulate ? *o + s : s;
    }
}

// Threads of a CTA and CTAs per SM.  Up to 1024 columns (512 in the backward pass, whose registers hold more) a warp takes a
// row; beyond, the CTA does, with two groups of columns per thread up to 4096 and four above.
struct LnShape {
    int kg;
    bool warp;
    unsigned threads, per_sm, min_rows;      // min_rows: rows that a CTA has at least, where there are more than 148 of them
};
static LnShape ln_shape(size_t D, bool backward)
{
    const unsigned n8 = (unsigned)(D / 8);
    LnShape s;
    s.warp = D <= (backward ? 512u : 1024u);
    if (s.warp) {
        s.kg = D <= 256 ? 1 : D <= 512 ? 2 : 4;
        s.threads = 256;
        s.min_rows = 1;
        s.per_sm = backward ? 2 : 3;
    } else {
        s.kg = D <= 4096 ? 2 : 4;
        s.threads = ((n8 + s.kg - 1) / s.kg + 31) & ~31u;
        s.per_sm = (backward || s.kg == 4 ? 512 : 768) / s.threads;
        if (s.per_sm < 1) s.per_sm = 1;
        s.min_rows = backward ? 8 : 1;          // fewer sums to add up behind the pass
    }
    return s;
}
static unsigned ln_grid(const LnShape &s, size_t T)
{
    const size_t rows = s.warp ? s.threads / 32 : s.min_rows;
    const size_t most = (size_t)148 * s.per_sm;
    size_t want = (T + rows - 1) / rows;
    if (!s.warp && want < 148) want = T < 148 ? T : 148;
    return (unsigned)(want < most ? want : most);
}

template <auto Kernel, int KG, int MAXT, typename P>
static int ln_launch(const P &p, const LnShape &s, unsigned int *amax, cudaStream_t st)
{
    if (ring_bytes<KG>(MAXT) > 40 * 1024) {
        const int rc = allow_shared<Kernel>((int)ring_bytes<KG>(MAXT));
        if (rc != FP8_OK) return rc;
    }
    return launch_behind_amax(Kernel, p.T * p.n8 * 8, amax, ln_grid(s, p.T), s.threads, ring_bytes<KG>(s.threads), st, p);
}

}  // namespace fp8dpa

using namespace fp8dpa;

static bool layernorm_shape_ok(size_t T, size_t D)
{
    return T > 0 && D > 0 && D % 8 == 0 && D <= 16384 && T <= 0x7FFFFFFFull;
}

static int layernorm_fwd(const char *who, const void *x, const float *gamma, const float *beta, const void *residual,
                         size_t T, size_t D, float eps, const float *q_scale, int fmt, void *out, uint8_t *out8,
                         float *mean, float *rstd, float *amax_out, void *stream)
{
    if (!x || !gamma || !beta || !out) {
        set_error("%s: NULL pointer", who);
        return FP8_ERR_NULL;
    }
    if (out8 && fmt != FP8_E4M3 && fmt != FP8_E5M2) {
        set_error("%s: fmt %d is not FP8_E4M3 / FP8_E5M2", who, fmt);
        return FP8_ERR_ENUM;
    }
    if (!layernorm_shape_ok(T, D) || !(eps >= 0.0f)) {
        set_error("%s: unsupported shape T=%zu D=%zu (D %% 8 == 0, D <= 16384) or eps < 0", who, T, D);
        return FP8_ERR_SHAPE;
    }
    if (!aligned16(x) || !aligned16(gamma) || !aligned16(beta) || !aligned16(residual) || !aligned16(out) || !aligned16(out8)) {
        set_error("%s: pointers must be 16-byte aligned", who);
        return FP8_ERR_ALIGN;
    }
    int rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    LnFwd p = {static_cast<const uint16_t *>(x), gamma, beta, static_cast<const uint16_t *>(residual), T, (unsigned)(D / 8), eps,
               static_cast<uint16_t *>(out), mean, rstd, reinterpret_cast<unsigned int *>(amax_out), q_scale, out8, fmt};
    const LnShape s = ln_shape(D, false);
    if (s.warp && s.kg == 1) return ln_launch<layernorm_fwd_kernel<1, true, 256, 3>, 1, 256>(p, s, p.amax_bits, st);
    if (s.warp && s.kg == 2) return ln_launch<layernorm_fwd_kernel<2, true, 256, 3>, 2, 256>(p, s, p.amax_bits, st);
    if (s.warp) return ln_launch<layernorm_fwd_kernel<4, true, 256, 2>, 4, 256>(p, s, p.amax_bits, st);
    if (s.kg == 2) return ln_launch<layernorm_fwd_kernel<2, false, 256, 3>, 2, 256>(p, s, p.amax_bits, st);
    return ln_launch<layernorm_fwd_kernel<4, false, 512, 1>, 4, 512>(p, s, p.amax_bits, st);
}

extern "C" int fp8_layernorm_fwd(const void *x_bf16, const float *gamma, const float *beta, const void *residual_bf16,
                                 size_t T, size_t D, float eps, void *out_bf16, float *mean, float *rstd, float *amax_out,
                                 void *stream)
{
    return layernorm_fwd("fp8_layernorm_fwd", x_bf16, gamma, beta, residual_bf16, T, D, eps, nullptr, 0, out_bf16, nullptr,
                         mean, rstd, amax_out, stream);
}

extern "C" int fp8_layernorm_fwd_q(const void *x_bf16, const float *gamma, const float *beta, const void *residual_bf16,
                                   size_t T, size_t D, float eps, const float *q_scale, int fmt, void *out_bf16,
                                   uint8_t *out8, float *mean, float *rstd, float *amax_out, void *stream)
{
    if (!out8 || !q_scale) {
        set_error("fp8_layernorm_fwd_q: NULL q_scale / out8");
        return FP8_ERR_NULL;
    }
    return layernorm_fwd("fp8_layernorm_fwd_q", x_bf16, gamma, beta, residual_bf16, T, D, eps, q_scale, fmt, out_bf16, out8,
                         mean, rstd, amax_out, stream);
}

extern "C" size_t fp8_layernorm_bwd_workspace_bytes(size_t T, size_t D)
{
    return layernorm_shape_ok(T, D) ? ((size_t)ln_grid(ln_shape(D, true), T) * 2 * D * sizeof(float) + 255) & ~(size_t)255 : 0;
}

extern "C" int fp8_layernorm_bwd(const void *dout_bf16, const void *x_bf16, const float *gamma, const float *mean,
                                 const float *rstd, size_t T, size_t D, void *dx_bf16, float *dgamma, float *dbeta,
                                 int accumulate, void *ws, size_t ws_bytes, void *stream)
{
    if (!dout_bf16 || !x_bf16 || !gamma || !mean || !rstd || !dx_bf16 || !dgamma || !dbeta) {
        set_error("fp8_layernorm_bwd: NULL pointer");
        return FP8_ERR_NULL;
    }
    if (!layernorm_shape_ok(T, D)) {
        set_error("fp8_layernorm_bwd: unsupported shape T=%zu D=%zu (D %% 8 == 0, D <= 16384)", T, D);
        return FP8_ERR_SHAPE;
    }
    if (!aligned16(dout_bf16) || !aligned16(x_bf16) || !aligned16(gamma) || !aligned16(dx_bf16)) {
        set_error("fp8_layernorm_bwd: pointers must be 16-byte aligned");
        return FP8_ERR_ALIGN;
    }
    const size_t need = fp8_layernorm_bwd_workspace_bytes(T, D);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("fp8_layernorm_bwd: workspace of %zu bytes, 256-byte aligned, needed (got %zu)", need, ws_bytes);
        return FP8_ERR_WORKSPACE;
    }
    int rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const LnShape s = ln_shape(D, true);
    float *partial = static_cast<float *>(ws);
    LnBwd p = {static_cast<const uint16_t *>(dout_bf16), static_cast<const uint16_t *>(x_bf16), gamma, mean, rstd, T,
               (unsigned)(D / 8), static_cast<uint16_t *>(dx_bf16), partial};
    if (s.warp && s.kg == 1) rc = ln_launch<layernorm_bwd_kernel<1, true, true, 256, 2>, 1, 256>(p, s, nullptr, st);
    else if (s.warp) rc = ln_launch<layernorm_bwd_kernel<2, true, true, 256, 2>, 2, 256>(p, s, nullptr, st);
    else if (s.kg == 2) rc = ln_launch<layernorm_bwd_kernel<2, false, true, 256, 2>, 2, 256>(p, s, nullptr, st);
    else rc = ln_launch<layernorm_bwd_kernel<4, false, false, 512, 1>, 4, 512>(p, s, nullptr, st);
    if (rc != FP8_OK) return rc;
    return launch_early(layernorm_bwd_sum_kernel, (unsigned)((2 * D + 31) / 32), 1024, 0, st, partial, (int)ln_grid(s, T),
                        (unsigned)D, dgamma, dbeta, accumulate ? 1 : 0);
}
