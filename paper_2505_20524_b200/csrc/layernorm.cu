// Layer norm: out = residual + gamma (x - mean) / sqrt(var + eps) + beta per token row, with the amax and the FP8 codes of
// the result for the next product, and its backward pass with the reduction of dgamma and dbeta.
#include <math.h>

#include "common.cuh"
#include "elementwise.cuh"

namespace fp8dpa {

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

// Who takes a row: 2^lanes_log2 lanes of a warp, a warp, or the CTA.
enum LnUnit { LN_LANES, LN_WARP, LN_CTA };

// A thread holds KG groups of eight columns of its unit's row, gamma and beta of them in registers for all the rows that the unit
// comes by (every n-th of n units': neighbours read neighbouring rows, 38.5 us against 41.8 with a contiguous share each at
// 8192 x 4096 with residual and codes), and the row itself between the two sums (the mean, then the squared distances from it:
// no cancellation however far the mean lies from zero) and the result: one read of x.  Persistent; the next rows travel while
// one is worked on.  Without a residual the instructions per row bind: addresses that only count on, columns behind the row as
// zeros instead of branches, and a kernel without the residual's code took 33.5M elements from 27 to 34 us to 24 to 26.
// With 50 to 64 KB per SM on their way memory does best, two rows ahead or, with a residual, one (8192 x 4096 with residual
// and codes: 38.5 us; 42 with two).  rstd by rsqrtf, off by 2 ulp of FP32 at most.
template <int KG, LnUnit UNIT, bool RES, int STAGES, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) layernorm_fwd_kernel(const LnFwd p, int lanes_log2)
{
    constexpr bool CTA = UNIT == LN_CTA;
    if (UNIT == LN_WARP) lanes_log2 = 5;
    extern __shared__ __align__(16) uint4 ring_mem[];
    __shared__ __align__(16) float red[2][MAXT / 32];
    const bool alone = amax_begin(p.amax_bits);
    const unsigned span = CTA ? blockDim.x : 1u << lanes_log2, lane = CTA ? threadIdx.x : threadIdx.x & (span - 1);
    const unsigned rows = CTA ? 1 : 32u >> lanes_log2, sub = CTA ? 0 : (threadIdx.x & 31) >> lanes_log2;    // rows at a time
    const size_t units = CTA ? gridDim.x : (size_t)gridDim.x * (blockDim.x >> 5);
    const size_t unit = CTA ? blockIdx.x : (size_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const size_t step = units * rows, pitch = step * p.n8;
    if (CTA) {
        if (threadIdx.x < MAXT / 32) red[0][threadIdx.x] = red[1][threadIdx.x] = 0.0f;
        __syncthreads();
    }
    const float qs = p.out8 ? __ldg(p.q_scale) : 1.0f;
    const float inv_d = 1.0f / (float)(p.n8 * 8);
    // places in shared memory of this thread's groups: [stage][tensor][k][thread]
    const uint32_t ring = smem_u32(ring_mem + threadIdx.x), per_k = blockDim.x * 16u, per_tensor = per_k * KG;
    const uint32_t per_stage = per_tensor * (RES ? 2u : 1u), ring_end = ring + STAGES * per_stage;
    bool in[KG];
    uint64_t g[KG][4], b[KG][4];
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        in[k] = k * span + lane < p.n8;
#pragma unroll
        for (int e = 0; e < 4; ++e) g[k][e] = b[k][e] = 0ull;
        if (in[k]) {
            load4x2(p.gamma + 8 * (k * span + lane), g[k]);
            load4x2(p.beta + 8 * (k * span + lane), b[k]);
        } else {                     // columns behind the row's: zeros that the loop below reads without asking
            for (uint32_t at = ring; at != ring_end; at += per_tensor) ring_put_zero(at + k * per_k);
        }
    }
    size_t t = unit * rows + sub;                             // this thread's row; the unit's first row decides for all
    size_t ahead = t, at = t * p.n8 + lane;
    const uint4 *next_x = reinterpret_cast<const uint4 *>(p.x) + at, *next_r = reinterpret_cast<const uint4 *>(p.residual) + at;
    const auto fetch = [&](uint32_t to) {
        if (ahead < p.T) {
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                if (!in[k]) continue;
                cp_async16(to + k * per_k, next_x + k * span);
                if (RES) cp_async16(to + per_tensor + k * per_k, next_r + k * span);
            }
        }
        cp_async_commit();
        ahead += step;
        next_x += pitch;
        if (RES) next_r += pitch;
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(ring + s * per_stage);
    uint32_t m = 0, now = ring, fill = ring + (STAGES - 1) * per_stage;
    for (size_t base = unit * rows; base < p.T; base += step, t += step, at += pitch) {
        cp_async_wait<STAGES - 2>();
        fetch(fill);                                          // the stage of the row before this one
        fill = now;
        uint64_t f[KG][4], s = 0ull;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            unpack4x2(ring_get(now + k * per_k), f[k]);
            s = add_f32x2(s, add_f32x2(add_f32x2(f[k][0], f[k][1]), add_f32x2(f[k][2], f[k][3])));
        }
        const float mean = row_sum<CTA, MAXT / 32>(add_halves(s), lanes_log2, red[0]) * inv_d;
        uint64_t ss = 0ull;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const uint64_t minus_mean = both(in[k] ? -mean : 0.0f);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f[k][e] = add_f32x2(f[k][e], minus_mean);
                ss = fma_f32x2(f[k][e], f[k][e], ss);
            }
        }
        const float rstd = rsqrtf(fmaf(row_sum<CTA, MAXT / 32>(add_halves(ss), lanes_log2, red[1]), inv_d, p.eps));
        const uint64_t rstd2 = both(rstd);
        const bool live = UNIT != LN_LANES || t < p.T;
        if (live && lane == 0) {
            if (p.mean) p.mean[t] = mean;
            if (p.rstd) p.rstd[t] = rstd;
        }
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            if (!live || !in[k]) continue;
            uint64_t r[4];
            if (RES) unpack4x2(ring_get(now + per_tensor + k * per_k), r);
            uint32_t o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint64_t y = fma_f32x2(mul_f32x2(f[k][q], rstd2), g[k][q], b[k][q]);
                if (RES) y = add_f32x2(y, r[q]);
                o[q] = round2(y);
                m = absmax2e(m, o[q]);
            }
            reinterpret_cast<uint4 *>(p.out)[at + k * span] = make_uint4(o[0], o[1], o[2], o[3]);
            if (p.out8) reinterpret_cast<uint2 *>(p.out8)[at + k * span] = bf16x8_to_fp8x8(o, qs, p.fmt);
        }
        now += per_stage;
        if (now == ring_end) now = ring;
    }
    amax_end(m, p.amax_bits, alone);
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
// layernorm_bwd_sum_kernel.  x and dout are read once, dx is written once.  A warp loads mean and rstd of 32 of its rows at a
// time: when all CTAs read those of neighbouring rows one by one, the few lines that hold them were what bound the kernel
// (8192 x 4096: 52.7 us).  Up to KG = 2 (8192 columns) xh, g and gamma stay in registers between the sums and dx (4000 x 8192:
// 37 us, memory's 30); with KG = 4 xh and g are formed again from the ring and gamma lies behind it, with one CTA per SM
// (2048 x 16384: 46 us, memory's 31; clusters of two and four CTAs per row with two groups per thread: 57 to 59, their
// barriers cost more than the second look at the row).
__host__ __device__ constexpr int ln_bwd_stages(int kg) { return kg > 2 ? 2 : 3; }
constexpr size_t ln_bwd_shared(int kg, unsigned threads) { return (size_t)(ln_bwd_stages(kg) + (kg > 2)) * 2 * kg * 16 * threads; }
template <int KG, LnUnit UNIT, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) layernorm_bwd_kernel(const LnBwd p, int lanes_log2)
{
    cudaTriggerProgrammaticLaunchCompletion();
    constexpr bool CTA = UNIT == LN_CTA, KEEP = KG <= 2;
    constexpr int STAGES = ln_bwd_stages(KG);
    if (UNIT == LN_WARP) lanes_log2 = 5;
    extern __shared__ __align__(16) uint4 ring_mem[];
    __shared__ __align__(16) float2 red[2][MAXT / 32];
    const unsigned span = CTA ? blockDim.x : 1u << lanes_log2, lane = CTA ? threadIdx.x : threadIdx.x & (span - 1);
    const unsigned groups = CTA ? 1 : blockDim.x >> 5, group = CTA ? 0 : threadIdx.x >> 5;
    const unsigned at_once = CTA ? 1 : 32u >> lanes_log2, sub = CTA ? 0 : (threadIdx.x & 31) >> lanes_log2;   // rows of a warp
    const Rows rows = rows_of((size_t)blockIdx.x * groups + group, (size_t)gridDim.x * groups, p.T);
    const float inv_d = 1.0f / (float)(p.n8 * 8);
    if (CTA) {
        if (threadIdx.x < MAXT / 32) red[0][threadIdx.x] = red[1][threadIdx.x] = make_float2(0.0f, 0.0f);
        __syncthreads();
    }
    // places in shared memory of this thread's groups: [stage][tensor][k][thread], then gamma [k][half][thread]
    const uint32_t ring = smem_u32(ring_mem + threadIdx.x), per_k = blockDim.x * 16u, per_tensor = per_k * KG;
    const uint32_t per_stage = 2 * per_tensor, ring_end = ring + STAGES * per_stage;
    constexpr int KK = KEEP ? KG : 1;
    bool in[KG];
    uint64_t dg[KG][4], db[KG][4], gm[KK][4];
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        in[k] = k * span + lane < p.n8;
#pragma unroll
        for (int e = 0; e < 4; ++e) dg[k][e] = db[k][e] = gm[KEEP ? k : 0][e] = 0ull;
        if (in[k]) load4x2(p.gamma + 8 * (k * span + lane), gm[KEEP ? k : 0]);
        else                         // columns behind the row's: zeros that the loop below reads without asking
            for (uint32_t at = ring; at != ring_end; at += per_tensor) ring_put_zero(at + k * per_k);
        if (!KEEP) {
            ring_put(ring_end + (2 * k) * per_k, gm[0][0], gm[0][1]);
            ring_put(ring_end + (2 * k + 1) * per_k, gm[0][2], gm[0][3]);
        }
    }
    const size_t pitch = (size_t)at_once * p.n8;
    size_t ahead = rows.begin + sub, at = ahead * p.n8 + lane;
    const uint4 *next_x = reinterpret_cast<const uint4 *>(p.x) + at, *next_d = reinterpret_cast<const uint4 *>(p.dout) + at;
    const auto fetch = [&](uint32_t to) {
        if (ahead < rows.end) {
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                if (!in[k]) continue;
                cp_async16(to + k * per_k, next_x + k * span);
                cp_async16(to + per_tensor + k * per_k, next_d + k * span);
            }
        }
        cp_async_commit();
        ahead += at_once;
        next_x += pitch;
        next_d += pitch;
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(ring + s * per_stage);
    uint32_t now = ring, fill = ring + (STAGES - 1) * per_stage;
    int flip = 0;
    float mu32 = 0.0f, rs32 = 0.0f, mu_ahead = 0.0f, rs_ahead = 0.0f;      // lane l: the statistics of row l of a batch of 32
    if (rows.begin + (threadIdx.x & 31) < rows.end) {
        mu_ahead = __ldg(p.mean + rows.begin + (threadIdx.x & 31));
        rs_ahead = __ldg(p.rstd + rows.begin + (threadIdx.x & 31));
    }
    for (size_t first = rows.begin; first < rows.end; first += at_once, at += pitch, flip ^= 1) {
        const bool live = UNIT != LN_LANES || first + sub < rows.end;
        cp_async_wait<STAGES - 2>();
        fetch(fill);                             // the stage of the row before this one
        fill = now;
        const unsigned in_batch = (unsigned)(first - rows.begin) & 31u;
        if (in_batch == 0) {                     // the next 32 rows' statistics; the batch behind them is on its way
            mu32 = mu_ahead;
            rs32 = rs_ahead;
            const size_t from = first + 32 + (threadIdx.x & 31);
            if (from < rows.end) {
                mu_ahead = __ldg(p.mean + from);
                rs_ahead = __ldg(p.rstd + from);
            }
        }
        const float mu = __shfl_sync(0xffffffffu, mu32, in_batch + sub), rs = __shfl_sync(0xffffffffu, rs32, in_batch + sub);
        const uint64_t minus_mu = both(-mu), rs2 = both(rs);
        uint64_t xh[KK][4], ge[KK][4], a1 = 0ull, a2 = 0ull;
        const auto load = [&](int k, int kk, uint64_t (&d)[4]) {
            unpack4x2(ring_get(now + k * per_k), xh[kk]);
            unpack4x2(ring_get(now + per_tensor + k * per_k), d);
            if (!KEEP) {
                ring_get(ring_end + (2 * k) * per_k, gm[0][0], gm[0][1]);
                ring_get(ring_end + (2 * k + 1) * per_k, gm[0][2], gm[0][3]);
            }
            const uint64_t shift = in[k] ? minus_mu : 0ull;      // columns behind the row's: 0, whatever mean * rstd is
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                xh[kk][e] = mul_f32x2(add_f32x2(xh[kk][e], shift), rs2);
                ge[kk][e] = mul_f32x2(d[e], gm[kk][e]);
            }
        };
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const int kk = KEEP ? k : 0;
            if (!live) continue;
            uint64_t d[4];
            load(k, kk, d);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                dg[k][e] = fma_f32x2(d[e], xh[kk][e], dg[k][e]);
                db[k][e] = add_f32x2(db[k][e], d[e]);
                a1 = add_f32x2(a1, ge[kk][e]);
                a2 = fma_f32x2(ge[kk][e], xh[kk][e], a2);
            }
        }
        float s1 = add_halves(a1), s2 = add_halves(a2);
        for (int off = UNIT != LN_LANES ? 16 : (1 << lanes_log2) >> 1; off > 0; off >>= 1) {
            s1 += __shfl_xor_sync(0xffffffffu, s1, off);
            s2 += __shfl_xor_sync(0xffffffffu, s2, off);
        }
        if (CTA) {           // two buffers in turn: the next row's writes do not meet this row's reads
            if ((threadIdx.x & 31) == 0) red[flip][threadIdx.x >> 5] = make_float2(s1, s2);
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int w = 0; w < MAXT / 32; w += 2) {
                const float4 v = *reinterpret_cast<const float4 *>(&red[flip][w]);
                s1 += v.x + v.z;
                s2 += v.y + v.w;
            }
        }
        const uint64_t minus_m1 = both(-s1 * inv_d), minus_m2 = both(-s2 * inv_d);
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const int kk = KEEP ? k : 0;
            if (!live || !in[k]) continue;
            uint64_t d[4];
            if (!KEEP) load(k, 0, d);
            uint32_t o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                o[q] = round2(mul_f32x2(rs2, fma_f32x2(xh[kk][q], minus_m2, add_f32x2(ge[kk][q], minus_m1))));
            reinterpret_cast<uint4 *>(p.dx)[at + k * span] = make_uint4(o[0], o[1], o[2], o[3]);
        }
        now += per_stage;
        if (now == ring_end) now = ring;
    }
    const size_t D = (size_t)p.n8 * 8;
    float *mine = p.partial + (size_t)blockIdx.x * 2 * D;
    if (CTA) {
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
    } else {                 // rows of a warp, then warps, hold the same columns: add them up in a fixed order
        for (unsigned off = 16; off >= span; off >>= 1) {
#pragma unroll
            for (int k = 0; k < KG; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    dg[k][e] = add_f32x2(dg[k][e], __shfl_xor_sync(0xffffffffu, dg[k][e], off));
                    db[k][e] = add_f32x2(db[k][e], __shfl_xor_sync(0xffffffffu, db[k][e], off));
                }
        }
        float4 *sum = reinterpret_cast<float4 *>(ring_mem);      // the ring is free: [2][KG * span][2]
        cp_async_wait<0>();
        __syncthreads();
        for (unsigned w = 0; w < groups; ++w) {
            if (group == w && sub == 0) {
#pragma unroll
                for (int k = 0; k < KG; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const unsigned at = (k * span + lane) * 2 + h, at2 = KG * span * 2 + at;
                        float4 a = quad(dg[k][2 * h], dg[k][2 * h + 1]), b = quad(db[k][2 * h], db[k][2 * h + 1]);
                        if (w) {
                            const float4 u = sum[at], v = sum[at2];
                            a = make_float4(u.x + a.x, u.y + a.y, u.z + a.z, u.w + a.w);
                            b = make_float4(v.x + b.x, v.y + b.y, v.z + b.z, v.w + b.w);
                        }
                        sum[at] = a;
                        sum[at2] = b;
                    }
            }
            __syncthreads();
        }
        const float *sums = reinterpret_cast<const float *>(ring_mem);
        for (unsigned j = threadIdx.x; j < p.n8 * 8; j += blockDim.x) {
            mine[j] = sums[j];
            mine[D + j] = sums[KG * span * 8 + j];
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

struct LnShape {
    bool cta;
    int lanes_log2;
    unsigned threads, grid;
};
static int log2_at_least(unsigned n)
{
    int l = 0;
    while ((1u << l) < n) ++l;
    return l;
}
// Forward: two groups of columns per thread on lanes of a warp up to 256 columns (65536 x 64: 5.0 us where a warp per row took
// 16.5, x 256: 14.1 where it took 17.2), on a warp up to 512, on the CTA between 1032 and 4096; four on a warp up to 1024
// and on the CTA above 4096.
static LnShape ln_fwd_shape(size_t T, size_t D)
{
    const unsigned kg = D <= 512 || (D > 1024 && D <= 4096) ? 2 : 4, lanes = ((unsigned)(D / 8) + kg - 1) / kg;
    LnShape s;
    s.cta = lanes > 32;
    s.lanes_log2 = s.cta ? 0 : D > 256 ? 5 : log2_at_least(lanes);
    s.threads = s.cta ? (lanes + 31) & ~31u : 256;
    const size_t at_once = s.cta ? 1 : s.threads >> s.lanes_log2, want = (T + at_once - 1) / at_once;
    const size_t most = 148 * (size_t)((kg == 2 ? 768 : 512) / s.threads);
    s.grid = (unsigned)(want < most ? want : most);
    return s;
}
// Backward: lanes of a warp with one group of columns each up to 128 columns, a warp with one up to 256 and two up to 512, then
// the CTA with two, above 8192 with four.  As many CTAs as registers allow; a CTA has eight rows at least where there are more
// than 148 of them (fewer sums to add up behind the pass).
static LnShape ln_bwd_shape(size_t T, size_t D)
{
    const unsigned n8 = (unsigned)(D / 8);
    LnShape s;
    s.cta = D > 512;
    s.lanes_log2 = s.cta || D > 128 ? 5 : log2_at_least(n8);
    const unsigned kg = D <= 8192 ? 2 : 4;
    s.threads = s.cta ? ((n8 + kg - 1) / kg + 31) & ~31u : 256;
    const size_t at_once = s.cta ? 8 : (size_t)8 << (5 - s.lanes_log2);
    const size_t most = 148 * (size_t)(s.cta ? 512 / s.threads : D <= 256 ? 3 : 2);
    size_t want = (T + at_once - 1) / at_once;
    if (s.cta && want < 148) want = T < 148 ? T : 148;
    s.grid = (unsigned)(want < most ? want : most);
    return s;
}

// `most`: the shared memory that the kernel's largest launch takes
template <auto Kernel, typename P>
static int ln_launch(const P &p, const LnShape &s, size_t smem, size_t most, unsigned int *amax, cudaStream_t st)
{
    if (most > 40 * 1024) {
        const int rc = allow_shared<Kernel>((int)most);
        if (rc != FP8_OK) return rc;
    }
    return launch_behind_amax<Kernel>(p.T * p.n8 * 8, amax, s.grid, s.threads, smem, st, p, s.lanes_log2);
}

template <int KG, LnUnit UNIT, bool RES, int STAGES, int MAXT, int MINB>
static int ln_fwd_launch(const LnFwd &p, const LnShape &s, cudaStream_t st)
{
    constexpr size_t per_thread = STAGES * (RES ? 2 : 1) * KG * 16;
    return ln_launch<layernorm_fwd_kernel<KG, UNIT, RES, STAGES, MAXT, MINB>>(p, s, per_thread * s.threads, per_thread * MAXT,
                                                                              p.amax_bits, st);
}
template <bool RES>
static int ln_fwd_run(const LnFwd &p, size_t D, cudaStream_t st)
{
    constexpr int STAGES = RES ? 2 : 3;
    const LnShape s = ln_fwd_shape(p.T, D);
    if (D <= 256) return ln_fwd_launch<2, LN_LANES, RES, STAGES, 256, 3>(p, s, st);
    if (D <= 512) return ln_fwd_launch<2, LN_WARP, RES, STAGES, 256, 3>(p, s, st);
    if (D <= 1024) return ln_fwd_launch<4, LN_WARP, RES, STAGES, 256, 2>(p, s, st);
    if (D <= 4096) return ln_fwd_launch<2, LN_CTA, RES, STAGES, 256, 3>(p, s, st);
    if (D <= 8192) return ln_fwd_launch<4, LN_CTA, RES, STAGES, 256, 2>(p, s, st);
    // one CTA of up to 384 threads per SM: with two stages too little travels (3000 x 10000 with codes: 42.0 us, 38.4 with three)
    if constexpr (RES)
        if (D <= 12288) return ln_fwd_launch<4, LN_CTA, true, 3, 384, 1>(p, s, st);
    return ln_fwd_launch<4, LN_CTA, RES, STAGES, 512, 1>(p, s, st);
}

template <int KG, LnUnit UNIT, int MAXT, int MINB>
static int ln_bwd_launch(const LnBwd &p, const LnShape &s, cudaStream_t st)
{
    return ln_launch<layernorm_bwd_kernel<KG, UNIT, MAXT, MINB>>(p, s, ln_bwd_shared(KG, s.threads), ln_bwd_shared(KG, MAXT),
                                                                 nullptr, st);
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
    return residual ? ln_fwd_run<true>(p, D, st) : ln_fwd_run<false>(p, D, st);
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
    return layernorm_shape_ok(T, D) ? ((size_t)ln_bwd_shape(T, D).grid * 2 * D * sizeof(float) + 255) & ~(size_t)255 : 0;
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
    const LnShape s = ln_bwd_shape(T, D);
    float *partial = static_cast<float *>(ws);
    LnBwd p = {static_cast<const uint16_t *>(dout_bf16), static_cast<const uint16_t *>(x_bf16), gamma, mean, rstd, T,
               (unsigned)(D / 8), static_cast<uint16_t *>(dx_bf16), partial};
    if (D <= 128) rc = ln_bwd_launch<1, LN_LANES, 256, 3>(p, s, st);
    else if (D <= 256) rc = ln_bwd_launch<1, LN_WARP, 256, 3>(p, s, st);
    else if (D <= 512) rc = ln_bwd_launch<2, LN_WARP, 256, 2>(p, s, st);
    else if (D <= 4096) rc = ln_bwd_launch<2, LN_CTA, 256, 2>(p, s, st);
    else if (D <= 8192) rc = ln_bwd_launch<2, LN_CTA, 512, 1>(p, s, st);
    else rc = ln_bwd_launch<4, LN_CTA, 512, 1>(p, s, st);
    if (rc != FP8_OK) return rc;
    return launch_early(layernorm_bwd_sum_kernel, (unsigned)((2 * D + 31) / 32), 1024, 0, st, partial, (int)s.grid,
                        (unsigned)D, dgamma, dbeta, accumulate ? 1 : 0);
}
