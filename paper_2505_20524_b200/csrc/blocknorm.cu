// The joint of two blocks: norm (or scale) behind a block, gate, residual scale and sum, norm in front of the next block with the
// amax and FP8 codes of its operand; and the gradient of all that.
#include <math.h>

#include "common.cuh"
#include "elementwise.cuh"
#include "rows.cuh"

namespace fp8dpa {

constexpr uint64_t TWO_ONES = 0x3F8000003F800000ull;

// sigmoid(v) of two values, s = 1 / (1 + e) with e = exp(-v), and 1 - s = e s (no cancellation where s is near 1).  A sigmoid below
// 2^-126 is 0, and the infinity that e may be there is kept out of e s; NaN stays NaN in both.
__device__ __forceinline__ uint64_t sigmoid2(uint64_t v, uint64_t &rest)
{
    float a, b;
    unpack_f32x2(mul_f32x2(v, both(-1.4426950408889634f)), a, b);
    a = ex2_approx(a);
    b = ex2_approx(b);
    const uint64_t e = pack_f32x2(fminf(a, 8.507059e37f), fminf(b, 8.507059e37f));      // 2^126
    unpack_f32x2(add_f32x2(pack_f32x2(a, b), both(1.0f)), a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    const uint64_t s = pack_f32x2(a, b);
    rest = mul_f32x2(e, s);
    return s;
}
// by the hardware's exp2 and reciprocal (good to 2^-22 of itself, then rounded to BF16 with the rest)
__device__ __forceinline__ uint64_t sigmoid2(uint64_t v)
{
    uint64_t unused;
    return sigmoid2(v, unused);
}

// A sum of products, each with its own rounding as written (the compiler joins packed sums with their products): without a norm
// or a sigmoid the joint is then what elementary operations give, bit for bit.
__device__ __forceinline__ uint64_t add_apart(uint64_t a, uint64_t b)
{
    float a0, a1, b0, b1;
    unpack_f32x2(a, a0, a1);
    unpack_f32x2(b, b0, b1);
    return pack_f32x2(__fadd_rn(a0, b0), __fadd_rn(a1, b1));
}

// ---------------------------------------------------------------- forward
struct BnFwd {
    const uint16_t *in[3];               // x, y, gate
    const float *gamma_post, *gamma_pre;
    size_t T;
    unsigned n8;
    float a, b, eps;
    int rms, sigmoid;
    uint16_t *h, *out;
    float *r_post, *r_pre;
    unsigned int *amax_bits;
    const float *q_scale;
    uint8_t *out8;
    int fmt;
};

// Rows and columns on threads as in the layer norm: a thread holds KG groups of eight columns of its unit's rows, both gammas of
// them in registers, and the next rows travel through its private ring.  NT tensors are read (x; y; gate); the sum of squares of
// y, the joint, its rounding to BF16, the sum of squares of that and the result follow in one pass: every tensor is read once and
// written once (8192 x 4096 with both norms and codes: 40.6 us in a graph, 235 MB at 5.8 TB/s; 43 with two CTAs per SM for three;
// with a gate 50.2 us, 6.0 TB/s).  The reciprocal roots by rsqrtf, off by 2 ulp of FP32 at most.
template <int KG, RowUnit UNIT, int NT, bool PRE, int STAGES, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) block_norm_fwd_kernel(const BnFwd p, int lanes_log2)
{
    constexpr bool CTA = UNIT == ROW_CTA;
    if (UNIT == ROW_WARP) lanes_log2 = 5;
    extern __shared__ __align__(16) uint4 ring_mem[];
    __shared__ __align__(16) float red[2][2][MAXT / 32];
    const bool alone = amax_begin(p.amax_bits);
    const unsigned span = CTA ? blockDim.x : 1u << lanes_log2, lane = CTA ? threadIdx.x : threadIdx.x & (span - 1);
    const unsigned rows = CTA ? 1 : 32u >> lanes_log2, sub = CTA ? 0 : (threadIdx.x & 31) >> lanes_log2;    // rows at a time
    const size_t units = CTA ? gridDim.x : (size_t)gridDim.x * (blockDim.x >> 5);
    const size_t unit = CTA ? blockIdx.x : (size_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const size_t step = units * rows, pitch = step * p.n8;
    if (CTA) {
        if (threadIdx.x < MAXT / 32)
            red[0][0][threadIdx.x] = red[0][1][threadIdx.x] = red[1][0][threadIdx.x] = red[1][1][threadIdx.x] = 0.0f;
        __syncthreads();
    }
    const uint64_t qs = both(p.out8 ? __ldg(p.q_scale) : 1.0f);
    const float inv_d = 1.0f / (float)(p.n8 * 8);
    const uint64_t a2 = both(p.a), b2 = both(p.b);
    // places in shared memory of this thread's groups: [stage][tensor][k][thread]
    const uint32_t ring = smem_u32(ring_mem + threadIdx.x), per_k = blockDim.x * 16u, per_tensor = per_k * KG;
    const uint32_t per_stage = per_tensor * NT, ring_end = ring + STAGES * per_stage;
    bool in[KG];
    uint64_t gq[KG][4], gp[KG][4];
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        in[k] = k * span + lane < p.n8;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            gq[k][e] = TWO_ONES;
            gp[k][e] = 0ull;
        }
        if (in[k]) {
            if (NT > 1 && p.gamma_post) load4x2(p.gamma_post + 8 * (k * span + lane), gq[k]);
            if (PRE) load4x2(p.gamma_pre + 8 * (k * span + lane), gp[k]);
        } else {                     // columns behind the row's: zeros that the loop below reads without asking
            for (uint32_t at = ring; at != ring_end; at += per_tensor) ring_put_zero(at + k * per_k);
        }
    }
    size_t t = unit * rows + sub;                             // this thread's row; the unit's first row decides for all
    size_t ahead = t, at = t * p.n8 + lane, at_ahead = at;
    const auto fetch = [&](uint32_t to) {
        if (ahead < p.T) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int k = 0; k < KG; ++k)
                    if (in[k]) cp_async16(to + i * per_tensor + k * per_k, reinterpret_cast<const uint4 *>(p.in[i]) + at_ahead + k * span);
        }
        cp_async_commit();
        ahead += step;
        at_ahead += pitch;
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(ring + s * per_stage);
    float m = 0.0f;
    uint32_t now = ring, fill = ring + (STAGES - 1) * per_stage;
    int flip = 0;
    for (size_t base = unit * rows; base < p.T; base += step, t += step, at += pitch, flip ^= 1) {
        cp_async_wait<STAGES - 2>();
        fetch(fill);                                          // the stage of the row before this one
        fill = now;
        const bool live = UNIT != ROW_LANES || t < p.T;
        uint64_t r2 = TWO_ONES;
        if (NT > 1 && p.rms) {
            uint64_t ss = 0ull;
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                uint64_t y[4];
                unpack4x2(ring_get(now + per_tensor + k * per_k), y);
#pragma unroll
                for (int e = 0; e < 4; ++e) ss = fma_f32x2(y[e], y[e], ss);
            }
            const float r = rsqrtf(fmaf(row_sum<CTA, MAXT / 32>(add_halves(ss), lanes_log2, red[flip][0]), inv_d, p.eps));
            if (live && lane == 0 && p.r_post) p.r_post[t] = r;
            r2 = both(r);
        }
        uint4 hw[KG];
        uint64_t ss = 0ull;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            uint64_t f[4];
            unpack4x2(ring_get(now + k * per_k), f);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = mul_f32x2(a2, f[e]);
            if (NT > 1) {
                uint64_t y[4];
                unpack4x2(ring_get(now + per_tensor + k * per_k), y);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = mul_f32x2(mul_f32x2(y[e], r2), gq[k][e]);
                if (NT > 2) {
                    uint64_t g[4];
                    unpack4x2(ring_get(now + 2 * per_tensor + k * per_k), g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = mul_f32x2(y[e], p.sigmoid ? sigmoid2(g[e]) : g[e]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = add_apart(f[e], mul_f32x2(b2, y[e]));
            }
            hw[k] = make_uint4(round2(f[0]), round2(f[1]), round2(f[2]), round2(f[3]));
            if (!in[k]) hw[k] = make_uint4(0u, 0u, 0u, 0u);   // 0 * inf where a row of zeros has no eps
            if (live && in[k] && p.h) reinterpret_cast<uint4 *>(p.h)[at + k * span] = hw[k];
            if (PRE) {
                unpack4x2(hw[k], f);
#pragma unroll
                for (int e = 0; e < 4; ++e) ss = fma_f32x2(f[e], f[e], ss);
            }
        }
        if (PRE) {
            const float r = rsqrtf(fmaf(row_sum<CTA, MAXT / 32>(add_halves(ss), lanes_log2, red[flip][1]), inv_d, p.eps));
            if (live && lane == 0 && p.r_pre) p.r_pre[t] = r;
            r2 = both(r);
        }
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            if (!live || !in[k]) continue;
            uint64_t f[4];
            uint4 o = hw[k];
            unpack4x2(o, f);
            if (PRE) {
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = mul_f32x2(mul_f32x2(f[e], r2), gp[k][e]);
                o = make_uint4(round2(f[0]), round2(f[1]), round2(f[2]), round2(f[3]));
                if (p.out) reinterpret_cast<uint4 *>(p.out)[at + k * span] = o;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) m = absmax3(m, f[e]);
            if (p.out8) reinterpret_cast<uint2 *>(p.out8)[at + k * span] = codes8(o, qs, p.fmt);
        }
        now += per_stage;
        if (now == ring_end) now = ring;
    }
    amax_end(pack_bf16x2(m, 0.0f), p.amax_bits, alone);
}

// ---------------------------------------------------------------- backward
struct BnBwd {
    const uint16_t *dout, *h, *dh, *y, *gate;
    const float *gamma_post, *gamma_pre, *r_post, *r_pre;
    size_t T;
    unsigned n8;
    float a, b;
    int rms, sigmoid, need_y;
    uint16_t *dx, *dy, *dgate;
    float *partial;
    unsigned int *maxima;                // behind them: the CTAs' largest dy, for the kernel that adds up the sums
    unsigned int *amax_bits;             // or, without sums, where it goes
    const float *q_scale;
    uint8_t *dy8;
    int fmt;
};

// With hh = h r_pre, e = gamma_pre dout:  D = dh + r_pre (e - hh mean(e hh)), dx = a D;  yh = y r_post, z = gamma_post yh,
// dgate = b D z s', dz = b D s, f = gamma_post dz:  dy = r_post (f - yh mean(f yh));  over rows dgamma_pre = sum dout hh and
// dgamma_post = sum dz yh, which a thread keeps in registers for its columns.  The two means are two sums over the row's
// threads, the second from what the first gives.  Every tensor is read once and written once.  The reciprocal roots go into
// scalars of the row: the loop forms e r_pre, dz r_post and f r_post and adds multiples of h and y to them, and the gammas lie in
// shared memory (8192 x 4096 with gate and codes: 106 -> 88 us in a graph, 503 MB at 5.7 TB/s; without a gate 67 us for 369 MB).
// Two barriers per row on 16 warps leave 0.55 instructions per cycle and scheduler; 512 threads with one group each, two CTAs
// per SM, have to do with 64 registers and spill (120 us).
// STAGES = 1: the ring holds one row, and a thread asks for the next row's piece as soon as it has read its own: above 8192
// columns, where two rows find no room (BF16 results without a gate, norm behind: 3000 x 10000 83 us, memory's 55; 2048 x 16384 114,
// memory's 62: 64 of 128 registers are the gammas' sums there, and one CTA fills an SM).
__host__ __device__ constexpr int bn_bwd_tensors(bool pre, bool gate) { return 2 + 2 * pre + gate; }
__host__ __device__ constexpr int bn_bwd_near(int kg, bool pre) { return kg <= 3 && pre ? 2 : 1; }
template <int KG, RowUnit UNIT, bool PRE, bool GATE, int STAGES, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) block_norm_bwd_kernel(const BnBwd p, int lanes_log2)
{
    cudaTriggerProgrammaticLaunchCompletion();
    constexpr bool CTA = UNIT == ROW_CTA;
    constexpr int PENDING = STAGES > 1 ? 2 * (STAGES - 2) : 0;       // copies that may be on their way when a row begins
    constexpr int NT = bn_bwd_tensors(PRE, GATE), DH = 0, Y = 1, DOUT = 2, H = 3, G = PRE ? 4 : 2;
    if (UNIT == ROW_WARP) lanes_log2 = 5;
    extern __shared__ __align__(16) uint4 ring_mem[];
    __shared__ __align__(16) float red[2][2][MAXT / 32];
    const bool alone = amax_begin(p.amax_bits);
    const unsigned span = CTA ? blockDim.x : 1u << lanes_log2, lane = CTA ? threadIdx.x : threadIdx.x & (span - 1);
    const unsigned groups = CTA ? 1 : blockDim.x >> 5, group = CTA ? 0 : threadIdx.x >> 5;
    const unsigned at_once = CTA ? 1 : 32u >> lanes_log2, sub = CTA ? 0 : (threadIdx.x & 31) >> lanes_log2;   // rows of a warp
    const Rows rows = rows_of((size_t)blockIdx.x * groups + group, (size_t)gridDim.x * groups, p.T);
    const float inv_d = 1.0f / (float)(p.n8 * 8);
    const uint64_t qs = both(p.dy8 ? __ldg(p.q_scale) : 1.0f);
    if (CTA) {
        if (threadIdx.x < MAXT / 32)
            red[0][0][threadIdx.x] = red[0][1][threadIdx.x] = red[1][0][threadIdx.x] = red[1][1][threadIdx.x] = 0.0f;
        __syncthreads();
    }
    const uint32_t ring = smem_u32(ring_mem + threadIdx.x), per_k = blockDim.x * 16u, per_tensor = per_k * KG;
    const uint32_t per_stage = NT * per_tensor, ring_end = ring + STAGES * per_stage;
    bool in[KG];
    uint64_t dgp[KG][4], dgq[KG][4];
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        in[k] = k * span + lane < p.n8;
#pragma unroll
        for (int e = 0; e < 4; ++e) dgp[k][e] = dgq[k][e] = 0ull;
        // columns behind the row's, and tensors that are not there: zeros that the loop below reads without asking
        for (uint32_t at = ring; at != ring_end; at += per_stage)
#pragma unroll
            for (int i = 0; i < NT; ++i)
                if (!in[k] || (i == DH && !p.dh) || (i == Y && !p.need_y)) ring_put_zero(at + i * per_tensor + k * per_k);
    }
    // gammas behind the ring, [which][k][half][thread], as many as there is room for; 1 for a missing one
    constexpr int NEAR = bn_bwd_near(KG, PRE), FIRST = KG > 3 && PRE ? 1 : 0;
#pragma unroll
    for (int i = FIRST; i < FIRST + NEAR; ++i)
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            uint64_t g[4] = {TWO_ONES, TWO_ONES, TWO_ONES, TWO_ONES};
            const float *from = i ? p.gamma_pre : p.gamma_post;
            if (in[k] && from) load4x2(from + 8 * (k * span + lane), g);
            ring_put(ring_end + (((i - FIRST) * KG + k) * 2) * per_k, g[0], g[1]);
            ring_put(ring_end + (((i - FIRST) * KG + k) * 2 + 1) * per_k, g[2], g[3]);
        }
    const auto gamma = [&](int i, int k, uint64_t (&g)[4]) {
        if (i >= FIRST && i < FIRST + NEAR) {
            ring_get(ring_end + (((i - FIRST) * KG + k) * 2) * per_k, g[0], g[1]);
            ring_get(ring_end + (((i - FIRST) * KG + k) * 2 + 1) * per_k, g[2], g[3]);
        } else if (i || p.gamma_post) {
            load4x2((i ? p.gamma_pre : p.gamma_post) + 8 * (k * span + lane), g);
        } else {
            g[0] = g[1] = g[2] = g[3] = TWO_ONES;
        }
    };
    const size_t pitch = (size_t)at_once * p.n8;
    size_t ahead = rows.begin + sub, at = ahead * p.n8 + lane, at_ahead = at;
    const auto ask = [&](uint32_t to, int i, const uint16_t *src) {
#pragma unroll
        for (int k = 0; k < KG; ++k)
            if (in[k]) cp_async16(to + i * per_tensor + k * per_k, reinterpret_cast<const uint4 *>(src) + at_ahead + k * span);
    };
    const auto fetch_first = [&](uint32_t to) {               // what the first sum and the joint's gradient need
        if (ahead < rows.end) {
            if (PRE) {
                ask(to, DOUT, p.dout);
                ask(to, H, p.h);
            }
            if (p.dh) ask(to, DH, p.dh);
        }
        cp_async_commit();
    };
    const auto fetch_second = [&](uint32_t to) {
        if (ahead < rows.end) {
            if (p.need_y) ask(to, Y, p.y);
            if (GATE) ask(to, G, p.gate);
        }
        cp_async_commit();
        ahead += at_once;
        at_ahead += pitch;
    };
#pragma unroll
    for (int s = 0; s < (STAGES > 1 ? STAGES - 1 : 1); ++s) {
        fetch_first(ring + s * per_stage);
        fetch_second(ring + s * per_stage);
    }
    float m = 0.0f;
    uint32_t now = ring, fill = ring + (STAGES - 1) * per_stage;
    int flip = 0;
    const uint64_t a2 = both(p.a);
    float rp32 = 1.0f, rq32 = 1.0f, rp_ahead = 1.0f, rq_ahead = 1.0f;      // lane l: the statistics of row l of a batch of 32
    if (rows.begin + (threadIdx.x & 31) < rows.end) {
        if (PRE) rp_ahead = __ldg(p.r_pre + rows.begin + (threadIdx.x & 31));
        if (p.rms) rq_ahead = __ldg(p.r_post + rows.begin + (threadIdx.x & 31));
    }
    for (size_t first = rows.begin; first < rows.end; first += at_once, at += pitch, flip ^= 1) {
        const bool live = UNIT != ROW_LANES || first + sub < rows.end;
        if (STAGES > 1) {
            cp_async_wait<PENDING>();
            fetch_first(fill);                   // the stage of the row before this one
            fetch_second(fill);
            fill = now;
        } else {
            cp_async_wait<1>();
        }
        const unsigned in_batch = (unsigned)(first - rows.begin) & 31u;
        if (in_batch == 0) {                     // the next 32 rows' statistics; the batch behind them is on its way
            rp32 = rp_ahead;
            rq32 = rq_ahead;
            const size_t from = first + 32 + (threadIdx.x & 31);
            if (from < rows.end) {
                if (PRE) rp_ahead = __ldg(p.r_pre + from);
                if (p.rms) rq_ahead = __ldg(p.r_post + from);
            }
        }
        const float rp = __shfl_sync(0xffffffffu, rp32, in_batch + sub), rq = __shfl_sync(0xffffffffu, rq32, in_batch + sub);
        uint64_t f[KG][4];
        float c1 = 0.0f;
        {
            uint64_t acc = 0ull;
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                unpack4x2(ring_get(now + DH * per_tensor + k * per_k), f[k]);
                if (!PRE || !live || !in[k]) continue;
                uint64_t d[4], h[4], g[4];
                unpack4x2(ring_get(now + DOUT * per_tensor + k * per_k), d);
                unpack4x2(ring_get(now + H * per_tensor + k * per_k), h);
                gamma(1, k, g);
#pragma unroll
                for (int e = 0; e < 4; ++e) {                 // e r_pre and sums of dout hh, e hh
                    d[e] = mul_f32x2(d[e], both(rp));
                    dgp[k][e] = fma_f32x2(d[e], h[e], dgp[k][e]);
                    d[e] = mul_f32x2(d[e], g[e]);
                    acc = fma_f32x2(d[e], h[e], acc);
                    f[k][e] = add_f32x2(f[k][e], d[e]);
                }
            }
            if (PRE) c1 = row_sum<CTA, MAXT / 32>(add_halves(acc), lanes_log2, red[flip][0]) * -inv_d * rp * rp;
        }
        if (STAGES == 1) cp_async_wait<0>();
        uint64_t acc = 0ull;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            if (!live || !in[k]) continue;
            uint64_t y[4], gq[4];
            if (PRE) {
                uint64_t h[4];
                unpack4x2(ring_get(now + H * per_tensor + k * per_k), h);
#pragma unroll
                for (int e = 0; e < 4; ++e) f[k][e] = fma_f32x2(h[e], both(c1), f[k][e]);
            }
            reinterpret_cast<uint4 *>(p.dx)[at + k * span] = make_uint4(round2(mul_f32x2(a2, f[k][0])), round2(mul_f32x2(a2, f[k][1])),
                                                                       round2(mul_f32x2(a2, f[k][2])), round2(mul_f32x2(a2, f[k][3])));
            unpack4x2(ring_get(now + Y * per_tensor + k * per_k), y);
            gamma(0, k, gq);
            if (GATE) {
                uint64_t g[4];
                uint32_t o[4];
                unpack4x2(ring_get(now + G * per_tensor + k * per_k), g);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f[k][e] = mul_f32x2(f[k][e], both(p.b * rq));
                    uint64_t slope = mul_f32x2(f[k][e], mul_f32x2(y[e], gq[e]));
                    if (p.sigmoid) {
                        uint64_t rest;
                        g[e] = sigmoid2(g[e], rest);
                        slope = mul_f32x2(slope, mul_f32x2(g[e], rest));
                    }
                    o[e] = round2(slope);
                    f[k][e] = mul_f32x2(f[k][e], g[e]);
                }
                reinterpret_cast<uint4 *>(p.dgate)[at + k * span] = make_uint4(o[0], o[1], o[2], o[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) f[k][e] = mul_f32x2(f[k][e], both(p.b * rq));
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {                     // dz r_post, f r_post and sums of dz yh, f yh
                dgq[k][e] = fma_f32x2(f[k][e], y[e], dgq[k][e]);
                f[k][e] = mul_f32x2(f[k][e], gq[e]);
                acc = fma_f32x2(f[k][e], y[e], acc);
            }
        }
        if (STAGES == 1) fetch_first(ring);
        float c2 = 0.0f;
        if (p.rms) c2 = row_sum<CTA, MAXT / 32>(add_halves(acc), lanes_log2, red[flip][1]) * -inv_d * rq * rq;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            if (!live || !in[k]) continue;
            if (p.rms) {
                uint64_t y[4];
                unpack4x2(ring_get(now + Y * per_tensor + k * per_k), y);
#pragma unroll
                for (int e = 0; e < 4; ++e) f[k][e] = fma_f32x2(y[e], both(c2), f[k][e]);
            }
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[e] = round2(f[k][e]);
                m = absmax3(m, f[k][e]);
            }
            if (p.dy) reinterpret_cast<uint4 *>(p.dy)[at + k * span] = make_uint4(o[0], o[1], o[2], o[3]);
            if (p.dy8) reinterpret_cast<uint2 *>(p.dy8)[at + k * span] = codes8(make_uint4(o[0], o[1], o[2], o[3]), qs, p.fmt);
        }
        if (STAGES == 1) fetch_second(ring);
        now += per_stage;
        if (now == ring_end) now = ring;
    }
    cp_async_wait<0>();
    if (p.maxima) {
        const uint32_t most = block_max_bf16(pack_bf16x2(m, 0.0f));
        if (threadIdx.x == 0) p.maxima[blockIdx.x] = most;
    }
    amax_end(pack_bf16x2(m, 0.0f), p.amax_bits, alone);
    if (!p.partial) return;
    const size_t D = (size_t)p.n8 * 8;
    float *mine = p.partial + (size_t)blockIdx.x * 2 * D;
    if (CTA) {
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const unsigned i = k * span + lane;
            if (i >= p.n8) continue;
            float4 *a = reinterpret_cast<float4 *>(mine + 8 * i), *b = reinterpret_cast<float4 *>(mine + D + 8 * i);
            a[0] = quad(dgp[k][0], dgp[k][1]);
            a[1] = quad(dgp[k][2], dgp[k][3]);
            b[0] = quad(dgq[k][0], dgq[k][1]);
            b[1] = quad(dgq[k][2], dgq[k][3]);
        }
    } else {                 // rows of a warp, then warps, hold the same columns: add them up in a fixed order
        for (unsigned off = 16; off >= span; off >>= 1) {
#pragma unroll
            for (int k = 0; k < KG; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    dgp[k][e] = add_f32x2(dgp[k][e], __shfl_xor_sync(0xffffffffu, dgp[k][e], off));
                    dgq[k][e] = add_f32x2(dgq[k][e], __shfl_xor_sync(0xffffffffu, dgq[k][e], off));
                }
        }
        float4 *sum = reinterpret_cast<float4 *>(ring_mem);      // the ring is free: [2][KG * span][2]
        __syncthreads();
        for (unsigned w = 0; w < groups; ++w) {
            if (group == w && sub == 0) {
#pragma unroll
                for (int k = 0; k < KG; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const unsigned to = (k * span + lane) * 2 + h, to2 = KG * span * 2 + to;
                        float4 a = quad(dgp[k][2 * h], dgp[k][2 * h + 1]), b = quad(dgq[k][2 * h], dgq[k][2 * h + 1]);
                        if (w) {
                            const float4 u = sum[to], v = sum[to2];
                            a = make_float4(u.x + a.x, u.y + a.y, u.z + a.z, u.w + a.w);
                            b = make_float4(v.x + b.x, v.y + b.y, v.z + b.z, v.w + b.w);
                        }
                        sum[to] = a;
                        sum[to2] = b;
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

// ---------------------------------------------------------------- launches
struct BnShape {
    bool cta;
    int lanes_log2;
    unsigned threads, grid;
};
// Forward: two groups of columns per thread on lanes of a warp up to 256 columns, on a warp up to 512, on the CTA up to 8192 (one
// group up to 2048 was 3 us slower at 16384 x 1024, four above 4096 1 to 3 us at 4096 x 8192), three up to 12288, then four.  As
// many CTAs per SM as 768 threads make, 640 above 4096 columns (6000 x 5120: 49 -> 38 us), one above 8192.  Above 4096 columns
// three rows travel instead of two, where they find room (4096 x 8192 without a norm in front 43 -> 40 us).
static BnShape bn_fwd_shape(size_t T, size_t D)
{
    const unsigned kg = D <= 8192 ? 2 : D <= 12288 ? 3 : 4, lanes = ((unsigned)(D / 8) + kg - 1) / kg;
    BnShape s;
    s.cta = D > 512;
    s.lanes_log2 = s.cta ? 0 : D > 256 ? 5 : log2_at_least(lanes);
    s.threads = s.cta ? (lanes + 31) & ~31u : 256;
    const size_t at_once = s.cta ? 1 : s.threads >> s.lanes_log2, want = (T + at_once - 1) / at_once;
    const size_t most = 148 * (size_t)((D <= 4096 ? 768 : D <= 8192 ? 640 : 512) / s.threads);
    s.grid = (unsigned)(want < most ? want : most);
    // up to 16 CTAs are one cluster, which sets the amax to zero itself; a second row per unit is less than a launch for that
    if (s.grid > 16 && s.grid <= 32) s.grid = 16;
    return s;
}
// Backward: lanes of a warp with one group of columns each up to 128 columns, a warp with one up to 256 and two up to 512, then
// the CTA with one up to 2048 (8192 x 2048 with a gate: 63 us with two, 52 with one), two up to 8192, three up to 12288 (3000 x
// 10000 with a gate: 154 us with four, 104 with three), four above.  A CTA has eight rows at least where there are more than 148 of
// them (fewer sums to add up behind the pass).
static BnShape bn_bwd_shape(size_t T, size_t D)
{
    const unsigned n8 = (unsigned)(D / 8);
    BnShape s;
    s.cta = D > 512;
    s.lanes_log2 = s.cta || D > 128 ? 5 : log2_at_least(n8);
    const unsigned kg = D <= 2048 ? 1 : D <= 8192 ? 2 : D <= 12288 ? 3 : 4;
    s.threads = s.cta ? ((n8 + kg - 1) / kg + 31) & ~31u : 256;
    const size_t at_once = s.cta ? 8 : (size_t)8 << (5 - s.lanes_log2);
    const size_t most = 148 * (size_t)(s.cta ? (kg == 1 ? 768 : 512) / s.threads : 2);
    size_t want = (T + at_once - 1) / at_once;
    if (s.cta && want < 148) want = T < 148 ? T : 148;
    s.grid = (unsigned)(want < most ? want : most);
    return s;
}

template <auto Kernel, typename P>
static int bn_launch(const P &p, const BnShape &s, size_t smem, size_t most, cudaStream_t st)
{
    if (most > 40 * 1024) {
        const int rc = allow_shared<Kernel>((int)most);
        if (rc != FP8_OK) return rc;
    }
    return launch_behind_amax<Kernel>(p.T * p.n8 * 8, p.amax_bits, s.grid, s.threads, smem, st, p, s.lanes_log2);
}
template <int KG, RowUnit UNIT, int NT, bool PRE, int STAGES, int MAXT, int MINB>
static int bn_fwd_launch(const BnFwd &p, const BnShape &s, cudaStream_t st)
{
    constexpr size_t per_thread = STAGES * NT * KG * 16;
    return bn_launch<block_norm_fwd_kernel<KG, UNIT, NT, PRE, STAGES, MAXT, MINB>>(p, s, per_thread * s.threads, per_thread * MAXT, st);
}
template <int NT, bool PRE>
static int bn_fwd_run(const BnFwd &p, size_t D, cudaStream_t st)
{
    const BnShape s = bn_fwd_shape(p.T, D);
    if (D <= 256) return bn_fwd_launch<2, ROW_LANES, NT, PRE, 2, 256, 3>(p, s, st);
    if (D <= 512) return bn_fwd_launch<2, ROW_WARP, NT, PRE, 2, 256, 3>(p, s, st);
    if (D <= 4096) return bn_fwd_launch<2, ROW_CTA, NT, PRE, 2, 256, 3>(p, s, st);
    if (D <= 8192) return bn_fwd_launch<2, ROW_CTA, NT, PRE, 3, 512, 1>(p, s, st);
    if (D <= 12288) return bn_fwd_launch<3, ROW_CTA, NT, PRE, 3, 512, 1>(p, s, st);
    return bn_fwd_launch<4, ROW_CTA, NT, PRE, 2, 512, 1>(p, s, st);
}
template <int KG, RowUnit UNIT, bool PRE, bool GATE, int STAGES, int MAXT, int MINB>
static int bn_bwd_launch(const BnBwd &p, const BnShape &s, cudaStream_t st)
{
    constexpr size_t per_thread = (STAGES * bn_bwd_tensors(PRE, GATE) + 2 * bn_bwd_near(KG, PRE)) * KG * 16;
    return bn_launch<block_norm_bwd_kernel<KG, UNIT, PRE, GATE, STAGES, MAXT, MINB>>(p, s, per_thread * s.threads, per_thread * MAXT, st);
}
template <bool PRE, bool GATE>
static int bn_bwd_run(const BnBwd &p, const BnShape &s, size_t D, cudaStream_t st)
{
    if (D <= 128) return bn_bwd_launch<1, ROW_LANES, PRE, GATE, 2, 256, 2>(p, s, st);
    if (D <= 256) return bn_bwd_launch<1, ROW_WARP, PRE, GATE, 2, 256, 2>(p, s, st);
    if (D <= 512) return bn_bwd_launch<2, ROW_WARP, PRE, GATE, 2, 256, 2>(p, s, st);
    if (D <= 2048) return bn_bwd_launch<1, ROW_CTA, PRE, GATE, 2, 256, 3>(p, s, st);
    if (D <= 4096) return bn_bwd_launch<2, ROW_CTA, PRE, GATE, 2, 256, 2>(p, s, st);
    if (D <= 8192) return bn_bwd_launch<2, ROW_CTA, PRE, GATE, 2, 512, 1>(p, s, st);
    if (D <= 12288) return bn_bwd_launch<3, ROW_CTA, PRE, GATE, 1, 512, 1>(p, s, st);
    return bn_bwd_launch<4, ROW_CTA, PRE, GATE, 1, 512, 1>(p, s, st);
}

// ---------------------------------------------------------------- checks
static bool finite_f(float v) { return v - v == 0.0f; }
static int bn_check(const char *who, size_t T, size_t D, const fp8_block_norm *c)
{
    if (!c) {
        set_error("%s: NULL configuration", who);
        return FP8_ERR_NULL;
    }
    if (c->post < FP8_NORM_RMS || c->post > FP8_NORM_NONE || (c->gate != FP8_GATE_LINEAR && c->gate != FP8_GATE_SIGMOID)) {
        set_error("%s: post %d / gate %d is not a known enum value", who, c->post, c->gate);
        return FP8_ERR_ENUM;
    }
    if (T == 0 || D == 0 || D % 8 || D > 16384 || T > 0x7FFFFFFFull || !(c->eps >= 0.0f) || !finite_f(c->x_scale) ||
        !finite_f(c->y_scale)) {
        set_error("%s: unsupported shape T=%zu D=%zu (D %% 8 == 0, D <= 16384), eps < 0 or a scale that is not finite", who, T, D);
        return FP8_ERR_SHAPE;
    }
    return FP8_OK;
}

static int bn_fwd(const char *who, const void *x, const void *y, const void *gate, const float *gamma_post, const float *gamma_pre,
                  size_t T, size_t D, const fp8_block_norm *c, const float *q_scale, int fmt, void *h, void *out, uint8_t *out8,
                  float *r_post, float *r_pre, float *amax_out, void *stream)
{
    int rc = bn_check(who, T, D, c);
    if (rc != FP8_OK) return rc;
    if (!x || (gate && !y) || (y && c->post != FP8_NORM_NONE && !gamma_post) || (gamma_pre && !out && !out8) || (!gamma_pre && !h)) {
        set_error("%s: NULL pointer (x; y with a gate; gamma_post with a norm or scale behind the block; an output: out or codes with "
                  "gamma_pre, else h)", who);
        return FP8_ERR_NULL;
    }
    if ((!gamma_pre && out) || (!h && (y || c->x_scale != 1.0f))) {
        set_error("%s: out goes with gamma_pre, and h may be left out where it is x", who);
        return FP8_ERR_SHAPE;
    }
    if (!aligned16(x) || !aligned16(y) || !aligned16(gate) || !aligned16(gamma_post) || !aligned16(gamma_pre) || !aligned16(h) ||
        !aligned16(out) || !aligned16(out8) || !aligned_to(q_scale, 4) || !aligned_to(r_post, 4) || !aligned_to(r_pre, 4) ||
        !aligned_to(amax_out, 4)) {
        set_error("%s: pointers must be 16-byte aligned, the scale, r_post, r_pre and amax_out to their type", who);
        return FP8_ERR_ALIGN;
    }
    rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    BnFwd p = {};
    p.in[0] = static_cast<const uint16_t *>(x);
    p.in[1] = static_cast<const uint16_t *>(y);
    p.in[2] = static_cast<const uint16_t *>(gate);
    p.gamma_post = c->post == FP8_NORM_NONE ? nullptr : gamma_post;
    p.gamma_pre = gamma_pre;
    p.T = T;
    p.n8 = (unsigned)(D / 8);
    p.a = c->x_scale;
    p.b = c->y_scale;
    p.eps = c->eps;
    p.rms = c->post == FP8_NORM_RMS;
    p.sigmoid = c->gate == FP8_GATE_SIGMOID;
    p.h = static_cast<uint16_t *>(h);
    p.out = static_cast<uint16_t *>(out);
    p.r_post = r_post;
    p.r_pre = r_pre;
    p.amax_bits = reinterpret_cast<unsigned int *>(amax_out);
    p.q_scale = q_scale;
    p.out8 = out8;
    p.fmt = fmt;
    if (gamma_pre) return gate ? bn_fwd_run<3, true>(p, D, st) : y ? bn_fwd_run<2, true>(p, D, st) : bn_fwd_run<1, true>(p, D, st);
    return gate ? bn_fwd_run<3, false>(p, D, st) : y ? bn_fwd_run<2, false>(p, D, st) : bn_fwd_run<1, false>(p, D, st);
}

static int bn_bwd(const char *who, const void *dout, const void *dh, const void *h, const void *y, const void *gate,
                  const float *gamma_post, const float *gamma_pre, const float *r_post, const float *r_pre, size_t T, size_t D,
                  const fp8_block_norm *c, const float *q_scale, int fmt, void *dx, void *dy, uint8_t *dy8, void *dgate,
                  float *dgamma_post, float *dgamma_pre, int accumulate, float *amax_out, void *ws, size_t ws_bytes, void *stream)
{
    int rc = bn_check(who, T, D, c);
    if (rc != FP8_OK) return rc;
    const bool pre = gamma_pre != nullptr, scaled = y && c->post != FP8_NORM_NONE, rms = y && c->post == FP8_NORM_RMS;
    if (!dx || (pre ? !dout || !h || !r_pre || !dgamma_pre : !dh) || (y && !dy && !dy8) || (gate && (!y || !dgate)) ||
        (scaled && (!gamma_post || !dgamma_post)) || (rms && !r_post)) {
        set_error("%s: NULL pointer (dx; with gamma_pre dout, h, r_pre and dgamma_pre, else dh; with y its gradient, and what its norm "
                  "and gate need)", who);
        return FP8_ERR_NULL;
    }
    if ((!pre && dout) || (!y && (dy || dy8 || amax_out)) || (!gate && dgate)) {
        set_error("%s: dout goes with gamma_pre, gradients of y and their amax with y, and dgate with a gate", who);
        return FP8_ERR_SHAPE;
    }
    if (!aligned16(dout) || !aligned16(dh) || !aligned16(h) || !aligned16(y) || !aligned16(gate) || !aligned16(gamma_post) ||
        !aligned16(gamma_pre) || !aligned16(dx) || !aligned16(dy) || !aligned16(dy8) || !aligned16(dgate) || !aligned_to(q_scale, 4) ||
        !aligned_to(r_post, 4) || !aligned_to(r_pre, 4) || !aligned_to(dgamma_post, 4) || !aligned_to(dgamma_pre, 4) || !aligned_to(amax_out, 4)) {
        set_error("%s: pointers must be 16-byte aligned, the scale, r_post, r_pre, dgamma_* and amax_out to their type", who);
        return FP8_ERR_ALIGN;
    }
    const size_t need = fp8_block_norm_bwd_workspace_bytes(T, D);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("%s: workspace of %zu bytes, 256-byte aligned, needed (got %zu)", who, need, ws_bytes);
        return FP8_ERR_WORKSPACE;
    }
    rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const BnShape s = bn_bwd_shape(T, D);
    BnBwd p = {};
    p.dout = static_cast<const uint16_t *>(dout);
    p.h = static_cast<const uint16_t *>(h);
    p.dh = static_cast<const uint16_t *>(dh);
    p.y = static_cast<const uint16_t *>(y);
    p.gate = static_cast<const uint16_t *>(gate);
    p.gamma_post = scaled ? gamma_post : nullptr;
    p.gamma_pre = gamma_pre;
    p.r_post = r_post;
    p.r_pre = r_pre;
    p.T = T;
    p.n8 = (unsigned)(D / 8);
    p.a = c->x_scale;
    p.b = c->y_scale;
    p.rms = rms;
    p.sigmoid = c->gate == FP8_GATE_SIGMOID;
    p.need_y = scaled || gate;
    p.dx = static_cast<uint16_t *>(dx);
    p.dy = static_cast<uint16_t *>(dy);
    p.dgate = static_cast<uint16_t *>(dgate);
    p.partial = pre || scaled ? static_cast<float *>(ws) : nullptr;
    unsigned int *const amax = reinterpret_cast<unsigned int *>(amax_out);
    p.maxima = p.partial && amax ? reinterpret_cast<unsigned int *>(p.partial + (size_t)s.grid * 2 * D) : nullptr;
    p.amax_bits = p.maxima ? nullptr : amax;
    p.q_scale = q_scale;
    p.dy8 = dy8;
    p.fmt = fmt;
    if (pre) rc = gate ? bn_bwd_run<true, true>(p, s, D, st) : bn_bwd_run<true, false>(p, s, D, st);
    else rc = gate ? bn_bwd_run<false, true>(p, s, D, st) : bn_bwd_run<false, false>(p, s, D, st);
    if (rc != FP8_OK || !p.partial) return rc;
    return launch_early(p.maxima ? column_sums_kernel<true> : column_sums_kernel<false>, (unsigned)((2 * D + 31) / 32), 1024, 0, st, p.partial, (int)s.grid, (unsigned)D,
                        pre ? dgamma_pre : nullptr, scaled ? dgamma_post : nullptr, accumulate ? 1 : 0,
                        static_cast<const unsigned int *>(p.maxima), amax);
}

}  // namespace fp8dpa

using namespace fp8dpa;

extern "C" int fp8_block_norm_fwd(const void *x_bf16, const void *y_bf16, const void *gate_bf16, const float *gamma_post,
                                  const float *gamma_pre, size_t T, size_t D, const fp8_block_norm *cfg, void *h_bf16,
                                  void *out_bf16, float *r_post, float *r_pre, float *amax_out, void *stream)
{
    return bn_fwd("fp8_block_norm_fwd", x_bf16, y_bf16, gate_bf16, gamma_post, gamma_pre, T, D, cfg, nullptr, 0, h_bf16, out_bf16,
                  nullptr, r_post, r_pre, amax_out, stream);
}

static int check_codes(const char *who, const void *scale, const void *codes, int fmt)
{
    if (!scale || !codes) {
        set_error("%s: NULL scale or codes", who);
        return FP8_ERR_NULL;
    }
    if (fmt != FP8_E4M3 && fmt != FP8_E5M2) {
        set_error("%s: fmt %d is not FP8_E4M3 / FP8_E5M2", who, fmt);
        return FP8_ERR_ENUM;
    }
    return FP8_OK;
}

extern "C" int fp8_block_norm_fwd_q(const void *x_bf16, const void *y_bf16, const void *gate_bf16, const float *gamma_post,
                                    const float *gamma_pre, size_t T, size_t D, const fp8_block_norm *cfg, const float *scale, int fmt,
                                    void *h_bf16, void *out_bf16, uint8_t *out8, float *r_post, float *r_pre, float *amax_out,
                                    void *stream)
{
    const int rc = check_codes("fp8_block_norm_fwd_q", scale, out8, fmt);
    if (rc != FP8_OK) return rc;
    return bn_fwd("fp8_block_norm_fwd_q", x_bf16, y_bf16, gate_bf16, gamma_post, gamma_pre, T, D, cfg, scale, fmt, h_bf16, out_bf16,
                  out8, r_post, r_pre, amax_out, stream);
}

extern "C" size_t fp8_block_norm_bwd_workspace_bytes(size_t T, size_t D)
{
    if (T == 0 || D == 0 || D % 8 || D > 16384 || T > 0x7FFFFFFFull) return 0;
    return ((size_t)bn_bwd_shape(T, D).grid * (2 * D + 1) * sizeof(float) + 255) & ~(size_t)255;
}

extern "C" int fp8_block_norm_bwd(const void *dout_bf16, const void *dh_bf16, const void *h_bf16, const void *y_bf16,
                                  const void *gate_bf16, const float *gamma_post, const float *gamma_pre, const float *r_post,
                                  const float *r_pre, size_t T, size_t D, const fp8_block_norm *cfg, void *dx_bf16, void *dy_bf16,
                                  void *dgate_bf16, float *dgamma_post, float *dgamma_pre, int accumulate, float *amax_out, void *ws,
                                  size_t ws_bytes, void *stream)
{
    return bn_bwd("fp8_block_norm_bwd", dout_bf16, dh_bf16, h_bf16, y_bf16, gate_bf16, gamma_post, gamma_pre, r_post, r_pre, T, D, cfg,
                  nullptr, 0, dx_bf16, dy_bf16, nullptr, dgate_bf16, dgamma_post, dgamma_pre, accumulate, amax_out, ws, ws_bytes,
                  stream);
}

extern "C" int fp8_block_norm_bwd_q(const void *dout_bf16, const void *dh_bf16, const void *h_bf16, const void *y_bf16,
                                    const void *gate_bf16, const float *gamma_post, const float *gamma_pre, const float *r_post,
                                    const float *r_pre, size_t T, size_t D, const fp8_block_norm *cfg, const float *scale, int fmt,
                                    void *dx_bf16, void *dy_bf16, uint8_t *dy8, void *dgate_bf16, float *dgamma_post,
                                    float *dgamma_pre, int accumulate, float *amax_out, void *ws, size_t ws_bytes, void *stream)
{
    const int rc = check_codes("fp8_block_norm_bwd_q", scale, dy8, fmt);
    if (rc != FP8_OK) return rc;
    return bn_bwd("fp8_block_norm_bwd_q", dout_bf16, dh_bf16, h_bf16, y_bf16, gate_bf16, gamma_post, gamma_pre, r_post, r_pre, T, D,
                  cfg, scale, fmt, dx_bf16, dy_bf16, dy8, dgate_bf16, dgamma_post, dgamma_pre, accumulate, amax_out, ws, ws_bytes,
                  stream);
}
