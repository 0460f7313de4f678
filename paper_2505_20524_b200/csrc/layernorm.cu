// Layer norm: out = residual + gamma (x - mean) / sqrt(var + eps) + beta per token row, with the amax and the FP8 codes of
// the result for the next product, and its backward pass with the reduction of dgamma and dbeta.
#include <math.h>

#include "common.cuh"
#include "elementwise.cuh"

namespace fp8dpa {

// Sum over the TPR threads that share a row.  TPR = 32: a warp; otherwise the whole CTA, through `red` (a buffer that this
// call alone uses until the next barrier).
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *red)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if (TPR > 32) {
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < TPR / 32; ++w) v += red[w];
    }
    return v;
}

__device__ __forceinline__ void unpack8(const uint4 v, float (&f)[8])
{
    f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
}
__device__ __forceinline__ void load8f(const float *p, float (&f)[8])
{
    const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

// ---------------------------------------------------------------- forward
// TPR threads per row, KG groups of eight columns per thread, the row in registers between the two sums (the mean, then the
// squared distances from it: no cancellation however far the mean lies from zero) and the result: one read of x.
template <int TPR, int KG>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) layernorm_fwd_kernel(
    const uint16_t *__restrict__ x, const float *__restrict__ gamma, const float *__restrict__ beta,
    const uint16_t *__restrict__ residual, size_t T, unsigned n8, float eps, uint16_t *__restrict__ out,
    float *__restrict__ mean_out, float *__restrict__ rstd_out, unsigned int *__restrict__ amax_bits,
    const float *__restrict__ q_scale, uint8_t *__restrict__ out8, int fmt)
{
    __shared__ float red[2][TPR / 32];
    const int lane = TPR == 32 ? (threadIdx.x & 31) : threadIdx.x;
    const size_t t = TPR == 32 ? (size_t)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
    const bool live = t < T;
    const float qs = out8 ? __ldg(q_scale) : 1.0f;
    const size_t row = (live ? t : 0) * n8;
    uint4 xv[KG], rv[KG];
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        const unsigned i = k * TPR + lane;
        xv[k] = rv[k] = make_uint4(0u, 0u, 0u, 0u);
        if (live && i < n8) {
            xv[k] = __ldg(reinterpret_cast<const uint4 *>(x) + row + i);
            if (residual) rv[k] = __ldg(reinterpret_cast<const uint4 *>(residual) + row + i);
        }
    }
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        float f[8];
        unpack8(xv[k], f);
        s += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
    }
    const float inv_d = 1.0f / (float)(n8 * 8);
    const float mean = row_sum<TPR>(s, red[0]) * inv_d;
    float ss = 0.0f;
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        if (k * TPR + lane >= n8) continue;
        float f[8];
        unpack8(xv[k], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(f[e] - mean, f[e] - mean, ss);
    }
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(ss, red[1]) * inv_d + eps);
    if (live && lane == 0) {
        if (mean_out) mean_out[t] = mean;
        if (rstd_out) rstd_out[t] = rstd;
    }
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < KG; ++k) {
        const unsigned i = k * TPR + lane;
        if (!live || i >= n8) continue;
        float f[8], r[8], g[8], b[8];
        unpack8(xv[k], f);
        unpack8(rv[k], r);
        load8f(gamma + 8 * i, g);
        load8f(beta + 8 * i, b);
        uint32_t o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float lo = fmaf((f[2 * q] - mean) * rstd, g[2 * q], b[2 * q]) + r[2 * q];
            const float hi = fmaf((f[2 * q + 1] - mean) * rstd, g[2 * q + 1], b[2 * q + 1]) + r[2 * q + 1];
            o[q] = pack_bf16x2(lo, hi);
            m = absmax2e(m, o[q]);
        }
        reinterpret_cast<uint4 *>(out)[row + i] = make_uint4(o[0], o[1], o[2], o[3]);
        if (out8) reinterpret_cast<uint2 *>(out8)[row + i] = bf16x8_to_fp8x8(o, qs, fmt);
    }
    if (amax_bits) block_max_bf16_to(m, amax_bits);
}

// ---------------------------------------------------------------- backward
// With xh = (x - mean) rstd and g = gamma dout:  dx = rstd (g - mean(g) - xh mean(g xh)), dgamma = sum over rows of dout xh,
// dbeta = sum over rows of dout.  Persistent CTAs; a thread keeps its columns' dgamma and dbeta in registers over all rows of
// its CTA (or warp, for short rows) and leaves them in `partial` [CTA][2][D]; layernorm_bwd_sum_kernel adds the CTAs up in a
// fixed order.  Reads x and dout once, writes dx once.
template <int TPR, int KG>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) layernorm_bwd_kernel(
    const uint16_t *__restrict__ dout, const uint16_t *__restrict__ x, const float *__restrict__ gamma,
    const float *__restrict__ mean, const float *__restrict__ rstd, size_t T, unsigned n8, uint16_t *__restrict__ dx,
    float *__restrict__ partial)
{
    constexpr int RG = TPR == 32 ? 8 : 1;           // rows a CTA works on at a time
    __shared__ float red[2][2][TPR / 32];
    const int lane = TPR == 32 ? (threadIdx.x & 31) : threadIdx.x, group = TPR == 32 ? (threadIdx.x >> 5) : 0;
    const float inv_d = 1.0f / (float)(n8 * 8);
    float dg[KG][8], db[KG][8];
#pragma unroll
    for (int k = 0; k < KG; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) dg[k][e] = db[k][e] = 0.0f;
    int flip = 0;
    for (size_t t0 = (size_t)blockIdx.x * RG; t0 < T; t0 += (size_t)gridDim.x * RG, flip ^= 1) {
        const size_t t = t0 + group;
        const bool live = t < T;
        const size_t row = (live ? t : 0) * n8;
        const float mu = live ? __ldg(mean + t) : 0.0f, rs = live ? __ldg(rstd + t) : 0.0f;
        uint4 xv[KG], dv[KG];
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const unsigned i = k * TPR + lane;
            xv[k] = dv[k] = make_uint4(0u, 0u, 0u, 0u);
            if (live && i < n8) {
                xv[k] = __ldg(reinterpret_cast<const uint4 *>(x) + row + i);
                dv[k] = __ldg(reinterpret_cast<const uint4 *>(dout) + row + i);
            }
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const unsigned i = k * TPR + lane;
            if (!live || i >= n8) continue;
            float f[8], d[8], g[8];
            unpack8(xv[k], f);
            unpack8(dv[k], d);
            load8f(gamma + 8 * i, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = (f[e] - mu) * rs, ge = d[e] * g[e];
                dg[k][e] = fmaf(d[e], xh, dg[k][e]);
                db[k][e] += d[e];
                s1 += ge;
                s2 = fmaf(ge, xh, s2);
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            s1 += __shfl_xor_sync(0xffffffffu, s1, off);
            s2 += __shfl_xor_sync(0xffffffffu, s2, off);
        }
        if (TPR > 32) {      // two buffers in turn: the next row's writes do not meet this row's reads
            if ((threadIdx.x & 31) == 0) {
                red[flip][0][threadIdx.x >> 5] = s1;
                red[flip][1][threadIdx.x >> 5] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int w = 0; w < TPR / 32; ++w) {
                s1 += red[flip][0][w];
                s2 += red[flip][1][w];
            }
        }
        s1 *= inv_d;
        s2 *= inv_d;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const unsigned i = k * TPR + lane;
            if (!live || i >= n8) continue;
            float f[8], d[8], g[8];
            unpack8(xv[k], f);
            unpack8(dv[k], d);
            load8f(gamma + 8 * i, g);
            uint32_t o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float xa = (f[2 * q] - mu) * rs, xb = (f[2 * q + 1] - mu) * rs;
                o[q] = pack_bf16x2(rs * (fmaf(d[2 * q], g[2 * q], -s1) - xa * s2),
                                   rs * (fmaf(d[2 * q + 1], g[2 * q + 1], -s1) - xb * s2));
            }
            reinterpret_cast<uint4 *>(dx)[row + i] = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
    const size_t D = (size_t)n8 * 8;
    float *mine = partial + (size_t)blockIdx.x * 2 * D;
    if (TPR > 32) {
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            const unsigned i = k * TPR + lane;
            if (i >= n8) continue;
            float4 *a = reinterpret_cast<float4 *>(mine + 8 * i), *b = reinterpret_cast<float4 *>(mine + D + 8 * i);
            a[0] = make_float4(dg[k][0], dg[k][1], dg[k][2], dg[k][3]);
            a[1] = make_float4(dg[k][4], dg[k][5], dg[k][6], dg[k][7]);
            b[0] = make_float4(db[k][0], db[k][1], db[k][2], db[k][3]);
            b[1] = make_float4(db[k][4], db[k][5], db[k][6], db[k][7]);
        }
    } else {                 // eight warps hold the same columns: add them in shared memory, warp by warp
        __shared__ float sum[2][KG * 32 * 8];
        for (int w = 0; w < 8; ++w) {
            if (group == w) {
#pragma unroll
                for (int k = 0; k < KG; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int at = (k * 32 + lane) * 8 + e;
                        sum[0][at] = w ? sum[0][at] + dg[k][e] : dg[k][e];
                        sum[1][at] = w ? sum[1][at] + db[k][e] : db[k][e];
                    }
            }
            __syncthreads();
        }
        for (unsigned j = threadIdx.x; j < n8 * 8; j += 256) {
            mine[j] = sum[0][j];
            mine[D + j] = sum[1][j];
        }
    }
}

// dgamma and dbeta from the CTAs' sums: 32 columns per CTA, eight threads per column take every eighth CTA.
__global__ void __launch_bounds__(256) layernorm_bwd_sum_kernel(const float *__restrict__ partial, int parts, unsigned D,
                                                                float *__restrict__ dgamma, float *__restrict__ dbeta,
                                                                int accumulate)
{
    __shared__ float red[8][33];
    const unsigned j = blockIdx.x * 32 + (threadIdx.x & 31);      // over [2][D]
    const int r = threadIdx.x >> 5;
    float s = 0.0f;
    if (j < 2 * D) {
#pragma unroll 4
        for (int c = r; c < parts; c += 8) s += __ldcg(partial + (size_t)c * 2 * D + j);
    }
    red[r][threadIdx.x & 31] = s;
    __syncthreads();
    if (r == 0 && j < 2 * D) {
#pragma unroll
        for (int w = 1; w < 8; ++w) s += red[w][threadIdx.x];
        float *o = j < D ? dgamma + j : dbeta + (j - D);
        *o = accumulate ? *o + s : s;
    }
}

// CTAs of the backward pass and so rows of its workspace: what keeps the SMs busy, no more than there is work for.
static size_t bwd_parts(size_t T, size_t D)
{
    const size_t rows = D <= 1024 ? 8 : 1;
    const size_t most = 148 * (size_t)(D <= 4096 ? 4 : D <= 8192 ? 2 : 1), want = (T + rows - 1) / rows;
    return want < most ? want : most;
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
    if (amax_out) FP8_CUDA_CHECK(cudaMemsetAsync(amax_out, 0, sizeof(float), st));
    const unsigned n8 = (unsigned)(D / 8);
#define FP8DPA_LAUNCH_LN(TPR, KG) \
    layernorm_fwd_kernel<TPR, KG><<<(unsigned)(TPR == 32 ? (T + 7) / 8 : T), TPR > 32 ? TPR : 256, 0, st>>>( \
        static_cast<const uint16_t *>(x), gamma, beta, static_cast<const uint16_t *>(residual), T, n8, eps, \
        static_cast<uint16_t *>(out), mean, rstd, reinterpret_cast<unsigned int *>(amax_out), q_scale, out8, fmt)
    if (D <= 256) FP8DPA_LAUNCH_LN(32, 1);
    else if (D <= 512) FP8DPA_LAUNCH_LN(32, 2);
    else if (D <= 1024) FP8DPA_LAUNCH_LN(32, 4);
    else if (D <= 2048) FP8DPA_LAUNCH_LN(128, 2);
    else if (D <= 4096) FP8DPA_LAUNCH_LN(256, 2);
    else if (D <= 8192) FP8DPA_LAUNCH_LN(512, 2);
    else FP8DPA_LAUNCH_LN(1024, 2);
#undef FP8DPA_LAUNCH_LN
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
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
    return layernorm_shape_ok(T, D) ? (bwd_parts(T, D) * 2 * D * sizeof(float) + 255) & ~(size_t)255 : 0;
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
    const unsigned n8 = (unsigned)(D / 8), parts = (unsigned)bwd_parts(T, D);
    float *partial = static_cast<float *>(ws);
#define FP8DPA_LAUNCH_LB(TPR, KG) \
    layernorm_bwd_kernel<TPR, KG><<<parts, TPR > 32 ? TPR : 256, 0, st>>>( \
        static_cast<const uint16_t *>(dout_bf16), static_cast<const uint16_t *>(x_bf16), gamma, mean, rstd, T, n8, \
        static_cast<uint16_t *>(dx_bf16), partial)
    if (D <= 256) FP8DPA_LAUNCH_LB(32, 1);
    else if (D <= 512) FP8DPA_LAUNCH_LB(32, 2);
    else if (D <= 1024) FP8DPA_LAUNCH_LB(32, 4);
    else if (D <= 2048) FP8DPA_LAUNCH_LB(256, 1);
    else if (D <= 4096) FP8DPA_LAUNCH_LB(512, 1);
    else if (D <= 8192) FP8DPA_LAUNCH_LB(512, 2);
    else FP8DPA_LAUNCH_LB(1024, 2);
#undef FP8DPA_LAUNCH_LB
    FP8_CUDA_CHECK(cudaGetLastError());
    layernorm_bwd_sum_kernel<<<(unsigned)((2 * D + 31) / 32), 256, 0, st>>>(partial, (int)parts, (unsigned)D, dgamma, dbeta,
                                                                           accumulate ? 1 : 0);
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
}
