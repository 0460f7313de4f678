// Router of the grouped (mixture-of-experts) products: experts and weights of every token, the counts and offsets and the
// order of rows that the grouped products read, the balance and z losses, and the gradient of the logits.
//
// A CTA owns a chunk of consecutive tokens in both forward kernels, so that the second can place its rows behind those of
// the chunks before it: a counting sort with the expert as its only digit, stable in (token, slot).  Probability sums are
// kept per CTA and added in the order of the CTAs: no floating-point atomics.
#include <math.h>

#include "common.cuh"
#include "stable_rank.cuh"

namespace fp8dpa {

constexpr int RT_THREADS = 256;
constexpr int RT_WARPS = RT_THREADS / 32;
constexpr int RT_MAX_E = 256;
constexpr int RT_MAX_K = 16;
constexpr size_t RT_MAX_CHUNKS = 148;

struct RouteParams {
    const void *logits;
    const float *bias;
    size_t T, chunk;                 // tokens per CTA
    int E, k, normalize;
    float balance_coef, z_coef;
    int *expert;
    float *weight;
    int *counts, *offsets, *rows, *n_routed;
    float *loss;
    int *cta_counts;                 // [CTAs][E]
    float *cta_probs;                // [CTAs][E]
    double *cta_z;                   // [CTAs]: sum of lse^2 (a row of the type's lowest value has lse^2 beyond FP32)
    int *cta_n;                      // [CTAs]: routed tokens
    int ctas;
    const int *n_in, *counts_in;     // backward
    const float *dloss, *dweight;
    void *dlogits;
};

// order-preserving map of binary32 (no NaN) to unsigned; -inf maps to 0x007FFFFF
__device__ __forceinline__ uint32_t float_key(float f)
{
    const uint32_t b = __float_as_uint(f + 0.0f);                 // -0 becomes +0: equal values, equal keys
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
constexpr uint32_t KEY_NEG_INF = 0x007FFFFFu;

template <bool F32>
__device__ __forceinline__ float load_logit(const void *p, size_t i)
{
    if (F32) return __ldg(static_cast<const float *>(p) + i);
    return __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t *>(p) + i) << 16);
}

// all-lane reductions over groups of G lanes (G a power of two)
template <int G> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int G> __device__ __forceinline__ float group_max(float v)
{
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <int G> __device__ __forceinline__ unsigned long long group_max64(unsigned long long v)
{
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) {
        const unsigned long long u = __shfl_xor_sync(0xffffffffu, v, o);
        v = u > v ? u : v;
    }
    return v;
}

// What both passes need of a token: its logits (lane l of the group holds experts l, l + G, ...), whether it is routed
// (a finite logit, nothing NaN or +inf), whether it is broken (NaN or +inf), the maximum and the sum of exponentials.
template <bool F32, int G, int PL>
struct Token {
    float l[PL], p[PL];
    float top, total;
    bool routed, broken;

    __device__ __forceinline__ void load(const void *logits, size_t t, int E, int gl, bool live)
    {
        float mx = -INFINITY;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            const int e = i * G + gl;
            l[i] = live && e < E ? load_logit<F32>(logits, t * E + e) : -INFINITY;
            bad |= !(l[i] < INFINITY);
            mx = fmaxf(mx, l[i]);
        }
        top = group_max<G>(mx);
        broken = group_max<G>(bad ? 1.0f : 0.0f) > 0.0f;
        routed = !broken && top > -INFINITY;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            p[i] = routed ? expf(l[i] - top) : 0.0f;
            s += p[i];
        }
        total = group_sum<G>(s);
        const float inv = routed ? 1.0f / total : broken ? NAN : 0.0f;
#pragma unroll
        for (int i = 0; i < PL; ++i) p[i] = broken ? (i * G + gl < E ? inv : 0.0f) : p[i] * inv;
    }
    __device__ __forceinline__ float lse() const { return broken ? NAN : routed ? top + logf(total) : 0.0f; }
};

// Forward, first kernel.  G lanes per token, PL experts per lane; a group takes the chunk's tokens in turn.
template <bool F32, int G, int PL>
__global__ void __launch_bounds__(RT_THREADS) route_choose_kernel(const RouteParams q)
{
    constexpr int GROUPS = RT_THREADS / G;
    __shared__ int cnt[RT_MAX_E];
    __shared__ float probs[RT_WARPS][G * PL];
    __shared__ double zsum[RT_WARPS];
    __shared__ int nsum[RT_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gl = tid & (G - 1), group = tid / G;
    for (int e = tid; e < q.E; e += RT_THREADS) cnt[e] = 0;
    __syncthreads();
    float ps[PL];
    double z = 0.0;
    int n = 0;
#pragma unroll
    for (int i = 0; i < PL; ++i) ps[i] = 0.0f;
    const size_t t0 = blockIdx.x * q.chunk, t1 = min(q.T, t0 + q.chunk);
    for (size_t base = t0; base < t1; base += GROUPS) {
        const size_t t = base + group;
        const bool live = t < t1;
        Token<F32, G, PL> tok;
        tok.load(q.logits, t, q.E, gl, live);
#pragma unroll
        for (int i = 0; i < PL; ++i) ps[i] += tok.p[i];
        const double lse = (double)tok.lse();
        const bool counted = gl == 0 && (tok.routed || tok.broken);
        z = counted ? fma(lse, lse, z) : z;
        n += counted ? 1 : 0;
        // the k largest scores, one maximum at a time; equal scores: the lowest expert
        unsigned long long key[PL];
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            const int e = i * G + gl;
            const float s = e < q.E ? (q.bias ? tok.l[i] + __ldg(q.bias + e) : tok.l[i]) : -INFINITY;
            const uint32_t k32 = tok.routed && s == s ? float_key(s) : 0u;
            key[i] = k32 > KEY_NEG_INF ? ((unsigned long long)k32 << 32) | (uint32_t)(0xFFFFFFFFu - e) : 0ull;
        }
        float wl[RT_MAX_K / 8 > 0 ? (RT_MAX_K + G - 1) / G : 1];   // slot j's logit (or probability), held by lane j % G
        int we[(RT_MAX_K + G - 1) / G];
#pragma unroll
        for (int i = 0; i < (RT_MAX_K + G - 1) / G; ++i) {
            wl[i] = -INFINITY;
            we[i] = -1;
        }
        for (int j = 0; j < q.k; ++j) {
            unsigned long long best = 0ull;
#pragma unroll
            for (int i = 0; i < PL; ++i) best = key[i] > best ? key[i] : best;
            best = group_max64<G>(best);
            const int e = best ? (int)(0xFFFFFFFFu - (uint32_t)best) : -1;
            float v = -INFINITY;
#pragma unroll
            for (int i = 0; i < PL; ++i)
                if (e >= 0 && i * G + gl == e) {
                    v = q.normalize ? tok.l[i] : tok.p[i];
                    key[i] = 0ull;
                }
            v = group_max<G>(v);
#pragma unroll
            for (int i = 0; i < (RT_MAX_K + G - 1) / G; ++i)
                if (j == i * G + gl) {
                    wl[i] = v;
                    we[i] = e;
                }
        }
        float high = -INFINITY, ws = 0.0f;
        if (q.normalize) {
#pragma unroll
            for (int i = 0; i < (RT_MAX_K + G - 1) / G; ++i) high = fmaxf(high, wl[i]);
            high = group_max<G>(high);
#pragma unroll
            for (int i = 0; i < (RT_MAX_K + G - 1) / G; ++i) {
                wl[i] = we[i] >= 0 ? expf(wl[i] - high) : 0.0f;
                ws += wl[i];
            }
            ws = group_sum<G>(ws);
        }
#pragma unroll
        for (int i = 0; i < (RT_MAX_K + G - 1) / G; ++i) {
            const int j = i * G + gl;
            if (live && j < q.k) {
                q.expert[t * q.k + j] = we[i];
                q.weight[t * q.k + j] = tok.broken ? NAN : we[i] < 0 ? 0.0f : q.normalize ? wl[i] / ws : wl[i];
                if (we[i] >= 0) atomicAdd(&cnt[we[i]], 1);
            }
        }
    }
    // sums over the groups of a warp, then over the warps in order
#pragma unroll
    for (int i = 0; i < PL; ++i) {
#pragma unroll
        for (int o = G; o < 32; o <<= 1) ps[i] += __shfl_xor_sync(0xffffffffu, ps[i], o);
        if (lane < G) probs[warp][i * G + lane] = ps[i];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) {
        zsum[warp] = z;
        nsum[warp] = n;
    }
    __syncthreads();
    for (int e = tid; e < q.E; e += RT_THREADS) {
        float s = probs[0][e];
#pragma unroll
        for (int w = 1; w < RT_WARPS; ++w) s += probs[w][e];
        q.cta_probs[(size_t)blockIdx.x * q.E + e] = s;
        q.cta_counts[(size_t)blockIdx.x * q.E + e] = cnt[e];
    }
    if (tid == 0) {
        for (int w = 1; w < RT_WARPS; ++w) {
            z += zsum[w];
            n += nsum[w];
        }
        q.cta_z[blockIdx.x] = z;
        q.cta_n[blockIdx.x] = n;
    }
}

// Forward, second kernel: thread e sums the chunks' counts of expert e.  Every CTA places its rows; the first one also
// writes counts, offsets, the token count and the losses; all clear the rows behind the last one.
__global__ void __launch_bounds__(RT_THREADS) route_place_kernel(const RouteParams q)
{
    __shared__ int warp_cnt[RT_WARPS][RT_MAX_E];
    __shared__ int base[RT_MAX_E];
    __shared__ int warp_sum[RT_WARPS];
    __shared__ double dred[RT_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int total = 0, mine = 0;
    if (tid < q.E) {
#pragma unroll 8
        for (int c = 0; c < q.ctas; ++c) {
            const int v = __ldcg(q.cta_counts + (size_t)c * q.E + tid);
            if (c < (int)blockIdx.x) mine += v;
            total += v;
        }
    }
    int scan = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += v;
    }
    if (lane == 31) warp_sum[warp] = scan;
    __syncthreads();
    int start = scan - total, all = 0;
    for (int w = 0; w < RT_WARPS; ++w) {
        if (w < warp) start += warp_sum[w];
        all += warp_sum[w];
    }
    base[tid] = start + mine;
    if (blockIdx.x == 0) {
        int n = 0;
        double z = 0.0;
        for (int c = tid; c < q.ctas; c += RT_THREADS) {
            n += __ldcg(q.cta_n + c);
            z += __ldcg(q.cta_z + c);
        }
        __shared__ int nred[RT_WARPS];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) {
            dred[warp] = z;
            nred[warp] = n;
        }
        __syncthreads();
        n = 0;
        z = 0.0;
        for (int w = 0; w < RT_WARPS; ++w) {
            n += nred[w];
            z += dred[w];
        }
        double f = 0.0;
        if (tid < q.E) {
            double p = 0.0;
#pragma unroll 8
            for (int c = 0; c < q.ctas; ++c) p += (double)__ldcg(q.cta_probs + (size_t)c * q.E + tid);
            f = (double)total * p;
            q.counts[tid] = total;
            q.offsets[tid] = start;
        }
        if (tid == 0) {
            q.offsets[q.E] = all;
            *q.n_routed = n;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) f += __shfl_xor_sync(0xffffffffu, f, o);
        __syncthreads();
        if (lane == 0) dred[warp] = f;
        __syncthreads();
        if (tid == 0) {
            f = 0.0;
            for (int w = 0; w < RT_WARPS; ++w) f += dred[w];
            const double dn = (double)n;
            q.loss[0] = n ? (float)((double)q.balance_coef * q.E * f / (dn * dn * q.k)) : 0.0f;
            q.loss[1] = n ? (float)((double)q.z_coef * z / dn) : 0.0f;
        }
    }
    if (!q.rows) return;
    const size_t copies = q.T * q.k;
    for (size_t i = (size_t)all + blockIdx.x * RT_THREADS + tid; i < copies; i += (size_t)gridDim.x * RT_THREADS) q.rows[i] = -1;
    const size_t i0 = blockIdx.x * q.chunk * q.k, i1 = min(copies, i0 + q.chunk * q.k);
    constexpr int ITEMS = 4;
    for (size_t tile = i0; tile < i1; tile += RT_THREADS * ITEMS) {
        for (int i = tid; i < RT_WARPS * RT_MAX_E; i += RT_THREADS) warp_cnt[i / RT_MAX_E][i % RT_MAX_E] = 0;
        __syncthreads();
        int e[ITEMS], rank[ITEMS];
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            const size_t i = tile + (size_t)warp * (32 * ITEMS) + j * 32 + lane;
            e[j] = i < i1 ? __ldcg(q.expert + i) : -1;
        }
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) rank[j] = warp_stable_rank(e[j], warp_cnt[warp], lane);
        __syncthreads();
        if (tid < q.E) {
            int at = base[tid];
#pragma unroll
            for (int w = 0; w < RT_WARPS; ++w) {
                const int v = warp_cnt[w][tid];
                warp_cnt[w][tid] = at;
                at += v;
            }
            base[tid] = at;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < ITEMS; ++j)
            if (e[j] >= 0) q.rows[warp_cnt[warp][e[j]] + rank[j]] = (int)(tile + (size_t)warp * (32 * ITEMS) + j * 32 + lane);
        __syncthreads();
    }
}

// Backward: one pass over the logits, everything of a token in its lane group.
//   u_e = dloss * balance_coef * E * counts_e / (k n^2)  (+ dweight of e's slot, without normalisation)
//   dl_e = p_e (u_e - sum u p) + dloss * z_coef * 2 lse / n * p_e  (+ w_j (dw_j - sum dw w) in slot j, with normalisation)
template <bool F32, int G, int PL>
__global__ void __launch_bounds__(RT_THREADS) route_bwd_kernel(const RouteParams q)
{
    constexpr int GROUPS = RT_THREADS / G;
    constexpr int SL = (RT_MAX_K + G - 1) / G;
    const int gl = threadIdx.x & (G - 1), group = threadIdx.x / G;
    const float d = q.dloss ? __ldg(q.dloss) : 1.0f;
    const float n = (float)__ldg(q.n_in);
    const float ub = n > 0.0f ? d * q.balance_coef * (float)q.E / (n * n * (float)q.k) : 0.0f;
    const float uz = n > 0.0f ? d * q.z_coef * 2.0f / n : 0.0f;
    float u0[PL];
#pragma unroll
    for (int i = 0; i < PL; ++i) u0[i] = i * G + gl < q.E ? ub * (float)__ldg(q.counts_in + i * G + gl) : 0.0f;
    for (size_t base = (size_t)blockIdx.x * GROUPS; base < q.T; base += (size_t)gridDim.x * GROUPS) {
        const size_t t = base + group;
        const bool live = t < q.T;
        Token<F32, G, PL> tok;
        tok.load(q.logits, t, q.E, gl, live);
        float u[PL], add[PL];
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            u[i] = u0[i];
            add[i] = 0.0f;
        }
        if (q.dweight) {
            int se[SL];
            float sd[SL], sw[SL];
            float high = -INFINITY;
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                const int j = i * G + gl;
                se[i] = live && j < q.k ? __ldg(q.expert + t * q.k + j) : -1;
                if (se[i] >= q.E) se[i] = -1;
                sd[i] = se[i] >= 0 ? __ldg(q.dweight + t * q.k + j) : 0.0f;
                sw[i] = q.normalize && se[i] >= 0 ? load_logit<F32>(q.logits, t * q.E + se[i]) : -INFINITY;
                high = fmaxf(high, sw[i]);
            }
            if (q.normalize) {
                high = group_max<G>(high);
                float s = 0.0f, sdw = 0.0f;
#pragma unroll
                for (int i = 0; i < SL; ++i) {
                    sw[i] = se[i] >= 0 ? expf(sw[i] - high) : 0.0f;
                    s += sw[i];
                }
                s = group_sum<G>(s);
                const float inv = s > 0.0f ? 1.0f / s : 0.0f;
#pragma unroll
                for (int i = 0; i < SL; ++i) {
                    sw[i] *= inv;
                    sdw = fmaf(sd[i], sw[i], sdw);
                }
                sdw = group_sum<G>(sdw);
#pragma unroll
                for (int i = 0; i < SL; ++i) sd[i] = sw[i] * (sd[i] - sdw);
            }
            for (int j = 0; j < q.k; ++j) {                       // slot j's expert and value to the lane that holds it
                int e = -1;
                float v = 0.0f;
#pragma unroll
                for (int i = 0; i < SL; ++i)
                    if (j / G == i) {
                        e = se[i];
                        v = sd[i];
                    }
                e = __shfl_sync(0xffffffffu, e, j % G, G);
                v = __shfl_sync(0xffffffffu, v, j % G, G);
#pragma unroll
                for (int i = 0; i < PL; ++i)
                    if (e == i * G + gl) {
                        if (q.normalize) add[i] += v;
                        else u[i] += v;
                    }
            }
        }
        float up = 0.0f;
#pragma unroll
        for (int i = 0; i < PL; ++i) up = fmaf(u[i], tok.p[i], up);
        up = group_sum<G>(up);
        const float zz = tok.routed ? uz * tok.lse() : 0.0f;
        if (!live) continue;
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            const int e = i * G + gl;
            if (e >= q.E) continue;
            const float g = tok.broken ? NAN : fmaf(tok.p[i], (u[i] - up) + zz, add[i]);
            if (F32) static_cast<float *>(q.dlogits)[t * q.E + e] = g;
            else static_cast<uint16_t *>(q.dlogits)[t * q.E + e] = (uint16_t)(pack_bf16x2(g, g) & 0xFFFFu);
        }
    }
}

static bool route_shape_ok(size_t T, int E)
{
    return T > 0 && T <= ((size_t)1 << 26) && E > 0 && E <= RT_MAX_E;
}
static size_t route_chunk(size_t T)
{
    const size_t c = (T + RT_MAX_CHUNKS - 1) / RT_MAX_CHUNKS;
    return c < 32 ? 32 : c;
}
static size_t route_ctas(size_t T) { return (T + route_chunk(T) - 1) / route_chunk(T); }

}  // namespace fp8dpa

using namespace fp8dpa;

#define FP8DPA_ROUTE_DISPATCH(KERNEL, GRID)                                          \
    do {                                                                             \
        if (q.E <= 8) FP8DPA_ROUTE_TYPE(KERNEL, GRID, 8, 1);                         \
        else if (q.E <= 16) FP8DPA_ROUTE_TYPE(KERNEL, GRID, 16, 1);                  \
        else if (q.E <= 32) FP8DPA_ROUTE_TYPE(KERNEL, GRID, 32, 1);                  \
        else if (q.E <= 64) FP8DPA_ROUTE_TYPE(KERNEL, GRID, 32, 2);                  \
        else if (q.E <= 128) FP8DPA_ROUTE_TYPE(KERNEL, GRID, 32, 4);                 \
        else FP8DPA_ROUTE_TYPE(KERNEL, GRID, 32, 8);                                 \
    } while (0)
#define FP8DPA_ROUTE_TYPE(KERNEL, GRID, G, PL)                                       \
    do {                                                                             \
        if (is_fp32) KERNEL<true, G, PL><<<GRID, RT_THREADS, 0, st>>>(q);            \
        else KERNEL<false, G, PL><<<GRID, RT_THREADS, 0, st>>>(q);                   \
    } while (0)

static int route_check(const char *who, size_t T, int E, int k, float balance_coef, float z_coef)
{
    if (!route_shape_ok(T, E) || k <= 0 || k > E || k > RT_MAX_K || !(balance_coef == balance_coef) || !(z_coef == z_coef)) {
        set_error("%s: unsupported shape T=%zu E=%d k=%d (T <= 2^26, E <= 256, k <= min(E, 16)) or a coefficient is NaN", who, T, E, k);
        return FP8_ERR_SHAPE;
    }
    return FP8_OK;
}

extern "C" size_t fp8_moe_route_workspace_bytes(size_t T, int E)
{
    return route_shape_ok(T, E) ? (route_ctas(T) * ((size_t)E * 8 + 12) + 255) & ~(size_t)255 : 0;
}

extern "C" int fp8_moe_route(const void *logits, int is_fp32, const float *bias, size_t T, int E, int k, int normalize,
                             float balance_coef, float z_coef, int *expert, float *weight, int *counts, int *offsets,
                             int *rows, int *n_routed, float *loss, void *ws, size_t ws_bytes, void *stream)
{
    if (!logits || !expert || !weight || !counts || !offsets || !n_routed || !loss) {
        set_error("fp8_moe_route: NULL pointer");
        return FP8_ERR_NULL;
    }
    int rc = route_check("fp8_moe_route", T, E, k, balance_coef, z_coef);
    if (rc != FP8_OK) return rc;
    if (!aligned16(logits) || !aligned16(expert) || !aligned16(weight)) {
        set_error("fp8_moe_route: tensor pointers must be 16-byte aligned");
        return FP8_ERR_ALIGN;
    }
    const size_t need = fp8_moe_route_workspace_bytes(T, E);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("fp8_moe_route: workspace of %zu bytes, 256-byte aligned, needed (got %zu)", need, ws_bytes);
        return FP8_ERR_WORKSPACE;
    }
    rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    RouteParams q = {};
    q.logits = logits; q.bias = bias; q.T = T; q.chunk = route_chunk(T); q.E = E; q.k = k; q.normalize = normalize ? 1 : 0;
    q.balance_coef = balance_coef; q.z_coef = z_coef;
    q.expert = expert; q.weight = weight; q.counts = counts; q.offsets = offsets; q.rows = rows; q.n_routed = n_routed;
    q.loss = loss;
    q.ctas = (int)route_ctas(T);
    q.cta_counts = static_cast<int *>(ws);
    q.cta_probs = reinterpret_cast<float *>(q.cta_counts + (size_t)q.ctas * E);
    q.cta_z = reinterpret_cast<double *>(q.cta_probs + (size_t)q.ctas * E);
    q.cta_n = reinterpret_cast<int *>(q.cta_z + q.ctas);
    FP8DPA_ROUTE_DISPATCH(route_choose_kernel, q.ctas);
    FP8_CUDA_CHECK(cudaGetLastError());
    route_place_kernel<<<rows ? q.ctas : 1, RT_THREADS, 0, st>>>(q);
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
}

extern "C" int fp8_moe_route_bwd(const void *logits, int is_fp32, const int *expert, const int *counts, const int *n_routed,
                                 size_t T, int E, int k, int normalize, float balance_coef, float z_coef,
                                 const float *dloss, const float *dweight, void *dlogits, void *stream)
{
    if (!logits || !counts || !n_routed || !dlogits || (dweight && !expert)) {
        set_error("fp8_moe_route_bwd: NULL pointer");
        return FP8_ERR_NULL;
    }
    int rc = route_check("fp8_moe_route_bwd", T, E, k, balance_coef, z_coef);
    if (rc != FP8_OK) return rc;
    if (!aligned16(logits) || !aligned16(expert) || !aligned16(dweight) || !aligned16(dlogits)) {
        set_error("fp8_moe_route_bwd: tensor pointers must be 16-byte aligned");
        return FP8_ERR_ALIGN;
    }
    rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    RouteParams q = {};
    q.logits = logits; q.T = T; q.E = E; q.k = k; q.normalize = normalize ? 1 : 0;
    q.balance_coef = balance_coef; q.z_coef = z_coef;
    q.expert = const_cast<int *>(expert); q.counts_in = counts; q.n_in = n_routed; q.dloss = dloss; q.dweight = dweight;
    q.dlogits = dlogits;
    const size_t groups = E <= 8 ? 32 : E <= 16 ? 16 : 8;
    size_t blocks = (T + groups - 1) / groups;
    const size_t cap = (size_t)sm_count() * 8;
    if (blocks > cap) blocks = cap;
    FP8DPA_ROUTE_DISPATCH(route_bwd_kernel, (unsigned)blocks);
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
}
