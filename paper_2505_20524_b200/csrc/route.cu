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

constexpr int RT_THREADS = 1024;     // of the forward kernels
constexpr int RT_WARPS = RT_THREADS / 32;
constexpr int RT_BWD_THREADS = 256;
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

// order-preserving map of binary32 (no NaN) to unsigned; -inf maps to KEY_NEG_INF
__device__ __forceinline__ uint32_t float_key(float f)
{
    const uint32_t b = __float_as_uint(f + 0.0f);                 // -0 becomes +0: equal values, equal keys
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_float(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k); }
constexpr uint32_t KEY_NEG_INF = 0x007FFFFFu;

template <bool F32>
__device__ __forceinline__ float load_logit(const void *p, size_t i)
{
    if (F32) return __ldg(static_cast<const float *>(p) + i);
    return __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t *>(p) + i) << 16);
}

// PL consecutive logits from index i (`there` of them inside the row, -inf behind); one vector load where the row's length is
// a multiple of PL
template <bool F32, int PL>
__device__ __forceinline__ void load_logits(const void *p, size_t i, int there, bool vec, float (&l)[PL])
{
    if (vec && there >= PL) {
        if (F32) {
            const float *q = static_cast<const float *>(p) + i;
            if constexpr (PL % 4 == 0) {
#pragma unroll
                for (int j = 0; j < PL / 4; ++j) {
                    const float4 v = __ldg(reinterpret_cast<const float4 *>(q) + j);
                    l[4 * j] = v.x; l[4 * j + 1] = v.y; l[4 * j + 2] = v.z; l[4 * j + 3] = v.w;
                }
            } else if constexpr (PL == 2) {
                const float2 v = __ldg(reinterpret_cast<const float2 *>(q));
                l[0] = v.x; l[1] = v.y;
            } else {
                l[0] = __ldg(q);
            }
        } else {
            const uint16_t *q = static_cast<const uint16_t *>(p) + i;
            uint32_t w[(PL + 1) / 2];
            if constexpr (PL % 8 == 0) {
#pragma unroll
                for (int j = 0; j < PL / 8; ++j) {
                    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(q) + j);
                    w[4 * j] = v.x; w[4 * j + 1] = v.y; w[4 * j + 2] = v.z; w[4 * j + 3] = v.w;
                }
            } else if constexpr (PL == 4) {
                const uint2 v = __ldg(reinterpret_cast<const uint2 *>(q));
                w[0] = v.x; w[1] = v.y;
            } else if constexpr (PL == 2) {
                w[0] = __ldg(reinterpret_cast<const uint32_t *>(q));
            } else {
                w[0] = __ldg(q);
            }
#pragma unroll
            for (int j = 0; j < PL; ++j) l[j] = j & 1 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < PL; ++j) l[j] = j < there ? load_logit<F32>(p, i + j) : -INFINITY;
}

// all-lane reductions over the G = 1 or 32 lanes that share a token
template <int G> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int G> __device__ __forceinline__ uint32_t group_max_u(uint32_t v)
{
    return G == 1 ? v : __reduce_max_sync(0xffffffffu, v);
}

// What both passes need of a token: its logits (lane gl of the token's G holds the experts gl PL ... gl PL + PL - 1), whether
// it is routed (a finite logit, nothing NaN or +inf), whether it is broken (NaN or +inf), the maximum, the sum of exponentials
// and the probabilities.
template <int G, int PL>
struct Token {
    float l[PL], p[PL];
    float top, total, inv;
    bool routed, broken;

    __device__ __forceinline__ void finish(int E, int gl)
    {
        uint32_t mx = 0u;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            const bool b = !(l[i] < INFINITY);
            bad |= b;
            mx = max(mx, b ? 0u : float_key(l[i]));
        }
        mx = group_max_u<G>(mx);
        broken = G == 1 ? bad : __any_sync(0xffffffffu, bad);
        routed = !broken && mx > KEY_NEG_INF;
        top = key_float(mx);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            p[i] = routed ? expf(l[i] - top) : 0.0f;
            s += p[i];
        }
        total = group_sum<G>(s);
        inv = routed ? 1.0f / total : broken ? NAN : 0.0f;
#pragma unroll
        for (int i = 0; i < PL; ++i) p[i] = broken ? (gl * PL + i < E ? inv : 0.0f) : p[i] * inv;
    }
    __device__ __forceinline__ float lse() const { return broken ? NAN : routed ? top + logf(total) : 0.0f; }
};

// The lane's best score and its (lowest) place
template <int PL>
__device__ __forceinline__ void local_best(const uint32_t (&key)[PL], uint32_t &best, int &at)
{
    best = key[0];
    at = 0;
#pragma unroll
    for (int i = 1; i < PL; ++i)
        if (key[i] > best) {
            best = key[i];
            at = i;
        }
}

// Forward, first kernel.  G lanes per token (1 up to 16 experts, a warp above), PL experts per lane; the tokens of the CTA's
// chunk go to the groups in turn.  Bound by latency: the k maxima of a token follow one another, one warp reduction each
// (16411 tokens of 160 experts, k = 6: 55.8 us with five shuffles per maximum and 8 warps per SM).
template <bool F32, int G, int PL>
__global__ void __launch_bounds__(RT_THREADS) route_choose_kernel(const RouteParams q)
{
    constexpr int GROUPS = RT_THREADS / G;
    constexpr int SLOTS = G == 1 ? PL : 1;            // slots a lane holds: all (k <= E <= PL), or the slot of its number
    __shared__ int cnt[RT_MAX_E];
    __shared__ float probs[RT_WARPS][G * PL];
    __shared__ double zsum[RT_WARPS];
    __shared__ int nsum[RT_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gl = G == 1 ? 0 : lane, group = tid / G;
    for (int e = tid; e < q.E; e += RT_THREADS) cnt[e] = 0;
    __syncthreads();
    float ps[PL], bias[PL];
    double z = 0.0;
    int n = 0;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        ps[i] = 0.0f;
        bias[i] = q.bias && gl * PL + i < q.E ? __ldg(q.bias + gl * PL + i) : 0.0f;
    }
    const bool vec = q.E % PL == 0;
    const size_t t0 = blockIdx.x * q.chunk, t1 = min(q.T, t0 + q.chunk);
    Token<G, PL> tok;
    float next[PL];
    load_logits<F32>(q.logits, (t0 + group) * q.E + gl * PL, t0 + group < t1 ? q.E - gl * PL : 0, vec, next);
    for (size_t base = t0; base < t1; base += GROUPS) {
        const size_t t = base + group;
        const bool live = t < t1;
#pragma unroll
        for (int i = 0; i < PL; ++i) tok.l[i] = next[i];
        load_logits<F32>(q.logits, (t + GROUPS) * q.E + gl * PL, t + GROUPS < t1 ? q.E - gl * PL : 0, vec, next);
        tok.finish(q.E, gl);
#pragma unroll
        for (int i = 0; i < PL; ++i) ps[i] += tok.p[i];
        const double lse = (double)tok.lse();
        const bool counted = gl == 0 && (tok.routed || tok.broken);
        z = counted ? fma(lse, lse, z) : z;
        n += counted ? 1 : 0;
        // the k largest scores, one maximum at a time; equal scores: the lowest expert
        uint32_t key[PL], best;
        int at;
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            const float s = tok.l[i] + bias[i];
            const uint32_t k32 = tok.routed && s == s ? float_key(s) : 0u;
            key[i] = k32 > KEY_NEG_INF ? k32 : 0u;
        }
        local_best(key, best, at);
        int we[SLOTS];
        float wl[SLOTS];
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
            we[j] = -1;
            wl[j] = -INFINITY;
        }
        if (G == 1) {
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) {
                if (j >= q.k) break;
                if (best) {
                    we[j] = at;
#pragma unroll
                    for (int i = 0; i < PL; ++i)
                        if (i == at) {
                            wl[j] = tok.l[i];
                            key[i] = 0u;
                        }
                    local_best(key, best, at);
                }
            }
        } else {
            for (int j = 0; j < q.k; ++j) {
                const uint32_t m = group_max_u<G>(best);
                const int src = __ffs(__ballot_sync(0xffffffffu, best == m)) - 1;
                const int e = __shfl_sync(0xffffffffu, gl * PL + at, src);
                if (lane == j) we[0] = m ? e : -1;
                if (m == 0u) break;
                if (lane == src) {
#pragma unroll
                    for (int i = 0; i < PL; ++i)
                        if (i == at) key[i] = 0u;
                    local_best(key, best, at);
                }
            }
            if (we[0] >= 0) wl[0] = load_logit<F32>(q.logits, t * q.E + we[0]);
        }
        float high = tok.top, inv = tok.inv;              // of the softmax that the weights are taken from
        if (q.normalize) {
            uint32_t h = 0u;
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) h = max(h, we[j] >= 0 ? float_key(wl[j]) : 0u);
            h = group_max_u<G>(h);
            high = key_float(h);
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) s += we[j] >= 0 ? expf(wl[j] - high) : 0.0f;
            s = group_sum<G>(s);
            inv = h ? 1.0f / s : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
            const int slot = G == 1 ? j : lane;
            if (live && slot < q.k) {
                q.expert[t * q.k + slot] = we[j];
                q.weight[t * q.k + slot] = tok.broken ? NAN : we[j] < 0 ? 0.0f : expf(wl[j] - high) * inv;
                if (we[j] >= 0) atomicAdd(&cnt[we[j]], 1);
            }
        }
    }
    // sums over the tokens of a warp (one lane each, if G = 1), then over the warps in order
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        if (G == 1) ps[i] = group_sum<32>(ps[i]);
        if (G == 32 || lane == 0) probs[warp][gl * PL + i] = ps[i];
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
    if (warp == RT_WARPS - 1) {
        z = zsum[lane];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        n = __reduce_add_sync(0xffffffffu, nsum[lane]);
        if (lane == 0) {
            q.cta_z[blockIdx.x] = z;
            q.cta_n[blockIdx.x] = n;
        }
    }
}

// Forward, second kernel.  Every CTA sums the chunks' counts per expert (RT_THREADS / E' threads per expert, E' the power of
// two that holds E) and places the rows of its chunk behind those of the chunks before it.  One more CTA, the last, writes
// counts, offsets, the token count and the losses.  All clear the rows behind the last used one.
__global__ void __launch_bounds__(RT_THREADS) route_place_kernel(const RouteParams q, int e_log2)
{
    __shared__ int warp_cnt[RT_WARPS][RT_MAX_E];
    __shared__ int part[2][RT_THREADS];
    __shared__ int base[RT_MAX_E], warp_sum[RT_MAX_E / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int slices = RT_THREADS >> e_log2, slice = tid >> e_log2, expert = tid & ((1 << e_log2) - 1);
    const bool stats = blockIdx.x == gridDim.x - 1;        // without rows it is the only one
    int total = 0, mine = 0;
    if (expert < q.E) {
#pragma unroll 8
        for (int c = slice; c < q.ctas; c += slices) {
            const int v = __ldcg(q.cta_counts + (size_t)c * q.E + expert);
            if (c < (int)blockIdx.x) mine += v;
            total += v;
        }
    }
    part[0][tid] = total;
    part[1][tid] = mine;
    if (!stats)
        for (int i = tid; i < RT_WARPS * RT_MAX_E; i += RT_THREADS) warp_cnt[i / RT_MAX_E][i % RT_MAX_E] = 0;
    __syncthreads();
    int scan = 0;
    total = mine = 0;
    if (tid < RT_MAX_E) {
        if (tid < 1 << e_log2) {
            for (int s = 0; s < slices; ++s) {
                total += part[0][(s << e_log2) + tid];
                mine += part[1][(s << e_log2) + tid];
            }
        }
        scan = total;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += v;
        }
        if (lane == 31) warp_sum[warp] = scan;
    }
    __syncthreads();
    int start = scan - total, all = 0;
#pragma unroll
    for (int w = 0; w < RT_MAX_E / 32; ++w) {
        if (w < warp) start += warp_sum[w];
        all += warp_sum[w];
    }
    if (tid < RT_MAX_E) base[tid] = start + mine;
    if (stats) {
        double *dred = reinterpret_cast<double *>(&warp_cnt[0][0]);          // [RT_THREADS], then [RT_WARPS] twice
        double p = 0.0, z = 0.0, f = 0.0;
        int n = 0;
        if (expert < q.E) {
#pragma unroll 8
            for (int c = slice; c < q.ctas; c += slices) p += (double)__ldcg(q.cta_probs + (size_t)c * q.E + expert);
        }
        dred[tid] = p;
        for (int c = tid; c < q.ctas; c += RT_THREADS) {
            n += __ldcg(q.cta_n + c);
            z += __ldcg(q.cta_z + c);
        }
        __syncthreads();
        if (tid < q.E) {
            for (int s = 1; s < slices; ++s) p += dred[(s << e_log2) + tid];
            f = (double)total * p;
            q.counts[tid] = total;
            q.offsets[tid] = start;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            z += __shfl_xor_sync(0xffffffffu, z, o);
            f += __shfl_xor_sync(0xffffffffu, f, o);
        }
        n = __reduce_add_sync(0xffffffffu, n);
        double *zred = dred + RT_THREADS, *fred = zred + RT_WARPS;
        if (lane == 0) {
            zred[warp] = z;
            fred[warp] = f;
            part[0][warp] = n;
        }
        __syncthreads();
        if (tid == 0) {
            z = f = 0.0;
            n = 0;
            for (int w = 0; w < RT_WARPS; ++w) {
                z += zred[w];
                f += fred[w];
                n += part[0][w];
            }
            const double dn = (double)n;
            q.offsets[q.E] = all;
            *q.n_routed = n;
            q.loss[0] = n ? (float)((double)q.balance_coef * q.E * f / (dn * dn * q.k)) : 0.0f;
            q.loss[1] = n ? (float)((double)q.z_coef * z / dn) : 0.0f;
        }
        return;
    }
    const size_t copies = q.T * q.k;
    for (size_t i = (size_t)all + blockIdx.x * RT_THREADS + tid; i < copies; i += (size_t)q.ctas * RT_THREADS) q.rows[i] = -1;
    const size_t i0 = blockIdx.x * q.chunk * q.k, i1 = min(copies, i0 + q.chunk * q.k);
    for (size_t tile = i0; tile < i1; tile += RT_THREADS) {
        if (tile != i0) {
            for (int i = tid; i < RT_WARPS * RT_MAX_E; i += RT_THREADS) warp_cnt[i / RT_MAX_E][i % RT_MAX_E] = 0;
        }
        __syncthreads();
        const size_t i = tile + tid;
        const int e = i < i1 ? __ldcg(q.expert + i) : -1;
        const int rank = warp_stable_rank(e, warp_cnt[warp], lane);
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
        if (e >= 0) q.rows[warp_cnt[warp][e] + rank] = (int)i;
        __syncthreads();
    }
}

// Backward: one pass over the logits, everything of a token in its lanes.
//   u_e = dloss * balance_coef * E * counts_e / (k n^2)  (+ dweight of e's slot, without normalisation)
//   dl_e = p_e (u_e - sum u p) + dloss * z_coef * 2 lse / n * p_e  (+ w_j (dw_j - sum dw w) in slot j, with normalisation)
template <bool F32, int G, int PL>
__global__ void __launch_bounds__(RT_BWD_THREADS) route_bwd_kernel(const RouteParams q)
{
    constexpr int GROUPS = RT_BWD_THREADS / G;
    constexpr int SLOTS = G == 1 ? PL : 1;
    const int lane = threadIdx.x & 31, gl = G == 1 ? 0 : lane, group = threadIdx.x / G;
    const float d = q.dloss ? __ldg(q.dloss) : 1.0f;
    const float n = (float)__ldg(q.n_in);
    const float ub = n > 0.0f ? d * q.balance_coef * (float)q.E / (n * n * (float)q.k) : 0.0f;
    const float uz = n > 0.0f ? d * q.z_coef * 2.0f / n : 0.0f;
    const bool vec = q.E % PL == 0;
    float u0[PL];
#pragma unroll
    for (int i = 0; i < PL; ++i) u0[i] = gl * PL + i < q.E ? ub * (float)__ldg(q.counts_in + gl * PL + i) : 0.0f;
    for (size_t base = (size_t)blockIdx.x * GROUPS; base < q.T; base += (size_t)gridDim.x * GROUPS) {
        const size_t t = base + group;
        const bool live = t < q.T;
        int se[SLOTS];
        float sd[SLOTS], sw[SLOTS];
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
            const int slot = G == 1 ? j : lane;
            se[j] = -1;
            sd[j] = 0.0f;
            if (q.dweight && live && slot < q.k) {
                se[j] = __ldg(q.expert + t * q.k + slot);
                sd[j] = __ldg(q.dweight + t * q.k + slot);
                if (se[j] < 0 || se[j] >= q.E) se[j] = -1;
            }
        }
        Token<G, PL> tok;
        load_logits<F32>(q.logits, t * q.E + gl * PL, live ? q.E - gl * PL : 0, vec, tok.l);
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) sw[j] = q.normalize && se[j] >= 0 ? load_logit<F32>(q.logits, t * q.E + se[j]) : -INFINITY;
        tok.finish(q.E, gl);
        float u[PL], add[PL];
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            u[i] = u0[i];
            add[i] = 0.0f;
        }
        if (q.dweight) {
            if (q.normalize) {
                uint32_t h = 0u;
#pragma unroll
                for (int j = 0; j < SLOTS; ++j) h = max(h, se[j] >= 0 && sw[j] < INFINITY ? float_key(sw[j]) : 0u);
                h = group_max_u<G>(h);
                const float high = key_float(h);
                float s = 0.0f, sdw = 0.0f;
#pragma unroll
                for (int j = 0; j < SLOTS; ++j) {
                    sw[j] = h && se[j] >= 0 ? expf(sw[j] - high) : 0.0f;
                    s += sw[j];
                }
                s = group_sum<G>(s);
                const float inv = s > 0.0f ? 1.0f / s : 0.0f;
#pragma unroll
                for (int j = 0; j < SLOTS; ++j) {
                    sw[j] *= inv;
                    sdw += se[j] >= 0 ? sd[j] * sw[j] : 0.0f;
                }
                sdw = group_sum<G>(sdw);
#pragma unroll
                for (int j = 0; j < SLOTS; ++j) sd[j] = sw[j] * (sd[j] - sdw);
            }
            if (G == 1) {
#pragma unroll
                for (int j = 0; j < SLOTS; ++j)
#pragma unroll
                    for (int i = 0; i < PL; ++i)
                        if (se[j] == i) {
                            if (q.normalize) add[i] += sd[j];
                            else u[i] += sd[j];
                        }
            } else {
                for (int j = 0; j < q.k; ++j) {
                    const int e = __shfl_sync(0xffffffffu, se[0], j);
                    const float v = __shfl_sync(0xffffffffu, sd[0], j);
#pragma unroll
                    for (int i = 0; i < PL; ++i)
                        if (e == gl * PL + i) {
                            if (q.normalize) add[i] += v;
                            else u[i] += v;
                        }
                }
            }
        }
        float up = 0.0f;
#pragma unroll
        for (int i = 0; i < PL; ++i) up = fmaf(u[i], tok.p[i], up);
        up = group_sum<G>(up);
        const float zz = tok.routed ? uz * tok.lse() : 0.0f;
        if (!live) continue;
        float g[PL];
#pragma unroll
        for (int i = 0; i < PL; ++i) g[i] = tok.broken ? NAN : fmaf(tok.p[i], (u[i] - up) + zz, add[i]);
        const size_t at = t * q.E + gl * PL;
        const int there = q.E - gl * PL;
        if (F32) {
            float *o = static_cast<float *>(q.dlogits) + at;
            if (PL % 4 == 0 && vec && there >= PL) {
#pragma unroll
                for (int i = 0; i + 3 < PL; i += 4) *reinterpret_cast<float4 *>(o + i) = make_float4(g[i], g[i + 1], g[i + 2], g[i + 3]);
            } else {
#pragma unroll
                for (int i = 0; i < PL; ++i)
                    if (i < there) o[i] = g[i];
            }
        } else {
            uint16_t *o = static_cast<uint16_t *>(q.dlogits) + at;
            if (PL % 8 == 0 && vec && there >= PL) {
#pragma unroll
                for (int i = 0; i + 7 < PL; i += 8)
                    *reinterpret_cast<uint4 *>(o + i) = make_uint4(pack_bf16x2(g[i], g[i + 1]), pack_bf16x2(g[i + 2], g[i + 3]),
                                                                   pack_bf16x2(g[i + 4], g[i + 5]), pack_bf16x2(g[i + 6], g[i + 7]));
            } else {
#pragma unroll
                for (int i = 0; i < PL; ++i)
                    if (i < there) o[i] = (uint16_t)(pack_bf16x2(g[i], g[i]) & 0xFFFFu);
            }
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

#define FP8DPA_ROUTE_DISPATCH(KERNEL, GRID, THREADS)                                 \
    do {                                                                             \
        if (q.E <= 8) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 1, 8);                \
        else if (q.E <= 16) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 1, 16);         \
        else if (q.E <= 32) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 32, 1);         \
        else if (q.E <= 64) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 32, 2);         \
        else if (q.E <= 128) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 32, 4);        \
        else FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 32, 8);                        \
    } while (0)
#define FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, G, PL)                              \
    do {                                                                             \
        if (is_fp32) KERNEL<true, G, PL><<<GRID, THREADS, 0, st>>>(q);               \
        else KERNEL<false, G, PL><<<GRID, THREADS, 0, st>>>(q);                      \
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
    FP8DPA_ROUTE_DISPATCH(route_choose_kernel, q.ctas, RT_THREADS);
    FP8_CUDA_CHECK(cudaGetLastError());
    int e_log2 = 0;
    while ((1 << e_log2) < E) ++e_log2;
    route_place_kernel<<<rows ? q.ctas + 1 : 1, RT_THREADS, 0, st>>>(q, e_log2);
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
    const size_t groups = E <= 16 ? RT_BWD_THREADS : RT_BWD_THREADS / 32;
    size_t blocks = (T + groups - 1) / groups;
    const size_t cap = (size_t)sm_count() * 8;
    if (blocks > cap) blocks = cap;
    FP8DPA_ROUTE_DISPATCH(route_bwd_kernel, (unsigned)blocks, RT_BWD_THREADS);
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
}
