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
constexpr size_t RT_MAX_CHUNKS = 147;    // one CTA per SM in the second kernel, whose last CTA has no chunk

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
    int *cta_counts;                 // [CTAs][stride]
    float *cta_probs;                // [CTAs][stride]
    int stride;                      // E rounded up to 4: rows are read four experts at a time
    double *cta_z;                   // [CTAs]: sum of lse^2 (a row of the type's lowest value has lse^2 beyond FP32)
    int *cta_n;                      // [CTAs]: routed tokens
    int ctas;
    const int *n_in, *counts_in;     // backward
    const float *dloss, *dweight;
    void *dlogits;
};

template <bool F32>
__device__ __forceinline__ float load_logit(const void *p, size_t i)
{
    if (F32) return __ldg(static_cast<const float *>(p) + i);
    return __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t *>(p) + i) << 16);
}

// A token's logits in its G = 1 or 32 lanes: lane gl holds the experts gl, gl + G, ... (-inf behind the row's end).  One lane
// reads its whole row with vector loads where the row's length allows it.
template <bool F32, int G, int PL>
__device__ __forceinline__ void load_logits(const void *p, size_t t, int E, int gl, bool live, float (&l)[PL])
{
    if constexpr (G == 1) {
        if (live && E == PL) {
#pragma unroll
            for (int j = 0; j < PL / 8; ++j) {
                if (F32) {
                    const float4 *q = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + t * PL + 8 * j);
                    const float4 v = __ldg(q), w = __ldg(q + 1);
                    l[8 * j] = v.x; l[8 * j + 1] = v.y; l[8 * j + 2] = v.z; l[8 * j + 3] = v.w;
                    l[8 * j + 4] = w.x; l[8 * j + 5] = w.y; l[8 * j + 6] = w.z; l[8 * j + 7] = w.w;
                } else {
                    const uint4 v = __ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + t * PL + 8 * j));
                    l[8 * j] = bf16_lo(v.x); l[8 * j + 1] = bf16_hi(v.x); l[8 * j + 2] = bf16_lo(v.y); l[8 * j + 3] = bf16_hi(v.y);
                    l[8 * j + 4] = bf16_lo(v.z); l[8 * j + 5] = bf16_hi(v.z); l[8 * j + 6] = bf16_lo(v.w); l[8 * j + 7] = bf16_hi(v.w);
                }
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < PL; ++i) l[i] = live && i * G + gl < E ? load_logit<F32>(p, t * E + i * G + gl) : -INFINITY;
}

// all-lane reductions over a token's lanes
template <int G> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int G> __device__ __forceinline__ float group_max(float v)
{
    if (G == 1) return v;
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// exp(x) for x <= 0 from the hardware's exp2 (relative error 2^-22).  The rounding of t = x log2 e, and of log2 e itself, moves
// the result by up to 1.5 |x| 2^-24 of itself: x - t ln 2, which one fma leaves with |x| 2^-28, is put back to first order.
// Results below 2^-126 are 0; -200 in place of -inf keeps the correction a number.
__device__ __forceinline__ float exp_neg(float x)
{
    x = fmaxf(x, -200.0f);
    const float t = x * 1.4426950408889634f, e = ex2_approx(t);
    return fmaf(e, fmaf(t, -0.6931471805599453f, x), e);
}

// What both passes need of a token: whether it is routed (a finite logit, nothing NaN or +inf), whether it is broken (NaN or
// +inf), the maximum, the sum of exponentials and the probabilities.
template <int G, int PL>
struct Token {
    float l[PL], p[PL];
    float top, total, inv;
    bool routed, broken;

    __device__ __forceinline__ void finish()
    {
        float mx = l[0];                                   // NaN if a logit is
#pragma unroll
        for (int i = 1; i < PL; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(mx) : "f"(l[i]));
        if (G > 1) asm volatile("redux.sync.max.NaN.f32 %0, %0, 0xffffffff;" : "+f"(mx));
        top = mx;
        broken = !(top < INFINITY);
        routed = !broken && top > -INFINITY;
        const float from = routed ? top : 0.0f;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            p[i] = exp_neg(l[i] - from);
            s += p[i];
        }
        total = group_sum<G>(s);
        inv = routed ? 1.0f / total : broken ? NAN : 0.0f;
#pragma unroll
        for (int i = 0; i < PL; ++i) p[i] *= inv;          // NaN in a broken token, behind the last expert too
    }
    __device__ __forceinline__ float lse() const { return broken ? NAN : routed ? top + logf(total) : 0.0f; }
};

// The lane's best score and its first place
template <int PL>
__device__ __forceinline__ void local_best(const float (&score)[PL], float &best, int &at)
{
    best = score[0];
    at = 0;
#pragma unroll
    for (int i = 1; i < PL; ++i)
        if (score[i] > best) {
            best = score[i];
            at = i;
        }
}

template <int PL>
__device__ __forceinline__ void without(float (&score)[PL], int at)
{
#pragma unroll
    for (int i = 0; i < PL; ++i)
        if (i == at) score[i] = -INFINITY;
}

// Forward, first kernel.  G lanes per token (1, or a warp), PL experts per lane; the tokens of the CTA's
// chunk go to the groups in turn.  Bound by instruction issue and by the latency of the k maxima, which follow one another:
// two warp reductions each (the largest score, the lowest expert that has it).
struct ChooseShared {
    int cnt[RT_MAX_E], nsum[RT_WARPS];
    double zsum[RT_WARPS];
};
template <bool F32, int G, int PL>
__device__ __forceinline__ void route_choose(const RouteParams &q, ChooseShared &sh, float (*probs)[G * PL])
{
    constexpr int SLOTS = G == 1 ? PL : 1;            // slots a lane holds: all (k <= E <= PL), or the slot of its number
    int *cnt = sh.cnt, *nsum = sh.nsum;
    double *zsum = sh.zsum;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gl = G == 1 ? 0 : lane, group = tid / G;
    const int warps = blockDim.x >> 5, groups = blockDim.x / G;
    for (int e = tid; e < q.E; e += blockDim.x) cnt[e] = 0;
    __syncthreads();
    float ps[PL], bias[PL], next[PL];
    double z = 0.0;
    int n = 0;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        ps[i] = 0.0f;
        bias[i] = q.bias && i * G + gl < q.E ? __ldg(q.bias + i * G + gl) : 0.0f;
    }
    const size_t t0 = blockIdx.x * q.chunk, t1 = min(q.T, t0 + q.chunk);
    load_logits<F32, G, PL>(q.logits, t0 + group, q.E, gl, t0 + group < t1, next);
    for (size_t first = t0; first < t1; first += groups) {
        const size_t t = first + group;
        const bool live = t < t1;
        Token<G, PL> tok;
#pragma unroll
        for (int i = 0; i < PL; ++i) tok.l[i] = next[i];
        load_logits<F32, G, PL>(q.logits, t + groups, q.E, gl, t + groups < t1, next);
        tok.finish();
#pragma unroll
        for (int i = 0; i < PL; ++i) ps[i] += tok.p[i];
        const double lse = (double)tok.lse();
        const bool counted = gl == 0 && (tok.routed || tok.broken);
        z = counted ? fma(lse, lse, z) : z;
        n += counted ? 1 : 0;
        // the k largest scores, one maximum at a time; equal scores: the lowest expert; -inf and NaN are no scores
        float score[PL], best;
        int at;
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            const float s = tok.l[i] + bias[i];
            score[i] = tok.routed && s == s ? s : -INFINITY;
        }
        local_best(score, best, at);
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
                if (j < q.k && best > -INFINITY) {
                    we[j] = at;
#pragma unroll
                    for (int i = 0; i < PL; ++i)
                        if (i == at) {
                            wl[j] = tok.l[i];
                            score[i] = -INFINITY;
                        }
                    local_best(score, best, at);
                }
            }
        } else {
            // A lane keeps its best two: the winner's second moves up at once, and only one that wins again looks at its
            // scores once more (8 of 256 for 32768 tokens: 25.4 us; 31.4 with a look after every win, which the warp waits for).
            float second = -INFINITY;
            int at2 = -1;
            if (PL > 1) {
                without(score, at);
                local_best(score, second, at2);
            }
            bool spent = false;                            // the second has moved up
            for (int j = 0; j < q.k; ++j) {
                const float m = group_max<G>(best);
                const int mine = at * G + gl;
                const int e = (int)__reduce_min_sync(0xffffffffu, best == m && m > -INFINITY ? (unsigned)mine : 0xFFFFFFFFu);
                if (lane == j) we[0] = e;                  // -1: no score left
                if (e == mine) {
                    if (PL == 1) {
                        best = -INFINITY;
                    } else if (PL > 2 && spent) {
                        without(score, at);
                        local_best(score, best, at);
                    } else {
                        best = spent ? -INFINITY : second;
                        at = at2;
                        spent = true;
                    }
                }
            }
            if (we[0] >= 0) wl[0] = load_logit<F32>(q.logits, t * q.E + we[0]);
        }
        float high = tok.top, inv = tok.inv;              // of the softmax that the weights are taken from
        if (q.normalize) {
            float h = -INFINITY;
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) h = fmaxf(h, wl[j]);
            high = group_max<G>(h);
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) s += we[j] >= 0 ? exp_neg(wl[j] - high) : 0.0f;
            s = group_sum<G>(s);
            inv = 1.0f / s;                                // of a token without a choice: not used
        }
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
            const int slot = G == 1 ? j : lane;
            if (live && slot < q.k) {
                q.expert[t * q.k + slot] = we[j];
                q.weight[t * q.k + slot] = tok.broken ? NAN : we[j] < 0 ? 0.0f : exp_neg(wl[j] - high) * inv;
                if (we[j] >= 0) atomicAdd(&cnt[we[j]], 1);
            }
        }
    }
    // sums over the tokens of a warp (one lane each, if G = 1), then over the warps in order
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        if (G == 1) ps[i] = group_sum<32>(ps[i]);
        if (G == 32 || lane == 0) probs[warp][i * G + gl] = ps[i];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) {
        zsum[warp] = z;
        nsum[warp] = n;
    }
    __syncthreads();
    for (int e = tid; e < q.E; e += blockDim.x) {
        float s = probs[0][e];
#pragma unroll
        for (int w = 1; w < RT_WARPS; ++w)
            if (w < warps) s += probs[w][e];
        q.cta_probs[(size_t)blockIdx.x * q.stride + e] = s;
        q.cta_counts[(size_t)blockIdx.x * q.stride + e] = cnt[e];
    }
    if (warp == warps - 1) {
        z = lane < warps ? zsum[lane] : 0.0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        n = __reduce_add_sync(0xffffffffu, lane < warps ? nsum[lane] : 0);
        if (lane == 0) {
            q.cta_z[blockIdx.x] = z;
            q.cta_n[blockIdx.x] = n;
        }
    }
}
template <bool F32, int G, int PL>
__global__ void __launch_bounds__(G == 1 ? 512 : RT_THREADS) route_choose_kernel(const RouteParams q)
{
    __shared__ ChooseShared sh;
    __shared__ float probs[RT_WARPS][G * PL];
    cudaTriggerProgrammaticLaunchCompletion();
    route_choose<F32, G, PL>(q, sh, probs);
}

// Forward, second kernel.  Every CTA sums the chunks' counts per expert (a thread four experts of every `slices`-th chunk) and
// places the rows of its chunk behind those of the chunks before it.  One more CTA, the last, writes counts, offsets, the
// token count and the losses.  All clear the rows behind the last used one.
struct PlaceShared {
    __align__(16) int warp_cnt[RT_WARPS][RT_MAX_E];       // before that: [2][slices][E' = 4 << quads_log2]
    int base[RT_MAX_E], warp_sum[RT_MAX_E / 32], nred[RT_WARPS];
    double zred[RT_WARPS], fred[RT_WARPS];
};
__device__ __forceinline__ void route_place(const RouteParams &q, int quads_log2, int slices, PlaceShared &sh)
{
    auto &warp_cnt = sh.warp_cnt;
    int *base = sh.base, *warp_sum = sh.warp_sum;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int slice = tid >> quads_log2, quad = tid & ((1 << quads_log2) - 1), e_pad = 4 << quads_log2;
    const bool stats = blockIdx.x == gridDim.x - 1;        // without rows it is the only one
    const size_t copies = q.T * q.k, i0 = blockIdx.x * q.chunk * q.k, i1 = min(copies, i0 + q.chunk * q.k);
    int e = !stats && i0 + tid < i1 ? __ldcg(q.expert + i0 + tid) : -1;       // the first tile's, on its way meanwhile
    if (slice < slices) {
        int4 total = make_int4(0, 0, 0, 0), mine = total;
        float4 prob = make_float4(0.f, 0.f, 0.f, 0.f);
        if (4 * quad < q.stride) {
#pragma unroll 10
            for (int c = slice; c < q.ctas; c += slices) {
                const int4 v = __ldcg(reinterpret_cast<const int4 *>(q.cta_counts + (size_t)c * q.stride) + quad);
                const int before = c < (int)blockIdx.x ? -1 : 0;
                mine.x += v.x & before; mine.y += v.y & before; mine.z += v.z & before; mine.w += v.w & before;
                total.x += v.x; total.y += v.y; total.z += v.z; total.w += v.w;
                if (stats) {
                    const float4 w = __ldcg(reinterpret_cast<const float4 *>(q.cta_probs + (size_t)c * q.stride) + quad);
                    prob.x += w.x; prob.y += w.y; prob.z += w.z; prob.w += w.w;
                }
            }
        }
        int4 *part = reinterpret_cast<int4 *>(&warp_cnt[0][0]) + ((size_t)slice << quads_log2) + quad;
        part[0] = total;
        if (stats) reinterpret_cast<float4 *>(part)[slices << quads_log2] = prob;
        else part[slices << quads_log2] = mine;
    }
    __syncthreads();
    int scan = 0, total = 0, mine = 0;
    double prob = 0.0;
    if (tid < RT_MAX_E) {
        if (tid < q.E) {
            const int *part = &warp_cnt[0][0] + tid;
#pragma unroll 16
            for (int s = 0; s < slices; ++s) {
                total += part[s * e_pad];
                const int v = part[(slices + s) * e_pad];
                if (stats) prob += (double)__int_as_float(v);
                else mine += v;
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
        if (tid < q.E) {
            q.counts[tid] = total;
            q.offsets[tid] = start;
        }
        double f = (double)total * prob, z = tid < q.ctas ? __ldcg(q.cta_z + tid) : 0.0;      // RT_MAX_CHUNKS at most
        int n = tid < q.ctas ? __ldcg(q.cta_n + tid) : 0;
#pragma unroll
        for (int round = 0; round < 2; ++round) {          // over the warp's lanes, then over the warps
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                z += __shfl_xor_sync(0xffffffffu, z, o);
                f += __shfl_xor_sync(0xffffffffu, f, o);
            }
            n = __reduce_add_sync(0xffffffffu, n);
            if (round == 0) {
                if (lane == 0) {
                    sh.zred[warp] = z;
                    sh.fred[warp] = f;
                    sh.nred[warp] = n;
                }
                __syncthreads();
                z = sh.zred[lane];
                f = sh.fred[lane];
                n = sh.nred[lane];
            }
        }
        if (tid == 0) {
            const double dn = (double)n;
            q.offsets[q.E] = all;
            *q.n_routed = n;
            q.loss[0] = n ? (float)((double)q.balance_coef * q.E * f / (dn * dn * q.k)) : 0.0f;
            q.loss[1] = n ? (float)((double)q.z_coef * z / dn) : 0.0f;
        }
        return;
    }
    for (size_t i = (size_t)all + blockIdx.x * RT_THREADS + tid; i < copies; i += (size_t)q.ctas * RT_THREADS) q.rows[i] = -1;
    for (size_t tile = i0; tile < i1; tile += RT_THREADS) {
        for (int i = lane; i < q.E; i += 32) warp_cnt[warp][i] = 0;        // a warp's own counters
        __syncwarp();
        const size_t i = tile + tid;
        if (tile != i0) e = i < i1 ? __ldcg(q.expert + i) : -1;
        const int rank = warp_stable_rank(e, quads_log2 + 2, warp_cnt[warp], lane);
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
        __syncwarp();
    }
}

__global__ void __launch_bounds__(RT_THREADS) route_place_kernel(const RouteParams q, int quads_log2, int slices)
{
    __shared__ PlaceShared sh;
    cudaGridDependencySynchronize();
    route_place(q, quads_log2, slices, sh);
}

// Few tokens: both kernels in one, a cluster of up to RT_CLUSTER CTAs (the last one has no chunk), with a cluster barrier where
// the second waits for the first.  A call of 1 to 224 tokens and 8 experts costs the host 10.6 us with its binding, 13.7 with two
// launches; the device takes 6.4 to 6.9 either way.
constexpr unsigned RT_CLUSTER = 8;
template <bool F32, int PL>
__global__ void __launch_bounds__(RT_THREADS) route_cluster_kernel(const RouteParams q, int quads_log2, int slices)
{
    __shared__ ChooseShared choose;
    __shared__ PlaceShared place;
    static_assert(sizeof(float) * 32 * PL <= sizeof(place.warp_cnt[0]), "the probabilities of a warp");
    const bool last = blockIdx.x == gridDim.x - 1;
    if (!last) route_choose<F32, 32, PL>(q, choose, reinterpret_cast<float(*)[32 * PL]>(&place.warp_cnt[0][0]));
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    if (q.rows || last) route_place(q, quads_log2, slices, place);
}

// Backward: one pass over the logits, everything of a token in its lanes.  Bound by instruction issue.
//   u_e = dloss * balance_coef * E * counts_e / (k n^2)  (+ dweight of e's slot, without normalisation)
//   dl_e = p_e (u_e - sum u p) + dloss * z_coef * 2 lse / n * p_e  (+ w_j (dw_j - sum dw w) in slot j, with normalisation)
template <bool F32, int G, int PL>
__global__ void __launch_bounds__(RT_BWD_THREADS, G == 1 ? 2 : 5) route_bwd_kernel(const RouteParams q)
{
    constexpr int GROUPS = RT_BWD_THREADS / G;
    constexpr int SLOTS = G == 1 ? PL : 1;
    __shared__ float slot_value[G == 1 ? 1 : GROUPS][G * PL];      // what the slots add, by expert; zero between tokens
    const int lane = threadIdx.x & 31, gl = G == 1 ? 0 : lane, group = threadIdx.x / G;
    const float d = q.dloss ? __ldg(q.dloss) : 1.0f;
    const float n = (float)__ldg(q.n_in);
    const float ub = n > 0.0f ? d * q.balance_coef * (float)q.E / (n * n * (float)q.k) : 0.0f;
    const float uz = n > 0.0f ? d * q.z_coef * 2.0f / n : 0.0f;
    float u0[PL];
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        u0[i] = i * G + gl < q.E ? ub * (float)__ldg(q.counts_in + i * G + gl) : 0.0f;
        if (G == 32) slot_value[group][i * G + gl] = 0.0f;
    }
    for (size_t first = (size_t)blockIdx.x * GROUPS; first < q.T; first += (size_t)gridDim.x * GROUPS) {
        const size_t t = first + group;
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
                if (se[j] < 0 || se[j] >= q.E) {
                    se[j] = -1;
                    sd[j] = 0.0f;
                }
            }
        }
        Token<G, PL> tok;
        load_logits<F32, G, PL>(q.logits, t, q.E, gl, live, tok.l);
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) sw[j] = q.normalize && se[j] >= 0 ? load_logit<F32>(q.logits, t * q.E + se[j]) : -INFINITY;
        tok.finish();
        if (q.dweight && q.normalize) {
            float h = -INFINITY;
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) h = fmaxf(h, sw[j]);
            h = group_max<G>(h);
            float s = 0.0f, sdw = 0.0f;
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) {
                sw[j] = h > -INFINITY ? exp_neg(sw[j] - h) : 0.0f;
                s += sw[j];
            }
            s = group_sum<G>(s);
            const float inv = s > 0.0f ? 1.0f / s : 0.0f;
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) {
                sw[j] *= inv;
                sdw = fmaf(sd[j], sw[j], sdw);
            }
            sdw = group_sum<G>(sdw);
#pragma unroll
            for (int j = 0; j < SLOTS; ++j) sd[j] = sw[j] * (sd[j] - sdw);
        }
        float add[PL];                                     // what the slots add, by expert
#pragma unroll
        for (int i = 0; i < PL; ++i) add[i] = 0.0f;
        if (q.dweight) {
            if (G == 1) {
#pragma unroll
                for (int j = 0; j < SLOTS; ++j)
#pragma unroll
                    for (int i = 0; i < PL; ++i)
                        if (se[j] == i) add[i] += sd[j];
            } else {
                __syncwarp();
                if (se[0] >= 0) slot_value[group][se[0]] = sd[0];
                __syncwarp();
#pragma unroll
                for (int i = 0; i < PL; ++i) add[i] = slot_value[group][i * G + gl];
                __syncwarp();
                if (se[0] >= 0) slot_value[group][se[0]] = 0.0f;
            }
        }
        float up = 0.0f;
#pragma unroll
        for (int i = 0; i < PL; ++i) up = fmaf(q.normalize ? u0[i] : u0[i] + add[i], tok.p[i], up);
        up = group_sum<G>(up);
        const float shift = (tok.routed ? uz * tok.lse() : 0.0f) - up;
        if (!live) continue;
        float g[PL];
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            g[i] = q.normalize ? fmaf(tok.p[i], u0[i] + shift, add[i]) : tok.p[i] * ((u0[i] + add[i]) + shift);
            if (!tok.routed) g[i] = tok.broken ? NAN : 0.0f;       // 0 whatever dloss is
        }
        if constexpr (G == 1) {
            if (q.E == PL) {
#pragma unroll
                for (int i = 0; i < PL; i += 8) {
                    if (F32) {
                        float4 *o = reinterpret_cast<float4 *>(static_cast<float *>(q.dlogits) + t * PL + i);
                        o[0] = make_float4(g[i], g[i + 1], g[i + 2], g[i + 3]);
                        o[1] = make_float4(g[i + 4], g[i + 5], g[i + 6], g[i + 7]);
                    } else {
                        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(q.dlogits) + t * PL + i) =
                            make_uint4(pack_bf16x2(g[i], g[i + 1]), pack_bf16x2(g[i + 2], g[i + 3]),
                                       pack_bf16x2(g[i + 4], g[i + 5]), pack_bf16x2(g[i + 6], g[i + 7]));
                    }
                }
                continue;
            }
        }
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            const int e = i * G + gl;
            if (e >= q.E) continue;
            if (F32) static_cast<float *>(q.dlogits)[t * q.E + e] = g[i];
            else static_cast<uint16_t *>(q.dlogits)[t * q.E + e] = (uint16_t)(pack_bf16x2(g[i], g[i]) & 0xFFFFu);
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
static int route_stride(int E) { return (E + 3) & ~3; }
static size_t route_ctas(size_t T) { return (T + route_chunk(T) - 1) / route_chunk(T); }

template <auto Kernel>
static int route_cluster(const RouteParams &q, int quads_log2, int slices, cudaStream_t st)
{
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)q.ctas + 1);
    c.blockDim = dim3(RT_THREADS);
    c.stream = st;
    cudaLaunchAttribute a[1];
    a[0].id = cudaLaunchAttributeClusterDimension;
    a[0].val.clusterDim.x = (unsigned)q.ctas + 1;
    a[0].val.clusterDim.y = a[0].val.clusterDim.z = 1;
    c.attrs = a;
    c.numAttrs = 1;
    FP8_CUDA_CHECK(cudaLaunchKernelEx(&c, Kernel, q, quads_log2, slices));
    return FP8_OK;
}

}  // namespace fp8dpa

using namespace fp8dpa;

// A lane per token (up to 16 experts) has a latency of its own, a warp per token one that grows with the tokens; one lane is
// faster above these many tokens.  us with a lane and with a warp per token, FP32 logits:
//   first forward kernel   E = 8: 4096 tokens 3.9, 3.4; 6144 3.9, 4.4    E = 16: 12288 7.1, 6.2; 16384 7.1, 7.4
//   gradient               E = 8: 8192 5.1, 4.4; 12288 5.2, 5.5          E = 16: 24576 11.3, 8.4; 131072 24.5, 35.1
static bool route_choose_by_lane(size_t T, int E) { return E <= 16 && T > (E <= 8 ? 4096 : 12288); }
static bool route_bwd_by_lane(size_t T, int E) { return E <= 16 && T > (E <= 8 ? 8192 : 32768); }

#define FP8DPA_ROUTE_DISPATCH(KERNEL, BY_LANE, GRID, THREADS)                        \
    do {                                                                             \
        if (BY_LANE && q.E <= 8) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 1, 8);     \
        else if (BY_LANE) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 1, 16);           \
        else if (q.E <= 32) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 32, 1);         \
        else if (q.E <= 64) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 32, 2);         \
        else if (q.E <= 96) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 32, 3);         \
        else if (q.E <= 128) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 32, 4);        \
        else if (q.E <= 160) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 32, 5);        \
        else if (q.E <= 192) FP8DPA_ROUTE_TYPE(KERNEL, GRID, THREADS, 32, 6);        \
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
    return route_shape_ok(T, E) ? (route_ctas(T) * ((size_t)route_stride(E) * 8 + 12) + 255) & ~(size_t)255 : 0;
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
    if (!aligned16(logits) || !aligned_to(expert, 4) || !aligned_to(weight, 4) || !aligned_to(rows, 4)) {
        set_error("fp8_moe_route: logits must be 16-byte aligned, the per-token outputs 4-byte");
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
    q.stride = route_stride(E);
    q.cta_probs = reinterpret_cast<float *>(q.cta_counts + (size_t)q.ctas * q.stride);
    q.cta_z = reinterpret_cast<double *>(q.cta_probs + (size_t)q.ctas * q.stride);
    q.cta_n = reinterpret_cast<int *>(q.cta_z + q.ctas);
    int quads_log2 = 0;
    while ((4 << quads_log2) < E) ++quads_log2;
    const int slices = (RT_THREADS >> quads_log2) < 32 ? RT_THREADS >> quads_log2 : 32;
    if ((unsigned)q.ctas < RT_CLUSTER) {
#define FP8DPA_ROUTE_CLUSTER(PL) \
    (is_fp32 ? route_cluster<route_cluster_kernel<true, PL>>(q, quads_log2, slices, st) : route_cluster<route_cluster_kernel<false, PL>>(q, quads_log2, slices, st))
        return E <= 32 ? FP8DPA_ROUTE_CLUSTER(1) : E <= 64 ? FP8DPA_ROUTE_CLUSTER(2) : E <= 128 ? FP8DPA_ROUTE_CLUSTER(4) : FP8DPA_ROUTE_CLUSTER(8);
#undef FP8DPA_ROUTE_CLUSTER
    }
    // one thread per token: no more threads than the chunk has tokens
    const bool by_lane = route_choose_by_lane(T, E);
    const unsigned threads = !by_lane ? RT_THREADS : (unsigned)(q.chunk < 512 ? (q.chunk + 31) & ~(size_t)31 : 512);
    FP8DPA_ROUTE_DISPATCH(route_choose_kernel, by_lane, q.ctas, threads);
    FP8_CUDA_CHECK(cudaGetLastError());
    return launch_early(route_place_kernel, rows ? q.ctas + 1 : 1, RT_THREADS, 0, st, q, quads_log2, slices);
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
    if (!aligned16(logits) || !aligned_to(expert, 4) || !aligned_to(dweight, 4) || !aligned16(dlogits)) {
        set_error("fp8_moe_route_bwd: logits and dlogits must be 16-byte aligned, expert and dweight 4-byte");
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
    const bool by_lane = route_bwd_by_lane(T, E);
    const size_t groups = by_lane ? RT_BWD_THREADS : RT_BWD_THREADS / 32;
    size_t blocks = (T + groups - 1) / groups;
    const size_t cap = (size_t)sm_count() * 8;
    if (blocks > cap) blocks = cap;
    FP8DPA_ROUTE_DISPATCH(route_bwd_kernel, by_lane, (unsigned)blocks, RT_BWD_THREADS);
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
}
