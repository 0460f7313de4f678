// AdamW over many tensors: clip, moments, decayed weights, their BF16 copy, FP8 codes and amax for the next step's products, with
// moments in FP32 or in 8 bits.
#include <math.h>

#include "common.cuh"
#include "elementwise.cuh"

namespace fp8dpa {

constexpr int AW_THREADS = 256;
constexpr int AW_PER_THREAD = 16;
constexpr int AW_CHUNK = AW_THREADS * AW_PER_THREAD;
constexpr int AW_ITEMS = 256;                             // tensors per launch (27 KB of kernel parameters)
constexpr int AW_BUCKETS = 1024;
constexpr int AW_BLOCK = 128;                             // values that share a scale in the 8-bit moments

struct AdamTable {
    float *p[AW_ITEMS];
    const void *g[AW_ITEMS];
    void *m[AW_ITEMS], *v[AW_ITEMS];
    uint8_t *m_exp[AW_ITEMS], *v_exp[AW_ITEMS];
    uint16_t *p16[AW_ITEMS];
    uint8_t *p8[AW_ITEMS];
    const float *q_scale[AW_ITEMS];
    unsigned int *amax[AW_ITEMS];
    unsigned long long n[AW_ITEMS], done[AW_ITEMS];       // elements here, and of the tensor in front of them
    unsigned first[AW_ITEMS + 1];                         // the tensor's first chunk
    float decay[AW_ITEMS];
    unsigned short start[AW_BUCKETS];                     // the tensor that holds chunk j << bucket_log2
    unsigned char types[AW_ITEMS];                        // bit 0: g is FP32, bit 1: moments in 8 bits, bit 2: codes are E5M2
    int items, bucket_log2, number;                       // number: of the first tensor in the caller's list
    unsigned chunks;
};

// What one thread works out for all: the step's number and what follows from it.
struct AdamStep {
    float factor, rate, inv_root, lr;                     // of the gradient; lr / (1 - beta1^t); 1 / sqrt(1 - beta2^t); lr
    uint32_t key;
    int skip;
};

// 32-bit integers to 32-bit integers that look random: xor-shifts and products with odd numbers (2^32 times the fractions of the
// golden ratio and of the square root of 2).  Every output bit changes with a probability within 0.011 of 1/2 with each input bit.
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x9E3779B9u;
    x = (x ^ (x >> 15)) * 0x6A09E667u;
    return x ^ (x >> 16);
}

__global__ void __launch_bounds__(AW_ITEMS) adamw_begin_kernel(const __grid_constant__ AdamTable t, AdamStep *out, const float *lr,
                                                              int *step, double log_beta1, double log_beta2, const float *norm,
                                                              float max_norm, uint32_t seed_lo, uint32_t seed_hi, int first_launch)
{
    cudaTriggerProgrammaticLaunchCompletion();
    const float n = norm ? *norm : 0.0f;
    const bool skip = !(n - n == 0.0f);                   // infinite or NaN
    if (!skip && threadIdx.x < t.items && t.done[threadIdx.x] == 0 && t.amax[threadIdx.x]) *t.amax[threadIdx.x] = 0u;
    if (threadIdx.x == 0 && first_launch) {
        AdamStep s;
        const int now = *step + 1;
        s.skip = skip;
        s.factor = 1.0f;
        if (norm) {
            const float f = max_norm / (n + 1e-6f);
            if (f < 1.0f) s.factor = f;
        }
        s.lr = *lr;
        s.rate = (float)((double)s.lr / -expm1((double)now * log_beta1));
        s.inv_root = (float)(1.0 / sqrt(-expm1((double)now * log_beta2)));
        s.key = mix32(mix32(mix32(seed_lo) ^ seed_hi) ^ (uint32_t)now);
        *out = s;
        if (!skip) *step = now;
    }
}

__device__ __forceinline__ int item_of_chunk(const AdamTable &t, unsigned c)
{
    int k = t.start[c >> t.bucket_log2];
    while (t.first[k + 1] <= c) ++k;
    return k;
}

// Eight consecutive values of a tensor; behind its end zeros, and nothing is stored.
__device__ __forceinline__ void load8(const float *p, int left, float (&f)[8])
{
    if (left >= 8) {
        const float4 a = __ldcs(reinterpret_cast<const float4 *>(p)), b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = e < left ? p[e] : 0.0f;
    }
}
__device__ __forceinline__ void load8(const uint16_t *p, int left, float (&f)[8])
{
    if (left >= 8) {
        const uint4 w = __ldcs(reinterpret_cast<const uint4 *>(p));
        f[0] = bf16_lo(w.x); f[1] = bf16_hi(w.x); f[2] = bf16_lo(w.y); f[3] = bf16_hi(w.y);
        f[4] = bf16_lo(w.z); f[5] = bf16_hi(w.z); f[6] = bf16_lo(w.w); f[7] = bf16_hi(w.w);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = e < left ? __uint_as_float((uint32_t)p[e] << 16) : 0.0f;
    }
}
__device__ __forceinline__ uint2 load8(const uint8_t *p, int left)
{
    if (left >= 8) return __ldcs(reinterpret_cast<const uint2 *>(p));
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < left) w[e >> 2] |= (uint32_t)p[e] << (8 * (e & 3));
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store8(float *p, int left, const float (&f)[8])
{
    if (left >= 8) {
        __stcs(reinterpret_cast<float4 *>(p), make_float4(f[0], f[1], f[2], f[3]));
        __stcs(reinterpret_cast<float4 *>(p) + 1, make_float4(f[4], f[5], f[6], f[7]));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = f[e];
    }
}
__device__ __forceinline__ void store8(uint16_t *p, int left, const uint32_t (&w)[4])
{
    if (left >= 8) {
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(w[0], w[1], w[2], w[3]));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
}
__device__ __forceinline__ void store8(uint8_t *p, int left, uint2 v)
{
    if (left >= 8) {
        __stcs(reinterpret_cast<uint2 *>(p), v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = (uint8_t)((e < 4 ? v.x : v.y) >> (8 * (e & 3)));
    }
}

__device__ __forceinline__ void decode8(uint2 codes, float scale, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint16_t two = (uint16_t)((i < 2 ? codes.x : codes.y) >> (16 * (i & 1)));
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
        float lo, hi;
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
        f[2 * i] = lo * scale;
        f[2 * i + 1] = hi * scale;
    }
}

// The codes of a block's values under the smallest power of two that leaves none above 448.  A value is rounded up in size with
// the probability of the part that is cut off (16 bits of it), so that a change far below a step is not lost over many steps but
// comes through on average.  FLOOR: values above zero get the smallest code at least (a root of zero in the update's denominator
// would let it through unchecked).  A value that is not finite gets the code of NaN.
template <bool FLOOR>
__device__ __forceinline__ uint2 encode8(const float (&f)[8], const uint32_t (&bits)[8], uint32_t &exponent)
{
    float most = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(f[e]));
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));   // the block's 16 lanes
    const int up = (int)((__float_as_uint(most) + 0x1FFFFFu) >> 23) - 8;
    exponent = (uint32_t)max(up, 1);
    const float inv = __uint_as_float((254u - exponent) << 23);
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float y = fabsf(f[e]) * inv, off = y < 0.015625f ? 0.015625f : 0.0f;     // below the normal numbers the step stays 2^-9
        const uint32_t rnd = FLOOR ? (bits[e] >> 16) << 4 : (bits[e] & 0xFFFFu) << 4;
        float q = __uint_as_float((__float_as_uint(y + off) + rnd) & 0xFFF00000u) - off;
        if (FLOOR && q == 0.0f && f[e] > 0.0f) q = 0.001953125f;
        q = y <= 448.0f ? q : __uint_as_float(0x7FC00000u);
        z[e] = FLOOR ? q : copysignf(q, f[e]);
    }
    return make_uint2(cvt_f32x4_to_fp8x4<0>(z[0], z[1], z[2], z[3]), cvt_f32x4_to_fp8x4<0>(z[4], z[5], z[6], z[7]));
}

struct AdamRates {
    float beta1, rest1, beta2, rest2, eps;                // rest = 1 - beta
};

template <typename G, bool EIGHT>
__device__ __forceinline__ uint32_t adamw_chunk(const AdamTable &t, int k, unsigned long long i, int left, const AdamStep &s,
                                               const AdamRates &a)
{
    const float keep = 1.0f - s.lr * t.decay[k], qs = t.p8[k] ? __ldg(t.q_scale[k]) : 1.0f;
    float *const p = t.p[k];
    const G *const g = static_cast<const G *>(t.g[k]);
    uint32_t m2 = 0u;
    i += threadIdx.x * 8;
    left -= threadIdx.x * 8;
#pragma unroll
    for (int u = 0; u < AW_PER_THREAD / 8; ++u, i += AW_THREADS * 8, left -= AW_THREADS * 8) {
        float w[8], d[8], m[8], v[8], r[8];
        const int some = max(left, 0);
        load8(p + i, some, w);
        load8(g + i, some, d);
        if (EIGHT) {
            const uint2 mc = load8(static_cast<const uint8_t *>(t.m[k]) + i, some), vc = load8(static_cast<const uint8_t *>(t.v[k]) + i, some);
            uint32_t me = 0u, ve = 0u;
            if (some) {
                me = t.m_exp[k][i / AW_BLOCK];
                ve = t.v_exp[k][i / AW_BLOCK];
            }
            decode8(mc, __uint_as_float(me << 23), m);
            decode8(vc, __uint_as_float(ve << 23), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= v[e];
        } else {
            load8(static_cast<const float *>(t.m[k]) + i, some, m);
            load8(static_cast<const float *>(t.v[k]) + i, some, v);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = __fmul_rn(d[e], s.factor);
            // one rounding per operation, in this order: the codes that random bits give are the same wherever they are worked out
            m[e] = __fadd_rn(__fmul_rn(a.beta1, m[e]), __fmul_rn(a.rest1, x));
            v[e] = __fadd_rn(__fmul_rn(a.beta2, v[e]), __fmul_rn(__fmul_rn(a.rest2, x), x));
            if (EIGHT) r[e] = __fsqrt_rn(v[e]);
            else asm("sqrt.approx.f32 %0, %1;" : "=f"(r[e]) : "f"(v[e]));
            w[e] = fmaf(-s.rate, __fdividef(m[e], fmaf(r[e], s.inv_root, a.eps)), w[e] * keep);
        }
        store8(p + i, some, w);
        if (EIGHT) {
            const unsigned long long at = t.done[k] + i;
            const uint32_t key = mix32(mix32(s.key + (uint32_t)(t.number + k)) + (uint32_t)(at >> 32)) + (uint32_t)at;
            uint32_t bits[8], me, ve;
#pragma unroll
            for (int e = 0; e < 8; ++e) bits[e] = mix32(key + e);
            const uint2 mc = encode8<false>(m, bits, me), vc = encode8<true>(r, bits, ve);
            store8(static_cast<uint8_t *>(t.m[k]) + i, some, mc);
            store8(static_cast<uint8_t *>(t.v[k]) + i, some, vc);
            if (some && (threadIdx.x & 15) == 0) {
                t.m_exp[k][i / AW_BLOCK] = (uint8_t)me;
                t.v_exp[k][i / AW_BLOCK] = (uint8_t)ve;
            }
        } else {
            store8(static_cast<float *>(t.m[k]) + i, some, m);
            store8(static_cast<float *>(t.v[k]) + i, some, v);
        }
        uint32_t o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = pack_bf16x2(w[2 * q], w[2 * q + 1]);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            m2 = absmax2e(m2, o[q] & (2 * q + 1 < some ? 0xFFFFFFFFu : 2 * q < some ? 0xFFFFu : 0u));
        if (t.p16[k]) store8(t.p16[k] + i, some, o);
        if (t.p8[k]) store8(t.p8[k] + i, some, bf16x8_to_fp8x8(o, qs, t.types[k] >> 2));
    }
    return m2;
}

__global__ void __launch_bounds__(AW_THREADS) adamw_kernel(const __grid_constant__ AdamTable t, const AdamStep *step, const AdamRates a)
{
    const unsigned c = blockIdx.x;
    const int k = item_of_chunk(t, c);
    const unsigned long long i = (unsigned long long)(c - t.first[k]) * AW_CHUNK, rest = t.n[k] - i;
    const int left = rest < AW_CHUNK ? (int)rest : AW_CHUNK;
    cudaGridDependencySynchronize();
    const AdamStep s = *step;
    if (s.skip) return;
    uint32_t m2;
    switch (t.types[k] & 3) {
    case 0: m2 = adamw_chunk<uint16_t, false>(t, k, i, left, s, a); break;
    case 1: m2 = adamw_chunk<float, false>(t, k, i, left, s, a); break;
    case 2: m2 = adamw_chunk<uint16_t, true>(t, k, i, left, s, a); break;
    default: m2 = adamw_chunk<float, true>(t, k, i, left, s, a); break;
    }
    if (t.amax[k]) block_max_bf16_to(m2, t.amax[k]);
}

static int adamw_check_items(const fp8_adamw_item *items, int n_items)
{
    for (int i = 0; i < n_items; ++i) {
        const fp8_adamw_item &it = items[i];
        if (it.n == 0) continue;
        const bool eight = it.state_bits == 8;
        if (!eight && it.state_bits != 32) {
            set_error("fp8_adamw: item %d: state_bits = %d is not 8 or 32", i, it.state_bits);
            return FP8_ERR_ENUM;
        }
        if (it.p8 && it.fmt != FP8_E4M3 && it.fmt != FP8_E5M2) {
            set_error("fp8_adamw: item %d: fmt %d is not FP8_E4M3 / FP8_E5M2", i, it.fmt);
            return FP8_ERR_ENUM;
        }
        if (!it.p || !it.g || !it.m || !it.v || (eight && (!it.m_exp || !it.v_exp)) || (it.p8 && !it.q_scale)) {
            set_error("fp8_adamw: item %d: NULL pointer", i);
            return FP8_ERR_NULL;
        }
        if (!aligned16(it.p) || !aligned16(it.g) || !aligned16(it.m) || !aligned16(it.v) || !aligned16(it.p_bf16) || !aligned16(it.p8)) {
            set_error("fp8_adamw: item %d: pointers must be 16-byte aligned", i);
            return FP8_ERR_ALIGN;
        }
        if (it.n > ((size_t)1 << 40) || !(it.weight_decay >= 0.0f) || isinf(it.weight_decay)) {
            set_error("fp8_adamw: item %d: n = %zu is over 2^40, or weight_decay = %g", i, it.n, (double)it.weight_decay);
            return FP8_ERR_SHAPE;
        }
    }
    return FP8_OK;
}

// The next launch's table from item *item on; chunk numbers stay below 2^30, one tensor may be cut for that.
static void adamw_fill(AdamTable &t, const fp8_adamw_item *items, int n_items, int &item, size_t &done)
{
    const size_t most = (size_t)1 << 30;
    t.items = 0;
    t.chunks = 0;
    t.number = item;
    while (item < n_items && t.items < AW_ITEMS && t.chunks < most) {
        const fp8_adamw_item &it = items[item];
        const int k = t.items++;                              // empty ones too: the number in the list is part of the key
        size_t n = it.n - done, chunks = (n + AW_CHUNK - 1) / AW_CHUNK;
        if (chunks > most - t.chunks) {
            chunks = most - t.chunks;
            n = chunks * AW_CHUNK;
        }
        const bool eight = it.state_bits == 8;
        t.p[k] = it.p + done;
        t.g[k] = static_cast<const char *>(it.g) + done * (it.g_is_fp32 ? 4 : 2);
        t.m[k] = static_cast<char *>(it.m) + done * (eight ? 1 : 4);
        t.v[k] = static_cast<char *>(it.v) + done * (eight ? 1 : 4);
        t.m_exp[k] = it.m_exp + (eight ? done / AW_BLOCK : 0);
        t.v_exp[k] = it.v_exp + (eight ? done / AW_BLOCK : 0);
        t.p16[k] = it.p_bf16 ? static_cast<uint16_t *>(it.p_bf16) + done : nullptr;
        t.p8[k] = it.p8 ? it.p8 + done : nullptr;
        t.q_scale[k] = it.q_scale;
        t.amax[k] = reinterpret_cast<unsigned int *>(it.amax);
        t.n[k] = n;
        t.done[k] = done;
        t.first[k] = t.chunks;
        t.decay[k] = it.weight_decay;
        t.types[k] = (it.g_is_fp32 ? 1 : 0) | (eight ? 2 : 0) | (it.fmt == FP8_E5M2 ? 4 : 0);
        t.chunks += (unsigned)chunks;
        done += n;
        if (done == it.n) {
            ++item;
            done = 0;
        }
    }
    t.first[t.items] = t.chunks;
    t.bucket_log2 = 0;
    while ((t.chunks >> t.bucket_log2) >= (unsigned)AW_BUCKETS) ++t.bucket_log2;
    int k = 0;
    for (unsigned j = 0; j << t.bucket_log2 < t.chunks; ++j) {
        while (t.first[k + 1] <= j << t.bucket_log2) ++k;
        t.start[j] = (unsigned short)k;
    }
}

}  // namespace fp8dpa

using namespace fp8dpa;

extern "C" size_t fp8_adamw_workspace_bytes(const fp8_adamw_item *items, int n_items)
{
    return items && n_items > 0 ? 256 : 0;
}

extern "C" int fp8_adamw(const fp8_adamw_item *items, int n_items, const float *lr, int *step, double beta1, double beta2, double eps,
                         const float *norm, float max_norm, uint64_t seed, void *ws, size_t ws_bytes, void *stream)
{
    if (!items || !lr || !step) {
        set_error("fp8_adamw: NULL items, lr or step");
        return FP8_ERR_NULL;
    }
    if (n_items <= 0) {
        set_error("fp8_adamw: n_items = %d", n_items);
        return FP8_ERR_SHAPE;
    }
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 1e-30 && eps <= 1e30) ||
        (norm && (!(max_norm > 0.0f) || isinf(max_norm)))) {
        set_error("fp8_adamw: beta1 = %g, beta2 = %g (in [0, 1)), eps = %g (1e-30 to 1e30), max_norm = %g (above 0 with a norm)", beta1,
                  beta2, eps, (double)max_norm);
        return FP8_ERR_SHAPE;
    }
    int rc = adamw_check_items(items, n_items);
    if (rc != FP8_OK) return rc;
    if (!aligned_to(lr, 4) || !aligned_to(step, 4) || !aligned_to(norm, 4)) {
        set_error("fp8_adamw: lr, step and norm must be aligned to their type");
        return FP8_ERR_ALIGN;
    }
    if (!ws || ws_bytes < 256 || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("fp8_adamw: workspace of 256 bytes, 256-byte aligned, needed (got %zu)", ws_bytes);
        return FP8_ERR_WORKSPACE;
    }
    rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    AdamStep *s = static_cast<AdamStep *>(ws);
    const AdamRates a = {(float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps};
    AdamTable t;
    int item = 0, first = 1;
    size_t done = 0;
    while (item < n_items) {
        adamw_fill(t, items, n_items, item, done);
        adamw_begin_kernel<<<1, AW_ITEMS, 0, st>>>(t, s, lr, step, log(beta1), log(beta2), norm, max_norm, (uint32_t)seed,
                                                   (uint32_t)(seed >> 32), first);
        FP8_CUDA_CHECK(cudaGetLastError());
        first = 0;
        if (t.chunks == 0) continue;
        rc = launch_early(adamw_kernel, t.chunks, AW_THREADS, 0, st, t, static_cast<const AdamStep *>(s), a);
        if (rc != FP8_OK) return rc;
    }
    return FP8_OK;
}
