// AdamW over many tensors: clip, moments, decayed weights, their BF16 copy, FP8 codes and amax for the next step's products, with
// moments in FP32 or in 8 bits.
//
// The tensors are cut into chunks, numbered through all of them, and a short CTA takes one, found through a table that travels with
// the launch.  With FP32 moments bytes bind (218 M weights, BF16 gradients and both copies: 924 us, 6.3 GB at 6.8 TB/s).  With 8
// bits 17 bytes are left per weight and the arithmetic comes up to them: 102 instructions per weight took 916 us, 60 take 562 to
// 566 in a graph (3.7 GB at 6.6 TB/s), 580 to 620 back to back (the longer it runs the lower the clocks that power allows).
#include <math.h>

#include "common.cuh"
#include "elementwise.cuh"
#include "rows.cuh"

namespace fp8dpa {

constexpr int AW_THREADS = 256;
// Elements of a thread in a launch: 16 where moments have 8 bits, whose arithmetic hides the second eight's loads (218 M weights:
// 563 us, 635 with 8), and 8 where all have 32 (921 us, 943 with 16).
constexpr int AW_PER_THREAD_8BIT = 16, AW_PER_THREAD = 8;
constexpr int AW_ITEMS = 304;                             // tensors per launch (31 KB of kernel parameters)
constexpr int AW_BUCKETS = 512;
constexpr int AW_MAXIMA = 512;                            // amaxes that one launch sets to zero
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
    unsigned long long n[AW_ITEMS];
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
__device__ __forceinline__ uint32_t mix32_products(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x9E3779B9u;
    return (x ^ (x >> 15)) * 0x6A09E667u;
}
__device__ __forceinline__ uint32_t mix32(uint32_t x)
{
    x = mix32_products(x);
    return x ^ (x >> 16);
}

struct AdamMaxima {
    unsigned int *amax[AW_MAXIMA];
    int n;
};
__global__ void __launch_bounds__(AW_MAXIMA) adamw_begin_kernel(const __grid_constant__ AdamMaxima maxima, AdamStep *out, const float *lr,
                                                                int *step, double log_beta1, double log_beta2, const float *norm,
                                                                float max_norm, uint32_t seed_lo, uint32_t seed_hi)
{
    cudaTriggerProgrammaticLaunchCompletion();
    const float n = norm ? *norm : 0.0f;
    const bool skip = !(n - n == 0.0f);                   // infinite or NaN
    if (!skip && threadIdx.x < maxima.n) *maxima.amax[threadIdx.x] = 0u;
    if (threadIdx.x < 32 && out) {                        // 1 - beta^t of both rates side by side, on two lanes
        AdamStep s;
        const int now = *step + 1;
        const double gone = -expm1((double)now * (threadIdx.x & 1 ? log_beta2 : log_beta1));
        const double gone2 = __shfl_sync(0xffffffffu, gone, 1);
        if (threadIdx.x != 0) return;
        s.skip = skip;
        s.factor = 1.0f;
        if (norm) {
            const float f = max_norm / (n + 1e-6f);
            if (f < 1.0f) s.factor = f;
        }
        s.lr = *lr;
        s.rate = (float)((double)s.lr / gone);
        s.inv_root = (float)(1.0 / sqrt(gone2));
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

// Four of these per eight values: the packed instructions work on two at a time.
__device__ __forceinline__ void decode8(uint2 codes, float scale, uint64_t (&f)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint16_t two = (uint16_t)((i < 2 ? codes.x : codes.y) >> (16 * (i & 1)));
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
        float lo, hi;
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
        f[i] = mul_f32x2(pack_f32x2(lo, hi), both(scale));
    }
}
// A sum that stays one: the compiler makes one rounding of a product and a sum of pairs, but not where they treat small numbers
// differently (0.9 m + 0.1 g in one rounding moved 181 of 218 M codes).  Terms and sums below the normal numbers are 0.
__device__ __forceinline__ uint64_t add_ftz2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// Square roots of two values that are 0 or normal numbers: the hardware's reciprocal root and one step of Newton's iteration on
// r^2 = v, r - (r^2 - v) / (2 r), with the difference exact: the correctly rounded root but where that lies within 2^-44 of the
// middle of two values (none of 8.4 M mantissas from 2^-102 on).  Below 2^-102 the difference has fewer bits, and the root may be the
// next value (of 2^-126 to 2^-125 a tenth are).  NaN of infinity.
__device__ __forceinline__ uint64_t root2(uint64_t v)
{
    float a, b, qa, qb;
    unpack_f32x2(v, a, b);
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(qa) : "f"(fmaxf(a, 1.17549435e-38f)));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(qb) : "f"(fmaxf(b, 1.17549435e-38f)));
    const uint64_t q = pack_f32x2(qa, qb), r = mul_f32x2(v, q);
    return fma_f32x2(fma_f32x2(r, r, mul_f32x2(v, both(-1.0f))), mul_f32x2(q, both(-0.5f)), r);
}
__device__ __forceinline__ float reciprocal(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// The same, and 0 of NaN: root2 makes NaN of an infinite second moment, and 8 bits store one as NaN, but an infinite root moves
// nothing.  (A gradient that is NaN or infinite has made the first moment so, too: the element is NaN all the same.)
__device__ __forceinline__ float reciprocal_or_zero(float v)
{
    asm("min.f32 %0, %0, %1;" : "+f"(v) : "f"(INFINITY));
    return reciprocal(v);
}
__device__ __forceinline__ uint32_t half_bits(uint64_t v, int i)
{
    float lo, hi;
    unpack_f32x2(v, lo, hi);
    return __float_as_uint(i ? hi : lo);
}

// The biased exponent of the smallest power of two that leaves none of a block's values above 448, from its largest one: 448 is
// 1.75 * 2^8, and a mantissa above 1.75 carries into the exponent.
__device__ __forceinline__ uint32_t exponent_of(float most) { return (__float_as_uint(most) + 0x1FFFFFu) >> 23; }

// A block's values as codes.  E4M3 with a fixed bias is FP32 with fewer bits: the value over its power of two and over 2^120 has
// its code in bits 20 to 26, down to the smallest, FP32's own denormal numbers being its too.  Rounding with random bits is then
// an addition below bit 20: away from zero with the probability of the part that is cut off (16 bits of it), so that a change far
// below a step is not lost over many steps but comes through on average.  ROOT: not negative, and values above zero get the
// smallest code at least (a root of zero in the update's denominator would let it through unchecked).
// FAR: blocks whose power of two and 2^-120 do not fit into one factor.
constexpr uint32_t AW_FAR = 134;
template <bool ROOT, bool FAR>
__device__ __forceinline__ uint2 encode8(const uint64_t (&f)[4], const uint32_t (&bits)[8], uint32_t exponent)
{
    const uint64_t inv = both(__uint_as_float((FAR ? 254u - exponent : 134u - exponent) << 23)), down = both(7.5231638e-37f);   // 2^-120
    uint32_t z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        uint64_t y = mul_f32x2(f[e >> 1], inv);
        if (FAR) y = mul_f32x2(y, down);
        const uint32_t cut = ROOT ? bits[e] >> 16 : (bits[e] ^ bits[e] >> 16) & 0xFFFFu;       // the halves of mix32's result
        z[e] = half_bits(y, e & 1) + (cut << 4);
        if (ROOT) z[e] = max(z[e], min(half_bits(f[e >> 1], e & 1), 0x100000u)) << 4;
        else z[e] = ((z[e] << 4) & 0x7FFFFFFFu) | (z[e] & 0x80000000u);
    }
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = __byte_perm(__byte_perm(z[4 * i], z[4 * i + 1], 0x0073), __byte_perm(z[4 * i + 2], z[4 * i + 3], 0x0073), 0x5410);
    return make_uint2(w[0], w[1]);
}
// The same for any block.  Values that are not finite get the code of NaN, the others are scaled by the largest of theirs.
// By all lanes of a warp together.
template <bool ROOT>
__device__ __noinline__ uint2 encode8_any(uint64_t f0, uint64_t f1, uint64_t f2, uint64_t f3, uint32_t key, uint32_t &exponent)
{
    uint64_t f[4] = {f0, f1, f2, f3};
    uint32_t bits[8], broken = 0u;
    float most = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        bits[e] = mix32_products(key + e);
        const float v = fabsf(__uint_as_float(half_bits(f[e >> 1], e & 1)));
        if (v < INFINITY) most = fmaxf(most, v);
        else broken |= 1u << e;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float lo, hi;
        unpack_f32x2(f[e], lo, hi);
        f[e] = pack_f32x2(broken >> (2 * e) & 1u ? 0.0f : lo, broken >> (2 * e + 1) & 1u ? 0.0f : hi);
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
    exponent = (uint32_t)max((int)exponent_of(most) - 8, 1);
    uint2 c = encode8<ROOT, true>(f, bits, exponent);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (broken >> e & 1u) (e < 4 ? c.x : c.y) |= 0x7Fu << (8 * (e & 3));
    return c;
}

struct AdamRates {
    float beta1, rest1, beta2, rest2, eps;                // rest = 1 - beta
};

// What a thread reads of eight elements.
template <typename G, bool EIGHT>
struct AdamIn {
    float w[8], g[8], m[EIGHT ? 1 : 8], v[EIGHT ? 1 : 8];
    uint2 mc, vc;
    uint32_t me, ve;
    __device__ __forceinline__ void load(const AdamTable &t, int k, unsigned long long i, int some)
    {
        load8(t.p[k] + i, some, w);
        load8(static_cast<const G *>(t.g[k]) + i, some, g);
        if constexpr (EIGHT) {
            mc = load8(static_cast<const uint8_t *>(t.m[k]) + i, some);
            vc = load8(static_cast<const uint8_t *>(t.v[k]) + i, some);
            me = some ? t.m_exp[k][i / AW_BLOCK] : 0u;
            ve = some ? t.v_exp[k][i / AW_BLOCK] : 0u;
        } else {
            load8(static_cast<const float *>(t.m[k]) + i, some, m);
            load8(static_cast<const float *>(t.v[k]) + i, some, v);
        }
    }
};

// The element's new weight and moments, two elements at a time.  The moments take one rounding per operation, in this order: the
// codes that random bits give are the same wherever they are worked out.
template <typename G, bool EIGHT, bool WHOLE, int PER_THREAD>
__device__ __forceinline__ void adamw_chunk(const AdamTable &t, int k, unsigned long long i, int left, const AdamStep *step,
                                            const AdamRates &a)
{
    i += threadIdx.x * 8;
    left -= threadIdx.x * 8;
    constexpr int U = PER_THREAD / 8, STEP = AW_THREADS * 8;
    AdamIn<G, EIGHT> in[EIGHT ? U : 1];
    const float scale = t.p8[k] ? __ldg(t.q_scale[k]) : 1.0f;
    // on their way before the step's numbers are there
#pragma unroll
    for (int u = 0; u < (EIGHT ? U : 1); ++u) in[u].load(t, k, i + u * STEP, WHOLE ? 8 : max(left - u * STEP, 0));
    cudaGridDependencySynchronize();
    const AdamStep s = *step;
    if (s.skip) return;
    const uint64_t keep = both(1.0f - s.lr * t.decay[k]), qs = both(scale);
    float most = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u, i += STEP, left -= STEP) {
        const int some = WHOLE ? 8 : max(left, 0);
        AdamIn<G, EIGHT> &x = in[EIGHT ? u : 0];
        if (!EIGHT && u > 0) x.load(t, k, i, some);
        uint64_t m[4], v[4], r[4], w[4];
        if constexpr (EIGHT) {
            decode8(x.mc, __fmul_rn(a.beta1, __uint_as_float(x.me << 23)), m);       // beta1 m: a power of two moves no rounding
            decode8(x.vc, __uint_as_float(x.ve << 23), v);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (EIGHT) {
                v[e] = mul_f32x2(v[e], v[e]);
            } else {
                m[e] = pack_f32x2(x.m[2 * e], x.m[2 * e + 1]);
                v[e] = pack_f32x2(x.v[2 * e], x.v[2 * e + 1]);
            }
            const uint64_t g = mul_f32x2(pack_f32x2(x.g[2 * e], x.g[2 * e + 1]), both(s.factor));
            const uint64_t rest = EIGHT ? m[e] : mul_f32x2(both(a.beta1), m[e]), new_m = mul_f32x2(both(a.rest1), g);
            const uint64_t old = mul_f32x2(both(a.beta2), v[e]), more = mul_f32x2(mul_f32x2(both(a.rest2), g), g);
            if constexpr (EIGHT) {
                m[e] = add_ftz2(rest, new_m);
                v[e] = add_ftz2(old, more);
                r[e] = root2(v[e]);
            } else {
                m[e] = add_f32x2(rest, new_m);
                v[e] = add_f32x2(old, more);
                float lo, hi;
                unpack_f32x2(v[e], lo, hi);
                asm("sqrt.approx.f32 %0, %1;" : "=f"(lo) : "f"(lo));
                asm("sqrt.approx.f32 %0, %1;" : "=f"(hi) : "f"(hi));
                r[e] = pack_f32x2(lo, hi);
            }
            float lo, hi;
            unpack_f32x2(fma_f32x2(r[e], both(s.inv_root), both(a.eps)), lo, hi);
            lo = EIGHT ? reciprocal_or_zero(lo) : reciprocal(lo);
            hi = EIGHT ? reciprocal_or_zero(hi) : reciprocal(hi);
            w[e] = fma_f32x2(mul_f32x2(m[e], pack_f32x2(lo, hi)), both(-s.rate),
                             mul_f32x2(pack_f32x2(x.w[2 * e], x.w[2 * e + 1]), keep));
            most = absmax3(most, w[e]);
            unpack_f32x2(w[e], x.w[2 * e], x.w[2 * e + 1]);
        }
        store8(t.p[k] + i, some, x.w);
        if constexpr (EIGHT) {
            const uint32_t key = mix32(mix32(s.key + (uint32_t)(t.number + k)) + (uint32_t)(i >> 32)) + (uint32_t)i;
            float top_m = 0.0f, top_r = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                top_m = absmax3(top_m, m[e]);
                top_r = absmax3(top_r, r[e]);
            }
            uint32_t up = exponent_of(top_m) << 16 | exponent_of(top_r);
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) up = __vmaxu2(up, __shfl_xor_sync(0xffffffffu, up, off));   // the block's 16 lanes
            uint32_t me = (uint32_t)max((int)(up >> 16) - 8, 1), ve = (uint32_t)max((int)(up & 0xFFFFu) - 8, 1);
            uint2 mc, vc;
            if (__any_sync(0xffffffffu, max(me, ve) >= AW_FAR)) {
                mc = encode8_any<false>(m[0], m[1], m[2], m[3], key, me);
                vc = encode8_any<true>(r[0], r[1], r[2], r[3], key, ve);
            } else {
                uint32_t bits[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) bits[e] = mix32_products(key + e);
                mc = encode8<false, false>(m, bits, me);
                vc = encode8<true, false>(r, bits, ve);
            }
            store8(static_cast<uint8_t *>(t.m[k]) + i, some, mc);
            store8(static_cast<uint8_t *>(t.v[k]) + i, some, vc);
            if ((threadIdx.x & 15) == 0 && some) {
                t.m_exp[k][i / AW_BLOCK] = (uint8_t)me;
                t.v_exp[k][i / AW_BLOCK] = (uint8_t)ve;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                unpack_f32x2(m[e], x.m[2 * e], x.m[2 * e + 1]);
                unpack_f32x2(v[e], x.v[2 * e], x.v[2 * e + 1]);
            }
            store8(static_cast<float *>(t.m[k]) + i, some, x.m);
            store8(static_cast<float *>(t.v[k]) + i, some, x.v);
        }
        const uint32_t o[4] = {round2(w[0]), round2(w[1]), round2(w[2]), round2(w[3])};
        if (t.p16[k]) store8(t.p16[k] + i, some, o);
        if (t.p8[k]) store8(t.p8[k] + i, some, codes8(make_uint4(o[0], o[1], o[2], o[3]), qs, t.types[k] >> 2));
    }
    if (t.amax[k]) block_max_bf16_to(pack_bf16x2(most, 0.0f), t.amax[k]);
}

template <int PER_THREAD>
__global__ void __launch_bounds__(AW_THREADS, 4) adamw_kernel(const __grid_constant__ AdamTable t, const AdamStep *step, const AdamRates a)
{
    cudaTriggerProgrammaticLaunchCompletion();            // the next launch's tensors are others
    constexpr int CHUNK = AW_THREADS * PER_THREAD;
    const unsigned c = blockIdx.x;
    const int k = item_of_chunk(t, c);
    const unsigned long long i = (unsigned long long)(c - t.first[k]) * CHUNK, rest = t.n[k] - i;
    const int left = rest < CHUNK ? (int)rest : CHUNK;
    const bool whole = left == CHUNK;
#define FP8DPA_ADAMW_CHUNK(G, EIGHT) \
    whole ? adamw_chunk<G, EIGHT, true, PER_THREAD>(t, k, i, left, step, a) : adamw_chunk<G, EIGHT, false, PER_THREAD>(t, k, i, left, step, a)
    if (PER_THREAD == AW_PER_THREAD_8BIT && t.types[k] & 2) {
        if (t.types[k] & 1) return FP8DPA_ADAMW_CHUNK(float, true);
        return FP8DPA_ADAMW_CHUNK(uint16_t, true);
    }
    if (t.types[k] & 1) return FP8DPA_ADAMW_CHUNK(float, false);
    return FP8DPA_ADAMW_CHUNK(uint16_t, false);
#undef FP8DPA_ADAMW_CHUNK
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
        if (!aligned16(it.p) || !aligned16(it.g) || !aligned16(it.m) || !aligned16(it.v) || !aligned16(it.p_bf16) || !aligned16(it.p8) ||
            !aligned_to(it.q_scale, 4) || !aligned_to(it.amax, 4)) {
            set_error("fp8_adamw: item %d: tensors must be 16-byte aligned, q_scale and amax to their type", i);
            return FP8_ERR_ALIGN;
        }
        if (it.n > ((size_t)1 << 40) || !(it.weight_decay >= 0.0f) || isinf(it.weight_decay)) {
            set_error("fp8_adamw: item %d: n = %zu is over 2^40, or weight_decay = %g", i, it.n, (double)it.weight_decay);
            return FP8_ERR_SHAPE;
        }
    }
    return FP8_OK;
}

// The next launch's table from `item` on, up to 2^30 chunks (a tensor has 2^29 at most).
static void adamw_fill(AdamTable &t, const fp8_adamw_item *items, int n_items, size_t chunk, int &item)
{
    t.items = 0;
    t.chunks = 0;
    t.number = item;
    for (; item < n_items && t.items < AW_ITEMS; ++item) {
        const fp8_adamw_item &it = items[item];
        const size_t chunks = (it.n + chunk - 1) / chunk;
        if (t.chunks + chunks > (size_t)1 << 30) break;
        const int k = t.items++;                              // empty ones too: the number in the list is part of the key
        t.p[k] = it.p;
        t.g[k] = it.g;
        t.m[k] = it.m;
        t.v[k] = it.v;
        t.m_exp[k] = it.m_exp;
        t.v_exp[k] = it.v_exp;
        t.p16[k] = static_cast<uint16_t *>(it.p_bf16);
        t.p8[k] = it.p8;
        t.q_scale[k] = it.q_scale;
        t.amax[k] = reinterpret_cast<unsigned int *>(it.amax);
        t.n[k] = it.n;
        t.first[k] = t.chunks;
        t.decay[k] = it.weight_decay;
        t.types[k] = (it.g_is_fp32 ? 1 : 0) | (it.state_bits == 8 ? 2 : 0) | (it.fmt == FP8_E5M2 ? 4 : 0);
        t.chunks += (unsigned)chunks;
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
    AdamMaxima maxima;
    int at = 0;
    do {                                                      // the step's numbers, and zeros where maxima will be
        const bool first = at == 0;
        maxima.n = 0;
        for (; at < n_items && maxima.n < AW_MAXIMA; ++at)
            if (items[at].n && items[at].amax) maxima.amax[maxima.n++] = reinterpret_cast<unsigned int *>(items[at].amax);
        adamw_begin_kernel<<<1, AW_MAXIMA, 0, st>>>(maxima, first ? s : nullptr, lr, step, log(beta1), log(beta2), norm, max_norm,
                                                    (uint32_t)seed, (uint32_t)(seed >> 32));
        FP8_CUDA_CHECK(cudaGetLastError());
    } while (at < n_items);
    bool eight = false;
    for (int i = 0; i < n_items; ++i) eight |= items[i].n && items[i].state_bits == 8;
    AdamTable t;
    for (int item = 0; item < n_items;) {
        adamw_fill(t, items, n_items, (size_t)AW_THREADS * (eight ? AW_PER_THREAD_8BIT : AW_PER_THREAD), item);
        if (t.chunks == 0) continue;
        rc = launch_early(eight ? adamw_kernel<AW_PER_THREAD_8BIT> : adamw_kernel<AW_PER_THREAD>, t.chunks, AW_THREADS, 0, st, t,
                          static_cast<const AdamStep *>(s), a);
        if (rc != FP8_OK) return rc;
    }
    return FP8_OK;
}
