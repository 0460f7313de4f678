// Rotary positions on the heads of the fused QKV projection, with the QK regulariser in front of them, the amax and FP8 codes of
// the attention's three operands behind them, the gradient of all that, and the table of angles for long contexts.
#include <math.h>

#include "common.cuh"
#include "elementwise.cuh"
#include "rows.cuh"

namespace fp8dpa {

// ---------------------------------------------------------------- table
constexpr int ROPE_MAX_PAIRS = 128;
struct RopeTable {
    double turns[ROPE_MAX_PAIRS];        // turns of each pair per position, and what its rounding to 64 bits left out
    double rest[ROPE_MAX_PAIRS];
    float *cos_t, *sin_t;
    size_t rows;
    int pairs;
    float magnitude;
};

// sin and cos of two angles of at most an eighth of a turn, in turns: their Taylor series up to the powers 9 and 10, of which the
// next terms are 1.8e-9 and 1.1e-10 there, with the powers of 2 pi in the coefficients and the rounding of 2 pi itself in the sine's
// second one.
__device__ __forceinline__ void sincos2(uint64_t x, uint64_t &sn, uint64_t &cs)
{
    constexpr double T = 6.283185307179586, T2 = T * T, T4 = T2 * T2, T8 = T4 * T4;
    constexpr float FULL = (float)T;
    const auto k = [](double v) { return pack_f32x2((float)v, (float)v); };
    const uint64_t q = mul_f32x2(x, x);
    uint64_t s = fma_f32x2(q, k(T8 * T / 362880.0), k(-T4 * T2 * T / 5040.0));
    s = fma_f32x2(s, q, k(T4 * T / 120.0));
    s = fma_f32x2(s, q, k(-T2 * T / 6.0));
    s = fma_f32x2(s, q, k(T - FULL));
    sn = fma_f32x2(x, k(FULL), mul_f32x2(s, x));
    uint64_t c = fma_f32x2(q, k(-T8 * T2 / 3628800.0), k(T8 / 40320.0));
    c = fma_f32x2(c, q, k(-T4 * T2 / 720.0));
    c = fma_f32x2(c, q, k(T4 / 24.0));
    c = fma_f32x2(c, q, k(-T2 / 2.0));
    cs = fma_f32x2(c, q, k(1.0));
}

// The angle in turns is the product of the position and a frequency kept as the sum of two doubles.  Adding 1.5 * 2^50 to the first's
// product leaves the nearest whole number of quarters (2^31 turns at most), in the low bits of the sum too.  What is left of the angle
// is the exact product less those, rounded once, and the second's product, so that nothing is lost next to a quarter turn: entries
// are good to 2 ulp (1.3 seen) wherever the position lies, next to their zeros too.  (A product rounded to 64 bits is off by 2^-53 of
// all turns: its cosine next to a zero by 2291 ulp below position 2^20, by 10^5 further out.)
// A thread keeps four frequencies, which one thread each brings to shared memory (lanes that ask the launch's parameters for different
// words wait for one another: 11.5 us for 131072 x 64 in a graph, 67 MB at 5.8 TB/s, and 15.3 without), and walks over the positions.
__global__ void __launch_bounds__(256) rope_table_kernel(const __grid_constant__ RopeTable t)
{
    const unsigned quads = t.pairs / 4, wide = 256 / quads, q = threadIdx.x % quads;
    __shared__ double2 frequency[4][ROPE_MAX_PAIRS / 4];
    if (threadIdx.x < t.pairs) frequency[threadIdx.x & 3][threadIdx.x >> 2] = make_double2(t.turns[threadIdx.x], t.rest[threadIdx.x]);
    __syncthreads();
    if (threadIdx.x >= wide * quads) return;
    double f[4], f_rest[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[e] = frequency[e][q].x;
        f_rest[e] = frequency[e][q].y;
    }
    const unsigned step = gridDim.x * wide;
#pragma unroll 2
    for (unsigned pos = blockIdx.x * wide + threadIdx.x / quads; pos < t.rows; pos += step) {
        const double at = (double)pos;
        float c[4], s[4], x[4];
        int k[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double shifted = fma(at, f[e], 1688849860263936.0), quarters = shifted - 1688849860263936.0;
            k[e] = __double2loint(shifted);
            x[e] = (float)fma(at, f_rest[e], fma(at, f[e], -quarters));
        }
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            uint64_t sn, cs;
            sincos2(pack_f32x2(x[e], x[e + 1]), sn, cs);
            unpack_f32x2(sn, s[e], s[e + 1]);
            unpack_f32x2(cs, c[e], c[e + 1]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float u = k[e] & 1 ? -s[e] : c[e], v = k[e] & 1 ? c[e] : s[e];
            c[e] = (k[e] & 2 ? -u : u) * t.magnitude;
            s[e] = (k[e] & 2 ? -v : v) * t.magnitude;
        }
        const size_t i = (size_t)pos * quads + q;
        __stcs(reinterpret_cast<float4 *>(t.cos_t) + i, make_float4(c[0], c[1], c[2], c[3]));
        __stcs(reinterpret_cast<float4 *>(t.sin_t) + i, make_float4(s[0], s[1], s[2], s[3]));
    }
}

// ---------------------------------------------------------------- heads
struct RopeArgs {
    const uint16_t *qkv;                 // rows of (Hq + 2 Hkv) heads, `pitch` elements apart (NULL: the gradient without a regulariser)
    size_t pitch;
    size_t T;
    int heads[3];                        // Hq, Hkv, Hkv
    int d, rot;                          // rot = 0: no rotation
    float alpha, eps, inv_d;
    const float *cos_t, *sin_t;
    size_t n_pos;
    const void *positions;
    int wide_positions;
    const uint16_t *grad[3];             // backward: gradients of q, k, v
    uint16_t *out[3];                    // forward: q, k, v; backward: out[0] = dqkv with rows `out_pitch` elements apart
    size_t out_pitch;
    uint8_t *out8[3];                    // forward: codes of q, k, v; backward: out8[0] = codes of dqkv, contiguous rows
    const float *scales;
    unsigned int *amax_bits;             // forward: three; backward: one
    unsigned words;                      // how many
    int fmt;
    int lanes_log2;                      // lanes per head: a power of two, at least d / 16
    int chunks[3];                       // pieces of ROPE_HEADS heads of each of q, k, v
    int per_cta, blocks;                 // pieces of a token on one CTA, and CTAs that share a token
    int tokens;                          // tokens of a CTA at a time (1 where CTAs share them)
};
constexpr int ROPE_HEADS = 4;

// A lane's cos and sin of a token, as the packed instructions take them: of partners in two groups (cos, sin, -sin of four pairs
// of places), or of neighbours (cos cos, -sin sin of each of eight pairs).
template <bool PAIRS>
struct Angles {
    uint64_t c[PAIRS ? 8 : 4], up[PAIRS ? 1 : 4], down[PAIRS ? 8 : 4];
    // from eight cos and eight sin, places 0 to 3 and 4 to 7 of the lane
    __device__ __forceinline__ void set(const uint4 c0, const uint4 c1, const uint4 s0, const uint4 s1, bool back)
    {
        const float cs[8] = {__uint_as_float(c0.x), __uint_as_float(c0.y), __uint_as_float(c0.z), __uint_as_float(c0.w),
                             __uint_as_float(c1.x), __uint_as_float(c1.y), __uint_as_float(c1.z), __uint_as_float(c1.w)};
        float sn[8] = {__uint_as_float(s0.x), __uint_as_float(s0.y), __uint_as_float(s0.z), __uint_as_float(s0.w),
                       __uint_as_float(s1.x), __uint_as_float(s1.y), __uint_as_float(s1.z), __uint_as_float(s1.w)};
#pragma unroll
        for (int e = 0; e < 8; ++e) sn[e] = back ? -sn[e] : sn[e];
#pragma unroll
        for (int e = 0; e < (PAIRS ? 8 : 4); ++e) {
            if (PAIRS) {
                c[e] = both(cs[e]);
                down[e] = pack_f32x2(-sn[e], sn[e]);
            } else {
                c[e] = pack_f32x2(cs[2 * e], cs[2 * e + 1]);
                up[PAIRS ? 0 : e] = pack_f32x2(sn[2 * e], sn[2 * e + 1]);
                down[e] = pack_f32x2(-sn[2 * e], -sn[2 * e + 1]);
            }
        }
    }
    // The rotation of a lane's two groups of eight: partners are the same places of the two groups, or neighbours in each.
    __device__ __forceinline__ void turn(uint64_t (&a)[4], uint64_t (&b)[4]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t x = a[e], y = b[e];
            if (PAIRS) {
                a[e] = fma_f32x2(x, c[e], mul_f32x2(swapped(x), down[e]));
                b[e] = fma_f32x2(y, c[PAIRS ? 4 + e : 0], mul_f32x2(swapped(y), down[PAIRS ? 4 + e : 0]));
            } else {
                a[e] = fma_f32x2(x, c[e], mul_f32x2(y, down[e]));
                b[e] = fma_f32x2(y, c[e], mul_f32x2(x, up[PAIRS ? 0 : e]));
            }
        }
    }
    static __device__ __forceinline__ uint64_t swapped(uint64_t v)
    {
        float lo, hi;
        unpack_f32x2(v, lo, hi);
        return pack_f32x2(hi, lo);
    }
};
__device__ __forceinline__ void scale8(uint64_t (&a)[4], float r)
{
    const uint64_t r2 = both(r);
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = mul_f32x2(a[e], r2);
}
__device__ __forceinline__ float dot16(const uint64_t (&a)[4], const uint64_t (&b)[4], const uint64_t (&x)[4], const uint64_t (&y)[4])
{
    uint64_t s = mul_f32x2(a[0], x[0]), t = mul_f32x2(b[0], y[0]);
#pragma unroll
    for (int e = 1; e < 4; ++e) {
        s = fma_f32x2(a[e], x[e], s);
        t = fma_f32x2(b[e], y[e], t);
    }
    return add_halves(add_f32x2(s, t));
}
template <typename F>
__device__ __forceinline__ void each8(uint64_t (&a)[4], F f)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float lo, hi;
        unpack_f32x2(a[e], lo, hi);
        a[e] = pack_f32x2(f(lo), f(hi));
    }
}

// 1 - tanh(x)^2 = 4 e / (1 + e)^2 with e = exp(-2 |x|): no cancellation where tanh is near 1.
__device__ __forceinline__ float sech2(float x)
{
    const float e = ex2_approx(-2.8853900817779268f * fabsf(x));
    return __fdividef(4.0f * e, (1.0f + e) * (1.0f + e));
}

template <int N>
__device__ __forceinline__ void block_max_each(const float (&m)[N], unsigned int *amax_bits)
{
    __shared__ uint32_t warp_max[N][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t most = __reduce_max_sync(0xffffffffu, pack_bf16x2(m[i], 0.0f) & 0xFFFFu);
        if (lane == 0) warp_max[i][warp] = most;
    }
    __syncthreads();
    const int nwarps = blockDim.x >> 5;
    for (int i = warp; i < N; i += nwarps) {
        const uint32_t most = __reduce_max_sync(0xffffffffu, lane < nwarps ? warp_max[i][lane] : 0u);
        if (lane == 0 && most != 0u) atomicMax(amax_bits + i, most << 16);
    }
}

// A head is on 2^lanes_log2 neighbouring lanes, 16 elements each: below `rot` lane j holds elements [8 j, 8 j + 8) and the same
// of the rotated part's second half, so that both kinds of partners are in one lane; behind it likewise, which passes through.
// A group of lanes takes up to ROPE_HEADS heads of one tensor of one token with the token's angles in registers.  Persistent: a
// group keeps its heads and walks over the tokens, and what it reads next travels through the threads' private ring.  Bytes
// bind: every element is read once and written once (8192 tokens of 32 + 2 x 8 heads of 128 with codes: 27.5 us in a graph, 153 MB
// at 5.6 TB/s; gradient 40.7 us, 237 MB at 5.8 TB/s; with a launch per call and whole-token CTAs that do not stay 47 and 72 us).
//
// Instructions are the next bound (23.7 M of a warp at first, 15.6 M now), so the usual case, all lanes of a warp with whole pieces
// of Q and K or of V, runs through four heads without a branch (33 -> 29.6 us, gradient 59 -> 43); V's pieces lie behind Q's and K's
// of all tokens of the CTA for that.  What is left takes the other path.  A second set of registers for the next token's angles or
// a branch around the rotation spills and costs 4 to 17 us.
// KIND: what is written, BF16 alone, codes alone in the direction's usual type (E4M3, E5M2 backward), or anything.
enum RopeKind { ROPE_BF16, ROPE_CODES, ROPE_ANY };
template <int MODE, bool BACK>
__host__ __device__ constexpr int rope_slots() { return ROPE_HEADS * (BACK && MODE != FP8_QK_NONE ? 4 : 2); }

// Sum over a head's lanes (D = 0: their number is not known).
template <int D>
__device__ __forceinline__ float head_sum(float v, int lanes)
{
#pragma unroll
    for (int off = D ? D / 32 : 8; off > 0; off >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, off);
        if (D || off < lanes) v += u;
    }
    return v;
}

// D: the head's size where it is one of the attention's and all of it is rotated (places are then known to the compiler: 18.7 -> 15.6 M
// instructions), else 0.
template <int D, int MODE, bool PAIRS, bool BACK, RopeKind KIND, int STAGES>
__global__ void __launch_bounds__(256, BACK ? 2 : 3) rope_kernel(const __grid_constant__ RopeArgs p, int /* of no use here */)
{
    extern __shared__ __align__(16) uint4 ring_mem[];
    constexpr bool SAVED = BACK && MODE != FP8_QK_NONE;
    constexpr int N = BACK ? 1 : 3;
    const bool alone = amax_begin(p.amax_bits, N);
    const int d = D ? D : p.d, rot = D ? D : p.rot;
    const int lanes = D ? D / 16 : 1 << p.lanes_log2, j = threadIdx.x & (lanes - 1), group = D ? threadIdx.x / (D ? D / 16 : 1) : threadIdx.x >> p.lanes_log2;
    const int turned = rot / 16, n_qk = p.chunks[0] + p.chunks[1], per_token = n_qk + p.chunks[2];
    const unsigned share = blockIdx.x % p.blocks, first = blockIdx.x / p.blocks, ctas = gridDim.x / p.blocks;
    int local, piece;
    if (p.blocks > 1) {
        local = 0;
        piece = group < p.per_cta ? share * p.per_cta + group : per_token;
    } else if (group < p.tokens * n_qk) {
        local = group / n_qk;
        piece = group - local * n_qk;
    } else {
        const int g = group - p.tokens * n_qk;
        local = p.chunks[2] ? g / p.chunks[2] : p.tokens;
        piece = n_qk + g - local * p.chunks[2];
    }
    const bool mine = (D || j < d / 16) && local < p.tokens && piece < per_token, turns = D || j < turned;
    piece = min(piece, per_token - 1);
    const int part = piece < p.chunks[0] ? 0 : piece < n_qk ? 1 : 2;
    if (part > 0) piece -= p.chunks[0];
    if (part > 1) piece -= p.chunks[1];
    const int h0 = piece * ROPE_HEADS, n_heads = p.heads[part], here = min(ROPE_HEADS, n_heads - h0);
    const int before = (part > 0 ? p.heads[0] : 0) + (part > 1 ? p.heads[1] : 0) + h0;       // heads of the row in front
    const int lo = turns ? 8 * j : rot + 8 * (j - turned), other = (turns ? rot : d - rot) / 2;
    const size_t in_row = (size_t)before * d + lo, in_part = (size_t)h0 * d + lo;
    const unsigned T = (unsigned)p.T, step = ctas * p.tokens;       // fewer than 2^31 tokens
    const size_t part_pitch = (size_t)n_heads * d, row_pitch = (size_t)(p.heads[0] + p.heads[1] + p.heads[2]) * d;
    unsigned t = first * p.tokens + local, ahead = t;
    // places in shared memory: [stage][slot][thread]; slots 2 hh, 2 hh + 1 are a head's groups, behind them those of what is saved
    const uint32_t per_slot = blockDim.x * 16u, per_stage = per_slot * rope_slots<MODE, BACK>();
    const uint32_t ring = smem_u32(ring_mem + threadIdx.x), ring_end = ring + STAGES * per_stage;
    // Forward: the angles lie behind them, [stage][token][cos, sin][rot / 2], copied by the first group of a token's for all (29.1
    // -> 27.5 us).  Backward has half the warps, whom the barrier for that costs more than the loads (42.4 us, 46.6 with it).
    constexpr bool SHARED = !BACK;
    const uint32_t tables = smem_u32(ring_mem) + STAGES * per_stage, per_table = p.tokens * rot * 4u;
    const bool copies = SHARED && mine && turns && part < 2 && (p.blocks > 1 ? group == 0 : group == local * n_qk);
    const uint32_t at0 = (PAIRS ? 4 * j : 8 * j) * 4u, at1 = (PAIRS ? rot / 4 + 4 * j : 8 * j + 4) * 4u, apart = rot * 2u;
    // A token's row of the tables, or -1 outside of them.
    const auto row_of = [&](unsigned t) -> int {
        if (!rot || !mine || t >= T) return 0;
        if (!p.positions) return (int)(t % (unsigned)p.n_pos);
        const long long at = p.wide_positions ? __ldg(static_cast<const long long *>(p.positions) + t)
                                              : (long long)__ldg(static_cast<const int *>(p.positions) + t);
        return at >= 0 && (unsigned long long)at < p.n_pos ? (int)at : -1;
    };
    int row_now = SHARED ? row_of(t) : 0, row_ahead = row_now;
    const uint16_t *next = (BACK ? p.grad[part] + in_part : p.qkv + in_row) + (size_t)ahead * (BACK ? part_pitch : p.pitch);
    const uint16_t *next_saved = SAVED ? p.qkv + in_row + (size_t)ahead * p.pitch : nullptr;
    const auto fetch = [&](uint32_t to, uint32_t table) {
        if (copies && ahead < T) {
            const size_t from = (size_t)max(row_ahead, 0) * (rot / 2);
            const uint32_t into = table + local * rot * 4u;
            const float *c = p.cos_t + from, *s = p.sin_t + from;
            cp_async16(into + at0, reinterpret_cast<const char *>(c) + at0);
            cp_async16(into + at1, reinterpret_cast<const char *>(c) + at1);
            cp_async16(into + apart + at0, reinterpret_cast<const char *>(s) + at0);
            cp_async16(into + apart + at1, reinterpret_cast<const char *>(s) + at1);
        }
        if (mine && ahead < T) {
#pragma unroll
            for (int hh = 0; hh < ROPE_HEADS; ++hh) {
                if (hh < here) {
                    cp_async16(to + (2 * hh) * per_slot, next + hh * d);
                    cp_async16(to + (2 * hh + 1) * per_slot, next + hh * d + other);
                    if (SAVED && part < 2) {
                        cp_async16(to + (2 * ROPE_HEADS + 2 * hh) * per_slot, next_saved + hh * d);
                        cp_async16(to + (2 * ROPE_HEADS + 2 * hh + 1) * per_slot, next_saved + hh * d + other);
                    }
                }
            }
        }
        cp_async_commit();
        ahead += step;
        if (SHARED) row_ahead = row_of(ahead);
        next += step * (BACK ? part_pitch : p.pitch);
        if (SAVED) next_saved += step * p.pitch;
    };
    static_assert(STAGES == 2, "row_ahead is one token ahead");
    fetch(ring, tables);
    const uint64_t qs2 = both(p.scales ? __ldg(p.scales + (BACK ? 0 : part)) : 1.0f);
    const size_t out_pitch = BACK ? p.out_pitch : part_pitch, out8_pitch = BACK ? row_pitch : part_pitch, out_at = BACK ? in_row : in_part;
    uint16_t *const out = BACK ? p.out[0] : p.out[part];
    uint8_t *const out8 = BACK ? p.out8[0] : p.out8[part];
    float m = 0.0f;
    uint32_t now = ring, fill = ring + (STAGES - 1) * per_stage, table = tables;

    // A lane's part of a head: what is read, regularised and rotated (or back), with `qk` false as it is.
    const auto work = [&](int hh, bool qk, bool every_lane_turns, const Angles<PAIRS> &angles, uint64_t (&a)[4], uint64_t (&b)[4]) {
        uint64_t x[4], y[4];
        unpack4x2(ring_get(now + (2 * hh) * per_slot), a);
        unpack4x2(ring_get(now + (2 * hh + 1) * per_slot), b);
        if (!qk) return;
        if (SAVED) {
            unpack4x2(ring_get(now + (2 * ROPE_HEADS + 2 * hh) * per_slot), x);
            unpack4x2(ring_get(now + (2 * ROPE_HEADS + 2 * hh + 1) * per_slot), y);
        }
        float r = 1.0f;
        if (MODE == FP8_QK_RMS) r = rsqrtf(fmaf(head_sum<D>(mine ? (BACK ? dot16(x, y, x, y) : dot16(a, b, a, b)) : 0.0f, lanes), p.inv_d, p.eps));
        if (!BACK) {
            if (MODE == FP8_QK_RMS) {
                scale8(a, r);
                scale8(b, r);
            } else if (MODE == FP8_QK_TANH) {
                each8(a, [&](float v) { return tanhf(p.alpha * v); });
                each8(b, [&](float v) { return tanhf(p.alpha * v); });
            }
        }
        if (every_lane_turns) {
            angles.turn(a, b);
        } else if (rot) {
            uint64_t u[4] = {a[0], a[1], a[2], a[3]}, w[4] = {b[0], b[1], b[2], b[3]};
            angles.turn(u, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] = turns ? u[e] : a[e];
                b[e] = turns ? w[e] : b[e];
            }
        }
        if (BACK && MODE == FP8_QK_RMS) {
            scale8(x, r);
            scale8(y, r);
            const uint64_t s2 = both(head_sum<D>(mine ? dot16(a, b, x, y) : 0.0f, lanes) * -p.inv_d);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] = fma_f32x2(s2, x[e], a[e]);
                b[e] = fma_f32x2(s2, y[e], b[e]);
            }
            scale8(a, r);
            scale8(b, r);
        }
        if (BACK && MODE == FP8_QK_TANH) {
            each8(x, [&](float v) { return p.alpha * sech2(p.alpha * v); });
            each8(y, [&](float v) { return p.alpha * sech2(p.alpha * v); });
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] = mul_f32x2(a[e], x[e]);
                b[e] = mul_f32x2(b[e], y[e]);
            }
        }
    };
    const auto store = [&](int hh, const uint64_t (&a)[4], const uint64_t (&b)[4], uint16_t *o, uint8_t *o8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) m = absmax3(absmax3(m, a[e]), b[e]);
        const uint4 oa = make_uint4(round2(a[0]), round2(a[1]), round2(a[2]), round2(a[3]));
        const uint4 ob = make_uint4(round2(b[0]), round2(b[1]), round2(b[2]), round2(b[3]));
        if (KIND == ROPE_BF16 || (KIND == ROPE_ANY && out)) {
            *reinterpret_cast<uint4 *>(o + hh * d) = oa;
            *reinterpret_cast<uint4 *>(o + hh * d + other) = ob;
        }
        if (KIND == ROPE_CODES || (KIND == ROPE_ANY && out8)) {
            const int fmt = KIND == ROPE_CODES ? BACK : p.fmt;
            *reinterpret_cast<uint2 *>(o8 + hh * d) = codes8(oa, qs2, fmt);
            *reinterpret_cast<uint2 *>(o8 + hh * d + other) = codes8(ob, qs2, fmt);
        }
    };
    const bool plain_lane = mine && here == ROPE_HEADS, whole_head = rot == d;
    const bool plain_qk = __all_sync(0xffffffffu, plain_lane && part < 2), plain_v = __all_sync(0xffffffffu, plain_lane && part == 2);
    for (unsigned base = first * p.tokens; base < T; base += step, t += step) {
        const int here_row = SHARED ? row_now : row_of(t);
        const bool live = mine && t < T, known = here_row >= 0;
        row_now = row_ahead;
        Angles<PAIRS> angles;
        if (!SHARED && turns && part < 2) {
            const size_t from = (size_t)max(here_row, 0) * (rot / 2);                  // row 0 for a token outside the table
            const char *c = reinterpret_cast<const char *>(p.cos_t + from), *s = reinterpret_cast<const char *>(p.sin_t + from);
            const auto get = [](const char *q) { return __ldg(reinterpret_cast<const uint4 *>(q)); };
            angles.set(get(c + at0), get(c + at1), get(s + at0), get(s + at1), BACK);
        }
        cp_async_wait<STAGES - 2>();
        if (SHARED) __syncthreads();                           // the token's angles are there, and the stage in front is read
        fetch(fill, table == tables ? tables + per_table : tables);
        fill = now;
        if (SHARED && turns && part < 2) {
            const uint32_t c = table + local * rot * 4u, s = c + apart;
            angles.set(ring_get(c + at0), ring_get(c + at1), ring_get(s + at0), ring_get(s + at1), BACK);
        }
        table = table == tables ? tables + per_table : tables;
        uint16_t *const o = out + (size_t)t * out_pitch + out_at;
        uint8_t *const o8 = out8 + (size_t)t * out8_pitch + out_at;
        const bool plain = __all_sync(0xffffffffu, live && known);
        if (plain && plain_qk) {
#pragma unroll
            for (int hh = 0; hh < ROPE_HEADS; ++hh) {
                uint64_t a[4], b[4];
                work(hh, true, whole_head, angles, a, b);
                store(hh, a, b, o, o8);
            }
        } else if (plain && plain_v) {
#pragma unroll
            for (int hh = 0; hh < ROPE_HEADS; ++hh) {
                uint64_t a[4], b[4];
                work(hh, false, false, angles, a, b);
                store(hh, a, b, o, o8);
            }
        } else {
#pragma unroll 1
            for (int hh = 0; hh < ROPE_HEADS; ++hh) {
                uint64_t a[4], b[4], u[4], w[4];
                work(hh, true, false, angles, a, b);           // all lanes: it has sums over lanes
                work(hh, false, false, angles, u, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    a[e] = !known ? 0ull : part < 2 ? a[e] : u[e];
                    b[e] = !known ? 0ull : part < 2 ? b[e] : w[e];
                }
                if (live && hh < here) store(hh, a, b, o, o8);
            }
        }
        now += per_stage;
        if (now == ring_end) now = ring;
    }
    cudaGridDependencySynchronize();
    if (alone) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    if (p.amax_bits) {
        float each[N];
#pragma unroll
        for (int i = 0; i < N; ++i) each[i] = BACK || part == i ? m : 0.0f;
        block_max_each(each, p.amax_bits);
    }
}

template <auto Kernel, bool SHARED>
static int rope_run(const RopeArgs &p, unsigned grid, unsigned threads, size_t per_thread, size_t elements, cudaStream_t st)
{
    const int rc = allow_shared<Kernel>((int)(256 * per_thread + (SHARED ? 2 * 16384 : 0)));      // of angles 16 KB at most a stage
    if (rc != FP8_OK) return rc;
    return launch_behind_amax<Kernel>(elements, p.amax_bits, grid, threads, threads * per_thread + (SHARED ? 8 * (size_t)p.tokens * p.rot : 0),
                                      st, p, 0, p.words);
}

template <bool BACK>
static int rope_launch(RopeArgs &p, int mode, bool pairs, cudaStream_t st)
{
    const int slots = p.d / 16;
    p.words = BACK ? 1 : 3;
    p.lanes_log2 = 0;
    while ((1 << p.lanes_log2) < slots) ++p.lanes_log2;
    int per_token = 0;
    for (int i = 0; i < 3; ++i) {
        // the forward leaves out what is not asked for
        const bool wanted = BACK || p.out[i] || p.out8[i] || p.amax_bits;
        p.chunks[i] = wanted ? (p.heads[i] + ROPE_HEADS - 1) / ROPE_HEADS : 0;
        per_token += p.chunks[i];
    }
    // CTAs of up to 256 threads take whole tokens, or several share one token's heads
    const int groups = 256 >> p.lanes_log2;
    p.blocks = (per_token + groups - 1) / groups;
    p.per_cta = (per_token + p.blocks - 1) / p.blocks;
    p.tokens = p.blocks > 1 ? 1 : groups / p.per_cta;
    if ((size_t)p.tokens > p.T) p.tokens = (int)p.T;
    const unsigned threads = (unsigned)((p.tokens * p.per_cta << p.lanes_log2) + 31) & ~31u;
    const size_t want = (p.T + p.tokens - 1) / p.tokens, most = 148 * (size_t)((BACK ? 512 : 768) / threads);
    size_t ctas = want * p.blocks <= most ? want : most / p.blocks;
    if (ctas == 0) ctas = 1;
    const unsigned grid = (unsigned)(ctas * p.blocks);
    const size_t elements = p.T * (size_t)(p.heads[0] + p.heads[1] + p.heads[2]) * p.d;
    bool bf16 = true, codes = true;
    for (int i = 0; i < (BACK ? 1 : 3); ++i) {
        if (!BACK && !p.chunks[i]) continue;
        bf16 &= p.out[i] && !p.out8[i];
        codes &= !p.out[i] && p.out8[i] && p.fmt == (BACK ? FP8_E5M2 : FP8_E4M3);
    }
    constexpr int STAGES = 2;
    const int whole = p.rot == p.d ? p.d : 0;
#define FP8DPA_ROPE_RUN(D, MODE, PAIRS, KIND) \
    return rope_run<rope_kernel<D, MODE, PAIRS, BACK, KIND, STAGES>, !BACK>(p, grid, threads, (size_t)STAGES * rope_slots<MODE, BACK>() * 16, elements, st)
#define FP8DPA_ROPE_SIZE(MODE, PAIRS, KIND) \
    do { \
        if (whole == 128) FP8DPA_ROPE_RUN(128, MODE, PAIRS, KIND); \
        if (whole == 64) FP8DPA_ROPE_RUN(64, MODE, PAIRS, KIND); \
        FP8DPA_ROPE_RUN(0, MODE, PAIRS, KIND); \
    } while (0)
#define FP8DPA_ROPE_PAIRS(MODE, PAIRS) \
    do { \
        if (bf16) FP8DPA_ROPE_SIZE(MODE, PAIRS, ROPE_BF16); \
        if (codes) FP8DPA_ROPE_SIZE(MODE, PAIRS, ROPE_CODES); \
        FP8DPA_ROPE_RUN(0, MODE, PAIRS, ROPE_ANY); \
    } while (0)
#define FP8DPA_LAUNCH_ROPE(MODE) \
    do { \
        if (pairs) FP8DPA_ROPE_PAIRS(MODE, true); \
        else FP8DPA_ROPE_PAIRS(MODE, false); \
    } while (0)
    if (mode == FP8_QK_RMS) FP8DPA_LAUNCH_ROPE(FP8_QK_RMS);
    else if (mode == FP8_QK_TANH) FP8DPA_LAUNCH_ROPE(FP8_QK_TANH);
    else FP8DPA_LAUNCH_ROPE(FP8_QK_NONE);
#undef FP8DPA_LAUNCH_ROPE
#undef FP8DPA_ROPE_PAIRS
#undef FP8DPA_ROPE_SIZE
#undef FP8DPA_ROPE_RUN
}

// What both directions check of an fp8_rope; 0 or a status.
static int rope_check(const char *who, size_t T, int Hq, int Hkv, int d, const fp8_rope *r)
{
    if (!r) {
        set_error("%s: NULL rope", who);
        return FP8_ERR_NULL;
    }
    if (r->mode < FP8_QK_RMS || r->mode > FP8_QK_NONE) {
        set_error("%s: mode %d is not FP8_QK_RMS / FP8_QK_TANH / FP8_QK_NONE", who, r->mode);
        return FP8_ERR_ENUM;
    }
    if (T == 0 || T > 0x7FFFFFFFull || Hq <= 0 || Hkv < 0 || Hq > 65536 || Hkv > 65536 || d <= 0 || d % 16 || d > 256) {
        set_error("%s: unsupported shape T=%zu Hq=%d Hkv=%d d=%d (d %% 16 == 0, d <= 256, up to 65536 heads)", who, T, Hq, Hkv, d);
        return FP8_ERR_SHAPE;
    }
    if (r->rot < 0 || r->rot > d || r->rot % 16 || (r->rot && (r->n_pos == 0 || r->n_pos > 0x7FFFFFFFull)) || !(r->eps >= 0.0f) ||
        !(r->alpha - r->alpha == 0.0f)) {
        set_error("%s: unsupported rot=%d (rot %% 16 == 0, rot <= d) or n_pos=%zu, eps < 0 or alpha not finite", who, r->rot, r->n_pos);
        return FP8_ERR_SHAPE;
    }
    if (r->rot && (!r->cos_table || !r->sin_table)) {
        set_error("%s: NULL table", who);
        return FP8_ERR_NULL;
    }
    if (!aligned16(r->cos_table) || !aligned16(r->sin_table) || !aligned_to(r->positions, r->positions_are_int64 ? 8 : 4)) {
        set_error("%s: tables must be 16-byte aligned, positions to their own type", who);
        return FP8_ERR_ALIGN;
    }
    return FP8_OK;
}

static void rope_fill(RopeArgs &p, size_t T, int Hq, int Hkv, int d, const fp8_rope *r, int fmt)
{
    p.T = T;
    p.heads[0] = Hq;
    p.heads[1] = p.heads[2] = Hkv;
    p.d = d;
    p.rot = r->rot;
    p.alpha = r->alpha;
    p.eps = r->eps;
    p.inv_d = 1.0f / (float)d;
    p.cos_t = r->cos_table;
    p.sin_t = r->sin_table;
    p.n_pos = r->n_pos;
    p.positions = r->rot ? r->positions : nullptr;
    p.wide_positions = r->positions_are_int64;
    p.fmt = fmt;
}

static int rope_fwd(const char *who, const void *qkv, size_t pitch, size_t T, int Hq, int Hkv, int d, const fp8_rope *r,
                    const float *scales, int fmt, void *q, void *k, void *v, uint8_t *q8, uint8_t *k8, uint8_t *v8, float *amax_out,
                    void *stream)
{
    int rc = rope_check(who, T, Hq, Hkv, d, r);
    if (rc != FP8_OK) return rc;
    if (!qkv || !(q || k || v || q8 || k8 || v8)) {
        set_error("%s: NULL qkv, or nothing to write", who);
        return FP8_ERR_NULL;
    }
    const size_t row = ((size_t)Hq + 2 * (size_t)Hkv) * d;
    if (pitch < row || pitch % 8 || pitch > ((size_t)1 << 40)) {
        set_error("%s: pitch of %zu elements (rows of %zu, multiples of 8)", who, pitch, row);
        return FP8_ERR_SHAPE;
    }
    if (Hkv == 0 && (k || v || k8 || v8)) {
        set_error("%s: outputs of K or V without heads of them", who);
        return FP8_ERR_SHAPE;
    }
    if (!aligned16(qkv) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q8) || !aligned16(k8) || !aligned16(v8) ||
        !aligned_to(scales, 4) || !aligned_to(amax_out, 4)) {
        set_error("%s: tensor pointers must be 16-byte aligned, scales and amax_out to their type", who);
        return FP8_ERR_ALIGN;
    }
    rc = check_arch();
    if (rc != FP8_OK) return rc;
    RopeArgs p = {};
    p.qkv = static_cast<const uint16_t *>(qkv);
    p.pitch = pitch;
    rope_fill(p, T, Hq, Hkv, d, r, fmt);
    void *const out[3] = {q, k, v};
    uint8_t *const out8[3] = {q8, k8, v8};
    for (int i = 0; i < 3; ++i) {
        p.out[i] = static_cast<uint16_t *>(out[i]);
        p.out8[i] = out8[i];
    }
    p.scales = scales;
    p.amax_bits = reinterpret_cast<unsigned int *>(amax_out);
    return rope_launch<false>(p, r->mode, r->interleaved != 0, static_cast<cudaStream_t>(stream));
}

static int rope_bwd(const char *who, const void *dq, const void *dk, const void *dv, const void *qkv, size_t pitch, size_t T,
                    int Hq, int Hkv, int d, const fp8_rope *r, const float *scale, int fmt, void *dqkv, size_t out_pitch,
                    uint8_t *dqkv8, float *amax_out, void *stream)
{
    int rc = rope_check(who, T, Hq, Hkv, d, r);
    if (rc != FP8_OK) return rc;
    if (!dq || (Hkv && (!dk || !dv)) || (!qkv && r->mode != FP8_QK_NONE)) {
        set_error("%s: NULL pointer (qkv may be missing with FP8_QK_NONE alone)", who);
        return FP8_ERR_NULL;
    }
    const size_t row = ((size_t)Hq + 2 * (size_t)Hkv) * d;
    if ((qkv && (pitch < row || pitch % 8 || pitch > ((size_t)1 << 40))) ||
        (dqkv && (out_pitch < row || out_pitch % 8 || out_pitch > ((size_t)1 << 40)))) {
        set_error("%s: pitches of %zu and %zu elements (rows of %zu, multiples of 8)", who, pitch, out_pitch, row);
        return FP8_ERR_SHAPE;
    }
    if (!aligned16(dq) || !aligned16(dk) || !aligned16(dv) || !aligned16(qkv) || !aligned16(dqkv) || !aligned16(dqkv8) ||
        !aligned_to(scale, 4) || !aligned_to(amax_out, 4)) {
        set_error("%s: tensor pointers must be 16-byte aligned, scale and amax_out to their type", who);
        return FP8_ERR_ALIGN;
    }
    rc = check_arch();
    if (rc != FP8_OK) return rc;
    RopeArgs p = {};
    p.qkv = static_cast<const uint16_t *>(qkv);
    p.pitch = pitch;
    rope_fill(p, T, Hq, Hkv, d, r, fmt);
    const void *const grad[3] = {dq, dk, dv};
    for (int i = 0; i < 3; ++i) p.grad[i] = static_cast<const uint16_t *>(grad[i]);
    p.out[0] = static_cast<uint16_t *>(dqkv);
    p.out_pitch = out_pitch;
    p.out8[0] = dqkv8;
    p.scales = scale;
    p.amax_bits = reinterpret_cast<unsigned int *>(amax_out);
    return rope_launch<true>(p, r->mode, r->interleaved != 0, static_cast<cudaStream_t>(stream));
}

static int check_codes(const char *who, const void *scale, int fmt, bool any)
{
    if (!scale || !any) {
        set_error("%s: NULL scale or codes", who);
        return FP8_ERR_NULL;
    }
    if (fmt != FP8_E4M3 && fmt != FP8_E5M2) {
        set_error("%s: fmt %d is not FP8_E4M3 / FP8_E5M2", who, fmt);
        return FP8_ERR_ENUM;
    }
    return FP8_OK;
}

// A number as the sum of two doubles that do not overlap: about 2^-104 of itself.
struct Wide {
    double hi, lo;
};
static Wide wide(double a) { return {a, 0.0}; }
static Wide wide_sum(double a, double b)
{
    const double s = a + b, t = s - a;
    return {s, (a - (s - t)) + (b - t)};
}
static Wide negative(Wide a) { return {-a.hi, -a.lo}; }
static Wide operator+(Wide a, Wide b)
{
    const Wide s = wide_sum(a.hi, b.hi);
    return wide_sum(s.hi, s.lo + (a.lo + b.lo));
}
static Wide operator*(Wide a, Wide b)
{
    const double p = a.hi * b.hi;
    return wide_sum(p, fma(a.hi, b.hi, -p) + (a.hi * b.lo + a.lo * b.hi));
}
static Wide operator/(Wide a, Wide b)
{
    const double q = a.hi / b.hi;
    return wide_sum(q, (a + negative(wide(q) * b)).hi / b.hi);
}
// x^(-1 / n): Newton's iteration y + y (1 - x y^n) / n from the nearest doubles, whose error it squares.  Whole n-th powers of two
// are taken out of x first, so that no power of y leaves the doubles' range.
static Wide inverse_root(double x, int n)
{
    int e;
    x = frexp(x, &e);
    const int out = (e - (e < 0 ? n - 1 : 0)) / n;                // e / n, rounded down
    x = ldexp(x, e - n * out);
    Wide y = wide(pow(x, -1.0 / n));
    for (int i = 0; i < 2; ++i) {
        Wide product = wide(x), square = y;
        for (int k = n; k > 0; k >>= 1, square = square * square)
            if (k & 1) product = product * square;
        y = y + y * ((wide(1.0) + negative(product)) / wide(n));
    }
    return {ldexp(y.hi, -out), ldexp(y.lo, -out)};
}

}  // namespace fp8dpa

using namespace fp8dpa;

extern "C" int fp8_rope_table(size_t n_pos, int rot, double base, int scaling, double factor, double original_len, double turns_low,
                              double turns_high, double magnitude, float *cos_table, float *sin_table, void *stream)
{
    if (!cos_table || !sin_table) {
        set_error("fp8_rope_table: NULL table");
        return FP8_ERR_NULL;
    }
    if (scaling < FP8_ROPE_PLAIN || scaling > FP8_ROPE_BY_PARTS) {
        set_error("fp8_rope_table: scaling %d is not a known enum value", scaling);
        return FP8_ERR_ENUM;
    }
    const bool scaled = scaling != FP8_ROPE_PLAIN, parts = scaling == FP8_ROPE_BY_PARTS;
    if (n_pos == 0 || n_pos > 0x7FFFFFFFull || rot <= 0 || rot % 16 || rot > 2 * ROPE_MAX_PAIRS || !(base > 0.0) || isinf(base) ||
        !(magnitude > 0.0) || isinf((float)magnitude) || (scaled && (!(factor > 0.0) || isinf(factor))) ||
        (parts && (!(original_len > 0.0) || isinf(original_len) || !(turns_high > turns_low) || isinf(turns_high) || isinf(turns_low)))) {
        set_error("fp8_rope_table: unsupported n_pos=%zu rot=%d (rot %% 16 == 0, rot <= 256) or a parameter that is not a positive "
                  "number", n_pos, rot);
        return FP8_ERR_SHAPE;
    }
    if (!aligned16(cos_table) || !aligned16(sin_table)) {
        set_error("fp8_rope_table: tables must be 16-byte aligned");
        return FP8_ERR_ALIGN;
    }
    RopeTable t = {};
    // Turns per position: powers of one ratio, of which 127 products in a row leave less than 2^-90 of error (positions below 2^31 need
    // that next to zeros).
    const Wide one = wide(1.0), share = scaling == FP8_ROPE_LINEAR || parts ? one / wide(factor) : one;
    const Wide span = parts ? one / wide_sum(turns_high, -turns_low) : one;
    Wide f = {0.15915494309189535, -9.839338337591243e-18}, ratio = inverse_root(base, rot / 2);             // 1 / 2 pi
    if (scaling == FP8_ROPE_NTK) ratio = ratio * inverse_root(factor, (rot - 2) / 2);      // factor^(-2 / (rot - 2))
    if (scaling == FP8_ROPE_LINEAR) f = f * share;
    bool too_many = false;
    for (int i = 0; i < rot / 2; ++i, f = f * ratio) {
        Wide turns = f;
        if (parts) {
            const Wide w = (f * wide(original_len) + wide(-turns_low)) * span;
            if (w.hi <= 0.0) turns = f * share;
            else if (!(w.hi >= 1.0)) turns = (one + negative(w)) * f * share + w * f;
        }
        t.turns[i] = turns.hi;
        t.rest[i] = turns.lo;
        too_many |= !(turns.hi * (double)n_pos <= 2147483648.0);
    }
    if (too_many) {
        set_error("fp8_rope_table: base=%g and factor=%g make more than 2^31 turns in %zu positions", base, factor, n_pos);
        return FP8_ERR_SHAPE;
    }
    int rc = check_arch();
    if (rc != FP8_OK) return rc;
    t.cos_t = cos_table;
    t.sin_t = sin_table;
    t.rows = n_pos;
    t.pairs = rot / 2;
    t.magnitude = (float)magnitude;
    const size_t wide = 256 / (rot / 8), want = (n_pos + wide - 1) / wide;       // positions of a CTA at a time
    rope_table_kernel<<<(unsigned)(want < 148 * 8 ? want : 148 * 8), 256, 0, static_cast<cudaStream_t>(stream)>>>(t);
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
}

extern "C" int fp8_rope_qkv_fwd(const void *qkv_bf16, size_t pitch, size_t T, int Hq, int Hkv, int d, const fp8_rope *rope,
                                void *q_bf16, void *k_bf16, void *v_bf16, float *amax_out, void *stream)
{
    return rope_fwd("fp8_rope_qkv_fwd", qkv_bf16, pitch, T, Hq, Hkv, d, rope, nullptr, 0, q_bf16, k_bf16, v_bf16, nullptr, nullptr,
                    nullptr, amax_out, stream);
}

extern "C" int fp8_rope_qkv_fwd_q(const void *qkv_bf16, size_t pitch, size_t T, int Hq, int Hkv, int d, const fp8_rope *rope,
                                  const float *scales, int fmt, void *q_bf16, void *k_bf16, void *v_bf16, uint8_t *q8, uint8_t *k8,
                                  uint8_t *v8, float *amax_out, void *stream)
{
    const int rc = check_codes("fp8_rope_qkv_fwd_q", scales, fmt, q8 || k8 || v8);
    if (rc != FP8_OK) return rc;
    return rope_fwd("fp8_rope_qkv_fwd_q", qkv_bf16, pitch, T, Hq, Hkv, d, rope, scales, fmt, q_bf16, k_bf16, v_bf16, q8, k8, v8,
                    amax_out, stream);
}

extern "C" int fp8_rope_qkv_bwd(const void *dq_bf16, const void *dk_bf16, const void *dv_bf16, const void *qkv_bf16, size_t pitch,
                                size_t T, int Hq, int Hkv, int d, const fp8_rope *rope, void *dqkv_bf16, size_t dqkv_pitch,
                                float *amax_out, void *stream)
{
    if (!dqkv_bf16) {
        set_error("fp8_rope_qkv_bwd: NULL dqkv");
        return FP8_ERR_NULL;
    }
    return rope_bwd("fp8_rope_qkv_bwd", dq_bf16, dk_bf16, dv_bf16, qkv_bf16, pitch, T, Hq, Hkv, d, rope, nullptr, 0, dqkv_bf16,
                    dqkv_pitch, nullptr, amax_out, stream);
}

extern "C" int fp8_rope_qkv_bwd_q(const void *dq_bf16, const void *dk_bf16, const void *dv_bf16, const void *qkv_bf16, size_t pitch,
                                  size_t T, int Hq, int Hkv, int d, const fp8_rope *rope, const float *scale, int fmt,
                                  void *dqkv_bf16, size_t dqkv_pitch, uint8_t *dqkv8, float *amax_out, void *stream)
{
    const int rc = check_codes("fp8_rope_qkv_bwd_q", scale, fmt, dqkv8 != nullptr);
    if (rc != FP8_OK) return rc;
    return rope_bwd("fp8_rope_qkv_bwd_q", dq_bf16, dk_bf16, dv_bf16, qkv_bf16, pitch, T, Hq, Hkv, d, rope, scale, fmt, dqkv_bf16,
                    dqkv_pitch, dqkv8, amax_out, stream);
}
