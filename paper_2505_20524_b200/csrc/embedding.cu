// Token embedding: out[t] = scale * table[id_t] (with the amax and the FP8 codes of the result, the operand of the next
// product in a block without pre-normalisation), and the gradient of the table by sorted tokens.
//
// Gradient.  dW[v] = scale * sum over the positions t with id_t = v of dy[t], summed in FP32 in ascending t.  The positions
// are put in the order of their ids by a stable counting sort of the id's digits, so that equal ids are neighbours and
// every row of dy is read once; no floating-point atomics, the result does not depend on the order in which blocks run.
#include <math.h>

#include "common.cuh"
#include "elementwise.cuh"
#include "stable_rank.cuh"

namespace fp8dpa {

// ---------------------------------------------------------------- forward
constexpr int EF_THREADS = 256;
constexpr int EF_ROWS = 4;       // table rows in flight per thread

template <typename IdT>
__device__ __forceinline__ int checked_id(const IdT *ids, size_t t, unsigned V)
{
    const IdT id = __ldg(ids + t);
    return id >= 0 && (unsigned long long)id < (unsigned long long)V ? (int)id : -1;
}

// `lanes` (a power of two) threads share a row; a CTA has 256 / lanes row slots with EF_ROWS rows each.  Bound by HBM:
// every thread keeps EF_ROWS 16-byte loads (32 bytes from an FP32 table) in flight.
template <typename IdT, bool F32>
__global__ void __launch_bounds__(EF_THREADS) embedding_fwd_kernel(const void *__restrict__ table, const IdT *__restrict__ ids,
                                                                   size_t T, unsigned V, unsigned n8, float scale,
                                                                   uint16_t *__restrict__ out,
                                                                   unsigned int *__restrict__ amax_bits,
                                                                   const float *__restrict__ q_scale,
                                                                   uint8_t *__restrict__ out8, int fmt, int lanes_log2)
{
    const float qs = out8 ? __ldg(q_scale) : 1.0f;
    const int lane = threadIdx.x & ((1 << lanes_log2) - 1), slot = threadIdx.x >> lanes_log2;
    const int slots = EF_THREADS >> lanes_log2;
    const size_t row0 = (size_t)blockIdx.x * (slots * EF_ROWS) + slot;
    int id[EF_ROWS];
#pragma unroll
    for (int j = 0; j < EF_ROWS; ++j) {
        const size_t t = row0 + (size_t)j * slots;
        id[j] = t < T ? checked_id(ids, t, V) : -1;
    }
    uint32_t m = 0;
    for (unsigned c = lane; c < n8; c += 1u << lanes_log2) {
        uint32_t w[EF_ROWS][4];
        if (F32) {
            float4 a[EF_ROWS], b[EF_ROWS];
#pragma unroll
            for (int j = 0; j < EF_ROWS; ++j) {
                a[j] = b[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (id[j] >= 0) {
                    const float4 *p = static_cast<const float4 *>(table) + 2 * ((size_t)id[j] * n8 + c);
                    a[j] = __ldg(p);
                    b[j] = __ldg(p + 1);
                }
            }
#pragma unroll
            for (int j = 0; j < EF_ROWS; ++j) {
                w[j][0] = pack_bf16x2(a[j].x * scale, a[j].y * scale);
                w[j][1] = pack_bf16x2(a[j].z * scale, a[j].w * scale);
                w[j][2] = pack_bf16x2(b[j].x * scale, b[j].y * scale);
                w[j][3] = pack_bf16x2(b[j].z * scale, b[j].w * scale);
            }
        } else {
            uint4 v[EF_ROWS];
#pragma unroll
            for (int j = 0; j < EF_ROWS; ++j) {
                v[j] = make_uint4(0u, 0u, 0u, 0u);
                if (id[j] >= 0) v[j] = __ldg(static_cast<const uint4 *>(table) + (size_t)id[j] * n8 + c);
            }
#pragma unroll
            for (int j = 0; j < EF_ROWS; ++j) {
                const uint32_t u[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                for (int q = 0; q < 4; ++q) w[j][q] = pack_bf16x2(bf16_lo(u[q]) * scale, bf16_hi(u[q]) * scale);
            }
        }
#pragma unroll
        for (int j = 0; j < EF_ROWS; ++j) {
            const size_t t = row0 + (size_t)j * slots;
            if (t >= T) continue;
            if (id[j] < 0) w[j][0] = w[j][1] = w[j][2] = w[j][3] = 0u;       // also for an infinite or NaN scale
#pragma unroll
            for (int q = 0; q < 4; ++q) m = absmax2e(m, w[j][q]);
            const size_t at = t * n8 + c;
            if (out) reinterpret_cast<uint4 *>(out)[at] = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
            if (out8) reinterpret_cast<uint2 *>(out8)[at] = bf16x8_to_fp8x8(w[j], qs, fmt);
        }
    }
    if (amax_bits) block_max_bf16_to(m, amax_bits);
}

// ---------------------------------------------------------------- gradient: order of the tokens
// Sort keys: the id, or V for a position whose id lies outside [0, V) (so those come last).  Digits of up to 10 bits,
// least significant first; a chunk is the run of positions one CTA ranks.
constexpr int ES_THREADS = 256;
constexpr int ES_WARPS = ES_THREADS / 32;
constexpr int ES_ITEMS = 8;                          // keys per thread and tile
constexpr int ES_TILE = ES_THREADS * ES_ITEMS;
constexpr int ES_MAX_BITS = 10;
constexpr int ES_MAX_DIGITS = 1 << ES_MAX_BITS;
constexpr int ES_MAX_CHUNKS = 256;                   // every scattering CTA sums up to this many rows of the count table

struct SortPlan {
    int passes, bits;                                // digit width
    size_t chunk_tiles, chunks;
};
static SortPlan sort_plan(size_t T, size_t V)
{
    SortPlan p;
    int total = 1;
    while (total < 32 && (V >> total)) ++total;      // bits of the largest key, V
    p.passes = (total + ES_MAX_BITS - 1) / ES_MAX_BITS;
    p.bits = (total + p.passes - 1) / p.passes;
    const size_t tiles = (T + ES_TILE - 1) / ES_TILE;
    p.chunk_tiles = (tiles + ES_MAX_CHUNKS - 1) / ES_MAX_CHUNKS;
    p.chunks = (tiles + p.chunk_tiles - 1) / p.chunk_tiles;
    return p;
}

// Counts of the first digit per chunk, the keys themselves, and a mark on every row of the table that is touched.
template <typename IdT>
__global__ void __launch_bounds__(ES_THREADS) embedding_count_kernel(const IdT *__restrict__ ids, size_t T, unsigned V,
                                                                     unsigned chunk_len, int bits, uint32_t *__restrict__ keys,
                                                                     int *__restrict__ table, uint8_t *__restrict__ touched)
{
    __shared__ int cnt[ES_MAX_DIGITS];
    const int digits = 1 << bits;
    for (int d = threadIdx.x; d < digits; d += ES_THREADS) cnt[d] = 0;
    __syncthreads();
    const size_t t0 = (size_t)blockIdx.x * chunk_len, t1 = min(T, t0 + chunk_len);
    for (size_t t = t0 + threadIdx.x; t < t1; t += ES_THREADS) {
        const int id = checked_id(ids, t, V);
        const uint32_t key = id < 0 ? V : (uint32_t)id;
        keys[t] = key;
        if (touched && id >= 0) touched[id] = 1;
        atomicAdd(&cnt[key & (digits - 1)], 1);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += ES_THREADS) table[(size_t)blockIdx.x * digits + d] = cnt[d];
}

// One stable pass: chunk b's keys go to the places that the counts of all chunks give, and the next digit is counted per
// chunk of the new order.  pos_in == NULL: the positions are 0, 1, 2, ...
__device__ __forceinline__ void sort_scatter(const uint32_t *__restrict__ keys, const int *__restrict__ pos_in, size_t T,
                                             unsigned chunk_len, unsigned chunks, unsigned chunk, int bits, int shift,
                                             const int *__restrict__ table, uint32_t *__restrict__ keys_out,
                                             int *__restrict__ pos_out, int *__restrict__ next_table)
{
    __shared__ int warp_cnt[ES_WARPS][ES_MAX_DIGITS];
    __shared__ int base[ES_MAX_DIGITS];
    __shared__ int warp_sum[ES_WARPS];
    const int digits = 1 << bits, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // where this chunk's keys of digit d start: keys of smaller digits, then those of d in earlier chunks
    const int per = (digits + ES_THREADS - 1) / ES_THREADS;      // digits per thread: tid * per ...
    int total[ES_MAX_DIGITS / ES_THREADS], mine[ES_MAX_DIGITS / ES_THREADS], sum = 0;
#pragma unroll
    for (int q = 0; q < ES_MAX_DIGITS / ES_THREADS; ++q) {
        total[q] = mine[q] = 0;
        const int d = tid * per + q;
        if (q < per && d < digits) {
#pragma unroll 4
            for (unsigned c = 0; c < chunks; ++c) {
                const int v = __ldcg(table + (size_t)c * digits + d);
                if (c < chunk) mine[q] += v;
                total[q] += v;
            }
            sum += total[q];
        }
    }
    int scan = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, scan, off);
        if (lane >= off) scan += v;
    }
    if (lane == 31) warp_sum[warp] = scan;
    __syncthreads();
    int start = scan - sum;
    for (int w = 0; w < warp; ++w) start += warp_sum[w];
#pragma unroll
    for (int q = 0; q < ES_MAX_DIGITS / ES_THREADS; ++q) {
        const int d = tid * per + q;
        if (q < per && d < digits) {
            base[d] = start + mine[q];
            start += total[q];
        }
    }
    const size_t t0 = (size_t)chunk * chunk_len, t1 = min(T, t0 + chunk_len);
    for (size_t tile = t0; tile < t1; tile += ES_TILE) {
        for (int i = tid; i < ES_WARPS * digits; i += ES_THREADS) warp_cnt[i >> bits][i & (digits - 1)] = 0;
        __syncthreads();
        uint32_t key[ES_ITEMS];
        int pos[ES_ITEMS], rank[ES_ITEMS];
#pragma unroll
        for (int j = 0; j < ES_ITEMS; ++j) {
            const size_t i = tile + (size_t)warp * (32 * ES_ITEMS) + j * 32 + lane;
            key[j] = i < t1 ? __ldcg(keys + i) : 0xFFFFFFFFu;
            pos[j] = i < t1 ? (pos_in ? __ldcg(pos_in + i) : (int)i) : -1;
        }
#pragma unroll
        for (int j = 0; j < ES_ITEMS; ++j)
            rank[j] = warp_stable_rank(pos[j] >= 0 ? (int)((key[j] >> shift) & (digits - 1)) : -1, warp_cnt[warp], lane);
        __syncthreads();
        for (int d = tid; d < digits; d += ES_THREADS) {         // the warps' counts become their starts
            int at = base[d];
#pragma unroll
            for (int w = 0; w < ES_WARPS; ++w) {
                const int v = warp_cnt[w][d];
                warp_cnt[w][d] = at;
                at += v;
            }
            base[d] = at;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < ES_ITEMS; ++j) {
            if (pos[j] < 0) continue;
            const int to = warp_cnt[warp][(key[j] >> shift) & (digits - 1)] + rank[j];
            keys_out[to] = key[j];
            pos_out[to] = pos[j];
            if (next_table) atomicAdd(next_table + (size_t)((unsigned)to / chunk_len) * digits + ((key[j] >> (shift + bits)) & (digits - 1)), 1);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- gradient: rows of zeros
// Rows [v0, v1) of the table that no token touches.
__device__ __forceinline__ void fill_rows(uint8_t *__restrict__ dtable, size_t row_bytes, const uint8_t *__restrict__ touched,
                                          size_t v0, size_t v1)
{
    for (size_t v = v0; v < v1; ++v) {
        if (__ldcg(touched + v)) continue;
        uint4 *row = reinterpret_cast<uint4 *>(dtable + v * row_bytes);
        for (size_t c = threadIdx.x; c < row_bytes / 16; c += blockDim.x) row[c] = make_uint4(0u, 0u, 0u, 0u);
    }
}

__global__ void __launch_bounds__(ES_THREADS) embedding_scatter_kernel(const uint32_t *__restrict__ keys,
                                                                       const int *__restrict__ pos_in, size_t T,
                                                                       unsigned chunk_len, unsigned chunks, int bits, int shift,
                                                                       const int *__restrict__ table,
                                                                       uint32_t *__restrict__ keys_out,
                                                                       int *__restrict__ pos_out, int *__restrict__ next_table)
{
    sort_scatter(keys, pos_in, T, chunk_len, chunks, blockIdx.x, bits, shift, table, keys_out, pos_out, next_table);
}

// ---------------------------------------------------------------- gradient: sums
constexpr int EG_THREADS = 256;
constexpr int EG_RUN = 32;          // sorted positions per work item
constexpr int EG_UNROLL = 4;        // rows of dy in flight per thread
constexpr int EG_JOIN = 4;          // partial sums in flight per thread

struct GradParams {
    const uint16_t *dy;
    const uint32_t *keys;
    const int *pos;
    size_t T;
    unsigned V, n8;
    float scale;
    void *dtable;
    int is_fp32, accumulate, lanes_log2;
    float *partial;                  // [items][2][D]: sums of the item's first and last run where they cross its ends
    size_t items, item_blocks, col_blocks;
    const uint8_t *touched;
    size_t fill_rows_per_block;
};

__device__ __forceinline__ void store_row8(const GradParams &p, uint32_t v, unsigned c, const float (&acc)[8])
{
    const size_t at = (size_t)v * p.n8 + c;
    float r[8];
    if (p.is_fp32) {
        float4 *o = static_cast<float4 *>(p.dtable) + 2 * at;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (p.accumulate) { a = o[0]; b = o[1]; }
        o[0] = make_float4(fmaf(acc[0], p.scale, a.x), fmaf(acc[1], p.scale, a.y), fmaf(acc[2], p.scale, a.z), fmaf(acc[3], p.scale, a.w));
        o[1] = make_float4(fmaf(acc[4], p.scale, b.x), fmaf(acc[5], p.scale, b.y), fmaf(acc[6], p.scale, b.z), fmaf(acc[7], p.scale, b.w));
    } else {
        uint4 *o = static_cast<uint4 *>(p.dtable) + at;
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (p.accumulate) u = *o;
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            r[2 * q] = fmaf(acc[2 * q], p.scale, bf16_lo(w[q]));
            r[2 * q + 1] = fmaf(acc[2 * q + 1], p.scale, bf16_hi(w[q]));
        }
        *o = make_uint4(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]), pack_bf16x2(r[4], r[5]), pack_bf16x2(r[6], r[7]));
    }
}

// Work item: EG_RUN neighbouring sorted positions, for the columns of one thread group (`lanes` threads, 8 columns each).
// A run of equal ids that lies inside the item is finished here; one that crosses the item's start or end leaves its sum
// in `partial` and is finished by embedding_join_kernel.  Blocks past the items write the untouched rows' zeros.
__global__ void __launch_bounds__(EG_THREADS) embedding_sum_kernel(const GradParams p)
{
    const size_t work_blocks = p.item_blocks * p.col_blocks;
    if (blockIdx.x >= work_blocks) {
        const size_t v0 = (blockIdx.x - work_blocks) * p.fill_rows_per_block;
        fill_rows(static_cast<uint8_t *>(p.dtable), (size_t)p.n8 * (p.is_fp32 ? 32 : 16), p.touched, v0,
                  min((size_t)p.V, v0 + p.fill_rows_per_block));
        return;
    }
    const int lanes = 1 << p.lanes_log2;
    const size_t item = (blockIdx.x / p.col_blocks) * (EG_THREADS >> p.lanes_log2) + (threadIdx.x >> p.lanes_log2);
    const unsigned c = (unsigned)(blockIdx.x % p.col_blocks) * lanes + (threadIdx.x & (lanes - 1));
    if (item >= p.items || c >= p.n8) return;
    const size_t i0 = item * EG_RUN, i1 = min(p.T, i0 + EG_RUN);
    const uint32_t first = __ldg(p.keys + i0);
    if (first >= p.V) return;                                   // padded positions: sorted behind every id
    const bool from_before = i0 > 0 && __ldg(p.keys + i0 - 1) == first;
    uint32_t cur = first;
    bool head = from_before;                                    // the current run began before this item
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const size_t D = (size_t)p.n8 * 8;
    for (size_t i = i0; i < i1; i += EG_UNROLL) {
        uint32_t key[EG_UNROLL];
        uint4 v[EG_UNROLL];
#pragma unroll
        for (int j = 0; j < EG_UNROLL; ++j) {
            key[j] = i + j < i1 ? __ldg(p.keys + i + j) : 0xFFFFFFFFu;
            if (key[j] < p.V) v[j] = __ldg(reinterpret_cast<const uint4 *>(p.dy) + (size_t)__ldg(p.pos + i + j) * p.n8 + c);
        }
#pragma unroll
        for (int j = 0; j < EG_UNROLL; ++j) {
            if (key[j] != cur && cur < p.V) {                    // the run ends
                if (head) {
                    float *o = p.partial + (item * 2) * D + (size_t)c * 8;
                    *reinterpret_cast<float4 *>(o) = make_float4(acc[0], acc[1], acc[2], acc[3]);
                    *reinterpret_cast<float4 *>(o + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
                } else if (i + j < i1 || i1 == p.T || __ldg(p.keys + i1) != cur) {
                    store_row8(p, cur, c, acc);
                } else {                                         // began here, goes on in the next item
                    float *o = p.partial + (item * 2 + 1) * D + (size_t)c * 8;
                    *reinterpret_cast<float4 *>(o) = make_float4(acc[0], acc[1], acc[2], acc[3]);
                    *reinterpret_cast<float4 *>(o + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
                head = false;
            }
            cur = key[j];
            if (cur < p.V) {
                const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    acc[2 * q] += bf16_lo(w[q]);
                    acc[2 * q + 1] += bf16_hi(w[q]);
                }
            }
        }
    }
    if (cur < p.V) {                                             // the item is full and its last run still open
        const bool goes_on = i1 < p.T && __ldg(p.keys + i1) == cur;
        if (head || goes_on) {
            float *o = p.partial + (item * 2 + (head ? 0 : 1)) * D + (size_t)c * 8;
            *reinterpret_cast<float4 *>(o) = make_float4(acc[0], acc[1], acc[2], acc[3]);
            *reinterpret_cast<float4 *>(o + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
        } else {
            store_row8(p, cur, c, acc);
        }
    }
}

// The runs that cross items: the item in which such a run begins adds the following items' sums in order.
__global__ void __launch_bounds__(EG_THREADS) embedding_join_kernel(const GradParams p)
{
    const int lanes = 1 << p.lanes_log2;
    const size_t item = (blockIdx.x / p.col_blocks) * (EG_THREADS >> p.lanes_log2) + (threadIdx.x >> p.lanes_log2);
    const unsigned c = (unsigned)(blockIdx.x % p.col_blocks) * lanes + (threadIdx.x & (lanes - 1));
    if (item + 1 >= p.items || c >= p.n8) return;
    const size_t i1 = (item + 1) * EG_RUN;
    const uint32_t key = __ldg(p.keys + i1 - 1);
    if (key >= p.V || __ldg(p.keys + i1) != key) return;                       // nothing goes on
    const size_t i0 = item * EG_RUN;
    if (__ldg(p.keys + i0) == key && i0 > 0 && __ldg(p.keys + i0 - 1) == key) return;   // it began earlier
    const size_t D = (size_t)p.n8 * 8;
    const float *src = p.partial + (item * 2 + 1) * D + (size_t)c * 8;
    const float4 a = __ldcg(reinterpret_cast<const float4 *>(src)), b = __ldcg(reinterpret_cast<const float4 *>(src) + 1);
    float acc[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    // the following items that the run reaches, EG_JOIN of them in flight at a time (loads past the run's end are unused)
    bool open = true;
    for (size_t k = item + 1; open && k < p.items; k += EG_JOIN) {
        float4 lo[EG_JOIN], hi[EG_JOIN];
        uint32_t at[EG_JOIN];
#pragma unroll
        for (int j = 0; j < EG_JOIN; ++j) {
            at[j] = 0xFFFFFFFFu;
            if (k + j >= p.items) continue;
            at[j] = __ldg(p.keys + (k + j) * EG_RUN);
            const float4 *q = reinterpret_cast<const float4 *>(p.partial + ((k + j) * 2) * D + (size_t)c * 8);
            lo[j] = __ldcg(q);
            hi[j] = __ldcg(q + 1);
        }
#pragma unroll
        for (int j = 0; j < EG_JOIN; ++j) {
            open = open && at[j] == key;
            if (!open) continue;
            acc[0] += lo[j].x; acc[1] += lo[j].y; acc[2] += lo[j].z; acc[3] += lo[j].w;
            acc[4] += hi[j].x; acc[5] += hi[j].y; acc[6] += hi[j].z; acc[7] += hi[j].w;
        }
    }
    store_row8(p, key, c, acc);
}

// ---------------------------------------------------------------- workspace of the gradient
struct GradWs {
    size_t keys0, keys1, pos0, pos1, table, touched, zero_bytes, partial, bytes;   // offsets; [table, table + zero_bytes) starts at zero
};
static GradWs grad_ws(size_t T, size_t V, size_t D)
{
    const SortPlan sp = sort_plan(T, V);
    const auto up = [](size_t b) { return (b + 255) & ~(size_t)255; };
    GradWs w;
    size_t at = 0;
    w.keys0 = at; at += up(T * 4);
    w.keys1 = at; at += up(T * 4);
    w.pos0 = at; at += up(T * 4);
    w.pos1 = at; at += up(T * 4);
    w.table = at; at += up((size_t)sp.passes * sp.chunks * ((size_t)4 << sp.bits));
    w.touched = at; at += up(V);
    w.zero_bytes = at - w.table;
    w.partial = at; at += up((T + EG_RUN - 1) / EG_RUN * 2 * D * sizeof(float));
    w.bytes = at;
    return w;
}

static int lanes_log2_for(size_t n8, int most)
{
    int l = 0;
    while (l < most && ((size_t)1 << l) < n8) ++l;
    return l;
}

}  // namespace fp8dpa

using namespace fp8dpa;

static bool embedding_shape_ok(size_t T, size_t V, size_t D)
{
    return T > 0 && V > 0 && D > 0 && D % 8 == 0 && T <= ((size_t)1 << 30) && V <= ((size_t)1 << 30) && D <= ((size_t)1 << 20);
}

static int embedding_fwd(const char *who, const void *table, int table_is_fp32, size_t V, size_t D, const void *ids,
                         int ids_are_int64, size_t T, float scale, const float *q_scale, int fmt, void *out_bf16,
                         uint8_t *out8, float *amax_out, void *stream)
{
    if (!table || !ids || (!out_bf16 && !out8)) {
        set_error("%s: NULL pointer", who);
        return FP8_ERR_NULL;
    }
    if (out8 && fmt != FP8_E4M3 && fmt != FP8_E5M2) {
        set_error("%s: fmt %d is not FP8_E4M3 / FP8_E5M2", who, fmt);
        return FP8_ERR_ENUM;
    }
    if (!embedding_shape_ok(T, V, D)) {
        set_error("%s: unsupported shape T=%zu V=%zu D=%zu (D %% 8 == 0, D <= 2^20, T and V <= 2^30)", who, T, V, D);
        return FP8_ERR_SHAPE;
    }
    if (!aligned16(table) || !aligned16(ids) || !aligned16(out_bf16) || !aligned16(out8)) {
        set_error("%s: pointers must be 16-byte aligned", who);
        return FP8_ERR_ALIGN;
    }
    int rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (amax_out) FP8_CUDA_CHECK(cudaMemsetAsync(amax_out, 0, sizeof(float), st));
    const unsigned n8 = (unsigned)(D / 8);
    const int ll = lanes_log2_for(n8, 8);
    const size_t per_block = (size_t)(EF_THREADS >> ll) * EF_ROWS;
    const unsigned blocks = (unsigned)((T + per_block - 1) / per_block);
    uint16_t *o = static_cast<uint16_t *>(out_bf16);
    unsigned int *ab = reinterpret_cast<unsigned int *>(amax_out);
#define FP8DPA_LAUNCH_EF(IdT, F32) \
    embedding_fwd_kernel<IdT, F32><<<blocks, EF_THREADS, 0, st>>>(table, static_cast<const IdT *>(ids), T, (unsigned)V, n8, \
                                                                  scale, o, ab, q_scale, out8, fmt, ll)
    if (ids_are_int64) {
        if (table_is_fp32) FP8DPA_LAUNCH_EF(long long, true);
        else FP8DPA_LAUNCH_EF(long long, false);
    } else {
        if (table_is_fp32) FP8DPA_LAUNCH_EF(int, true);
        else FP8DPA_LAUNCH_EF(int, false);
    }
#undef FP8DPA_LAUNCH_EF
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
}

extern "C" int fp8_embedding_fwd(const void *table, int table_is_fp32, size_t V, size_t D, const void *ids,
                                 int ids_are_int64, size_t T, float scale, void *out_bf16, float *amax_out, void *stream)
{
    return embedding_fwd("fp8_embedding_fwd", table, table_is_fp32, V, D, ids, ids_are_int64, T, scale, nullptr, 0, out_bf16,
                         nullptr, amax_out, stream);
}

extern "C" int fp8_embedding_fwd_q(const void *table, int table_is_fp32, size_t V, size_t D, const void *ids,
                                   int ids_are_int64, size_t T, float scale, const float *q_scale, int fmt, void *out_bf16,
                                   uint8_t *out8, float *amax_out, void *stream)
{
    if (!out8 || !q_scale) {
        set_error("fp8_embedding_fwd_q: NULL q_scale / out8");
        return FP8_ERR_NULL;
    }
    return embedding_fwd("fp8_embedding_fwd_q", table, table_is_fp32, V, D, ids, ids_are_int64, T, scale, q_scale, fmt,
                         out_bf16, out8, amax_out, stream);
}

extern "C" size_t fp8_embedding_bwd_workspace_bytes(size_t T, size_t V, size_t D)
{
    return embedding_shape_ok(T, V, D) ? grad_ws(T, V, D).bytes : 0;
}

extern "C" int fp8_embedding_bwd(const void *dy_bf16, const void *ids, int ids_are_int64, size_t T, size_t V, size_t D,
                                 float scale, void *dtable, int out_is_fp32, int accumulate, void *ws, size_t ws_bytes,
                                 void *stream)
{
    if (!dy_bf16 || !ids || !dtable) {
        set_error("fp8_embedding_bwd: NULL pointer");
        return FP8_ERR_NULL;
    }
    if (!embedding_shape_ok(T, V, D)) {
        set_error("fp8_embedding_bwd: unsupported shape T=%zu V=%zu D=%zu (D %% 8 == 0, D <= 2^20, T and V <= 2^30)", T, V, D);
        return FP8_ERR_SHAPE;
    }
    if (!aligned16(dy_bf16) || !aligned16(ids) || !aligned16(dtable)) {
        set_error("fp8_embedding_bwd: pointers must be 16-byte aligned");
        return FP8_ERR_ALIGN;
    }
    const GradWs w = grad_ws(T, V, D);
    if (!ws || ws_bytes < w.bytes || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("fp8_embedding_bwd: workspace of %zu bytes, 256-byte aligned, needed (got %zu)", w.bytes, ws_bytes);
        return FP8_ERR_WORKSPACE;
    }
    int rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t *base = static_cast<uint8_t *>(ws);
    uint32_t *keys[2] = {reinterpret_cast<uint32_t *>(base + w.keys0), reinterpret_cast<uint32_t *>(base + w.keys1)};
    int *pos[2] = {reinterpret_cast<int *>(base + w.pos0), reinterpret_cast<int *>(base + w.pos1)};
    int *table = reinterpret_cast<int *>(base + w.table);
    uint8_t *touched = base + w.touched;
    const SortPlan sp = sort_plan(T, V);
    const unsigned chunk_len = (unsigned)(sp.chunk_tiles * ES_TILE), chunks = (unsigned)sp.chunks;
    const size_t table_len = sp.chunks << sp.bits;
    FP8_CUDA_CHECK(cudaMemsetAsync(table, 0, w.zero_bytes, st));
    if (ids_are_int64)
        embedding_count_kernel<long long><<<chunks, ES_THREADS, 0, st>>>(
            static_cast<const long long *>(ids), T, (unsigned)V, chunk_len, sp.bits, keys[0], table, accumulate ? nullptr : touched);
    else
        embedding_count_kernel<int><<<chunks, ES_THREADS, 0, st>>>(
            static_cast<const int *>(ids), T, (unsigned)V, chunk_len, sp.bits, keys[0], table, accumulate ? nullptr : touched);
    FP8_CUDA_CHECK(cudaGetLastError());
    for (int i = 0; i < sp.passes; ++i) {
        embedding_scatter_kernel<<<chunks, ES_THREADS, 0, st>>>(
            keys[i & 1], i ? pos[i & 1] : nullptr, T, chunk_len, chunks, sp.bits, i * sp.bits, table + i * table_len,
            keys[(i + 1) & 1], pos[(i + 1) & 1], i + 1 < sp.passes ? table + (i + 1) * table_len : nullptr);
        FP8_CUDA_CHECK(cudaGetLastError());
    }
    GradParams p;
    p.dy = static_cast<const uint16_t *>(dy_bf16);
    p.keys = keys[sp.passes & 1];
    p.pos = pos[sp.passes & 1];
    p.T = T;
    p.V = (unsigned)V;
    p.n8 = (unsigned)(D / 8);
    p.scale = scale;
    p.dtable = dtable;
    p.is_fp32 = out_is_fp32 ? 1 : 0;
    p.accumulate = accumulate ? 1 : 0;
    p.lanes_log2 = lanes_log2_for(p.n8, 8);
    p.partial = reinterpret_cast<float *>(base + w.partial);
    p.items = (T + EG_RUN - 1) / EG_RUN;
    const size_t slots = EG_THREADS >> p.lanes_log2;
    p.item_blocks = (p.items + slots - 1) / slots;
    p.col_blocks = (p.n8 + (1u << p.lanes_log2) - 1) >> p.lanes_log2;
    p.touched = touched;
    const size_t row_bytes = D * (out_is_fp32 ? 4 : 2);
    p.fill_rows_per_block = row_bytes >= 65536 ? 1 : 65536 / row_bytes;
    const size_t work = p.item_blocks * p.col_blocks;
    const size_t fill = accumulate ? 0 : (V + p.fill_rows_per_block - 1) / p.fill_rows_per_block;
    if (work + fill > 0x7FFFFFFFull) {
        set_error("fp8_embedding_bwd: T=%zu V=%zu D=%zu needs more blocks than a grid holds", T, V, D);
        return FP8_ERR_SHAPE;
    }
    embedding_sum_kernel<<<(unsigned)(work + fill), EG_THREADS, 0, st>>>(p);
    FP8_CUDA_CHECK(cudaGetLastError());
    if (p.items > 1) {
        embedding_join_kernel<<<(unsigned)work, EG_THREADS, 0, st>>>(p);
        FP8_CUDA_CHECK(cudaGetLastError());
    }
    return FP8_OK;
}
