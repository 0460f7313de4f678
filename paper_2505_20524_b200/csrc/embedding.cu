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
// every thread keeps EF_ROWS 16-byte loads (32 bytes from an FP32 table) in flight.  8192 tokens x 4096 with codes and amax:
// 25.1 us (100 MB written, 32 MB of distinct rows read); 1, 2 and 4 rows and 128 threads are within 4 % of it.
struct EmbedFwd {
    const void *table, *ids;
    size_t T;
    unsigned V, n8;
    float scale;
    uint16_t *out;
    unsigned int *amax_bits;
    const float *q_scale;
    uint8_t *out8;
    int fmt;
};
template <typename IdT, bool F32>
__global__ void __launch_bounds__(EF_THREADS) embedding_fwd_kernel(const EmbedFwd p, int lanes_log2)
{
    const bool alone = amax_begin(p.amax_bits);
    const void *__restrict__ table = p.table;
    const IdT *__restrict__ ids = static_cast<const IdT *>(p.ids);
    uint16_t *__restrict__ out = p.out;
    uint8_t *__restrict__ out8 = p.out8;
    const size_t T = p.T;
    const unsigned V = p.V, n8 = p.n8;
    const float scale = p.scale, qs = out8 ? __ldg(p.q_scale) : 1.0f;
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
            if (out8) reinterpret_cast<uint2 *>(out8)[at] = bf16x8_to_fp8x8(w[j], qs, p.fmt);
        }
    }
    amax_end(m, p.amax_bits, alone);
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

// Counts of the first digit per chunk, and the keys themselves.
template <typename IdT>
__global__ void __launch_bounds__(ES_THREADS) embedding_count_kernel(const IdT *__restrict__ ids, size_t T, unsigned V,
                                                                     unsigned chunk_len, int bits, uint32_t *__restrict__ keys,
                                                                     int *__restrict__ table, int *__restrict__ split_count)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) *split_count = 0;
    __shared__ int cnt[ES_MAX_DIGITS];
    const int digits = 1 << bits;
    for (int d = threadIdx.x; d < digits; d += ES_THREADS) cnt[d] = 0;
    __syncthreads();
    const size_t t0 = (size_t)blockIdx.x * chunk_len, t1 = min(T, t0 + chunk_len);
    for (size_t t = t0 + threadIdx.x; t < t1; t += ES_THREADS) {
        const int id = checked_id(ids, t, V);
        const uint32_t key = id < 0 ? V : (uint32_t)id;
        keys[t] = key;
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
            rank[j] = warp_stable_rank(pos[j] >= 0 ? (int)((key[j] >> shift) & (digits - 1)) : -1, bits, warp_cnt[warp], lane);
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

__global__ void __launch_bounds__(ES_THREADS) embedding_scatter_kernel(const uint32_t *__restrict__ keys,
                                                                       const int *__restrict__ pos_in, size_t T,
                                                                       unsigned chunk_len, unsigned chunks, int bits, int shift,
                                                                       const int *__restrict__ table,
                                                                       uint32_t *__restrict__ keys_out,
                                                                       int *__restrict__ pos_out, int *__restrict__ next_table)
{
    sort_scatter(keys, pos_in, T, chunk_len, chunks, blockIdx.x, bits, shift, table, keys_out, pos_out, next_table);
}

// Up to ER_MAX_T positions find their places by counting: position i comes behind every j with a smaller key, and behind every
// j < i with the same.  A CTA counts for 32 positions, one to a lane; its 8 warps share the keys among them.  No step waits for
// another CTA, and all SMs take part: T^2 comparisons in 3.7 us for 1024 positions, 4.2 for 2048 and 6.2 for 4096, where the
// cluster below takes 8.5 to 9.2; with more positions than 32 per SM it falls behind (64 to a CTA, 8192: 14.5 against 9.5).
constexpr int ER_THREADS = 256;
constexpr int ER_WARPS = ER_THREADS / 32;
constexpr int ER_TILE = 256;              // keys that a warp stages at a time
constexpr size_t ER_MAX_T = 32 * 148;

struct RankIds {
    const void *ids;
    unsigned T, V;
    uint32_t *keys;                       // out, in order
    int *pos;
    int *split_count;                     // set to zero for the kernels behind
};
template <typename IdT>
__device__ __forceinline__ uint32_t id_key(const void *ids, unsigned V, unsigned i)
{
    const int id = checked_id(static_cast<const IdT *>(ids), i, V);
    return id < 0 ? V : (uint32_t)id;
}

template <typename IdT>
__global__ void __launch_bounds__(ER_THREADS) embedding_rank_kernel(const RankIds p)
{
    __shared__ __align__(16) uint32_t tile[ER_WARPS][2][ER_TILE];
    __shared__ int counts[ER_WARPS][32];
    cudaTriggerProgrammaticLaunchCompletion();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.split_count = 0;
    const unsigned p0 = blockIdx.x * 32, i = p0 + lane;
    const uint32_t mine = i < p.T ? id_key<IdT>(p.ids, p.V, i) : 0u;
    int cnt = 0;
    // the warp's keys: tiles warp, warp + 8, ...; the next one is on its way while one is compared
    uint32_t next[ER_TILE / 32];
    const auto fetch = [&](unsigned j0) {
#pragma unroll
        for (int m = 0; m < ER_TILE / 32; ++m) {
            const unsigned j = j0 + m * 32 + lane;
            next[m] = j < p.T ? id_key<IdT>(p.ids, p.V, j) : 0xFFFFFFFFu;
        }
    };
    fetch(warp * ER_TILE);
    int buffer = 0;
    for (unsigned j0 = warp * ER_TILE; j0 < p.T; j0 += ER_WARPS * ER_TILE, buffer ^= 1) {
        uint32_t *keys = tile[warp][buffer];
#pragma unroll
        for (int m = 0; m < ER_TILE / 32; ++m) keys[m * 32 + lane] = next[m];
        __syncwarp();
        fetch(j0 + ER_WARPS * ER_TILE);
        if (j0 + ER_TILE <= p0 || j0 >= p0 + 32) {                // all before the CTA's positions, or all behind them
            const uint32_t below = mine + (j0 < p0 ? 1u : 0u);
#pragma unroll 8
            for (int q = 0; q < ER_TILE / 4; ++q) {
                const uint4 k = *reinterpret_cast<const uint4 *>(keys + 4 * q);
                cnt += (k.x < below ? 1 : 0) + (k.y < below ? 1 : 0) + (k.z < below ? 1 : 0) + (k.w < below ? 1 : 0);
            }
        } else {
            const int at = (int)i - (int)j0;                      // the lane's own place in the tile
#pragma unroll 4
            for (int q = 0; q < ER_TILE / 4; ++q) {
                const uint4 v = *reinterpret_cast<const uint4 *>(keys + 4 * q);
                const uint32_t k[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) cnt += k[e] < mine + (4 * q + e < at ? 1u : 0u) ? 1 : 0;
            }
        }
    }
    counts[warp][lane] = cnt;
    __syncthreads();
    if (warp == 0 && i < p.T) {
        int rank = 0;
#pragma unroll
        for (int w = 0; w < ER_WARPS; ++w) rank += counts[w][lane];
        p.keys[rank] = mine;
        p.pos[rank] = (int)i;
    }
}

// Up to CS_MAX_T positions are sorted by one cluster of 8 CTAs, which read one another's counts and hand the keys on through
// distributed shared memory; the chunked form above takes the rest, with a launch per pass.  Both are chains of latencies:
// loads, ranks, scans, scattered stores (two passes: 9.5 us for 8192 positions, 12.5 for 12345, 2 us more when the keys pass
// through L2; five launches of the chunked form took 22 us for 12345, one CTA that sorts alone 41).
constexpr int CS_THREADS = 1024;
constexpr int CS_WARPS = CS_THREADS / 32;
constexpr int CS_ITEMS = 8;
constexpr int CS_CTAS = 8;
constexpr size_t CS_MAX_T = (size_t)CS_CTAS * CS_THREADS * CS_ITEMS;

struct ClusterSort {
    const void *ids;
    unsigned T, V;
    int passes, bits, items;              // items: keys per thread; CTA c ranks positions c * items * 1024 ...
    uint32_t *keys;                       // out, in order
    int *pos;
    int *split_count;                     // set to zero for the kernels behind
};

// Sum over the threads before this one, of the CTA's 1024 (`warp_sum`: CS_WARPS entries).  Ends with a barrier behind its reads.
__device__ __forceinline__ int scan_before(int v, int *warp_sum)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int scan = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, scan, off);
        if (lane >= off) scan += u;
    }
    if (lane == 31) warp_sum[warp] = scan;
    __syncthreads();
    const int before = __reduce_add_sync(0xffffffffu, warp > lane ? warp_sum[lane] : 0);
    __syncthreads();
    return before + scan - v;
}

// The warps' counts of digit `tid` become their starts within the CTA; returns the digit's total.
__device__ __forceinline__ int starts_of_warps(uint16_t *cnt, int digits)
{
    int at = 0;
#pragma unroll
    for (int w = 0; w < CS_WARPS; ++w) {
        const int v = cnt[w * digits + threadIdx.x];
        cnt[w * digits + threadIdx.x] = (uint16_t)at;
        at += v;
    }
    return at;
}

__device__ __forceinline__ int load_cluster_int(uint32_t saddr, int cta)
{
    int v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr(saddr, cta)) : "memory");
    return v;
}

__device__ __forceinline__ void store_cluster(uint32_t saddr, unsigned cta, uint32_t v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(saddr, cta)), "r"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <typename IdT>
__global__ void __launch_bounds__(CS_THREADS, 1) embedding_cluster_sort_kernel(const ClusterSort p)
{
    extern __shared__ __align__(16) uint32_t sort_mem[];
    cudaTriggerProgrammaticLaunchCompletion();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = (int)cluster_ctarank();
    const int digits = 1 << p.bits;
    if (cta == 0 && tid == 0) *p.split_count = 0;
    uint16_t *cnt = reinterpret_cast<uint16_t *>(sort_mem);                       // [CS_WARPS][digits]: at most 8192 in a CTA
    int *tot = reinterpret_cast<int *>(cnt + CS_WARPS * digits);                  // [digits]: this CTA's keys per digit
    int *base = tot + digits;                                                     // [digits]
    const unsigned held = (unsigned)p.items * CS_THREADS;                         // places of the order that a CTA holds
    uint32_t *skey = reinterpret_cast<uint32_t *>(base + digits);                 // [held]: keys between the passes
    int *spos = reinterpret_cast<int *>(skey + held);                             // [held]: their positions
    __shared__ int warp_sum[CS_WARPS];
    uint16_t *my_cnt = cnt + warp * digits;
    const unsigned first = ((unsigned)cta * CS_WARPS + warp) * 32u * p.items + lane;
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = pass * p.bits;
        for (int d = lane; d < digits / 2; d += 32) reinterpret_cast<uint32_t *>(my_cnt)[d] = 0u;
        uint32_t key[CS_ITEMS];
        int pos[CS_ITEMS], rank[CS_ITEMS];
#pragma unroll
        for (int j = 0; j < CS_ITEMS; ++j) {
            const unsigned i = first + 32u * j;
            key[j] = 0u;
            pos[j] = -1;
            if (j < p.items && i < p.T) {
                if (pass == 0) {
                    key[j] = id_key<IdT>(p.ids, p.V, i);
                    pos[j] = (int)i;
                } else {
                    key[j] = skey[i - cta * held];
                    pos[j] = spos[i - cta * held];
                }
            }
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < CS_ITEMS; ++j)
            if (j < p.items) rank[j] = warp_stable_rank(pos[j] >= 0 ? (int)((key[j] >> shift) & (digits - 1)) : -1, p.bits, my_cnt, lane);
        __syncthreads();
        if (tid < digits) tot[tid] = starts_of_warps(cnt, digits);
        cluster_sync_all();
        int total = 0, mine = 0;
        if (tid < digits) {
            const uint32_t a = smem_u32(tot + tid);
#pragma unroll
            for (int c = 0; c < CS_CTAS; ++c) {
                const int v = load_cluster_int(a, c);
                if (c < cta) mine += v;
                total += v;
            }
        }
        const int before = scan_before(total, warp_sum);
        if (tid < digits) base[tid] = before + mine;
        __syncthreads();
        const bool last = pass + 1 == p.passes;
        if (last) cluster_arrive();             // done with the others' `tot`
#pragma unroll
        for (int j = 0; j < CS_ITEMS; ++j) {
            if (j >= p.items || pos[j] < 0) continue;
            const int d = (key[j] >> shift) & (digits - 1);
            const unsigned to = base[d] + my_cnt[d] + rank[j];
            if (last) {
                p.keys[to] = key[j];
                p.pos[to] = pos[j];
            } else {
                const unsigned there = (to / CS_THREADS) / (unsigned)p.items;     // the CTA that holds this place
                store_cluster(smem_u32(skey + (to - there * held)), there, key[j]);
                store_cluster(smem_u32(spos + (to - there * held)), there, (uint32_t)pos[j]);
            }
        }
        if (last) cluster_wait();               // nobody leaves while its `tot` may be read
        else cluster_sync_all();                // the stores above, and everybody's reads of `tot`
    }
}

// ---------------------------------------------------------------- gradient: sums
constexpr int EG_THREADS = 256;
constexpr unsigned EG_JOIN_BLOCKS = 148 * 8;
constexpr int EG_FILL_ROWS = 4096;  // rows of the table per filling block, at most

struct GradParams {
    const uint16_t *dy;
    const uint32_t *keys;
    const int *pos;
    size_t T;
    unsigned V, n8;
    float scale;
    void *dtable;
    int is_fp32, accumulate, lanes_log2;
    int run_log2;                    // sorted positions per work item
    int *split_count;                // the runs that go on from the item they begin in to the next: how many,
    uint2 *split;                    // and (item, id) of each
    float *partial;                  // [items][2][D]: sums of the item's first and last run where they cross its ends
    size_t items, item_blocks, col_blocks;
    size_t fill_rows, fill_from;     // rows of the table per filling block, and the first of them
};

// First place in the sorted keys that is not below v: a warp probes 32 places at a time.
__device__ __forceinline__ size_t lower_bound(const uint32_t *keys, size_t T, uint32_t v, int lane)
{
    size_t lo = 0, hi = T;
    while (lo < hi) {
        const size_t step = (hi - lo + 31) / 32, at = lo + lane * step;
        const int below = __popc(__ballot_sync(0xffffffffu, at < hi && __ldcg(keys + min(at, hi - 1)) < v));
        if (below == 0) return lo;
        hi = min(hi, lo + below * step);
        lo += (below - 1) * step + 1;
    }
    return lo;
}

// Zeros in the rows [v0, v1) that no token points at.
__device__ __forceinline__ void fill_rows(const GradParams &p, size_t v0, size_t v1)
{
    __shared__ uint8_t touched[EG_FILL_ROWS];
    __shared__ size_t range[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (size_t i = threadIdx.x; i < v1 - v0; i += EG_THREADS) touched[i] = 0;
    if (warp < 2) {
        const size_t at = lower_bound(p.keys, p.T, (uint32_t)(warp ? v1 : v0), lane);
        if (lane == 0) range[warp] = at;
    }
    __syncthreads();
    for (size_t i = range[0] + threadIdx.x; i < range[1]; i += EG_THREADS) touched[__ldcg(p.keys + i) - v0] = 1;
    __syncthreads();
    const size_t quads = (size_t)p.n8 * (p.is_fp32 ? 2 : 1);       // 16-byte words per row
    uint4 *out = static_cast<uint4 *>(p.dtable) + v0 * quads;
    if (quads >= 32) {                          // a warp per row
        for (size_t r = warp; r < v1 - v0; r += EG_THREADS / 32) {
            if (touched[r]) continue;
            for (size_t c = lane; c < quads; c += 32) out[r * quads + c] = make_uint4(0u, 0u, 0u, 0u);
        }
    } else {
        for (size_t i = threadIdx.x; i < (v1 - v0) * quads; i += EG_THREADS)
            if (!touched[(unsigned)i / (unsigned)quads]) out[i] = make_uint4(0u, 0u, 0u, 0u);
    }
}

// Zeros for the first words of a table that is overwritten, on the SMs that do not sort.  Launched behind the sort's kernel and
// beside it; rows among them that a token points at are written later, by the kernels that wait for this one.  Its last block
// waits for the sort, so that whoever waits for this kernel has waited for both.
constexpr unsigned EC_WORDS = 4096;       // 16-byte words per block
// what is written while the sort takes its 10 us (131072 x 4096 in BF16: 182 us with none, 178.0 with 40 MB, 176.3 with 60 and
// 80, 178.4 with 100); a table below EC_MIN_BYTES is not worth the launch.  Up to ER_MAX_T positions the order takes 4 to 6 us and
// less fits beside it, which large tables do not feel (4096 positions: 131072 x 4096 167.6 us with 24 MB, 166.9 with 64; 50257 x
// 2048 FP32 78 and 77) and one that is cleared whole does (32000 x 1024 BF16: 31.8 with 24 or 40 MB, 33.8 with 64)
constexpr size_t EC_BYTES = (size_t)64 << 20, EC_MIN_BYTES = (size_t)4 << 20;
__global__ void __launch_bounds__(EG_THREADS) embedding_clear_kernel(uint4 *__restrict__ out, size_t words)
{
    cudaTriggerProgrammaticLaunchCompletion();
    const size_t i0 = (size_t)blockIdx.x * EC_WORDS + threadIdx.x;
#pragma unroll
    for (unsigned j = 0; j < EC_WORDS; j += EG_THREADS)
        if (i0 + j < words) out[i0 + j] = make_uint4(0u, 0u, 0u, 0u);
    if (blockIdx.x == gridDim.x - 1) cudaGridDependencySynchronize();
}

// Eight gradients of a row as they stand: one or two 16-byte words
template <bool F32>
struct Row8 {
    uint4 w[F32 ? 2 : 1];
};
template <bool F32>
__device__ __forceinline__ Row8<F32> load_row8(const GradParams &p, uint32_t v, unsigned c)
{
    Row8<F32> r;
    const uint4 *o = static_cast<const uint4 *>(p.dtable) + ((size_t)v * p.n8 + c) * (F32 ? 2 : 1);
    r.w[0] = o[0];
    if (F32) r.w[F32 ? 1 : 0] = o[1];
    return r;
}
template <bool F32>
__device__ __forceinline__ void store_row8(const GradParams &p, uint32_t v, unsigned c, const float (&acc)[8], const Row8<F32> &old)
{
    uint4 *o = static_cast<uint4 *>(p.dtable) + ((size_t)v * p.n8 + c) * (F32 ? 2 : 1);
    float r[8];
    if (F32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 u = old.w[F32 ? h : 0];
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) r[4 * h + q] = fmaf(acc[4 * h + q], p.scale, __uint_as_float(w[q]));
            reinterpret_cast<float4 *>(o)[h] = make_float4(r[4 * h], r[4 * h + 1], r[4 * h + 2], r[4 * h + 3]);
        }
    } else {
        const uint32_t w[4] = {old.w[0].x, old.w[0].y, old.w[0].z, old.w[0].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            r[2 * q] = fmaf(acc[2 * q], p.scale, bf16_lo(w[q]));
            r[2 * q + 1] = fmaf(acc[2 * q + 1], p.scale, bf16_hi(w[q]));
        }
        *o = make_uint4(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]), pack_bf16x2(r[4], r[5]), pack_bf16x2(r[6], r[7]));
    }
}
template <bool F32>
__device__ __forceinline__ Row8<F32> zero_row8()
{
    Row8<F32> r;
    r.w[0] = r.w[F32 ? 1 : 0] = make_uint4(0u, 0u, 0u, 0u);
    return r;
}

// Work item: 2^run_log2 neighbouring sorted positions, for the columns of one thread group (`lanes` threads, 8 columns each).
// A run of equal ids that lies inside the item is finished here; one that crosses the item's start or end leaves its sum
// in `partial` ([item][0] the one that began before, [item][1] the one that goes on) and is finished by
// embedding_join_kernel, which takes the runs from a list of the items that they begin in.  Blocks past the items write the untouched rows' zeros.
// U rows of dy travel at a time, and with them the old gradients of the runs that end among them (loaded when their run ends
// they cost 10 us more: 12345 tokens into 50257 x 2048 FP32, 20 us for the 132 MB that move).
template <bool F32, bool ACC, int U>
__global__ void __launch_bounds__(EG_THREADS) embedding_sum_kernel(const GradParams p)
{
    extern __shared__ __align__(16) uint32_t item_mem[];
    cudaTriggerProgrammaticLaunchCompletion();
    cudaGridDependencySynchronize();
    const size_t work_blocks = p.item_blocks * p.col_blocks;
    if (blockIdx.x >= work_blocks) {
        const size_t v0 = p.fill_from + (blockIdx.x - work_blocks) * p.fill_rows;
        fill_rows(p, v0, min((size_t)p.V, v0 + p.fill_rows));
        return;
    }
    const int run = 1 << p.run_log2, lanes = 1 << p.lanes_log2, slots = EG_THREADS >> p.lanes_log2, slot = threadIdx.x >> p.lanes_log2;
    // the block's keys, one before and one behind them, and its positions
    uint32_t *skey = item_mem + 1;
    int *spos = reinterpret_cast<int *>(item_mem + slots * run + 2);
    const size_t block0 = (blockIdx.x / p.col_blocks) * slots * run;
    for (int i = (int)threadIdx.x - 1; i <= slots * run; i += EG_THREADS) {
        const bool in = (i >= 0 || block0 > 0) && block0 + i < p.T;
        skey[i] = in ? __ldcg(p.keys + block0 + i) : 0xFFFFFFFFu;
        if (in && i >= 0 && i < slots * run) spos[i] = __ldcg(p.pos + block0 + i);
    }
    __syncthreads();
    const size_t item = (blockIdx.x / p.col_blocks) * slots + slot;
    const unsigned c = (unsigned)(blockIdx.x % p.col_blocks) * lanes + (threadIdx.x & (lanes - 1));
    if (item >= p.items || c >= p.n8) return;
    const uint32_t *key = skey + slot * run;
    const int *pos = spos + slot * run;
    const uint32_t before = key[-1];                             // 0xFFFFFFFF in front of the first position
    const int count = (int)min((size_t)run, p.T - item * run);
    const size_t D = (size_t)p.n8 * 8;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < count && key[i] < p.V; i += U) {         // ids outside the table are sorted behind the others
        uint4 v[U];
        Row8<F32> old[ACC ? U : 1];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (i + j >= count || key[i + j] >= p.V) continue;
            v[j] = __ldg(reinterpret_cast<const uint4 *>(p.dy) + (size_t)pos[i + j] * p.n8 + c);
            if (ACC && key[i + j + 1] != key[i + j] && key[i + j] != before) old[ACC ? j : 0] = load_row8<F32>(p, key[i + j], c);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (i + j >= count) continue;
            const uint32_t k = key[i + j];
            if (k >= p.V) continue;
            const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                acc[2 * q] += bf16_lo(w[q]);
                acc[2 * q + 1] += bf16_hi(w[q]);
            }
            const bool ends = key[i + j + 1] != k;
            if (!ends && i + j + 1 < count) continue;
            if (ends && k != before) {
                if (ACC) store_row8<F32>(p, k, c, acc, old[ACC ? j : 0]);
                else store_row8<F32>(p, k, c, acc, zero_row8<F32>());
            } else {
                float *o = p.partial + (item * 2 + (k == before ? 0 : 1)) * D + (size_t)c * 8;
                *reinterpret_cast<float4 *>(o) = make_float4(acc[0], acc[1], acc[2], acc[3]);
                *reinterpret_cast<float4 *>(o + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
                if (c == 0 && k != before) p.split[atomicAdd(p.split_count, 1)] = make_uint2((unsigned)item, k);      // in any order
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
        }
    }
}

// The runs that cross items.  A CTA takes a run and up to 128 lanes of its columns; its 256 / lanes thread groups share the
// items that the run reaches (group g the g-th, g + groups-th, ..., J of them in flight), then add up in pairs: a fixed order,
// whichever CTA it is.
template <bool F32, int J>
__global__ void __launch_bounds__(EG_THREADS) embedding_join_kernel(const GradParams p, int lanes_log2, unsigned col_blocks)
{
    __shared__ float4 red[2][EG_THREADS];
    cudaGridDependencySynchronize();
    const int lanes = 1 << lanes_log2, groups = EG_THREADS >> lanes_log2, group = threadIdx.x >> lanes_log2;
    const size_t D = (size_t)p.n8 * 8, run = (size_t)1 << p.run_log2;
    uint2 entry = __ldcg(p.split + blockIdx.x / col_blocks);     // on its way with the count; used if there are so many
    const size_t pieces = (size_t)__ldcg(p.split_count) * col_blocks;
    for (size_t piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
        if (piece != blockIdx.x) entry = __ldcg(p.split + piece / col_blocks);
        const size_t item = entry.x;
        const uint32_t key = entry.y;
        const unsigned c = (unsigned)(piece % col_blocks) * lanes + (threadIdx.x & (lanes - 1));
        const bool in = c < p.n8;
        Row8<F32> old = zero_row8<F32>();
        float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (in && group == 0) {
            if (p.accumulate) old = load_row8<F32>(p, key, c);
            const float4 *q = reinterpret_cast<const float4 *>(p.partial + (item * 2 + 1) * D + (size_t)c * 8);
            const float4 a = __ldcg(q), b = __ldcg(q + 1);
            acc[0] = a.x; acc[1] = a.y; acc[2] = a.z; acc[3] = a.w; acc[4] = b.x; acc[5] = b.y; acc[6] = b.z; acc[7] = b.w;
        }
        bool open = in;                                          // loads past the run's end are unused
        for (size_t k = item + 1 + group; open && k < p.items; k += (size_t)J * groups) {
            float4 lo[J], hi[J];
            uint32_t at[J];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const size_t n = k + (size_t)j * groups;
                at[j] = 0xFFFFFFFFu;
                if (n >= p.items) continue;
                at[j] = __ldcg(p.keys + n * run);
                const float4 *q = reinterpret_cast<const float4 *>(p.partial + n * 2 * D + (size_t)c * 8);
                lo[j] = __ldcg(q);
                hi[j] = __ldcg(q + 1);
            }
#pragma unroll
            for (int j = 0; j < J; ++j) {
                open = open && at[j] == key;
                if (!open) continue;
                acc[0] += lo[j].x; acc[1] += lo[j].y; acc[2] += lo[j].z; acc[3] += lo[j].w;
                acc[4] += hi[j].x; acc[5] += hi[j].y; acc[6] += hi[j].z; acc[7] += hi[j].w;
            }
        }
        for (int half = groups / 2; half > 0; half /= 2) {
            red[0][threadIdx.x] = make_float4(acc[0], acc[1], acc[2], acc[3]);
            red[1][threadIdx.x] = make_float4(acc[4], acc[5], acc[6], acc[7]);
            __syncthreads();
            if (group < half) {
                const float4 a = red[0][threadIdx.x + half * lanes], b = red[1][threadIdx.x + half * lanes];
                acc[0] += a.x; acc[1] += a.y; acc[2] += a.z; acc[3] += a.w;
                acc[4] += b.x; acc[5] += b.y; acc[6] += b.z; acc[7] += b.w;
            }
            __syncthreads();
        }
        if (in && group == 0) store_row8<F32>(p, key, c, acc, old);
    }
}

// ---------------------------------------------------------------- workspace of the gradient
// Sorted positions per work item.  Rows of up to 64 columns take few threads: shorter items give them more groups to work at
// once, and the join shares out the longer list of sums.  (Longer rows: 16 takes the same time as 32, with twice the sums.)
static int eg_run_log2(size_t D) { return D <= 64 ? 3 : 5; }

struct GradWs {
    size_t keys0, keys1, pos0, pos1, table, split, partial, bytes;     // offsets
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
    w.table = at; at += T <= CS_MAX_T ? 0 : up((size_t)sp.passes * sp.chunks * ((size_t)4 << sp.bits));
    const size_t items = ((T - 1) >> eg_run_log2(D)) + 1;
    w.split = at; at += up((items + 1) * sizeof(uint2));
    w.partial = at; at += up(items * 2 * D * sizeof(float));
    w.bytes = at;
    return w;
}

constexpr int EMB_MAX_SHARED = 160 * 1024;          // of the cluster's sort: counts of 32 warps x 1024 digits and two more rows (72 KB), 64 KB of keys
template <typename IdT>
static int launch_cluster_sort(const ClusterSort &p, size_t smem, cudaStream_t st)
{
    if (smem > 40 * 1024) {
        const int rc = allow_shared<embedding_cluster_sort_kernel<IdT>>(EMB_MAX_SHARED);
        if (rc != FP8_OK) return rc;
    }
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(CS_CTAS);
    c.blockDim = dim3(CS_THREADS);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    cudaLaunchAttribute a[1];
    a[0].id = cudaLaunchAttributeClusterDimension;
    a[0].val.clusterDim.x = CS_CTAS;
    a[0].val.clusterDim.y = a[0].val.clusterDim.z = 1;
    c.attrs = a;
    c.numAttrs = 1;
    FP8_CUDA_CHECK(cudaLaunchKernelEx(&c, embedding_cluster_sort_kernel<IdT>, p));
    return FP8_OK;
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
    if (!aligned16(table) || !aligned_to(ids, ids_are_int64 ? 8 : 4) || !aligned16(out_bf16) || !aligned16(out8)) {
        set_error("%s: pointers must be 16-byte aligned (ids: to their own size)", who);
        return FP8_ERR_ALIGN;
    }
    int rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const unsigned n8 = (unsigned)(D / 8);
    const int ll = lanes_log2_for(n8, 8);
    const size_t per_block = (size_t)(EF_THREADS >> ll) * EF_ROWS;
    const unsigned blocks = (unsigned)((T + per_block - 1) / per_block);
    const EmbedFwd p = {table, ids, T, (unsigned)V, n8, scale, static_cast<uint16_t *>(out_bf16),
                        reinterpret_cast<unsigned int *>(amax_out), q_scale, out8, fmt};
#define FP8DPA_LAUNCH_EF(IdT, F32) \
    return launch_behind_amax<embedding_fwd_kernel<IdT, F32>>(T * D, p.amax_bits, blocks, EF_THREADS, 0, st, p, ll)
    if (ids_are_int64) {
        if (table_is_fp32) FP8DPA_LAUNCH_EF(long long, true);
        else FP8DPA_LAUNCH_EF(long long, false);
    } else {
        if (table_is_fp32) FP8DPA_LAUNCH_EF(int, true);
        else FP8DPA_LAUNCH_EF(int, false);
    }
#undef FP8DPA_LAUNCH_EF
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
    if (!aligned16(dy_bf16) || !aligned_to(ids, ids_are_int64 ? 8 : 4) || !aligned16(dtable)) {
        set_error("fp8_embedding_bwd: pointers must be 16-byte aligned (ids: to their own size)");
        return FP8_ERR_ALIGN;
    }
    const GradWs w = grad_ws(T, V, D);
    if (!ws || ws_bytes < w.bytes || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("fp8_embedding_bwd: workspace of %zu bytes, 256-byte aligned, needed (got %zu)", w.bytes, ws_bytes);
        return FP8_ERR_WORKSPACE;
    }
    uint8_t *base = static_cast<uint8_t *>(ws);
    uint32_t *keys[2] = {reinterpret_cast<uint32_t *>(base + w.keys0), reinterpret_cast<uint32_t *>(base + w.keys1)};
    int *pos[2] = {reinterpret_cast<int *>(base + w.pos0), reinterpret_cast<int *>(base + w.pos1)};
    int *table = reinterpret_cast<int *>(base + w.table);
    const SortPlan sp = sort_plan(T, V);
    const size_t row_bytes = D * (out_is_fp32 ? 4 : 2);
    size_t cleared = accumulate || T > CS_MAX_T || V * row_bytes < EC_MIN_BYTES ? 0 : EC_BYTES / row_bytes;
    if (cleared > V) cleared = V;
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
    p.run_log2 = eg_run_log2(D);
    p.split_count = reinterpret_cast<int *>(base + w.split);
    p.split = reinterpret_cast<uint2 *>(p.split_count) + 1;
    p.items = ((T - 1) >> p.run_log2) + 1;
    const size_t slots = EG_THREADS >> p.lanes_log2;
    p.item_blocks = (p.items + slots - 1) / slots;
    p.col_blocks = (p.n8 + (1u << p.lanes_log2) - 1) >> p.lanes_log2;
    p.fill_from = cleared;
    p.fill_rows = row_bytes >= 131072 ? 1 : 131072 / row_bytes;
    if (p.fill_rows > EG_FILL_ROWS) p.fill_rows = EG_FILL_ROWS;
    const size_t work = p.item_blocks * p.col_blocks;
    const size_t fill = accumulate ? 0 : (V - cleared + p.fill_rows - 1) / p.fill_rows;
    if (work + fill > 0x7FFFFFFFull) {
        set_error("fp8_embedding_bwd: T=%zu V=%zu D=%zu needs more blocks than a grid holds", T, V, D);
        return FP8_ERR_SHAPE;
    }
    int rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T <= CS_MAX_T) {
        if (T <= ER_MAX_T) {
            const RankIds s = {ids, (unsigned)T, (unsigned)V, keys[sp.passes & 1], pos[sp.passes & 1], p.split_count};
            const unsigned grid = (unsigned)((T + 31) / 32);
            if (ids_are_int64) embedding_rank_kernel<long long><<<grid, ER_THREADS, 0, st>>>(s);
            else embedding_rank_kernel<int><<<grid, ER_THREADS, 0, st>>>(s);
            FP8_CUDA_CHECK(cudaGetLastError());
        } else {
            ClusterSort s;
            s.ids = ids;
            s.T = (unsigned)T;
            s.V = (unsigned)V;
            s.passes = sp.passes;
            s.bits = sp.bits;
            s.items = (int)((T + CS_CTAS * CS_THREADS - 1) / (CS_CTAS * CS_THREADS));
            s.keys = keys[sp.passes & 1];
            s.pos = pos[sp.passes & 1];
            s.split_count = p.split_count;
            const size_t smem = (((size_t)CS_WARPS * 2 + 8) << sp.bits) + (size_t)s.items * CS_THREADS * 8;
            rc = ids_are_int64 ? launch_cluster_sort<long long>(s, smem, st) : launch_cluster_sort<int>(s, smem, st);
            if (rc != FP8_OK) return rc;
        }
        if (cleared) {
            const size_t words = cleared * row_bytes / 16;
            rc = launch_early(embedding_clear_kernel, (unsigned)((words + EC_WORDS - 1) / EC_WORDS), EG_THREADS, 0, st,
                              static_cast<uint4 *>(dtable), words);
            if (rc != FP8_OK) return rc;
        }
    } else {
        const unsigned chunk_len = (unsigned)(sp.chunk_tiles * ES_TILE), chunks = (unsigned)sp.chunks;
        const size_t table_len = sp.chunks << sp.bits;
        if (sp.passes > 1) FP8_CUDA_CHECK(cudaMemsetAsync(table + table_len, 0, (sp.passes - 1) * table_len * sizeof(int), st));
        if (ids_are_int64)
            embedding_count_kernel<long long><<<chunks, ES_THREADS, 0, st>>>(static_cast<const long long *>(ids), T, (unsigned)V,
                                                                             chunk_len, sp.bits, keys[0], table, p.split_count);
        else
            embedding_count_kernel<int><<<chunks, ES_THREADS, 0, st>>>(static_cast<const int *>(ids), T, (unsigned)V, chunk_len,
                                                                       sp.bits, keys[0], table, p.split_count);
        FP8_CUDA_CHECK(cudaGetLastError());
        for (int i = 0; i < sp.passes; ++i) {
            embedding_scatter_kernel<<<chunks, ES_THREADS, 0, st>>>(
                keys[i & 1], i ? pos[i & 1] : nullptr, T, chunk_len, chunks, sp.bits, i * sp.bits, table + i * table_len,
                keys[(i + 1) & 1], pos[(i + 1) & 1], i + 1 < sp.passes ? table + (i + 1) * table_len : nullptr);
            FP8_CUDA_CHECK(cudaGetLastError());
        }
    }
    const size_t smem = ((slots << p.run_log2) * 2 + 2) * sizeof(uint32_t);       // 16 KB at most (8 columns: 256 slots of 8)
    const unsigned blocks = (unsigned)(work + fill);
    if (p.is_fp32 && p.accumulate) rc = launch_early(embedding_sum_kernel<true, true, 4>, blocks, EG_THREADS, smem, st, p);
    else if (p.is_fp32) rc = launch_early(embedding_sum_kernel<true, false, 8>, blocks, EG_THREADS, smem, st, p);
    else if (p.accumulate) rc = launch_early(embedding_sum_kernel<false, true, 4>, blocks, EG_THREADS, smem, st, p);
    else rc = launch_early(embedding_sum_kernel<false, false, 8>, blocks, EG_THREADS, smem, st, p);
    if (rc != FP8_OK || p.items == 1) return rc;
    // narrow rows have a group for (almost) every item that a run reaches, wide ones few groups
    const int jl = lanes_log2_for(p.n8, 7);
    const unsigned cols = (p.n8 + (1u << jl) - 1) >> jl;
    const size_t most = p.items * cols;
    const unsigned grid = (unsigned)(most < EG_JOIN_BLOCKS ? most : EG_JOIN_BLOCKS);
    if (p.is_fp32 && jl > 3) rc = launch_early(embedding_join_kernel<true, 8>, grid, EG_THREADS, 0, st, p, jl, cols);
    else if (p.is_fp32) rc = launch_early(embedding_join_kernel<true, 2>, grid, EG_THREADS, 0, st, p, jl, cols);
    else if (jl > 3) rc = launch_early(embedding_join_kernel<false, 8>, grid, EG_THREADS, 0, st, p, jl, cols);
    else rc = launch_early(embedding_join_kernel<false, 2>, grid, EG_THREADS, 0, st, p, jl, cols);
    return rc;
}
