// Global gradient norm over many tensors and the scaling that clips it.
//
// The tensors are cut into chunks of GC_CHUNK elements, numbered through all tensors; a CTA takes a contiguous share of them,
// whose first tensor the host looks up, and streams through the tensors' parts in it.  The assignment, and with it the order
// of every sum, depends on the sizes alone.
#include <math.h>

#include "common.cuh"

namespace fp8dpa {

constexpr int GC_THREADS = 256;
constexpr int GC_CHUNK = GC_THREADS * 8;
constexpr int GC_ITEMS = 512;                             // tensors per launch (17 KB of kernel parameters)
constexpr unsigned GC_MAX_BLOCKS = 148 * 8;
// The clip keeps 32 elements of a thread in flight (four CTAs per SM), or 16 (eight) where a CTA's share is below this many
// chunks and latency counts: 12.3 M FP32 elements in 389 tensors (5 chunks per CTA) take 17.4 us with 32 and 12.7 with 16,
// 218 M BF16 elements (90 chunks per CTA) 218 us with 32 and 229 with 16.
constexpr unsigned GC_SMALL_SHARE = 16;

struct GradTable {
    const void *g[GC_ITEMS];
    void *out[GC_ITEMS];
    unsigned long long n[GC_ITEMS];
    unsigned first[GC_ITEMS + 1];                         // the tensor's first chunk
    unsigned short start[GC_MAX_BLOCKS];                  // the CTA's first tensor
    unsigned char types[GC_ITEMS];                        // bit 0: g is FP32, bit 1: out is FP32
    int items;
    unsigned chunks;
};
__device__ __forceinline__ unsigned first_chunk_of(unsigned chunks, unsigned block, unsigned blocks)
{
    return (unsigned)((unsigned long long)chunks * block / blocks);
}

// V consecutive values (V x 2 or 4 bytes: one 8- or 16-byte access) of a BF16 or FP32 tensor
template <bool F32, int V>
__device__ __forceinline__ void load_v(const void *p, unsigned long long i, float (&f)[V])
{
    if constexpr (F32) {
        static_assert(V == 4, "16 bytes");
        const float4 v = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(p) + i));
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else if constexpr (V == 8) {
        const uint4 v = __ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + i));
        f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
        f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
    } else {
        const uint2 v = __ldg(reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + i));
        f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    }
}
template <bool F32>
__device__ __forceinline__ float load_1(const void *p, unsigned long long i)
{
    return F32 ? static_cast<const float *>(p)[i] : __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[i] << 16);
}
template <bool F32, int V>
__device__ __forceinline__ void store_v(void *p, unsigned long long i, const float (&f)[V])
{
    if constexpr (F32) {
        *reinterpret_cast<float4 *>(static_cast<float *>(p) + i) = make_float4(f[0], f[1], f[2], f[3]);
    } else if constexpr (V == 8) {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + i) =
            make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    } else {
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p) + i) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
    }
}
template <bool F32>
__device__ __forceinline__ void store_1(void *p, unsigned long long i, float f)
{
    if (F32) static_cast<float *>(p)[i] = f;
    else static_cast<uint16_t *>(p)[i] = (uint16_t)(pack_bf16x2(f, f) & 0xFFFFu);
}

// Squares of the elements [i, end): FP32 for 32 of a thread's at a time, FP64 above.
template <bool F32>
__device__ __forceinline__ double span_squares(const void *g, unsigned long long i, unsigned long long end)
{
    constexpr int V = F32 ? 4 : 8, U = 32 / V;
    constexpr unsigned ROW = GC_THREADS * V;
    double acc = 0.0;
    for (; i + (unsigned long long)U * ROW <= end; i += (unsigned long long)U * ROW) {
        float f[U][V], s = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) load_v<F32, V>(g, i + u * ROW + threadIdx.x * V, f[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) s = fmaf(f[u][e], f[u][e], s);
        acc += (double)s;
    }
    float s = 0.0f;                                       // fewer than U rows are left
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned long long at = i + u * ROW + threadIdx.x * V;
        if (at + V <= end) {
            float f[V];
            load_v<F32, V>(g, at, f);
#pragma unroll
            for (int e = 0; e < V; ++e) s = fmaf(f[e], f[e], s);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float f = at + e < end ? load_1<F32>(g, at + e) : 0.0f;
                s = fmaf(f, f, s);
            }
        }
    }
    return acc + (double)s;
}

__global__ void __launch_bounds__(GC_THREADS) grad_norm_kernel(const __grid_constant__ GradTable t, double *__restrict__ partial)
{
    cudaTriggerProgrammaticLaunchCompletion();
    __shared__ double red[GC_THREADS / 32];
    double acc = 0.0;
    const unsigned end = first_chunk_of(t.chunks, blockIdx.x + 1, gridDim.x);
    unsigned c = first_chunk_of(t.chunks, blockIdx.x, gridDim.x);
    for (int k = t.start[blockIdx.x]; c < end; ++k) {
        const unsigned first = t.first[k], stop = min(end, t.first[k + 1]);
        const unsigned long long i = (unsigned long long)(c - first) * GC_CHUNK;
        const unsigned long long to = min(t.n[k], (unsigned long long)(stop - first) * GC_CHUNK);
        acc += (t.types[k] & 1) ? span_squares<true>(t.g[k], i, to) : span_squares<false>(t.g[k], i, to);
        c = stop;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, off);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < GC_THREADS / 32; ++w) acc += red[w];
        partial[blockIdx.x] = acc;
    }
}

__global__ void __launch_bounds__(1024) grad_norm_join_kernel(const double *__restrict__ partial, size_t parts,
                                                              float *__restrict__ norm)
{
    cudaGridDependencySynchronize();
    __shared__ double red[32];
    double acc = 0.0;
    for (size_t i = threadIdx.x; i < parts; i += 1024) acc += __ldcg(partial + i);
#pragma unroll
    for (int round = 0; round < 2; ++round) {             // over a warp's lanes, then over the warps
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, off);
        if (round == 0) {
            if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = acc;
            __syncthreads();
            acc = red[threadIdx.x & 31];
        }
    }
    if (threadIdx.x == 0) *norm = (float)sqrt(acc);
}

template <bool IN32, bool OUT32, int PER>
__device__ __forceinline__ void span_scale(const void *g, void *o, unsigned long long begin, unsigned long long end, float c)
{
    constexpr int V = IN32 || OUT32 ? 4 : 8, U = PER / V;  // full 16-byte accesses of the wider side
    constexpr unsigned ROW = GC_THREADS * V;
    // last part first: what the norm read last is still in L2
    const unsigned long long blocks = (end - begin) / ((unsigned long long)U * ROW);
    const unsigned long long tail = begin + blocks * ((unsigned long long)U * ROW);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned long long at = tail + u * ROW + threadIdx.x * V;
        if (at + V <= end) {
            float f[V];
            load_v<IN32, V>(g, at, f);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] *= c;
            store_v<OUT32, V>(o, at, f);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (at + e < end) store_1<OUT32>(o, at + e, load_1<IN32>(g, at + e) * c);
        }
    }
    for (unsigned long long b = blocks; b > 0; --b) {
        const unsigned long long i = begin + (b - 1) * ((unsigned long long)U * ROW) + threadIdx.x * V;
        float f[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) load_v<IN32, V>(g, i + u * ROW, f[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int e = 0; e < V; ++e) f[u][e] *= c;
            store_v<OUT32, V>(o, i + u * ROW, f[u]);
        }
    }
}

// out = g * min(1, max_norm / (norm + 1e-6)).  A tensor that is clipped in place under a factor of 1 stays untouched.
// PER elements of a thread are in flight.
template <int PER>
__global__ void __launch_bounds__(GC_THREADS, PER == 16 ? 8 : 1) grad_clip_kernel(const __grid_constant__ GradTable t, const float *__restrict__ norm,
                                                               float max_norm)
{
    float f = max_norm / (__ldg(norm) + 1e-6f);
    if (f > 1.0f) f = 1.0f;                               // a NaN norm stays NaN
    const unsigned end = first_chunk_of(t.chunks, blockIdx.x + 1, gridDim.x);
    unsigned c = first_chunk_of(t.chunks, blockIdx.x, gridDim.x);
    for (int k = t.start[blockIdx.x]; c < end; ++k) {
        const unsigned first = t.first[k], stop = min(end, t.first[k + 1]);
        const unsigned long long i = (unsigned long long)(c - first) * GC_CHUNK;
        const unsigned long long to = min(t.n[k], (unsigned long long)(stop - first) * GC_CHUNK);
        const void *g = t.g[k];
        void *o = t.out[k];
        c = stop;
        if (f == 1.0f && o == g) continue;
        switch (t.types[k]) {
        case 0: span_scale<false, false, PER>(g, o, i, to, f); break;
        case 1: span_scale<true, false, PER>(g, o, i, to, f); break;
        case 2: span_scale<false, true, PER>(g, o, i, to, f); break;
        default: span_scale<true, true, PER>(g, o, i, to, f); break;
        }
    }
}

static int check_items(const char *who, const fp8_grad_item *items, int n_items, bool need_out)
{
    if (!items) {
        set_error("%s: NULL items", who);
        return FP8_ERR_NULL;
    }
    if (n_items <= 0) {
        set_error("%s: n_items = %d", who, n_items);
        return FP8_ERR_SHAPE;
    }
    for (int i = 0; i < n_items; ++i) {
        const fp8_grad_item &it = items[i];
        if (it.n == 0) continue;
        if (!it.g || (need_out && !it.out)) {
            set_error("%s: item %d: NULL pointer", who, i);
            return FP8_ERR_NULL;
        }
        if (!aligned16(it.g) || (need_out && !aligned16(it.out))) {
            set_error("%s: item %d: pointers must be 16-byte aligned", who, i);
            return FP8_ERR_ALIGN;
        }
        if (it.n > ((size_t)1 << 40) || (need_out && it.out == it.g && !it.out_is_fp32 != !it.g_is_fp32)) {
            set_error("%s: item %d: n = %zu is over 2^40, or it is clipped in place with two types", who, i, it.n);
            return FP8_ERR_SHAPE;
        }
    }
    return FP8_OK;
}

static unsigned grid_of(const GradTable &t) { return t.chunks < GC_MAX_BLOCKS ? t.chunks : GC_MAX_BLOCKS; }

// The next launch's table from item *at on; chunk numbers stay below 2^31, one tensor may be cut for that.
struct Cursor {
    int item = 0;
    size_t done = 0;                                      // elements of `item` that earlier launches took
};
static void fill_table(GradTable &t, const fp8_grad_item *items, int n_items, Cursor &at)
{
    const size_t most = (size_t)1 << 30;                  // chunks per launch
    t.items = 0;
    t.chunks = 0;
    while (at.item < n_items && t.items < GC_ITEMS && t.chunks < most) {
        const fp8_grad_item &it = items[at.item];
        if (it.n == 0) {
            ++at.item;
            continue;
        }
        size_t n = it.n - at.done;
        size_t chunks = (n + GC_CHUNK - 1) / GC_CHUNK;
        if (chunks > most - t.chunks) {
            chunks = most - t.chunks;
            n = chunks * GC_CHUNK;
        }
        const int k = t.items++;
        t.g[k] = static_cast<const char *>(it.g) + at.done * (it.g_is_fp32 ? 4 : 2);
        t.out[k] = it.out ? static_cast<char *>(it.out) + at.done * (it.out_is_fp32 ? 4 : 2) : nullptr;
        t.n[k] = n;
        t.first[k] = t.chunks;
        t.types[k] = (it.g_is_fp32 ? 1 : 0) | (it.out_is_fp32 ? 2 : 0);
        t.chunks += (unsigned)chunks;
        at.done += n;
        if (at.done == it.n) {
            ++at.item;
            at.done = 0;
        }
    }
    t.first[t.items] = t.chunks;
}
// The tensor in which each CTA's share, chunks * b / blocks on, begins.
static void fill_starts(GradTable &t)
{
    const unsigned blocks = grid_of(t);
    if (!blocks) return;
    const unsigned whole = t.chunks / blocks, rest = t.chunks % blocks;
    unsigned c = 0, part = 0;
    int k = 0;
    for (unsigned b = 0; b < blocks; ++b) {
        while (t.first[k + 1] <= c) ++k;
        t.start[b] = (unsigned short)k;
        c += whole;
        part += rest;
        if (part >= blocks) {
            part -= blocks;
            ++c;
        }
    }
}

}  // namespace fp8dpa

using namespace fp8dpa;

extern "C" size_t fp8_grad_norm_workspace_bytes(const fp8_grad_item *items, int n_items)
{
    if (!items || n_items <= 0) return 0;
    // a launch takes GC_ITEMS tensors or 2^30 chunks, and leaves a sum per CTA
    size_t chunks = 0;
    for (int i = 0; i < n_items; ++i) chunks += items[i].n / GC_CHUNK + 1;
    const size_t launches = (size_t)n_items / GC_ITEMS + 1 + 2 * (chunks >> 30);
    const size_t parts = launches > 1 ? launches * GC_MAX_BLOCKS : chunks < GC_MAX_BLOCKS ? chunks : GC_MAX_BLOCKS;
    return (parts * sizeof(double) + 255) & ~(size_t)255;
}

extern "C" int fp8_grad_norm(const fp8_grad_item *items, int n_items, float *norm, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_items("fp8_grad_norm", items, n_items, false);
    if (rc != FP8_OK) return rc;
    if (!norm) {
        set_error("fp8_grad_norm: NULL norm");
        return FP8_ERR_NULL;
    }
    const size_t need = fp8_grad_norm_workspace_bytes(items, n_items);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("fp8_grad_norm: workspace of %zu bytes, 256-byte aligned, needed (got %zu)", need, ws_bytes);
        return FP8_ERR_WORKSPACE;
    }
    rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    double *partial = static_cast<double *>(ws);
    Cursor at;
    GradTable t;
    size_t parts = 0;
    while (at.item < n_items) {
        fill_table(t, items, n_items, at);
        fill_starts(t);
        const unsigned grid = grid_of(t);
        if (grid == 0) break;                             // only empty tensors were left
        grad_norm_kernel<<<grid, GC_THREADS, 0, st>>>(t, partial + parts);
        FP8_CUDA_CHECK(cudaGetLastError());
        parts += grid;
    }
    if (parts == 0) {                                     // nothing but empty tensors
        FP8_CUDA_CHECK(cudaMemsetAsync(norm, 0, sizeof(float), st));
        return FP8_OK;
    }
    return launch_early(grad_norm_join_kernel, 1, 1024, 0, st, partial, parts, norm);
}

extern "C" int fp8_grad_clip(const fp8_grad_item *items, int n_items, const float *norm, float max_norm, void *stream)
{
    int rc = check_items("fp8_grad_clip", items, n_items, true);
    if (rc != FP8_OK) return rc;
    if (!norm) {
        set_error("fp8_grad_clip: NULL norm");
        return FP8_ERR_NULL;
    }
    if (!(max_norm > 0.0f) || isinf(max_norm)) {
        set_error("fp8_grad_clip: max_norm = %g is not a positive number", (double)max_norm);
        return FP8_ERR_SHAPE;
    }
    rc = check_arch();
    if (rc != FP8_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Cursor at;
    GradTable t;
    while (at.item < n_items) {
        fill_table(t, items, n_items, at);
        fill_starts(t);
        const unsigned grid = grid_of(t);
        if (grid == 0) break;
        if (t.chunks < GC_SMALL_SHARE * grid) grad_clip_kernel<16><<<grid, GC_THREADS, 0, st>>>(t, norm, max_norm);
        else grad_clip_kernel<32><<<grid, GC_THREADS, 0, st>>>(t, norm, max_norm);
        FP8_CUDA_CHECK(cudaGetLastError());
    }
    return FP8_OK;
}
