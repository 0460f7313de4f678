// Global gradient norm over many tensors and the scaling that clips it.
//
// The tensors are cut into chunks of GC_CHUNK elements, numbered through all tensors.  A CTA of the clip takes one chunk, one
// of the norm GC_NORM_CHUNKS of them, and finds its tensor in a table that travels with the launch; the assignment, and with
// it the order of every sum, depends on the sizes alone.  Many short CTAs in order, not a few that stay: 218 M BF16 elements
// to FP32 are scaled at 6.7 TB/s in blocks of 4096 and at 5.5 to 6.0 by 148 x 2 ... 8 CTAs that loop (a share each, or every
// grid-th block), and read at 7.1 TB/s against 6.6.
#include <math.h>

#include "common.cuh"

namespace fp8dpa {

constexpr int GC_THREADS = 256;
constexpr int GC_PER_THREAD = 16;
constexpr int GC_CHUNK = GC_THREADS * GC_PER_THREAD;
constexpr int GC_NORM_CHUNKS = 4;
constexpr int GC_ITEMS = 512;                             // tensors per launch (17 KB of kernel parameters)
constexpr int GC_BUCKETS = 1024;

struct GradTable {
    const void *g[GC_ITEMS];
    void *out[GC_ITEMS];
    unsigned long long n[GC_ITEMS];
    unsigned first[GC_ITEMS + 1];                         // the tensor's first chunk
    unsigned short start[GC_BUCKETS];                     // the tensor that holds chunk j << bucket_log2
    unsigned char types[GC_ITEMS];                        // bit 0: g is FP32, bit 1: out is FP32
    int items, bucket_log2;
    unsigned chunks;
};
__device__ __forceinline__ int item_of_chunk(const GradTable &t, unsigned c)
{
    int k = t.start[c >> t.bucket_log2];
    while (t.first[k + 1] <= c) ++k;
    return k;
}

// V consecutive values (V x 2 or 4 bytes: one 8- or 16-byte access) of a BF16 or FP32 tensor.  CONST: memory that the kernel
// does not write, through the read-only path.  The clip may write what it reads (`out` can be the gradient itself), which that
// path does not allow: it loads from L2, in the same time (218 M BF16 to FP32 with the norm 278.8 us; 297 through L1).
template <bool CONST, typename W>
__device__ __forceinline__ W load_words(const void *p)
{
    return CONST ? __ldg(static_cast<const W *>(p)) : __ldcg(static_cast<const W *>(p));
}
template <bool F32, int V, bool CONST>
__device__ __forceinline__ void load_v(const void *p, unsigned long long i, float (&f)[V])
{
    if constexpr (F32) {
        static_assert(V == 4, "16 bytes");
        const float4 v = load_words<CONST, float4>(static_cast<const float *>(p) + i);
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else if constexpr (V == 8) {
        const uint4 v = load_words<CONST, uint4>(static_cast<const uint16_t *>(p) + i);
        f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
        f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
    } else {
        const uint2 v = load_words<CONST, uint2>(static_cast<const uint16_t *>(p) + i);
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
    for (; i < end; i += (unsigned long long)U * ROW) {
        float f[U][V], s = 0.0f;
        if (i + (unsigned long long)U * ROW <= end) {     // without conditions between them the loads go out together
#pragma unroll
            for (int u = 0; u < U; ++u) load_v<F32, V, true>(g, i + u * ROW + threadIdx.x * V, f[u]);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const unsigned long long at = i + u * ROW + threadIdx.x * V;
#pragma unroll
                for (int e = 0; e < V; ++e) f[u][e] = 0.0f;
                if (at + V <= end) {
                    load_v<F32, V, true>(g, at, f[u]);
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        if (at + e < end) f[u][e] = load_1<F32>(g, at + e);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) s = fmaf(f[u][e], f[u][e], s);
        acc += (double)s;
    }
    return acc;
}

__global__ void __launch_bounds__(GC_THREADS) grad_norm_kernel(const __grid_constant__ GradTable t, double *__restrict__ partial)
{
    cudaTriggerProgrammaticLaunchCompletion();
    __shared__ double red[GC_THREADS / 32];
    double acc = 0.0;
    unsigned c = blockIdx.x * GC_NORM_CHUNKS;
    const unsigned end = min(t.chunks, c + GC_NORM_CHUNKS);
    for (int k = item_of_chunk(t, c); c < end; ++k) {
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
#pragma unroll 8
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

template <bool IN32, bool OUT32>
__device__ __forceinline__ void scale_chunk(const void *g, void *o, unsigned long long i, unsigned long long end, float c)
{
    constexpr int V = IN32 || OUT32 ? 4 : 8, U = GC_PER_THREAD / V;      // full 16-byte accesses of the wider side
    constexpr unsigned ROW = GC_THREADS * V;
    i += threadIdx.x * V;
    float f[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (i + u * ROW + V <= end) load_v<IN32, V, false>(g, i + u * ROW, f[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const unsigned long long at = i + u * ROW;
        if (at + V <= end) {
#pragma unroll
            for (int e = 0; e < V; ++e) f[u][e] *= c;
            store_v<OUT32, V>(o, at, f[u]);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (at + e < end) store_1<OUT32>(o, at + e, load_1<IN32>(g, at + e) * c);
        }
    }
}

// out = g * min(1, max_norm / (norm + 1e-6)).  A tensor that is clipped in place under a factor of 1 stays untouched.  The last
// chunk first: what the norm read last is still in L2.
__global__ void __launch_bounds__(GC_THREADS, 8) grad_clip_kernel(const __grid_constant__ GradTable t,
                                                                  const float *__restrict__ norm, float max_norm)
{
    float f = max_norm / (__ldg(norm) + 1e-6f);
    if (f > 1.0f) f = 1.0f;                               // a NaN norm stays NaN
    const unsigned c = t.chunks - 1 - blockIdx.x;
    const int k = item_of_chunk(t, c);
    const void *g = t.g[k];
    void *o = t.out[k];
    if (f == 1.0f && o == g) return;
    const unsigned long long i = (unsigned long long)(c - t.first[k]) * GC_CHUNK, end = min(t.n[k], i + GC_CHUNK);
    switch (t.types[k]) {
    case 0: return scale_chunk<false, false>(g, o, i, end, f);
    case 1: return scale_chunk<true, false>(g, o, i, end, f);
    case 2: return scale_chunk<false, true>(g, o, i, end, f);
    default: return scale_chunk<true, true>(g, o, i, end, f);
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
// Where a CTA begins to look for its tensor.
static void fill_starts(GradTable &t)
{
    t.bucket_log2 = 0;
    while ((t.chunks >> t.bucket_log2) >= (unsigned)GC_BUCKETS) ++t.bucket_log2;
    int k = 0;
    for (unsigned j = 0; j << t.bucket_log2 < t.chunks; ++j) {
        while (t.first[k + 1] <= j << t.bucket_log2) ++k;
        t.start[j] = (unsigned short)k;
    }
}

}  // namespace fp8dpa

using namespace fp8dpa;

extern "C" size_t fp8_grad_norm_workspace_bytes(const fp8_grad_item *items, int n_items)
{
    if (!items || n_items <= 0) return 0;
    // a sum per GC_NORM_CHUNKS chunks, and one more for each launch (of GC_ITEMS tensors or 2^30 chunks)
    size_t chunks = 0;
    for (int i = 0; i < n_items; ++i) chunks += (items[i].n + GC_CHUNK - 1) / GC_CHUNK;
    const size_t parts = chunks / GC_NORM_CHUNKS + (size_t)n_items / GC_ITEMS + 2 * (chunks >> 30) + 2;
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
        if (t.chunks == 0) break;                         // only empty tensors were left
        fill_starts(t);
        const unsigned grid = (t.chunks + GC_NORM_CHUNKS - 1) / GC_NORM_CHUNKS;
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
        if (t.chunks == 0) break;
        fill_starts(t);
        grad_clip_kernel<<<t.chunks, GC_THREADS, 0, st>>>(t, norm, max_norm);
        FP8_CUDA_CHECK(cudaGetLastError());
    }
    return FP8_OK;
}
