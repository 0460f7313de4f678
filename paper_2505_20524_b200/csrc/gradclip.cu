// Global gradient norm over many tensors and the scaling that clips it.
//
// The tensors are cut into chunks of GC_CHUNK elements; chunk c belongs to the tensor whose first chunk is the last one
// not behind c (a search in the table of first chunks that travels with the launch).  CTA b takes the chunks b, b + grid,
// ...: the assignment, and with it the order of every sum, depends on the sizes alone.
#include <math.h>

#include "common.cuh"

namespace fp8dpa {

constexpr int GC_THREADS = 256;
constexpr int GC_PER_THREAD = 32;                         // elements: four groups of eight
constexpr int GC_CHUNK = GC_THREADS * GC_PER_THREAD;
constexpr int GC_ITEMS = 512;                             // tensors per launch (16 KB of kernel parameters)
constexpr unsigned GC_MAX_BLOCKS = 148 * 8;

struct GradTable {
    const void *g[GC_ITEMS];
    void *out[GC_ITEMS];
    unsigned long long n[GC_ITEMS];
    unsigned first[GC_ITEMS];                             // the tensor's first chunk
    unsigned char types[GC_ITEMS];                        // bit 0: g is FP32, bit 1: out is FP32
    int items;
    unsigned chunks;
};

__device__ __forceinline__ int item_of_chunk(const GradTable &t, unsigned c)
{
    int lo = 0, hi = t.items;                             // first[lo] <= c < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

// eight elements from index i of a tensor of n, zeros behind its end
__device__ __forceinline__ void load8(const void *g, bool fp32, unsigned long long i, unsigned long long n, float (&f)[8])
{
    if (i + 8 <= n) {
        if (fp32) {
            const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(g) + i);
            const float4 a = p[0], b = p[1];
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        } else {
            const uint4 v = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(g) + i);
            f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
            f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        f[e] = 0.0f;
        if (i + e < n)
            f[e] = fp32 ? static_cast<const float *>(g)[i + e] : __uint_as_float((uint32_t)static_cast<const uint16_t *>(g)[i + e] << 16);
    }
}

__device__ __forceinline__ void store8(void *o, bool fp32, unsigned long long i, unsigned long long n, const float (&f)[8])
{
    const uint32_t w[4] = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
    if (i + 8 <= n) {
        if (fp32) {
            float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(o) + i);
            p[0] = make_float4(f[0], f[1], f[2], f[3]);
            p[1] = make_float4(f[4], f[5], f[6], f[7]);
        } else {
            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(o) + i) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (i + e >= n) continue;
        if (fp32) static_cast<float *>(o)[i + e] = f[e];
        else static_cast<uint16_t *>(o)[i + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
}

// Sum of squares of the CTA's chunks.  Squares and the 32 of a thread's chunk in FP32, everything above in FP64.
__global__ void __launch_bounds__(GC_THREADS) grad_norm_kernel(const __grid_constant__ GradTable t, double *__restrict__ partial)
{
    __shared__ double red[GC_THREADS / 32];
    double acc = 0.0;
    for (unsigned c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int k = item_of_chunk(t, c);
        const void *g = t.g[k];
        const unsigned long long n = t.n[k], i0 = (unsigned long long)(c - t.first[k]) * GC_CHUNK + threadIdx.x * 8;
        const bool fp32 = t.types[k] & 1;
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < GC_PER_THREAD / 8; ++j) {
            float f[8];
            load8(g, fp32, i0 + (unsigned long long)j * (GC_THREADS * 8), n, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf(f[e], f[e], s);
        }
        acc += (double)s;
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
    __shared__ double red[32];
    double acc = 0.0;
    for (size_t i = threadIdx.x; i < parts; i += 1024) acc += __ldcg(partial + i);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, off);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 32; ++w) acc += red[w];
        *norm = (float)sqrt(acc);
    }
}

// out = g * min(1, max_norm / (norm + 1e-6)).  A tensor that is clipped in place under a factor of 1 stays untouched.
__global__ void __launch_bounds__(GC_THREADS) grad_clip_kernel(const __grid_constant__ GradTable t, const float *__restrict__ norm,
                                                               float max_norm)
{
    float f = max_norm / (__ldg(norm) + 1e-6f);
    if (f > 1.0f) f = 1.0f;                               // a NaN norm stays NaN
    for (unsigned c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        const int k = item_of_chunk(t, c);
        const void *g = t.g[k];
        void *o = t.out[k];
        if (f == 1.0f && o == g) continue;
        const unsigned long long n = t.n[k], i0 = (unsigned long long)(c - t.first[k]) * GC_CHUNK + threadIdx.x * 8;
        const bool in32 = t.types[k] & 1, out32 = t.types[k] & 2;
        float v[GC_PER_THREAD / 8][8];
#pragma unroll
        for (int j = 0; j < GC_PER_THREAD / 8; ++j) load8(g, in32, i0 + (unsigned long long)j * (GC_THREADS * 8), n, v[j]);
#pragma unroll
        for (int j = 0; j < GC_PER_THREAD / 8; ++j) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] *= f;
            store8(o, out32, i0 + (unsigned long long)j * (GC_THREADS * 8), n, v[j]);
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
}
static unsigned grid_of(const GradTable &t) { return t.chunks < GC_MAX_BLOCKS ? t.chunks : GC_MAX_BLOCKS; }

}  // namespace fp8dpa

using namespace fp8dpa;

extern "C" size_t fp8_grad_norm_workspace_bytes(const fp8_grad_item *items, int n_items)
{
    if (!items || n_items <= 0) return 0;
    Cursor at;
    GradTable t;
    size_t parts = 0;
    while (at.item < n_items) {
        fill_table(t, items, n_items, at);
        parts += grid_of(t);
    }
    const size_t bytes = (parts * sizeof(double) + 255) & ~(size_t)255;
    return bytes ? bytes : 256;
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
        const unsigned grid = grid_of(t);
        if (grid == 0) break;                             // only empty tensors were left
        grad_norm_kernel<<<grid, GC_THREADS, 0, st>>>(t, partial + parts);
        FP8_CUDA_CHECK(cudaGetLastError());
        parts += grid;
    }
    grad_norm_join_kernel<<<1, 1024, 0, st>>>(partial, parts, norm);
    FP8_CUDA_CHECK(cudaGetLastError());
    return FP8_OK;
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
        const unsigned grid = grid_of(t);
        if (grid == 0) break;
        grad_clip_kernel<<<grid, GC_THREADS, 0, st>>>(t, norm, max_norm);
        FP8_CUDA_CHECK(cudaGetLastError());
    }
    return FP8_OK;
}
