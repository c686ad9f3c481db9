// The global norm of a list of gradients, and clipping: norm = sqrt(sum over all tensors and elements of g^2), and
// g * min(1, max_norm / (norm + 1e-6)).
//
// The list becomes a table in device memory (ecrm_grads_bind): the tensors, and for each chunk of kGradChunk elements of one
// tensor which tensor it is -- so that one launch goes over any number of tensors of any sizes, a workgroup a chunk at a
// time.  What bounds both: memory, every element read once (and written once).
// Squares are summed in 64 bits: squares of 32-bit values neither overflow nor vanish there, and no order of the sum can be
// seen in the 32 bits of the norm.
#include <math.h>
#include <new>
#include <string.h>

#include "types.h"

using namespace ecrm;

namespace ecrm {

constexpr int kGradThreads = 256;
constexpr uint32_t kGradChunk = 8192;     // elements
constexpr uint32_t kGradBlocks = 2048;    // workgroups of a launch, at most
constexpr uint32_t kGradPart = 48;        // tensors that one launch writes into the table

struct GradTensor {
    void *data;
    uint64_t elements;
    const uint64_t *rows;                 // null: all elements are there; else *rows * row_elements of them
    uint32_t row_elements, type;
    uint32_t first_chunk;
    uint32_t skew;                        // elements from the 16-byte boundary at or before data to data
};
struct GradPart { GradTensor t[kGradPart]; };
struct GradTable {
    const GradTensor *tensors;
    const uint32_t *chunk_tensor;         // [chunks]
    double *part;                         // [kGradBlocks]
    uint32_t *arrived;
    uint32_t chunks;
};

__global__ void write_table_kernel(GradPart p, uint32_t first, uint32_t cnt, GradTensor *to, uint32_t *arrived)
{
    if (threadIdx.x < cnt) to[first + threadIdx.x] = p.t[threadIdx.x];
    if (threadIdx.x == 0) *arrived = 0;
}

__global__ __launch_bounds__(kGradThreads) void write_chunks_kernel(const GradTensor *t, uint32_t count, uint32_t chunks,
                                                                    uint32_t *chunk_tensor)
{
    const uint32_t i = blockIdx.x * kGradThreads + threadIdx.x;
    if (i >= chunks) return;
    uint32_t lo = 0, hi = count;          // the last tensor whose first chunk is not behind i
    while (hi - lo > 1u) {
        const uint32_t mid = lo + (hi - lo) / 2u;
        if (t[mid].first_chunk <= i) lo = mid;
        else hi = mid;
    }
    chunk_tensor[i] = lo;
}

// The elements of a chunk: [lo, hi) of the tensor counted from the 16-byte boundary before it, so that a lane's 16 bytes are
// aligned; elements below `skew` or behind the tensor are not there.
struct Span { uint64_t lo, hi, from, to; };
__device__ __forceinline__ Span span_of(const GradTensor &t, uint32_t chunk)
{
    uint64_t n = t.elements;
    if (t.rows) {
        const uint64_t r = *t.rows, most = t.elements / t.row_elements;
        n = (r < most ? r : most) * t.row_elements;
    }
    Span s;
    s.lo = (uint64_t)(chunk - t.first_chunk) * kGradChunk;
    s.from = t.skew;
    s.to = t.skew + n;
    s.hi = s.lo + kGradChunk < s.to ? s.lo + kGradChunk : s.to;
    return s;
}

template <typename T>
struct Sixteen {                          // 16 bytes of elements
    static constexpr uint32_t N = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(N)));
};

template <typename T>
__device__ __forceinline__ typename Sixteen<T>::type load16(const T *p, uint64_t v, const Span &s)
{
    typedef typename Sixteen<T>::type Vec;
    constexpr uint32_t N = Sixteen<T>::N;
    if (v >= s.from && v + N <= s.to) return *(const Vec *)(p + v);
    Vec r;
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) r[j] = v + j >= s.from && v + j < s.to ? p[v + j] : (T)0.0f;
    return r;
}

template <typename T>
__device__ __forceinline__ double square_chunk(const GradTensor &t, const Span &s)
{
    constexpr uint32_t N = Sixteen<T>::N, U = 4;
    const T *p = (const T *)t.data - t.skew;
    double acc[2] = {0, 0};
    for (uint64_t v0 = s.lo; v0 < s.hi; v0 += U * N * kGradThreads) {
        typename Sixteen<T>::type x[U];
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) x[q] = load16<T>(p, v0 + (q * kGradThreads + threadIdx.x) * N, s);
#pragma unroll
        for (uint32_t q = 0; q < U; ++q)
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) {
                const double g = (double)(float)x[q][j];
                acc[j & 1] = fma(g, g, acc[j & 1]);
            }
    }
    return acc[0] + acc[1];
}

// sum over the workgroup, in an order that does not change, to thread 0
__device__ __forceinline__ double block_sum(double v, double *s_wave)
{
#pragma unroll
    for (int d = kWave / 2; d; d >>= 1) v += __shfl_down(v, d, kWave);
    if (lane_id() == 0) s_wave[threadIdx.x / kWave] = v;
    __syncthreads();
    double sum = 0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kGradThreads / kWave; ++w) sum += s_wave[w];
    return sum;
}

__global__ __launch_bounds__(kGradThreads) void norm_kernel(GradTable g, float *norm)
{
    __shared__ double s_wave[kGradThreads / kWave];
    __shared__ bool s_last;
    double acc = 0;
    for (uint32_t c = blockIdx.x; c < g.chunks; c += gridDim.x) {
        const GradTensor t = g.tensors[g.chunk_tensor[c]];
        const Span s = span_of(t, c);
        if (t.type == ECRM_BF16) acc += square_chunk<__bf16>(t, s);
        else if (t.type == ECRM_F16) acc += square_chunk<_Float16>(t, s);
        else acc += square_chunk<float>(t, s);
    }
    const double sum = block_sum(acc, s_wave);
    // the last workgroup adds up what all have left, in the order of their numbers
    if (threadIdx.x == 0) {
        __hip_atomic_store(&g.part[blockIdx.x], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = __hip_atomic_fetch_add(g.arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1u;
    }
    __syncthreads();
    if (!s_last) return;
    acc = 0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kGradThreads)
        acc += __hip_atomic_load(&g.part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const double total = block_sum(acc, s_wave);
    if (threadIdx.x == 0) {
        *norm = (float)sqrt(total);
        __hip_atomic_store(g.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next call
    }
}

// 16 bytes' worth of source elements, N of them, to [v, v + N) of the output
template <typename TO, uint32_t N>
__device__ __forceinline__ void store_some(TO *p, uint64_t v, const Span &s, const float (&y)[N])
{
    if (v >= s.from && v + N <= s.to && ((uintptr_t)(p + v) & (N * sizeof(TO) < 16 ? N * sizeof(TO) - 1 : 15)) == 0) {
        constexpr uint32_t M = N * sizeof(TO) < 16 ? N : 16 / sizeof(TO);      // to a store
        typedef TO Vec __attribute__((ext_vector_type(M)));
#pragma unroll
        for (uint32_t j0 = 0; j0 < N; j0 += M) {
            Vec r;
#pragma unroll
            for (uint32_t j = 0; j < M; ++j) r[j] = (TO)y[j0 + j];
            *(Vec *)(p + v + j0) = r;
        }
        return;
    }
#pragma unroll
    for (uint32_t j = 0; j < N; ++j)
        if (v + j >= s.from && v + j < s.to) p[v + j] = (TO)y[j];
}

template <typename T, typename TO>
__device__ __forceinline__ void clip_chunk(const GradTensor &t, const Span &s, void *out, double factor)
{
    constexpr uint32_t N = Sixteen<T>::N, U = 4;
    const T *p = (const T *)t.data - t.skew;
    TO *o = (TO *)out - t.skew;
    for (uint64_t v0 = s.lo; v0 < s.hi; v0 += U * N * kGradThreads) {
        typename Sixteen<T>::type x[U];
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) x[q] = load16<T>(p, v0 + (q * kGradThreads + threadIdx.x) * N, s);
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) {
            const uint64_t v = v0 + (q * kGradThreads + threadIdx.x) * N;
            float y[N];
            // the product in 64 bits, so that a 32-bit gradient is rounded once (a 16-bit one in 32 bits first)
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) y[j] = (float)((double)(float)x[q][j] * factor);
            if (v < s.hi) store_some<TO, N>(o, v, s, y);
        }
    }
}

template <typename T>
__device__ __forceinline__ void clip_to(const GradTensor &t, const Span &s, void *out, uint32_t type, double factor)
{
    if (type == ECRM_BF16) clip_chunk<T, __bf16>(t, s, out, factor);
    else if (type == ECRM_F16) clip_chunk<T, _Float16>(t, s, out, factor);
    else clip_chunk<T, float>(t, s, out, factor);
}

// out: null, or a table of as many tensors of as many elements
__global__ __launch_bounds__(kGradThreads) void clip_kernel(GradTable g, const GradTensor *out, const float *norm, double max_norm)
{
    double factor = max_norm / ((double)*norm + 1e-6);
    if (factor > 1.0) factor = 1.0;                      // not a number stays that
    if (factor == 1.0 && !out) return;                   // in place there is nothing to write
    for (uint32_t c = blockIdx.x; c < g.chunks; c += gridDim.x) {
        const uint32_t i = g.chunk_tensor[c];
        const GradTensor t = g.tensors[i];
        const Span s = span_of(t, c);
        void *to = out ? out[i].data : t.data;
        const uint32_t type = out ? out[i].type : t.type;
        if (t.type == ECRM_BF16) clip_to<__bf16>(t, s, to, type, factor);
        else if (t.type == ECRM_F16) clip_to<_Float16>(t, s, to, type, factor);
        else clip_to<float>(t, s, to, type, factor);
    }
}

}  // namespace ecrm

// ---- C ABI -----------------------------------------------------------------------------------------------------------------
struct ecrm_grads {
    GradTensor *list;                     // [count], host memory
    uint32_t count, chunks;
    size_t off_chunks, off_part, off_arrived, bytes;
    char *table;                          // bound device memory
};

static GradTable table_of(const ecrm_grads *g)
{
    GradTable t;
    t.tensors = (const GradTensor *)g->table;
    t.chunk_tensor = (const uint32_t *)(g->table + g->off_chunks);
    t.part = (double *)(g->table + g->off_part);
    t.arrived = (uint32_t *)(g->table + g->off_arrived);
    t.chunks = g->chunks;
    return t;
}

static int launched() { return hipGetLastError() == hipSuccess ? ECRM_OK : ECRM_EHIP; }

extern "C" {

int ecrm_grads_create(const ecrm_tensor *tensors, uint32_t count, ecrm_grads **out)
{
    if (!out || (count && !tensors)) return ECRM_EINVAL;
    *out = nullptr;
    if (count > (1u << 24)) return ECRM_EINVAL;
    uint64_t chunks = 0;
    for (uint32_t i = 0; i < count; ++i) {
        const ecrm_tensor &t = tensors[i];
        if (t.type > ECRM_F16 || (t.elements && !t.data) || (uintptr_t)t.data % type_bytes(t.type)) return ECRM_EINVAL;
        if (t.elements > (1ull << 48)) return ECRM_EINVAL;
        if (t.rows && ((uintptr_t)t.rows % 8 || !t.row_elements || t.elements % t.row_elements)) return ECRM_EINVAL;
        chunks += (t.elements + 15u) / kGradChunk + 1u;
    }
    if (chunks > 0xFFFFFFFFull) return ECRM_EINVAL;
    ecrm_grads *g = new (std::nothrow) ecrm_grads;
    GradTensor *list = new (std::nothrow) GradTensor[count ? count : 1];
    if (!g || !list) {
        delete g;
        delete[] list;
        return ECRM_EINVAL;
    }
    memset(g, 0, sizeof(*g));
    g->list = list;
    g->count = count;
    for (uint32_t i = 0; i < count; ++i) {
        const ecrm_tensor &t = tensors[i];
        GradTensor &to = list[i];
        to.data = t.data;
        to.elements = t.elements;
        to.rows = t.rows;
        to.row_elements = t.row_elements;
        to.type = t.type;
        to.first_chunk = g->chunks;
        to.skew = (uint32_t)((uintptr_t)t.data % 16 / type_bytes(t.type));
        if (t.elements) g->chunks += (uint32_t)((t.elements + to.skew + kGradChunk - 1) / kGradChunk);
    }
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
    take((size_t)count * sizeof(GradTensor));
    g->off_chunks = take((size_t)g->chunks * 4);
    g->off_part = take((size_t)kGradBlocks * sizeof(double));
    g->off_arrived = take(4);
    g->bytes = off;
    *out = g;
    return ECRM_OK;
}

void ecrm_grads_destroy(ecrm_grads *g)
{
    if (!g) return;
    delete[] g->list;
    delete g;
}

size_t ecrm_grads_bytes(const ecrm_grads *g) { return g ? g->bytes : 0; }

int ecrm_grads_bind(ecrm_grads *g, void *table, size_t table_bytes, void *stream)
{
    if (!g) return ECRM_EINVAL;
    if (!table || (uintptr_t)table % 256 || table_bytes < g->bytes) return ECRM_ESCRATCH;
    g->table = (char *)table;
    hipStream_t st = (hipStream_t)stream;
    const GradTable t = table_of(g);
    uint32_t first = 0;
    do {                                  // in the kernels' arguments: the list's own memory may go when the call returns
        GradPart p;
        memset(&p, 0, sizeof(p));
        const uint32_t cnt = g->count - first < kGradPart ? g->count - first : kGradPart;
        memcpy(p.t, g->list + first, cnt * sizeof(GradTensor));
        hipLaunchKernelGGL(write_table_kernel, dim3(1), dim3(64), 0, st, p, first, cnt, (GradTensor *)g->table, t.arrived);
        first += cnt;
    } while (first < g->count);
    if (g->chunks)
        hipLaunchKernelGGL(write_chunks_kernel, dim3((g->chunks + kGradThreads - 1) / kGradThreads), dim3(kGradThreads), 0, st,
                           t.tensors, g->count, g->chunks, (uint32_t *)t.chunk_tensor);
    return launched();
}

int ecrm_grads_norm(ecrm_grads *g, float *norm, void *stream)
{
    if (!g) return ECRM_EINVAL;
    if (!g->table) return ECRM_ENOTBOUND;
    if (!norm || (uintptr_t)norm % 4) return ECRM_EINVAL;
    const uint32_t blocks = g->chunks < kGradBlocks ? (g->chunks ? g->chunks : 1u) : kGradBlocks;
    hipLaunchKernelGGL(norm_kernel, dim3(blocks), dim3(kGradThreads), 0, (hipStream_t)stream, table_of(g), norm);
    return launched();
}

int ecrm_grads_clip(ecrm_grads *g, const ecrm_grads *out, const float *norm, float max_norm, void *stream)
{
    if (!g) return ECRM_EINVAL;
    if (!g->table || (out && !out->table)) return ECRM_ENOTBOUND;
    if (!norm || (uintptr_t)norm % 4 || !isfinite(max_norm) || max_norm < 0.0f) return ECRM_EINVAL;
    if (out) {
        if (out->count != g->count) return ECRM_EINVAL;
        for (uint32_t i = 0; i < g->count; ++i)
            if (out->list[i].elements != g->list[i].elements) return ECRM_EINVAL;
    }
    if (!g->chunks) return ECRM_OK;
    const uint32_t blocks = g->chunks < kGradBlocks ? g->chunks : kGradBlocks;
    hipLaunchKernelGGL(clip_kernel, dim3(blocks), dim3(kGradThreads), 0, (hipStream_t)stream, table_of(g),
                       out ? (const GradTensor *)out->table : (const GradTensor *)nullptr, norm, (double)max_norm);
    return launched();
}

}  // extern "C"
