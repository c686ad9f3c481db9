// The global norm of a list of gradients, and clipping: norm = sqrt(sum over all tensors and elements of g^2), and
// g * min(1, max_norm / (norm + 1e-6)).
//
// The list becomes a table in device memory (ecrm_grads_bind): the tensors, and for each chunk of one tensor's memory which
// tensor's it is and where -- so that one launch goes over any number of tensors of any sizes, a workgroup a chunk at a time.  What bounds both: memory, every element read once (and written once): the norm of 562 MB takes 89 us, 6.3 TB/s.
// Squares are summed in 64 bits: squares of 32-bit values neither overflow nor vanish there.  The order of the sum follows from the
// list, the 16-byte alignment of its addresses included, so that two runs give the same bits.
#include <math.h>
#include <new>
#include <string.h>

#include "types.h"

using namespace ecrm;

namespace ecrm {

constexpr int kGradThreads = 256;
// Of a chunk, in a list of up to kLongList: two 16-byte loads of a lane, in a longer one four.  4 KB, 8 KB, 16 KB: norm and clipping of 8 MB
// into 17 MB 14.4, 13.8, 15.0 us, of 34 MB into as many 24.3, 24.2, 26.0; the norm of 34 MB 10.8, 10.6, 12.2, of 537 MB 91, 88, 87; norm and
// clipping of 268 MB into as many 139, 142, 134.
constexpr uint32_t kShortChunk = 8192, kLongChunk = 16384;
// Of a list longer than the memory-side cache's 256 MiB what the norm reads last is what clipping, from the end on, finds there:
// the last kNearChunks are read as usual, the others, and all that clipping moves in a list of more than kLongList, past the
// caches.  2^28 elements, 562 MB: norm 95 us as usual, 87 all past the caches, 89 so; norm and clipping of 268 MB into as many: 164
// as usual, 156 with loads past the caches, 135 with stores, 134 so (128 MiB near: 139).  A list of 8 MB into 17: 15.5 as usual, 16.3.
constexpr uint64_t kLongList = 128ull << 20;
constexpr uint32_t kNearChunks = (192u << 20) / kLongChunk;
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
// A chunk: some bytes of one tensor's memory from a 16-byte boundary on, of which the elements [from, to) are the tensor's.
struct GradChunk {
    const void *base;
    uint64_t first;                       // element of the tensor that base would be, from <= 0 where the tensor begins behind it
    uint32_t from, to;
    uint32_t tensor;
    uint32_t type;                        // and kCounted: the device knows how many rows there are
};
constexpr uint32_t kCounted = 16;
struct GradTable {
    const GradTensor *tensors;
    const GradChunk *chunk;               // [chunks]
    double *part;                         // [kGradBlocks]
    uint32_t *arrived;                    // [1 + kGroups][kGroupWords]
    uint32_t chunks;
};
// Workgroups count themselves in groups, and the groups in one counter: 2048 on one counter are 12 us, one after the other.
constexpr uint32_t kGroups = 32, kGroupWords = 64;

__global__ void write_table_kernel(GradPart p, uint32_t first, uint32_t cnt, GradTensor *to, uint32_t *arrived)
{
    if (threadIdx.x < cnt) to[first + threadIdx.x] = p.t[threadIdx.x];
    if (threadIdx.x <= kGroups) arrived[threadIdx.x * kGroupWords] = 0;
}

__global__ __launch_bounds__(kGradThreads) void write_chunks_kernel(const GradTensor *tensors, uint32_t count, uint32_t chunks,
                                                                    uint32_t chunk_bytes, GradChunk *chunk)
{
    const uint32_t i = blockIdx.x * kGradThreads + threadIdx.x;
    if (i >= chunks) return;
    uint32_t lo = 0, hi = count;          // the last tensor whose first chunk is not behind i
    while (hi - lo > 1u) {
        const uint32_t mid = lo + (hi - lo) / 2u;
        if (tensors[mid].first_chunk <= i) lo = mid;
        else hi = mid;
    }
    const GradTensor t = tensors[lo];
    const uint32_t each = chunk_bytes / type_bytes(t.type);
    const uint64_t nth = i - t.first_chunk, end = t.elements + t.skew - nth * each;
    GradChunk c;
    c.base = (const char *)t.data - (size_t)t.skew * type_bytes(t.type) + nth * chunk_bytes;
    c.first = nth * each - t.skew;
    c.from = nth ? 0u : t.skew;
    c.to = (uint32_t)(end < each ? end : each);
    c.tensor = lo;
    c.type = t.type | (t.rows ? kCounted : 0u);
    chunk[i] = c;
}

// how much of the chunk is there
__device__ __forceinline__ uint32_t counted_end(const GradTable &g, const GradChunk &c)
{
    if (!(c.type & kCounted)) return c.to;
    const GradTensor &t = g.tensors[c.tensor];
    const uint64_t r = *t.rows, most = t.elements / t.row_elements, n = (r < most ? r : most) * t.row_elements;
    const int64_t end = (int64_t)(n - c.first);          // from base
    return end <= (int64_t)c.from ? c.from : end < (int64_t)c.to ? (uint32_t)end : c.to;
}

template <typename T, uint32_t N>
struct Several {
    typedef T type __attribute__((ext_vector_type(N)));
};

// elements [v, v + N) of a chunk, zeros where they are not the tensor's
template <typename T, uint32_t N>
__device__ __forceinline__ typename Several<T, N>::type some_of(const T *p, uint32_t v, uint32_t from, uint32_t to)
{
    typename Several<T, N>::type r;
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) r[j] = v + j >= from && v + j < to ? p[v + j] : (T)0.0f;
    return r;
}

// A lane's elements of a chunk, N at a time: f(first of them, the N).  A chunk that is the tensor's as a whole -- most are --
// is loaded without a branch, all of it in flight.
// STREAM: it is not read again soon.
template <typename T, uint32_t N, uint32_t BYTES, bool STREAM, typename F>
__device__ __forceinline__ void over_chunk(const void *base, uint32_t from, uint32_t to, F f)
{
    typedef typename Several<T, N>::type Vec;
    constexpr uint32_t U = BYTES / (N * sizeof(T)) / kGradThreads;
    const T *p = (const T *)base;
    if (from == 0 && to == U * N * kGradThreads) {
        Vec x[U];
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) {
            const Vec *at = (const Vec *)p + q * kGradThreads + threadIdx.x;
            x[q] = STREAM ? __builtin_nontemporal_load(at) : *at;
        }
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) f((q * kGradThreads + threadIdx.x) * N, x[q]);
        return;
    }
    for (uint32_t q = 0; q < U; ++q) {
        const uint32_t v = (q * kGradThreads + threadIdx.x) * N;
        if (v >= to) break;
        f(v, v >= from && v + N <= to ? *(const Vec *)(p + v) : some_of<T, N>(p, v, from, to));
    }
}

template <typename T, uint32_t BYTES, bool STREAM>
__device__ __forceinline__ double square_chunk(const GradChunk &c, uint32_t to)
{
    constexpr uint32_t N = 16 / sizeof(T);
    double acc[2] = {0, 0};
    over_chunk<T, N, BYTES, STREAM>(c.base, c.from, to, [&](uint32_t, const typename Several<T, N>::type &x) {
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) {
            const double g = (double)(float)x[j];
            acc[j & 1] = fma(g, g, acc[j & 1]);
        }
    });
    return acc[0] + acc[1];
}

template <uint32_t BYTES, bool STREAM>
__device__ __forceinline__ double squares(const GradChunk &c, uint32_t to, uint32_t type)
{
    if (type == ECRM_BF16) return square_chunk<__bf16, BYTES, STREAM>(c, to);
    if (type == ECRM_F16) return square_chunk<_Float16, BYTES, STREAM>(c, to);
    return square_chunk<float, BYTES, STREAM>(c, to);
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

// Is the caller the last of `members` to arrive?  The counter is left as it was.
__device__ __forceinline__ bool arrive(uint32_t *counter, uint32_t members)
{
    if (__hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u != members) return false;
    __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}

// LONG: of a list of more than kLongList
template <bool LONG>
__global__ __launch_bounds__(kGradThreads) void norm_kernel(GradTable g, float *norm)
{
    __shared__ double s_wave[kGradThreads / kWave];
    __shared__ bool s_last;
    double acc = 0;
    GradChunk next = g.chunk[min(blockIdx.x, max(g.chunks, 1u) - 1u)];
    for (uint32_t i = blockIdx.x; i < g.chunks; i += gridDim.x) {
        const GradChunk c = next;
        next = g.chunk[min(i + gridDim.x, g.chunks - 1u)];
        const uint32_t to = counted_end(g, c), type = c.type & ~kCounted;
        if (!LONG) acc += squares<kShortChunk, false>(c, to, type);
        else acc += i + kNearChunks < g.chunks ? squares<kLongChunk, true>(c, to, type) : squares<kLongChunk, false>(c, to, type);
    }
    const double sum = block_sum(acc, s_wave);
    // the last workgroup adds up what all have left, in the order of their numbers
    if (threadIdx.x == 0) {
        shared_store(&g.part[blockIdx.x], sum);
        published();
        const uint32_t group = blockIdx.x % kGroups, members = (gridDim.x - group + kGroups - 1) / kGroups;
        s_last = arrive(g.arrived + (1u + group) * kGroupWords, members) && arrive(g.arrived, min(gridDim.x, kGroups));
    }
    __syncthreads();
    if (!s_last) return;
    acc = 0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kGradThreads) acc += shared_load(&g.part[i]);
    const double total = block_sum(acc, s_wave);
    if (threadIdx.x == 0) *norm = (float)sqrt(total);
}

// to elements p[0 .. N), of which [from, to) are there
template <typename TO, bool STREAM, uint32_t N>
__device__ __forceinline__ void store_some(TO *p, int64_t from, int64_t to, const float (&y)[N])
{
    if (from <= 0 && to >= (int64_t)N && (uintptr_t)p % (N * sizeof(TO)) == 0) {
        typedef typename Several<TO, N>::type Vec;
        Vec r;
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) r[j] = (TO)y[j];
        if (STREAM) __builtin_nontemporal_store(r, (Vec *)p);
        else *(Vec *)p = r;
        return;
    }
#pragma unroll
    for (uint32_t j = 0; j < N; ++j)
        if ((int64_t)j >= from && (int64_t)j < to) p[j] = (TO)y[j];
}

template <typename T, typename TO, bool LONG>
__device__ __forceinline__ void clip_chunk(const GradChunk &c, uint32_t to, void *out, double factor)
{
    constexpr uint32_t N = 16 / (sizeof(T) > sizeof(TO) ? sizeof(T) : sizeof(TO));      // 16 bytes of the wider
    TO *o = (TO *)out + (int64_t)c.first;
    over_chunk<T, N, LONG ? kLongChunk : kShortChunk, LONG>(c.base, c.from, to, [&](uint32_t v, const typename Several<T, N>::type &x) {
        float y[N];
        // the product in 64 bits, so that a 32-bit gradient is rounded once (a 16-bit one in 32 bits first)
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) y[j] = (float)((double)(float)x[j] * factor);
        store_some<TO, LONG, N>(o + v, (int64_t)c.from - v, (int64_t)to - v, y);
    });
}

template <typename T, bool LONG>
__device__ __forceinline__ void clip_to(const GradChunk &c, uint32_t to, void *out, uint32_t type, double factor)
{
    if (type == ECRM_BF16) clip_chunk<T, __bf16, LONG>(c, to, out, factor);
    else if (type == ECRM_F16) clip_chunk<T, _Float16, LONG>(c, to, out, factor);
    else clip_chunk<T, float, LONG>(c, to, out, factor);
}

// out: a table of as many tensors of as many elements; where it is the list's own, the call is in place
template <bool LONG>
__global__ __launch_bounds__(kGradThreads) void clip_kernel(GradTable g, const GradTensor *out, const float *norm, double max_norm)
{
    double factor = max_norm / ((double)*norm + 1e-6);
    if (factor > 1.0) factor = 1.0;                      // not a number stays that
    if (factor == 1.0 && out == g.tensors) return;       // nothing to write
    // from the end on: what the norm has read last may be near still
    GradChunk next = g.chunk[g.chunks - 1u - min(blockIdx.x, g.chunks - 1u)];
    for (uint32_t i = blockIdx.x; i < g.chunks; i += gridDim.x) {
        const GradChunk c = next;
        next = g.chunk[g.chunks - 1u - min(i + gridDim.x, g.chunks - 1u)];
        void *o = out[c.tensor].data;
        const uint32_t to = counted_end(g, c), type = c.type & ~kCounted, out_type = out[c.tensor].type;
        if (type == ECRM_BF16) clip_to<__bf16, LONG>(c, to, o, out_type, factor);
        else if (type == ECRM_F16) clip_to<_Float16, LONG>(c, to, o, out_type, factor);
        else clip_to<float, LONG>(c, to, o, out_type, factor);
    }
}

}  // namespace ecrm

// ---- C ABI -----------------------------------------------------------------------------------------------------------------
struct ecrm_grads {
    GradTensor *list;                     // [count], host memory
    uint32_t count, chunks;
    bool is_long;
    size_t off_chunks, off_part, off_arrived, bytes;
    char *table;                          // bound device memory
};

static GradTable table_of(const ecrm_grads *g)
{
    GradTable t;
    t.tensors = (const GradTensor *)g->table;
    t.chunk = (const GradChunk *)(g->table + g->off_chunks);
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
    uint64_t chunks = 0, bytes = 0;
    for (uint32_t i = 0; i < count; ++i) {
        const ecrm_tensor &t = tensors[i];
        if (t.type > ECRM_F16 || (t.elements && !t.data) || (uintptr_t)t.data % type_bytes(t.type)) return ECRM_EINVAL;
        if (t.elements > (1ull << 48)) return ECRM_EINVAL;
        if (t.rows && ((uintptr_t)t.rows % 8 || !t.row_elements || t.elements % t.row_elements)) return ECRM_EINVAL;
        bytes += t.elements * type_bytes(t.type);
        chunks += (t.elements + 8u) / (kShortChunk / type_bytes(t.type)) + 1u;
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
    g->is_long = bytes > kLongList;
    const uint32_t chunk_bytes = g->is_long ? kLongChunk : kShortChunk;
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
        const uint32_t each = chunk_bytes / type_bytes(t.type);
        if (t.elements) g->chunks += (uint32_t)((t.elements + to.skew + each - 1) / each);
    }
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
    take((size_t)count * sizeof(GradTensor));
    g->off_chunks = take((size_t)g->chunks * sizeof(GradChunk));
    g->off_part = take((size_t)kGradBlocks * sizeof(double));
    g->off_arrived = take((size_t)(1 + kGroups) * kGroupWords * 4);
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
                           t.tensors, g->count, g->chunks, g->is_long ? kLongChunk : kShortChunk, (GradChunk *)t.chunk);
    return launched();
}

int ecrm_grads_norm(ecrm_grads *g, float *norm, void *stream)
{
    if (!g) return ECRM_EINVAL;
    if (!g->table) return ECRM_ENOTBOUND;
    if (!norm || (uintptr_t)norm % 4) return ECRM_EINVAL;
    const uint32_t blocks = g->chunks < kGradBlocks ? (g->chunks ? g->chunks : 1u) : kGradBlocks;
    hipLaunchKernelGGL((g->is_long ? norm_kernel<true> : norm_kernel<false>), dim3(blocks), dim3(kGradThreads), 0, (hipStream_t)stream,
                       table_of(g), norm);
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
    hipLaunchKernelGGL((g->is_long ? clip_kernel<true> : clip_kernel<false>), dim3(blocks), dim3(kGradThreads), 0, (hipStream_t)stream,
                       table_of(g), (const GradTensor *)(out ? out : g)->table, norm, (double)max_norm);
    return launched();
}

}  // extern "C"
