// Gradient of the lookup by sorted tokens: the gradient of row x is scale * the sum of the gradients of the looked-up rows
// whose token is x.  The tokens are sorted, stably, with the index of their row; the sorted positions are cut into chunks of
// equal length, whatever the runs of equal tokens in them, so that a token that is a tenth of a batch takes no longer than
// others.  A team of D / 4 lanes, four columns to a lane, walks a chunk: the sum of a run that lies inside the chunk is
// written at once, what a chunk has of runs that go on before or behind it is joined in LDS by the workgroup, and what a
// workgroup has of runs that go on in its neighbours by a launch behind.  Sums are carried in 64 bits and rounded once, in
// an order that follows from the sorted positions, n and D alone: no atomics, two runs give the same bits.
#include "types.h"

namespace ecrm {

constexpr int kSumThreads = 256;
constexpr uint32_t kSumMost = 1024;       // sorted positions of a workgroup, at most
constexpr uint32_t kSumBlocks = 2048;     // workgroups, unless that would be more positions to one than there is room for
constexpr uint32_t kChunkMin = 4, kChunkMax = 128;
constexpr int kTokenThreads = 256, kTokenTile = 1024;

// What a workgroup has of a run that goes on before it (and maybe behind it) and of one that begins in it and goes on behind it.
enum { kPartHead = 1, kPartThrough = 2, kPartTail = 4 };

struct SumArgs {
    const uint32_t *sk, *si;         // sorted: row (`rows` for the padding token), index of the gradient
    uint32_t n, rows, D;
    Divider d4;                      // by D / 4
    uint32_t teams, chunk, per;      // teams of a workgroup, positions of a chunk, of a workgroup
    uint32_t blocks;
    const void *d;                   // [n][stride] gradients of the looked-up rows
    uint64_t stride;
    double scale;
    uint32_t accumulate;             // dense: add to what is there
    TokenControl *ctl;
    uint32_t *first;                 // [blocks] distinct rows that begin before the workgroup's positions
    uint32_t *state;                 // [blocks] kPart*
    uint32_t *dest;                  // [blocks] row of the output that a kPartTail belongs to
    double *part;                    // [blocks][2][D]: head, tail
    uint64_t *out_keys;              // rows form
    float *out;
    uint64_t *count;
};

__global__ void token_begin_kernel(TokenControl *ctl)
{
    if (threadIdx.x == 0) ctl->bad = 0;
}

// row ids and indices for the sort; the padding token sorts behind every row
__global__ __launch_bounds__(kTokenThreads) void token_keys_kernel(const uint64_t *keys, uint32_t n, uint64_t padding,
                                                                   uint32_t rows, uint32_t *k, uint32_t *v, Header *hdr,
                                                                   TokenControl *ctl)
{
    const uint32_t end = min(n - blockIdx.x * kTokenTile, (uint32_t)kTokenTile) + blockIdx.x * kTokenTile;
    bool bad = false;
    for (uint32_t i = blockIdx.x * kTokenTile + threadIdx.x; i < end; i += kTokenThreads) {
        const uint64_t key = keys[i];
        const bool pad = key == padding && key != ECRM_NO_PADDING;
        bad |= !pad && key >= (uint64_t)rows;
        k[i] = pad ? rows : (uint32_t)key;
        v[i] = i;
    }
    if (__ballot(bad) && lane_id() == 0) {
        atomicOr(&ctl->bad, 1u);
        atomicOr(&hdr->err_sticky, 1u);
    }
}

// is sorted position p the first of a row?
__device__ __forceinline__ bool run_head(const uint32_t *sk, uint32_t p, uint32_t rows)
{
    const uint32_t key = sk[p];
    return key < rows && (p == 0 || sk[p - 1] != key);
}

__global__ __launch_bounds__(kSumThreads) void count_heads_kernel(SumArgs a)
{
    __shared__ uint32_t s_count;
    if (threadIdx.x == 0) s_count = 0;
    __syncthreads();
    const uint64_t pos0 = (uint64_t)blockIdx.x * a.per;
    const uint32_t cnt = (uint32_t)min((uint64_t)a.per, a.n - pos0);
    for (uint32_t i0 = 0; i0 < cnt; i0 += kSumThreads) {
        const uint32_t i = i0 + threadIdx.x;
        const unsigned long long m = __ballot(i < cnt && run_head(a.sk, (uint32_t)pos0 + i, a.rows));
        if (lane_id() == 0 && m) atomicAdd(&s_count, (uint32_t)__popcll(m));
    }
    __syncthreads();
    if (threadIdx.x == 0) a.first[blockIdx.x] = s_count;
}

// exclusive sums of the workgroups' counts in place; their total is the number of distinct rows
__global__ __launch_bounds__(kSumThreads) void scan_heads_kernel(SumArgs a)
{
    __shared__ uint32_t s_sum[kSumThreads];
    const uint32_t tid = threadIdx.x, each = (a.blocks + kSumThreads - 1) / kSumThreads;
    const uint32_t lo = min(tid * each, a.blocks), hi = min(lo + each, a.blocks);
    uint32_t sum = 0;
    for (uint32_t i = lo; i < hi; ++i) sum += a.first[i];
    s_sum[tid] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (uint32_t t = 0; t < tid; ++t) before += s_sum[t];
    for (uint32_t i = lo; i < hi; ++i) {
        const uint32_t c = a.first[i];
        a.first[i] = before;
        before += c;
    }
    if (tid == kSumThreads - 1) {
        a.ctl->distinct = a.ctl->bad ? 0u : before;
        if (a.count) *a.count = a.ctl->bad ? 0u : before;
    }
}

__device__ __forceinline__ void write_sum(const SumArgs &a, uint32_t row, uint32_t c, const double (&v)[4])
{
    f32x4 *to = (f32x4 *)(a.out + (size_t)row * a.D + c);
    double s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = v[i] * a.scale;
    if (a.accumulate) {
        const f32x4 old = *to;
        s[0] += (double)old.x;
        s[1] += (double)old.y;
        s[2] += (double)old.z;
        s[3] += (double)old.w;
    }
    *to = f32x4{(float)s[0], (float)s[1], (float)s[2], (float)s[3]};
}

template <typename T, bool DENSE>
__global__ __launch_bounds__(kSumThreads) void sum_runs_kernel(SumArgs a)
{
    typedef typename Quad<T>::type Four;
    constexpr uint32_t U = 4;                            // rows in flight
    __shared__ uint32_t s_key[kSumMost + 2];             // position i's at i + 1
    __shared__ uint32_t s_idx[kSumMost];
    __shared__ unsigned long long s_head[kSumMost / kWave];
    __shared__ uint32_t s_rank[kSumMost / kWave];        // of the heads in it and before
    __shared__ uint32_t s_state[kSumThreads], s_all, s_dest;
    __shared__ double s_part[2][kSumThreads][4];
    const uint32_t tid = threadIdx.x, b = blockIdx.x;
    const uint32_t pos0 = b * a.per, cnt = min(a.per, a.n - pos0);
    const uint32_t distinct = a.ctl->distinct;
    if (a.ctl->bad) {
        if (!DENSE)
            for (uint32_t i = tid; i < cnt; i += kSumThreads) a.out_keys[pos0 + i] = ECRM_NO_KEY;
        if (tid == 0) a.state[b] = 0;
        return;
    }
    for (uint32_t i = tid; i < cnt + 2u; i += kSumThreads) {
        const bool in = pos0 + i >= 1u && pos0 + i - 1u < a.n;
        s_key[i] = in ? a.sk[pos0 + i - 1u] : kNoKey;
        if (i < cnt) s_idx[i] = a.si[pos0 + i];
    }
    s_state[tid] = 0;
    if (tid == 0) s_all = 0;
    __syncthreads();
    for (uint32_t i0 = 0; i0 < cnt; i0 += kSumThreads) {
        const uint32_t i = i0 + tid;
        const bool head = i < cnt && s_key[i + 1] < a.rows && s_key[i + 1] != s_key[i];
        const unsigned long long m = __ballot(head);
        if (lane_id() == 0 && i < cnt) s_head[i / kWave] = m;
    }
    __syncthreads();
    if (tid < (cnt + kWave - 1) / kWave) {
        uint32_t before = a.first[b];
        for (uint32_t w = 0; w < tid; ++w) before += (uint32_t)__popcll(s_head[w]);
        s_rank[tid] = before;
    }
    __syncthreads();
    // the how-manieth distinct row position i has
    auto rank = [&](uint32_t i) {
        return s_rank[i / kWave] + (uint32_t)__popcll(s_head[i / kWave] & (~0ull >> (kWave - 1u - i % kWave))) - 1u;
    };
    if (!DENSE)
        for (uint32_t i = tid; i < cnt; i += kSumThreads) {
            if (s_key[i + 1] < a.rows && s_key[i + 1] != s_key[i]) a.out_keys[rank(i)] = s_key[i + 1];
            if (pos0 + i >= distinct) a.out_keys[pos0 + i] = ECRM_NO_KEY;
        }

    const uint32_t team = a.d4.div(tid), unit = tid - team * a.d4.d, c = unit * 4u;
    const bool live = team < a.teams;
    const T *d = (const T *)a.d + c;
    uint32_t tail_at = 0;
    if (live) {
        const uint32_t lo = team * a.chunk, hi = min(lo + a.chunk, cnt);
        uint32_t state = 0;
        double acc[4] = {0, 0, 0, 0};
        bool before = lo < hi && s_key[lo] == s_key[lo + 1], open = false;     // the run begins before the chunk; is not at its end
        for (uint32_t i0 = lo; i0 < hi; i0 += U) {
            if (s_key[i0 + 1] >= a.rows) break;
            Four v[U];
#pragma unroll
            for (uint32_t q = 0; q < U; ++q) v[q] = *(const Four *)(d + (size_t)s_idx[min(i0 + q, hi - 1u)] * a.stride);
#pragma unroll
            for (uint32_t q = 0; q < U; ++q) {
                const uint32_t i = i0 + q;
                if (i >= hi || s_key[i + 1] >= a.rows) break;
                const f32x4 g = widen4<T>(v[q]);
                acc[0] += (double)g.x;
                acc[1] += (double)g.y;
                acc[2] += (double)g.z;
                acc[3] += (double)g.w;
                open = s_key[i + 2] == s_key[i + 1];
                if (open) continue;
                if (before) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) s_part[0][tid][j] = acc[j];
                    state = kPartHead;
                    before = false;
                } else {
                    write_sum(a, DENSE ? s_key[i + 1] : rank(i), c, acc);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = 0;
            }
        }
        if (open) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s_part[before ? 0 : 1][tid][j] = acc[j];
            state |= before ? kPartHead | kPartThrough : kPartTail;
            tail_at = hi - 1u;
        }
        if (unit == 0) s_state[team] = state;
    }
    __syncthreads();
    if (live) {
        const uint32_t state = s_state[team];
        auto join = [&](uint32_t t, double (&acc)[4], bool through) {       // the run goes on behind team t
            while (through && ++t < a.teams) {
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] += s_part[0][t * a.d4.d + unit][j];
                through = (s_state[t] & kPartThrough) != 0;
            }
            return through;
        };
        if (team == 0 && (state & kPartHead)) {
            double acc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = s_part[0][tid][j];
            const bool through = join(0, acc, (state & kPartThrough) != 0);
            double *to = a.part + (size_t)b * 2u * a.D + c;
#pragma unroll
            for (int j = 0; j < 4; ++j) to[j] = acc[j];
            if (unit == 0) atomicOr(&s_all, through ? kPartHead | kPartThrough : kPartHead);
        }
        if (state & kPartTail) {
            double acc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = s_part[1][tid][j];
            const uint32_t row = DENSE ? s_key[tail_at + 1] : rank(tail_at);
            if (join(team, acc, true)) {
                double *to = a.part + ((size_t)b * 2u + 1u) * a.D + c;
#pragma unroll
                for (int j = 0; j < 4; ++j) to[j] = acc[j];
                if (unit == 0) {
                    atomicOr(&s_all, (uint32_t)kPartTail);
                    s_dest = row;
                }
            } else {
                write_sum(a, row, c, acc);
            }
        }
    }
    __syncthreads();
    if (tid == 0) {
        a.state[b] = s_all;
        if (s_all & kPartTail) a.dest[b] = s_dest;
    }
}

// The runs that began in one workgroup of sum_runs_kernel and ended in a later one.
__global__ __launch_bounds__(kSumThreads) void join_runs_kernel(SumArgs a)
{
    __shared__ double s_part[kSumThreads][4];
    const uint32_t b = blockIdx.x, tid = threadIdx.x, lane = lane_id();
    if (!(a.state[b] & kPartTail)) return;
    uint32_t end = b + 1u;                               // one behind the last workgroup that has a part of the run
    for (;;) {
        const bool through = end + lane < a.blocks && (a.state[end + lane] & kPartThrough);
        const unsigned long long ends = ~__ballot(through);
        if (ends) {
            end += (uint32_t)__builtin_ctzll(ends) + 1u;
            break;
        }
        end += kWave;
    }
    end = min(end, a.blocks);
    const uint32_t team = a.d4.div(tid), unit = tid - team * a.d4.d, c = unit * 4u;
    const uint32_t parts = end - (b + 1u), each = (parts + a.teams - 1) / a.teams;
    double acc[4] = {0, 0, 0, 0};
    if (team < a.teams) {
        const uint32_t lo = min(b + 1u + team * each, end), hi = min(lo + each, end);
#pragma unroll 4
        for (uint32_t t = lo; t < hi; ++t) {
            const double2 *p = (const double2 *)(a.part + (size_t)t * 2u * a.D + c);
            const double2 x = p[0], y = p[1];
            acc[0] += x.x;
            acc[1] += x.y;
            acc[2] += y.x;
            acc[3] += y.y;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) s_part[tid][j] = acc[j];
    }
    __syncthreads();
    if (team != 0) return;
    const double2 *p = (const double2 *)(a.part + ((size_t)b * 2u + 1u) * a.D + c);
    const double2 x = p[0], y = p[1];
    acc[0] = x.x;
    acc[1] = x.y;
    acc[2] = y.x;
    acc[3] = y.y;
    for (uint32_t t = 0; t < a.teams; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += s_part[t * a.d4.d + unit][j];
    write_sum(a, a.dest[b], c, acc);
}

__global__ __launch_bounds__(kSumThreads) void clear_rows_kernel(const TokenControl *ctl, f32x4 *to, uint64_t n)
{
    if (ctl && ctl->bad) return;
    for (uint64_t i = (uint64_t)blockIdx.x * kSumThreads + threadIdx.x; i < n; i += (uint64_t)gridDim.x * kSumThreads)
        to[i] = f32x4{0.f, 0.f, 0.f, 0.f};
}

__global__ void no_rows_kernel(uint64_t *count)
{
    if (threadIdx.x == 0) *count = 0;
}

// ---- host side -------------------------------------------------------------------------------------------------------------
struct SumPlan { uint32_t teams, chunk, per, blocks; };
static SumPlan sum_plan(uint32_t n, uint32_t D)
{
    SumPlan p;
    p.teams = (uint32_t)kSumThreads / (D / 4u);
    const uint32_t most = kSumMost / p.teams < kChunkMax ? kSumMost / p.teams : kChunkMax;
    p.chunk = (uint32_t)(((uint64_t)n + (uint64_t)p.teams * kSumBlocks - 1) / ((uint64_t)p.teams * kSumBlocks));
    if (p.chunk < kChunkMin) p.chunk = kChunkMin;
    if (p.chunk > most) p.chunk = most;
    p.per = p.teams * p.chunk;
    p.blocks = (n + p.per - 1) / p.per;
    return p;
}

EmbedGradLayout embed_grad_layout(size_t off, uint32_t max_batch, uint32_t D)
{
    // the most workgroups that any batch of up to max_batch tokens takes
    const SumPlan p = sum_plan(max_batch, D);
    const uint64_t least = ((uint64_t)max_batch + (uint64_t)p.teams * kChunkMin - 1) / ((uint64_t)p.teams * kChunkMin);
    const uint32_t blocks = p.blocks > kSumBlocks ? p.blocks : (uint32_t)(least < kSumBlocks ? least : kSumBlocks);
    EmbedGradLayout l;
    auto take = [&](size_t bytes) { const size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
    l.off_ctl = take(sizeof(TokenControl));
    l.off_first = take((size_t)blocks * 4);
    l.off_state = take((size_t)blocks * 4);
    l.off_dest = take((size_t)blocks * 4);
    l.off_part = take((size_t)blocks * 2 * D * sizeof(double));
    l.end = off;
    return l;
}

void launch_embed_grad(const Scratch &s, const EmbedGradLayout &l, const Geometry &g, int key_bits, const uint64_t *keys,
                       const void *d, uint32_t type, uint64_t stride, uint32_t n, uint64_t padding, float scale,
                       uint64_t *out_keys, float *out, uint64_t *count, bool accumulate, int cus, hipStream_t st)
{
    const bool dense = !out_keys;
    const dim3 clear_grid((uint32_t)cus * 8u), threads(kSumThreads);
    const uint64_t quads = (uint64_t)g.rows * (g.D / 4u);
    if (n == 0) {
        if (!dense) hipLaunchKernelGGL(no_rows_kernel, dim3(1), dim3(64), 0, st, count);
        else if (!accumulate)
            hipLaunchKernelGGL(clear_rows_kernel, clear_grid, threads, 0, st, (const TokenControl *)nullptr, (f32x4 *)out, quads);
        return;
    }
    char *base = (char *)s.hdr;
    SumArgs a{};
    const SumPlan p = sum_plan(n, g.D);
    a.n = n; a.rows = g.rows; a.D = g.D; a.d4 = make_divider(g.D / 4u);
    a.teams = p.teams; a.chunk = p.chunk; a.per = p.per; a.blocks = p.blocks;
    a.d = d; a.stride = stride; a.scale = (double)scale; a.accumulate = accumulate ? 1u : 0u;
    a.ctl = (TokenControl *)(base + l.off_ctl);
    a.first = (uint32_t *)(base + l.off_first);
    a.state = (uint32_t *)(base + l.off_state);
    a.dest = (uint32_t *)(base + l.off_dest);
    a.part = (double *)(base + l.off_part);
    a.out_keys = out_keys; a.out = out; a.count = count;
    hipLaunchKernelGGL(token_begin_kernel, dim3(1), dim3(64), 0, st, a.ctl);
    hipLaunchKernelGGL(token_keys_kernel, dim3((n + kTokenTile - 1) / kTokenTile), dim3(kTokenThreads), 0, st, keys, n, padding,
                       g.rows, s.keys[1], s.vals[1], s.hdr, a.ctl);
    if (dense && !accumulate) hipLaunchKernelGGL(clear_rows_kernel, clear_grid, threads, 0, st, a.ctl, (f32x4 *)out, quads);
    uint32_t *sk, *si;
    launch_sort_pairs(s, g, n, key_bits, &sk, &si, st);
    a.sk = sk; a.si = si;
    hipLaunchKernelGGL(count_heads_kernel, dim3(a.blocks), threads, 0, st, a);
    hipLaunchKernelGGL(scan_heads_kernel, dim3(1), threads, 0, st, a);
    with_type(type, [&](auto t) {
        if (dense) hipLaunchKernelGGL((sum_runs_kernel<decltype(t), true>), dim3(a.blocks), threads, 0, st, a);
        else hipLaunchKernelGGL((sum_runs_kernel<decltype(t), false>), dim3(a.blocks), threads, 0, st, a);
    });
    hipLaunchKernelGGL(join_runs_kernel, dim3(a.blocks), threads, 0, st, a);
}

}  // namespace ecrm
