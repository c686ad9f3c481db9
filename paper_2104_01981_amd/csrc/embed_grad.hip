// Gradient of the lookup by sorted tokens: the gradient of row x is scale * the sum of the gradients of the looked-up rows
// whose token is x.  The tokens are sorted, stably, with the index of their row; the sorted positions are cut into chunks of
// equal length, whatever the runs of equal tokens in them, so that a token that is a tenth of a batch takes no longer than
// others.  A team of D / 4 lanes, four columns to a lane, walks a chunk: the sum of a run that lies inside the chunk is
// written at once, what a chunk has of runs that go on before or behind it is joined in LDS by the workgroup, and what a
// workgroup has of runs that go on in its neighbours by a launch behind.  Sums are carried in 64 bits and rounded once, in
// an order that follows from the sorted positions, n and D alone: no atomics, two runs give the same bits.
//
// What bounds it: in large batches memory -- 2^20 tokens of 128 floats, hardly any twice, 228 us, of which the sums 164: 933 MB
// at 5.7 TB/s, in part from the memory-side cache --, in small ones the trips to memory that follow from one another: a launch (up to
// kSortHere tokens, 6.8 us for 64), two (up to kOneBlock, 11 us for 600), three (up to kRankMost), five (up to 2^16; four for the dense
// form, which counts no rows), then two for each digit of the sort, or three, and three or four behind it: five to nine up to 2^18
// tokens, six to sixteen beyond (twelve for rows of 19 to 27 bits).  Of 2^16 tokens of text with 256 floats in bf16, 42 us, the sums
// take 16, the sort 20 and the join 4; with dropout (mask.h), which the sums draw again, the sums take 20, of 2^20 tokens 177.
#include "mask.h"

namespace ecrm {

constexpr int kSumThreads = 256;
constexpr uint32_t kSumMost = 2048;       // sorted positions of a workgroup, at most
// Batches of up to kSortHere tokens are sorted by every workgroup for itself (64 tokens: 6.8 us, with a launch for it 9.6; 256: 8.5
// and 10).  Batches of up to kOneBlock tokens are cut by columns, not by positions: nothing is left to join (1024 tokens of text
// 12.9 us, 14.8 with positions cut; 2048 18.1 and 16.0), kOneUnits times four columns to a workgroup (1, 2, 4: 600 tokens 11.1,
// 11.3, 12.6, all one token 13.2, 13.1, 12.5; 1024 of 1024 floats 15.8, 14.0, 14.9).
constexpr uint32_t kSortHere = 256, kOneBlock = 1536, kOneUnits = 2;
// Workgroups, unless that would be more positions to one than there is room for.  2^16 tokens of 256 floats with 1024, 1536, 2048,
// 4096 (with the radix sort): 44.3, 45.0, 46.7, 51.2 us (a run that goes over several costs a join); 2^20 of 128 floats 251, 253, 252, 243, so at most
// chunk_max (below) positions to a team.
constexpr uint32_t kSumBlocks = 1024;
constexpr uint32_t kPerMin = 8;           // positions of a workgroup, at least (4, 8, 16 of 1024 floats: 4096 tokens 24.7, 23.1, 24.8 us)
constexpr uint32_t kChunkMin = 4;         // positions of a team, which are on their way together
constexpr uint32_t kCountThreads = 1024;
constexpr uint32_t kCountGroup = 8;       // workgroups whose distinct rows are counted together
constexpr uint32_t kScanGroups = 1024;    // from more on these counts are added up by a launch of its own
// Where more than this goes in and out -- the rows, and the output as if no token came twice --, rows are read and written past the
// caches, eight of a team in flight instead of four.  Whether that pays depends on where the rows are, which nobody here knows.  Time
// so / as usual, widths 64 to 1024, 16 and 32 bits (rows; dense; added to what is there), in batches by turns, 600 MiB of them:
// up to 60 MiB 0.98; 1.03; 1.04, 60 to 100 1.05; 0.98; 0.96, 100 to 200 of text 0.98; 0.98; 0.96, of unlike tokens 1.03; 1.02; 0.98,
// 200 to 300 of text 0.96; 0.94; 0.91, of unlike tokens 1.07; 1.02; 0.97, beyond 400 0.94 for rows, beyond 300 0.90 to 0.99 for the others.
// With one batch again and again, which the memory-side cache holds as a whole, it loses 3 to 14 % up to 300 MiB and gains as much beyond 400.
constexpr uint64_t kStreamBytes = 100ull << 20;
// Of these rows a quarter, but no more than kNearBytes, is read into the memory-side cache beside the sort, the first ones: what was
// written last is there anyway.  120 MB: of 2^20 items 160 MB took 231 us, 240 MB 235.  2^20 items of 128 floats 239 us without, 228 so; 65536 of 512 floats 77.6 and 73.0, with half of the
// rows 71.8; 18001 of 1024 in bf16 45.6 and 44.9; 2^19 of text with 128 in bf16 99.7 and 100.9, with half of them 103.4.
constexpr uint64_t kNearBytes = 114ull << 20;
constexpr uint32_t kJoinUnits = 16;       // of four columns, of a job
constexpr uint32_t kLongJoin = 16;        // workgroups from which on a run is a long one

// What a workgroup has of a run that goes on before it (and maybe behind it) and of one that begins in it and goes on behind it
// (by more than kLongJoin workgroups).
enum { kPartHead = 1, kPartThrough = 2, kPartTail = 4, kPartLong = 8 };
// Where the number of distinct rows before a workgroup's positions comes from.
enum { kCountKeys = 0, kAddCounts = 1, kScanned = 2, kAllHere = 3 };

struct SumArgs {
    const uint64_t *keys;            // up to kSortHere tokens: the caller's
    uint64_t padding;
    uint32_t rows;
    Header *hdr;
    const uint32_t *sk, *si;         // sorted: row, index of the gradient
    uint32_t n, D;
    uint32_t quads;                  // D / 4
    Divider units;                   // by the quads of a workgroup: all, or, where one workgroup has all positions, a few
    uint32_t teams, chunk, per;      // teams of a workgroup, positions of a chunk, of a workgroup
    uint32_t blocks;
    uint32_t counting;
    const void *d;                   // [n][stride] gradients of the looked-up rows
    uint64_t stride;
    MaskArgs mask;                   // with dropout: which elements of d count; its factor is in the scale
    double scale;
    uint32_t accumulate;             // dense: add to what is there
    TokenControl *ctl;
    uint32_t groups;                 // of kCountGroup workgroups
    uint32_t *first;                 // [blocks] distinct rows that begin in the group's positions before the workgroup's
    uint32_t *group;                 // [groups] distinct rows that begin in it; scanned: before it
    uint32_t *state;                 // [blocks] kPart*
    uint32_t *dest;                  // [blocks] row of the output that a kPartTail belongs to
    uint32_t *join;                  // [blocks] workgroups with a kPartLong, in any order
    double *part;                    // [blocks][2][D]: head, tail
    uint64_t *out_keys;              // rows form
    float *out;
    uint64_t *count;
};

// sums of v and w over the workgroup, to all
__device__ __forceinline__ uint32_t block_totals(uint32_t v, uint32_t w, uint2 *s_wave, uint32_t &of_w)
{
#pragma unroll
    for (int by = 1; by < kWave; by <<= 1) {
        v += (uint32_t)__shfl_xor((int)v, by, kWave);
        w += (uint32_t)__shfl_xor((int)w, by, kWave);
    }
    if (lane_id() == 0) s_wave[threadIdx.x / kWave] = uint2{v, w};
    __syncthreads();
    v = of_w = 0;
#pragma unroll
    for (int i = 0; i < kSumThreads / kWave; ++i) {
        v += s_wave[i].x;
        of_w += s_wave[i].y;
    }
    return v;
}

__global__ __launch_bounds__(kCountThreads) void count_heads_kernel(SumArgs a)
{
    __shared__ uint32_t s_heads[kCountGroup];
    const uint32_t tid = threadIdx.x;
    if (tid < kCountGroup) s_heads[tid] = 0;
    __syncthreads();
    const uint64_t pos0 = (uint64_t)blockIdx.x * kCountGroup * a.per;
    const uint32_t cnt = (uint32_t)min((uint64_t)kCountGroup * a.per, a.n - pos0), valid = a.ctl->valid;
    for (uint32_t i0 = 0; i0 < cnt; i0 += kCountThreads) {
        const uint32_t i = i0 + tid, p = min((uint32_t)pos0 + i, a.n - 1u), key = a.sk[p], last = a.sk[p ? p - 1u : 0u];
        const bool head = i < cnt && p < valid && (p == 0 || key != last);
        // a wave's at once where they are one workgroup's
        const uint32_t w0 = (i - lane_id()) / a.per;
        if ((i - lane_id() + kWave - 1u) / a.per == w0) {
            const unsigned long long m = __ballot(head);
            if (lane_id() == 0 && m) atomicAdd(&s_heads[w0], (uint32_t)__popcll(m));
        } else if (head) {
            atomicAdd(&s_heads[i / a.per], 1u);
        }
    }
    __syncthreads();
    if (tid >= kCountGroup) return;
    uint32_t before = 0;
    for (uint32_t j = 0; j < tid; ++j) before += s_heads[j];
    const uint32_t b = blockIdx.x * kCountGroup + tid;
    if (b < a.blocks) a.first[b] = before;
    if (tid == kCountGroup - 1) a.group[blockIdx.x] = before + s_heads[tid];
}

// exclusive sums of the groups' counts in place; their total is the number of distinct rows
__global__ __launch_bounds__(1024) void scan_heads_kernel(SumArgs a)
{
    __shared__ uint32_t s_wave[16];
    uint32_t carry = 0;
    for (uint32_t b0 = 0; b0 < a.groups; b0 += 1024u) {
        const uint32_t i = b0 + threadIdx.x, v = i < a.groups ? a.group[i] : 0u;
        uint32_t incl = v;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const uint32_t t = (uint32_t)__shfl_up((int)incl, d, kWave);
            if (lane_id() >= (uint32_t)d) incl += t;
        }
        if (lane_id() == kWave - 1) s_wave[threadIdx.x / kWave] = incl;
        __syncthreads();
        uint32_t before = carry;
        for (uint32_t w = 0; w < 16u; ++w) {
            if (w < threadIdx.x / kWave) before += s_wave[w];
            carry += s_wave[w];
        }
        if (i < a.groups) a.group[i] = before + incl - v;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.ctl->distinct = carry;
}

// The distinct rows before sorted position pos0, and (valid, not SCANNED) in all.
__device__ __forceinline__ uint32_t distinct_before(const SumArgs &a, uint32_t pos0, uint32_t valid, uint2 *s_wave, uint32_t &distinct)
{
    if (a.counting == kScanned) {
        distinct = a.ctl->distinct;
        return a.group[blockIdx.x / kCountGroup] + a.first[blockIdx.x];
    }
    const uint32_t tid = threadIdx.x;
    uint32_t before = 0, all = 0;
    if (a.counting == kAddCounts) {
        const uint32_t own = blockIdx.x / kCountGroup;
        const uint32_t here = a.first[blockIdx.x];
#pragma unroll
        for (uint32_t j = 0; j < kScanGroups / kSumThreads; ++j) {
            const uint32_t g = j * kSumThreads + tid, c = a.group[min(g, a.groups - 1u)];
            all += g < a.groups ? c : 0u;
            before += g < own ? c : 0u;
        }
        if (tid == 0) before += here;
    } else {
#pragma unroll 2
        for (uint32_t p = tid * 4u; p < valid; p += 4u * kSumThreads) {
            const uint4 k = *(const uint4 *)(a.sk + p);        // room for a multiple of four
            const uint32_t left = a.sk[p ? p - 1u : 0u], last = p ? left : kNoKey;
            const uint32_t h[4] = {k.x != last ? 1u : 0u, k.y != k.x ? 1u : 0u, k.z != k.y ? 1u : 0u, k.w != k.z ? 1u : 0u};
#pragma unroll
            for (uint32_t q = 0; q < 4u; ++q) {
                all += p + q < valid ? h[q] : 0u;
                before += p + q < valid && p + q < pos0 ? h[q] : 0u;
            }
        }
    }
    return block_totals(before, all, s_wave, distinct);
}

template <bool STREAM>
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
    const f32x4 sum = {(float)s[0], (float)s[1], (float)s[2], (float)s[3]};
    if (STREAM) __builtin_nontemporal_store(sum, to);
    else *to = sum;
}

// Sorts the batch's tokens, one to a thread, into s_key (position i's at i + 1) and s_idx: how many are rows; none if one is bad.
__device__ __forceinline__ uint32_t sort_here(const SumArgs &a, uint32_t *s_raw, uint32_t *s_key, uint32_t *s_idx, uint2 *s_wave)
{
    const uint32_t tid = threadIdx.x, n = a.n;
    const uint64_t word = a.keys[min(tid, n - 1u)];
    const bool in = tid < n, pad = in && is_padding(word, a.padding), bad = in && !pad && word >= (uint64_t)a.rows;
    const uint32_t key = in && !pad ? (uint32_t)word : kNoKey;
    s_raw[tid] = key;
    uint32_t bads;
    const uint32_t pads = block_totals(pad ? 1u : 0u, bad ? 1u : 0u, s_wave, bads);      // a barrier
    const uint32_t valid = bads ? 0u : n - pads, wave0 = tid / kWave * kWave, end = (n + 3u) / 4u * 4u;
    if (bads && tid == 0 && blockIdx.y == 0) atomicOr(&a.hdr->err_sticky, 1u);
    uint32_t at = 0;                                     // tokens before: of equal ones those of smaller index
#pragma unroll 8
    for (uint32_t j = 0; j < wave0; j += 4u) {
        const uint4 k = *(const uint4 *)(s_raw + j);
        at += (k.x <= key ? 1u : 0u) + (k.y <= key ? 1u : 0u) + (k.z <= key ? 1u : 0u) + (k.w <= key ? 1u : 0u);
    }
#pragma unroll 4
    for (uint32_t j = wave0; j < min(wave0 + kWave, end); j += 4u) {
        const uint4 k = *(const uint4 *)(s_raw + j);
        at += (k.x < key || (k.x == key && j < tid) ? 1u : 0u) + (k.y < key || (k.y == key && j + 1u < tid) ? 1u : 0u) +
              (k.z < key || (k.z == key && j + 2u < tid) ? 1u : 0u) + (k.w < key || (k.w == key && j + 3u < tid) ? 1u : 0u);
    }
#pragma unroll 8
    for (uint32_t j = wave0 + kWave; j < end; j += 4u) {
        const uint4 k = *(const uint4 *)(s_raw + j);
        at += (k.x < key ? 1u : 0u) + (k.y < key ? 1u : 0u) + (k.z < key ? 1u : 0u) + (k.w < key ? 1u : 0u);
    }
    if (in && !pad && !bads) {
        s_key[at + 1u] = key;
        s_idx[at] = tid;
    }
    if (tid == 0) s_key[0] = s_key[valid + 1u] = kNoKey;
    return valid;
}

// STREAM: rows are moved past the caches (kStreamBytes).  HERE: up to kSortHere tokens, sorted here.  DROP: the lookup had dropout.
template <typename T, bool DENSE, bool STREAM, bool HERE, bool DROP>
__global__ __launch_bounds__(kSumThreads) void sum_runs_kernel(SumArgs a)
{
    typedef typename Quad<T>::type Four;
    constexpr uint32_t U = STREAM ? 8 : 4;               // rows in flight
    extern __shared__ uint32_t lds[];
    uint32_t *s_key = lds, *s_idx = lds + a.per + 2u;    // position i's key at i + 1
    __shared__ unsigned long long s_head[DENSE ? 1 : kSumMost / kWave];
    __shared__ uint32_t s_rank[DENSE ? 1 : kSumMost / kWave];          // of the heads before it
    __shared__ uint32_t s_state[kSumThreads], s_all, s_dest, s_key_of_tail, s_all_heads;
    __shared__ uint2 s_wave[kSumThreads / kWave];
    __shared__ unsigned long long s_through[kSumThreads / kWave];
    __shared__ double s_part[2][kSumThreads][4];
    const uint32_t tid = threadIdx.x, b = blockIdx.x;
    const uint32_t pos0 = b * a.per, room = min(a.per, a.n - pos0);
    const bool lists = !DENSE && blockIdx.y == 0;        // the keys are written once, not for every slice of columns
    uint32_t valid;
    s_state[tid] = 0;
    if (tid == 0) s_all = 0;
    if (HERE) {
        __shared__ __align__(16) uint32_t s_raw[HERE ? kSortHere : 1];
        valid = sort_here(a, s_raw, s_key, s_idx, s_wave);
    } else {
        for (uint32_t i0 = 0; i0 < room + 2u; i0 += 4u * kSumThreads) {    // behind `valid` the buffers hold anything
            uint32_t key[4], idx[4];
#pragma unroll
            for (uint32_t q = 0; q < 4u; ++q) {
                const uint32_t i = i0 + q * kSumThreads + tid;
                key[q] = a.sk[min(max(pos0 + i, 1u) - 1u, a.n - 1u)];
                idx[q] = a.si[min(pos0 + i, a.n - 1u)];
            }
#pragma unroll
            for (uint32_t q = 0; q < 4u; ++q) {
                const uint32_t i = i0 + q * kSumThreads + tid;
                if (i < room + 2u) s_key[i] = pos0 + i >= 1u && pos0 + i - 1u < a.n ? key[q] : kNoKey;
                if (i < room) s_idx[i] = idx[q];
            }
        }
        valid = a.ctl->bad ? 0u : a.ctl->valid;
    }
    const uint32_t cnt = pos0 < valid ? min(room, valid - pos0) : 0u;
    __syncthreads();
    if (!HERE && (cnt < room || pos0 + room == valid)) {
        if (tid == 0) s_key[cnt + 1u] = kNoKey;
        __syncthreads();
    }

    // the first rows are on their way while the heads are counted
    const uint32_t team = a.units.div(tid), mine = tid - team * a.units.d, unit = blockIdx.y * a.units.d + mine, c = unit * 4u;
    const uint32_t lo = min(team * a.chunk, cnt), hi = min(lo + a.chunk, cnt);
    const bool live = team < a.teams && unit < a.quads;
    const T *d = (const T *)a.d + c;
    Four v[U];
    auto load = [&](uint32_t i0) {
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) {
            const Four *row = (const Four *)(d + (size_t)s_idx[min(i0 + q, hi - 1u)] * a.stride);
            v[q] = STREAM ? __builtin_nontemporal_load(row) : *row;
        }
    };
    if (live && lo < hi) load(lo);
    if (!DENSE) {
        for (uint32_t i0 = 0; i0 < cnt; i0 += kSumThreads) {
            const uint32_t i = i0 + tid;
            const unsigned long long m = __ballot(i < cnt && s_key[min(i, cnt) + 1u] != s_key[min(i, cnt)]);
            if (lane_id() == 0 && i < cnt) s_head[i / kWave] = m;
        }
        uint32_t distinct = 0, first = 0;
        if (a.counting != kAllHere) first = distinct_before(a, pos0, valid, s_wave, distinct);
        __syncthreads();
        if (tid < kWave) {                               // at most 32 words
            const uint32_t words = (cnt + kWave - 1) / kWave, heads = tid < words ? (uint32_t)__popcll(s_head[tid]) : 0u;
            uint32_t incl = heads;
#pragma unroll
            for (int by = 1; by < kWave / 2; by <<= 1) {
                const uint32_t t = (uint32_t)__shfl_up((int)incl, by, kWave);
                if (tid >= (uint32_t)by) incl += t;
            }
            if (tid < words) s_rank[tid] = first + incl - heads;
            if (tid == kWave / 2 - 1) s_all_heads = incl;
        }
        __syncthreads();
        if (a.counting == kAllHere) distinct = s_all_heads;
        if (valid == 0) distinct = 0;
        if (lists) {
            if (b == 0 && tid == 0) *a.count = distinct;
            for (uint32_t i = tid; i < room; i += kSumThreads)
                if (pos0 + i >= distinct) a.out_keys[pos0 + i] = ECRM_NO_KEY;
        }
    }
    // the how-manieth distinct row position i has
    auto rank = [&](uint32_t i) {
        return s_rank[i / kWave] + (uint32_t)__popcll(s_head[i / kWave] & (~0ull >> (kWave - 1u - i % kWave))) - 1u;
    };
    if (lists)
        for (uint32_t i = tid; i < cnt; i += kSumThreads)
            if (s_key[i + 1] != s_key[i]) a.out_keys[rank(i)] = s_key[i + 1];

    uint32_t tail_at = 0;
    if (live) {
        uint32_t state = 0;
        double acc[4] = {0, 0, 0, 0};
        MaskKey mask{};
        if (DROP) mask = mask_key(a.mask);
        bool before = lo < hi && s_key[lo] == s_key[lo + 1], open = false;     // the run begins before the chunk; is not at its end
        for (uint32_t i0 = lo; i0 < hi; i0 += U) {
            if (i0 != lo) load(i0);
            uint2 bits[U];
            if (DROP) {                                  // lanes 2i and 2i + 1 have columns 8j and 8j + 4 if teams begin at even ones
                uint32_t row[U], col[U];
#pragma unroll
                for (uint32_t q = 0; q < U; ++q) {
                    row[q] = s_idx[min(i0 + q, hi - 1u)];
                    col[q] = c;
                }
                mask_quads<U>(mask, row, col, a.units.d % 2u == 0 && a.quads % 2u == 0, bits);
            }
#pragma unroll
            for (uint32_t q = 0; q < U; ++q) {
                const uint32_t i = i0 + q;
                if (i >= hi) break;
                f32x4 g = widen4<T>(v[q]);
                if (DROP) g = keep4(g, bits[q], mask.border);
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
                    write_sum<STREAM>(a, DENSE ? s_key[i + 1] : rank(i), c, acc);
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
        if (mine == 0) s_state[team] = state;
    }
    __syncthreads();
    const unsigned long long through = __ballot((s_state[tid] & kPartThrough) != 0);       // of teams; there are no more than threads
    if (lane_id() == 0) s_through[tid / kWave] = through;
    __syncthreads();
    if (live) {
        const uint32_t state = s_state[team];
        // adds the parts behind team t's of a run that goes on there: does it go on behind the workgroup, too?
        auto join = [&](uint32_t t, double (&acc)[4]) {
            uint32_t end = a.teams;                      // the first behind t that the run does not go on behind
            for (uint32_t w = (t + 1u) / kWave; w < (uint32_t)(kSumThreads / kWave); ++w) {
                unsigned long long ends = ~s_through[w];
                if (w == (t + 1u) / kWave) ends &= ~0ull << ((t + 1u) % kWave);
                if (ends) {
                    end = min(end, w * kWave + (uint32_t)__builtin_ctzll(ends));
                    break;
                }
            }
            const uint32_t last = min(end + 1u, a.teams);
#pragma unroll 4
            for (uint32_t p = t + 1u; p < last; ++p)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] += s_part[0][p * a.units.d + mine][j];
            return end == a.teams;
        };
        if (team == 0 && (state & kPartHead)) {
            double acc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = s_part[0][tid][j];
            const bool on = (state & kPartThrough) && join(0, acc);
            double *to = a.part + (size_t)b * 2u * a.D + c;
#pragma unroll
            for (int j = 0; j < 4; ++j) to[j] = acc[j];
            if (mine == 0) atomicOr(&s_all, on ? kPartHead | kPartThrough : kPartHead);
        }
        if (state & kPartTail) {
            double acc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = s_part[1][tid][j];
            const uint32_t row = DENSE ? s_key[tail_at + 1] : rank(tail_at);
            if (join(team, acc)) {
                double *to = a.part + ((size_t)b * 2u + 1u) * a.D + c;
#pragma unroll
                for (int j = 0; j < 4; ++j) to[j] = acc[j];
                if (mine == 0) {
                    atomicOr(&s_all, (uint32_t)kPartTail);
                    s_dest = row;
                    s_key_of_tail = s_key[tail_at + 1];
                }
            } else {
                write_sum<STREAM>(a, row, c, acc);
            }
        }
    }
    if (a.blocks == 1) return;
    __syncthreads();
    if (tid == 0) {
        uint32_t state = s_all;
        if (state & kPartTail) {
            a.dest[b] = s_dest;
            const uint64_t far = ((uint64_t)b + kLongJoin) * a.per;
            if (far < valid && a.sk[far] == s_key_of_tail) {
                state |= kPartLong;
                a.join[atomicAdd(&a.ctl->joins, 1u)] = b;
            }
        }
        a.state[b] = state;
    }
}

// one behind the last workgroup that has a part of the run that begins in b
__device__ __forceinline__ uint32_t run_end(const SumArgs &a, uint32_t b)
{
    uint32_t end = b + 1u;
    for (;;) {
        const uint32_t at = end + lane_id();
        const unsigned long long ends = ~__ballot(at < a.blocks && (a.state[at] & kPartThrough));
        if (ends) return min(end + (uint32_t)__builtin_ctzll(ends) + 1u, a.blocks);
        end += kWave;
    }
}

__device__ __forceinline__ void add_part(const SumArgs &a, uint32_t b, uint32_t which, uint32_t c, double (&acc)[4])
{
    const double2 *p = (const double2 *)(a.part + ((size_t)b * 2u + which) * a.D + c);
    const double2 x = p[0], y = p[1];
    acc[0] += x.x;
    acc[1] += x.y;
    acc[2] += y.x;
    acc[3] += y.y;
}

// The runs that began in one workgroup of sum_runs_kernel and ended in a later one.  Short ones: a team each, part after part.
// Long ones, by the last `wide` workgroups: a job is a run and 64 columns, whose parts are added up by as many lanes side by side
// as there are, each a range of them in order.
__global__ __launch_bounds__(kSumThreads) void join_runs_kernel(SumArgs a, uint32_t wide)
{
    __shared__ double s_part[kSumThreads][4];
    const uint32_t tid = threadIdx.x, narrow = gridDim.x - wide;
    if (blockIdx.x < narrow) {
        const uint32_t team = a.units.div(tid), c = (tid - team * a.units.d) * 4u;
        if (team >= a.teams) return;
        for (uint32_t first = blockIdx.x * a.teams + team; first < a.blocks; first += narrow * a.teams) {
            if ((a.state[first] & (kPartTail | kPartLong)) != kPartTail) continue;
            const uint32_t to = a.dest[first];
            double acc[4] = {0, 0, 0, 0};
            add_part(a, first, 1u, c, acc);
            uint32_t on = 0;                             // the workgroups behind: does the run go on behind them, too?
#pragma unroll
            for (uint32_t j = 0; j < kLongJoin; ++j) on |= (a.state[min(first + 1u + j, a.blocks - 1u)] & kPartThrough ? 1u : 0u) << j;
            const uint32_t parts = (uint32_t)__builtin_ctz(~on) + 1u;
#pragma unroll 4
            for (uint32_t j = 0; j < parts; ++j) add_part(a, first + 1u + j, 0u, c, acc);
            write_sum<false>(a, to, c, acc);
        }
        return;
    }
    const uint32_t units = min(a.quads, kJoinUnits), groups = (a.quads + units - 1) / units, slices = kSumThreads / units;
    const uint32_t slice = tid / units, jobs = a.ctl->joins * groups;
    for (uint32_t job = blockIdx.x - narrow; job < jobs; job += wide) {
        const uint32_t first = a.join[job / groups];
        const uint32_t unit = job % groups * units + tid % units, c = unit * 4u;
        const uint32_t begin = first + 1u, parts = run_end(a, first) - begin, each = (parts + slices - 1) / slices;
        const bool live = slice < slices && unit < a.quads;
        double acc[4] = {0, 0, 0, 0};
        if (live) {
            const uint32_t lo = min(slice * each, parts), hi = min(lo + each, parts);
#pragma unroll 4
            for (uint32_t t = lo; t < hi; ++t) add_part(a, begin + t, 0u, c, acc);
#pragma unroll
            for (int j = 0; j < 4; ++j) s_part[tid][j] = acc[j];
        }
        __syncthreads();
        if (live && slice == 0) {
            double all[4] = {0, 0, 0, 0};
            add_part(a, first, 1u, c, all);
            for (uint32_t t = 0; t < slices && t * each < parts; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) all[j] += s_part[t * units + tid][j];
            write_sum<false>(a, a.dest[first], c, all);
        }
        __syncthreads();
    }
}

__global__ __launch_bounds__(kSumThreads) void clear_rows_kernel(f32x4 *to, uint64_t n)
{
    for (uint64_t i = (uint64_t)blockIdx.x * kSumThreads + threadIdx.x; i < n; i += (uint64_t)gridDim.x * kSumThreads)
        to[i] = f32x4{0.f, 0.f, 0.f, 0.f};
}

__global__ void no_rows_kernel(uint64_t *count)
{
    if (threadIdx.x == 0) *count = 0;
}

// ---- host side -------------------------------------------------------------------------------------------------------------
struct SumPlan { uint32_t units, teams, chunk, per, blocks, slices; };
static SumPlan sum_plan(uint32_t n, uint32_t D)
{
    SumPlan p;
    const uint32_t quads = D / 4u;
    p.units = n <= kOneBlock && quads > kOneUnits ? kOneUnits : quads;
    p.slices = (quads + p.units - 1) / p.units;
    p.teams = (uint32_t)kSumThreads / p.units;
    // What the parts of runs take in the scratch buffer grows with D * D / chunk_max: of large batches 32, 64, 128 bytes a token.  The
    // up to kSumBlocks workgroups of smaller ones have 16 * D each, however few their tokens: 2 KB a token of 8192 with 1024 floats.
    const uint32_t room = kSumMost / p.teams, chunk_max = D <= 256 ? 32u : D <= 512 ? 64u : 128u;
    const uint32_t most = n <= kOneBlock || room < chunk_max ? room : chunk_max;
    const uint64_t wanted = n <= kOneBlock ? p.teams : (uint64_t)p.teams * kSumBlocks;
    p.chunk = (uint32_t)((n + wanted - 1) / wanted);
    const uint32_t chunk_min = p.teams * kChunkMin < kPerMin ? kPerMin / p.teams : kChunkMin;
    if (p.chunk < chunk_min) p.chunk = chunk_min;
    if (p.chunk > most) p.chunk = most;
    p.per = p.teams * p.chunk;
    p.blocks = (n + p.per - 1) / p.per;
    return p;
}

EmbedGradLayout embed_grad_layout(size_t off, uint32_t max_batch, uint32_t D, int key_bits)
{
    EmbedGradLayout l;
    l.sort = token_sort_layout(off, max_batch, key_bits);
    off = l.sort.end;
    // the most workgroups that any batch of up to max_batch tokens takes: more than kSumBlocks have as many positions as one can
    const SumPlan p = sum_plan(max_batch, D);
    const uint32_t per_min = p.teams * kChunkMin < kPerMin ? kPerMin : p.teams * kChunkMin;
    const uint32_t least = (uint32_t)(((uint64_t)max_batch + per_min - 1) / per_min);
    const uint32_t few = least < kSumBlocks ? least : kSumBlocks, blocks = max_batch <= kOneBlock ? 1u : p.blocks > few ? p.blocks : few;
    auto take = [&](size_t bytes) { const size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
    l.off_first = take((size_t)blocks * 4);
    l.off_group = take(((size_t)blocks / kCountGroup + 1) * 4);
    l.off_state = take((size_t)blocks * 4);
    l.off_dest = take((size_t)blocks * 4);
    l.off_join = take((size_t)blocks * 4);
    l.off_part = take((size_t)blocks * 2 * D * sizeof(double));
    l.end = off;
    return l;
}

template <typename T, bool DENSE, bool DROP>
static void launch_sum(const SumArgs &a, dim3 grid, size_t lds, bool stream, hipStream_t st)
{
    const dim3 threads(kSumThreads);
    if (a.keys) hipLaunchKernelGGL((sum_runs_kernel<T, DENSE, false, true, DROP>), grid, threads, lds, st, a);
    else if (stream) hipLaunchKernelGGL((sum_runs_kernel<T, DENSE, true, false, DROP>), grid, threads, lds, st, a);
    else hipLaunchKernelGGL((sum_runs_kernel<T, DENSE, false, false, DROP>), grid, threads, lds, st, a);
}

void launch_embed_grad(const Scratch &s, const EmbedGradLayout &l, const Geometry &g, int key_bits, const uint64_t *keys,
                       const void *d, uint32_t type, uint64_t stride, uint32_t n, uint64_t padding, double scale,
                       const MaskArgs *mask, uint64_t *out_keys, float *out, uint64_t *count, bool accumulate, int cus,
                       hipStream_t st)
{
    const bool dense = !out_keys;
    const dim3 threads(kSumThreads);
    BesideJob beside{};
    if (dense && !accumulate) {
        beside.to = out;
        beside.count = (uint64_t)g.rows * (g.D / 4u);
    }
    if (n == 0) {
        if (!dense) hipLaunchKernelGGL(no_rows_kernel, dim3(1), dim3(64), 0, st, count);
        if (beside.to) hipLaunchKernelGGL(clear_rows_kernel, dim3((uint32_t)cus * 8u), threads, 0, st, (f32x4 *)beside.to, beside.count);
        return;
    }
    const uint32_t size = type_bytes(type);
    const uint64_t moved = (uint64_t)n * g.D * size + (dense ? (uint64_t)g.rows : n) * g.D * 4u;
    const bool stream = moved > kStreamBytes;
    if (stream && !beside.to && n > kRankMost && g.D * size % 16u == 0 && stride * size % 16u == 0 && (uintptr_t)d % 16u == 0) {
        const uint64_t units = (uint64_t)n * (g.D * size / 16u);
        beside.from = (const char *)d;
        beside.stride = stride * size;
        beside.row = make_divider(g.D * size / 16u);
        beside.count = units / 4u < kNearBytes / 16u ? units / 4u : kNearBytes / 16u;
    }
    char *base = (char *)s.hdr;
    SumArgs a{};
    // every workgroup of the sums reads the tokens where it sorts them itself: not where the first one writes the distinct keys
    const bool in_place = out_keys && out_keys < keys + n && keys < out_keys + n;
    if (n <= kSortHere && !beside.to && !in_place) {
        a.keys = keys; a.padding = padding; a.rows = g.rows; a.hdr = s.hdr;
    } else {
        const TokenSort sorted = launch_token_sort(s, l.sort, keys, n, padding, g.rows, key_bits, beside, cus, st);
        a.sk = sorted.sk; a.si = sorted.si; a.ctl = sorted.ctl;
    }
    const SumPlan p = sum_plan(n, g.D);
    a.n = n; a.D = g.D; a.quads = g.D / 4u; a.units = make_divider(p.units);
    a.teams = p.teams; a.chunk = p.chunk; a.per = p.per; a.blocks = p.blocks;
    a.d = d; a.stride = stride; a.scale = scale; a.accumulate = accumulate ? 1u : 0u;
    a.first = (uint32_t *)(base + l.off_first);
    a.group = (uint32_t *)(base + l.off_group);
    a.groups = (a.blocks + kCountGroup - 1) / kCountGroup;
    a.state = (uint32_t *)(base + l.off_state);
    a.dest = (uint32_t *)(base + l.off_dest);
    a.join = (uint32_t *)(base + l.off_join);
    a.part = (double *)(base + l.off_part);
    a.out_keys = out_keys; a.out = out; a.count = count;
    if (mask) a.mask = *mask;
    a.counting = a.blocks == 1 ? kAllHere : n <= kRankMost ? kCountKeys : a.groups <= kScanGroups ? kAddCounts : kScanned;
    if (!dense && (a.counting == kAddCounts || a.counting == kScanned)) {
        hipLaunchKernelGGL(count_heads_kernel, dim3(a.groups), dim3(kCountThreads), 0, st, a);
        if (a.counting == kScanned) hipLaunchKernelGGL(scan_heads_kernel, dim3(1), dim3(1024), 0, st, a);
    }
    const size_t lds = ((size_t)a.per * 2 + 2) * 4;
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        const dim3 grid(a.blocks, p.slices);
        if (mask && dense) launch_sum<T, true, true>(a, grid, lds, stream, st);
        else if (mask) launch_sum<T, false, true>(a, grid, lds, stream, st);
        else if (dense) launch_sum<T, true, false>(a, grid, lds, stream, st);
        else launch_sum<T, false, false>(a, grid, lds, stream, st);
    });
    if (a.blocks > 1) {
        const uint32_t narrow = (a.blocks + a.teams - 1) / a.teams, most = (uint32_t)cus * 8u, wide = (uint32_t)cus;
        hipLaunchKernelGGL(join_runs_kernel, dim3((narrow < most ? narrow : most) + wide), threads, 0, st, a, wide);
    }
}

}  // namespace ecrm
