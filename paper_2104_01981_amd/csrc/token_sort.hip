// Groups a batch's tokens for the gradient of the lookup: (row, index) pairs in ascending order of the row, and of the index for
// one row.  Padding tokens are left out, a token that is no row marks the batch.
//
// Up to kRankMost tokens: one launch.  A token's place is the number of tokens before it in the order, and each wave counts
// that for eight tokens over all keys in LDS -- n^2 comparisons, which the device does at 10^13 a second: 4.7 us for 600 tokens.
// (A gradient of 8192 tokens takes 23.2 us so, 24.3 with the next.)
// Up to kMergeMost: two launches.  Tiles are sorted in LDS (7.4 us for 64 of them, three digits), then a token's place is what the
// other tiles have below it, by binary search, all tiles going through the LDS of every workgroup (13 us: about 5 for the 700
// steps of a token, 4 for the tiles' way to LDS).  A gradient of 12 000 tokens 25 us, of 2^16 with 256 floats 41.8; with the radix
// sort 33 and 43.5.  (Tiles of 2048: 11 and 11 us instead of 7.4 and 13.)
// More: a radix sort of digits of up to 11 bits, two launches to a digit: counts of each tile, then a stable scatter that ranks
// a tile's items with wave ballots and writes them in runs.  Every workgroup of the scatter adds up the counts of the tiles before
// its own by itself; of more than kDirectTiles tiles they are first added up in groups, by a launch in between.  What bounds it is
// latency.  2^20 items of 22 bits: three digits of 4.9 (counts), 4.9 (groups), 11 us (scatter, of which 1 goes into the counts of the
// other tiles, 1.5 into the ranks, 1 into the sums over the workgroup, 0.5 into the writes).
// (The counts of 257 tiles without groups: a scatter of 21 us instead of 12.)
#include "ecrm_internal.h"

namespace ecrm {

constexpr int kRankThreads = 256;
constexpr uint32_t kRankItems = 8;                       // tokens of a wave
constexpr int kTokenThreads = 512;
constexpr int kTokenWaves = kTokenThreads / kWave;
constexpr int kTokenBits = 11;                           // of a digit, at most
constexpr uint32_t kDirectTiles = 128;
constexpr uint32_t kLargeBatch = 2048u * 1024u;
constexpr uint32_t kMergeTile = 1024, kMergeItems = 256, kMergeThreads = 1024;
constexpr uint32_t kMergeMost = 64u * kMergeTile;        // tokens of a batch that is sorted in tiles, which are then merged
constexpr uint32_t kBadTile = 0x80000000u;

struct TokenPass {
    const uint64_t *keys64;                              // first digit: the caller's
    const uint32_t *keys, *vals;                         // others
    uint32_t *keys_out, *vals_out;
    uint32_t n;
    uint64_t padding;
    uint32_t rows;
    int shift, bits;
    uint32_t tiles, group, groups;                       // group: tiles of one
    uint16_t *table;                                     // [tiles][bins]; grouped: of 32 bits
    uint32_t *sums;                                      // [groups][bins]
    uint32_t *flags;                                     // [tiles] padding tokens, kBadTile
    TokenControl *ctl;
    Header *hdr;
    BesideJob beside;                                    // by the workgroups behind the tiles'
};

// a share of the job for each of `blocks` workgroups
__device__ __forceinline__ void share_of(const BesideJob &job, uint32_t block, uint32_t blocks, uint32_t threads)
{
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    if (job.to) {
        u4 *to = (u4 *)job.to + job.first;
        for (uint64_t i = (uint64_t)block * threads + threadIdx.x; i < job.count; i += (uint64_t)blocks * threads)
            to[i] = u4{0u, 0u, 0u, 0u};
        return;
    }
    constexpr uint32_t U = 8;                            // loads in flight
    const uint32_t lane = lane_id(), count = (uint32_t)job.count, waves = blocks * (threads / kWave);
    for (uint32_t i0 = (block * (threads / kWave) + threadIdx.x / kWave) * (U * kWave); i0 < count; i0 += waves * (U * kWave)) {
        u4 x[U];
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) {
            const uint32_t i = (uint32_t)job.first + min(i0 + q * kWave + lane, count - 1u), r = job.row.div(i);
            x[q] = *(const u4 *)(job.from + r * job.stride + (size_t)(i - r * job.row.d) * 16u);
        }
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) asm volatile("" : : "v"(x[q]));        // to be in the cache is all
    }
}

// inclusive sum over the wave: within rows of 16 lanes, then over the rows
__device__ __forceinline__ uint32_t wave_sums(uint32_t v)
{
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false);       // row_shr:1, 2, 4, 8
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);       // row_bcast:15 to rows 1 and 3
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);       // row_bcast:31 to rows 2 and 3
    return v;
}

__global__ __launch_bounds__(kRankThreads) void token_rank_kernel(TokenPass a)
{
    __shared__ __align__(16) uint32_t s_key[kRankMost];
    __shared__ uint32_t s_pads, s_bad;
    if (blockIdx.x >= a.tiles) {
        share_of(a.beside, blockIdx.x - a.tiles, gridDim.x - a.tiles, kRankThreads);
        return;
    }
    const uint32_t tid = threadIdx.x, lane = lane_id(), wave = tid / kWave, n = a.n;
    if (tid == 0) s_pads = s_bad = 0;
    __syncthreads();
    const uint32_t room = (n + 255u) / 256u * 256u;      // what a wave looks at a time
    uint32_t pads = 0;
    bool bad = false;
#pragma unroll 4
    for (uint32_t i = tid; i < room; i += kRankThreads) {
        const uint64_t key = a.keys64[min(i, n - 1u)];
        const bool pad = i < n && is_padding(key, a.padding);
        bad |= i < n && !pad && key >= (uint64_t)a.rows;
        pads += pad ? 1u : 0u;
        s_key[i] = i < n && !pad ? (uint32_t)key : kNoKey;
    }
    if (blockIdx.x == 0) {
        if (pads) atomicAdd(&s_pads, pads);
        if (bad) s_bad = 1;
    }
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        a.ctl->bad = s_bad;
        a.ctl->valid = n - s_pads;
        a.ctl->joins = 0;
        if (s_bad) atomicOr(&a.hdr->err_sticky, 1u);
    }
    const uint32_t i0 = (blockIdx.x * (kRankThreads / kWave) + wave) * kRankItems;
    if (i0 >= n) return;
    uint32_t key[kRankItems], less[kRankItems];
#pragma unroll
    for (uint32_t q = 0; q < kRankItems; ++q) {
        key[q] = s_key[i0 + q];                          // i0 + q < room
        less[q] = 0;
    }
    // below: every token; of equal ones those before it.  The eight themselves are looked at last.
    for (uint32_t j = lane * 4u; j < room; j += 4u * kWave) {
        const uint4 k = *(const uint4 *)(s_key + j);
        const bool own = j / kRankItems == i0 / kRankItems;
        const uint32_t one = j < i0 ? 1u : 0u;
#pragma unroll
        for (uint32_t q = 0; q < kRankItems; ++q) {
            const uint32_t below = own ? 0u : key[q] + one;
            less[q] += (k.x < below ? 1u : 0u) + (k.y < below ? 1u : 0u) + (k.z < below ? 1u : 0u) + (k.w < below ? 1u : 0u);
        }
    }
    // eight sums over the wave: halves are exchanged, so that lane l ends up with that of token bits(l)
#pragma unroll
    for (uint32_t h = kRankItems / 2u, by = 1; h; h /= 2u, by *= 2u) {
        const bool upper = (lane & by) != 0;
#pragma unroll
        for (uint32_t q = 0; q < h; ++q) {
            const uint32_t keep = upper ? less[q + h] : less[q], give = upper ? less[q] : less[q + h];
            less[q] = keep + (uint32_t)__shfl_xor((int)give, (int)by, kWave);
        }
    }
#pragma unroll
    for (int by = kRankItems; by < kWave; by *= 2) less[0] += (uint32_t)__shfl_xor((int)less[0], by, kWave);
    if (lane >= kRankItems) return;
    const uint32_t mine = ((lane & 1u) << 2) | (lane & 2u) | (lane >> 2), i = i0 + mine, x = s_key[i];
    uint32_t at = less[0];
#pragma unroll
    for (uint32_t q = 0; q < kRankItems; ++q) {
        const uint32_t k = s_key[i0 + q];
        at += k < x || (k == x && q < mine) ? 1u : 0u;
    }
    if (i < n && x != kNoKey) {                          // no padding token
        a.keys_out[at] = x;
        a.vals_out[at] = i;
    }
}

// ---- tiles sorted, then merged -------------------------------------------------------------------------------------------------
// Sorts a tile of kMergeTile tokens by `bits` bits, enough for rows and one value more: what is not a row comes last, as kNoKey.
// Digits of up to 8 bits; a token's place is what the waves have of smaller digits, and the waves before of its own, and its rank
// among the wave's.
__global__ __launch_bounds__(kMergeTile) void token_tile_kernel(TokenPass a)
{
    constexpr uint32_t kWaves = kMergeTile / kWave, kBits = 8, kPer = (kWaves << kBits) / kMergeTile;
    __shared__ uint32_t s_key[kMergeTile], s_val[kMergeTile], s_wave[kWaves], s_pads, s_bad;
    __shared__ __align__(16) uint32_t s_cnt[kWaves << kBits];                      // [digit][wave]
    if (blockIdx.x >= a.tiles) {
        share_of(a.beside, blockIdx.x - a.tiles, gridDim.x - a.tiles, kMergeTile);
        return;
    }
    const uint32_t tid = threadIdx.x, wave = tid / kWave, lane = lane_id(), i = blockIdx.x * kMergeTile + tid;
    const uint64_t word = a.keys64[min(i, a.n - 1u)];
    const bool in = i < a.n, pad = in && is_padding(word, a.padding), bad = in && !pad && word >= (uint64_t)a.rows;
    uint32_t key = in && !pad ? (uint32_t)word : a.rows, val = i;
    if (tid == 0) s_pads = s_bad = 0;
    const int passes = (a.bits + (int)kBits - 1) / (int)kBits;
    int shift = 0;
    for (int p = 0; p < passes; ++p) {
        const int bits = (a.bits - shift + passes - p - 1) / (passes - p);
        const uint32_t digit = (key >> shift) & ((1u << bits) - 1u), counters = kWaves << bits;
        typedef uint32_t Counts __attribute__((ext_vector_type(kPer)));
        Counts *mine = (Counts *)s_cnt + tid;            // kPer counters to a thread
        const bool counting = tid * kPer < counters;
        if (counting) *mine = (Counts)0u;
        unsigned long long peers = ~0ull;                // of the wave's: those with the same digit
        for (int b = 0; b < bits; ++b) {
            const bool bit = (digit >> b) & 1u;
            const unsigned long long bal = __ballot(bit);
            peers &= bit ? bal : ~bal;
        }
        const uint32_t below = (uint32_t)__popcll(peers & ((1ull << lane) - 1ull));
        __syncthreads();
        if (below == 0) s_cnt[digit * kWaves + wave] = (uint32_t)__popcll(peers);
        __syncthreads();
        const Counts c = counting ? *mine : (Counts)0u;
        uint32_t total = 0;
#pragma unroll
        for (uint32_t q = 0; q < kPer; ++q) total += c[q];
        const uint32_t incl = wave_sums(total);
        if (lane == kWave - 1) s_wave[wave] = incl;
        __syncthreads();
        uint32_t before = incl - total;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) before += w < wave ? s_wave[w] : 0u;
        Counts start;
#pragma unroll
        for (uint32_t q = 0; q < kPer; ++q) {
            start[q] = before;
            before += c[q];
        }
        if (counting) *mine = start;
        __syncthreads();
        const uint32_t at = s_cnt[digit * kWaves + wave] + below;
        s_key[at] = key;
        s_val[at] = val;
        __syncthreads();
        key = s_key[tid];
        val = s_val[tid];
        shift += bits;
    }
    if (in) {                                            // the places behind the batch's last token are the last ones here, too
        a.keys_out[i] = key < a.rows ? key : kNoKey;
        a.vals_out[i] = val;
    }
    const unsigned long long pads = __ballot(pad);
    if (lane == 0 && pads) atomicAdd(&s_pads, (uint32_t)__popcll(pads));
    if (bad) s_bad = 1;
    __syncthreads();
    if (tid == 0) {
        a.flags[blockIdx.x] = s_pads | (s_bad ? kBadTile : 0u);
        if (s_bad) atomicOr(&a.hdr->err_sticky, 1u);
        if (blockIdx.x == 0) a.ctl->joins = 0;
    }
}

// tokens of a sorted tile that are below `key`
__device__ __forceinline__ uint32_t below_in_tile(const uint32_t *s_tile, uint32_t key)
{
    uint32_t at = 0;
#pragma unroll
    for (uint32_t step = kMergeTile / 2u; step; step /= 2u) at += s_tile[at + step - 1u] < key ? step : 0u;
    return at + (s_tile[at] < key ? 1u : 0u);
}

// Places the tokens of sorted tiles: a workgroup kMergeItems of them, each by four lanes, which look its key up in a quarter of the
// other tiles.  A token comes behind equal ones of earlier tiles and before those of later ones.
__global__ __launch_bounds__(kMergeThreads) void token_merge_kernel(TokenPass a)
{
    constexpr uint32_t kRound = 16, kParts = kMergeThreads / kMergeItems, kEach = kRound / kParts;
    constexpr uint32_t kQuads = kRound * kMergeTile / 4u / kMergeThreads;               // 16-byte loads of a thread in a round
    __shared__ __align__(16) uint32_t s_key[kRound * kMergeTile];
    __shared__ uint32_t s_sum[kParts][kMergeItems], s_pads, s_bad;
    const uint32_t tid = threadIdx.x, n = a.n, blocks = (n + kMergeItems - 1) / kMergeItems;
    if (blockIdx.x >= blocks) {
        share_of(a.beside, blockIdx.x - blocks, gridDim.x - blocks, kMergeThreads);
        return;
    }
    const uint32_t item = tid % kMergeItems, part = tid / kMergeItems, i = blockIdx.x * kMergeItems + item, own = i / kMergeTile;
    const uint32_t flag = a.flags[min(tid, a.tiles - 1u)];                         // no more tiles than threads
    const uint32_t key = a.keys[min(i, n - 1u)], val = a.vals[min(i, n - 1u)];
    uint4 next[kQuads];
    auto load = [&](uint32_t u0) {
#pragma unroll
        for (uint32_t q = 0; q < kQuads; ++q) {
            const uint32_t at = u0 * kMergeTile + (q * kMergeThreads + tid) * 4u;
            next[q] = *(const uint4 *)(a.keys + min(at, (n - 1u) / 4u * 4u));      // room for a multiple of four
            if (at >= n) next[q].x = kNoKey;
            if (at + 1u >= n) next[q].y = kNoKey;
            if (at + 2u >= n) next[q].z = kNoKey;
            if (at + 3u >= n) next[q].w = kNoKey;
        }
    };
    load(0);
    if (tid == 0) s_pads = s_bad = 0;
    __syncthreads();
    if (tid < a.tiles) {
        if (flag & ~kBadTile) atomicAdd(&s_pads, flag & ~kBadTile);
        if (flag & kBadTile) s_bad = 1;
    }
    uint32_t before = 0;
    for (uint32_t u0 = 0; u0 < a.tiles; u0 += kRound) {
        if (u0) __syncthreads();                         // everybody is done with the round before
#pragma unroll
        for (uint32_t q = 0; q < kQuads; ++q) *(uint4 *)(s_key + (q * kMergeThreads + tid) * 4u) = next[q];
        __syncthreads();
        if (u0 + kRound < a.tiles) load(u0 + kRound);
        uint32_t got[kEach];
#pragma unroll
        for (uint32_t q = 0; q < kEach; ++q) {
            const uint32_t u = u0 + part * kEach + q;
            got[q] = below_in_tile(s_key + (part * kEach + q) * kMergeTile, key + (u < own ? 1u : 0u));
            if (u == own) got[q] = 0;
        }
#pragma unroll
        for (uint32_t q = 0; q < kEach; ++q) before += got[q];
    }
    if (blockIdx.x == 0 && tid == 0) {
        a.ctl->valid = n - s_pads;
        a.ctl->bad = s_bad;
    }
    if (s_bad) return;                                   // such tiles are not sorted
    s_sum[part][item] = before;
    __syncthreads();
    if (part || i >= n || key == kNoKey) return;
    uint32_t at = i - own * kMergeTile;
#pragma unroll
    for (uint32_t p = 0; p < kParts; ++p) at += s_sum[p][item];
    a.keys_out[at] = key;
    a.vals_out[at] = val;
}

// ---- radix sort ------------------------------------------------------------------------------------------------------------------
// Item i's word, or the last one's: loads without a branch, so that a thread's are in flight together.  Behind `valid` the
// buffers of the later digits hold anything.
template <bool FIRST>
__device__ __forceinline__ uint64_t token_word(const TokenPass &a, uint32_t i)
{
    const uint32_t at = min(i, a.n - 1u);
    return FIRST ? a.keys64[at] : (uint64_t)a.keys[at];
}
// Is item i's word one to be sorted?  Its low 32 bits are its row; of a bad one too: the batch is rejected anyway.
template <bool FIRST>
__device__ __forceinline__ bool is_token(const TokenPass &a, uint32_t i, uint32_t n, uint64_t word, bool &pad, bool &bad)
{
    pad = FIRST && i < n && is_padding(word, a.padding);
    bad = FIRST && i < n && !pad && word >= (uint64_t)a.rows;
    return i < n && !pad;
}

template <bool FIRST, int IPT, bool GROUPED>
__global__ __launch_bounds__(kTokenThreads) void token_hist_kernel(TokenPass a)
{
    __shared__ uint32_t s_hist[1 << kTokenBits];
    __shared__ uint32_t s_pads, s_bad;
    const uint32_t tid = threadIdx.x, bins = 1u << a.bits, n = FIRST ? a.n : a.ctl->valid;
    for (uint32_t i = tid; i < bins; i += kTokenThreads) s_hist[i] = 0;
    if (FIRST && tid == 0) s_pads = s_bad = 0;
    __syncthreads();
    const uint32_t tile = tile_of_block(blockIdx.x, a.tiles), tile0 = tile * (uint32_t)(kTokenThreads * IPT);
    uint32_t pads = 0;
    bool any_bad = false;
    uint64_t word[IPT];
#pragma unroll
    for (int r = 0; r < IPT; ++r) word[r] = token_word<FIRST>(a, tile0 + r * kTokenThreads + tid);
#pragma unroll
    for (int r = 0; r < IPT; ++r) {
        bool pad, bad;
        if (is_token<FIRST>(a, tile0 + r * kTokenThreads + tid, n, word[r], pad, bad))
            atomicAdd(&s_hist[((uint32_t)word[r] >> a.shift) & (bins - 1u)], 1u);
        pads += pad ? 1u : 0u;
        any_bad |= bad;
    }
    if (FIRST) {
        if (pads) atomicAdd(&s_pads, pads);
        if (any_bad) s_bad = 1;
    }
    __syncthreads();
    for (uint32_t i = tid; i < bins; i += kTokenThreads) {
        if (GROUPED) ((uint32_t *)a.table)[(size_t)tile * bins + i] = s_hist[i];
        else a.table[(size_t)tile * bins + i] = (uint16_t)s_hist[i];
    }
    if (FIRST && tid == 0) {
        a.flags[tile] = s_pads | (s_bad ? kBadTile : 0u);
        if (s_bad) atomicOr(&a.hdr->err_sticky, 1u);
        if (tile == 0) a.ctl->joins = 0;
    }
}

// Of a group of tiles and a digit value: exclusive sums over the group's tiles in place, and their total.
__global__ __launch_bounds__(256) void token_groups_kernel(TokenPass a)
{
    const uint32_t bins = 1u << a.bits, bin = blockIdx.y * 256u + threadIdx.x, g = blockIdx.x;
    if (bin >= bins) return;
    uint32_t *at = (uint32_t *)a.table + (size_t)g * a.group * bins + bin;
    const uint32_t cnt = min(a.group, a.tiles - g * a.group);
    uint32_t sum = 0;
    constexpr uint32_t U = 32;
    for (uint32_t t0 = 0; t0 < cnt; t0 += U) {
        uint32_t c[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) c[u] = at[(size_t)min(t0 + u, cnt - 1u) * bins];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            if (t0 + u >= cnt) continue;
            at[(size_t)(t0 + u) * bins] = sum;
            sum += c[u];
        }
    }
    a.sums[(size_t)g * bins + bin] = sum;
}

// exclusive sum of v over the workgroup
template <typename N>
__device__ __forceinline__ N sum_before(N v, N *s_wave)
{
    const uint32_t lane = lane_id(), wave = threadIdx.x / kWave;
    N incl = v;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const N t = __shfl_up(incl, d, kWave);
        if (lane >= (uint32_t)d) incl += t;
    }
    if (lane == kWave - 1) s_wave[wave] = incl;
    __syncthreads();
    N before = incl - v;
#pragma unroll
    for (uint32_t w = 0; w < (uint32_t)kTokenWaves; ++w) before += w < wave ? s_wave[w] : (N)0;
    __syncthreads();
    return before;
}

// LDS of a scatter
static size_t scatter_lds(int bits, int ipt)
{
    const size_t bins = (size_t)1 << bits, tile = (size_t)kTokenThreads * ipt;
    return tile * 8 + bins * 8 + kTokenWaves * bins * 2;
}

// PER: digit values of a thread
template <bool FIRST, int IPT, int PER, bool GROUPED>
__global__ __launch_bounds__(kTokenThreads) void token_scatter_kernel(TokenPass a)
{
    constexpr uint32_t kTile = kTokenThreads * IPT;
    extern __shared__ __align__(16) uint32_t lds[];
    __shared__ unsigned long long s_wave[kTokenWaves];
    const uint32_t tid = threadIdx.x, wave = tid / kWave, lane = lane_id();
    const uint32_t bins = 1u << a.bits;
    uint32_t *s_keys = lds, *s_vals = lds + kTile, *s_start = lds + 2 * kTile, *s_base = s_start + bins;
    uint16_t *s_cnt = (uint16_t *)(s_base + bins);       // [waves][bins] counts, then offsets, of a wave
    if (blockIdx.x >= a.tiles) {
        share_of(a.beside, blockIdx.x - a.tiles, gridDim.x - a.tiles, kTokenThreads);
        return;
    }
    const uint32_t n = FIRST ? a.n : a.ctl->valid;
    const uint32_t tile = tile_of_block(blockIdx.x, a.tiles), tile0 = tile * kTile;
    if (FIRST && blockIdx.x == 0) {                      // what the first counting has found
        uint32_t pads = 0, bad = 0;
        for (uint32_t t = tid; t < a.tiles; t += kTokenThreads) {
            pads += a.flags[t] & ~kBadTile;
            bad |= a.flags[t] & kBadTile;
        }
        const unsigned long long own = (unsigned long long)(bad ? 1u : 0u) << 32 | pads, sums = sum_before(own, s_wave) + own;
        if (tid == kTokenThreads - 1) {
            a.ctl->valid = a.n - (uint32_t)sums;
            a.ctl->bad = sums >> 32 ? 1u : 0u;
        }
    }
    uint32_t key[IPT], val[IPT], rank[IPT];
    bool there[IPT];
    {
        uint64_t word[IPT];
        const uint32_t i0 = tile0 + wave * (kWave * IPT) + lane;
#pragma unroll
        for (int r = 0; r < IPT; ++r) {
            word[r] = token_word<FIRST>(a, i0 + r * kWave);
            val[r] = FIRST ? i0 + r * kWave : a.vals[min(i0 + r * kWave, a.n - 1u)];
        }
#pragma unroll
        for (int r = 0; r < IPT; ++r) {
            bool pad, bad;
            there[r] = is_token<FIRST>(a, i0 + r * kWave, n, word[r], pad, bad);
            key[r] = (uint32_t)word[r];
        }
    }
    if (tile0 >= n) return;
    // the thread's digit values: items of them in the tiles before, and in all
    const uint32_t bin = tid * PER;
    uint32_t before[PER] = {}, all[PER] = {};
    if (bin < bins) {
        if (GROUPED) {
            constexpr uint32_t U = 32 / PER;
            typedef uint32_t Counts __attribute__((ext_vector_type(PER)));
            const uint32_t g = tile / a.group;
            const Counts here = *(const Counts *)((const uint32_t *)a.table + (size_t)tile * bins + bin);
            for (uint32_t t0 = 0; t0 < a.groups; t0 += U) {
                Counts c[U];
#pragma unroll
                for (uint32_t u = 0; u < U; ++u) c[u] = *(const Counts *)(a.sums + (size_t)min(t0 + u, a.groups - 1u) * bins + bin);
#pragma unroll
                for (uint32_t u = 0; u < U; ++u)
#pragma unroll
                    for (int q = 0; q < PER; ++q) {
                        all[q] += t0 + u < a.groups ? c[u][q] : 0u;
                        before[q] += t0 + u < g ? c[u][q] : 0u;
                    }
            }
#pragma unroll
            for (int q = 0; q < PER; ++q) before[q] += here[q];
        } else {
            constexpr uint32_t U = 64 / PER;
            typedef uint16_t Counts __attribute__((ext_vector_type(PER)));
            for (uint32_t t0 = 0; t0 < a.tiles; t0 += U) {
                Counts c[U];
#pragma unroll
                for (uint32_t u = 0; u < U; ++u) c[u] = *(const Counts *)(a.table + (size_t)min(t0 + u, a.tiles - 1u) * bins + bin);
#pragma unroll
                for (uint32_t u = 0; u < U; ++u)
#pragma unroll
                    for (int q = 0; q < PER; ++q) {
                        all[q] += t0 + u < a.tiles ? (uint32_t)c[u][q] : 0u;
                        before[q] += t0 + u < tile ? (uint32_t)c[u][q] : 0u;
                    }
            }
        }
    }
    for (uint32_t i = tid; i < kTokenWaves * bins / 2u; i += kTokenThreads) ((uint32_t *)s_cnt)[i] = 0;
    __syncthreads();

    // rank inside the wave, whose items are ordered (r, lane): equal digits are matched with ballots
    uint16_t *cnt = s_cnt + wave * bins;
#pragma unroll
    for (int r = 0; r < IPT; ++r) {
        const uint32_t digit = (key[r] >> a.shift) & (bins - 1u);
        unsigned long long peers = __ballot(there[r]);
        auto match = [&](int b) {
            const bool bit = (digit >> b) & 1u;
            const unsigned long long bal = __ballot(bit);
            peers &= bit ? bal : ~bal;
        };
        if (PER == 1) {
            for (int b = 0; b < a.bits; ++b) match(b);
        } else {                                         // 10 bits, or 11
#pragma unroll
            for (int b = 0; b < (PER == 2 ? 10 : 11); ++b) match(b);
        }
        const uint32_t below = (uint32_t)__popcll(peers & ((1ull << lane) - 1ull));
        const uint32_t old = cnt[digit];
        __builtin_amdgcn_wave_barrier();
        if (there[r] && below == 0) cnt[digit] = (uint16_t)(old + (uint32_t)__popcll(peers));
        __builtin_amdgcn_wave_barrier();
        rank[r] = old + below;
    }
    __syncthreads();

    uint32_t total[PER] = {}, mine = 0, in_all = 0;
    if (bin < bins) {
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            uint32_t t[kTokenWaves];
#pragma unroll
            for (int w = 0; w < kTokenWaves; ++w) t[w] = s_cnt[w * bins + bin + q];
#pragma unroll
            for (int w = 0; w < kTokenWaves; ++w) {
                s_cnt[w * bins + bin + q] = (uint16_t)total[q];
                total[q] += t[w];
            }
            mine += total[q];
            in_all += all[q];
        }
    }
    // both sums at once
    const unsigned long long sums = sum_before((unsigned long long)in_all << 32 | mine, s_wave);
    uint32_t start = (uint32_t)sums, global = (uint32_t)(sums >> 32);
    if (bin < bins) {
#pragma unroll
        for (int q = 0; q < PER; ++q) {
            s_start[bin + q] = start;
            s_base[bin + q] = global + before[q] - start;
            start += total[q];
            global += all[q];
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < IPT; ++r) {
        if (!there[r]) continue;
        const uint32_t digit = (key[r] >> a.shift) & (bins - 1u), at = s_start[digit] + cnt[digit] + rank[r];
        s_keys[at] = key[r];
        s_vals[at] = val[r];
    }
    // items of the tile
    if (tid == kTokenThreads - 1) s_wave[0] = start;
    __syncthreads();
    const uint32_t items = (uint32_t)s_wave[0];
    for (uint32_t i = tid; i < items; i += kTokenThreads) {
        const uint32_t k = s_keys[i], to = s_base[(k >> a.shift) & (bins - 1u)] + i;
        a.keys_out[to] = k;
        a.vals_out[to] = s_vals[i];
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------------
static int items_of(uint32_t n) { return n <= kLargeBatch ? 4 : 8; }     // of a thread (2^20 items with eight: 267 us for 252)
static bool is_grouped(uint32_t tiles) { return tiles > kDirectTiles; }
// Digits: wide ones for few launches; in large batches at most 9 bits, so that what a tile writes of one digit value is some
// tens of bytes on end (2^20 items, two digits of 11 bits: scatters of 43 us instead of 12).
static int token_passes(int key_bits, bool grouped)
{
    const int most = grouped ? 9 : kTokenBits;
    return (key_bits + most - 1) / most;
}
static int digit_of(int bits_left, int passes_left)      // spread evenly, wider ones first; eight values at least
{
    const int bits = (bits_left + passes_left - 1) / passes_left;
    return bits < 3 ? 3 : bits;
}
static uint32_t group_of(uint32_t tiles)                 // tiles of a group: as many groups, about
{
    uint32_t g = 8;
    while ((uint64_t)g * g < tiles) ++g;
    return g;
}
static uint32_t tiles_of(uint32_t n, int ipt) { return (uint32_t)(((uint64_t)n + kTokenThreads * ipt - 1) / (kTokenThreads * ipt)); }

TokenSortLayout token_sort_layout(size_t off, uint32_t max_batch, int key_bits)
{
    TokenSortLayout l;
    auto take = [&](size_t bytes) { const size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
    size_t tiles = 0, table = 0, sums = 0;
    const uint32_t ends[3] = {kDirectTiles * 4u * kTokenThreads, kLargeBatch, 0xFFFFFFFFu};
    if (max_batch > kRankMost) tiles = kMergeMost / kMergeTile;
    for (int c = 0; c < 3 && max_batch > kMergeMost; ++c) {      // the largest batch of each kind
        const uint32_t n = max_batch < ends[c] ? max_batch : ends[c];
        const size_t t = tiles_of(n, items_of(n)), g = group_of((uint32_t)t);
        const bool grouped = is_grouped((uint32_t)t);
        const size_t bins = (size_t)1 << digit_of(key_bits, token_passes(key_bits, grouped));
        if (t > tiles) tiles = t;
        if (t * bins * (grouped ? 4 : 2) > table) table = t * bins * (grouped ? 4 : 2);
        if (grouped && (t + g - 1) / g * bins > sums) sums = (t + g - 1) / g * bins;
    }
    l.off_ctl = take(sizeof(TokenControl));
    l.off_flags = take(tiles * 4);
    l.off_table = take(table);
    l.off_groups = take(sums * 4);
    l.end = off;
    return l;
}

template <bool FIRST, int IPT, bool GROUPED>
static void launch_token_pass(const TokenPass &a, uint32_t helpers, hipStream_t st)
{
    const dim3 hist(a.tiles), scatter(a.tiles + helpers), block(kTokenThreads);
    const size_t lds = scatter_lds(a.bits, IPT);
    hipLaunchKernelGGL((token_hist_kernel<FIRST, IPT, GROUPED>), hist, block, 0, st, a);
    if (GROUPED) hipLaunchKernelGGL(token_groups_kernel, dim3(a.groups, ((1u << a.bits) + 255u) / 256u), dim3(256), 0, st, a);
    if (a.bits <= 9) hipLaunchKernelGGL((token_scatter_kernel<FIRST, IPT, 1, GROUPED>), scatter, block, lds, st, a);
    else if (GROUPED) return;                            // digits are narrower there
    else if (a.bits == 10) hipLaunchKernelGGL((token_scatter_kernel<FIRST, IPT, GROUPED ? 1 : 2, GROUPED>), scatter, block, lds, st, a);
    else hipLaunchKernelGGL((token_scatter_kernel<FIRST, IPT, GROUPED ? 1 : 4, GROUPED>), scatter, block, lds, st, a);
}

template <bool FIRST>
static void launch_token_pass(const TokenPass &a, int ipt, uint32_t helpers, hipStream_t st)
{
    if (ipt == 8) launch_token_pass<FIRST, 8, true>(a, helpers, st);
    else if (is_grouped(a.tiles)) launch_token_pass<FIRST, 4, true>(a, helpers, st);
    else launch_token_pass<FIRST, 4, false>(a, helpers, st);
}

TokenSort launch_token_sort(const Scratch &s, const TokenSortLayout &l, const uint64_t *keys, uint32_t n, uint64_t padding, uint32_t rows,
                            int key_bits, const BesideJob &beside, int cus, hipStream_t st)
{
    char *base = (char *)s.hdr;
    TokenPass a{};
    a.keys64 = keys; a.n = n; a.padding = padding; a.rows = rows; a.hdr = s.hdr;
    a.ctl = (TokenControl *)(base + l.off_ctl);
    a.flags = (uint32_t *)(base + l.off_flags);
    a.table = (uint16_t *)(base + l.off_table);
    a.sums = (uint32_t *)(base + l.off_groups);
    a.beside = beside;
    TokenSort r;
    r.ctl = a.ctl;
    const uint32_t helpers = beside.count ? (uint32_t)cus * 4u : 0u;
    if (n <= kRankMost) {
        const uint32_t each = kRankItems * (kRankThreads / kWave);
        a.tiles = (n + each - 1) / each;
        a.keys_out = s.keys[0]; a.vals_out = s.vals[0];
        hipLaunchKernelGGL(token_rank_kernel, dim3(a.tiles + helpers), dim3(kRankThreads), 0, st, a);
        r.sk = s.keys[0];
        r.si = s.vals[0];
        return r;
    }
    if (n <= kMergeMost) {
        const uint32_t blocks = (n + kMergeItems - 1) / kMergeItems;
        a.tiles = (n + kMergeTile - 1) / kMergeTile;
        a.bits = key_bits;
        while (a.bits < 32 && (1ull << a.bits) <= rows) ++a.bits;
        a.keys_out = s.keys[1]; a.vals_out = s.vals[1];
        a.beside.count = beside.count / 2u;              // half of the job beside either
        hipLaunchKernelGGL(token_tile_kernel, dim3(a.tiles + helpers), dim3(kMergeTile), 0, st, a);
        a.keys = s.keys[1]; a.vals = s.vals[1];
        a.keys_out = s.keys[0]; a.vals_out = s.vals[0];
        a.beside.first = a.beside.count;
        a.beside.count = beside.count - a.beside.first;
        hipLaunchKernelGGL(token_merge_kernel, dim3(blocks + helpers), dim3(kMergeThreads), 0, st, a);
        r.sk = s.keys[0];
        r.si = s.vals[0];
        return r;
    }
    const int ipt = items_of(n);
    a.tiles = tiles_of(n, ipt);
    const int passes = token_passes(key_bits, is_grouped(a.tiles));
    a.group = group_of(a.tiles);
    a.groups = (a.tiles + a.group - 1) / a.group;
    int shift = 0;
    for (int p = 0; p < passes; ++p) {
        const int out = p & 1;
        a.shift = shift;
        a.bits = digit_of(key_bits - shift, passes - p);
        a.keys = s.keys[out ^ 1]; a.vals = s.vals[out ^ 1];
        a.keys_out = s.keys[out]; a.vals_out = s.vals[out];
        a.beside.first = beside.count * p / passes;      // a part of the job beside each digit's scatter
        a.beside.count = beside.count * (p + 1) / passes - a.beside.first;
        if (p == 0) launch_token_pass<true>(a, ipt, helpers, st);
        else launch_token_pass<false>(a, ipt, helpers, st);
        shift += a.bits;
        r.sk = s.keys[out];
        r.si = s.vals[out];
    }
    return r;
}

}  // namespace ecrm
