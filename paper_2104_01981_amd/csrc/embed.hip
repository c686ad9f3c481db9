// Lookup of tokens: out[i] = scale * entry keys[i], rounded to the type of the activations, a row of zeros for the padding
// token, and an entry of a server that is down decoded from its stripe (Sec. 3.2) on the way.
//
// What bounds it: memory -- D floats read and D elements written for each token.  A lane moves 16 bytes of whatever row they
// belong to, so that rows of any width use all lanes, and keeps several of them in flight; what is written is read by somebody
// else later.  2^20 tokens of 128 floats to bf16, out of 2^22 rows: 157 us, 4.8 TB/s, what a copy reaches (163 with the stores
// kept in the caches; 162 with loads past them, too), with dropout 153; 2^16 to fp32 while a server is down 16 us.  With dropout
// (mask.h) batches that the caches hold are bound by drawing the masks: 2^16 tokens to bf16 8.8 us instead of 6.1.
#include "mask.h"

namespace ecrm {

constexpr int kEmbedThreads = 256;
constexpr int kEmbedWaves = kEmbedThreads / kWave;
constexpr uint64_t kEmbedSlice = 1ull << 30;         // tokens of a launch, at most

struct EmbedArgs {
    const float *E, *PE;
    const uint64_t *keys;
    uint64_t n, padding;
    uint32_t per;            // consecutive tokens of a wave, at most 64
    uint32_t lost;           // server whose entries are decoded, or none
    float scale;
    void *out;
    uint64_t stride;
    Header *hdr;
    Geometry geo;
    Divider d4;              // by D / 4
    MaskArgs mask;           // with dropout
    uint32_t first;          // row of the first token in the mask
};

// The tokens of a wave that are handled alike, row and place in the wave's range: how many there are.
__device__ __forceinline__ uint32_t gather_tokens(bool mine, uint32_t x, uint2 *list)
{
    const uint32_t lane = lane_id();
    const unsigned long long m = __ballot(mine);
    if (mine) list[__popcll(m & ((1ull << lane) - 1ull))] = uint2{x, lane};
    __builtin_amdgcn_wave_barrier();
    return (uint32_t)__popcll(m);
}

// Four floats of a lost entry: its parity minus the other members by increasing member, rounded as the decoder stores it.
__device__ __forceinline__ f32x4 decode4(const EmbedArgs &a, uint32_t x, uint32_t c)
{
    constexpr uint32_t U = 4;                            // members in flight
    const uint32_t D = a.geo.D, k = a.geo.k, g = a.geo.dk.div(x), j = x - g * k;
    const f32x4 p = *(const f32x4 *)(a.PE + (size_t)g * D + c);
    double v[4] = {(double)p.x, (double)p.y, (double)p.z, (double)p.w};
    for (uint32_t m0 = 0; m0 + 1u < k; m0 += U) {        // the survivors: member m, or m + 1 from the lost one on
        f32x4 o[U];
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) {
            const uint32_t m = min(m0 + q, k - 2u);
            o[q] = *(const f32x4 *)(a.E + ((size_t)g * k + (m < j ? m : m + 1u)) * D + c);
        }
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) {
            if (m0 + q >= k - 1u) continue;
            v[0] -= (double)o[q].x;
            v[1] -= (double)o[q].y;
            v[2] -= (double)o[q].z;
            v[3] -= (double)o[q].w;
        }
    }
    return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}

template <typename T, bool DROP>
__global__ __launch_bounds__(kEmbedThreads) void embed_kernel(EmbedArgs a)
{
    typedef typename Quad<T>::type Four;
    __shared__ uint2 s_list[kEmbedWaves][kWave];
    const uint32_t lane = lane_id(), wave = threadIdx.x / kWave, D = a.geo.D;
    uint2 *list = s_list[wave];
    const uint64_t first = ((uint64_t)blockIdx.x * kEmbedWaves + wave) * a.per;
    if (first >= a.n) return;
    const uint32_t cnt = (uint32_t)(a.n - first < a.per ? a.n - first : a.per);
    const bool in = lane < cnt;
    const uint64_t key = in ? a.keys[first + lane] : 0ull;
    const bool pad = in && is_padding(key, a.padding), bad = in && !pad && key >= (uint64_t)a.geo.rows;
    if (bad) atomicOr(&a.hdr->err_sticky, 1u);
    const uint32_t x = pad ? kNoKey : (uint32_t)key;
    bool lost = false;
    if (a.lost != ECRM_NO_SERVER && in && !pad && !bad) {
        const uint32_t g = a.geo.dk.div(x), j = x - g * a.geo.k;
        lost = a.geo.dS.mod(g + 1u + j) == a.lost;
    }
    T *out = (T *)a.out + first * a.stride;
    MaskKey mask{};
    if (DROP) mask = mask_key(a.mask);
    const uint32_t row0 = a.first + (uint32_t)first;     // with dropout there are at most 2^32

    // the product is formed in 32 bits, then rounded to the type: half a step of the type and 2^-24 in all
    const uint32_t plain = gather_tokens(in && !bad && !lost, x, list), total = plain * a.d4.d;
    constexpr uint32_t U = 4;                            // (2, 4, 8: 162, 163, 162 us of 2^20 tokens, 5.7, 5.8, 8.4 of 20011)
    for (uint32_t u0 = 0; u0 < total; u0 += U * kWave) {
        f32x4 e[U];
        size_t to[U];
        uint32_t row[U], col[U];
        uint2 bits[U] = {};
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) {
            const uint32_t u = min(u0 + q * kWave + lane, total - 1u), r = a.d4.div(u), c = (u - r * a.d4.d) * 4u;
            const uint2 what = list[r];
            to[q] = what.y * a.stride + c;
            row[q] = row0 + what.y;
            col[q] = c;
            e[q] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (what.x != kNoKey) e[q] = *(const f32x4 *)(a.E + (size_t)what.x * D + c) * a.scale;
        }
        if (DROP) {                                      // lanes 2i and 2i + 1 have quads 2j and 2j + 1 if a row has an even number
            mask_quads<U, true>(mask, row, col, a.d4.d % 2u == 0, bits, (total - u0 + kWave - 1u) / kWave);
#pragma unroll
            for (uint32_t q = 0; q < U; ++q) e[q] = drop4(e[q], bits[q], mask);
        }
#pragma unroll
        for (uint32_t q = 0; q < U; ++q)
            if (u0 + q * kWave + lane < total) __builtin_nontemporal_store(round4<T>(e[q]), (Four *)(out + to[q]));
    }
    if (a.lost == ECRM_NO_SERVER) return;
    __builtin_amdgcn_wave_barrier();
    const uint32_t decoded = gather_tokens(lost, x, list) * a.d4.d;
    for (uint32_t u = lane; u < decoded; u += kWave) {
        const uint32_t r = a.d4.div(u), c = (u - r * a.d4.d) * 4u;
        const uint2 what = list[r];
        f32x4 e = decode4(a, what.x, c) * a.scale;
        if (DROP) e = drop4(e, mask_quad(mask, row0 + what.y, c), mask);
        __builtin_nontemporal_store(round4<T>(e), (Four *)(out + what.y * a.stride + c));
    }
}

void launch_embed(const Scratch &s, const Geometry &g, const float *E, const float *PE, const uint64_t *keys, uint64_t n,
                  uint64_t padding, float scale, uint32_t lost, const MaskArgs *mask, void *out, uint32_t type, uint64_t stride,
                  int cus, hipStream_t st)
{
    EmbedArgs a{};
    a.E = E; a.PE = PE; a.hdr = s.hdr; a.geo = g; a.lost = lost; a.scale = scale; a.padding = padding; a.stride = stride;
    a.d4 = make_divider(g.D / 4u);
    if (mask) a.mask = *mask;
    for (uint64_t at = 0; at < n; at += kEmbedSlice) {
        a.n = n - at < kEmbedSlice ? n - at : kEmbedSlice;
        a.keys = keys + at;
        a.first = (uint32_t)at;
        a.out = (char *)out + at * stride * type_bytes(type);
        const uint64_t waves = (uint64_t)cus * 32u;              // as many as are resident
        a.per = (uint32_t)((a.n + waves - 1) / waves);
        // with dropout a wave has two places' quads for every lane, which share what is drawn (8192 tokens of 128 floats in bf16: 3.4 us, with
        // one 3.9, with a token to each wave 5.7, without dropout 4.2; 600 3.0, 3.0, 3.1, 2.7)
        if (mask && a.per < 2u * kWave / a.d4.d) a.per = 2u * kWave / a.d4.d;
        if (a.per > (uint32_t)kWave) a.per = kWave;
        const uint64_t per_block = (uint64_t)a.per * kEmbedWaves;
        const dim3 grid((uint32_t)((a.n + per_block - 1) / per_block)), block(kEmbedThreads);
        with_type(type, [&](auto t) {
            if (mask) hipLaunchKernelGGL((embed_kernel<decltype(t), true>), grid, block, 0, st, a);
            else hipLaunchKernelGGL((embed_kernel<decltype(t), false>), grid, block, 0, st, a);
        });
    }
}

}  // namespace ecrm
