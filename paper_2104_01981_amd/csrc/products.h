// Matrix products of the feed-forward block on the matrix cores: tiles of BM x BN results, whose operands go from memory to LDS
// without passing through registers, 128 bytes of K (64 elements of 16 bits, 32 of 32) at a time, the next ones on their way while the
// present ones are multiplied.
//
// An operand is a matrix whose rows lie along K ("rows": x, h, the weights in the forward pass) or across it ("columns": the
// weights in the backward pass, both operands of weight gradients).
//   rows:    LDS holds [BM][128 bytes].  A wave's load fills eight rows; within a row its eight 16-byte chunks are exchanged by
//            (row / 2) % 8, so that the 16 rows of a fragment's read lie in different banks.
//   columns: LDS holds [K][BM]; 16-bit fragments are read transposed (ds_read_b64_tr_b16: the 16 lanes that read 4 x 16 elements get
//            a column of four each), their 32-byte chunks exchanged by K % 4 and K / 8 % 2; 32-bit ones are read word by word, 64-byte
//            chunks exchanged by K / 4 % 4.
// The buffer descriptors end with the operand, rows or K: what lies behind comes back as zeros (load_range.h).  Rows along K need two more
// precautions where K ends inside a tile, because the next row follows: lanes whose chunk lies behind K read out of range, and the
// upper half of a chunk that K ends in the middle of (K % 8 == 4, 16 bits) is cleared in LDS.  Both operands, since
// zero times what is not finite is not zero.
//
// The results' 16 x 16 blocks are held transposed (b is the first operand of the instruction): a lane has four consecutive columns of
// a row.  Of 16-bit results two blocks make a pair, the columns dealt out to them by fours, so that a lane has eight: 16 bytes to an access.
//
// What bounds the loop: 256 x 256 tiles, one workgroup of eight waves to a CU, move 64 KB from the caches for 8.4 MFLOP.  16384 x 4096, K =
// 4096, bf16: 415 to 440 us, 1250 to 1320 TFLOP/s; with all rows in one place, so that nothing but L1 is asked, 385 (1430), a
// bf16 product of 8192^3 by the library 1460: the clock under this load is what is left.  LDS is read a fifth of the time, without
// conflicts.  Fragments read ahead of the barrier changed nothing (1 %), K rotated by tile, so that tiles ask unlike channels, cost 10 %.
#pragma once

#include "ffn_plan.h"
#include "load_range.h"
#include "mask.h"

namespace ecrm {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_t;

// What becomes of a product.
enum {
    kGate = 0,      // both projections, the activation and the product: h, and g and u where they are saved
    kOut = 1,       // the block's output: dropout, residual
    kBack = 2,      // gradient of h; dg, du and h again
    kInput = 3,     // gradient of x, added to something
    kWeights = 4    // weight gradients
};

struct Operand {
    const void *p[2];          // kGate: of the gate's and the up projection's weights; kInput: of the first and the second half of K
    uint64_t stride[2];        // elements
};

struct Product {
    Operand a, b;              // a: M rows of the result, b: N columns
    uint32_t M, N, K;          // kInput: K of each half;  kGate: N of each projection
    void *out;
    uint64_t out_stride;
    const void *in;            // kOut: residual;  kInput: what is added;  kBack: saved g and u
    uint64_t in_stride;
    void *out2, *out3;         // kGate: saved g and u (or null);  kBack: du, h
    float scale;               // kBack, kWeights: of the sums (the dropout's factor, which e comes without: that is exact in every type)
    uint32_t kind;             // kInput or kWeights, where they are worked off side by side
    uint32_t tiles_m, tiles_n;
    uint32_t splits, each;     // K tiles: cut into so many parts of at most so many
    uint32_t first;            // workgroup of its first tile's first part
    uint32_t part;             // of several parts: its first tile's first one in ProductArgs::part, in tiles;
    uint32_t counter;          // its first tile's in ProductArgs::arrived
};

struct ProductArgs {
    Product p[4];
    uint32_t products, workgroups;
    float *part;
    uint32_t *arrived;                 // parts of a tile that are there
    uint32_t clear;                    // so many of them are cleared by the first launch of a call, for those behind it
    uint32_t activation;
    uint32_t masked, first_row;        // row of the mask that row 0 of the results has
    MaskArgs mask;
    uint32_t accumulate, wide;         // kWeights: added to; in 32 bits whatever the type
};

template <typename T>
struct Fragment;
template <>
struct Fragment<__bf16> {
    typedef __bf16 type __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 multiply(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(type, a), __builtin_bit_cast(type, b), c, 0, 0, 0);
    }
};
template <>
struct Fragment<_Float16> {
    typedef _Float16 type __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 multiply(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(type, a), __builtin_bit_cast(type, b), c, 0, 0, 0);
    }
};
template <>
struct Fragment<float> {
    static __device__ __forceinline__ f32x4 multiply(u32x4 a, u32x4 b, f32x4 c)
    {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
        return c;
    }
};


// A value that is the same for the wave, in scalar registers: what a division gives lies in vector registers, and a load whose descriptor
// or LDS address does would be made lane by lane.
__device__ __forceinline__ uint32_t scalar(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

__device__ __forceinline__ const char *scalar(const char *p)
{
    return (const char *)((uint64_t)scalar((uint32_t)((uint64_t)p >> 32)) << 32 | scalar((uint32_t)(uint64_t)p));
}

// 64 lanes' 16 bytes each from a buffer (zeros behind its end) to the 1 KB of LDS at `to` + BEHIND.  Written out because the compiler,
// which does not tell the tiles' two halves apart where fragments are read transposed, waits for the load before the next such read
// (kInput with K = 4096: 980 TFLOP/s that way, 1310 so).  It does not count these loads either: before the tile is read there have to be
// a wait for all of them and a barrier.  Nor does it keep the distances that it keeps for a load of its own: M0 is written two instructions
// before its use, and scalar registers that a vector instruction may have written last (readfirstlane) five at least, in the
// first of several loads, which have them in common.
template <uint32_t BEHIND>
__device__ __forceinline__ void load_to_lds(u32x4 buffer, uint32_t at, uint32_t from, uint32_t to)
{
    if (BEHIND == 0)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :: "s"(to), "v"(at), "s"(buffer), "s"(from) : "memory", "m0");
    else
        asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds"
                     :: "s"(to), "i"(BEHIND), "v"(at), "s"(buffer), "s"(from) : "memory", "scc", "m0");
}
// f(Constant<0>()), f(Constant<1>()) .. f(Constant<N - 1>())
template <uint32_t V>
struct Constant { static constexpr uint32_t value = V; };
template <uint32_t N, uint32_t I = 0, typename F>
__device__ __forceinline__ void for_each(F f)
{
    if constexpr (I < N) {
        f(Constant<I>());
        for_each<N, I + 1>(f);
    }
}
__device__ __forceinline__ u32x4 buffer_of(const char *base, uint32_t bytes)
{
    return u32x4{(uint32_t)(uint64_t)base, (uint32_t)((uint64_t)base >> 32), bytes, 0x00020000u};
}

// ---- from memory to LDS ----------------------------------------------------------------------------------------------------------
// Where two blocks of 16 columns lie in pairs, so that a lane's four results of either are eight consecutive ones: the column that row
// r of the operand's tile is.
__device__ __forceinline__ uint32_t column_of(uint32_t r) { return (r & ~31u) | (r >> 2 & 3u) << 3 | (r >> 4 & 1u) << 2 | (r & 3u); }

// The part of a tile of ROWS rows (or columns) that a wave loads.
template <typename T, bool COLUMNS, int ROWS, int WAVES, bool PAIRS>
struct Loader {
    static constexpr uint32_t kLoads = ROWS * kRowBytes / 1024 / WAVES, kElements = kRowBytes / sizeof(T);
    static_assert(kLoads >= 1 && ROWS * kRowBytes % (1024 * WAVES) == 0, "whole loads of a wave");
    uint32_t at[kLoads];
    const char *base;                            // rows: the tile's first row; columns: its first column
    uint32_t stride, end;                        // bytes; rows: the operand's size from base on; columns: of a row
    uint32_t K;

    // `first`: of the operand's rows; `load`: the wave's first load, the rows of the tile's load j are first + (j - row0) * 8
    __device__ __forceinline__ void set(const void *p, uint64_t elements, uint32_t first, uint32_t count, uint32_t k, uint32_t load, uint32_t row0)
    {
        const uint32_t lane = lane_id();
        K = k;
        stride = (uint32_t)(elements * sizeof(T));
        if (!COLUMNS) {
            base = scalar((const char *)p + (uint64_t)first * stride);
            end = scalar(rows_end(count, first, (uint32_t)ROWS, stride, K * (uint32_t)sizeof(T)));
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i) {
                const uint32_t j = load + i, chunk = (lane % 8u) ^ ((lane / 16u) | (j & 1u) << 2);
                const uint32_t row = (j - row0) * 8u + lane / 8u;
                at[i] = (PAIRS ? column_of(row) : row) * stride + chunk * 16u;
            }
        } else {
            constexpr uint32_t kBytes = ROWS * sizeof(T);
            base = scalar((const char *)p + (uint64_t)first * sizeof(T));
            end = scalar((count > first ? count - first : 0u) * (uint32_t)sizeof(T));
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i) {
                const uint32_t byte = (load + i) * 1024u + lane * 16u, row = byte / kBytes, chunk = byte % kBytes / 16u;
                const uint32_t by = sizeof(T) == 2 ? (((row & 3u) | (row >> 3 & 1u) << 2) & (kBytes / 32u - 1u)) << 1 : (row >> 2 & 3u & (kBytes / 64u - 1u)) << 2;
                at[i] = row * stride + (chunk ^ by) * 16u;
            }
        }
    }

    // K from k0 on, into the tile at `tile`
    __device__ __forceinline__ void issue(uint32_t k0, const char *tile, uint32_t load) const
    {
        const uint32_t lane = lane_id(), left = K - k0;  // more than 0
        const uint32_t to = scalar((uint32_t)(uintptr_t)(lds_t *)tile + load * 1024u);
        if (!COLUMNS) {
            const u32x4 buffer = buffer_of(base, end);
            const uint32_t from = scalar(rows_from(end, k0 * (uint32_t)sizeof(T)));
            if (left >= kElements) {
                for_each<kLoads>([&](auto i) { load_to_lds<decltype(i)::value * 1024u>(buffer, at[decltype(i)::value], from, to); });
            } else {
                for_each<kLoads>([&](auto i) {
                    const uint32_t chunk = (lane % 8u) ^ ((lane / 16u) | ((load + decltype(i)::value) & 1u) << 2);
                    const bool outside = chunk * (16u / (uint32_t)sizeof(T)) >= left;
                    load_to_lds<decltype(i)::value * 1024u>(buffer, outside ? kOutside : at[decltype(i)::value], from, to);
                });
            }
        } else {
            const u32x4 buffer = buffer_of(scalar(base + (uint64_t)k0 * stride), scalar(columns_end(min(left, kElements), stride, end)));
            for_each<kLoads>([&](auto i) { load_to_lds<decltype(i)::value * 1024u>(buffer, at[decltype(i)::value], 0u, to); });
        }
    }
};

// K ends in the middle of a 16-byte chunk, `left` 16-bit elements from the tile's begin: what is behind it in the chunk is cleared in all rows.
template <int ROWS, int THREADS>
__device__ __forceinline__ void clear_behind(char *tile, uint32_t left, uint32_t tid)
{
    for (uint32_t r = tid; r < ROWS; r += THREADS)
        *(uint2 *)(tile + r * kRowBytes + (left / 8u ^ (r / 2u) % 8u) * 16u + 8u) = uint2{0u, 0u};
}

// ---- from LDS to registers -------------------------------------------------------------------------------------------------------
// Fragments of the tile's 16-row blocks first .. first + N - 1, of half `s` of its K.
template <typename T, bool COLUMNS, int ROWS, bool PAIRS, int N>
__device__ __forceinline__ void read_fragments(const char *tile, uint32_t first, uint32_t s, u32x4 (&f)[N])
{
    const uint32_t lane = lane_id(), i = lane % 16u, q = lane / 16u;
    if (!COLUMNS) {
        const char *p = tile + (first * 16u + i) * kRowBytes + (((s * 4u + q) ^ (i >> 1)) * 16u);
#pragma unroll
        for (int b = 0; b < N; ++b) f[b] = *(const u32x4 *)(p + b * 16 * (int)kRowBytes);
    } else if (sizeof(T) == 2) {
        typedef short s4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s4 lds4;
        constexpr uint32_t kBytes = ROWS * sizeof(T);
        const uint32_t row = s * 32u + q * 8u + i / 4u, by = ((i / 4u) | (q & 1u) << 2) & (kBytes / 32u - 1u);
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const uint32_t block = first + b;
            const uint32_t chunk = PAIRS ? (block & ~1u) + i % 4u / 2u : block, in = PAIRS ? i % 2u * 16u + (block & 1u) * 8u : i % 4u * 8u;
            const char *p = tile + row * kBytes + (chunk ^ by) * 32u + in;
            const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(p + 4u * kBytes));
            const uint2 x = __builtin_bit_cast(uint2, lo), y = __builtin_bit_cast(uint2, hi);
            f[b] = u32x4{x.x, x.y, y.x, y.y};
        }
    } else {
        constexpr uint32_t kBytes = ROWS * sizeof(T);
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const char *p = tile + (s * 16u + q * 4u) * kBytes + (((first + b) ^ (q & (kBytes / 64u - 1u))) * 64u) + i * 4u;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[b][j] = *(const uint32_t *)(p + j * (int)kBytes);
        }
    }
}

// ---- what becomes of four consecutive results ------------------------------------------------------------------------------------
// In 16-bit types the functions below are off by a few 2^-22 of the larger of 1 and their value, the rounding behind them by 2^-9 or 2^-12.
template <typename T>
__device__ __forceinline__ float logistic(float g)
{
    if (sizeof(T) == 4) return 1.0f / (1.0f + expf(-g));
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));
}
// (1 + erf(g / sqrt 2)) / 2 and e^(-g^2 / 2).  16 bits: M. Abramowitz, I. Stegun, "Handbook of Mathematical Functions", 7.1.26 (1.5e-7).
template <typename T>
__device__ __forceinline__ float normal(float g, float &density)
{
    if (sizeof(T) == 4) {
        density = expf(-0.5f * g * g);
        return 0.5f * erfcf(g * -0.70710678f);
    }
    const float x = fabsf(g) * 0.70710678f, t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * x);
    density = __builtin_amdgcn_exp2f(x * x * -1.44269504f);
    const float poly = t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    const float tail = 0.5f * poly * density;            // of the side g is on
    return g < 0.f ? tail : 1.0f - tail;
}
template <typename T, uint32_t ACT>
__device__ __forceinline__ float activation(float g, float &slope)
{
    if (ACT == ECRM_SILU) {
        const float q = logistic<T>(g);
        slope = q * (1.0f + g * (1.0f - q));
        return g * q;
    }
    if (ACT == ECRM_GELU) {
        float density;
        const float q = normal<T>(g, density);
        slope = q + g * density * 0.39894228f;
        return g * q;
    }
    slope = g > 0.f ? 1.0f : 0.f;
    return g > 0.f ? g : g != g ? g : 0.f;
}

// f(Constant<activation>()): one branch for all that f does
template <typename F>
__device__ __forceinline__ void with_activation(uint32_t kind, F f)
{
    if (kind == ECRM_SILU) f(Constant<ECRM_SILU>());
    else if (kind == ECRM_GELU) f(Constant<ECRM_GELU>());
    else f(Constant<ECRM_RELU>());
}

// 16 bytes of a row: eight consecutive elements of 16 bits, four of 32, in `quads` fours of which there are 1 or 2 (16 bits), or none.
template <typename T>
struct Piece {
    static constexpr int kQuads = 16 / (4 * sizeof(T));
    typedef u32x4 Loose __attribute__((aligned(8)));     // elements are aligned by fours
    static __device__ __forceinline__ u32x4 read(const T *p, uint32_t quads)
    {
        if (quads >= (uint32_t)kQuads) return *(const Loose *)p;
        const uint2 half = quads ? *(const uint2 *)p : uint2{0u, 0u};
        return u32x4{half.x, half.y, 0u, 0u};
    }
    static __device__ __forceinline__ u32x4 read_or_zero(const T *p, uint32_t quads)
    {
        return quads ? read(p, quads) : u32x4{0u, 0u, 0u, 0u};
    }
    static __device__ __forceinline__ void write_past(T *p, uint32_t quads, u32x4 v)
    {
        if (quads >= (uint32_t)kQuads) __builtin_nontemporal_store((Loose)v, (Loose *)p);
        else write(p, quads, v);
    }
    static __device__ __forceinline__ void write(T *p, uint32_t quads, u32x4 v)
    {
        if (quads >= (uint32_t)kQuads) *(Loose *)p = v;
        else if (quads) *(uint2 *)p = uint2{v.x, v.y};
    }
    static __device__ __forceinline__ void widen(u32x4 v, f32x4 (&to)[kQuads])
    {
        if constexpr (sizeof(T) == 4) {
            to[0] = __builtin_bit_cast(f32x4, v);
        } else {
            to[0] = widen4<T>(__builtin_bit_cast(typename Quad<T>::type, uint2{v.x, v.y}));
            to[1] = widen4<T>(__builtin_bit_cast(typename Quad<T>::type, uint2{v.z, v.w}));
        }
    }
    static __device__ __forceinline__ u32x4 round(const f32x4 (&v)[kQuads])
    {
        if constexpr (sizeof(T) == 4) {
            return __builtin_bit_cast(u32x4, v[0]);
        } else {
            const uint2 a = __builtin_bit_cast(uint2, round4<T>(v[0])), b = __builtin_bit_cast(uint2, round4<T>(v[1]));
            return u32x4{a.x, a.y, b.x, b.y};
        }
    }
};

// Lanes l and l ^ 8 exchange: where a is a lane's 16 bytes of its row in one run of 64 bytes (of four lanes 16 apart), b those in the
// next run, then afterwards a is of row l % 8, b of row l % 8 + 8, both in the first run for l % 16 < 8 and in the second for others: eight
// rows of 128 bytes to an access instead of 16 of 64, whole lines.  And back.
__device__ __forceinline__ void exchange(u32x4 &a, u32x4 &b)
{
    const bool upper = threadIdx.x & 8u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t give = upper ? a[i] : b[i];
        const uint32_t got = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)give, 0x128, 0xF, 0xF, true);      // eight lanes on, of 16
        a[i] = upper ? got : a[i];
        b[i] = upper ? b[i] : got;
    }
}

// What a lane reads for a piece of the results, and writes.
enum { kReads = 2, kWrites = 3 };

// W quads of results v (kGate: of the gate, w those of the up projection) with what was read, x and y, to what is written: v, and kGate
// and kBack x and y.
template <typename T, int KIND, int W>
__device__ __forceinline__ void finish(const ProductArgs &a, const Product &p, const MaskKey &mask, uint32_t row, uint32_t col, f32x4 (&v)[W],
                                       const f32x4 (&w)[W], f32x4 (&x)[W], f32x4 (&y)[W])
{
    if (KIND == kGate) {
        with_activation(a.activation, [&](auto act) {
#pragma unroll
            for (int q = 0; q < W; ++q) {
                x[q] = v[q];
                y[q] = w[q];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float slope;
                    v[q][i] = activation<T, decltype(act)::value>(v[q][i], slope) * w[q][i];
                }
            }
        });
    } else if (KIND == kBack) {
        with_activation(a.activation, [&](auto act) {
#pragma unroll
            for (int q = 0; q < W; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[q][i] *= p.scale;
                    float slope;
                    const float value = activation<T, decltype(act)::value>(x[q][i], slope);
                    x[q][i] = v[q][i] * value;
                    v[q][i] *= y[q][i] * slope;
                    y[q][i] *= value;
                }
        });
    } else {
        if (KIND == kOut && a.masked) {
            const uint4 bits = mask_block(mask, a.first_row + row, col / 8u);
            const bool upper = W == 1 && (col & 4u);
            v[0] = drop4(v[0], upper ? uint2{bits.z, bits.w} : uint2{bits.x, bits.y}, mask);
            if (W == 2) v[W - 1] = drop4(v[W - 1], uint2{bits.z, bits.w}, mask);
        }
        if (KIND == kWeights)
#pragma unroll
            for (int q = 0; q < W; ++q) v[q] *= p.scale;
        if (KIND == kWeights ? a.accumulate != 0u : p.in != nullptr)
#pragma unroll
            for (int q = 0; q < W; ++q) v[q] += x[q];
    }
}

// kWeights, results in 32 bits of operands in 16
template <int W>
__device__ __forceinline__ void write_wide(const ProductArgs &a, const Product &p, uint32_t row, uint32_t col, f32x4 (&v)[W])
{
    float *to = (float *)p.out + (uint64_t)row * p.out_stride + col;
#pragma unroll
    for (uint32_t q = 0; q < (uint32_t)W; ++q) {
        if (row >= p.M || col + q * 4u >= p.N) break;
        v[q] *= p.scale;
        if (a.accumulate) v[q] += *(const f32x4 *)(to + q * 4u);
        *(f32x4 *)(to + q * 4u) = v[q];
    }
}

// Where tile t of a product lies: the tiles of eight rows of tiles go column by column, so that those that run at one time share operands.
__device__ __forceinline__ void find_tile(const Product &p, uint32_t t, uint32_t &m, uint32_t &n)
{
    const uint32_t group = 8u * p.tiles_n, g = scalar(t / group), in = t - g * group, rows = min(8u, p.tiles_m - g * 8u);
    n = scalar(in / rows);
    m = scalar(g * 8u + in - n * rows);
}

template <typename T, int KIND, int BM, int BN, int WM, int WN>
struct Tiling {
    static constexpr bool kColumnsA = KIND == kWeights, kColumnsB = KIND == kBack || KIND == kInput || KIND == kWeights;
    static constexpr bool kFirst = KIND == kGate || KIND == kBack;       // of the launches of a call
    static constexpr bool kDual = KIND == kGate;         // half of the columns of a wave are the gate's, half the up projection's
    static constexpr int kWaves = WM * WN, kThreads = kWaves * kWave;
    static constexpr int MB = BM / WM / 16, NB = BN / WN / 16, kNeed = kDual ? NB / 2 : NB;
    static constexpr uint32_t kColumns = kDual ? BN / 2 : BN, kElements = kRowBytes / sizeof(T);
    // 16-bit results: two blocks of 16 columns in a pair, eight consecutive results to a lane.  A unit: the four lanes' 64 bytes of a row.
    static constexpr int kPair = Piece<T>::kQuads, kUnits = kNeed / kPair, kTogether = kUnits % 2 ? 1 : 2, kGroups = kUnits / kTogether;
    static_assert(kNeed % kPair == 0, "whole pairs");

    // Of a lane: row and column of unit u of the wave's rows of blocks i.
    static __device__ __forceinline__ void place(uint32_t m, uint32_t n, uint32_t i, uint32_t u, uint32_t &row, uint32_t &col)
    {
        const uint32_t lane = lane_id(), wave = scalar(threadIdx.x / kWave), wm = wave / WN, wn = wave % WN;
        row = m * BM + (wm * MB + i) * 16u + lane % 16u;
        col = n * kColumns + (wn * kNeed + u * kPair) * 16u + lane / 16u * 4u * kPair;
    }
    // Where the k-th of its pieces of group g lies in memory: as computed, or exchanged.
    static __device__ __forceinline__ void place_line(uint32_t m, uint32_t n, uint32_t i, uint32_t g, uint32_t k, uint32_t &row, uint32_t &col)
    {
        const uint32_t lane = lane_id();
        if (kTogether == 1) return place(m, n, i, g, row, col);
        place(m, n, i, g * 2u + (lane >> 3 & 1u), row, col);
        row = (row & ~15u) + (lane & 7u) + k * 8u;
    }

    // What another call reads is written past the caches, where whole lines are, and leaves them to the operands: g and u of 16384 x 4096, K =
    // 1024, bf16, 282 -> 265 us (with h, which the next launch reads, 273); 8192 x 512, K = 128, in all of a forward pass 18.2 -> 16.9.
    static __device__ __forceinline__ void write_far(T *p, uint32_t quads, u32x4 v)
    {
        if (kTogether == 2) Piece<T>::write_past(p, quads, v);
        else Piece<T>::write(p, quads, v);
    }

    struct In { u32x4 x[kTogether][kReads]; };
    static __device__ __forceinline__ void fetch(const ProductArgs &a, const Product &p, uint32_t m, uint32_t n, uint32_t i, uint32_t g, In &in)
    {
        const bool any = KIND == kBack || ((KIND == kOut || KIND == kInput) && p.in) || (KIND == kWeights && a.accumulate && !a.wide);
        if (!any) return;
#pragma unroll
        for (uint32_t k = 0; k < kTogether; ++k) {
            uint32_t row, col;
            place_line(m, n, i, g, k, row, col);
            const uint32_t quads = row < p.M && col < p.N ? (p.N - col) / 4u : 0u;
            if (KIND == kBack) {
                const T *s = (const T *)p.in + (uint64_t)row * 2u * p.N + col;
                in.x[k][0] = Piece<T>::read(s, quads);
                in.x[k][1] = Piece<T>::read(s + p.N, quads);
            } else if (KIND == kWeights) {
                in.x[k][0] = Piece<T>::read((const T *)p.out + (uint64_t)row * p.out_stride + col, quads);
            } else {
                in.x[k][0] = Piece<T>::read((const T *)p.in + (uint64_t)row * p.in_stride + col, quads);
            }
        }
    }
    // The group's results: of(k, q) and of_up(k, q) are unit k's quad q.
    template <typename F, typename G>
    static __device__ __forceinline__ void finish_group(const ProductArgs &a, const Product &p, const MaskKey &mask, uint32_t m, uint32_t n, uint32_t i,
                                                        uint32_t g, In &in, F of, G of_up)
    {
        constexpr int kIn = KIND == kBack ? 2 : KIND == kGate ? 0 : 1, kOuts = KIND == kBack || KIND == kGate ? 3 : 1;
        u32x4 out[kTogether][kWrites];
        if (kTogether == 2)
#pragma unroll
            for (int r = 0; r < kIn; ++r) exchange(in.x[0][r], in.x[kTogether - 1][r]);
#pragma unroll
        for (uint32_t k = 0; k < kTogether; ++k) {
            uint32_t row, col;
            place(m, n, i, g * kTogether + k, row, col);
            f32x4 v[kPair], w[kPair];
#pragma unroll
            for (int q = 0; q < kPair; ++q) {
                v[q] = of(k, q);
                w[q] = of_up(k, q);
            }
            if (KIND == kWeights && a.wide) {
                write_wide<kPair>(a, p, row, col, v);
                continue;
            }
            f32x4 x[kPair], y[kPair];
            if (kIn >= 1) Piece<T>::widen(in.x[k][0], x);
            if (kIn >= 2) Piece<T>::widen(in.x[k][1], y);
            finish<T, KIND, kPair>(a, p, mask, row, col, v, w, x, y);
            out[k][0] = Piece<T>::round(v);
            if (kOuts == 3) {
                out[k][1] = Piece<T>::round(x);
                out[k][2] = Piece<T>::round(y);
            }
        }
        if (KIND == kWeights && a.wide) return;
        if (kTogether == 2)
#pragma unroll
            for (int r = 0; r < kOuts; ++r) exchange(out[0][r], out[kTogether - 1][r]);
#pragma unroll
        for (uint32_t k = 0; k < kTogether; ++k) {
            uint32_t row, col;
            place_line(m, n, i, g, k, row, col);
            const uint32_t quads = row < p.M && col < p.N ? (p.N - col) / 4u : 0u;
            const uint64_t at = (uint64_t)row * p.out_stride + col;
            Piece<T>::write((T *)p.out + at, quads, out[k][0]);
            if (KIND == kGate && p.out2) {
                T *s = (T *)p.out2 + (uint64_t)row * 2u * p.N + col;
                write_far(s, quads, out[k][1]);
                write_far(s + p.N, quads, out[k][2]);
            } else if (KIND == kBack) {
                Piece<T>::write((T *)p.out2 + at, quads, out[k][1]);
                Piece<T>::write((T *)p.out3 + at, quads, out[k][2]);
            }
        }
    }
};

// Four sums of each of N threads, p this one's first place: the halves of all of them side by side, so that a wave writes whole lines (8191
// rows, D = 128, F = 512, fp16: backward 36.9 us with eight bytes of every sixteen at a time, 34.7 so).
template <uint32_t N>
__device__ __forceinline__ void store_part(double *p, f32x4 v)
{
    const double2 d = __builtin_bit_cast(double2, v);
    shared_store(p, d.x);
    shared_store(p + N, d.y);
}
template <uint32_t N>
__device__ __forceinline__ f32x4 load_part(const double *p)
{
    double2 d;
    d.x = shared_load(p);
    d.y = shared_load(p + N);
    return __builtin_bit_cast(f32x4, d);
}

// One part of K of one tile of product p; `local`: the workgroup's place among those of the product.
template <typename T, int KIND, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void run_tile(const ProductArgs &a, const Product &p, uint32_t local, char *s_a0, char *s_b0, char *s_a1, char *s_b1)
{
    typedef Tiling<T, KIND, BM, BN, WM, WN> L;
    constexpr int MB = L::MB, NB = L::NB, kWaves = L::kWaves;
    const uint32_t tid = threadIdx.x, wave = scalar(tid / kWave), wm = wave / WN, wn = wave % WN;

    // consecutive tiles on one XCD (workgroups go to the eight by turns), the parts of K one after the other
    const uint32_t tiles = p.tiles_m * p.tiles_n, all = tiles * p.splits, per = all / 8u, more = all % 8u, xcd = local % 8u;
    const uint32_t index = xcd * per + min(xcd, more) + local / 8u;
    const uint32_t split = scalar(index / tiles), tile = index - split * tiles;
    uint32_t m, n;
    find_tile(p, tile, m, n);

    const uint32_t K = p.K, half_tiles = (K + L::kElements - 1u) / L::kElements, k_tiles = KIND == kInput ? 2u * half_tiles : half_tiles;
    const uint32_t begin = split * p.each, stop = min(begin + p.each, k_tiles);

    typedef Loader<T, L::kColumnsA, BM, kWaves, false> LoadA;
    typedef Loader<T, L::kColumnsB, BN, kWaves, L::kPair == 2> LoadB;
    LoadA la;
    LoadB lb;
    const uint32_t load_a = wave * LoadA::kLoads, load_b = wave * LoadB::kLoads;
    auto set = [&](uint32_t half) {
        la.set(p.a.p[half], p.a.stride[half], m * BM, p.M, p.K, load_a, 0u);
        lb.set(p.b.p[half], p.b.stride[half], n * BN, p.N, p.K, load_b, 0u);
    };
    if (KIND == kGate) {
        // the tile's columns in the order gate, up, gate, up, NB / 2 blocks of 16 each: a wave loads of one projection alone
        constexpr uint32_t kLoadsEach = NB / 2 * 2;          // loads of eight rows to NB / 2 blocks
        static_assert(kLoadsEach % LoadB::kLoads == 0, "a wave loads of one projection");
        const uint32_t part = load_b / kLoadsEach, up = part & 1u;
        la.set(p.a.p[0], p.a.stride[0], m * BM, p.M, p.K, load_a, 0u);
        const uint32_t first = n * L::kColumns + part / 2u * (NB / 2 * 16u);
        lb.set(p.b.p[up], p.b.stride[up], first, p.N, p.K, load_b, part * kLoadsEach);
        // of the rows from `first` on the projection has so many, and no other wave's
    } else {
        set(KIND == kInput && begin >= half_tiles ? 1u : 0u);
    }
    auto issue = [&](uint32_t t, char *to_a, char *to_b) {
        uint32_t k0 = t * L::kElements;
        if (KIND == kInput) {
            if (t == half_tiles && t != begin) set(1u);
            if (t >= half_tiles) k0 = (t - half_tiles) * L::kElements;
        }
        la.issue(k0, to_a, load_a);
        lb.issue(k0, to_b, load_b);
    };

    f32x4 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto multiply = [&](const char *ta, const char *tb) {
#pragma unroll
        for (uint32_t s = 0; s < 2; ++s) {
            u32x4 fa[MB], fb[NB];
            read_fragments<T, L::kColumnsA, BM, false, MB>(ta, wm * MB, s, fa);
            read_fragments<T, L::kColumnsB, BN, L::kPair == 2, NB>(tb, wn * NB, s, fb);
            // before the other wave's reads (1 to 2 % with a's rows along K, nothing or less with weight gradients)
            if (!L::kColumnsA) __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = Fragment<T>::multiply(fb[j], fa[i], acc[i][j]);
            if (!L::kColumnsA) __builtin_amdgcn_s_setprio(0);
        }
    };
    // tile t is there, all of it
    auto arrive = [&](uint32_t t, char *ta, char *tb) {
        __builtin_amdgcn_s_waitcnt(0);                   // this wave's part of it ...
        __syncthreads();                                 // ... and everybody's; nobody reads the other tile any more
        const uint32_t left = K - (KIND == kInput && t >= half_tiles ? t - half_tiles : t) * L::kElements;
        if (sizeof(T) == 2 && !(L::kColumnsA && L::kColumnsB) && left < L::kElements && left % 8u) {
            if (!L::kColumnsA) clear_behind<BM, L::kThreads>(ta, left, tid);
            if (!L::kColumnsB) clear_behind<BN, L::kThreads>(tb, left, tid);
            __syncthreads();
        }
    };
    auto step = [&](uint32_t t, char *ta, char *tb, char *next_a, char *next_b) {
        arrive(t, ta, tb);
        issue(t + 1u, next_a, next_b);
        multiply(ta, tb);
    };
    if (begin < stop) issue(begin, s_a0, s_b0);
    for (uint32_t t = begin; t + 1u < stop; t += 2u) {
        step(t, s_a0, s_b0, s_a1, s_b1);
        if (t + 2u < stop) step(t + 1u, s_a1, s_b1, s_a0, s_b0);
    }
    // What the first rows' results are finished with is on its way before the last multiplications, and then always that of the next: a
    // store could change it for all the compiler knows, which would wait for one block's after the other (kBack 16384 x 4096, K = 1024:
    // 497 us; one row of blocks ahead 303).
    constexpr uint32_t G = L::kGroups, kAhead = KIND == kBack && MB < 8 ? MB : 1;      // as the registers allow
    typename L::In in[kAhead + 1][G];
    if (begin < stop) {
        const bool first = (stop - begin) % 2u;          // the last tile lies in the first place
        char *ta = first ? s_a0 : s_a1, *tb = first ? s_b0 : s_b1;
        arrive(stop - 1u, ta, tb);
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i)
#pragma unroll
            for (uint32_t g = 0; g < G; ++g) L::fetch(a, p, m, n, i, g, in[i][g]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(ta, tb);
    }

    if (!L::kFirst && p.splits > 1u) {
        const uint64_t size = MB * NB * 2 * L::kThreads; // of a part, in pairs of sums
        double *parts = (double *)a.part + (uint64_t)(p.part + tile * p.splits) * size + tid;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) store_part<L::kThreads>(parts + split * size + (i * NB + j) * 2 * L::kThreads, acc[i][j]);
        // the one that is there last joins them, in order
        published();
        __syncthreads();
        uint32_t *s_last = (uint32_t *)s_a0;
        if (tid == 0) {
            const uint32_t before = __hip_atomic_fetch_add(a.arrived + p.counter + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            *s_last = before + 1u == p.splits;
            if (before + 1u == p.splits) __hip_atomic_store(a.arrived + p.counter + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!scalar(*s_last)) return;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (uint32_t s = 0; s < p.splits; ++s)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] += load_part<L::kThreads>(parts + s * size + (i * NB + j) * 2 * L::kThreads);
    }
    MaskKey mask{};
    if (KIND == kOut && a.masked) mask = mask_key(a.mask);
#pragma unroll
    for (uint32_t i = 0; i < MB; ++i) {
        if (i + kAhead < MB)
#pragma unroll
            for (uint32_t g = 0; g < G; ++g) L::fetch(a, p, m, n, i + kAhead, g, in[(i + kAhead) % (kAhead + 1)][g]);
#pragma unroll
        for (uint32_t g = 0; g < G; ++g)
            L::finish_group(a, p, mask, m, n, i, g, in[i % (kAhead + 1)][g],
                            [&](uint32_t k, int q) { return acc[i][(g * L::kTogether + k) * L::kPair + q]; },
                            [&](uint32_t k, int q) { return acc[i][((g * L::kTogether + k) * L::kPair + q + L::kNeed) % NB]; });
    }
}

template <typename T, int KIND, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * kWave, 2) void product_kernel(ProductArgs a)
{
    __shared__ __align__(1024) char s_a0[BM * kRowBytes], s_b0[BN * kRowBytes], s_a1[BM * kRowBytes], s_b1[BN * kRowBytes];
    if (Tiling<T, KIND, BM, BN, WM, WN>::kFirst && blockIdx.x == 0)
        for (uint32_t c = threadIdx.x; c < a.clear; c += blockDim.x) a.arrived[c] = 0u;
    run_tile<T, KIND, BM, BN, WM, WN>(a, a.p[0], blockIdx.x, s_a0, s_b0, s_a1, s_b1);
}

// The gradients of x and of the weights side by side: products that do not wait for each other, the tiles that take longest first.
template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * kWave, 2) void gradients_kernel(ProductArgs a)
{
    __shared__ __align__(1024) char s_a0[BM * kRowBytes], s_b0[BN * kRowBytes], s_a1[BM * kRowBytes], s_b1[BN * kRowBytes];
    uint32_t which = 0;
#pragma unroll
    for (uint32_t i = 1; i < 4; ++i) which = i < a.products && blockIdx.x >= a.p[i].first ? i : which;
    const Product &p = a.p[which];
    if (p.kind == kInput) run_tile<T, kInput, BM, BN, WM, WN>(a, p, blockIdx.x - p.first, s_a0, s_b0, s_a1, s_b1);
    else run_tile<T, kWeights, BM, BN, WM, WN>(a, p, blockIdx.x - p.first, s_a0, s_b0, s_a1, s_b1);
}

// ---- few rows --------------------------------------------------------------------------------------------------------------------
// Up to 16 * XB rows: what counts is that all of the weights are on their way at once.  A workgroup has 16 columns of the results (of
// both projections) and all of K or, where there are few columns and a long K, a part of it; its waves share that, every one with up to
// kAtOnce steps of 64 bytes of 16 rows of weights in flight, straight into the registers of the matrix instructions, whose second operand
// are the rows.  The waves' sums are added up in LDS, in order; those of several workgroups by the one that is there last, in order, too.
template <int XB>
struct Skinny { static constexpr uint32_t kWaves = XB == 1 ? 16 : 8; };          // as the registers allow

template <typename T, int KIND, int XB>
__global__ __launch_bounds__(Skinny<XB>::kWaves * kWave) void skinny_kernel(ProductArgs a)
{
    constexpr int B = KIND == kGate ? 2 : 1;             // matrices of weights
    constexpr uint32_t kChunk = 16 / sizeof(T), kStep = 4 * kChunk;
    __shared__ f32x4 s_part[Skinny<XB>::kWaves][B * XB][kWave];
    const Product &p = a.p[0];
    const uint32_t lane = lane_id(), i = lane % 16u, q = lane / 16u, wave = scalar(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const uint32_t col0 = blockIdx.x * 16u, K = p.K, steps = (K + kStep - 1u) / kStep, sharing = waves * gridDim.y;
    const uint32_t each = scalar((steps + sharing - 1u) / sharing), begin = (blockIdx.y * waves + wave) * each, stop = min(begin + each, steps);
    if (KIND == kGate && blockIdx.x == 0 && blockIdx.y == 0)             // for the launch behind, kOut's
        for (uint32_t c = threadIdx.x; c < a.clear; c += blockDim.x) a.arrived[c] = 0u;

    const T *w[B], *x[XB];
#pragma unroll
    for (int b = 0; b < B; ++b) w[b] = (const T *)p.b.p[b] + (uint64_t)min(col0 + i, p.N - 1u) * p.b.stride[b] + q * kChunk;
#pragma unroll
    for (int r = 0; r < XB; ++r) x[r] = (const T *)p.a.p[0] + (uint64_t)min((uint32_t)r * 16u + i, p.M - 1u) * p.a.stride[0] + q * kChunk;

    f32x4 acc[B][XB];
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
        for (int r = 0; r < XB; ++r) acc[b][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (uint32_t s0 = begin; s0 < stop; s0 += kAtOnce) {
        u32x4 fw[kAtOnce][B], fx[kAtOnce][XB];
        if (s0 + kAtOnce <= stop && (s0 + kAtOnce) * kStep <= K) {
#pragma unroll
            for (uint32_t s = 0; s < kAtOnce; ++s) {
#pragma unroll
                for (int b = 0; b < B; ++b) fw[s][b] = Piece<T>::read(w[b] + (s0 + s) * kStep, 2u);
#pragma unroll
                for (int r = 0; r < XB; ++r) fx[s][r] = Piece<T>::read(x[r] + (s0 + s) * kStep, 2u);
            }
        } else {
#pragma unroll
            for (uint32_t s = 0; s < kAtOnce; ++s) {     // what is behind K, or the wave's part of it, is zero on both sides
                const uint32_t k = (s0 + s) * kStep + q * kChunk, quads = s0 + s < stop && k < K ? (K - k) / 4u : 0u;
#pragma unroll
                for (int b = 0; b < B; ++b) fw[s][b] = Piece<T>::read_or_zero(w[b] + (s0 + s) * kStep, quads);
#pragma unroll
                for (int r = 0; r < XB; ++r) fx[s][r] = Piece<T>::read_or_zero(x[r] + (s0 + s) * kStep, quads);
            }
        }
#pragma unroll
        for (uint32_t s = 0; s < kAtOnce; ++s)
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int r = 0; r < XB; ++r) acc[b][r] = Fragment<T>::multiply(fw[s][b], fx[s][r], acc[b][r]);
    }
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
        for (int r = 0; r < XB; ++r) s_part[wave][b * XB + r][lane] = acc[b][r];
    __syncthreads();

    // wave r finishes rows 16 r .. 16 r + 15 (where there are as few waves as rows of blocks, one may have several)
    for (uint32_t r = wave; r < (uint32_t)XB; r += waves) {
        const uint32_t row = r * 16u + i, col = col0 + q * 4u;
        const bool there = row < p.M && col < p.N;
        f32x4 v[1], up[1], in[1], y[1];
        v[0] = up[0] = in[0] = y[0] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (KIND == kOut && p.in && there) in[0] = widen4<T>(*(const typename Quad<T>::type *)((const T *)p.in + (uint64_t)row * p.in_stride + col));
        for (uint32_t s = 0; s < waves; ++s) {
            v[0] += s_part[s][r][lane];
            if (KIND == kGate) up[0] += s_part[s][(B - 1) * XB + r][lane];
        }
        if (KIND == kOut && gridDim.y > 1u) {
            const uint32_t slot = blockIdx.x * XB + r;
            double *parts = (double *)a.part + (uint64_t)slot * gridDim.y * 2u * kWave + lane;
            store_part<kWave>(parts + blockIdx.y * 2u * kWave, v[0]);
            published();
            uint32_t before = 0;
            if (lane == 0) before = __hip_atomic_fetch_add(a.arrived + slot, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (scalar(before) + 1u < gridDim.y) continue;
            v[0] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (uint32_t s = 0; s < gridDim.y; ++s) v[0] += load_part<kWave>(parts + s * 2u * kWave);
        }
        MaskKey mask{};
        if (KIND == kOut && a.masked) mask = mask_key(a.mask);
        finish<T, KIND, 1>(a, p, mask, row, col, v, up, in, y);
        if (!there) continue;
        typedef typename Quad<T>::type Four;
        *(Four *)((T *)p.out + (uint64_t)row * p.out_stride + col) = round4<T>(v[0]);
        if (KIND == kGate && p.out2) {
            T *s = (T *)p.out2 + (uint64_t)row * 2u * p.N + col;
            *(Four *)s = round4<T>(in[0]);
            *(Four *)(s + p.N) = round4<T>(y[0]);
        }
    }
}

}  // namespace ecrm
