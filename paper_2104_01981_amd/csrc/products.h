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
// The buffer descriptors end with the operand, rows or K: what lies behind comes back as zeros.  Rows along K need two more
// precautions where K ends inside a tile, because the next row follows: lanes whose chunk lies behind K read out of range, and the
// upper half of a chunk that K ends in the middle of (K % 8 == 4, 16 bits) is cleared in LDS.  Both operands, since
// zero times what is not finite is not zero.
//
// The results' 16 x 16 blocks are held transposed (weights are the first operand of the instruction): a lane has four consecutive
// columns of a row.
#pragma once

#include "mask.h"

namespace ecrm {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;
typedef __attribute__((address_space(3))) char lds_t;

// What becomes of a product.
enum {
    kGate = 0,      // both projections, the activation and the product: h, and g and u where they are saved
    kOut = 1,       // the block's output: dropout, residual
    kBack = 2,      // gradient of h; dg, du and h again
    kInput = 3,     // gradient of x, added to something
    kWeights = 4,   // weight gradients
    kKinds = 5
};

struct Operand {
    const void *p[2];          // kGate: of the gate's and the up projection's weights; kInput: of the first and the second half of K
    uint64_t stride[2];        // elements
};

struct Product {
    Operand a, b;              // a: M rows of the result, b: N columns
    uint32_t M, N, K;          // kInput: K of each half;  kGate: N of each projection
    uint32_t tiles_m, tiles_n;
    void *out;
    uint64_t out_stride;
    const void *in;            // kOut: residual;  kInput: what is added;  kBack: saved g and u
    uint64_t in_stride;
    void *out2, *out3;         // kGate: saved g and u (or null);  kBack: du, h
};

struct ProductArgs {
    Product p[3];
    uint32_t products, first[3];       // tile of each product's first
    uint32_t tiles;                    // in all
    uint32_t splits, each;             // K tiles: cut into so many parts of at most so many
    float *part;                       // [tiles][splits][threads][..] where there are several
    uint32_t activation;
    uint32_t masked;
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

constexpr uint32_t kRowBytes = 128;              // of K, in a tile
constexpr uint32_t kOutside = 0x7FFFFFFFu;       // an offset behind any operand's end

// ---- from memory to LDS ----------------------------------------------------------------------------------------------------------
// The part of a tile of ROWS rows (or columns) that a wave loads.
template <typename T, bool COLUMNS, int ROWS, int WAVES>
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
            base = (const char *)p + (uint64_t)first * stride;
            const uint32_t rows = count > first ? min(count - first, (uint32_t)ROWS) : 0u;
            end = rows ? (rows - 1u) * stride + K * (uint32_t)sizeof(T) : 0u;
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i) {
                const uint32_t j = load + i, chunk = (lane % 8u) ^ ((lane / 16u) | (j & 1u) << 2);
                at[i] = ((j - row0) * 8u + lane / 8u) * stride + chunk * 16u;
            }
        } else {
            constexpr uint32_t kBytes = ROWS * sizeof(T);
            base = (const char *)p + (uint64_t)first * sizeof(T);
            end = (count > first ? count - first : 0u) * (uint32_t)sizeof(T);
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i) {
                const uint32_t byte = (load + i) * 1024u + lane * 16u, row = byte / kBytes, chunk = byte % kBytes / 16u;
                const uint32_t by = sizeof(T) == 2 ? (((row & 3u) | (row >> 3 & 1u) << 2) & (kBytes / 32u - 1u)) << 1 : (row >> 2 & 3u) << 2;
                at[i] = row * stride + (chunk ^ by) * 16u;
            }
        }
    }

    // K from k0 on, into the tile at `to`
    __device__ __forceinline__ void issue(uint32_t k0, char *to, uint32_t load) const
    {
        const uint32_t lane = lane_id();
        const uint32_t left = K - k0;            // more than 0
        if (!COLUMNS) {
            const rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)end, 0x00020000);
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i) {
                uint32_t from = at[i];
                if (left < kElements) {
                    const uint32_t chunk = (lane % 8u) ^ ((lane / 16u) | ((load + i) & 1u) << 2);
                    if (chunk * (16u / (uint32_t)sizeof(T)) >= left) from = kOutside;
                }
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_t *)(to + (load + i) * 1024u), 16, (int)from,
                                                         (int)(k0 * (uint32_t)sizeof(T)), 0, 0);
            }
        } else {
            const uint32_t rows = min(left, kElements), bytes = end ? (rows - 1u) * stride + end : 0u;
            const rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)(base + (uint64_t)k0 * stride), 0, (int)bytes, 0x00020000);
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_t *)(to + (load + i) * 1024u), 16, (int)at[i], 0, 0, 0);
        }
    }
};

// K ends in the middle of a chunk of 16 bits a element, `left` elements from the tile's begin: what is behind is cleared in all rows.
template <int ROWS, int THREADS>
__device__ __forceinline__ void clear_behind(char *tile, uint32_t left, uint32_t tid)
{
    for (uint32_t r = tid; r < ROWS; r += THREADS)
        *(uint2 *)(tile + r * kRowBytes + (left / 8u ^ (r / 2u) % 8u) * 16u + 8u) = uint2{0u, 0u};
}

// ---- from LDS to registers -------------------------------------------------------------------------------------------------------
// Fragments of the tile's 16-row blocks first .. first + N - 1, of half `s` of its K.
template <typename T, bool COLUMNS, int ROWS, int N>
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
            const char *p = tile + row * kBytes + (((first + b) ^ by) * 32u) + (i % 4u) * 8u;
            const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(p + 4u * kBytes));
            const uint2 x = __builtin_bit_cast(uint2, lo), y = __builtin_bit_cast(uint2, hi);
            f[b] = u32x4{x.x, x.y, y.x, y.y};
        }
    } else {
        constexpr uint32_t kBytes = ROWS * sizeof(T);
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const char *p = tile + (s * 16u + q * 4u) * kBytes + (((first + b) ^ q) * 64u) + i * 4u;
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
template <typename T>
__device__ __forceinline__ float activation(uint32_t kind, float g, float &slope)
{
    if (kind == ECRM_SILU) {
        const float q = logistic<T>(g);
        slope = q * (1.0f + g * (1.0f - q));
        return g * q;
    }
    if (kind == ECRM_GELU) {
        float density;
        const float q = normal<T>(g, density);
        slope = q + g * density * 0.39894228f;
        return g * q;
    }
    slope = g > 0.f ? 1.0f : 0.f;
    return g > 0.f ? g : g != g ? g : 0.f;
}

// v: results (row, col .. col + 3); kGate: of the gate, w those of the up projection
template <typename T, int KIND>
__device__ __forceinline__ void finish(const ProductArgs &a, const Product &p, const MaskKey &mask, uint32_t row, uint32_t col, f32x4 v, f32x4 w)
{
    typedef typename Quad<T>::type Four;
    if (row >= p.M || col >= p.N) return;
    if (KIND == kGate) {
        if (p.out2) {
            T *s = (T *)p.out2 + (uint64_t)row * 2u * p.N + col;
            *(Four *)s = round4<T>(v);
            *(Four *)(s + p.N) = round4<T>(w);
        }
        f32x4 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float slope;
            h[i] = activation<T>(a.activation, v[i], slope) * w[i];
        }
        *(Four *)((T *)p.out + (uint64_t)row * p.out_stride + col) = round4<T>(h);
    } else if (KIND == kOut) {
        if (a.masked) v = drop4(v, mask_quad(mask, row, col), mask);
        if (p.in) v += widen4<T>(*(const Four *)((const T *)p.in + (uint64_t)row * p.in_stride + col));
        *(Four *)((T *)p.out + (uint64_t)row * p.out_stride + col) = round4<T>(v);
    } else if (KIND == kBack) {
        const T *s = (const T *)p.in + (uint64_t)row * 2u * p.N + col;
        const f32x4 g = widen4<T>(*(const Four *)s), u = widen4<T>(*(const Four *)(s + p.N));
        f32x4 dg, du, h;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float slope;
            const float x = activation<T>(a.activation, g[i], slope);
            dg[i] = v[i] * u[i] * slope;
            du[i] = v[i] * x;
            h[i] = x * u[i];
        }
        const uint64_t to = (uint64_t)row * p.out_stride + col;
        *(Four *)((T *)p.out + to) = round4<T>(dg);
        *(Four *)((T *)p.out2 + to) = round4<T>(du);
        *(Four *)((T *)p.out3 + to) = round4<T>(h);
    } else if (KIND == kInput) {
        if (p.in) v += widen4<T>(*(const Four *)((const T *)p.in + (uint64_t)row * p.in_stride + col));
        *(Four *)((T *)p.out + (uint64_t)row * p.out_stride + col) = round4<T>(v);
    } else {
        const uint64_t at = (uint64_t)row * p.out_stride + col;
        if (a.wide) {
            f32x4 *to = (f32x4 *)((float *)p.out + at);
            if (a.accumulate) v += *to;
            *to = v;
        } else {
            Four *to = (Four *)((T *)p.out + at);
            if (a.accumulate) v += widen4<T>(*to);
            *to = round4<T>(v);
        }
    }
}

// Which product and tile: the tiles of eight rows of tiles go column by column, so that those that run at one time share operands.
__device__ __forceinline__ uint32_t find_tile(const ProductArgs &a, uint32_t tile, uint32_t &m, uint32_t &n)
{
    uint32_t which = 0;
    if (a.products > 1 && tile >= a.first[1]) which = 1;
    if (a.products > 2 && tile >= a.first[2]) which = 2;
    const Product &p = a.p[which];
    const uint32_t t = tile - a.first[which], group = 8u * p.tiles_n, g = t / group, in = t - g * group;
    const uint32_t rows = min(8u, p.tiles_m - g * 8u);
    n = in / rows;
    m = g * 8u + in - n * rows;
    return which;
}

template <typename T, int KIND, int BM, int BN, int WM, int WN>
struct Tiling {
    static constexpr bool kColumnsA = KIND == kWeights, kColumnsB = KIND == kBack || KIND == kInput || KIND == kWeights;
    static constexpr bool kDual = KIND == kGate;         // half of the columns of a wave are the gate's, half the up projection's
    static constexpr int kWaves = WM * WN, kThreads = kWaves * kWave;
    static constexpr int MB = BM / WM / 16, NB = BN / WN / 16, kNeed = kDual ? NB / 2 : NB;
    static constexpr uint32_t kColumns = kDual ? BN / 2 : BN, kElements = kRowBytes / sizeof(T);
    static __device__ __forceinline__ void place(uint32_t m, uint32_t n, uint32_t tid, int mb, int nb, uint32_t &row, uint32_t &col)
    {
        const uint32_t lane = tid % kWave, wave = tid / kWave, wm = wave / WN, wn = wave % WN;
        row = m * BM + (wm * MB + mb) * 16u + lane % 16u;
        col = n * kColumns + (wn * kNeed + nb) * 16u + lane / 16u * 4u;
    }
};

template <typename T, int KIND, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * kWave) void product_kernel(ProductArgs a)
{
    typedef Tiling<T, KIND, BM, BN, WM, WN> L;
    constexpr int MB = L::MB, NB = L::NB, kWaves = L::kWaves;
    __shared__ __align__(1024) char s_a0[BM * kRowBytes], s_b0[BN * kRowBytes], s_a1[BM * kRowBytes], s_b1[BN * kRowBytes];
    const uint32_t tid = threadIdx.x, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid / kWave)), wm = wave / WN, wn = wave % WN;

    // consecutive tiles on one XCD (workgroups go to the eight by turns), the parts of K one after the other
    const uint32_t all = a.tiles * a.splits, per = all / 8u, more = all % 8u, xcd = blockIdx.x % 8u;
    const uint32_t index = xcd * per + min(xcd, more) + blockIdx.x / 8u;
    const uint32_t split = index / a.tiles, tile = index - split * a.tiles;
    uint32_t m, n;
    const Product &p = a.p[find_tile(a, tile, m, n)];

    const uint32_t half_tiles = (p.K + L::kElements - 1u) / L::kElements, k_tiles = KIND == kInput ? 2u * half_tiles : half_tiles;
    const uint32_t begin = split * a.each, stop = min(begin + a.each, k_tiles);

    typedef Loader<T, L::kColumnsA, BM, kWaves> LoadA;
    typedef Loader<T, L::kColumnsB, BN, kWaves> LoadB;
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
            read_fragments<T, L::kColumnsA, BM, MB>(ta, wm * MB, s, fa);
            read_fragments<T, L::kColumnsB, BN, NB>(tb, wn * NB, s, fb);
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = Fragment<T>::multiply(fb[j], fa[i], acc[i][j]);
        }
    };
    auto step = [&](uint32_t t, char *ta, char *tb, char *next_a, char *next_b) {
        __builtin_amdgcn_s_waitcnt(0);                   // this wave's part of the tile is there ...
        __syncthreads();                                 // ... and everybody's; nobody reads the other tile any more
        const uint32_t left = p.K - (KIND == kInput && t >= half_tiles ? t - half_tiles : t) * L::kElements;
        if (sizeof(T) == 2 && !(L::kColumnsA && L::kColumnsB) && left < L::kElements && left % 8u) {
            if (!L::kColumnsA) clear_behind<BM, L::kThreads>(ta, left, tid);
            if (!L::kColumnsB) clear_behind<BN, L::kThreads>(tb, left, tid);
            __syncthreads();
        }
        if (t + 1u < stop) issue(t + 1u, next_a, next_b);
        multiply(ta, tb);
    };
    if (begin < stop) issue(begin, s_a0, s_b0);
    for (uint32_t t = begin; t < stop; t += 2u) {
        step(t, s_a0, s_b0, s_a1, s_b1);
        if (t + 1u < stop) step(t + 1u, s_a1, s_b1, s_a0, s_b0);
    }

    if (a.splits > 1u) {
        f32x4 *to = (f32x4 *)a.part + ((uint64_t)tile * a.splits + split) * (MB * NB * L::kThreads) + tid;
#pragma unroll
        for (int i = 0; i < MB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) to[(i * NB + j) * L::kThreads] = acc[i][j];
        return;
    }
    MaskKey mask{};
    if (KIND == kOut && a.masked) mask = mask_key(a.mask);
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < L::kNeed; ++j) {
            uint32_t row, col;
            L::place(m, n, tid, i, j, row, col);
            finish<T, KIND>(a, p, mask, row, col, acc[i][j], acc[i][(j + L::kNeed) % NB]);
        }
}

// Adds up what the parts of K gave, in order; a workgroup has one block of each of a tile's waves.
template <typename T, int KIND, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * kWave) void join_kernel(ProductArgs a)
{
    typedef Tiling<T, KIND, BM, BN, WM, WN> L;
    constexpr int NB = L::NB, MB = L::MB;
    const uint32_t tile = blockIdx.x, tid = threadIdx.x, i = blockIdx.y / L::kNeed, j = blockIdx.y % L::kNeed;
    uint32_t m, n, row, col;
    const Product &p = a.p[find_tile(a, tile, m, n)];
    const f32x4 *from = (const f32x4 *)a.part + (uint64_t)tile * a.splits * (MB * NB * L::kThreads) + (i * NB + j) * L::kThreads + tid;
    f32x4 v = {0.f, 0.f, 0.f, 0.f}, w = v;
#pragma unroll 4
    for (uint32_t s = 0; s < a.splits; ++s) {
        v += from[(uint64_t)s * (MB * NB * L::kThreads)];
        if (L::kDual) w += from[(uint64_t)s * (MB * NB * L::kThreads) + L::kNeed * L::kThreads];
    }
    MaskKey mask{};
    if (KIND == kOut && a.masked) mask = mask_key(a.mask);
    L::place(m, n, tid, (int)i, (int)j, row, col);
    finish<T, KIND>(a, p, mask, row, col, v, w);
}

}  // namespace ecrm
