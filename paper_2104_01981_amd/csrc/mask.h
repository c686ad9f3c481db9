// The masks of dropout: drawn anew wherever they are needed, from the seed, the mask's number, the row and the column, and never stored.
//
// Eight columns of a row are one block of Philox 4x32 with ten rounds (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011), counter (column / 8, row, number, number >> 32) and key (seed, seed >> 32); an element has
// 16 of its 128 bits, the lower half of a word before the upper one.  It is dropped where they are below border = 2^16 p, rounded,
// and multiplied by 2^16 / (2^16 - border) elsewhere, so that the expected value is the element's own whatever p was rounded to.
// Twenty 32-bit products for eight elements, two and a half each: half of what 32 bits for an element would take.
#pragma once

#include "types.h"

namespace ecrm {

struct MaskArgs {
    const uint64_t *state;   // device: seed, masks drawn before
    uint64_t offset;         // added to the latter
    uint32_t border;
    float factor;            // of what is kept; 0 where everything is dropped
};

struct MaskKey { uint32_t seed0, seed1, number0, number1, border; float factor; };

__device__ __forceinline__ MaskKey mask_key(const MaskArgs &a)
{
    const uint64_t seed = a.state[0], number = a.state[1] + a.offset;
    return MaskKey{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)number, (uint32_t)(number >> 32), a.border, a.factor};
}

__device__ __forceinline__ uint32_t xor3(uint32_t x, uint32_t y, uint32_t z) { return __builtin_amdgcn_bitop3_b32(x, y, z, 0x96); }

// the 128 bits of columns 8 * block .. 8 * block + 7
__device__ __forceinline__ uint4 mask_block(const MaskKey &k, uint32_t row, uint32_t block)
{
    uint32_t x = block, y = row, z = k.number0, w = k.number1, s0 = k.seed0, s1 = k.seed1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)x * 0xD2511F53u, b = (uint64_t)z * 0xCD9E8D57u;
        const uint32_t nx = xor3((uint32_t)(b >> 32), y, s0), nz = xor3((uint32_t)(a >> 32), w, s1);
        x = nx;
        y = (uint32_t)b;
        z = nz;
        w = (uint32_t)a;
        s0 += 0x9E3779B9u;
        s1 += 0xBB67AE85u;
    }
    return uint4{x, y, z, w};
}

// of the four columns from c (a multiple of four) on
__device__ __forceinline__ uint2 mask_quad(const MaskKey &k, uint32_t row, uint32_t c)
{
    const uint4 b = mask_block(k, row, c / 8u);
    return c & 4u ? uint2{b.z, b.w} : uint2{b.x, b.y};
}

// The bits of N places in lanes' quads, all of them by turns where both lanes of a pair (2i, 2i + 1) have the halves of one block
// each time (`paired`, the same for the wave; both lanes of a pair get here together): a lane draws every other one and hands its
// neighbour the half that it has no use for.  FEW: only the first `used` places count (the same for the wave).
template <int N, bool FEW = false>
__device__ __forceinline__ void mask_quads(const MaskKey &k, const uint32_t (&row)[N], const uint32_t (&c)[N], bool paired, uint2 (&bits)[N],
                                           uint32_t used = N)
{
    static_assert(N % 2 == 0, "places are taken in twos");
    if (!paired) {
#pragma unroll
        for (int q = 0; q < N; ++q)
            if (!FEW || (uint32_t)q < used) bits[q] = mask_quad(k, row[q], c[q]);
        return;
    }
    const bool odd = threadIdx.x & 1u;
#pragma unroll
    for (int q = 0; q < N; q += 2) {
        if (FEW && (uint32_t)q >= used) break;
        const uint4 b = mask_block(k, odd ? row[q + 1] : row[q], (odd ? c[q + 1] : c[q]) / 8u);
        const int s0 = (int)(odd ? b.x : b.z), s1 = (int)(odd ? b.y : b.w);
        constexpr int kSwap = 0xB1;                      // lanes 1, 0, 3, 2 of each four
        const uint2 got = {(uint32_t)__builtin_amdgcn_mov_dpp(s0, kSwap, 0xF, 0xF, true),
                           (uint32_t)__builtin_amdgcn_mov_dpp(s1, kSwap, 0xF, 0xF, true)};
        bits[q] = odd ? got : uint2{b.x, b.y};
        bits[q + 1] = odd ? uint2{b.z, b.w} : got;
    }
}

// What is dropped becomes zero whatever it was.
__device__ __forceinline__ f32x4 keep4(f32x4 v, uint2 bits, uint32_t border)
{
    return f32x4{(bits.x & 0xFFFFu) >= border ? v.x : 0.f, (bits.x >> 16) >= border ? v.y : 0.f,
                 (bits.y & 0xFFFFu) >= border ? v.z : 0.f, (bits.y >> 16) >= border ? v.w : 0.f};
}
__device__ __forceinline__ f32x4 drop4(f32x4 v, uint2 bits, const MaskKey &k) { return keep4(v * k.factor, bits, k.border); }

// ---- host side -------------------------------------------------------------------------------------------------------------
// false: a bad mask.  `factor`: that of MaskArgs in 64 bits.
bool make_mask(const ecrm_mask *mask, MaskArgs &to, double &factor);

// out = residual + the mask's factor times what it keeps of x; arguments have been checked.
void launch_dropout(MaskArgs mask, const void *x, uint64_t x_stride, const void *residual, uint64_t residual_stride, void *out, uint64_t out_stride,
                    uint32_t type, uint64_t rows, uint32_t cols, hipStream_t st);

// Have the rows of a and of b no byte in common?  Rows of one stride may lie between each other; of unlike strides, a whole range of
// rows lies before the other.
bool strided_apart(const void *a, uint64_t a_rows, uint64_t a_row_bytes, uint64_t a_stride_bytes, const void *b, uint64_t b_rows,
                   uint64_t b_row_bytes, uint64_t b_stride_bytes);

}  // namespace ecrm
