// Dropout of an activation, with what it is added to in the same pass: out = residual + c m x, m drawn in registers (mask.h).  Its
// gradient is the same call on the gradient.
//
// What bounds it: memory, rows * cols elements in (twice with a residual) and out; 262 149 x 512 in bf16 with a residual 159 us, 5.1 TB/s, where a
// copy of 4 GiB moves 4.7.  A lane takes the eight columns of a block and keeps four blocks in flight: drawing the masks, twenty wide
// products for a block, stays behind that.  A small tensor (600 x 128) is the call: kernel 2.4 us.
#include "mask.h"

#include <math.h>

namespace ecrm {

constexpr int kDropThreads = 256;
constexpr uint32_t kDropUnits = 1u << 30;            // blocks of a launch, at most

struct DropArgs {
    const void *x, *residual;
    void *out;
    uint64_t x_stride, residual_stride, out_stride;
    uint32_t first_row, units, cols;
    Divider blocks;                                  // by the blocks of a row
    MaskArgs mask;
};

template <typename T>
struct Octet {
    typedef T type __attribute__((ext_vector_type(8)));
};

// 8 or (in a row's last block) 4 elements.  WIDE: rows and strides allow 16 bytes at a time.
template <typename T, bool WIDE>
__device__ __forceinline__ void read8(const T *p, bool whole, f32x4 (&v)[2])
{
    typedef typename Quad<T>::type Four;
    if (WIDE && sizeof(T) == 2) {
        const typename Octet<T>::type e = *(const typename Octet<T>::type *)p;
        v[0] = widen4<T>(__builtin_shufflevector(e, e, 0, 1, 2, 3));
        v[1] = widen4<T>(__builtin_shufflevector(e, e, 4, 5, 6, 7));
    } else {
        v[0] = widen4<T>(*(const Four *)p);
        v[1] = widen4<T>(((const Four *)p)[whole ? 1 : 0]);
    }
}
template <typename T, bool WIDE>
__device__ __forceinline__ void write8(T *p, bool whole, const f32x4 (&v)[2])
{
    typedef typename Quad<T>::type Four;
    const Four a = round4<T>(v[0]), b = round4<T>(v[1]);
    if (WIDE && sizeof(T) == 2) {
        __builtin_nontemporal_store((typename Octet<T>::type)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7), (typename Octet<T>::type *)p);
    } else {
        __builtin_nontemporal_store(a, (Four *)p);
        if (whole) __builtin_nontemporal_store(b, (Four *)p + 1);
    }
}

template <typename T, bool WIDE, bool RESIDUAL>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(DropArgs a)
{
    constexpr uint32_t U = 4;
    const MaskKey key = mask_key(a.mask);
    const uint32_t step = gridDim.x * kDropThreads;
    for (uint32_t u0 = blockIdx.x * kDropThreads + threadIdx.x; u0 < a.units; u0 += U * step) {
        f32x4 v[U][2], r[U][2];
        uint32_t row[U], block[U];
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) {
            const uint32_t u = (uint32_t)min((uint64_t)u0 + (uint64_t)q * step, (uint64_t)a.units - 1u);
            row[q] = a.blocks.div(u);
            block[q] = u - row[q] * a.blocks.d;
            const bool whole = block[q] * 8u + 4u < a.cols;
            read8<T, WIDE>((const T *)a.x + row[q] * a.x_stride + block[q] * 8u, whole, v[q]);
            if (RESIDUAL) read8<T, WIDE>((const T *)a.residual + row[q] * a.residual_stride + block[q] * 8u, whole, r[q]);
        }
#pragma unroll
        for (uint32_t q = 0; q < U; ++q) {
            if ((uint64_t)u0 + (uint64_t)q * step >= a.units) break;
            const uint4 bits = mask_block(key, a.first_row + row[q], block[q]);
            v[q][0] = drop4(v[q][0], uint2{bits.x, bits.y}, key);
            v[q][1] = drop4(v[q][1], uint2{bits.z, bits.w}, key);
            if (RESIDUAL) {
                v[q][0] += r[q][0];
                v[q][1] += r[q][1];
            }
            write8<T, WIDE>((T *)a.out + row[q] * a.out_stride + block[q] * 8u, block[q] * 8u + 4u < a.cols, v[q]);
        }
    }
}

void launch_dropout(MaskArgs mask, const void *x, uint64_t x_stride, const void *residual, uint64_t residual_stride, void *out, uint64_t out_stride,
                    uint32_t type, uint64_t rows, uint32_t cols, hipStream_t st)
{
    DropArgs a{};
    const uint32_t size = type_bytes(type);
    a.mask = mask;
    a.cols = cols;
    a.x_stride = x_stride; a.residual_stride = residual_stride; a.out_stride = out_stride;
    const uint32_t blocks = (cols + 7u) / 8u;
    a.blocks = make_divider(blocks);
    auto wide_rows = [&](const void *p, uint64_t stride) { return (uintptr_t)p % 16 == 0 && stride * size % 16 == 0; };
    const bool wide = cols % 8 == 0 && wide_rows(x, x_stride) && wide_rows(out, out_stride) && (!residual || wide_rows(residual, residual_stride));
    const uint64_t slice = kDropUnits / blocks;
    for (uint64_t at = 0; at < rows; at += slice) {
        const uint64_t cnt = rows - at < slice ? rows - at : slice;
        a.first_row = (uint32_t)at;
        a.units = (uint32_t)(cnt * blocks);
        a.x = (const char *)x + at * x_stride * size;
        a.residual = residual ? (const char *)residual + at * residual_stride * size : nullptr;
        a.out = (char *)out + at * out_stride * size;
        const uint32_t most = 256u * 8u, wanted = (a.units + kDropThreads - 1) / kDropThreads;
        const dim3 grid(wanted < most ? wanted : most), threads(kDropThreads);
        with_type(type, [&](auto t) {
            typedef decltype(t) T;
            if (wide && residual) hipLaunchKernelGGL((dropout_kernel<T, true, true>), grid, threads, 0, st, a);
            else if (wide) hipLaunchKernelGGL((dropout_kernel<T, true, false>), grid, threads, 0, st, a);
            else if (residual) hipLaunchKernelGGL((dropout_kernel<T, false, true>), grid, threads, 0, st, a);
            else hipLaunchKernelGGL((dropout_kernel<T, false, false>), grid, threads, 0, st, a);
        });
    }
}

bool make_mask(const ecrm_mask *mask, MaskArgs &to, double &factor)
{
    if (!mask->state || (uintptr_t)mask->state % 8 || !(mask->p >= 0.0 && mask->p <= 1.0)) return false;
    to.state = mask->state;
    to.offset = mask->offset;
    to.border = (uint32_t)llrint(mask->p * 65536.0);
    factor = to.border < 65536u ? 65536.0 / (double)(65536u - to.border) : 0.0;
    to.factor = (float)factor;
    return true;
}

bool strided_apart(const void *a, uint64_t a_rows, uint64_t a_row, uint64_t a_stride, const void *b, uint64_t b_rows, uint64_t b_row,
                   uint64_t b_stride)
{
    if (!a_rows || !b_rows || !a_row || !b_row) return true;
    const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
    const uintptr_t a_end = pa + (a_rows - 1) * a_stride + a_row, b_end = pb + (b_rows - 1) * b_stride + b_row;
    if (a_end <= pb || b_end <= pa) return true;
    if (a_rows == 1 || b_rows == 1) {                    // one row against several: what of the several is there
        const bool one = a_rows == 1;
        const uintptr_t p = one ? pa : pb, row = one ? a_row : b_row, q = one ? pb : pa;
        const uint64_t rows = one ? b_rows : a_rows, q_row = one ? b_row : a_row, stride = one ? b_stride : a_stride;
        const uint64_t i = p < q + q_row ? 0 : (p - q - q_row) / stride + 1;        // the first of them that ends behind p
        return i >= rows || q + i * stride >= p + row;
    }
    if (a_stride != b_stride) return false;
    // in step with each other: b's rows begin where a's have ended, and end where a's next begin
    const uint64_t by = pb >= pa ? (pb - pa) % a_stride : (a_stride - (pa - pb) % a_stride) % a_stride;
    return by >= a_row && by + b_row <= a_stride;
}

}  // namespace ecrm

using namespace ecrm;

extern "C" int ecrm_dropout(const ecrm_mask *mask, const void *x, uint64_t x_stride, const void *residual, uint64_t residual_stride,
                            void *out, uint64_t out_stride, uint32_t type, uint64_t rows, uint32_t cols, void *stream)
{
    DropArgs a{};
    double factor;
    if (!mask || !make_mask(mask, a.mask, factor)) return ECRM_EINVAL;
    if (type > ECRM_F16 || cols < 4 || cols % 4 || cols > (1u << 24) || rows > (1ull << 32)) return ECRM_EINVAL;
    if (!rows) return ECRM_OK;
    const uint32_t size = type_bytes(type);
    const uint64_t row = (uint64_t)cols * size;
    auto ok = [&](const void *p, uint64_t stride) {
        return p && (uintptr_t)p % (4 * size) == 0 && stride >= cols && stride % 4 == 0 && (rows == 1 || stride <= (1ull << 48) / (rows - 1));
    };
    if (rows == 1) x_stride = residual_stride = out_stride = cols;          // of one row it says nothing
    if (!ok(x, x_stride) || !ok(out, out_stride) || (residual && !ok(residual, residual_stride))) return ECRM_EINVAL;
    auto same_or_apart = [&](const void *p, uint64_t stride) {              // in place, or clear of it
        return (p == out && stride == out_stride) || strided_apart(p, rows, row, stride * size, out, rows, row, out_stride * size);
    };
    if (!same_or_apart(x, x_stride) || (residual && !same_or_apart(residual, residual_stride)) ||
        !strided_apart(mask->state, 1, 16, 16, out, rows, row, out_stride * size))
        return ECRM_EINVAL;
    launch_dropout(a.mask, x, x_stride, residual, residual_stride, out, out_stride, type, rows, cols, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? ECRM_OK : ECRM_EHIP;
}
