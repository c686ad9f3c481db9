// Element types of looked-up rows and of gradients, four elements at a time.
#pragma once

#include "ecrm_internal.h"

namespace ecrm {

typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename T>
struct Quad {
    typedef T type __attribute__((ext_vector_type(4)));
};

// p: aligned to four elements
template <typename T>
__device__ __forceinline__ f32x4 widen4(typename Quad<T>::type v) { return __builtin_convertvector(v, f32x4); }
template <typename T>
__device__ __forceinline__ typename Quad<T>::type round4(f32x4 v)       // to nearest, ties to even
{
    return __builtin_convertvector(v, typename Quad<T>::type);
}

__host__ __device__ __forceinline__ uint32_t type_bytes(uint32_t type) { return type == ECRM_F32 ? 4u : 2u; }

// f(T()) for the element type
template <typename F>
static inline void with_type(uint32_t type, F f)
{
    if (type == ECRM_BF16) f(__bf16());
    else if (type == ECRM_F16) f(_Float16());
    else f(float());
}

}  // namespace ecrm
