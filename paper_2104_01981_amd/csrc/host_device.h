// Plain arithmetic that kernels and host share; it compiles without HIP, too, so that tests can ask the very same functions.
#pragma once

#include <stdint.h>

#ifdef __HIP__
#include <hip/hip_runtime.h>
#define ECRM_HD __host__ __device__ __forceinline__
#else
#define ECRM_HD inline
#endif
