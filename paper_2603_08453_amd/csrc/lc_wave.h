// Matrix operands and the exchanges between a wavefront's 16-lane rows that the attention kernels share.
#pragma once

#include "lc_device.h"

typedef __bf16 lc_bf16x8 __attribute__((ext_vector_type(8)));
typedef float lc_f32x4 __attribute__((ext_vector_type(4)));

// a in the lower half of the wavefront and b in the upper half, each summed over the two halves
__device__ __forceinline__ float lc_add_halves(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// a in the even 16-lane rows and b in the odd ones, each summed over a row and its neighbour
__device__ __forceinline__ float lc_add_rows(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// maximum over the four 16-lane groups, in every lane
__device__ __forceinline__ float lc_max_groups(float v) {
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
