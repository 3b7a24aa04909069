// Rows of a cache in 4 bits: 128 values in 68 bytes.
//   bytes 0..63   e2m1 codes, value 2 i in the low half of byte i: sign, two bits of exponent, one of mantissa, that is 0, .5, 1, 1.5, 2, 3, 4, 6
//   bytes 64..67  for each 32 values an e8m0 byte s: the codes stand for multiples of 2^(s - 127); 255: the block holds no numbers
// gfx950 has instructions that turn two bfloat16 values into two codes and back (the scale as a float whose exponent is s), so
// neither way costs arithmetic of its own, and since a code has at most two significant bits, every value is exact in bfloat16.
#pragma once

#include "lc_device.h"
#include "lc_wave.h"
#include "lychee.h"

#define LC_ROW4 LC_CACHE4_ROW     // bytes of a row

typedef __bf16 lc_bf16x2 __attribute__((ext_vector_type(2)));

// The scale byte as the conversions take it.
__device__ __forceinline__ float lc_scale4(uint32_t s) { return __uint_as_float(s << 23); }

// Eight codes -> eight bfloat16 values, in order.
__device__ __forceinline__ uint4 lc_unpack4(uint32_t codes, float scale) {
    uint4 v;
    v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return v;
}

// A row by its 16 lanes: lane `sub` has values [8 sub, 8 sub + 8) in v and gets their codes; *scale is the byte of its block of 32 (four
// lanes, the same in each).  The power of two is the smallest at which the block's largest value is rounded by no more than half a step: up to
// 7 times the power, which the largest code, 6, stands for.  Its exponent and upper mantissa bits tell that (bfloat16 bits of magnitudes order as
// the magnitudes do).  A block with a value that is not finite holds no numbers; with the power 2^126 the code of 4 would be an
// infinity: 3 stands in for it.
__device__ __forceinline__ uint32_t lc_pack4(const uint4& v, uint32_t* scale) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    auto mag = [](uint32_t w) { return __builtin_bit_cast(u16x2, w & 0x7fff7fffu); };
    const u16x2 m2 = __builtin_elementwise_max(__builtin_elementwise_max(mag(v.x), mag(v.y)), __builtin_elementwise_max(mag(v.z), mag(v.w)));
    int top = m2.x > m2.y ? m2.x : m2.y;
    top = max(top, __builtin_amdgcn_update_dpp(0, top, 0xB1, 0xF, 0xF, true));      // quad_perm [1,0,3,2]
    top = max(top, __builtin_amdgcn_update_dpp(0, top, 0x4E, 0xF, 0xF, true));      // quad_perm [2,3,0,1]
    const int exponent = top >> 7;
    if (exponent == 255) {
        *scale = 255u;
        return 0u;
    }
    const int s = max(0, exponent - 2 + ((top & 0x7f) > 0x60 ? 1 : 0));
    *scale = (uint32_t)s;
    const float f = lc_scale4((uint32_t)s);
    uint32_t c = 0u;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(lc_bf16x2, v.x), f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(lc_bf16x2, v.y), f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(lc_bf16x2, v.z), f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(lc_bf16x2, v.w), f, 3);
    if (s == 253) {
        const uint32_t four = (c >> 2) & (c >> 1) & 0x11111111u;                     // codes 6 and 7
        c = (c & ~(7u * four)) | (5u * four);
    }
    return c;
}
