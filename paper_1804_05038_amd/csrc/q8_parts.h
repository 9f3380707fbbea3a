// q8_parts.h -- fp32 numbers as the sum of two fp16 numbers, for products on the fp16 matrix cores that are as exact as sums in fp32: times a
// power of two that puts the largest of them below 2^14, a number is hi + lo within 2^-22 of itself (2^-38 of the largest where that is more).
#pragma once

#include "q8_device.h"

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// The power of two for values up to m: 2^-e m in [2^13, 2^14), as (inv = 2^-e, returned 2^e); m < 2^-100 counts as zeros (inv = 0).
__device__ __forceinline__ float parts_scale(float m, float &inv)
{
    if (!(m >= 0x1p-100f)) { inv = 0.0f; return 1.0f; }
    const unsigned e = (__float_as_uint(m) >> 23) - 13u;                    // 14 .. 242
    inv = __uint_as_float((254u - e) << 23);
    return __uint_as_float(e << 23);
}

// x minus the low or high fp16 number of a pair, in one instruction that takes it as it is (the compiler converts first).
__device__ __forceinline__ float minus_half(float x, unsigned pair, bool high)
{
    float r;
    if (high) asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(pair), "v"(x));
    else asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(pair), "v"(x));
    return r;
}

// Four values times inv as hi and lo parts (two conversions an instruction).
__device__ __forceinline__ void parts4(float x, float y, float z, float w, float inv, uint2 &hi, uint2 &lo)
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    auto pair = [](float a, float b) { return __builtin_bit_cast(unsigned, __builtin_convertvector(((v2f){a, b}), v2h)); };
    const float v[4] = {x * inv, y * inv, z * inv, w * inv};
    hi = make_uint2(pair(v[0], v[1]), pair(v[2], v[3]));
    lo = make_uint2(pair(minus_half(v[0], hi.x, false), minus_half(v[1], hi.x, true)), pair(minus_half(v[2], hi.y, false), minus_half(v[3], hi.y, true)));
}
