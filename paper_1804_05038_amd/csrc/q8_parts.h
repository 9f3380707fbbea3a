// q8_parts.h -- fp32 numbers as the sum of two fp16 numbers, for products on the fp16 matrix cores that are as exact as sums in fp32: times a
// power of two that puts the largest of them below 2^14, a number is hi + lo within 2^-22 of itself (2^-39 of the largest where that is more).
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

// Four values times inv as hi and lo parts (two conversions an instruction, the rest in one that takes an fp16 number as it is).
__device__ __forceinline__ void parts4(float x, float y, float z, float w, float inv, uint2 &hi, uint2 &lo)
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    const float v[4] = {x * inv, y * inv, z * inv, w * inv};
    const v2h a = __builtin_convertvector(((v2f){v[0], v[1]}), v2h), b = __builtin_convertvector(((v2f){v[2], v[3]}), v2h);
    const v2f c = {fmaf((float)a[0], -1.0f, v[0]), fmaf((float)a[1], -1.0f, v[1])}, d = {fmaf((float)b[0], -1.0f, v[2]), fmaf((float)b[1], -1.0f, v[3])};
    hi = make_uint2(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b));
    lo = make_uint2(__builtin_bit_cast(unsigned, __builtin_convertvector(c, v2h)), __builtin_bit_cast(unsigned, __builtin_convertvector(d, v2h)));
}
