// Rows in 8 bits: codes of -127 to 127 and a scale, max|x| / 127, for each row or block of one.
#pragma once

#include "common.h"

struct RowScale { float scale, inv; };        // value = code * scale, code = rint(value * inv)

// Of rows (or blocks) whose largest magnitude is `most`, which is finite.
__device__ __forceinline__ RowScale row_scale(float most)
{
    RowScale r;
    r.scale = fmaxf(most / 127.f, 0x1p-126f);
    // 127 / most, rounded up.  Half of the largest value is a tie for every block (63.5: 64), and with a factor that is too small by its rounding it came out as 63.  (Other ties need a
    // largest value of 127 times a power of two, whose factor is exact; and quotients of bf16 that are no ties are 7e-6 and more from one.)
    float inv = 127.f / most;
    if (fmaf(inv, most, -127.f) < 0.f) inv = __uint_as_float(__float_as_uint(inv) + 1u);
    r.inv = most > 0.f ? fminf(inv, 0x1p126f) : 0.f;
    return r;
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// Largest magnitudes of eight bf16, one in either half.  Magnitudes of bf16 order as their bits do, infinities and NaN highest.
__device__ __forceinline__ uint32_t top_of_bf16x8(const uint4 &v)
{
    constexpr uint32_t MAG = 0x7fff7fffu;
    return max_u16x2(max_u16x2(v.x & MAG, v.y & MAG), max_u16x2(v.z & MAG, v.w & MAG));
}

__device__ __forceinline__ uint2 codes_of(const float *f, float inv)
{
    int c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = (int)rintf(f[e] * inv) & 0xff;
    return make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
}
