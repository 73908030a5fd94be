// Conversions of the cache in 4 bits (packed.h): codes in e2m1 to fp16 pairs and back.
#pragma once

#include <cuda_fp16.h>

#include "packed.h"

namespace da {

// The 8 codes of a word as four fp16 pairs (exact: every magnitude has two significant bits).  The instruction runs at
// about half the rate of an fp16 multiplication.
__device__ __forceinline__ void packed_unpack(uint32_t w, uint32_t (&r)[4])
{
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
        : "r"(w));
}

// The scale of 32 values whose largest magnitude is amax: amax / 6 in fp16, finite.  65,504, the largest fp16 value, would have the
// scale 10,920 and be held as 65,520, which fp16 (of expanded pages, of the operands of V) rounds to infinity: its scale is 10,912.
__device__ __forceinline__ __half packed_scale(float amax)
{
    const float s = fminf(__fdiv_rn(amax, 6.0f), 65504.0f);
    return __float2half_rn(fabsf(s - 10920.0f) < 4.0f ? 10912.0f : s);          // (what rounds to 10,920: half a step of 8 to either side)
}

// Two codes from a value's quotients: nearest, ties to the even code, at most 6.
__device__ __forceinline__ uint32_t packed_pair(float lo, float hi)
{
    uint32_t r;
    asm("{\n\t.reg .b8 b;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %2, %1;\n\t"
        "cvt.u32.u8 %0, b;\n\t}"
        : "=r"(r)
        : "f"(lo), "f"(hi));
    return r;
}

// Eight codes of the values x (of a 16-bit type), whose block has the scale s: those of the definition, without a division a
// value.  A quotient lies between two codes at one of the ties b = 1/4, 3/4, .. 5 or, since b * s has 14 significant bits and x has
// at most 11, at least 2^-14 of b beside it.  The product with the reciprocal is off by at most 2^-23; rounded to 19 bits it is a tie
// itself where the quotient is, and on the quotient's side of it elsewhere.  (1,900 rows of 16 heads of 128: 8.4 us by divisions, 6.8 so.)
__device__ __forceinline__ uint32_t packed_word(const float (&x)[8], __half s)
{
    const float f = __half2float(s);
    if (f == 0.f) return 0u;
    const float r = __frcp_rn(f);
    auto quotient = [&](float v) { return __uint_as_float((__float_as_uint(v * r) + 16u) & ~31u); };
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= packed_pair(quotient(x[2 * i]), quotient(x[2 * i + 1])) << (8 * i);
    return w;
}

}  // namespace da
