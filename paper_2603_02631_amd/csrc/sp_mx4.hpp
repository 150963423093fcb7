// Microscaled 4-bit elements as kernels make and take them: E2M1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a byte, the lower
// element in the lower bits, and for 32 elements of a row a power of two s, held as its exponent + 127 in a byte (255: NaN).
//   s = the smallest power of two >= 2^-64 with max |x| <= 6 s, code = E2M1(x / s) rounded to nearest, halfway to the even code.
// No code stands for what is not finite: a group that holds any gets scale 255 and codes of zero, and so is NaN as a whole.
#pragma once

#include "sp_common.hpp"

namespace sp {

constexpr int kMx4Group = SP_MX4_GROUP;
constexpr int kMx4Floor = -64;          // log2 of the smallest scale
constexpr int kMx4NaN = 255;

// A magnitude's bits order as the magnitude does, what is not finite above all else.
__device__ __forceinline__ uint32_t mx4_magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// The scale's byte for a largest magnitude with bits m: m = f 2^e with f in [1, 2) needs 2^(e - 2), or 2^(e - 1) where f > 1.5.
__device__ __forceinline__ int mx4_scale(uint32_t m)
{
    if (m >= 0x7f800000u) return kMx4NaN;
    const int b = (int)(m >> 23) - 2 + ((m & 0x7fffffu) > 0x400000u ? 1 : 0);
    return b < 127 + kMx4Floor ? 127 + kMx4Floor : b;
}

// Codes of eight elements under the scale with byte b, the first in the lowest bits. The conversion divides by the power of two and rounds once.
__device__ __forceinline__ uint32_t mx4_codes(const float (&x)[8], int b)
{
    if (b == kMx4NaN) return 0;
    const float s = __uint_as_float((uint32_t)b << 23);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
    return r;
}

}  // namespace sp
