// 4-bit numbers as the kernels hold them (MXFP4 of the OCP microscaling formats):
// e2m1 elements, two to a byte, the first in the low half, and for every 32 of a row
// one byte e for the power of two 2^(e - 127) that multiplies them; e = 255 makes
// them NaN.  Internal to libtileattn.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tileattn_mx {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int GROUP = 32;

// The scale's byte as the number it stands for, in the form that the conversions take:
// they look at the exponent alone (0 is 2^-127 there, 255 NaN)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// The two numbers of byte B of w times the scale, as a pair of bf16, exactly
template <int B>
__device__ __forceinline__ uint32_t pair(uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}

// (B a constant after unrolling)
__device__ __forceinline__ uint32_t pair_at(uint32_t w, float scale, int b)
{
    return b == 0 ? pair<0>(w, scale) : b == 1 ? pair<1>(w, scale) : b == 2 ? pair<2>(w, scale) : pair<3>(w, scale);
}

// The eight numbers of w, one group's, as an operand of the matrix cores
__device__ __forceinline__ bf16x8 eight(uint32_t w, float scale)
{
    return __builtin_bit_cast(bf16x8, u32x4{pair<0>(w, scale), pair<1>(w, scale), pair<2>(w, scale), pair<3>(w, scale)});
}

// The scale's byte for a group whose largest number has these bits (sign 0): the
// power of two that puts it between 3.5 and 7, so that it rounds to 4 or 6 (a power
// that put it between 4 and 8 would clip what lies past 7 to 6).  An infinity counts
// as the largest finite number, NaN gives 255.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    if (top > 0x7F800000u)
        return 255;
    top = top < 0x7F7FFFFFu ? top : 0x7F7FFFFFu;
    const int e = (int)((top + 0x200000u) >> 23) - 2;
    return (uint32_t)(e < 1 ? 1 : e > 252 ? 252 : e);
}

// Eight numbers over the scale, rounded to the nearest e2m1 (to even), beyond 6 as 6
__device__ __forceinline__ uint32_t pack(const float (&x)[8], float scale)
{
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

}  // namespace tileattn_mx
