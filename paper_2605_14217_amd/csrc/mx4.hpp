// Pages of 4-bit numbers: where they lie, and the two conversions.
//
// A number is a sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6; 32 consecutive ones of a head share a power of two, kept as a byte, 127 more than its exponent (255: the
// 32 are NaN).  That is the 4-bit format of the OCP Microscaling specification (E2M1 elements, E8M0 scales), which the vector units convert from and to in one
// instruction for two numbers.  A page holds, head after head, the numbers of its tokens (two a byte, the first in the low bits), then their powers.
#pragma once
#include "common.hpp"

namespace preft {

constexpr int MX4_BLOCK = 32;

template <int D> struct Mx4Page {
    static constexpr int NUMBERS = D / 2, POWERS = D / MX4_BLOCK;       // bytes of a token
    static constexpr int TOKEN = NUMBERS + POWERS;
    // bytes of one head of a page
    static __host__ __device__ __forceinline__ int64_t head_bytes(int page_shift) { return (int64_t)TOKEN << page_shift; }
};

// The power's byte for 32 numbers whose largest magnitude has these bits: the least power at which it is below 7 (what is between 6 and 7 becomes 6, no further off than a
// rounding there), as far as there is one between 2^-125 and 2^125: no value is then subnormal or infinite.
__device__ __forceinline__ uint32_t mx4_power(uint32_t top)
{
    if (top >= 0x7f800000u) return 255u;
    const int32_t e = (int32_t)((top + 0x200000u) >> 23) - 2;           // from 1.75 times a power of two on: the next one
    return (uint32_t)max(2, min(e, 252));
}
// 2^-(exponent), to multiply with: exact, also where a number is subnormal; of NaN it does not matter
__device__ __forceinline__ float mx4_inverse(uint32_t power) { return __uint_as_float((254u - min(power, 252u)) << 23); }
__device__ __forceinline__ float mx4_scale(uint32_t power) { return __uint_as_float(power << 23); }   // 255: the conversions below give NaN

// eight numbers, already divided by their power: to nearest, in the middle to even, no larger than 6
__device__ __forceinline__ uint32_t mx4_pack(const float (&x)[8])
{
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], 1.0f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], 1.0f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], 1.0f, 3);
}
// the values of eight numbers: every one is a bf16 number
__device__ __forceinline__ u32x4_t mx4_bf16(uint32_t numbers, float scale)
{
    return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(numbers, scale, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(numbers, scale, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(numbers, scale, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(numbers, scale, 3))};
}

}  // namespace preft
