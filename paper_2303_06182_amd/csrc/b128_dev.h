// Device helpers of the calls on e4m3 operands with a scale per block of 128.
#pragma once

#include "b128_internal.h"

namespace moe355 {

// Scale byte of a block: the smallest n >= -126 with largest <= 448 * 2^n, plus 127; 127 where largest is 0.  From the bits: with
// largest = 1.m * 2^e, 448 = 1.75 * 2^8.  (largest is finite and not negative; below 2^-118 the answer is 1 in any case.)
__device__ __forceinline__ int b128_scale_byte(uint32_t largest_bits)
{
    if (largest_bits == 0) return 127;
    const int n = (int)(largest_bits >> 23) - 8 + ((largest_bits & 0x7fffffu) > 0x600000u);
    return n < 1 ? 1 : n;
}
// 1 / scale: 2^(127 - byte), for bytes of 1 to 253 (a finite number's byte is at most 247)
__device__ __forceinline__ float b128_inverse(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

__device__ __forceinline__ uint32_t finite_bits(float x)
{
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0;
}
// Four numbers of at most 448, NaN or infinity to e4m3 to nearest even; the latter two to NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d)
{
    int word = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, word, true);
}

}  // namespace moe355
