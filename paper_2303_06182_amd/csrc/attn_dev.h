// Device helpers shared by the attention kernels.
#pragma once

#include "attn_internal.h"
#include "gemm_bf16_dev.h"

namespace moe355 {

static constexpr float kLn2 = 0.69314718055994530942f;

template <int NS>
struct Pieces {
    bf16x8 x[NS];
};
// eight fp32 numbers as NS bf16 pieces: rounded, the rest rounded, ..
template <int NS>
__device__ __forceinline__ Pieces<NS> split(const float (&v)[8])
{
    Pieces<NS> r;
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = v[i];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = pack_bf16(rest[2 * i], rest[2 * i + 1]);
            rest[2 * i] -= __uint_as_float(w[i] << 16);
            rest[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
        }
        const uint4 q = make_uint4(w[0], w[1], w[2], w[3]);
        r.x[n] = __builtin_bit_cast(bf16x8, q);
    }
    return r;
}

// eight e4m3 numbers times a power of two, which the conversion takes
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi, float scale = 1.f)
{
    uint4 w;
    w.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
    w.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
    w.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
    w.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
    return __builtin_bit_cast(bf16x8, w);
}

// out[c] = byte c of r0, r1, r2, r3, for c = 0 .. 3
__device__ __forceinline__ void transpose4(uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3, uint32_t (&out)[4])
{
    const uint32_t a = __builtin_amdgcn_perm(r1, r0, 0x05010400), b = __builtin_amdgcn_perm(r1, r0, 0x07030602);
    const uint32_t c = __builtin_amdgcn_perm(r3, r2, 0x05010400), d = __builtin_amdgcn_perm(r3, r2, 0x07030602);
    out[0] = __builtin_amdgcn_perm(c, a, 0x05040100);
    out[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
    out[2] = __builtin_amdgcn_perm(d, b, 0x05040100);
    out[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}

}  // namespace moe355
