// Device helpers of the calls on e4m3 operands with a scale per block of 128.
#pragma once

#include "b128_internal.h"
#include "gemm_bf16_dev.h"

namespace moe355 {

// Scale byte of a block: the smallest n >= -126 with largest <= 448 * 2^n, plus 127; 127 where largest is 0.  From the bits: with
// largest = 1.m * 2^e, 448 = 1.75 * 2^8.  (largest is finite and not negative; below 2^-118 the answer is 1 in any case.)
__device__ __forceinline__ int b128_scale_byte(uint32_t largest_bits)
{
    if (largest_bits == 0) return 127;
    const int n = (int)(largest_bits >> 23) - 8 + ((largest_bits & 0x7fffffu) > 0x600000u);
    return n < 1 ? 1 : n;
}
__device__ __forceinline__ float scale_value(int byte) { return __uint_as_float((uint32_t)byte << 23); }  // bytes of 1 to 254

// N consecutive elements of a row, as they are stored.  The scaled conversions divide by the scale and round to nearest even once, as a
// multiplication by its inverse and the plain conversion do (compared on all bf16 numbers and 7e8 fp32 ones), and turn NaN into NaN.
template <bool BF16, int N> struct Elements;
typedef __attribute__((ext_vector_type(2))) short i16x2_b128;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2_b128;
template <int N> struct Elements<true, N> {
    uint32_t x[N / 2];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) x[i] = 0;
    }
    // elements at .. at + 7, a load of 16 bytes; i: in the row
    __device__ __forceinline__ void load8(const void *row, int64_t i, int at)
    {
        const uint4 r = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(row) + i);
        x[at / 2] = r.x, x[at / 2 + 1] = r.y, x[at / 2 + 2] = r.z, x[at / 2 + 3] = r.w;
    }
    // bits of the largest absolute value as fp32; those of infinity or more if an element is not finite
    __device__ __forceinline__ uint32_t largest() const
    {
        u16x2_b128 m = {0, 0};
#pragma unroll
        for (int i = 0; i < N / 2; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_b128, x[i] & 0x7fff7fffu));
        return (uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16;
    }
    // the rare way: infinities become NaN, -> bits of the largest finite one
    __device__ __forceinline__ uint32_t largest_finite()
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const uint32_t lo = x[i] & 0x7fffu, hi = x[i] >> 16 & 0x7fffu;
            if (lo >= 0x7f80u) x[i] = (x[i] & 0xffff0000u) | 0x7fc0u;
            else m = max(m, lo);
            if (hi >= 0x7f80u) x[i] = (x[i] & 0xffffu) | 0x7fc00000u;
            else m = max(m, hi);
        }
        return m << 16;
    }
    // four of them over the scale, as e4m3
    __device__ __forceinline__ uint32_t pack4(int at, float scale) const
    {
        i16x2_b128 w = {0, 0};
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, x[at / 2]), scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, x[at / 2 + 1]), scale, true);
        return __builtin_bit_cast(uint32_t, w);
    }
};
template <int N> struct Elements<false, N> {
    float x[N];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = 0.f;
    }
    __device__ __forceinline__ void load8(const void *row, int64_t i, int at)
    {
        const float4 a = *reinterpret_cast<const float4 *>(static_cast<const float *>(row) + i);
        const float4 b = *reinterpret_cast<const float4 *>(static_cast<const float *>(row) + i + 4);
        x[at] = a.x, x[at + 1] = a.y, x[at + 2] = a.z, x[at + 3] = a.w, x[at + 4] = b.x, x[at + 5] = b.y, x[at + 6] = b.z, x[at + 7] = b.w;
    }
    __device__ __forceinline__ uint32_t largest() const
    {
        float m = 0.f;  // fmaxf leaves NaN out, which the conversion then finds by itself
#pragma unroll
        for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(x[i]));
        return __float_as_uint(m);
    }
    __device__ __forceinline__ uint32_t largest_finite()
    {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
            if (b >= 0x7f800000u) x[i] = __uint_as_float(0x7fc00000u);
            else m = max(m, b);
        }
        return m;
    }
    __device__ __forceinline__ uint32_t pack4(int at, float scale) const
    {
        i16x2_b128 w = {0, 0};
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[at], x[at + 1], scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[at + 2], x[at + 3], scale, true);
        return __builtin_bit_cast(uint32_t, w);
    }
};
// Scale byte of the block whose elements lie in the lanes that `join` finds the maximum over (the same for all of them).
template <typename Elem, typename Join>
__device__ __forceinline__ int b128_block_byte(Elem &e, const Join &join)
{
    uint32_t most = join(e.largest());
    if (most >= 0x7f800000u) most = join(e.largest_finite());
    return b128_scale_byte(most);
}
__device__ __forceinline__ uint32_t lanes_max(uint32_t m, int off) { return max(m, (uint32_t)__shfl_xor((int)m, off, 64)); }

// ---- operands of the matrix instructions: a lane's 32 bytes of a block of a row, 16 at k and 16 at k + 64
typedef __attribute__((ext_vector_type(8))) int Fragment;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

__device__ __forceinline__ Fragment whole(const u32x4 &lo, const u32x4 &hi)
{
    return Fragment{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// at: where the lane's bytes are; k and K, multiples of 16: zeros from K on
__device__ __forceinline__ Fragment load_fragment(const uint8_t *at, int k, int K)
{
    u32x4 lo = {0, 0, 0, 0}, hi = lo;
    if (k < K) lo = *reinterpret_cast<const u32x4 *>(at);
    if (k + 64 < K) hi = *reinterpret_cast<const u32x4 *>(at + 64);
    return whole(lo, hi);
}

// Eight of them as bf16, times a power of two: exact, as bf16 has four more bits.
__device__ __forceinline__ bf16x8 widen(const Fragment &f, int q, float scale)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        w[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * q + i], scale, false));
        w[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * q + i], scale, true));
    }
    return __builtin_bit_cast(bf16x8, w);
}
// g / (1 + exp(-g)).  By the hardware's exponential and reciprocal off by less than (|g| + 4) 2^-23 of it, which is more than the sums are, but far below what bf16 results
// show; EXACT, for fp32: by 2^-22, at 2 us of one token's 22.  Where the exponential passes fp32 the result is -0.
template <bool EXACT>
__device__ __forceinline__ float silu(float g)
{
    if constexpr (!EXACT) return g * __builtin_amdgcn_rcpf(1.f + __expf(-g));
    const float d = 1.f + expf(-g), r = __builtin_amdgcn_rcpf(d);
    return g * (d < INFINITY ? fmaf(fmaf(-d, r, 1.f), r, r) : 0.f);
}
__device__ __forceinline__ float relu(float g) { return g > 0.f ? g : g != g ? g : 0.f; }

// ---- the expert of a block and its rows
struct ExpertRows {
    int expert, first, end;
};
// The expert that a grid's row y is for: y itself, or, where the grid has fewer rows than there are experts (there are fewer rows of A then), the y-th that
// has rows.  expert -1: there is none.
__device__ __forceinline__ ExpertRows expert_rows(const GemmB128 &g, int y, int grid_rows)
{
    if (!g.offsets) return {0, 0, g.n_rows};
    if (grid_rows == g.E) {
        const int first = min(max(g.offsets[y], 0), g.n_rows);
        return {y, first, min(max(g.offsets[y + 1], first), g.n_rows)};
    }
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < g.E; base += 64) {
        int first = 0, end = 0;
        if (base + lane < g.E) {
            first = min(max(g.offsets[base + lane], 0), g.n_rows);
            end = min(max(g.offsets[base + lane + 1], first), g.n_rows);
        }
        unsigned long long some = __ballot(end > first);
        const int n = __popcll(some);
        if (y < n) {
            for (; y > 0; --y) some &= some - 1;
            const int src = __builtin_ctzll(some);
            return {base + src, __builtin_amdgcn_readlane(first, src), __builtin_amdgcn_readlane(end, src)};
        }
        y -= n;
    }
    return {-1, 0, 0};
}

}  // namespace moe355
