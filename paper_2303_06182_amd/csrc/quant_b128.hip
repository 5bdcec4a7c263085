// Quantisation to e4m3 with a power of two as scale for each block of 128: of a row (activations), or of 128 rows (weights).
//
// s = the smallest 2^n, n >= -126, with max |x| <= 448 s over the block's finite elements (1 for a block of zeros); q = e4m3(x / s), to
// nearest even.  A power of two, so the division is exact: each element is rounded once, by half a step of e4m3 (2^-4 of it; below
// 2^-6 s by 2^-10 s).  An element that is not finite becomes NaN and moves no scale.
//
// Bound by HBM: elements are read once, and wait in registers for their block's maximum.  16 lanes hold a row's 128 elements, 8 each.
#include "b128_dev.h"

namespace moe355 {

namespace {

constexpr int kThreads = 256;
constexpr int kRowItems = 4;  // blocks a group of 16 lanes takes at once

template <bool BF16>
__device__ __forceinline__ void load8(const void *x, int64_t i, float (&v)[8])
{
    if (BF16) {
        const uint4 r = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(x) + i);
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[2 * j] = __uint_as_float(w[j] << 16), v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    } else {
        const float4 a = *reinterpret_cast<const float4 *>(static_cast<const float *>(x) + i);
        const float4 b = *reinterpret_cast<const float4 *>(static_cast<const float *>(x) + i + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
}

__device__ __forceinline__ uint32_t largest8(const float (&v)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, finite_bits(v[j]));
    return m;
}

__device__ __forceinline__ uint2 pack8(const float (&v)[8], float inv)
{
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = finite_bits(v[j]) == 0 && v[j] != 0.f ? __uint_as_float(0x7fc00000u) : v[j] * inv;
    return make_uint2(pack_e4m3(y[0], y[1], y[2], y[3]), pack_e4m3(y[4], y[5], y[6], y[7]));
}

__device__ __forceinline__ uint32_t largest_of_16_lanes(uint32_t m)
{
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off, 64));
    return m;
}

// blocks: of a row, those behind its end (bytes of 127, no elements) among them
template <bool BF16>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(const void *x, int64_t stride, int64_t rows, int cols, int blocks, uint8_t *q, uint8_t *scale)
{
    const int part = threadIdx.x & 15;
    const int64_t items = rows * blocks, step = (int64_t)gridDim.x * (kThreads / 16);
    for (int64_t first = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4); first < items; first += step * kRowItems) {
        float v[kRowItems][8];
        int64_t row[kRowItems];
        int b[kRowItems];
        bool live[kRowItems];
#pragma unroll
        for (int u = 0; u < kRowItems; ++u) {
            const int64_t item = first + u * step;
            row[u] = item / blocks;
            b[u] = (int)(item - row[u] * blocks);
            live[u] = item < items && b[u] * kBlock + part * 8 < cols;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[u][j] = 0.f;
            if (live[u]) load8<BF16>(x, row[u] * stride + b[u] * kBlock + part * 8, v[u]);
        }
#pragma unroll
        for (int u = 0; u < kRowItems; ++u) {
            const int byte = b128_scale_byte(largest_of_16_lanes(largest8(v[u])));
            if (live[u]) *reinterpret_cast<uint2 *>(q + row[u] * cols + b[u] * kBlock + part * 8) = pack8(v[u], b128_inverse(byte));
            if (part == 0 && first + u * step < items) scale[first + u * step] = (uint8_t)byte;
        }
    }
}

// A block of 128 x 128 a thread block: 16 rows at a time, 8 times.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void quantize_blocks_kernel(const void *x, int64_t stride, int64_t matrices, int rows, int cols, int blocks, uint8_t *q,
                                                                  uint8_t *scale)
{
    __shared__ uint32_t of_wave[kThreads / 64];
    const int part = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const int row_blocks = ceil_div(rows, kBlock);
    const int64_t items = matrices * row_blocks * blocks;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t rb = item / blocks, m = rb / row_blocks;
        const int b = (int)(item - rb * blocks), first = (int)(rb - m * row_blocks) * kBlock;
        const int col = b * kBlock + part * 8;
        float v[8][8];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
            const int r = first + r0 + 16 * i;
            if (r < rows && col < cols) load8<BF16>(x, (m * rows + r) * stride + col, v[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) most = max(most, largest8(v[i]));
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, off, 64));
        if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) most = max(most, of_wave[w]);
        __syncthreads();
        const int byte = b128_scale_byte(most);
        const float inv = b128_inverse(byte);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = first + r0 + 16 * i;
            if (r < rows && col < cols) *reinterpret_cast<uint2 *>(q + (m * rows + r) * cols + col) = pack8(v[i], inv);
        }
        if (threadIdx.x == 0) scale[item] = (uint8_t)byte;
    }
}

// The experts' activation on the first product's fp32 results, quantised by rows.
__global__ __launch_bounds__(kThreads) void act_quantize_kernel(const float *gu, int gated, int n_rows, int F, int blocks, const int32_t *offsets, int E,
                                                                uint8_t *q, uint8_t *scale)
{
    const int part = threadIdx.x & 15;
    const int64_t rows = offsets ? min(max(offsets[E], 0), n_rows) : n_rows;
    const int64_t items = rows * blocks, step = (int64_t)gridDim.x * (kThreads / 16);
    for (int64_t item = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4); item < items; item += step) {
        const int64_t row = item / blocks;
        const int b = (int)(item - row * blocks), col = b * kBlock + part * 8;
        float h[8] = {};
        if (col < F) {
            const float *g = gu + row * F * (gated ? 2 : 1) + col;
            load8<false>(g, 0, h);
            float u[8];
            if (gated) load8<false>(g + F, 0, u);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = gated ? h[j] / (1.f + __expf(-h[j])) * u[j] : h[j] > 0.f ? h[j] : h[j] != h[j] ? h[j] : 0.f;
        }
        const int byte = b128_scale_byte(largest_of_16_lanes(largest8(h)));
        if (col < F) *reinterpret_cast<uint2 *>(q + row * F + col) = pack8(h, b128_inverse(byte));
        if (part == 0) scale[item] = (uint8_t)byte;
    }
}

unsigned grid_for(int64_t items, int64_t most) { return (unsigned)(items < 1 ? 1 : items < most ? items : most); }

}  // namespace

int launch_quantize_b128(const void *x, int dtype, int64_t stride, int64_t matrices, int rows, int cols, int block_rows, uint8_t *q, uint8_t *scale,
                         hipStream_t s)
{
    const int blocks = (int)b128_scale_cols(cols);
    const bool bf16 = dtype == MOE_DTYPE_BF16;
    if (block_rows == 1) {
        const int64_t all = matrices * rows, per = (int64_t)(kThreads / 16) * kRowItems;
        const dim3 grid(grid_for((all * blocks + per - 1) / per, 1 << 20));
        if (bf16) hipLaunchKernelGGL(quantize_rows_kernel<true>, grid, dim3(kThreads), 0, s, x, stride, all, cols, blocks, q, scale);
        else hipLaunchKernelGGL(quantize_rows_kernel<false>, grid, dim3(kThreads), 0, s, x, stride, all, cols, blocks, q, scale);
        MOE_LAUNCH_CHECK("quantize_rows_kernel");
    } else {
        const dim3 grid(grid_for(matrices * ceil_div(rows, kBlock) * blocks, 1 << 20));
        if (bf16) hipLaunchKernelGGL(quantize_blocks_kernel<true>, grid, dim3(kThreads), 0, s, x, stride, matrices, rows, cols, blocks, q, scale);
        else hipLaunchKernelGGL(quantize_blocks_kernel<false>, grid, dim3(kThreads), 0, s, x, stride, matrices, rows, cols, blocks, q, scale);
        MOE_LAUNCH_CHECK("quantize_blocks_kernel");
    }
    return MOE_OK;
}

int launch_act_quantize(const float *gu, int gated, int n_rows, int F, const int32_t *offsets, int E, uint8_t *q, uint8_t *scale, hipStream_t s)
{
    const int blocks = (int)b128_scale_cols(F);
    ProfScope ps("act_quantize", s);
    hipLaunchKernelGGL(act_quantize_kernel, dim3(grid_for(((int64_t)n_rows * blocks + 15) / 16, 1 << 16)), dim3(kThreads), 0, s, gu, gated, n_rows, F,
                       blocks, offsets, E, q, scale);
    MOE_LAUNCH_CHECK("act_quantize_kernel");
    return MOE_OK;
}

}  // namespace moe355
