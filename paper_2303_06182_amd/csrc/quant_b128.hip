// Quantisation to e4m3 with a power of two as scale for each block of 128: of a row (activations), or of 128 rows (weights).
//
// s = the smallest 2^n, n >= -126, with max |x| <= 448 s over the block's finite elements (1 for a block of zeros); q = e4m3(x / s), to
// nearest even.  A power of two, so the division is exact: each element is rounded once, by half a step of e4m3 (2^-4 of it; below
// 2^-6 s by 2^-10 s).  An element that is not finite becomes NaN and moves no scale.
//
// Bound by HBM: elements are read once, and wait in registers for their block's maximum.  16 lanes hold a row's 128 elements, 8 each: 16 bytes of bf16
// a lane and load, whole lines a row.  65536 x 2000 by rows 71 us, 16 x 8192 x 2048 by blocks 143 us (bf16; 5.5 TB/s read and written, a large copy 5.0); 64 x 2048 4 us, a launch.
#include "b128_dev.h"

namespace moe355 {

namespace {

constexpr int kThreads = 256;
constexpr int kRowItems = 4;  // blocks a group of 16 lanes takes at once

template <typename Elem>
__device__ __forceinline__ uint2 pack8(const Elem &e, float scale) { return make_uint2(e.pack4(0, scale), e.pack4(4, scale)); }
__device__ __forceinline__ uint32_t over_16_lanes(uint32_t m) { return lanes_max(lanes_max(lanes_max(lanes_max(m, 8), 4), 2), 1); }

// blocks: of a row, those behind its end (bytes of 127, no elements) among them
template <bool BF16>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(const void *x, int64_t stride, int64_t rows, int cols, int blocks, uint8_t *q, uint8_t *scale)
{
    const int part = threadIdx.x & 15;
    const int64_t items = rows * blocks, step = (int64_t)gridDim.x * (kThreads / 16);
    for (int64_t first = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4); first < items; first += step * kRowItems) {
        Elements<BF16, 8> v[kRowItems];
        int64_t row[kRowItems];
        int b[kRowItems];
        bool live[kRowItems];
#pragma unroll
        for (int u = 0; u < kRowItems; ++u) {
            const int64_t item = first + u * step;
            row[u] = item / blocks;
            b[u] = (int)(item - row[u] * blocks);
            live[u] = item < items && b[u] * kBlock + part * 8 < cols;
            v[u].zero();
            if (live[u]) v[u].load8(x, row[u] * stride + b[u] * kBlock + part * 8, 0);
        }
#pragma unroll
        for (int u = 0; u < kRowItems; ++u) {
            const int byte = b128_block_byte(v[u], over_16_lanes);
            if (live[u]) *reinterpret_cast<uint2 *>(q + row[u] * cols + b[u] * kBlock + part * 8) = pack8(v[u], scale_value(byte));
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
    const int row_blocks = (rows - 1) / kBlock + 1;
    const int64_t items = matrices * row_blocks * blocks;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t rb = item / blocks, m = rb / row_blocks;
        const int b = (int)(item - rb * blocks), first = (int)(rb - m * row_blocks) * kBlock;
        const int col = b * kBlock + part * 8;
        Elements<BF16, 64> v;
        v.zero();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = first + r0 + 16 * i;
            if (r < rows && col < cols) v.load8(x, (m * rows + r) * stride + col, 8 * i);
        }
        const int byte = b128_block_byte(v, [&](uint32_t most) {
            most = over_16_lanes(lanes_max(lanes_max(most, 32), 16));
            if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = most;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kThreads / 64; ++w) most = max(most, of_wave[w]);
            __syncthreads();
            return most;
        });
        const float scale_of = scale_value(byte);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = first + r0 + 16 * i;
            if (r < rows && col < cols) *reinterpret_cast<uint2 *>(q + (m * rows + r) * cols + col) = make_uint2(v.pack4(8 * i, scale_of), v.pack4(8 * i + 4, scale_of));
        }
        if (threadIdx.x == 0) scale[item] = (uint8_t)byte;
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
        const dim3 grid(grid_for(matrices * ((rows - 1) / kBlock + 1) * blocks, 1 << 20));
        if (bf16) hipLaunchKernelGGL(quantize_blocks_kernel<true>, grid, dim3(kThreads), 0, s, x, stride, matrices, rows, cols, blocks, q, scale);
        else hipLaunchKernelGGL(quantize_blocks_kernel<false>, grid, dim3(kThreads), 0, s, x, stride, matrices, rows, cols, blocks, q, scale);
        MOE_LAUNCH_CHECK("quantize_blocks_kernel");
    }
    return MOE_OK;
}

}  // namespace moe355
