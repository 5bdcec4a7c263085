// Internal declarations of the calls on e4m3 operands with a scale per block of 128 and of the selection in front of them.
#pragma once

#include "moe_internal.h"

namespace moe355 {

constexpr int kBlock = 128;  // k of a block, and weight rows of one

// Scale bytes of a row: one per block, in groups of four so that four blocks' are one word.
__host__ __device__ __forceinline__ int64_t b128_scale_cols(int64_t cols) { return (cols + 4 * kBlock - 1) / (4 * kBlock) * 4; }

// ---- selection (select_experts.hip)
struct SelectParams {
    const void *logits;  // [T, E], `stride` elements from row to row
    int64_t stride;
    const float *bias;  // [E] or NULL
    int T, E, k;
    int softmax;         // scores: 1 softmax, 0 sigmoid
    int groups, kept, group_top;
    int renorm;
    float scale;
    int32_t *idx;  // [T, k]
    float *w;      // [T, k]
    // fp32 logits in slices along the gate's K: the sums go to sum_out, which is `logits`
    int n_parts;  // slices further than `logits`
    const float *parts;
    int64_t part_stride;
    float *sum_out;
};
int launch_select(const SelectParams &p, int dtype, hipStream_t s);
int check_select(const moe_select_config_t *c);
SelectParams select_params(const moe_select_config_t &c);

// ---- quantisation (quant_b128.hip)
int launch_quantize_b128(const void *x, int dtype, int64_t stride, int64_t matrices, int rows, int cols, int block_rows, uint8_t *q, uint8_t *scale,
                         hipStream_t s);
// ---- products
enum { kRowsE4m3, kRowsBf16, kRowsF32 };    // what A is: bytes and scales, or rows that are quantised on the way (few rows only)
enum { kActNone, kActRelu, kActSilu };      // of the results; silu: of the first matrix's, times the second's
struct GemmB128 {
    int rows, act;
    const uint8_t *a, *a_scale;  // [a_count, K], [a_count, scale columns]
    int a_count;
    const int32_t *a_rows;       // row r of the product is row a_rows[r] of a (NULL: r)
    const uint8_t *w, *w_scale;  // [E, N, K], [E, N / Nh, ceil(Nh / 128), scale columns]
    const int32_t *offsets;      // [E + 1] or NULL: one expert with all rows
    int E, n_rows, N, K;
    int Nh;  // weight rows of a matrix: an expert has N / Nh of them one after the other, each with scales of its own
    void *c;  // [n_rows, N], with an activation [n_rows, Nh]; tiles with an activation: bytes, with
    uint8_t *c_scale;  // [n_rows, scale columns of Nh]
    int c_dtype;
    bool precise;  // sums in fp32 throughout (gemm_b128_tile.hip)
    bool deep;         // with an activation: sums of sums of 256 products (gemm_b128_tile.hip)
    const char *name;  // of the launch for the event profiler
};
// few rows an expert, which it quantises itself (gemm_b128_stream.hip)
bool b128_few_rows(int n_rows, int E);
int64_t b128_few_rows_most(int E);  // rows that are few, at most
int launch_gemm_b128_stream(const GemmB128 &g, hipStream_t s);
// many (gemm_b128_tile.hip).  kTileTime: what a K tile of a tile of 64, 128, 192 or 256 rows takes, fast and precise, in units of 50 ns
constexpr int kTileTime[2][4] = {{16, 16, 22, 28}, {22, 35, 46, 56}};
bool b128_tiles_ok(const GemmB128 &g);
int launch_gemm_b128_tile(const GemmB128 &g, hipStream_t s);
// few output tiles, and what the tiles cannot address, without an activation (gemm_b128_small.hip)
int launch_gemm_b128_small(const GemmB128 &g, hipStream_t s);
int launch_gemm_b128(const GemmB128 &g, hipStream_t s);  // the one or the other, of operands in e4m3

}  // namespace moe355
