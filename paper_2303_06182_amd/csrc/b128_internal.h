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
// h = act(gu) and its quantised rows: gu fp32 [rows, gated ? 2 : 1, F]; rows from offsets[0] to offsets[E] (NULL: all n_rows)
int launch_act_quantize(const float *gu, int gated, int n_rows, int F, const int32_t *offsets, int E, uint8_t *q, uint8_t *scale, hipStream_t s);

// ---- products (gemm_b128.hip)
struct GemmB128 {
    const uint8_t *a, *a_scale;  // [a_count, K], [a_count, scale columns]
    int a_count;
    const int32_t *a_rows;  // row r of the product is row a_rows[r] of a (NULL: r)
    const uint8_t *w, *w_scale;  // [E, N, K], [E, ceil(N / 128), scale columns]
    const int32_t *offsets;  // [E + 1] or NULL: one expert with all rows
    int E, n_rows, N, K;
    int Nh;  // weight rows of a matrix: an expert has N / Nh of them one after the other, each with scales of its own
    void *c;
    int c_dtype;
    bool precise;  // sums in fp32 throughout: see gemm_b128.hip
    const char *name;  // of the launch for the event profiler
};
int launch_gemm_b128(const GemmB128 &g, hipStream_t s);

}  // namespace moe355
