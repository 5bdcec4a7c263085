// The feed-forward's products for few rows an expert: bound by reading the weights.
//
// A wave takes 16 weight rows (of each of the two matrices of a gated pair), or 32, of one expert and up to 32 rows of A, which the block
// holds in LDS; it reads its weights straight into registers, P blocks of k ahead.  Waves of a block share the k of the same weight rows (KS of them,
// joined in LDS at the end) where there is too little work for one each.  A lane of weight row r holds bytes 16 (lane / 16) and 64 + 16 (lane / 16) of the
// row's 128, so that a pair of loads takes whole lines of 16 rows; either operand's k lie in that order.  Both operands are widened to bf16 and go through
// v_mfma_f32_16x16x32_bf16, exact products and fp32 sums: the matrix cores have time here.
//
// The rows come as they are, bf16 or fp32, and are quantised on their way to LDS: of few rows that costs less than a launch
// and a trip through memory.  The quantisation is that of quant_b128.hip, bit for bit.
//
// 64 tokens x 8 over 128 experts, 2048 -> 2 x 1024 -> 2048: 105 + 61 us, 5.1 and 4.4 TB/s of the weights.  Without the products it takes as long (measured in
// a copy): it waits for memory.  Blocks of k begun at another place a wave, loads past the caches: no faster; a block for several groups of rows one
// after the other: 10 % slower for two.  With fewer rows than experts the grid has a row for each expert that has some: one token's 8 of 64 experts 33 -> 23 us.
#include <mutex>

#include "b128_dev.h"

namespace moe355 {

namespace {

constexpr int NW = 8, kThreads = NW * 64;
constexpr int P = 3;   // blocks of k on their way: with two waves of rows, what 128 registers hold
constexpr int NC = 2;  // blocks of 16 weight rows

// k of A that LDS holds at once: 64 KB, so that a CU has room for two blocks
constexpr int held_k(int mr) { return 4096 / mr; }
constexpr int kRowPad = 16;  // bytes behind a row, which put 16 rows' chunks of 16 bytes on all banks

struct Stage {
    uint8_t *a;   // [16 MR][k + kRowPad]
    uint8_t *as;  // [blocks][16 MR]
    int ld;
};

// Rows row0 .. of A, k0 .. k1 of them, to LDS.
template <int A, int MR>
__device__ __forceinline__ void stage_rows(const GemmB128 &g, const Stage &st, int row0, int rows, int k0, int k1)
{
    const int part = threadIdx.x & 15, blocks = ceil_div(k1 - k0, kBlock);
    for (int i = threadIdx.x >> 4; i < rows * blocks; i += kThreads / 16) {
        const int row = i / blocks, b = i - row * blocks;
        int at = row0 + row;
        if (g.a_rows) at = min(max(g.a_rows[at], 0), g.a_count - 1);
        const int k = k0 + b * kBlock + part * 8;
        Elements<A == kRowsBf16, 8> e;
        e.zero();
        if (k < k1) e.load8(g.a + (int64_t)at * g.K * (A == kRowsF32 ? 4 : 2), k, 0);
        const int byte = b128_block_byte(e, [](uint32_t m) { return lanes_max(lanes_max(lanes_max(lanes_max(m, 8), 4), 2), 1); });
        *reinterpret_cast<uint2 *>(st.a + row * st.ld + b * kBlock + part * 8) = make_uint2(e.pack4(0, scale_value(byte)), e.pack4(4, scale_value(byte)));
        if (part == 0) st.as[b * 16 * MR + row] = (uint8_t)byte;
    }
}

// Rows row0 .. row0 + rows - 1 (16 MR at most) of expert e against all of the block's weight rows.
template <int A, int ACT, int MR, int KS>
__device__ __forceinline__ void stream_rows(const GemmB128 &g, uint8_t *smem, int e, int row0, int rows)
{
    constexpr int CW = NW / KS;                       // groups of weight rows a block works on at once
    constexpr int COLS = ACT == kActSilu ? 16 : 32;   // of the result, of a group
    constexpr int KC = held_k(MR);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, part = lane >> 4;
    const int kw = wave % KS, cw = wave / KS;
    const int K = g.K, KB = ceil_div(K, kBlock), chunks = ceil_div(K, KC);
    const int groups = ceil_div(g.Nh, COLS), n_blocks = ceil_div(g.Nh, kBlock);
    const int scale_cols = (int)b128_scale_cols(K);
    const int held = min(K, KC);
    Stage st;
    st.ld = ceil_div(held, kBlock) * kBlock + kRowPad;
    st.a = smem;
    st.as = smem + 16 * MR * st.ld;
    float *const join = reinterpret_cast<float *>(smem + 16 * MR * st.ld + align_up(ceil_div(held, kBlock) * 16 * MR, 16));
    const int its = (groups - (int)blockIdx.x * CW + (int)gridDim.x * CW - 1) / ((int)gridDim.x * CW);  // the same for all waves

    {
        // ---- this wave's stream of weights: its groups, and of each the blocks of k that are kw modulo KS
        int l_it = 0, l_b = kw;
        __amdgpu_buffer_rsrc_t buf[NC];
        const uint8_t *ws[NC];
        auto aim = [&]() __attribute__((always_inline)) {
            const int group = ((int)blockIdx.x + l_it * (int)gridDim.x) * CW + cw;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int half = ACT == kActSilu ? c : 0, col = group * COLS + (ACT == kActSilu ? 0 : c * 16);
                const int live = __builtin_amdgcn_readfirstlane(min(max(g.Nh - col, 0), 16));
                const int at = live ? col : 0;
                const uint8_t *base = g.w + ((int64_t)e * g.N + (int64_t)half * g.Nh + at) * K;
                buf[c] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), 0, live * K, 0x00020000);
                ws[c] = g.w_scale + ((int64_t)(e * (g.N / g.Nh) + half) * n_blocks + at / kBlock) * scale_cols;
            }
        };
        struct Raw {
            u32x4 w[NC][2];
            int s[NC];
        } raw[P];
        auto load = [&](Raw &f) __attribute__((always_inline)) {
            if (l_it >= its) return;
            const int k = l_b * kBlock + part * 16;
            const uint32_t off = (uint32_t)(r * K + part * 16);
#pragma unroll
            for (int c = 0; c < NC; ++c) {
#pragma unroll
                for (int h = 0; h < 2; ++h)  // past the end of the buffer: zeros
                    f.w[c][h] = __builtin_amdgcn_raw_buffer_load_b128(buf[c], k + 64 * h < K ? off + 64 * h : 0x80000000u, l_b * kBlock, 0);
                f.s[c] = ws[c][l_b];
            }
            l_b += KS;
            if (l_b >= KB) {
                l_b = kw;
                ++l_it;
                if (l_it < its) aim();
            }
        };
        if (kw < KB) {
            aim();
#pragma unroll
            for (int j = 0; j < P; ++j) load(raw[j]);
        }
        int slot = 0;
        for (int it = 0; it < its; ++it) {
            const int group = ((int)blockIdx.x + it * (int)gridDim.x) * CW + cw;
            f32x4 acc[MR][NC] = {};
            for (int chunk = 0; chunk < chunks; ++chunk) {
                if (it == 0 || chunks > 1) {
                    __syncthreads();
                    stage_rows<A, MR>(g, st, row0, rows, chunk * KC, min(K, (chunk + 1) * KC));
                    __syncthreads();
                }
                const int b0 = chunk * (KC / kBlock), b1 = min(KB, b0 + KC / kBlock);
                int b = kw;  // KC / 128 is a multiple of KS
                auto multiply = [&](const Raw &f) __attribute__((always_inline)) {
                    const int at = b;
                    Fragment af[MR];
                    float as[MR];
#pragma unroll
                    for (int m = 0; m < MR; ++m) {
                        const uint8_t *row = st.a + (16 * m + r) * st.ld + at * kBlock + part * 16;
                        const u32x4 lo = *reinterpret_cast<const u32x4 *>(row), hi = *reinterpret_cast<const u32x4 *>(row + 64);
                        af[m] = whole(lo, hi);
                        as[m] = scale_value(st.as[at * 16 * MR + 16 * m + r]);
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        bf16x8 aw[MR];
#pragma unroll
                        for (int m = 0; m < MR; ++m) aw[m] = widen(af[m], q, as[m]);
#pragma unroll
                        for (int c = 0; c < NC; ++c) {
                            const bf16x8 ww = widen(whole(f.w[c][0], f.w[c][1]), q, scale_value(f.s[c]));
#pragma unroll
                            for (int m = 0; m < MR; ++m) acc[m][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ww, aw[m], acc[m][c], 0, 0, 0);
                        }
                    }
                };
                // the ring's places are compile-time: a switch into the unrolled loop where a pass begins in its middle
                while (b < b1 - b0) {
#pragma unroll
                    for (int j = 0; j < P; ++j)
                        if (slot == j && b < b1 - b0) {
                            multiply(raw[j]);
                            load(raw[j]);
                            b += KS;
                            slot = (j + 1) % P;
                        }
                }
            }
            // ---- join and store: lane r holds columns 4 part .. of row r
            if constexpr (KS > 1) {
                __syncthreads();
                if (kw > 0)
#pragma unroll
                    for (int m = 0; m < MR; ++m)
#pragma unroll
                        for (int c = 0; c < NC; ++c)
                            *reinterpret_cast<f32x4 *>(join + (((cw * (KS - 1) + kw - 1) * MR + m) * NC + c) * 256 + lane * 4) = acc[m][c];
                __syncthreads();
                if (kw == 0)
#pragma unroll
                    for (int m = 0; m < MR; ++m)
#pragma unroll
                        for (int c = 0; c < NC; ++c)
                            for (int x = 0; x < KS - 1; ++x)
                                acc[m][c] += *reinterpret_cast<const f32x4 *>(join + (((cw * (KS - 1) + x) * MR + m) * NC + c) * 256 + lane * 4);
                if (kw > 0) continue;
            }
            if (group >= groups) continue;
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                const int row = 16 * m + r;
                if (row >= rows) continue;
#pragma unroll
                for (int c = 0; c < (ACT == kActSilu ? 1 : NC); ++c) {
                    const int col = group * COLS + c * 16 + part * 4;
                    if (col >= g.Nh) continue;  // a multiple of 8
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = ACT == kActSilu ? silu<A == kRowsF32>(acc[m][0][j]) * acc[m][1][j] : ACT == kActRelu ? relu(acc[m][c][j]) : acc[m][c][j];
                    const int64_t at = (int64_t)(row0 + row) * g.Nh + col;
                    if (g.c_dtype == MOE_DTYPE_F32) *reinterpret_cast<float4 *>(static_cast<float *>(g.c) + at) = make_float4(v[0], v[1], v[2], v[3]);
                    else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(g.c) + at) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
                }
            }
        }
    }
}

template <int A, int ACT, int KS>
__global__ __launch_bounds__(kThreads, 4) void gemm_b128_stream_kernel(GemmB128 g)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const ExpertRows rows_of = expert_rows(g, blockIdx.y, gridDim.y);
    const int e = rows_of.expert, first = rows_of.first, end = rows_of.end;
    if (e < 0) return;
    for (int row0 = first + blockIdx.z * 32; row0 < end; row0 += gridDim.z * 32) {
        const int rows = min(end - row0, 32);
        if (rows <= 16) stream_rows<A, ACT, 1, KS>(g, smem, e, row0, rows);
        else stream_rows<A, ACT, 2, KS>(g, smem, e, row0, rows);
    }
}

// LDS of 16 MR rows
size_t stream_lds(int mr, int K, int ks)
{
    const int blocks = ceil_div(K < held_k(mr) ? K : held_k(mr), kBlock);
    return 16 * mr * (blocks * kBlock + kRowPad) + align_up(blocks * 16 * mr, 16) + (ks > 1 ? NW / ks * (ks - 1) * mr * NC * 1024 : 0);
}

template <int A, int ACT, int KS>
int launch_ks(const GemmB128 &g, hipStream_t s)
{
    constexpr int COLS = ACT == kActSilu ? 16 : 32, CW = NW / KS;
    const size_t one = stream_lds(1, g.K, KS), two = stream_lds(2, g.K, KS), smem = one > two ? one : two;
    auto kern = gemm_b128_stream_kernel<A, ACT, KS>;
    static std::once_flag once;  // per instantiation
    static hipError_t setup_rc = hipSuccess;
    std::call_once(once, [&]() { setup_rc = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024); });
    MOE_HIP_CHECK(setup_rc);
    const int across = ceil_div(ceil_div(g.Nh, COLS), CW), per = ceil_div(g.n_rows, g.E * 32);
    const dim3 grid(across < 4096 ? across : 4096, g.E < g.n_rows ? g.E : g.n_rows, per < 64 ? per : 64);
    hipLaunchKernelGGL(kern, grid, dim3(kThreads), smem, s, g);
    MOE_LAUNCH_CHECK("gemm_b128_stream_kernel");
    return MOE_OK;
}

template <int A, int ACT>
int launch_as(const GemmB128 &g, hipStream_t s)
{
    constexpr int COLS = ACT == kActSilu ? 16 : 32;
    // waves that read weights, one for each group of rows, as far as the host knows; a CU runs 16
    const int64_t groups = (int64_t)(g.E < g.n_rows ? g.E : g.n_rows) * ceil_div(g.Nh, COLS);
    if (groups >= 4096) return launch_ks<A, ACT, 1>(g, s);
    if (groups >= 2048) return launch_ks<A, ACT, 2>(g, s);
    if (groups >= 1024) return launch_ks<A, ACT, 4>(g, s);
    return launch_ks<A, ACT, 8>(g, s);
}

}  // namespace

// Up to so many rows an expert on average the feed-forward's two products run here, beyond them in tiles.  Stream / tiles, us, at 4, 8 and 16 rows: 128 experts
// 2048 -> 2 x 1024 -> 2048 172 / 203, 209 / 213, 268 / 224; 32 experts 4096 -> 2 x 2048 182 / 205, --, 267 / 214; 16 experts 2048 -> 2 x 8192 170 / 220 (2 rows),
// 208 / 229, 253 / 233; 64 experts 512 -> 2 x 512 19 / 29 (2 rows), 32 / 31, 46 / 32.
int64_t b128_few_rows_most(int E) { return 8 * (int64_t)E; }
bool b128_few_rows(int n_rows, int E) { return n_rows <= b128_few_rows_most(E); }

int launch_gemm_b128_stream(const GemmB128 &g, hipStream_t s)
{
    ProfScope ps(g.name ? g.name : "gemm_b128", s);
    if (g.rows == kRowsBf16) return g.act == kActSilu ? launch_as<kRowsBf16, kActSilu>(g, s) : launch_as<kRowsBf16, kActRelu>(g, s);
    if (g.act == kActNone) return launch_as<kRowsF32, kActNone>(g, s);
    return g.act == kActSilu ? launch_as<kRowsF32, kActSilu>(g, s) : launch_as<kRowsF32, kActRelu>(g, s);
}

}  // namespace moe355
