// Products of e4m3 operands in blocks of 128 where whole tiles would leave most CUs without work.
//
// A block takes 16 MR rows by 32 weight rows of an expert; its 8 waves share the blocks of k (wave w takes w, w + 8, ...), read both operands from memory
// (which for sizes like these is the L2) straight into registers, a block of k ahead, and work alone until one join in LDS.  What bounds it is
// latency: a wave has two to eight blocks of k, one after the other.
// Fragments: lane l holds bytes 16 (l / 16) and 64 + 16 (l / 16) of row l % 16's 128; either operand's k lie in that order.  Fast and precise: as in
// gemm_b128_tile.hip, with the instructions for 16 x 16.
#include "b128_dev.h"

namespace moe355 {

namespace {

constexpr int NW = 8, kThreads = NW * 64, NC = 2, COLS = NC * 16, LD = COLS + 4;

template <bool PRECISE, int MR>
__global__ __launch_bounds__(kThreads) void gemm_b128_small_kernel(GemmB128 g)
{
    __shared__ __align__(16) float join[NW * 16 * LD];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, part = lane >> 4;
    const int K = g.K, KB = ceil_div(K, kBlock), scale_cols = (int)b128_scale_cols(K), n_blocks = ceil_div(g.N, kBlock);
    const int n0 = blockIdx.x * COLS;
    const ExpertRows rows_of = expert_rows(g, blockIdx.y, gridDim.y);
    const int e = rows_of.expert, first = rows_of.first, end = rows_of.end;
    if (e < 0) return;
    for (int row0 = first + blockIdx.z * 16 * MR; row0 < end; row0 += gridDim.z * 16 * MR) {
        // rows that are not there repeat the last one, of either operand; what comes of them is not stored
        const uint8_t *w[NC], *a[MR], *as[MR];
#pragma unroll
        for (int c = 0; c < NC; ++c) w[c] = g.w + ((int64_t)e * g.N + min(n0 + c * 16 + r, g.N - 1)) * K + part * 16;
        const uint8_t *const ws = g.w_scale + ((int64_t)e * n_blocks + n0 / kBlock) * scale_cols;  // 32 weight rows lie in one block
#pragma unroll
        for (int m = 0; m < MR; ++m) {
            int at = min(row0 + 16 * m + r, end - 1);
            if (g.a_rows) at = min(max(g.a_rows[at], 0), g.a_count - 1);
            a[m] = g.a + (int64_t)at * K + part * 16;
            as[m] = g.a_scale + (int64_t)at * scale_cols;
        }
        struct Raw {
            Fragment w[NC], a[MR];
            int ws, as[MR];
        };
        auto load = [&](Raw &f, int b) __attribute__((always_inline)) {
            const int k = b * kBlock;
            f.ws = ws[b];
#pragma unroll
            for (int m = 0; m < MR; ++m) f.as[m] = as[m][b];
            if (k + kBlock <= K) {
#pragma unroll
                for (int c = 0; c < NC; ++c) f.w[c] = load_fragment(w[c] + k, 0, kBlock);
#pragma unroll
                for (int m = 0; m < MR; ++m) f.a[m] = load_fragment(a[m] + k, 0, kBlock);
            } else {  // the last block of k may be short: zeros
#pragma unroll
                for (int c = 0; c < NC; ++c) f.w[c] = load_fragment(w[c] + k, part * 16, K - k);
#pragma unroll
                for (int m = 0; m < MR; ++m) f.a[m] = load_fragment(a[m] + k, part * 16, K - k);
            }
        };
        f32x4 acc[MR][NC] = {};
        auto multiply = [&](const Raw &f) __attribute__((always_inline)) {
            if constexpr (PRECISE) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    bf16x8 ww[NC];
#pragma unroll
                    for (int c = 0; c < NC; ++c) ww[c] = widen(f.w[c], q, scale_value(f.ws));
#pragma unroll
                    for (int m = 0; m < MR; ++m) {
                        const bf16x8 aw = widen(f.a[m], q, scale_value(f.as[m]));
#pragma unroll
                        for (int c = 0; c < NC; ++c) acc[m][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ww[c], aw, acc[m][c], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int m = 0; m < MR; ++m)
#pragma unroll
                    for (int c = 0; c < NC; ++c) acc[m][c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(f.w[c], f.a[m], acc[m][c], 0, 0, 0, f.ws, 0, f.as[m]);
            }
        };
        int b = wave;
        if constexpr (MR < 4) {
            Raw f[2];
            if (b < KB) load(f[0], b);
            while (b < KB) {
                if (b + NW < KB) load(f[1], b + NW);
                multiply(f[0]);
                b += NW;
                if (b >= KB) break;
                if (b + NW < KB) load(f[0], b + NW);
                multiply(f[1]);
                b += NW;
            }
        } else {  // two blocks of k do not fit the registers beside the sums: 64 rows, 2048 -> 8192 13.1 us with them, 11.5 without (precise 17.4, 12.3)
            for (; b < KB; b += NW) {
                Raw f;
                load(f, b);
                multiply(f);
            }
        }
        const int waves = min(NW, KB);  // the others have nothing to add
#pragma unroll
        for (int m = 0; m < MR; ++m) {
            if (row0 + 16 * m >= end) break;
            __syncthreads();
#pragma unroll
            for (int c = 0; c < NC; ++c) *reinterpret_cast<f32x4 *>(join + (wave * 16 + r) * LD + c * 16 + part * 4) = acc[m][c];
            __syncthreads();
            if (tid < 16 * COLS / 4) {  // four columns a thread; N is a multiple of 8
                const int row = tid / (COLS / 4), col = tid % (COLS / 4) * 4;
                if (row0 + 16 * m + row < end && n0 + col < g.N) {
                    f32x4 v = {0.f, 0.f, 0.f, 0.f};
                    for (int x = 0; x < waves; ++x) v += *reinterpret_cast<const f32x4 *>(join + (x * 16 + row) * LD + col);
                    const int64_t at = (int64_t)(row0 + 16 * m + row) * g.N + n0 + col;
                    if (g.c_dtype == MOE_DTYPE_F32) *reinterpret_cast<f32x4 *>(static_cast<float *>(g.c) + at) = v;
                    else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(g.c) + at) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
                }
            }
        }
    }
}

template <bool PRECISE, int MR>
int launch_rows(const GemmB128 &g, hipStream_t s)
{
    const int per = ceil_div(g.n_rows, g.E * 16 * MR);
    const dim3 grid(ceil_div(g.N, COLS), g.E < g.n_rows ? g.E : g.n_rows, per < 64 ? per : 64);
    hipLaunchKernelGGL((gemm_b128_small_kernel<PRECISE, MR>), grid, dim3(kThreads), 0, s, g);
    MOE_LAUNCH_CHECK("gemm_b128_small_kernel");
    return MOE_OK;
}

// What a call takes at 16 mr rows a block, estimated in units of 50 ns: rounds of blocks, each with a beginning and an end and its waves' blocks of k.
int64_t small_time(const GemmB128 &g, int mr)
{
    static const int kIteration[2][3] = {{32, 48, 80}, {34, 50, 84}};
    const int64_t active = g.E < g.n_rows ? g.E : g.n_rows, rows = (g.n_rows + active - 1) / active;
    constexpr int resident = 256;  // where a CU has two, as it can of 16 rows, each takes twice as long (64 to 96 rows, 8192 -> 2048: 16 -> 28 us)
    const int64_t blocks = active * ceil_div(g.N, COLS) * ((rows + 16 * mr - 1) / (16 * mr));
    return (blocks + resident - 1) / resident * (40 + (int64_t)ceil_div(ceil_div(g.K, kBlock), NW) * kIteration[g.precise][mr == 4 ? 2 : mr - 1]);
}

// Few columns: more blocks of fewer rows, which read the same weights out of L2.
int best_rows(const GemmB128 &g)
{
    int best = 4;
    for (int mr = 2; mr >= 1; --mr)
        if (small_time(g, mr) < small_time(g, best)) best = mr;
    return best;
}

}  // namespace

int launch_gemm_b128_small(const GemmB128 &g, hipStream_t s)
{
    ProfScope ps(g.name ? g.name : "gemm_b128", s);
    switch (best_rows(g)) {
    case 1: return g.precise ? launch_rows<true, 1>(g, s) : launch_rows<false, 1>(g, s);
    case 2: return g.precise ? launch_rows<true, 2>(g, s) : launch_rows<false, 2>(g, s);
    default: return g.precise ? launch_rows<true, 4>(g, s) : launch_rows<false, 4>(g, s);
    }
}

// Which of the two takes less, estimated in units of 50 ns.  Here: rounds of blocks, each with a beginning and an end and its waves' blocks of k.  Tiles: rounds of
// tiles, of the height that suits best.  Measured, small / tiles, us, bf16 results: one expert 2048 -> 8192, 16 rows 6.4 / 19, 64 rows 11 / 20, 128 rows 20 / 21.5,
// 192 rows 29 / 21; 8192 -> 2048, 64 to 256 rows 33 / 58 to 62, 512 rows 63 / 62; 8 experts of 16 rows, 2048 -> 8192 38 / 28, 8192 -> 2048 47 / 70, of 48 rows
// 58 / 76 (taken for 64, which have as many rounds of blocks: 91 / 77), of 96 113 / 81; 64 experts of 16 rows, 512 -> 4096 49 / 31.  fp32 results: 128 rows, 2048 -> 8192
// 21 / 28; 512 rows, 8192 -> 2048 65 / 82; 8 experts of 64 rows, 8192 -> 2048 92 / 107.
static bool small_pays(const GemmB128 &g)
{
    const int64_t active = g.E < g.n_rows ? g.E : g.n_rows, rows = (g.n_rows + active - 1) / active;
    const int KT = ceil_div(g.K, kBlock);
    const int64_t here = small_time(g, best_rows(g));
    int64_t there = INT64_MAX;
    for (int h = 1; h <= 4; ++h) {
        const int64_t tiles = active * ceil_div((int)((rows + 63) / 64), h) * ceil_div(g.N, 256);
        const int64_t t = (tiles + 255) / 256 * ((KT + 9) * (int64_t)kTileTime[g.precise][h - 1]);
        if (t < there) there = t;
    }
    return here <= there;
}

int launch_gemm_b128(const GemmB128 &g, hipStream_t s) { return !b128_tiles_ok(g) || small_pays(g) ? launch_gemm_b128_small(g, s) : launch_gemm_b128_tile(g, s); }

}  // namespace moe355
