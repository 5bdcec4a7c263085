// Products of e4m3 operands in blocks of 128 where whole tiles would leave most CUs without work.
//
// A block takes 16 MR rows by 16 or 32 weight rows of an expert; its 8 waves share the blocks of k (wave w takes w, w + 8, ...), read both operands from memory
// (which for sizes like these is the L2) straight into registers, up to P blocks of k at once, and work alone until one join in LDS.  What bounds it: latency, where
// a wave has two blocks of k (17 rows, 2048 -> 8192: 7.5 us), and else what one CU can have on its way, about 20 bytes a ns; so that more and smaller blocks pay until every CU has
// one (8192 -> 2048: 16 rows by 32 / by 16 columns 15.3 / 11.8 us; 64 rows in blocks of 64 / of 16 33 / 16 us).
// Fragments: lane l holds bytes 16 (l / 16) and 64 + 16 (l / 16) of row l % 16's 128; either operand's k lie in that order.  Fast and precise: as in
// gemm_b128_tile.hip, with the instructions for 16 x 16.
#include "b128_dev.h"

namespace moe355 {

namespace {

constexpr int NW = 8, kThreads = NW * 64;

// NC: blocks of 16 weight rows
template <bool PRECISE, int MR, int NC>
__global__ __launch_bounds__(kThreads) void gemm_b128_small_kernel(GemmB128 g)
{
    constexpr int COLS = NC * 16, LD = COLS + 4;
    // blocks of k that a wave has at once
    constexpr int P = MR == 1 ? 4 : MR == 2 ? 2 : 1;
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
        const uint8_t *const ws = g.w_scale + ((int64_t)e * n_blocks + n0 / kBlock) * scale_cols;  // 32 neighbouring weight rows lie in one block
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
        Raw f[P];
#pragma unroll
        for (int j = 0; j + 1 < P; ++j)
            if (wave + j * NW < KB) load(f[j], wave + j * NW);
        for (int b = wave; b < KB;) {
#pragma unroll
            for (int j = 0; j < P; ++j) {
                if (b + (P - 1) * NW < KB) load(f[(j + P - 1) % P], b + (P - 1) * NW);
                multiply(f[j]);
                b += NW;
                if (b >= KB) break;
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

template <bool PRECISE, int MR, int NC>
int launch_as(const GemmB128 &g, hipStream_t s)
{
    const int per = ceil_div(g.n_rows, g.E * 16 * MR);
    const dim3 grid(ceil_div(g.N, NC * 16), g.E < g.n_rows ? g.E : g.n_rows, per < 64 ? per : 64);
    hipLaunchKernelGGL((gemm_b128_small_kernel<PRECISE, MR, NC>), grid, dim3(kThreads), 0, s, g);
    MOE_LAUNCH_CHECK("gemm_b128_small_kernel");
    return MOE_OK;
}

struct Shape {
    int mr, nc;
    int64_t time;
};
// The rows and columns of a block that take least, estimated in units of 50 ns: rounds of blocks, each with a beginning and an end and its waves' blocks of k, which cost about
// what they load.  Few columns: more blocks, of fewer rows or columns; those that read the same weights find them in the L2.  A CU runs one block a round: where it has two, as it
// can of 16 rows, each takes twice as long (64 and 96 rows, 8192 -> 2048: 16 and 28 us).
Shape best_shape(const GemmB128 &g)
{
    static const struct { int mr, nc, iteration[2]; } kShapes[] = {{4, 2, {80, 84}}, {2, 2, {48, 50}}, {1, 2, {32, 34}}, {1, 1, {22, 24}}};
    const int64_t active = g.E < g.n_rows ? g.E : g.n_rows, rows = (g.n_rows + active - 1) / active;
    Shape best = {0, 0, INT64_MAX};
    for (const auto &k : kShapes) {
        const int64_t blocks = active * ceil_div(g.N, k.nc * 16) * ((rows + 16 * k.mr - 1) / (16 * k.mr));
        const int64_t t = (blocks + 255) / 256 * (40 + (int64_t)ceil_div(ceil_div(g.K, kBlock), NW) * k.iteration[g.precise]);
        if (t < best.time) best = {k.mr, k.nc, t};
    }
    return best;
}

template <bool PRECISE>
int launch_shape(const GemmB128 &g, const Shape &shape, hipStream_t s)
{
    if (shape.nc == 1) return launch_as<PRECISE, 1, 1>(g, s);
    return shape.mr == 1 ? launch_as<PRECISE, 1, 2>(g, s) : shape.mr == 2 ? launch_as<PRECISE, 2, 2>(g, s) : launch_as<PRECISE, 4, 2>(g, s);
}

}  // namespace

int launch_gemm_b128_small(const GemmB128 &g, hipStream_t s)
{
    ProfScope ps(g.name ? g.name : "gemm_b128", s);
    return g.precise ? launch_shape<true>(g, best_shape(g), s) : launch_shape<false>(g, best_shape(g), s);
}

// Which of the two takes less, this or tiles: rounds of tiles, of the height that suits best, each as long as nine K tiles more than it has (six for a tile's beginning and
// end, as in gemm_b128_tile.hip, and three for the rest of a launch).  Measured, small / tiles, us, bf16 results: one expert 2048 -> 8192,
// 16 rows 6.2 / 19, 64 rows 11 / 20, 128 rows 20 / 21.5, 192 rows 29 / 21; 8192 -> 2048, 16 rows 11.8 / 56, 64 rows 16 / 58, 256 rows 33 / 62, 512 rows 63 / 62; 8 experts of
// 16 rows, 2048 -> 8192 38 / 28, 8192 -> 2048 44 / 70, of 48 rows 58 / 76 (tiles are taken), of 64 rows 91 / 77; 64 experts of 16 rows, 512 -> 4096 49 / 31.
// fp32 results: 128 rows, 2048 -> 8192 21 / 28; 512 rows, 8192 -> 2048 65 / 82; 8 experts of 64 rows, 8192 -> 2048 92 / 107.
static bool small_pays(const GemmB128 &g)
{
    const int64_t active = g.E < g.n_rows ? g.E : g.n_rows, rows = (g.n_rows + active - 1) / active;
    const int KT = ceil_div(g.K, kBlock);
    const int64_t here = best_shape(g).time;
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
