// C = A W[e]^T for e4m3 operands with a scale 2^(byte - 127) per row and block of 128 k (A) and per 128 x 128 (W), fp32 sums.
//
// The scaled MFMA 16x16x128 takes a scale byte for every 32 k of each row of either operand, so a block of 128 k is one MFMA and its
// scales cost nothing.  What it computes: products exactly, but among 8 neighbouring k it aligns them to the largest and drops what lies
// 2^-14 below that; between those groups and with the accumulator it is fp32.  On normally distributed operands its results are off by 1.4e-5
// of their standard deviation (measured against 64 bits; the unscaled fp8 MFMA is the same), where rounding them to bf16 is off by 1.7e-3.
// That is why it serves bf16 results; fp32 results widen both operands to bf16, which holds e4m3 numbers times powers of two, and take
// the bf16 MFMA, whose sums are fp32 throughout.
#include "b128_dev.h"
#include "gemm_bf16_dev.h"

namespace moe355 {

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kThreads = 256;

struct RowTile {
    int expert, row0, row_end;
};

// Tile `index` among all experts' row tiles of `height` rows, in order; expert -1 behind the last one.  A wave's lanes look at 64 experts at a time.
__device__ __forceinline__ RowTile find_tile(const int32_t *offsets, int E, int n_rows, int height, int index)
{
    const int lane = threadIdx.x & 63;
    if (!offsets) {
        const int row0 = index * height;
        return row0 < n_rows ? RowTile{0, row0, min(n_rows, row0 + height)} : RowTile{-1, 0, 0};
    }
    for (int base = 0; base < E; base += 64) {
        int first = 0, end = 0;
        if (base + lane < E) {
            first = min(max(offsets[base + lane], 0), n_rows);
            end = min(max(offsets[base + lane + 1], first), n_rows);
        }
        const int tiles = (end - first + height - 1) / height;
        int incl = tiles;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int up = __shfl_up(incl, off, 64);
            if (lane >= off) incl += up;
        }
        const int total = __builtin_amdgcn_readlane(incl, 63);
        if (index < total) {
            const int src = __builtin_ctzll(__ballot(incl > index));
            const int row0 = __builtin_amdgcn_readlane(first, src) + (index - __builtin_amdgcn_readlane(incl - tiles, src)) * height;
            return RowTile{base + src, row0, min(__builtin_amdgcn_readlane(end, src), row0 + height)};
        }
        index -= total;
    }
    return RowTile{-1, 0, 0};
}

__device__ __forceinline__ i32x8 load_fragment(const uint8_t *row, int k, int K, bool live)
{
    // a lane's 32 bytes of a block: 16 at k and 16 at k + 64; either operand's k lie in the same order
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    if (live && k < K) lo = *reinterpret_cast<const uint4 *>(row + k);
    if (live && k + 64 < K) hi = *reinterpret_cast<const uint4 *>(row + k + 64);
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}

__device__ __forceinline__ bf16x8 widen(const i32x8 &f, int q, float scale)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        w[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * q + i], scale, false));
        w[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * q + i], scale, true));
    }
    return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ float scale_value(int byte) { return byte ? __uint_as_float((uint32_t)byte << 23) : __uint_as_float(1u << 22); }

constexpr int kRows = 64;

// A block: 64 rows x 64 columns, a wave 16 columns of them, fragments straight from memory.
template <bool PRECISE>
__global__ __launch_bounds__(kThreads) void gemm_b128_kernel(GemmB128 g)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, part = lane >> 4;
    const int64_t scale_cols = b128_scale_cols(g.K);
    for (int index = blockIdx.y;; index += gridDim.y) {
        const RowTile t = find_tile(g.offsets, g.E, g.n_rows, kRows, index);
        if (t.expert < 0) return;
        for (int n0 = blockIdx.x * 64 + wave * 16; n0 < g.N; n0 += gridDim.x * 64) {
            const bool n_live = n0 + r < g.N;
            const uint8_t *w = g.w + ((int64_t)t.expert * g.N + (n_live ? n0 + r : 0)) * g.K;
            const uint8_t *ws = g.w_scale + ((int64_t)t.expert * (g.N / g.Nh) * ceil_div(g.Nh, kBlock) + n0 / g.Nh * ceil_div(g.Nh, kBlock) + n0 % g.Nh / kBlock) * scale_cols;
            const uint8_t *a[4], *as[4];
            bool m_live[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int m = t.row0 + 16 * i + r;
                m_live[i] = m < t.row_end;
                int at = m_live[i] ? m : t.row0;
                if (g.a_rows) at = min(max(g.a_rows[at], 0), g.a_count - 1);
                a[i] = g.a + (int64_t)at * g.K;
                as[i] = g.a_scale + (int64_t)at * scale_cols;
            }
            f32x4 acc[4] = {};
            for (int b = 0; b * kBlock < g.K; ++b) {
                const int k = b * kBlock + part * 16;
                const i32x8 wf = load_fragment(w, k, g.K, n_live);
                const int wsc = ws[b];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const i32x8 af = load_fragment(a[i], k, g.K, m_live[i]);
                    if constexpr (PRECISE) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(wf, q, scale_value(wsc)), widen(af, q, scale_value(as[i][b])), acc[i], 0, 0, 0);
                    } else {
                        acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf, af, acc[i], 0, 0, 0, wsc, 0, as[i][b]);
                    }
                }
            }
            const int col = n0 + part * 4;
            if (col >= g.N) continue;  // N is a multiple of 8
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!m_live[i]) continue;
                const int64_t at = (int64_t)(t.row0 + 16 * i + r) * g.N + col;
                if (g.c_dtype == MOE_DTYPE_F32)
                    *reinterpret_cast<float4 *>(static_cast<float *>(g.c) + at) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
                else
                    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(g.c) + at) = make_uint2(pack_bf16(acc[i][0], acc[i][1]), pack_bf16(acc[i][2], acc[i][3]));
            }
        }
    }
}

}  // namespace

int launch_gemm_b128(const GemmB128 &g, hipStream_t s)
{
    if (g.n_rows == 0) return MOE_OK;
    ProfScope ps(g.name ? g.name : "gemm_b128", s);
    const int64_t tiles = (int64_t)g.n_rows / kRows + (g.offsets ? g.E : 0) + 1;
    const int columns = ceil_div(g.N, 64);
    const dim3 grid(columns < 1024 ? columns : 1024, (unsigned)(tiles < 8192 ? tiles : 8192));
    if (g.precise) hipLaunchKernelGGL(gemm_b128_kernel<true>, grid, dim3(kThreads), 0, s, g);
    else hipLaunchKernelGGL(gemm_b128_kernel<false>, grid, dim3(kThreads), 0, s, g);
    MOE_LAUNCH_CHECK("gemm_b128_kernel");
    return MOE_OK;
}

}  // namespace moe355
