// Attention over a paged e4m3 cache for few query rows per key head (decoder steps).
//
// The queries of a (sequence, key head) that are served together -- the heads of a group, the new tokens -- are the columns of
// 16-wide MFMA tiles; a wave walks tiles of kTile keys with a running maximum and sum (one pass over the cache), everything in
// registers:
//   scores  S^T = K Q^T    A = keys as they lie in the cache (16 rows x 64 bytes a load instruction), B = queries
//   output  O^T = V^T P^T  A = values (bytes of eight keys gathered with v_perm_b32), B = the weights where the first product left
//                          them: a lane of S^T holds keys 4g .. 4g+3 of a 16-key block for query column lane & 15, and the order of
//                          the keys inside a product is free, so no weight ever changes lanes.
// e4m3 bytes become bf16 exactly (v_cvt_scalef32_pk_bf16_fp8), keys' scales multiply the scores, values' scales the weights.
// fp32 queries and weights are three bf16 numbers each (8 bits of the mantissa a piece), one MFMA per piece: the bytes are bf16
// exactly, so nothing else is lost.
//
// Bound by HBM: 2 DH bytes a key, at 16 columns 32 MFMAs of 16 cycles per 16 KB and SIMD, far below.  Split: the tiles of all
// (sequence, rows, head) units lie in one row and every block takes the same number of them, whatever the lengths are; a unit
// that several blocks share leaves partial results that a second kernel joins.
#include "attn_dev.h"

namespace moe355 {

namespace {

static constexpr int kThreads = 256, kWaves = 4;

constexpr int tile_keys(int dh) { return dh <= 128 ? 64 : 32; }

// Tiles of a sequence's key range that any of its new tokens sees, and the first of them.  At least one tile where there are
// new tokens, so that every row is written.
__device__ __forceinline__ void seq_range(const AttnParams &p, const Seq &sq, int tile, int &first, int &count)
{
    int lo = 0;
    if (p.window > 0) lo = max(0, sq.kv - sq.n - p.window + 1);
    first = min(lo, sq.kv) / tile;
    count = max(1, ceil_div(sq.kv, tile) - first);
}

__device__ __forceinline__ int64_t seq_cost(const AttnParams &p, int b, int tile)
{
    const Seq sq = load_seq(p, b);
    if (sq.n == 0 || sq.n * p.group > p.few_rows) return 0;
    int first, count;
    seq_range(p, sq, tile, first, count);
    return (int64_t)count * ceil_div(sq.n * p.group, 16) * p.n_kv_heads;
}

// Exclusive prefix of the sequences' tiles into begin[0 .. B] (LDS).  All threads.
__device__ void scan_sequences(const AttnParams &p, int tile, int64_t *begin, int64_t *wave_sum)
{
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int64_t carry = 0;
    for (int base = 0; base < p.B; base += kThreads) {
        const int b = base + tid;
        const int64_t mine = b < p.B ? seq_cost(p, b, tile) : 0;
        int64_t sum = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int64_t other = __shfl_up(sum, off, 64);
            if (lane >= off) sum += other;
        }
        if (lane == 63) wave_sum[w] = sum;
        __syncthreads();
        int64_t before = carry;
        for (int i = 0; i < kWaves; ++i) {
            if (i < w) before += wave_sum[i];
            carry += wave_sum[i];
        }
        if (b < p.B) begin[b] = before + sum - mine;
        __syncthreads();
    }
    if (tid == 0) begin[p.B] = carry;
    __syncthreads();
}

// Tiles a block takes: equal parts of them all, at least one for each wave.
__device__ __forceinline__ int64_t tiles_per_block(int64_t total, int n_blocks)
{
    const int64_t per = (total + n_blocks - 1) / n_blocks;
    return max((int64_t)kWaves, (per + kWaves - 1) / kWaves * kWaves);
}

// A partial result: 16 rows of DH outputs (not divided by the sum), then the 16 maxima and the 16 sums
template <int DH>
constexpr int part_floats() { return 16 * DH + 32; }

template <int DH>
struct TileData {
    static constexpr int kBlocks = tile_keys(DH) / 16, kChunks = DH / 64, kWords = DH / 64;
    uint4 k[kBlocks][kChunks];
    uint32_t v[kBlocks][4][kWords];  // [block][i]: key 16 block + 4 g + i, DH/16 bytes from dimension DH/16 * (lane & 15)
    float ks[kBlocks], vs[kBlocks];
    bool held[kBlocks];              // the block's page exists
};

template <int DH>
__device__ __forceinline__ void load_tile(const AttnParams &p, const int32_t *table, int kv, int h, int key0, int lane, TileData<DH> &d)
{
    const int l15 = lane & 15, g = lane >> 4;
    const int page_mask = (1 << p.page_shift) - 1;
#pragma unroll
    for (int b = 0; b < TileData<DH>::kBlocks; ++b) {
        const int key = key0 + 16 * b;
        const int page = key < kv ? table[key >> p.page_shift] : -1;
        d.held[b] = page >= 0 && page < p.num_pages;
        const int64_t unit = (int64_t)(d.held[b] ? page : 0) * p.n_kv_heads + h;
        d.ks[b] = p.k_scale[unit];
        d.vs[b] = p.v_scale[unit];
        const int64_t at = ((unit << p.page_shift) + (key & page_mask)) * DH;
        const uint8_t *kp = p.k + at + l15 * DH + 16 * g, *vp = p.v + at + 4 * g * DH + (DH / 16) * l15;
#pragma unroll
        for (int c = 0; c < TileData<DH>::kChunks; ++c) d.k[b][c] = *reinterpret_cast<const uint4 *>(kp + 64 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (DH == 64) d.v[b][i][0] = *reinterpret_cast<const uint32_t *>(vp + i * DH);
            if (DH == 128) {
                const uint2 w = *reinterpret_cast<const uint2 *>(vp + i * DH);
                d.v[b][i][0] = w.x;
                d.v[b][i][DH / 64 - 1] = w.y;
            }
            if (DH == 256) {
                const uint4 w = *reinterpret_cast<const uint4 *>(vp + i * DH);
                d.v[b][i][0] = w.x;
                d.v[b][i][1 % (DH / 64)] = w.y;
                d.v[b][i][2 % (DH / 64)] = w.z;
                d.v[b][i][DH / 64 - 1] = w.w;
            }
        }
    }
}

// DH: head dimension; NS: bf16 pieces of an fp32 number (1: bf16 queries and weights rounded once)
template <int DH, int NS>
__global__ __launch_bounds__(kThreads, 2) void attn_decode_kernel(AttnParams p)
{
    static constexpr int kTile = tile_keys(DH), kBlocks = kTile / 16, kChunks = DH / 64, kCols = DH / 16, kWords = DH / 64;
    extern __shared__ __align__(16) uint8_t lds[];
    float *merge = reinterpret_cast<float *>(lds);                                       // [waves][16][DH]
    float *merge_m = merge + kWaves * 16 * DH, *merge_l = merge_m + kWaves * 16;           // [waves][16]
    int64_t *wave_sum = reinterpret_cast<int64_t *>(merge_l + kWaves * 16);                // [waves]
    int64_t *begin = wave_sum + kWaves;                                                    // [B + 1]
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, g = lane >> 4;

    scan_sequences(p, kTile, begin, wave_sum);
    const int64_t total = begin[p.B], per = tiles_per_block(total, p.n_blocks);
    if (blockIdx.x == 0 && p.seq_tiles)  // for the kernel that joins
        for (int b = tid; b <= p.B; b += kThreads) p.seq_tiles[b] = begin[b];
    const int64_t t_begin = (int64_t)blockIdx.x * per, t_end = min(total, t_begin + per);
    if (t_begin >= t_end) return;
    int b = 0;
    {   // the sequence that holds t_begin: the last one that begins at or before it
        int lo = 0, hi = p.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (begin[mid] <= t_begin) lo = mid;
            else hi = mid;
        }
        b = lo;
    }
    for (int64_t t = t_begin; t < t_end;) {
        while (begin[b + 1] <= t) ++b;
        const int bu = __builtin_amdgcn_readfirstlane(b);
        const Seq sq = load_seq(p, bu);
        int first, count;
        seq_range(p, sq, kTile, first, count);
        const int local = (int)(t - begin[bu]);
        const int unit = __builtin_amdgcn_readfirstlane(local / count), tile0 = __builtin_amdgcn_readfirstlane(local - unit * count);
        const int run = __builtin_amdgcn_readfirstlane((int)min(t_end - t, (int64_t)(count - tile0)));
        const int rt = unit / p.n_kv_heads, h = unit - rt * p.n_kv_heads;
        const int32_t *table = p.page_table + (int64_t)bu * p.max_pages;

        // this lane's query: row r of the sequence's n * group rows
        const int r = rt * 16 + l15;
        const int tok = r / p.group, head = h * p.group + (r - tok * p.group);
        const bool live = tok < sq.n;
        const int pos = sq.kv - sq.n + tok;
        const int key_end = !live ? 0 : p.causal ? min(pos + 1, sq.kv) : sq.kv;
        const int key_begin = p.window > 0 ? max(0, pos - p.window + 1) : 0;
        Pieces<NS> q[kChunks][2];
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int64_t at = (int64_t)(sq.first + tok) * p.q_stride + (int64_t)head * DH + 64 * c + 16 * g + 8 * half;
                if (NS == 1) {
                    uint4 x = make_uint4(0, 0, 0, 0);
                    if (live) x = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.q) + at);
                    q[c][half].x[0] = __builtin_bit_cast(bf16x8, x);
                } else {
                    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    if (live) {
                        const float4 lo = *reinterpret_cast<const float4 *>(static_cast<const float *>(p.q) + at);
                        const float4 hi = *reinterpret_cast<const float4 *>(static_cast<const float *>(p.q) + at + 4);
                        x[0] = lo.x, x[1] = lo.y, x[2] = lo.z, x[3] = lo.w, x[4] = hi.x, x[5] = hi.y, x[6] = hi.z, x[7] = hi.w;
                    }
                    q[c][half] = split<NS>(x);
                }
            }

        f32x4 o[kCols];
#pragma unroll
        for (int c = 0; c < kCols; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        // keys that every row of this wave sees, so tiles inside need no mask: the largest begin and the smallest end over the lanes
        int all_begin = live ? key_begin : 0, all_end = live ? key_end : 0x7fffffff;
#pragma unroll
        for (int off = 8; off >= 1; off >>= 1) {
            all_begin = max(all_begin, __shfl_xor(all_begin, off, 64));
            all_end = min(all_end, __shfl_xor(all_end, off, 64));
        }
        all_begin = __builtin_amdgcn_readfirstlane(all_begin);
        all_end = min(__builtin_amdgcn_readfirstlane(all_end), sq.kv);

        TileData<DH> d, next;
        int tile = tile0 + w;
        const int tile_end = tile0 + run;
        if (tile < tile_end) load_tile<DH>(p, table, sq.kv, h, (first + tile) * kTile, lane, next);
        for (; tile < tile_end; tile += kWaves) {
            d = next;
            const int key0 = (first + tile) * kTile;
            if (tile + kWaves < tile_end) load_tile<DH>(p, table, sq.kv, h, key0 + kWaves * kTile, lane, next);
            f32x4 s[kBlocks];
            bool whole = key0 >= all_begin && key0 + kTile <= all_end;
#pragma unroll
            for (int n = 0; n < kBlocks; ++n) {
                s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
                whole = whole && d.held[n];
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {
                    const bf16x8 lo = widen(d.k[n][c].x, d.k[n][c].y), hi = widen(d.k[n][c].z, d.k[n][c].w);
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, q[c][0].x[i], s[n], 0, 0, 0);
                        s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, q[c][1].x[i], s[n], 0, 0, 0);
                    }
                }
                const float scale = d.ks[n] * p.scale_log2e;
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][i] *= scale;
            }
            if (!whole) {
#pragma unroll
                for (int n = 0; n < kBlocks; ++n) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = key0 + 16 * n + 4 * g + i;
                        const bool sees = d.held[n] && key >= key_begin && key < key_end;
                        s[n][i] = sees ? s[n][i] : -INFINITY;
                        // bytes that nobody wrote may be NaN, which no weight of zero takes away
                        const bool there = d.held[n] && key < sq.kv;
#pragma unroll
                        for (int x = 0; x < kWords; ++x) d.v[n][i][x] = there ? d.v[n][i][x] : 0u;
                    }
                    d.vs[n] = d.held[n] ? d.vs[n] : 0.f;
                }
            }
            float top = s[0][0];
#pragma unroll
            for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[n][i]);
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float m_new = fmaxf(m, top);
            const float base = m_new == -INFINITY ? 0.f : m_new;  // a row that has seen nothing: every weight is 0
            const float alpha = __builtin_amdgcn_exp2f(m - base);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[c][i] *= alpha;
#pragma unroll
            for (int pair = 0; pair < kBlocks / 2; ++pair) {
                float weight[8];
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float e = __builtin_amdgcn_exp2f(s[2 * pair + half][i] - base);
                        l += e;
                        weight[4 * half + i] = e * d.vs[2 * pair + half];
                    }
                const Pieces<NS> wp = split<NS>(weight);
#pragma unroll
                for (int x = 0; x < kWords; ++x) {
                    uint32_t lo[4], hi[4];
                    transpose4(d.v[2 * pair][0][x], d.v[2 * pair][1][x], d.v[2 * pair][2][x], d.v[2 * pair][3][x], lo);
                    transpose4(d.v[2 * pair + 1][0][x], d.v[2 * pair + 1][1][x], d.v[2 * pair + 1][2][x], d.v[2 * pair + 1][3][x], hi);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const bf16x8 value = widen(lo[y], hi[y]);
#pragma unroll
                        for (int i = 0; i < NS; ++i) o[4 * x + y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value, wp.x[i], o[4 * x + y], 0, 0, 0);
                    }
                }
            }
        }
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);

        // join the waves: o[c][i] of a lane is dimension kCols * (4 g + i) + c of query row l15
        if (g == 0) {
            merge_m[w * 16 + l15] = m;
            merge_l[w * 16 + l15] = l;
        }
        __syncthreads();
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) top = fmaxf(top, merge_m[i * 16 + l15]);
        const float mine = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < kCols; c += 4)
                *reinterpret_cast<float4 *>(merge + (w * 16 + l15) * DH + kCols * (4 * g + i) + c) =
                    make_float4(o[c][i] * mine, o[c + 1][i] * mine, o[c + 2][i] * mine, o[c + 3][i] * mine);
        __syncthreads();
        const bool all = run == count;
        float *part = nullptr;
        if (!all) part = p.part + ((int64_t)blockIdx.x * 2 + (t == t_begin ? 0 : 1)) * part_floats<DH>();
        for (int e = tid * 4; e < 16 * DH; e += kThreads * 4) {
            const int row = e / DH, dim = e - row * DH;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const float4 x = *reinterpret_cast<const float4 *>(merge + (i * 16 + row) * DH + dim);
                sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
            }
            float row_top = -INFINITY, row_l = 0.f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) row_top = fmaxf(row_top, merge_m[i * 16 + row]);
#pragma unroll
            for (int i = 0; i < kWaves; ++i)
                row_l += merge_m[i * 16 + row] == -INFINITY ? 0.f : merge_l[i * 16 + row] * __builtin_amdgcn_exp2f(merge_m[i * 16 + row] - row_top);
            if (!all) {
                *reinterpret_cast<float4 *>(part + e) = sum;
                if (dim == 0) {
                    part[16 * DH + row] = row_top;
                    part[16 * DH + 16 + row] = row_l;
                }
                continue;
            }
            const int rr = rt * 16 + row, token = rr / p.group;
            if (token >= sq.n) continue;
            const int64_t at = (int64_t)(sq.first + token) * p.n_heads + h * p.group + (rr - token * p.group);
            const float inv = row_l > 0.f ? 1.f / row_l : 0.f;
            if (NS == 1)
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + at * DH + dim) =
                    make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
            else
                *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + at * DH + dim) =
                    make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
            if (dim == 0 && p.lse) p.lse[at] = row_l > 0.f ? row_top * kLn2 + logf(row_l) : -INFINITY;
        }
        __syncthreads();
        t += run;
    }
}

// Joins the partial results of the units that more than one block worked on.  A block per unit (x: unit of a sequence, y: sequence).
template <int DH, int NS>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnParams p)
{
    static constexpr int kTile = tile_keys(DH);
    const int b = blockIdx.y, unit = blockIdx.x, tid = threadIdx.x;
    const Seq sq = load_seq(p, b);
    if (sq.n == 0 || sq.n * p.group > p.few_rows || unit >= ceil_div(sq.n * p.group, 16) * p.n_kv_heads) return;
    int first, count;
    seq_range(p, sq, kTile, first, count);
    const int64_t per = tiles_per_block(p.seq_tiles[p.B], p.n_blocks);
    const int64_t t0 = p.seq_tiles[b] + (int64_t)unit * count, t1 = t0 + count;
    const int64_t b0 = t0 / per, b1 = (t1 - 1) / per;
    if (b0 == b1) return;
    const int rt = unit / p.n_kv_heads, h = unit - rt * p.n_kv_heads;
    for (int e = tid * 4; e < 16 * DH; e += kThreads * 4) {
        const int row = e / DH, dim = e - row * DH;
        const int rr = rt * 16 + row, token = rr / p.group;
        if (token >= sq.n) continue;
        float top = -INFINITY, l = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int64_t k = b0; k <= b1; ++k) {
            const float *part = p.part + (2 * k + (t0 > k * per ? 1 : 0)) * part_floats<DH>();
            const float pm = part[16 * DH + row], pl = part[16 * DH + 16 + row];
            const float4 x = *reinterpret_cast<const float4 *>(part + e);
            const float m_new = fmaxf(top, pm), base = m_new == -INFINITY ? 0.f : m_new;
            const float keep = __builtin_amdgcn_exp2f(top - base), add = __builtin_amdgcn_exp2f(pm - base);
            top = m_new;
            l = l * keep + pl * add;
            sum.x = sum.x * keep + x.x * add;
            sum.y = sum.y * keep + x.y * add;
            sum.z = sum.z * keep + x.z * add;
            sum.w = sum.w * keep + x.w * add;
        }
        const int64_t at = (int64_t)(sq.first + token) * p.n_heads + h * p.group + (rr - token * p.group);
        const float inv = l > 0.f ? 1.f / l : 0.f;
        if (NS == 1)
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + at * DH + dim) =
                make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
        else
            *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + at * DH + dim) = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
        if (dim == 0 && p.lse) p.lse[at] = l > 0.f ? top * kLn2 + logf(l) : -INFINITY;
    }
}

template <int DH, int NS>
int launch_as(const AttnParams &p, hipStream_t s)
{
    const size_t lds = (size_t)(kWaves * 16 * DH + 2 * kWaves * 16) * 4 + (kWaves + p.B + 1) * 8;
    if (lds > 64 * 1024)
        MOE_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(attn_decode_kernel<DH, NS>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    {
        ProfScope ps("attn_decode", s);
        hipLaunchKernelGGL((attn_decode_kernel<DH, NS>), dim3(p.n_blocks), dim3(kThreads), lds, s, p);
        MOE_LAUNCH_CHECK("attn_decode_kernel");
    }
    ProfScope ps("attn_join", s);
    const int units = ceil_div((int)((int64_t)p.max_q * p.group < p.few_rows ? (int64_t)p.max_q * p.group : p.few_rows), 16) * p.n_kv_heads;
    hipLaunchKernelGGL((attn_join_kernel<DH, NS>), dim3(units, p.B), dim3(kThreads), 0, s, p);
    MOE_LAUNCH_CHECK("attn_join_kernel");
    return MOE_OK;
}

int decode_blocks(int num_cus) { return 2 * num_cus; }

}  // namespace

// partial results of two units a block
int64_t attn_decode_workspace(int head_dim, int num_cus)
{
    return align_up((int64_t)decode_blocks(num_cus) * 2 * (16 * head_dim + 32) * 4, 256);
}

int launch_attn_decode(int dtype, int head_dim, AttnParams p, int num_cus, hipStream_t s)
{
    p.n_blocks = decode_blocks(num_cus);
    const bool bf = dtype == MOE_DTYPE_BF16;
    if (head_dim == 64) return bf ? launch_as<64, 1>(p, s) : launch_as<64, 3>(p, s);
    if (head_dim == 128) return bf ? launch_as<128, 1>(p, s) : launch_as<128, 3>(p, s);
    return bf ? launch_as<256, 1>(p, s) : launch_as<256, 3>(p, s);
}

}  // namespace moe355
