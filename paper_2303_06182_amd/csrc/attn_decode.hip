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
// exactly, so nothing else is lost.  With bf16 queries a weight is rounded once to bf16, 2^-9 of it, and the sum has it unrounded; weights are relative to
// the row's largest so far, which is 1 and rounds to itself.  Outputs are then off by 1.8e-3 where fp32 weights, rounded to bf16 at the output alone, give
// 1.6e-3 (64 sequences of up to 16384 keys; with two bf16 numbers for a weight 44.2 us there, with one 43.3).
//
// Bound by HBM: 2 DH bytes a key, at 16 columns 32 MFMAs of 16 cycles per 16 KB and SIMD, far below; short calls by latency.  Split: where
// the units (sequence, 16 rows, key head) are short, a block a unit and each wave an equal part of its tiles, joined in LDS.  Else the tiles of all
// units lie in one row; every block takes the same number of them, whatever the lengths are, and every wave
// a quarter of the block's.  A wave works alone until its tiles are done: units that lie inside its part are written at once, the one
// or two that do not are left in LDS, where the block joins them; what reaches past the block is joined by a second kernel.
// (With the waves of a block on one unit at a time, joined after each, short sequences cost a block 8 us a unit: 32 sequences of up to
// 1111 keys, 16 heads of 64, fp32 41 us.)
// Measured: 64 sequences of up to 16384 keys, 32 heads over 4 of 128, 116 MB: 31 us, 3.7 TB/s (a kernel that only sums reads 4.0), and 6 to join.
#include "attn_dev.h"

#include <mutex>

namespace moe355 {

namespace {

static constexpr int kThreads = 256, kWaves = 4;

constexpr int tile_keys(int dh) { return dh <= 128 ? 64 : 32; }

// Tiles of a sequence's key range that any of its new tokens sees, and the first of them.  At least one tile where there are
// new tokens, so that every row is written.
__device__ __forceinline__ void seq_range(const AttnParams &p, const Seq &sq, int tile, int &first, int &count)
{
    int lo = 0;
    if (p.window > 0) lo = max(0, sq.begin - p.window + 1);
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
template <int W>
__device__ void scan_sequences(const AttnParams &p, int tile, int64_t *begin, int64_t *wave_sum)
{
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int64_t carry = 0;
    for (int base = 0; base < p.B; base += 64 * W) {
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
        for (int i = 0; i < W; ++i) {
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

// What a wave (or a block, in memory) has of a unit that it shares: 16 rows of DH outputs (not divided by the sum), the 16 maxima, the 16
// sums.  In LDS the rows are 4 floats further apart, so that the 16 lanes that write a dimension each meet other banks.
struct Piece {
    int64_t unit_begin;  // first tile of the unit, -1: nothing here
    int b, unit, run, count;
};
template <int DH, int W>
struct Shared {
    static constexpr int kRow = DH + 4;
    Piece piece[W][2];
    float m[W][2][16], l[W][2][16];
    int64_t wave_sum[W];
    float o[W][2][16 * kRow];
};

// four outputs of a row, from dimension dim on
template <int NS>
__device__ __forceinline__ void store_out(const AttnParams &p, int64_t at, float4 x)
{
    if (NS == 1)
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + at) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
    else
        *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + at) = x;
}

// The unit `unit` of a sequence: its rows' tile and its key head; a row's output begins at element row_out() * DH, -1: there is no such row
__device__ __forceinline__ int64_t row_out(const AttnParams &p, const Seq &sq, int unit, int row)
{
    const int rt = unit / p.n_kv_heads, h = unit - rt * p.n_kv_heads;
    const int r = rt * 16 + row, tok = r / p.group;
    return tok < sq.n ? (int64_t)(sq.first + tok) * p.n_heads + h * p.group + (r - tok * p.group) : -1;
}

// DH: head dimension; NS: bf16 pieces of an fp32 number (1: bf16 queries and weights rounded once); M: blocks a CU holds; W: waves.
// WHOLE: a block takes a whole unit
template <int DH, int NS, int M, int W, bool WHOLE>
__global__ __launch_bounds__(64 * W, M) void attn_decode_kernel(AttnParams p)
{
    static constexpr int kTile = tile_keys(DH), kBlocks = kTile / 16, kChunks = DH / 64, kCols = DH / 16, kWords = DH / 64;
    static constexpr int kRow = Shared<DH, W>::kRow;
    extern __shared__ __align__(16) uint8_t lds[];
    Shared<DH, W> &sh = *reinterpret_cast<Shared<DH, W> *>(lds);
    int64_t *begin = reinterpret_cast<int64_t *>(lds + sizeof(Shared<DH, W>));  // [B + 1]
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l15 = lane & 15, g = lane >> 4;

    if (tid < 2 * W) sh.piece[tid >> 1][tid & 1].unit_begin = -1;
    // this block's unit, or its part of the tiles and this wave's of it
    int64_t t_begin = 0, w_begin = 0, w_end = 1;
    int b = WHOLE ? (int)blockIdx.x / p.units : 0;
    if (!WHOLE) {
        scan_sequences<W>(p, kTile, begin, sh.wave_sum);
        const int64_t total = begin[p.B], per = tiles_per_block(total, p.n_blocks);
        if (blockIdx.x == 0)  // for the kernel that joins
            for (int i = tid; i <= p.B; i += 64 * W) p.seq_tiles[i] = begin[i];
        t_begin = (int64_t)blockIdx.x * per;
        const int64_t t_end = min(total, t_begin + per);
        if (t_begin >= t_end) return;
        w_begin = t_begin + w * (per / W), w_end = min(t_end, w_begin + per / W);
    }
    if (!WHOLE && w_begin < w_end) {  // the sequence that holds w_begin: the last one that begins at or before it
        int lo = 0, hi = p.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (begin[mid] <= w_begin) lo = mid;
            else hi = mid;
        }
        b = lo;
    }
    for (int64_t t = w_begin; t < w_end;) {
        if (!WHOLE)
            while (begin[b + 1] <= t) ++b;
        const int bu = __builtin_amdgcn_readfirstlane(b);
        const Seq sq = load_seq(p, bu);
        int first, count;
        seq_range(p, sq, kTile, first, count);
        int unit, tile0, run;
        if (WHOLE) {
            const int each = ceil_div(count, W);
            unit = (int)blockIdx.x % p.units;
            if (sq.n * p.group > p.few_rows || unit >= ceil_div(sq.n * p.group, 16) * p.n_kv_heads) return;
            tile0 = w * each;
            run = min(each, count - tile0);
            if (run <= 0) break;
        } else {
            // a sequence's tiles of all its units may pass 32 bits; a division of 64 is left for those
            const int64_t local = t - begin[bu];
            unit = local <= 0x7fffffff ? (int)local / count : (int)(local / count);
            tile0 = (int)(local - (int64_t)unit * count);
            run = (int)min(w_end - t, (int64_t)(count - tile0));
        }
        unit = __builtin_amdgcn_readfirstlane(unit);
        tile0 = __builtin_amdgcn_readfirstlane(tile0);
        run = __builtin_amdgcn_readfirstlane(run);
        const int rt = unit / p.n_kv_heads, h = unit - rt * p.n_kv_heads;
        const int32_t *table = p.page_table + (int64_t)bu * p.max_pages;

        TileData<DH> d, next;
        load_tile<DH>(p, table, sq.kv, h, (first + tile0) * kTile, lane, next);

        // this lane's query: row r of the sequence's n * group rows
        const int r = rt * 16 + l15;
        const int tok = r / p.group, head = h * p.group + (r - tok * p.group);
        const bool live = tok < sq.n;
        const int pos = sq.begin + tok;
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

        for (int tile = tile0; tile < tile0 + run; ++tile) {
            d = next;
            const int key0 = (first + tile) * kTile;
            if (tile + 1 < tile0 + run) load_tile<DH>(p, table, sq.kv, h, key0 + kTile, lane, next);
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

        // o[c][i] of a lane is dimension kCols * (4 g + i) + c of query row l15
        if (run == count) {
            const int64_t at = row_out(p, sq, unit, l15);
            const float inv = l > 0.f ? 1.f / l : 0.f;
            if (at >= 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < kCols; c += 4)
                        store_out<NS>(p, at * DH + kCols * (4 * g + i) + c, make_float4(o[c][i] * inv, o[c + 1][i] * inv, o[c + 2][i] * inv, o[c + 3][i] * inv));
                if (g == 0 && p.lse) p.lse[at] = l > 0.f ? m * kLn2 + logf(l) : -INFINITY;
            }
        } else {
            const int slot = t == w_begin ? 0 : 1;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < kCols; c += 4)
                    *reinterpret_cast<float4 *>(sh.o[w][slot] + l15 * kRow + kCols * (4 * g + i) + c) = make_float4(o[c][i], o[c + 1][i], o[c + 2][i], o[c + 3][i]);
            if (g == 0) {
                sh.m[w][slot][l15] = m;
                sh.l[w][slot][l15] = l;
            }
            if (lane == 0) sh.piece[w][slot] = {WHOLE ? 0 : begin[bu] + (int64_t)unit * count, bu, unit, run, count};
        }
        t += WHOLE ? 1 : run;
    }
    __syncthreads();
    if (WHOLE) {  // what the first waves have, all as much, of one unit
        const Piece piece = sh.piece[0][0];
        if (piece.unit_begin < 0) return;
        const int waves = ceil_div(piece.count, piece.run);
        const Seq sq = load_seq(p, piece.b);
        for (int e = tid * 4; e < 16 * DH; e += 64 * W * 4) {
            const int row = e / DH, dim = e - row * DH;
            float m[W], l = 0.f, top = -INFINITY;
            float4 x[W], sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < W; ++k) {
                m[k] = k < waves ? sh.m[k][0][row] : -INFINITY;
                x[k] = *reinterpret_cast<const float4 *>(sh.o[k < waves ? k : 0][0] + row * kRow + dim);
                top = fmaxf(top, m[k]);
            }
#pragma unroll
            for (int k = 0; k < W; ++k) {
                const float scale = m[k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[k] - top);
                l = fmaf(sh.l[k < waves ? k : 0][0][row], scale, l);
                sum.x = fmaf(x[k].x, scale, sum.x), sum.y = fmaf(x[k].y, scale, sum.y), sum.z = fmaf(x[k].z, scale, sum.z), sum.w = fmaf(x[k].w, scale, sum.w);
            }
            const int64_t at = row_out(p, sq, piece.unit, row);
            if (at < 0) continue;
            const float inv = l > 0.f ? 1.f / l : 0.f;
            store_out<NS>(p, at * DH + dim, make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
            if (dim == 0 && p.lse) p.lse[at] = l > 0.f ? top * kLn2 + logf(l) : -INFINITY;
        }
        return;
    }
    // the block's pieces, in the order of the tiles; those of one unit follow each other
    for (int i = 0; i < 2 * W;) {
        const Piece piece = sh.piece[i >> 1][i & 1];
        if (piece.unit_begin < 0) {
            ++i;
            continue;
        }
        int end = i + 1, run = piece.run;
        for (; end < 2 * W; ++end) {
            const Piece &other = sh.piece[end >> 1][end & 1];
            if (other.unit_begin >= 0 && other.unit_begin != piece.unit_begin) break;
            if (other.unit_begin >= 0) run += other.run;
        }
        const Seq sq = load_seq(p, piece.b);
        float *part = p.part + ((int64_t)blockIdx.x * 2 + (piece.unit_begin > t_begin ? 1 : 0)) * part_floats<DH>();
        for (int e = tid * 4; e < 16 * DH; e += 64 * W * 4) {
            const int row = e / DH, dim = e - row * DH;
            float top = -INFINITY, l = 0.f;
            for (int k = i; k < end; ++k)
                if (sh.piece[k >> 1][k & 1].unit_begin >= 0) top = fmaxf(top, sh.m[k >> 1][k & 1][row]);
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = i; k < end; ++k) {
                if (sh.piece[k >> 1][k & 1].unit_begin < 0) continue;
                const float mk = sh.m[k >> 1][k & 1][row], scale = mk == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mk - top);
                const float4 x = *reinterpret_cast<const float4 *>(sh.o[k >> 1][k & 1] + row * kRow + dim);
                l = fmaf(sh.l[k >> 1][k & 1][row], scale, l);
                sum.x = fmaf(x.x, scale, sum.x), sum.y = fmaf(x.y, scale, sum.y), sum.z = fmaf(x.z, scale, sum.z), sum.w = fmaf(x.w, scale, sum.w);
            }
            if (run < piece.count) {
                *reinterpret_cast<float4 *>(part + e) = sum;
                if (dim == 0) {
                    part[16 * DH + row] = top;
                    part[16 * DH + 16 + row] = l;
                }
                continue;
            }
            const int64_t at = row_out(p, sq, piece.unit, row);
            if (at < 0) continue;
            const float inv = l > 0.f ? 1.f / l : 0.f;
            store_out<NS>(p, at * DH + dim, make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
            if (dim == 0 && p.lse) p.lse[at] = l > 0.f ? top * kLn2 + logf(l) : -INFINITY;
        }
        i = end;
    }
}

// Joins the partial results of the units that more than one block worked on.  A block per unit (x: row of a unit of a sequence, y: sequence)
// and row; DH / 4 threads hold the row, the block's other threads take other partial results.  (A block a unit, one partial result after
// the other: two sequences of 131072 keys, two heads, 128 results a unit: 49 us.)
template <int DH, int NS>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnParams p, int rows)
{
    static constexpr int kTile = tile_keys(DH), kLanes = DH / 4, kGroups = kThreads / kLanes;
    __shared__ float4 sums[kGroups][kLanes];
    __shared__ float tops[kGroups], ls[kGroups];
    const int b = blockIdx.y, unit = blockIdx.x / rows, row = blockIdx.x - unit * rows;
    const Seq sq = load_seq(p, b);
    if (sq.n == 0 || sq.n * p.group > p.few_rows || unit >= ceil_div(sq.n * p.group, 16) * p.n_kv_heads) return;
    const int64_t at = row_out(p, sq, unit, row);
    if (at < 0) return;
    int first, count;
    seq_range(p, sq, kTile, first, count);
    const int64_t per = tiles_per_block(p.seq_tiles[p.B], p.n_blocks);
    const int64_t t0 = p.seq_tiles[b] + (int64_t)unit * count, t1 = t0 + count;
    const int64_t b0 = t0 / per, b1 = (t1 - 1) / per;
    if (b0 == b1) return;
    const int x = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    float top = -INFINITY, l = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const auto add = [&](float pm, float pl, float4 v) {
        const float m_new = fmaxf(top, pm), base = m_new == -INFINITY ? 0.f : m_new;
        const float keep = __builtin_amdgcn_exp2f(top - base), more = __builtin_amdgcn_exp2f(pm - base);
        top = m_new;
        l = l * keep + pl * more;
        sum.x = sum.x * keep + v.x * more;
        sum.y = sum.y * keep + v.y * more;
        sum.z = sum.z * keep + v.z * more;
        sum.w = sum.w * keep + v.w * more;
    };
#pragma unroll 4
    for (int64_t k = b0 + group; k <= b1; k += kGroups) {
        const float *part = p.part + (2 * k + (t0 > k * per ? 1 : 0)) * part_floats<DH>();
        add(part[16 * DH + row], part[16 * DH + 16 + row], *reinterpret_cast<const float4 *>(part + row * DH + 4 * x));
    }
    if (x == 0) {
        tops[group] = top;
        ls[group] = l;
    }
    sums[group][x] = sum;
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int k = 1; k < kGroups; ++k) add(tops[k], ls[k], sums[k][x]);
    const float inv = l > 0.f ? 1.f / l : 0.f;
    store_out<NS>(p, at * DH + 4 * x, make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
    if (x == 0 && p.lse) p.lse[at] = l > 0.f ? top * kLn2 + logf(l) : -INFINITY;
}

// Blocks a CU: two; one where a wave needs the registers of two (fp32 over 128 dimensions, 256 dimensions)
template <int DH, int NS>
constexpr int blocks_per_cu() { return DH == 256 || (DH == 128 && NS == 3) ? 1 : 2; }

template <int DH, int NS, int W, bool WHOLE>
int launch_waves(const AttnParams &p, int64_t blocks, hipStream_t s)
{
    static constexpr int M = W == kWaves ? blocks_per_cu<DH, NS>() : 1;  // waves of 256 registers in any case
    static constexpr size_t kMost = sizeof(Shared<DH, W>) + (MOE_ATTN_MAX_B + 1) * 8;
    static_assert(kMost <= 160 * 1024, "the sequences' places have to fit the LDS beside the pieces");
    const size_t lds = sizeof(Shared<DH, W>) + (WHOLE ? 0 : (p.B + 1) * 8);
    static std::once_flag once;
    static hipError_t setup_rc = hipSuccess;
    std::call_once(once, [&]() {
        setup_rc = hipFuncSetAttribute(reinterpret_cast<const void *>(attn_decode_kernel<DH, NS, M, W, WHOLE>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMost);
    });
    MOE_HIP_CHECK(setup_rc);
    hipLaunchKernelGGL((attn_decode_kernel<DH, NS, M, W, WHOLE>), dim3((unsigned)blocks), dim3(64 * W), lds, s, p);
    MOE_LAUNCH_CHECK("attn_decode_kernel");
    return MOE_OK;
}

template <int DH, int NS>
int launch_as(AttnParams p, int num_cus, hipStream_t s)
{
    p.n_blocks = blocks_per_cu<DH, NS>() * num_cus;
    const int64_t rows = (int64_t)p.max_q * p.group < p.few_rows ? (int64_t)p.max_q * p.group : p.few_rows;
    p.units = ceil_div((int)rows, 16) * p.n_kv_heads;
    const int unit_rows = rows < 16 ? (int)rows : 16;
    // Where no unit has more than four tiles a wave, or eight and there are units for every CU, a block takes a whole unit: it need not look for its
    // part, and nothing is left to join.  Where there are not, and a CU has the registers, twice the waves take it.  us a call, whole / in parts / by
    // eight waves:
    //    1 x 1000 keys, 16 heads of 64     10.5 / 13.5 / 10.4       1 x 1000, 8 heads of 128    14.3 / 19.2 / 12.7
    //    8 x 2000 keys, 16 heads of 64        - / 18.1 / 14.1       8 x 2000, 8 heads of 128       - / 19.4 / 19.6
    //   64 x 2000 keys, 16 heads of 64     51.7 / 74.0 / 56.5     256 x 500, 16 heads of 64     55.6 / -    / 92.0
    // It goes by the caller's bound, as the lengths are on the device: 900 keys of 16 heads of 64, captured, 7.9 us with bounds of 2048 and less, 12.8 above.
    static constexpr bool kTwice = blocks_per_cu<DH, NS>() == 2;
    const int tiles = ceil_div(p.max_kv, tile_keys(DH));
    const bool every = (int64_t)p.units * p.B >= num_cus;
    if (tiles <= 4 * kWaves || (tiles <= 8 * kWaves && (every || (kTwice && DH == 64)))) {
        if (kTwice && !every && tiles > kWaves) return launch_waves<DH, NS, kTwice ? 2 * kWaves : kWaves, true>(p, (int64_t)p.units * p.B, s);
        return launch_waves<DH, NS, kWaves, true>(p, (int64_t)p.units * p.B, s);
    }
    const int failed = launch_waves<DH, NS, kWaves, false>(p, p.n_blocks, s);
    if (failed) return failed;
    hipLaunchKernelGGL((attn_join_kernel<DH, NS>), dim3(p.units * unit_rows, p.B), dim3(kThreads), 0, s, p, unit_rows);
    MOE_LAUNCH_CHECK("attn_join_kernel");
    return MOE_OK;
}

}  // namespace

// partial results of two units a block
int64_t attn_decode_workspace(int head_dim, int num_cus)
{
    return align_up((int64_t)2 * num_cus * 2 * (16 * head_dim + 32) * 4, 256);
}

int launch_attn_decode(int dtype, int head_dim, const AttnParams &p, int num_cus, hipStream_t s)
{
    const bool bf = dtype == MOE_DTYPE_BF16;
    if (head_dim == 64) return bf ? launch_as<64, 1>(p, num_cus, s) : launch_as<64, 3>(p, num_cus, s);
    if (head_dim == 128) return bf ? launch_as<128, 1>(p, num_cus, s) : launch_as<128, 3>(p, num_cus, s);
    return bf ? launch_as<256, 1>(p, num_cus, s) : launch_as<256, 3>(p, num_cus, s);
}

}  // namespace moe355
