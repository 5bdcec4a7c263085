// Attention over a paged e4m3 cache for many query rows per key head (prefill, chunks of it, cross attention).
//
// A block owns 32 W query rows (new tokens x heads of a group) of a (sequence, key head), a wave 32 of them, and walks tiles of 64
// keys with a running maximum and sum.  Keys and values are widened to bf16 once for the block on their way into LDS:
//   K    [64 keys][DH], V^T [DH][64 keys], 16-byte chunks swizzled so that 16 lanes that read a fragment, and 16 that write, meet each
//        bank once (V's writes: twice); two or four buffers, a later tile's bytes are in flight while this one is computed
//   S^T = K Q^T and O^T = V^T P^T by 32x32x16 MFMAs; queries stay in registers.  A lane holds 4 keys in 8 of one query; a chunk of
//        V^T holds just those keys in just that order, so the weights are the second product's operand where the first left them.
// The maximum, the sum and the rescaling of a query are its lane's own; two lanes share a query.  The scales are powers of two, which the
// conversion to bf16 multiplies by for nothing, and no later step knows of them.  (In the exponent instead, a key's as part of its factor and
// a value's as its offset, they cost instructions per 16 keys, and the scale of a page of zeros, 2^-126, takes its weights out of fp32.)
// Products below 2^-126 may be lost: what they weigh is less than that, too.
//
// With bf16 queries a weight is rounded once to bf16 for the second product, 2^-9 of it; the sum has it unrounded.  The weights are relative to the row's
// largest so far, so that the largest is 1 and rounds to itself: where a key or two take nearly all of a row, as they do, little else is left to round.
// (A maximum that may be behind by a factor of 256 rescales the output less often, but rounds the largest weight like the rest: 8192 tokens 298 us and an
// error of 2.2e-3 of the outputs, with this 303 and 1.8e-3; fp32 weights rounded to bf16 at the output alone 1.6e-3.  Weights as two bf16 numbers: 390.
// fp32 queries have three pieces of everything, and none of this.)
//
// Bound by the matrix cores and the exponentials (a quarter of the rate of other instructions) in about equal parts: per 32 x 64 weights
// and wave 32 MFMAs of 32 cycles, 32 exponentials of 16 and some 110 others of 4.  Two waves a SIMD overlap them.  Measured: 8192 tokens, 16
// heads of 128, bf16, causal: 299 to 305 us, 900 to 920 TFLOP/s; matrix pipes busy 36 %, vector issue 45 %, LDS reads about 40 %.  (Half of the waves held half
// a tile behind the others by barriers, so that products meet exponentials: 327 where this took 307; other priorities of the waves: no difference.)
// Over 256 dimensions a wave has no registers left: 25 of them spill with bf16 queries, 161 with fp32.
//
// Blocks begin with the last rows, which see the most keys; a sequence's heads stay on one XCD and its L2.  Where there are too few
// blocks for the chip, the keys are cut into parts, joined by a second kernel.
#include "attn_dev.h"

#include <mutex>

namespace moe355 {

namespace {

static constexpr int kTile = 64;

struct PrefillParams {
    AttnParams a;
    int row_tiles, splits;  // bounds for all sequences
};

template <int DH>
struct alignas(16) Buffer {
    uint16_t k[kTile * DH];
    uint16_t v[DH * kTile];
    int held[4];  // 16 keys each: the page table names a page for them
    int whole;    // all of them
};

template <int DH>
__device__ __forceinline__ int k_at(int row, int chunk)  // element of a 16-byte chunk of K
{
    return row * DH + (DH == 64 ? chunk ^ ((row >> 1) & 7) : chunk ^ (row & 15)) * 8;
}
__device__ __forceinline__ int v_at(int dim, int chunk)
{
    return dim * kTile + (chunk ^ ((dim >> 1) & 7) ^ ((dim >> 4) & 1)) * 8;
}

// The tiles of keys that rows [row0, row0 + rows) of a sequence see: first, count.
__device__ __forceinline__ void tile_range(const AttnParams &p, const Seq &sq, int row0, int rows, int &first, int &count)
{
    const int tok0 = row0 / p.group, tok1 = min((row0 + rows - 1) / p.group, sq.n - 1);
    const int pos0 = sq.begin + tok0, pos1 = sq.begin + tok1;
    const int end = p.causal ? min(sq.kv, max(pos1 + 1, 0)) : sq.kv;
    const int begin = p.window > 0 ? min(max(0, pos0 - p.window + 1), end) : 0;
    first = begin / kTile;
    count = ceil_div(end, kTile) - first;
}

// Tiles between two barriers: while these are computed the next ones are stored.  With two, waves need not keep step so closely, and 8 waves' block
// has the LDS for four buffers (8192 tokens of 16 heads of 128: 294 us where one takes 307).  A block of 4 shares its CU with another.
template <int W>
constexpr int kTogether = W == 8 ? 2 : 1;

// A partial result: the rows' outputs (not divided by the sum), maxima, sums
template <int DH, int W>
constexpr int64_t part_floats() { return (int64_t)32 * W * (DH + 2); }

template <int DH, int NS, int W>
__global__ __launch_bounds__(64 * W, NS == 1 && DH <= 128 ? 2 : 1) void attn_prefill_kernel(PrefillParams pp)
{
    static constexpr int kThreads = 64 * W, kRows = 32 * W, kRole = kThreads / 2;
    static constexpr int kKItems = (4 * DH + kRole - 1) / kRole;  // 16 bytes of a key each
    static constexpr int kVItems = (2 * DH + kRole - 1) / kRole;  // 4 dimensions of 8 values each
    static constexpr int kWords = kKItems * 4 > kVItems * 8 ? kKItems * 4 : kVItems * 8;
    static constexpr int kSteps = DH / 16, kCols = DH / 32, kNext = kTogether<W>;
    static constexpr int kValues = DH <= 128 ? 2 : 1;  // fragments of the values in registers: of this 16 keys and the next, where they fit
    extern __shared__ __align__(16) uint8_t lds[];
    Buffer<DH> *buffer = reinterpret_cast<Buffer<DH> *>(lds);
    const AttnParams &p = pp.a;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l31 = lane & 31, half = lane >> 5;

    const int per_tile = p.B * p.n_kv_heads * pp.splits;
    const int index = (int)(blockIdx.y * gridDim.x + blockIdx.x);
    const int rt = pp.row_tiles - 1 - index / per_tile;
    if (rt < 0) return;  // the last row of the grid may have too many
    const int rest = index % per_tile;
    const int part = rest % pp.splits, h = rest / pp.splits % p.n_kv_heads, b = rest / pp.splits / p.n_kv_heads;
    const Seq sq = load_seq(p, b);
    if (sq.n * p.group <= p.few_rows || rt * kRows >= sq.n * p.group) return;
    int first, count;
    tile_range(p, sq, rt * kRows, kRows, first, count);
    if (pp.splits > 1) {
        const int each = ceil_div(count, pp.splits);
        first += part * each;
        count = min(each, max(0, count - part * each));
    }
    const int32_t *table = p.page_table + (int64_t)b * p.max_pages;

    const int r = rt * kRows + w * 32 + l31;
    const int tok = r / p.group, head = h * p.group + (r - tok * p.group);
    const bool live = tok < sq.n;
    const int pos = sq.begin + tok;
    const int key_end = !live ? 0 : p.causal ? min(pos + 1, sq.kv) : sq.kv;
    const int key_begin = p.window > 0 ? max(0, pos - p.window + 1) : 0;
    // over the wave's rows: keys that all see, and that any sees
    int all_begin = live ? key_begin : 0, all_end = live ? key_end : 0x7fffffff;
    int any_begin = live ? key_begin : 0x7fffffff, any_end = key_end;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) {
        all_begin = max(all_begin, __shfl_xor(all_begin, off, 64));
        all_end = min(all_end, __shfl_xor(all_end, off, 64));
        any_begin = min(any_begin, __shfl_xor(any_begin, off, 64));
        any_end = max(any_end, __shfl_xor(any_end, off, 64));
    }
    all_begin = __builtin_amdgcn_readfirstlane(all_begin);
    all_end = min(__builtin_amdgcn_readfirstlane(all_end), sq.kv);
    any_begin = __builtin_amdgcn_readfirstlane(any_begin);
    any_end = __builtin_amdgcn_readfirstlane(any_end);

    // queries; a negative scale and one of zero are theirs, so that the factor in front of the exponent is positive (times a masked score's infinity
    // zero is no number)
    const bool negative = p.scale_log2e < 0.f, asks = live && p.scale_log2e != 0.f;
    const float scale = p.scale_log2e != 0.f ? fabsf(p.scale_log2e) : 1.f;
    Pieces<NS> q[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int64_t at = (int64_t)(sq.first + tok) * p.q_stride + (int64_t)head * DH + 16 * s + 8 * half;
        if (NS == 1) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (asks) x = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.q) + at);
            if (negative) x = make_uint4(x.x ^ 0x80008000u, x.y ^ 0x80008000u, x.z ^ 0x80008000u, x.w ^ 0x80008000u);
            q[s].x[0] = __builtin_bit_cast(bf16x8, x);
        } else {
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (asks) {
                const float4 lo = *reinterpret_cast<const float4 *>(static_cast<const float *>(p.q) + at);
                const float4 hi = *reinterpret_cast<const float4 *>(static_cast<const float *>(p.q) + at + 4);
                x[0] = lo.x, x[1] = lo.y, x[2] = lo.z, x[3] = lo.w, x[4] = hi.x, x[5] = hi.y, x[6] = hi.z, x[7] = hi.w;
            }
            if (negative)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = -x[i];
            q[s] = split<NS>(x);
        }
    }

    // staging: the first half of the waves brings keys, the other values
    const bool brings_k = w < W / 2;
    const int role = brings_k ? tid : tid - kRole;
    const int page_mask = (1 << p.page_shift) - 1;
    uint32_t words[kWords];
    float unit_scale[kKItems > kVItems ? kKItems : kVItems];
    int page[kKItems > kVItems ? kKItems : kVItems], group_page = -1;
    // Where this thread's bytes lie in a page, without the page: in tiles that are there as a whole, nearly all of them, the loads then take an
    // address and offsets that are part of the instruction.  (With a predicate and an address of its own for each: 348 us where this took 313.)
    int in_tile[kKItems > kVItems ? kKItems : kVItems];
#pragma unroll
    for (int i = 0; i < (kKItems > kVItems ? kKItems : kVItems); ++i) {
        const int item = i * kRole + role;
        in_tile[i] = brings_k ? min(item / (DH / 16), kTile - 1) : 16 * (min(item / (DH / 4), 7) >> 1) + 4 * (item / (DH / 4) & 1);
    }
    const auto page_of = [&](int key) { return key < sq.kv ? table[key >> p.page_shift] : -1; };
    const auto look_up = [&](int key0) {  // the pages of a tile, a tile ahead of its bytes
        if (brings_k) {
#pragma unroll
            for (int i = 0; i < kKItems; ++i) page[i] = page_of(key0 + in_tile[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kVItems; ++i) page[i] = page_of(key0 + in_tile[i]);
        }
        if (tid < 4) group_page = page_of(key0 + 16 * tid);
    };
    bool group_held = false;
    const auto load = [&](int key0) {
        bool there = key0 + kTile <= sq.kv;
#pragma unroll
        for (int i = 0; i < (kKItems > kVItems ? kKItems : kVItems); ++i)
            if (i < (brings_k ? kKItems : kVItems)) there = there && (uint32_t)page[i] < (uint32_t)p.num_pages;
        const bool whole = __all(there);
        if (brings_k) {
#pragma unroll
            for (int i = 0; i < kKItems; ++i) {
                const int item = i * kRole + role, row = in_tile[i], c = item % (DH / 16);
                const bool held = whole || (key0 + row < sq.kv && (uint32_t)page[i] < (uint32_t)p.num_pages);
                const int64_t unit = (int64_t)(held ? page[i] : 0) * p.n_kv_heads + h;
                const uint8_t *src = p.k + ((unit << p.page_shift) + ((key0 + row) & page_mask)) * DH + 16 * c;
                unit_scale[i] = held ? p.k_scale[unit] : 1.f;
                uint4 x;
                if (whole) x = *reinterpret_cast<const uint4 *>(src);
                else x = held ? *reinterpret_cast<const uint4 *>(src) : make_uint4(0, 0, 0, 0);
                words[4 * i] = x.x, words[4 * i + 1] = x.y, words[4 * i + 2] = x.z, words[4 * i + 3] = x.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVItems; ++i) {
                const int quad = (i * kRole + role) % (DH / 4), row0 = in_tile[i];
                const bool held = whole || (uint32_t)page[i] < (uint32_t)p.num_pages;
                const int64_t unit = (int64_t)(held ? page[i] : 0) * p.n_kv_heads + h;
                const uint8_t *src = p.v + ((unit << p.page_shift) + ((key0 + row0) & page_mask)) * DH + 4 * quad;
                unit_scale[i] = held ? p.v_scale[unit] : 1.f;
                if (whole) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) words[8 * i + j] = *reinterpret_cast<const uint32_t *>(src + ((j & 3) + 8 * (j >> 2)) * DH);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int row = (j & 3) + 8 * (j >> 2);
                        words[8 * i + j] = held && key0 + row0 + row < sq.kv ? *reinterpret_cast<const uint32_t *>(src + row * DH) : 0u;
                    }
                }
            }
        }
        if (tid < 4) group_held = (uint32_t)group_page < (uint32_t)p.num_pages;
    };
    const auto store = [&](Buffer<DH> &to) {
        if (brings_k) {
#pragma unroll
            for (int i = 0; i < kKItems; ++i) {
                const int item = i * kRole + role, row = item / (DH / 16), c = item - row * (DH / 16);
                if (row >= kTile) continue;
                *reinterpret_cast<bf16x8 *>(to.k + k_at<DH>(row, 2 * c)) = widen(words[4 * i], words[4 * i + 1], unit_scale[i]);
                *reinterpret_cast<bf16x8 *>(to.k + k_at<DH>(row, 2 * c + 1)) = widen(words[4 * i + 2], words[4 * i + 3], unit_scale[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVItems; ++i) {
                const int item = i * kRole + role, c = item / (DH / 4), quad = item - c * (DH / 4);
                if (c >= 8) continue;
                uint32_t lo[4], hi[4];
                transpose4(words[8 * i], words[8 * i + 1], words[8 * i + 2], words[8 * i + 3], lo);
                transpose4(words[8 * i + 4], words[8 * i + 5], words[8 * i + 6], words[8 * i + 7], hi);
#pragma unroll
                for (int y = 0; y < 4; ++y) *reinterpret_cast<bf16x8 *>(to.v + v_at(4 * quad + y, c)) = widen(lo[y], hi[y], unit_scale[i]);
            }
        }
        if (w == 0) {
            const bool all = __all(tid >= 4 || group_held);
            if (tid == 0) to.whole = all;
            if (tid < 4) to.held[tid] = group_held;
        }
    };

    f32x16 o[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    if (count > 0) {
        look_up(first * kTile);
#pragma unroll
        for (int i = 0; i < kNext; ++i) {  // past the last tile: zeros, which nobody reads
            load((first + i) * kTile);
            look_up((first + i + 1) * kTile);
            store(buffer[i]);
        }
        __syncthreads();
    }
    for (int t = 0; t < count; ++t) {
        const int key0 = (first + t) * kTile;
        if (t + kNext < count) {
            load(key0 + kNext * kTile);
            look_up(key0 + (kNext + 1) * kTile);
        }
        const Buffer<DH> &buf = buffer[t % (2 * kNext)];
        if (key0 < any_end && key0 + kTile > any_begin) {
            // Fragments are asked for kAhead steps before their MFMAs, and the order is kept by scheduling barriers: left to itself the
            // compiler asks for two and waits for them (prefill of 8192 tokens 355 us, matrix pipes busy 30 %).
            static constexpr int kAhead = kSteps < 4 ? kSteps : 4;
            f32x16 s[2];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[n][i] = 0.f;
            bf16x8 key[kAhead][2], value[kValues][kCols];
#pragma unroll
            for (int x = 0; x < kAhead; ++x)
#pragma unroll
                for (int n = 0; n < 2; ++n) key[x][n] = *reinterpret_cast<const bf16x8 *>(buf.k + k_at<DH>(32 * n + l31, 2 * x + half));
            const int all_held = buf.whole;
            __builtin_amdgcn_s_setprio(1);  // the wave that has products goes before the one that has exponentials (1 %)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < kSteps; ++x) {
                bf16x8 now[2] = {key[x % kAhead][0], key[x % kAhead][1]};
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < NS; ++i) s[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(now[n], q[x].x[i], s[n], 0, 0, 0);
                if (x + kAhead < kSteps)
#pragma unroll
                    for (int n = 0; n < 2; ++n) key[x % kAhead][n] = *reinterpret_cast<const bf16x8 *>(buf.k + k_at<DH>(32 * n + l31, 2 * (x + kAhead) + half));
                __builtin_amdgcn_sched_barrier(0);
            }
            if (kValues == 2)
#pragma unroll
                for (int c = 0; c < kCols; ++c) value[0][c] = *reinterpret_cast<const bf16x8 *>(buf.v + v_at(32 * c + l31, half));
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
            const bool whole = key0 >= all_begin && key0 + kTile <= all_end && __builtin_amdgcn_readfirstlane(all_held);
            if (!whole) {
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = key0 + 32 * n + 8 * (i >> 2) + 4 * half + (i & 3);
                        s[n][i] = buf.held[2 * n + (i >> 3)] && key >= key_begin && key < key_end ? s[n][i] : -INFINITY;
                    }
            }
            float top = -INFINITY;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
            top = fmaxf(top, __shfl_xor(top, 32, 64)) * scale;
            if (__any(top > m)) {  // m is -infinity until a row has seen a key
                const float m_new = fmaxf(m, top);
                const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
                m = m_new;
                l *= alpha;
#pragma unroll
                for (int c = 0; c < kCols; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[c][i] *= alpha;
            }
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int ask = g + kValues - 1;
                if (ask < 4)
#pragma unroll
                    for (int c = 0; c < kCols; ++c) value[ask % kValues][c] = *reinterpret_cast<const bf16x8 *>(buf.v + v_at(32 * c + l31, 2 * ask + half));
                __builtin_amdgcn_sched_barrier(0);
                float weight[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    weight[i] = __builtin_amdgcn_exp2f(fmaf(s[g >> 1][8 * (g & 1) + i], scale, -base));
                    l += weight[i];
                }
                const Pieces<NS> wp = split<NS>(weight);
#pragma unroll
                for (int c = 0; c < kCols; ++c)
#pragma unroll
                    for (int i = 0; i < NS; ++i) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value[g % kValues][c], wp.x[i], o[c], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (t + kNext < count) store(buffer[(t + kNext) % (2 * kNext)]);
        if (t % kNext == kNext - 1) __syncthreads();
    }
    l += __shfl_xor(l, 32, 64);
    // o[c][i] of a lane is dimension 32 c + 8 (i / 4) + 4 half + i % 4 of its query
    if (pp.splits > 1) {
        const int64_t slot = ((int64_t)rt * p.B * p.n_kv_heads + (int64_t)b * p.n_kv_heads + h) * pp.splits + part;
        float *to = p.part + slot * part_floats<DH, W>();
        const int row = w * 32 + l31;
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<float4 *>(to + (int64_t)row * DH + 32 * c + 2 * i + 4 * half) = make_float4(o[c][i], o[c][i + 1], o[c][i + 2], o[c][i + 3]);
        if (half == 0) {
            to[(int64_t)kRows * DH + row] = m;
            to[(int64_t)kRows * DH + kRows + row] = l;
        }
        return;
    }
    if (!live) return;
    const int64_t at = (int64_t)(sq.first + tok) * p.n_heads + head;
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int64_t dim = at * DH + 32 * c + 2 * i + 4 * half;
            if (NS == 1)
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + dim) =
                    make_uint2(pack_bf16(o[c][i] * inv, o[c][i + 1] * inv), pack_bf16(o[c][i + 2] * inv, o[c][i + 3] * inv));
            else
                *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + dim) = make_float4(o[c][i] * inv, o[c][i + 1] * inv, o[c][i + 2] * inv, o[c][i + 3] * inv);
        }
    if (half == 0 && p.lse) p.lse[at] = l > 0.f ? m * kLn2 + logf(l) : -INFINITY;
}

// Joins the parts of the keys: a block per 16 rows of a unit.
template <int DH, int NS, int W>
__global__ __launch_bounds__(256) void attn_prefill_join_kernel(PrefillParams pp)
{
    static constexpr int kRows = 32 * W, kPieces = kRows / 16;
    const AttnParams &p = pp.a;
    const int piece = blockIdx.x % kPieces, unit = blockIdx.x / kPieces;
    const int h = unit % p.n_kv_heads, b = unit / p.n_kv_heads % p.B, rt = unit / p.n_kv_heads / p.B;
    const Seq sq = load_seq(p, b);
    if (sq.n * p.group <= p.few_rows) return;
    for (int e = threadIdx.x * 4; e < 16 * DH; e += 256 * 4) {
        const int row = piece * 16 + e / DH, dim = e % DH, r = rt * kRows + row, tok = r / p.group;
        if (tok >= sq.n) continue;
        float top = -INFINITY, l = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < pp.splits; ++k) {
            const float *part = p.part + ((int64_t)unit * pp.splits + k) * part_floats<DH, W>();
            const float pm = part[(int64_t)kRows * DH + row], pl = part[(int64_t)kRows * DH + kRows + row];
            const float4 x = *reinterpret_cast<const float4 *>(part + (int64_t)row * DH + dim);
            const float m_new = fmaxf(top, pm), base = m_new == -INFINITY ? 0.f : m_new;
            const float keep = __builtin_amdgcn_exp2f(top - base), add = __builtin_amdgcn_exp2f(pm - base);
            top = m_new;
            l = l * keep + pl * add;
            sum.x = sum.x * keep + x.x * add;
            sum.y = sum.y * keep + x.y * add;
            sum.z = sum.z * keep + x.z * add;
            sum.w = sum.w * keep + x.w * add;
        }
        const int64_t at = (int64_t)(sq.first + tok) * p.n_heads + h * p.group + (r - tok * p.group);
        const float inv = l > 0.f ? 1.f / l : 0.f;
        if (NS == 1)
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + at * DH + dim) =
                make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
        else
            *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + at * DH + dim) = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
        if (dim == 0 && p.lse) p.lse[at] = l > 0.f ? top * kLn2 + logf(l) : -INFINITY;
    }
}

// Parts of the keys: none where the units give every CU two blocks, else so many that they do, of four tiles at least (a part of 256 rows and 128
// dimensions costs 133 KB written and read again, as much as two tiles).  units: blocks of the grid; filled: about how many of them have rows.
// Part buffers: 4 a CU.
int splits_for(int64_t units, int64_t filled, int tiles, int num_cus)
{
    int64_t n = filled >= 2 * num_cus ? 1 : 2 * num_cus / (filled > 0 ? filled : 1);
    if (n > (tiles + 3) / 4) n = (tiles + 3) / 4;
    if (n > 4 * num_cus / units) n = 4 * num_cus / units;
    return n < 1 ? 1 : (int)n;
}

template <int DH, int NS, int W>
int launch_as(PrefillParams pp, int num_cus, hipStream_t s)
{
    static constexpr size_t kLds = 2 * kTogether<W> * sizeof(Buffer<DH>);
    static std::once_flag once;
    static hipError_t setup_rc = hipSuccess;
    std::call_once(once, [&]() {
        setup_rc = hipFuncSetAttribute(reinterpret_cast<const void *>(attn_prefill_kernel<DH, NS, W>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds);
    });
    MOE_HIP_CHECK(setup_rc);
    const AttnParams &p = pp.a;
    pp.row_tiles = (int)(((int64_t)p.max_q * p.group + 32 * W - 1) / (32 * W));
    const int64_t units = (int64_t)pp.row_tiles * p.B * p.n_kv_heads;
    const int64_t filled = ((int64_t)p.T * p.group / (32 * W) + p.B) * p.n_kv_heads;
    pp.splits = splits_for(units, filled < units ? filled : units, ceil_div(p.max_kv, kTile), num_cus);
    // rows of the grid of 2^22 blocks: a launch of 2^32 threads in one dimension starts fewer and says nothing
    const int64_t blocks = units * pp.splits, row = 1 << 22;
    if (blocks >= (1ll << 31) - row) {
        set_error("moe_attn_forward: %lld blocks", (long long)blocks);
        return MOE_ERR_INVALID_ARG;
    }
    hipLaunchKernelGGL((attn_prefill_kernel<DH, NS, W>), dim3((unsigned)(blocks < row ? blocks : row), (unsigned)((blocks + row - 1) / row)), dim3(64 * W), kLds, s, pp);
    MOE_LAUNCH_CHECK("attn_prefill_kernel");
    if (pp.splits > 1) {
        hipLaunchKernelGGL((attn_prefill_join_kernel<DH, NS, W>), dim3((unsigned)(units * 2 * W)), dim3(256), 0, s, pp);
        MOE_LAUNCH_CHECK("attn_prefill_join_kernel");
    }
    return MOE_OK;
}

}  // namespace

int64_t attn_prefill_workspace(int head_dim, int num_cus)
{
    const int w = head_dim <= 128 ? 8 : 4;
    return align_up((int64_t)4 * num_cus * 32 * w * (head_dim + 2) * 4, 256);
}

// p.part: attn_prefill_workspace() bytes
int launch_attn_prefill(int dtype, int head_dim, const AttnParams &p, int num_cus, hipStream_t s)
{
    const PrefillParams pp = {p, 0, 1};
    const bool bf = dtype == MOE_DTYPE_BF16;
    // Rows of 256 and two waves a SIMD; fp32 and 256 dimensions need the registers of both.  Rows of 128 too where tiles of 256 would be fewer than
    // the CUs: staging costs twice as much a row then (8192 tokens of 16 heads: 467 us, 313 with 256 at the time), but more CUs work.
    const bool small = ((int64_t)p.T * p.group / 256 + p.B) * p.n_kv_heads < num_cus;
    if (bf && small && head_dim == 64) return launch_as<64, 1, 4>(pp, num_cus, s);
    if (bf && small && head_dim == 128) return launch_as<128, 1, 4>(pp, num_cus, s);
    if (head_dim == 64) return bf ? launch_as<64, 1, 8>(pp, num_cus, s) : launch_as<64, 3, 4>(pp, num_cus, s);
    if (head_dim == 128) return bf ? launch_as<128, 1, 8>(pp, num_cus, s) : launch_as<128, 3, 4>(pp, num_cus, s);
    return bf ? launch_as<256, 1, 4>(pp, num_cus, s) : launch_as<256, 3, 4>(pp, num_cus, s);
}

}  // namespace moe355
