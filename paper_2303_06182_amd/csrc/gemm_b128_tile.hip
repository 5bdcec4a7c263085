// Products of e4m3 operands in blocks of 128 on one persistent block per CU: tiles of up to 256 rows by 256 weight rows.
//
// What bounds them: the matrix cores where an expert has rows enough, the stream of the weights where it has few.  8 waves, 2 x 4; each owns up to 4
// blocks of 32 rows and 2 of 32 weight rows (the weights are the first operand, so that a lane's sums are 16 neighbouring columns of one
// row).  A tile costs what its rows cost: its 32-row blocks are dealt to the two rows of waves in turn and the K loop exists once per block count.
//
// Measured: 8192^3 fast 440 to 460 us (2.4 to 2.5 PFLOP/s, matrix cores 63 % busy at 1.85 GHz; a library product of e4m3 numbers 420), precise 877; 24 experts of 5003 rows in all,
// 1200 -> 1640, 29 us in one round of tiles (66 MB: 13 us); 65536 rows, 128 -> 8192 311 us (3.5 TB/s, nearly all written).
//
// Fast (bf16 results): v_mfma_scale_f32_32x32x64_f8f6f4, which takes the scales as exponents.  A K tile of 128 bytes goes to LDS in two halves
// of 64; five half slots of 32 KB make a ring that is filled by direct-to-LDS loads.  Step u (64 k) multiplies the fragments of slot u mod 5, which were
// read into registers during step u - 1:
//   1. the products of row block 0;
//   2. wait for this wave's LDS reads, on odd steps also for its loads of the next K tile; barrier.  Behind it slots u - 1 and u are free,
//      and the next K tile has landed for everybody;
//   3. the other products; behind them the reads of step u + 1's fragments and the loads of the K tile two ahead, weights in
//      the even step, rows in the odd one (the other way round in small tiles).
//
// Precise (results in fp32, or activated and quantised again): both operands are widened to bf16 in registers and go through
// v_mfma_f32_32x32x16_bf16, with fp32 sums throughout and twice the time.  Four half slots, that is two K tiles; fragments are read 32 k ahead of
// their products, and there is one barrier a K tile, behind which the loads of the K tile two ahead go out.
// Why the first product of a feed-forward is precise: its results are rounded to e4m3, and what the fast instruction is off by (1.4e-5 of
// their deviation) sends some elements in ten thousand to the other side of a border.  With it the output's error against 64 bits was 2.2e-3
// to 2.5e-3, without it 1.7e-3, which is the output's own rounding to bf16.
//
// Deep (first product of a feed-forward in fp32): there nothing hides a hidden element that falls to the other side of a border of e4m3.  A sum of n roundings is off
// by the sum of its partial sums' squares, n^2 / 2; sums of 16 steps (256 k) and then of those sums by 8 n + n^2 / 32, which at K = 2048 is 0.4 of the
// error.  The second sums take registers, so a tile has 128 rows at most: 16384 tokens x 2 over 16 experts, 2048 -> 8192 -> 2048, 1.94 -> 2.17 ms.  Of 28 drawn cases 11 had
// elements on the other side of a border than 64-bit sums, and 8 have (a plain program in fp32: 7).
//
// A slot row is 64 bytes: 16-byte chunk c of row r sits at position c ^ ((r >> 2) & 3), which keeps the 16 lanes x 16 bytes of a
// fragment read on 16 different bank groups.  A lane's 16 bytes of a row are the same k for either operand, whatever their order.
// Weight row permutation: LDS row i of a block of 32 holds column 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3), so that the 16 sums of a lane are
// columns 16 * (lane / 32) ... of row lane % 32 and leave as whole 16-byte stores.
//
// Launch: one block per CU, no list on the device: every block works out from the offsets which output tiles its XCD has (an eighth of all, by cost)
// and takes every 32nd of them.  The load cursor walks the block's whole sequence of (tile, K tile), so the first K tiles of the next tile are
// loaded during the last steps of the current one.
#include <mutex>
#include <type_traits>

#include "b128_dev.h"

namespace moe355 {

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;

constexpr int BM = 256, BN = 256, WN = 4, NWAVE = 8, kThreads = NWAVE * 64;
constexpr int SLOT = (BM + BN) * 64;
constexpr int MI = 4, NI = 2;     // 32-row blocks of a wave, at most, and blocks of 32 weight rows
constexpr int kFewItems = 1024;  // output tiles that are dealt to the XCDs by number
constexpr int GROUP_M = 4;        // row tiles that are walked across all columns together
constexpr uint32_t kNowhere = 0xfc000000u;  // byte offset past the end of every operand, also with a K tile's offset added

enum { kEpiPlain, kEpiRelu, kEpiSilu };

struct Tile {
    int row0, row_end, expert, n0;
};

// The same value in a scalar register, of which the optimiser knows nothing: a chain of tests on such values stays a chain.
__device__ __forceinline__ int opaque(int v)
{
    asm volatile("" : "+s"(v));
    return __builtin_amdgcn_readfirstlane(v);
}

// acc += w * a, in place: an accumulator that lives across basic blocks gets a second set of registers from the compiler.  What its hazard handling
// then no longer sees is padded by hand: accumulators are written by vector instructions at the head of a tile and read at its end; an operand that a
// vector instruction has written (a widened one, a scale, a copy where two blocks of code join) has two wait states behind it, the PAD.
template <bool PAD>
__device__ __forceinline__ void mfma_fp8(f32x16_t &acc, const Fragment &w, const Fragment &a, int sw, int sa)
{
    if constexpr (PAD)
        asm volatile("s_nop 1\n\tv_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]" : "+v"(acc) : "v"(w), "v"(a), "v"(sw), "v"(sa));
    else
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]" : "+v"(acc) : "v"(w), "v"(a), "v"(sw), "v"(sa));
}
template <bool PAD>
__device__ __forceinline__ void mfma_bf16(f32x16_t &acc, const bf16x8 &w, const bf16x8 &a)
{
    if constexpr (PAD)
        asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(w), "v"(a));
    else
        asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(w), "v"(a));
}

// 8 of a chunk's 16 bytes as bf16, times the scale
__device__ __forceinline__ bf16x8 widen8(const u32x4 &c, int q, float scale)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        w[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * q + i], scale, false));
        w[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * q + i], scale, true));
    }
    return __builtin_bit_cast(bf16x8, w);
}

}  // namespace

// DEEP: precise, with sums of sums
template <bool PRECISE, int EPI, bool DEEP>
__global__ __launch_bounds__(kThreads, 1) void gemm_b128_tile_kernel(GemmB128 g)
{
    constexpr int MOST = DEEP ? 2 : MI;  // 32-row blocks of a wave
    constexpr int SLOTS = PRECISE ? 4 : 5;
    constexpr int TILE_N = EPI == kEpiSilu ? BN / 2 : BN;  // columns of the result
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int K = g.K, KT = max((K + kBlock - 1) / kBlock, 2);  // two at least, for the load stream; the second may be all zeros
    const int n_tiles = (g.Nh + TILE_N - 1) / TILE_N;
    const int scale_cols = (int)b128_scale_cols(K), n_blocks = (g.Nh + kBlock - 1) / kBlock;

    // ---- the block's tiles.  Experts, 64 at a time, one per lane: rows, tiles along them, output tiles before it.
    int w_base = 0, w_pos = 0, w_total = 0;
    int w_row0, w_row_end, w_cuts, w_excl;
    int cap = MOST;  // height of a tile, in units of 64 rows
    auto load_window = [&]() __attribute__((always_inline)) {
        w_row0 = 0, w_row_end = 0;
        const int e = w_base + lane;
        if (e < g.E) {
            w_row_end = g.n_rows;
            if (g.offsets) {
                w_row0 = min(max(g.offsets[e], 0), g.n_rows);
                w_row_end = min(max(g.offsets[e + 1], w_row0), g.n_rows);
            }
        }
        const int units = (w_row_end - w_row0 + 63) >> 6;  // of 64 rows
        w_cuts = cap == 4 ? (units + 3) >> 2 : cap == 3 ? (units + 2) / 3 : cap == 2 ? (units + 1) >> 1 : units;
        int incl = w_cuts;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int up = __shfl_up(incl, off, 64);
            if (lane >= off) incl += up;
        }
        w_excl = (incl - w_cuts) * n_tiles;
        w_total = __builtin_amdgcn_readlane(incl, 63) * n_tiles;
    };
    // The height at which the rounds of all blocks take least: a round costs a K loop, whose K tiles take about so many units by a tile's height, and as much as six
    // more of its K tiles for its beginning and end.  Only ratios count here, so what every height has alike is left out: the launch, and the work before the first tile
    // (the choice between these tiles and gemm_b128_small.hip counts them, as three more).
    if (g.n_rows > 64) {
        int tiles[4] = {0, 0, 0, 0};
        for (w_base = 0; w_base < g.E; w_base += 64) {
            load_window();
            const int units = (w_row_end - w_row0 + 63) >> 6;
#pragma unroll
            for (int h = 1; h <= 4; ++h) tiles[h - 1] += (units + h - 1) / h;
        }
        float best = 0.f;
#pragma unroll
        for (int h = MOST; h >= (PRECISE ? 1 : 2); --h) {
            int n = tiles[h - 1];
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) n += __shfl_xor(n, off, 64);
            const float out = (float)n * (float)n_tiles, rounds = ceilf(out * (1.f / 256.f));
            const float t = rounds * (float)((KT + 6) * kTileTime[PRECISE][h - 1]);
            if (h == MOST || t < 0.97f * best) best = t, cap = h;
            if (h == MOST && rounds > 3.f) break;  // blocks of several rounds even out by themselves
        }
        cap = __builtin_amdgcn_readfirstlane(cap);
    }
    // What a window's expert costs, in units of 64 rows by a column tile: its rows, but half a full tile at least for the weights' stream, and as much
    // as three units for a tile's beginning and end.
    auto cost = [&]() __attribute__((always_inline)) -> float {
        const int units = (w_row_end - w_row0 + 63) >> 6;
        return (float)n_tiles * (float)(max(units, 2 * w_cuts) + 3 * w_cuts);
    };
    int pos, pos_last;
    {
        float total = 0.f;
        for (w_base = 0; w_base < g.E; w_base += 64) {
            load_window();
            float c = cost();
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) c += __shfl_xor(c, off, 64);
            total += c;
        }
        const int x = blockIdx.x & 7;
        const float from = total * (float)x * 0.125f, to = total * (float)(x + 1) * 0.125f;
        float before = 0.f;
        int items = 0, lo = -1, hi = -1;
        for (w_base = 0; w_base < g.E; w_base += 64) {
            load_window();
            const float c = cost();
            float incl = c;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const float up = __shfl_up(incl, off, 64);
                if (lane >= off) incl += up;
            }
            auto place = [&](float t, int &at) __attribute__((always_inline)) {
                const unsigned long long past = __ballot(before + incl > t && w_cuts > 0);
                if (at >= 0 || past == 0) return;
                const int src = __builtin_ctzll(past);
                const int n = __builtin_amdgcn_readlane(w_cuts, src) * n_tiles;
                const float first = before + (__shfl(incl, src, 64) - __shfl(c, src, 64));
                const int in = (int)((t - first) / __shfl(c, src, 64) * (float)n);
                at = items + __builtin_amdgcn_readlane(w_excl, src) + min(max(in, 0), n);
            };
            place(from, lo);
            place(to, hi);
            before += __shfl(incl, 63, 64);
            items += w_total;
        }
        lo = x == 0 ? 0 : lo < 0 ? items : lo;
        hi = x == 7 || hi < 0 ? items : hi;
        if (items <= kFewItems) {
            // few rounds: as many tiles for each XCD, or one of them has a round more (24 experts, 238 tiles: 46 us by cost, 25 by number)
            const int share = (items + 7) >> 3;
            lo = min(x * share, items);
            hi = min(lo + share, items);
        }
        pos = __builtin_amdgcn_readfirstlane(lo) + (blockIdx.x >> 3);
        pos_last = __builtin_amdgcn_readfirstlane(hi);
    }
    int pos_next = pos + 63 - 2 * (int)(blockIdx.x >> 3);  // every second round the other way round
    w_base = 0;
    load_window();
    Tile nx;  // the stream's next tile
    auto next_tile_pos = [&]() __attribute__((always_inline)) -> bool {
        if (pos >= pos_last) return false;
        while (pos - w_pos >= w_total) {
            w_pos += w_total;
            w_base += 64;
            if (w_base >= g.E) return false;
            load_window();
        }
        const int at = pos - w_pos;
        const int src = 63 - __builtin_clzll(__ballot(w_excl <= at && w_cuts > 0));
        const int row0 = __builtin_amdgcn_readlane(w_row0, src), row_end = __builtin_amdgcn_readlane(w_row_end, src);
        const int cuts = __builtin_amdgcn_readlane(w_cuts, src), units = (row_end - row0 + 63) >> 6;
        const int in = at - __builtin_amdgcn_readlane(w_excl, src);
        const int grp = in / (GROUP_M * n_tiles), within = in - grp * (GROUP_M * n_tiles);
        const int gsz = min(GROUP_M, cuts - grp * GROUP_M);
        const int nt = within / gsz, mt = grp * GROUP_M + within - nt * gsz;
        nx.expert = __builtin_amdgcn_readfirstlane(w_base + src);
        nx.n0 = __builtin_amdgcn_readfirstlane(nt * TILE_N);
        const int each = units / cuts, more = units - each * cuts;  // the first `more` tiles have a unit more
        const int first = row0 + 64 * (mt * each + min(mt, more));
        nx.row0 = __builtin_amdgcn_readfirstlane(first);
        nx.row_end = __builtin_amdgcn_readfirstlane(min(row_end, first + 64 * (each + (mt < more))));
        const int after = pos + 64;
        pos = pos_next;
        pos_next = after;
        return true;
    };
    if (!next_tile_pos()) return;

    f32x16_t acc[MI][NI];
    const int row32 = lane & 31, kg = lane >> 5, swz = (row32 >> 2) & 3;
    // chunk kg of a row, and (16 * (kg + 2) ^ ...: the same with bit 1 of the position turned) chunk kg + 2
    const int frag_off = row32 * 64 + ((kg ^ swz) << 4), frag_far = row32 * 64 + (((kg + 2) ^ swz) << 4);
    const uint8_t *const fragA = smem + wm * 2048;
    const uint8_t *const fragB = smem + BM * 64 + wn * 4096;
    auto chunk_of = [&](const uint8_t *frag, int slot, int at, int far) __attribute__((always_inline)) {
        return *reinterpret_cast<const u32x4 *>(frag + slot * SLOT + at + (far ? frag_far : frag_off));
    };
    auto read_a = [&](int slot, int mi) __attribute__((always_inline)) { return whole(chunk_of(fragA, slot, mi * 4096, 0), chunk_of(fragA, slot, mi * 4096, 1)); };
    auto read_b = [&](int slot, int ni) __attribute__((always_inline)) { return whole(chunk_of(fragB, slot, ni * 2048, 0), chunk_of(fragB, slot, ni * 2048, 1)); };

    // ---- load stream.  An offset past a buffer's end costs no memory traffic and fills zeros, which is what rows past a tile's end, weight rows past
    // the last and the chunks past K need.
    int l_kt = 0;
    bool l_more = true;
    int w_slot = 0;  // slot of the first half of the K tile the stream is at
    // A and its scales: all of them where rows are chosen by index, else from the tile's first row on
    __amdgpu_buffer_rsrc_t bufA = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(g.a), 0, (int)kNowhere, 0x00020000);
    __amdgpu_buffer_rsrc_t bufAS = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(g.a_scale), 0, (int)kNowhere, 0x00020000);
    __amdgpu_buffer_rsrc_t bufB = bufA, bufBS = bufAS;  // the expert's weights and their scales
    uint32_t a_voff[2], b_voff[2], as_voff[MI], bs_off[NI];
    const int ld_row = lane >> 2;                         // row inside a 16-row group
    const int ld_chunk = (lane & 3) ^ ((lane >> 4) & 3);  // chunk this lane fetches for its LDS position
    auto row_of = [&](int r) __attribute__((always_inline)) -> int {  // of bufA, of row r of the stream's tile
        const int in = min(r, nx.row_end - 1 - nx.row0);
        return g.a_rows ? min(max(g.a_rows[nx.row0 + in], 0), g.a_count - 1) : in;
    };
    auto set_ptrs = [&]() __attribute__((always_inline)) {
        const int64_t mats = (int64_t)nx.expert * (g.N / g.Nh);
        if (!g.a_rows) {
            bufA = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(g.a + (int64_t)nx.row0 * K), 0, (int)kNowhere, 0x00020000);
            bufAS = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(g.a_scale + (int64_t)nx.row0 * scale_cols), 0, (int)kNowhere, 0x00020000);
        }
        bufB = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(g.w + (int64_t)nx.expert * g.N * K), 0, (int)kNowhere, 0x00020000);
        bufBS = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(g.w_scale + mats * n_blocks * scale_cols), 0, (int)kNowhere, 0x00020000);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = (i * NWAVE + wave) * 16 + ld_row;
            a_voff[i] = nx.row0 + r < nx.row_end ? (uint32_t)row_of(r) * (uint32_t)K + ld_chunk * 16 : kNowhere;
            const int rho = (wave * 2 + i) * 16 + ld_row, x = rho & 31, c = 16 * ((x >> 2) & 1) + 4 * (x >> 3) + (x & 3);
            const int half = EPI == kEpiSilu ? (rho >> 5) & 1 : 0;
            const int col = nx.n0 + (EPI == kEpiSilu ? (rho >> 6) * 32 + c : (rho & ~31) + c);
            b_voff[i] = col < g.Nh ? (uint32_t)(half * g.Nh + col) * (uint32_t)K + ld_chunk * 16 : kNowhere;
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) as_voff[i] = (uint32_t)row_of((2 * i + wm) * 32 + row32) * (uint32_t)scale_cols;
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            const int block = EPI == kEpiSilu ? n * n_blocks + nx.n0 / kBlock : min((nx.n0 + wn * 64) / kBlock, n_blocks - 1);
            bs_off[n] = (uint32_t)__builtin_amdgcn_readfirstlane(block * scale_cols);
        }
    };
    auto issue = [&](__amdgpu_buffer_rsrc_t buf, uint32_t voff, int h, int lds_off) __attribute__((always_inline)) {
        int slot = w_slot + h;
        if (slot >= SLOTS) slot -= SLOTS;
        if (l_kt * kBlock + h * 64 + ld_chunk * 16 >= K) voff = kNowhere;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lds_void *)(smem + slot * SLOT + lds_off), 16, voff, l_kt * kBlock + h * 64, 0, 0);
    };
    auto issue_a = [&](int i, int h) __attribute__((always_inline)) { issue(bufA, a_voff[i], h, (i * NWAVE + wave) * 1024); };
    auto issue_b = [&](int i, int h) __attribute__((always_inline)) { issue(bufB, b_voff[i], h, BM * 64 + (wave * 2 + i) * 1024); };
    // scale bytes, those of four K tiles a word: of the K tile being multiplied in the lowest byte, and the next word
    int sa[MI], sb[NI], sa_next[MI], sb_next[NI];
    auto issue_scales = [&](int group) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MI; ++i) sa_next[i] = __builtin_amdgcn_raw_buffer_load_b32(bufAS, as_voff[i], group * 4, 0);
#pragma unroll
        for (int n = 0; n < NI; ++n) sb_next[n] = __builtin_amdgcn_raw_buffer_load_b32(bufBS, 0, bs_off[n] + group * 4, 0);
    };
    auto take_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MI; ++i) sa[i] = sa_next[i];
#pragma unroll
        for (int n = 0; n < NI; ++n) sb[n] = PRECISE ? __builtin_amdgcn_readfirstlane(sb_next[n]) : sb_next[n];  // the same in all lanes
    };
    auto landed_scales = [&]() __attribute__((always_inline)) {  // behind a wait that covers them: the compiler need not look for one later
#pragma unroll
        for (int i = 0; i < MI; ++i) asm volatile("" : "+v"(sa_next[i]));
#pragma unroll
        for (int n = 0; n < NI; ++n) asm volatile("" : "+v"(sb_next[n]));
    };
    auto next_k = [&]() __attribute__((always_inline)) {
        ++l_kt;
        w_slot += 2;
        if (w_slot >= SLOTS) w_slot -= SLOTS;
    };
    auto next_tile = [&]() __attribute__((always_inline)) {
        l_more = next_tile_pos();
        if (l_more) {
            l_kt = 0;
            set_ptrs();
        } else {
            l_kt = KT - 2;  // past the end: K tiles again, into slots nobody reads
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): no scalar load is in flight in the K loop, whose waits count LDS reads
    };
    // Words are asked for at the head of a K tile and have landed with the wait in its last step: this tile's next one where kt % 4 = 0, the next tile's
    // first one behind next_tile and behind the use of this tile's last.
    const int last_group = (KT - 1) >> 2, ask_next = max(KT - 2, 4 * last_group);
    auto ask_scales = [&](int kt) __attribute__((always_inline)) {
        if (kt == ask_next) issue_scales(0);
        else if ((kt & 3) == 0 && kt >> 2 < last_group) issue_scales((kt >> 2) + 1);
    };
    auto turn_scales = [&](int kt) __attribute__((always_inline)) {  // behind K tile kt
        if (kt == 0 && K <= kBlock) {  // a K tile of zeros, whatever byte stands there
#pragma unroll
            for (int i = 0; i < MI; ++i) sa[i] = 127;
#pragma unroll
            for (int n = 0; n < NI; ++n) sb[n] = 127;
        } else if (kt + 1 == KT || ((kt + 1) & 3) == 0) {
            take_scales();
        } else {
#pragma unroll
            for (int i = 0; i < MI; ++i) sa[i] = (int)((uint32_t)sa[i] >> 8);
#pragma unroll
            for (int n = 0; n < NI; ++n) sb[n] = (int)((uint32_t)sb[n] >> 8);
        }
    };

    // ---- results
    auto epilogue = [&](const Tile &ti, auto blocks) __attribute__((always_inline)) {
        constexpr int M = decltype(blocks)::value;
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");  // see mfma_fp8
#pragma unroll
        for (int mi = 0; mi < M; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) asm volatile("" : "+v"(acc[mi][ni]));
        if constexpr (EPI == kEpiPlain) {
            const bool f32 = g.c_dtype == MOE_DTYPE_F32;
            const uint32_t es = f32 ? 4 : 2;
            const __amdgpu_buffer_rsrc_t bufC =
                __builtin_amdgcn_make_buffer_rsrc(static_cast<uint8_t *>(g.c) + (int64_t)ti.row0 * g.N * es, 0, (int)kNowhere, 0x00020000);
            const int col = ti.n0 + wn * 64 + kg * 16;
#pragma unroll
            for (int mi = 0; mi < M; ++mi) {
                const int row = (2 * mi + wm) * 32 + row32;
                const bool row_live = ti.row0 + row < ti.row_end;
                const uint32_t off = ((uint32_t)row * (uint32_t)g.N + (uint32_t)col) * es;
#pragma unroll
                for (int ni = 0; ni < NI; ++ni) {
                    if (PRECISE && f32) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)  // N is a multiple of 8
                            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{acc[mi][ni][4 * j], acc[mi][ni][4 * j + 1], acc[mi][ni][4 * j + 2], acc[mi][ni][4 * j + 3]}), bufC,
                                                                   row_live && col + ni * 32 + 4 * j < g.N ? off + ni * 128 + 16 * j : kNowhere, 0, 0);
                    } else {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            u32x4 o;
#pragma unroll
                            for (int q = 0; q < 4; ++q) o[q] = pack_bf16(acc[mi][ni][8 * j + 2 * q], acc[mi][ni][8 * j + 2 * q + 1]);
                            __builtin_amdgcn_raw_buffer_store_b128(o, bufC, row_live && col + ni * 32 + 8 * j < g.N ? off + ni * 64 + 16 * j : kNowhere, 0, 0);
                        }
                    }
                }
            }
        } else {
            // h, its largest element over the block's 128 columns (16 or 32 a lane, two lanes, and 4 or 2 waves), and its bytes
            constexpr int H = EPI == kEpiSilu ? 16 : 32;
            uint32_t *const most = reinterpret_cast<uint32_t *>(smem + opaque(SLOTS * SLOT));  // [4][256]; addresses made here, not held across the K loop
            const int F = g.Nh, hidden_cols = (int)b128_scale_cols(F);
            const int first = ti.n0 + (EPI == kEpiSilu ? wn * 32 : wn * 64) + kg * 16;
            uint8_t *const hq = static_cast<uint8_t *>(g.c);
#pragma unroll
            for (int mi = 0; mi < M; ++mi) {
                Elements<false, H> h;
#pragma unroll
                for (int j = 0; j < H; ++j) h.x[j] = EPI == kEpiSilu ? silu<DEEP>(acc[mi][0][j & 15]) * acc[mi][1][j & 15] : relu(acc[mi][j >> 4][j & 15]);
                // in place: the sums are not needed any more
#pragma unroll
                for (int j = 0; j < H; ++j) acc[mi][j >> 4][j & 15] = h.x[j];
                uint32_t m = h.largest();
                if (m >= 0x7f800000u) {
                    m = h.largest_finite();
#pragma unroll
                    for (int j = 0; j < H; ++j) acc[mi][j >> 4][j & 15] = h.x[j];
                }
                m = lanes_max(m, 32);
                if (kg == 0) most[wn * 256 + (2 * mi + wm) * 32 + row32] = m;
            }
            __builtin_amdgcn_s_waitcnt(0xc07f);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int mi = 0; mi < M; ++mi) {
                const int row = (2 * mi + wm) * 32 + row32;
                uint32_t m = 0;
                if constexpr (EPI == kEpiSilu) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) m = max(m, *reinterpret_cast<const u32_lds *>(most + w * 256 + row));
                } else {
#pragma unroll
                    for (int w = 0; w < 2; ++w) m = max(m, *reinterpret_cast<const u32_lds *>(most + ((wn & 2) + w) * 256 + row));
                }
                const int byte = b128_scale_byte(m);
                if (ti.row0 + row >= ti.row_end) continue;
                Elements<false, H> h;
#pragma unroll
                for (int j = 0; j < H; ++j) h.x[j] = acc[mi][j >> 4][j & 15];
                const int64_t at = ti.row0 + row;
#pragma unroll
                for (int b = 0; b < H / 16; ++b)
                    if (first + 32 * b < F)  // F is a multiple of 16
                        *reinterpret_cast<uint4 *>(hq + at * F + first + 32 * b) = make_uint4(h.pack4(16 * b, scale_value(byte)), h.pack4(16 * b + 4, scale_value(byte)),
                                                                                              h.pack4(16 * b + 8, scale_value(byte)), h.pack4(16 * b + 12, scale_value(byte)));
                if (kg == 0 && (EPI == kEpiSilu ? wn == 0 : (wn & 1) == 0) && first < F) g.c_scale[at * hidden_cols + first / kBlock] = (uint8_t)byte;
            }
        }
    };
    auto zero_acc = [&](auto blocks) __attribute__((always_inline)) {
        constexpr int M = decltype(blocks)::value;
#pragma unroll
        for (int mi = 0; mi < M; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[mi][ni][r] = 0.f;
                asm volatile("" : "+v"(acc[mi][ni]));
            }
        asm volatile("s_nop 7");
    };

    int r_slot = 0;  // slot of the step being multiplied
    if constexpr (!PRECISE) {
        // a[M - 1 + P]: the last row block has a register set per step parity, so that its read for the next step goes out with the first ones
        Fragment a[MI + 1], w[2][NI];
        auto step = [&](auto parity, auto blocks) __attribute__((always_inline)) {
            constexpr int P = decltype(parity)::value, M = decltype(blocks)::value;
            constexpr int POST = (M - 1) * NI;
            auto mfma = [&](auto pad, int mi, int ni) __attribute__((always_inline)) {
                mfma_fp8<decltype(pad)::value>(acc[mi][ni], w[P][ni], a[mi == M - 1 ? mi + P : mi], sb[ni], sa[mi]);
            };
            mfma(std::true_type{}, 0, 0);
#pragma unroll
            for (int ni = 1; ni < NI; ++ni) mfma(std::false_type{}, 0, ni);
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("" ::: "memory");
            if (P == 1) {
                __builtin_amdgcn_s_waitcnt(0x0070 | 4);  // lgkmcnt(0), and at most the even step's loads in flight
                landed_scales();
            } else {
                __builtin_amdgcn_s_waitcnt(0xc07f);
            }
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            const int nslot = r_slot + 1 == SLOTS ? 0 : r_slot + 1;
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) w[P ^ 1][ni] = read_b(nslot, ni);
            a[0] = read_a(nslot, 0);
            a[M - 1 + (P ^ 1)] = read_a(nslot, M - 1);
            __builtin_amdgcn_sched_barrier(0);
            auto loads_at = [&](int at) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j * POST / 4 == at) {
                        if ((M <= 2) == (P == 0)) issue_a(j >> 1, j & 1);
                        else issue_b(j >> 1, j & 1);
                    }
            };
#pragma unroll
            for (int mi = 1; mi < M; ++mi)
#pragma unroll
                for (int ni = 0; ni < NI; ++ni) {
                    mfma(std::false_type{}, mi, ni);
                    if (ni == NI - 1 && mi < M - 1) a[mi] = read_a(nslot, mi);
                    loads_at((mi - 1) * NI + ni);
                    __builtin_amdgcn_sched_barrier(0);
                }
            r_slot = nslot;
            __builtin_amdgcn_sched_barrier(0);
        };
        auto run_tile = [&](const Tile &ti, auto blocks) __attribute__((always_inline)) {
            constexpr int M = decltype(blocks)::value;
            zero_acc(blocks);
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) w[0][ni] = read_b(r_slot, ni);
#pragma unroll
            for (int mi = 0; mi < M; ++mi) a[mi] = read_a(r_slot, mi);
            for (int kt = 0; kt < KT; ++kt) {
                if (kt == KT - 2) next_tile();
                ask_scales(kt);
                step(std::integral_constant<int, 0>{}, blocks);
                step(std::integral_constant<int, 1>{}, blocks);
                next_k();
                turn_scales(kt);
            }
            epilogue(ti, blocks);
        };
        Tile t = nx;
        set_ptrs();
        issue_scales(0);
#pragma unroll 1
        for (int rep = 0; rep < 2; ++rep) {
#pragma unroll
            for (int j = 0; j < 4; ++j) issue_b(j >> 1, j & 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) issue_a(j >> 1, j & 1);
            next_k();
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0f70 | 8);  // the first K tile and its scales have landed
        landed_scales();
        take_scales();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        while (true) {
            const int blocks = max(2, (t.row_end - t.row0 + 63) >> 6);
            if (opaque(blocks) == 4) run_tile(t, std::integral_constant<int, 4>{});
            if (opaque(blocks) == 3) run_tile(t, std::integral_constant<int, 3>{});
            if (opaque(blocks) == 2) run_tile(t, std::integral_constant<int, 2>{});
            if (!l_more) break;
            t = nx;
        }
    } else {
        u32x4 ra[2][MI], rb[2][NI];  // chunks of one phase (32 k) and of the next
        auto read_phase = [&](int set, int slot, int far, auto blocks) __attribute__((always_inline)) {
            constexpr int M = decltype(blocks)::value;
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) rb[set][ni] = chunk_of(fragB, slot, ni * 2048, far);
#pragma unroll
            for (int mi = 0; mi < M; ++mi) ra[set][mi] = chunk_of(fragA, slot, mi * 4096, far);
        };
        auto run_tile = [&](const Tile &ti, auto blocks) __attribute__((always_inline)) {
            constexpr int M = decltype(blocks)::value;
            zero_acc(blocks);
            f32x16_t sum[DEEP ? M : 1][NI] = {};
            read_phase(0, r_slot, 0, blocks);
            for (int kt = 0; kt < KT; ++kt) {
                if (kt == KT - 2) next_tile();
                float fa[M], fb[NI];
#pragma unroll
                for (int i = 0; i < M; ++i) fa[i] = scale_value(sa[i] & 255);
#pragma unroll
                for (int n = 0; n < NI; ++n) fb[n] = scale_value(sb[n] & 255);
                const int slot1 = r_slot + 1 == SLOTS ? 0 : r_slot + 1, slot2 = slot1 + 1 == SLOTS ? 0 : slot1 + 1;
                ask_scales(kt);
                // phases 0 .. 3: chunks kg and kg + 2 of the first half, of the second half
#pragma unroll
                for (int ph = 0; ph < 4; ++ph) {
                    constexpr int kLoads = 8;
                    if (ph == 3) {
                        // this wave's reads of the K tile are done, its loads of the next have landed; behind the barrier everybody's
                        __builtin_amdgcn_sched_barrier(0);
                        asm volatile("" ::: "memory");
                        __builtin_amdgcn_s_waitcnt(0x0070);
                        landed_scales();
                        __builtin_amdgcn_s_barrier();
                        asm volatile("" ::: "memory");
                        __builtin_amdgcn_sched_barrier(0);
                        read_phase(0, slot2, 0, blocks);
                    } else {
                        read_phase((ph + 1) & 1, ph == 0 ? r_slot : slot1, ph == 1 ? 0 : 1, blocks);
                    }
                    const int set = ph & 1;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        bf16x8 bw[NI];
#pragma unroll
                        for (int ni = 0; ni < NI; ++ni) bw[ni] = widen8(rb[set][ni], q, fb[ni]);
#pragma unroll
                        for (int mi = 0; mi < M; ++mi) {
                            const bf16x8 aw = widen8(ra[set][mi], q, fa[mi]);
                            mfma_bf16<true>(acc[mi][0], bw[0], aw);
                            mfma_bf16<false>(acc[mi][1], bw[1], aw);
                            if (ph == 3) {
                                const int at = q * M + mi;  // of 2 M
#pragma unroll
                                for (int j = 0; j < kLoads; ++j)
                                    if (j * 2 * M / kLoads == at) {
                                        if (j < 4) issue_b(j >> 1, j & 1);
                                        else issue_a((j - 4) >> 1, j & 1);
                                    }
                            }
                        }
                    }
                }
                next_k();
                r_slot = slot2;
                turn_scales(kt);
                if constexpr (DEEP) {
                    if ((kt & 1) || kt + 1 == KT) {
                        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");  // see mfma_fp8
#pragma unroll
                        for (int mi = 0; mi < M; ++mi)
#pragma unroll
                            for (int ni = 0; ni < NI; ++ni) {
                                asm volatile("" : "+v"(acc[mi][ni]));
                                sum[mi][ni] += acc[mi][ni];
                            }
                        zero_acc(blocks);
                    }
                }
            }
            if constexpr (DEEP) {
#pragma unroll
                for (int mi = 0; mi < M; ++mi)
#pragma unroll
                    for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = sum[mi][ni];
            }
            epilogue(ti, blocks);
        };
        Tile t = nx;
        set_ptrs();
        issue_scales(0);
#pragma unroll 1
        for (int rep = 0; rep < 2; ++rep) {
#pragma unroll
            for (int j = 0; j < 4; ++j) issue_b(j >> 1, j & 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) issue_a(j >> 1, j & 1);
            next_k();
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0f70 | 8);
        landed_scales();
        take_scales();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        while (true) {
            const int blocks = (t.row_end - t.row0 + 63) >> 6;
            if constexpr (!DEEP) {
                if (opaque(blocks) == 4) run_tile(t, std::integral_constant<int, 4>{});
                if (opaque(blocks) == 3) run_tile(t, std::integral_constant<int, 3>{});
            }
            if (opaque(blocks) == 2) run_tile(t, std::integral_constant<int, 2>{});
            if (opaque(blocks) == 1) run_tile(t, std::integral_constant<int, 1>{});
            if (!l_more) break;
            t = nx;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no LDS write may outlive the block
}

template <bool PRECISE, int EPI, bool DEEP = false>
static int launch_tile_as(const GemmB128 &g, hipStream_t s)
{
    const size_t smem = (PRECISE ? 4 : 5) * SLOT + (EPI != kEpiPlain ? 4 * 256 * 4 : 0);
    auto kern = gemm_b128_tile_kernel<PRECISE, EPI, DEEP>;
    static std::once_flag once;  // per instantiation
    static hipError_t setup_rc = hipSuccess;
    std::call_once(once, [&]() { setup_rc = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
    MOE_HIP_CHECK(setup_rc);
    hipLaunchKernelGGL(kern, dim3(256), dim3(kThreads), smem, s, g);
    MOE_LAUNCH_CHECK("gemm_b128_tile_kernel");
    return MOE_OK;
}

// The kernel addresses an expert's weights, a tile's rows of A, and all of A where rows are chosen by index, with 32-bit byte offsets, and counts output tiles
// in 32 bits.
bool b128_tiles_ok(const GemmB128 &g)
{
    return g.K <= 1 << 23 && g.N <= 1 << 20 && (!g.a_rows || (int64_t)g.a_count * g.K <= (int64_t)kNowhere) && (int64_t)g.N * g.K <= (int64_t)kNowhere &&
           ((int64_t)g.n_rows / 64 + g.E) * ceil_div(g.N, 128) < 1 << 30;
}

int launch_gemm_b128_tile(const GemmB128 &g, hipStream_t s)
{
    ProfScope ps(g.name ? g.name : "gemm_b128", s);
    if (g.act == kActSilu) return g.deep ? launch_tile_as<true, kEpiSilu, true>(g, s) : launch_tile_as<true, kEpiSilu>(g, s);
    if (g.act == kActRelu) return g.deep ? launch_tile_as<true, kEpiRelu, true>(g, s) : launch_tile_as<true, kEpiRelu>(g, s);
    return g.precise ? launch_tile_as<true, kEpiPlain>(g, s) : launch_tile_as<false, kEpiPlain>(g, s);
}

}  // namespace moe355
