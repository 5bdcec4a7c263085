// Position rotation of new queries and keys, and the new keys and values into a paged cache of e4m3 bytes with one
// power-of-two scale per (page, key head).
//
// One launch.  Blocks of the first kind own a (sequence, page that its new tokens touch, key head): they hold the new rows
// of the page in registers, take the largest element, settle the page's scale and write the bytes, so the rows are read
// once.  Blocks of the second kind turn queries.  Work items are 16 elements of a row, eight pairs that turn together: the
// angle of a pair is computed once for both of its elements.
//
// Angles are position * frequency in 64 bits: at position 10^5 an fp32 product is off by 4e-3 rad, more than bf16 keeps.  sin and
// cos of the remainder too, by their series over an eighth of a turn (below), so the rotated key is the fp32 number nearest to
// the exact one nearly always, and a page's scale does not depend on how the rotation was computed.
//
// Bound by HBM for many tokens, by latency for few.  Measured: 24 sequences, 6272 tokens, 16 heads of 128, half of them turned: 37 us for 128 MB,
// 3.5 TB/s (a large copy: 4.8); 256 sequences of one token, 32 / 8 heads of 128: 7.9 us; one token: 4.8.
#include "attn_internal.h"

namespace moe355 {

namespace {

// cos and sin of an angle in radians: the turns t = angle / (2 pi) less the nearest quarter, r in [-1/8, 1/8], then the Taylor
// series of sin and cos at x = 2 pi r, |x| <= pi/4: the first terms left out are x^15 / 15! = 2e-14 and x^14 / 14! = 4e-13.
// The product angle / (2 pi) is kept with its rounding error: alone it would be off by 1e-10 radians at angles of 1e6.
__device__ __forceinline__ void cos_sin(double angle, double &c, double &s)
{
    const double kTurn = 0.15915494309189535, kTurnLow = -9.839338337591243e-18;  // 1 / (2 pi) in two parts
    const double t = angle * kTurn;
    const double rest = fma(angle, kTurnLow, fma(angle, kTurn, -t));
    const double quarter = rint(t * 4.0);
    const double x = (fma(quarter, -0.25, t) + rest) * 6.28318530717958647693;
    const double z = x * x;
    double sp = 1.0 / 6227020800.0;
    sp = fma(sp, z, -1.0 / 39916800.0);
    sp = fma(sp, z, 1.0 / 362880.0);
    sp = fma(sp, z, -1.0 / 5040.0);
    sp = fma(sp, z, 1.0 / 120.0);
    sp = fma(sp, z, -1.0 / 6.0);
    sp = fma(sp * z, x, x);
    double cp = 1.0 / 479001600.0;
    cp = fma(cp, z, -1.0 / 3628800.0);
    cp = fma(cp, z, 1.0 / 40320.0);
    cp = fma(cp, z, -1.0 / 720.0);
    cp = fma(cp, z, 1.0 / 24.0);
    cp = fma(cp, z, -0.5);
    cp = fma(cp, z, 1.0);
    // which quarter: quarter is a whole number below 2^53, its two lowest bits say
    const int n = (int)(quarter - 4.0 * floor(quarter * 0.25));
    const double a = n & 1 ? sp : cp, b = n & 1 ? cp : sp;
    c = (n == 1 || n == 2) ? -a : a;
    s = n >= 2 ? -b : b;
}

// eight elements as they lie in memory
template <bool BF16>
struct Raw {
    uint4 q[BF16 ? 1 : 2];
};
template <bool BF16>
__device__ __forceinline__ Raw<BF16> load8(const void *p, int64_t at)
{
    Raw<BF16> r;
    const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p) + at * (BF16 ? 2 : 4));
    r.q[0] = src[0];
    if (!BF16) r.q[BF16 ? 0 : 1] = src[1];
    return r;
}
template <bool BF16>
__device__ __forceinline__ void floats(const Raw<BF16> &r, float (&v)[8])
{
    const uint4 a = r.q[0], b = r.q[BF16 ? 0 : 1];
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(!BF16 ? w[i] : i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
}

template <bool BF16>
__device__ __forceinline__ void store8(void *p, int64_t at, const float (&v)[8])
{
    if (BF16) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t lo = __float_as_uint(v[2 * i]), hi = __float_as_uint(v[2 * i + 1]);
            lo += 0x7fffu + ((lo >> 16) & 1u);
            hi += 0x7fffu + ((hi >> 16) & 1u);
            w[i] = (lo >> 16) | (hi & 0xffff0000u);
        }
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        *reinterpret_cast<float4 *>(static_cast<float *>(p) + at) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(static_cast<float *>(p) + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// Where the 16 elements of item e of a row lie: two groups of eight, and whether they turn.  The eight angles are
// inv_freq[8 e .. 8 e + 7] in both forms of pairing.
struct Item {
    int a, b;
    bool turns;
};
__device__ __forceinline__ Item item_of(int e, int rot_dim, int interleaved)
{
    const bool turns = 16 * e < rot_dim;
    if (turns && !interleaved) return {8 * e, 8 * e + rot_dim / 2, true};
    return {16 * e, 16 * e + 8, turns};
}

// x, y: the two groups.  Half apart: (x[i], y[i]) turn by angle i.  Interleaved: (x[0], x[1]), .. , (y[6], y[7]).
__device__ __forceinline__ void turn(float (&x)[8], float (&y)[8], const double (&c)[8], const double (&s)[8], int interleaved)
{
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double p = x[2 * i], q = x[2 * i + 1], u = y[2 * i], w = y[2 * i + 1];
            x[2 * i] = (float)(p * c[i] - q * s[i]);
            x[2 * i + 1] = (float)(q * c[i] + p * s[i]);
            y[2 * i] = (float)(u * c[4 + i] - w * s[4 + i]);
            y[2 * i + 1] = (float)(w * c[4 + i] + u * s[4 + i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double p = x[i], q = y[i];
            x[i] = (float)(p * c[i] - q * s[i]);
            y[i] = (float)(q * c[i] + p * s[i]);
        }
    }
}

__device__ __forceinline__ void angles(const double *inv_freq, int e, int pos, double (&c)[8], double (&s)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) cos_sin((double)pos * inv_freq[8 * e + i], c[i], s[i]);
}

// Exponent n of the smallest power of two 2^n >= 2^-126 with largest <= 448 * 2^n, without a division: largest = m 2^e with
// m in [0.5, 1) and 448 = 0.875 * 2^9.
__device__ __forceinline__ int needed_exponent(float largest)
{
    if (!(largest > 0.f)) return -126;
    int e;
    const float m = frexpf(largest, &e);
    const int n = m <= 0.875f ? e - 9 : e - 8;
    return min(max(n, -126), 120);
}
__device__ __forceinline__ float two_to(int n) { return __uint_as_float((uint32_t)(n + 127) << 23); }  // -126 <= n <= 127

__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ uint2 to_e4m3(const float (&v)[8], float inv)
{
    return make_uint2(to_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv), to_e4m3(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
}

// rows below r0 of a page of one head, scale s_old, rounded anew for s_new
__device__ __forceinline__ void round_anew(uint8_t *page, int bytes, float ratio, int tid, int threads)
{
    for (int i = tid * 4; i < bytes; i += threads * 4) {
        uint32_t *w = reinterpret_cast<uint32_t *>(page + i);
        typedef __attribute__((ext_vector_type(2))) float f32x2_t;
        const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)*w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)*w, true);
        *w = to_e4m3(lo.x * ratio, lo.y * ratio, hi.x * ratio, hi.y * ratio);
    }
}

// Heads of queries a thread turns by the same angles: their loads are in flight together, the angles' 40 operations in 64 bits a pair shared.
constexpr int kQHeads = 4;

// A sequence's new tokens; its keys end with the last of them.
__device__ __forceinline__ Seq load_new(const AttnParams &p, int b)
{
    int lo = p.q_offsets[b], hi = p.q_offsets[b + 1];
    lo = min(max(lo, 0), p.T);
    hi = min(max(hi, lo), p.T);
    const int begin = min(max(p.kv_len[b], 0), p.room) - (hi - lo), n = min(hi - lo, p.max_q);
    return {lo, n, begin + n, begin};
}

// Pages that a sequence's new tokens touch, and the first of them.
__device__ __forceinline__ int pages_of(const AttnParams &p, const Seq &sq, int &first)
{
    const int lo = max(sq.begin, 0);
    first = lo >> p.page_shift;
    return sq.kv > lo ? ((sq.kv - 1) >> p.page_shift) - first + 1 : 0;
}

// The sequence of the index-th touched page of all, and which of its pages that is: every wave adds up the sequences' pages, 64 at a
// time.  -1: there are not so many.
__device__ __forceinline__ int page_owner(const AttnParams &p, int index, int &m)
{
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < p.B; base += 64) {
        int first, sum = 0;
        if (base + lane < p.B) sum = pages_of(p, load_new(p, base + lane), first);
        const int mine = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(sum, off, 64);
            if (lane >= off) sum += o;
        }
        const unsigned long long past = __ballot(sum > index);
        if (past) {
            const int owner = __ffsll(past) - 1;
            m = index - __shfl(sum - mine, owner, 64);
            return base + owner;
        }
        index -= __shfl(sum, 63, 64);
    }
    return -1;
}

// NT threads, each with at most U items of a page's keys and values.  kv_units: blocks of the first kind; pages: 0 where these are
// counted over the pages that are touched, else pages of a sequence at most (a decoder step: one, and nothing has to be added up).
template <int DH, bool BF16, int NT, int U>
__global__ __launch_bounds__(NT) void kv_append_kernel(AppendParams p, int kv_units, int pages)
{
    static constexpr int kItems = DH / 16;
    const int unit = blockIdx.x;
    const int tid = threadIdx.x;
    if (unit >= kv_units) {  // queries: an item of a token, the same of kQHeads heads
        const int64_t at = (int64_t)(unit - kv_units) * NT + tid, per_group = (int64_t)p.a.T * kItems;
        const int group = (int)(at / per_group), item = (int)(at - group * per_group), t = item / kItems, e = item - t * kItems;
        if (group * kQHeads >= p.a.n_heads) return;
        int lo = 0, hi = p.a.B;  // the last sequence that begins at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (p.a.q_offsets[mid] <= t) lo = mid;
            else hi = mid;
        }
        const Seq sq = load_new(p.a, lo);
        const int i = t - sq.first;
        if (i < 0 || i >= sq.n) return;
        const Item it = item_of(e, p.rot_dim, p.interleaved);
        Raw<BF16> rx[kQHeads], ry[kQHeads];
#pragma unroll
        for (int k = 0; k < kQHeads; ++k) {
            const int h = min(group * kQHeads + k, p.a.n_heads - 1);
            rx[k] = load8<BF16>(p.a.q, (int64_t)t * p.a.q_stride + (int64_t)h * DH + it.a);
            ry[k] = load8<BF16>(p.a.q, (int64_t)t * p.a.q_stride + (int64_t)h * DH + it.b);
        }
        double c[8], s[8];
        if (it.turns) angles(p.inv_freq, e, sq.begin + i, c, s);
#pragma unroll
        for (int k = 0; k < kQHeads; ++k) {
            const int h = group * kQHeads + k;
            if (h >= p.a.n_heads) break;
            float x[8], y[8];
            floats<BF16>(rx[k], x);
            floats<BF16>(ry[k], y);
            if (it.turns) turn(x, y, c, s, p.interleaved);
            store8<BF16>(p.q_out, ((int64_t)t * p.a.n_heads + h) * DH + it.a, x);
            store8<BF16>(p.q_out, ((int64_t)t * p.a.n_heads + h) * DH + it.b, y);
        }
        return;
    }
    const int page_size = 1 << p.a.page_shift;
    const int index = unit / p.a.n_kv_heads, h = unit - index * p.a.n_kv_heads;
    int m = 0, b = index;
    if (!pages) b = page_owner(p.a, index, m);
    else if (pages > 1) b = index / pages, m = index - b * pages;
    if (b < 0) return;
    const Seq sq = load_new(p.a, b);
    int slot;
    if (m >= pages_of(p.a, sq, slot)) return;
    slot += m;
    const int lo = max(max(sq.begin, 0), slot << p.a.page_shift), hi = min(sq.kv, (slot + 1) << p.a.page_shift);
    if (lo >= hi || slot >= p.a.max_pages) return;
    const int r0 = lo - (slot << p.a.page_shift), rows = hi - lo, items = rows * kItems;
    // the new rows, and beside them the page and its scales
    Raw<BF16> rx[U], ry[U];
    Item it[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int id = min(tid + u * NT, 2 * items - 1);
        const bool is_v = id >= items;
        const int r = (is_v ? id - items : id) / kItems, e = (is_v ? id - items : id) - r * kItems;
        it[u] = is_v ? Item{16 * e, 16 * e + 8, false} : item_of(e, p.rot_dim, p.interleaved);
        const int64_t t = sq.first + (lo - sq.begin) + r;
        const void *src = is_v ? p.v_new : p.k_new;
        const int64_t at = t * (is_v ? p.v_stride : p.k_stride) + (int64_t)h * DH;
        rx[u] = load8<BF16>(src, at + it[u].a);
        ry[u] = load8<BF16>(src, at + it[u].b);
    }
    const int page = p.a.page_table[(int64_t)b * p.a.max_pages + slot];
    if (page < 0 || page >= p.a.num_pages) return;
    const int64_t unit_at = (int64_t)page * p.a.n_kv_heads + h;
    const float old_k = p.a.k_scale[unit_at], old_v = p.a.v_scale[unit_at];

    float x[U][8], y[U][8];
    float top_k = 0.f, top_v = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int id = tid + u * NT;
        if (id >= 2 * items) continue;
        const bool is_v = id >= items;
        floats<BF16>(rx[u], x[u]);
        floats<BF16>(ry[u], y[u]);
        if (it[u].turns) {
            const int r = id / kItems, e = id - r * kItems;
            double c[8], s[8];
            angles(p.inv_freq, e, lo + r, c, s);
            turn(x[u], y[u], c, s, p.interleaved);
        }
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fmaxf(fabsf(x[u][i]), fabsf(y[u][i])));
        top_k = fmaxf(top_k, is_v ? 0.f : top);
        top_v = fmaxf(top_v, is_v ? top : 0.f);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        top_k = fmaxf(top_k, __shfl_xor(top_k, off, 64));
        top_v = fmaxf(top_v, __shfl_xor(top_v, off, 64));
    }
    if (NT > 64) {
        __shared__ float part[2][NT / 64 + 1];
        if ((tid & 63) == 0) {
            part[0][tid >> 6] = top_k;
            part[1][tid >> 6] = top_v;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) {
            top_k = fmaxf(top_k, part[0][w]);
            top_v = fmaxf(top_v, part[1][w]);
        }
    }
    const int need_k = needed_exponent(top_k), need_v = needed_exponent(top_v);
    const float s_k = r0 ? fmaxf(old_k, two_to(need_k)) : two_to(need_k);
    const float s_v = r0 ? fmaxf(old_v, two_to(need_v)) : two_to(need_v);
    uint8_t *kp = p.a.k + unit_at * page_size * DH, *vp = p.a.v + unit_at * page_size * DH;
    const float inv_k = 1.f / s_k, inv_v = 1.f / s_v;  // powers of two: exact
    if (r0 && s_k > old_k) round_anew(kp, r0 * DH, old_k * inv_k, tid, NT);
    if (r0 && s_v > old_v) round_anew(vp, r0 * DH, old_v * inv_v, tid, NT);
    if (tid == 0) {
        p.a.k_scale[unit_at] = s_k;
        p.a.v_scale[unit_at] = s_v;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int id = tid + u * NT;
        if (id >= 2 * items) continue;
        const bool is_v = id >= items;
        const int r = (is_v ? id - items : id) / kItems;
        uint8_t *row = (is_v ? vp : kp) + (int64_t)(r0 + r) * DH;
        const float inv = is_v ? inv_v : inv_k;
        *reinterpret_cast<uint2 *>(row + it[u].a) = to_e4m3(x[u], inv);
        *reinterpret_cast<uint2 *>(row + it[u].b) = to_e4m3(y[u], inv);
    }
}

template <int DH, bool BF16, int NT, int U>
int launch_as(const AppendParams &p, hipStream_t s)
{
    // touched pages: at most (n - 2) / page_size + 2 of each sequence, and T / page_size + 2 B of all
    const int page_size = 1 << p.a.page_shift;
    const int each = (p.a.max_q + page_size - 2) / page_size + 1;
    const int64_t all = (int64_t)p.a.T / page_size + 2 * p.a.B;
    const bool counted = (int64_t)each * p.a.B > all;
    const int64_t kv_units = (counted ? all : (int64_t)each * p.a.B) * p.a.n_kv_heads;
    const int64_t q_units = p.a.q ? ((int64_t)ceil_div(p.a.n_heads, kQHeads) * p.a.T * (DH / 16) + NT - 1) / NT : 0;
    const int64_t blocks = kv_units + q_units;
    if (blocks >= (1ll << 31)) {
        set_error("moe_kv_append: %lld blocks", (long long)blocks);
        return MOE_ERR_INVALID_ARG;
    }
    hipLaunchKernelGGL((kv_append_kernel<DH, BF16, NT, U>), dim3((unsigned)blocks), dim3(NT), 0, s, p, (int)kv_units, counted ? 0 : each);
    MOE_LAUNCH_CHECK("kv_append_kernel");
    return MOE_OK;
}

template <int DH, bool BF16>
int launch_sized(const AppendParams &p, hipStream_t s)
{
    const int rows = p.a.max_q < (1 << p.a.page_shift) ? p.a.max_q : 1 << p.a.page_shift;
    const int items = 2 * rows * (DH / 16);  // of keys and values in a block
    // A key's and a value's item a thread, so that a block's loads are all in flight at once; 124 registers leave room for four waves a SIMD (fp32: 148,
    // three).  Blocks of 1024 threads have 128 a thread: fp32 spills 24 of them, four items a thread (pages of 128 rows of 256) 56, fp32 104.
    if (items <= 64) return launch_as<DH, BF16, 64, 1>(p, s);
    if (items <= 128) return launch_as<DH, BF16, 64, 2>(p, s);
    if (items <= 512) return launch_as<DH, BF16, 256, 2>(p, s);
    if (items <= 1024) return launch_as<DH, BF16, 512, 2>(p, s);
    if (items <= 2048) return launch_as<DH, BF16, 1024, 2>(p, s);
    return launch_as<DH, BF16, 1024, 4>(p, s);
}

}  // namespace

int launch_kv_append(int dtype, int head_dim, const AppendParams &p, hipStream_t s)
{
    const bool bf = dtype == MOE_DTYPE_BF16;
    if (head_dim == 64) return bf ? launch_sized<64, true>(p, s) : launch_sized<64, false>(p, s);
    if (head_dim == 128) return bf ? launch_sized<128, true>(p, s) : launch_sized<128, false>(p, s);
    return bf ? launch_sized<256, true>(p, s) : launch_sized<256, false>(p, s);
}

}  // namespace moe355
