// Selection of experts from logits: scores, a bias that moves the selection and not the weights, groups, top-k, weights.
//
//   s_e = 1 / (1 + exp(-l_e))  or  exp(l_e - max l) / sum exp(l - max l);   key_e = s_e + b_e
// in 64 bits: two keys that differ are then told apart as any other 64-bit program tells them (in 32 bits a large part of the
// scores near 1 would be equal), and equal ones go to the lower index.  An expert without a key (logit -infinity or NaN, or bias
// -infinity or NaN) is ordered behind all others and has weight 0.
//
// Few tokens: one wave a token (select_kernel), whose lanes hold the 64-bit keys of E / 64 experts each and find the largest k times.
//
// Many tokens: four lanes a token (select_many_kernel), 16 tokens a wave with their logits in LDS.  A lane goes through every fourth expert with
// 32-bit keys and keeps the k + 2 largest in a sorted list; the four lists become one, whose entries get 64-bit keys and are ranked by them.
// What the 32-bit keys may have decided wrongly -- the last group that stays against the first that does not, the k-th key against what fell
// off the list -- is checked with their error bound; a token that fails is done again by the whole wave as above.  Of normally distributed
// logits fewer than one in a thousand fail; of logits with many equal ones at the border, all may.
// Bound by issuing vector instructions (the lists, mostly), not by memory, and by how few waves LDS leaves a CU where there are many experts (16 rows of logits a wave: 16 waves
// at 128 experts, 8 at 256, 4 at 512, 2 at 1024).  One wave a token / four lanes a token, us, launches of a graph one after the other: 65536 x 128 experts, 8 groups, k = 6
// 156 / 32 (fp32, sigmoid), 170 / 44 (softmax), 203 / 63 (256 experts), 399 / 225 (512 experts, k = 8), 955 / 711 (1024 experts, k = 8), 58 / 17 (128 experts, no groups, k = 2);
// 8192 tokens 24 / 19, 26 / 27, 30 / 24, 56 / 63, 119 / 115, 10.4 / 9.0; 6144 tokens 20 / 20, 21 / 23, 24 / 26, 43 / 61, 89 / 103, 8.6 / 9.0; 4096 tokens 15 / 17, 16 / 25, 17 / 24,
// 33 / 62, 61 / 96, 6.8 / 7.8.  One lane a token, 64 a wave: 55 for the first, as it leaves a wave a SIMD.
#include <mutex>
#include <type_traits>

#include "b128_internal.h"

namespace moe355 {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kManyFrom = 6144;  // tokens: about where either takes as long with up to 256 experts; with more that is at 8192 and later
constexpr int kManyTokens = 16;  // of a wave of select_many_kernel
// words from row to row there: four lanes of a token read four neighbours, and the rows of 16 tokens lie four banks apart
__host__ __device__ constexpr int many_row(int E) { return (E + 59) / 64 * 64 + 4; }
// words for keys or groups' sums
__host__ __device__ inline int many_groups(const SelectParams &p) { return p.kept == p.groups ? 0 : 2 * p.E > p.groups * kManyTokens ? 2 * p.E : p.groups * kManyTokens; }
typedef unsigned long long u64;

// Keys as whole numbers in the same order; 0: no key.
__device__ __forceinline__ u64 ordered(double key)
{
    if (!(key > -INFINITY)) return 0;
    const u64 b = (u64)__double_as_longlong(key);
    return b >> 63 ? ~b : b | 1ull << 63;
}

template <bool BF16>
__device__ __forceinline__ float logit(const void *row, int e)
{
    return BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(row)[e] << 16) : static_cast<const float *>(row)[e];
}

__device__ __forceinline__ double sigmoid(float l) { return 1. / (1. + exp(-(double)l)); }

// One token by a wave.  l: logits of the lane's experts lane + 64 i, -infinity past the last; keys: room for E numbers, of this wave alone.
// All waves of a block come here together.
template <int V>
__device__ __forceinline__ void select_token(const SelectParams &p, const float (&l)[V], double *keys, int64_t t, bool live)
{
    const int lane = threadIdx.x & 63, E = p.E, size = E / p.groups;
    double s[V];
    u64 key[V];
    if (p.softmax) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < V; ++i) top = fmaxf(top, l[i]);
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        double sum = 0.;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s[i] = l[i] == -INFINITY ? 0. : l[i] == top ? 1. : top == INFINITY ? 0. : exp((double)l[i] - (double)top);
            sum += s[i];
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = sum > 0. ? s[i] / sum : 0.;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = sigmoid(l[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane + 64 * i;
        const double k = e < E && l[i] != -INFINITY ? s[i] + (p.bias ? (double)p.bias[e] : 0.) : -INFINITY;
        key[i] = ordered(k);
        if (key[i] == 0) s[i] = 0.;
        if (p.kept < p.groups && e < E) keys[e] = key[i] ? k : -INFINITY;
    }
    u64 groups = ~0ull;
    if (p.kept < p.groups) {
        // a lane a group
        __syncthreads();
        double best = -INFINITY, second = -INFINITY;
        if (lane < p.groups)
            for (int j = 0; j < size; ++j) {
                const double k = keys[lane * size + j];
                second = fmax(second, fmin(best, k));
                best = fmax(best, k);
            }
        const u64 score = lane < p.groups ? ordered(p.group_top == 2 && second > -INFINITY ? best + second : best) : 0;
        int before = 0;
        for (int g = 0; g < p.groups; ++g) {
            const u64 other = __shfl(score, g, 64);
            before += other > score || (other == score && g < lane);
        }
        groups = __ballot(lane < p.groups && before < p.kept);
        __syncthreads();
    }
    // index of an expert that is still to be had, E of one that is not
    int at[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane + 64 * i;
        at[i] = e < E && groups >> (p.kept < p.groups ? e / size : 0) & 1 ? e : E;
        if (at[i] == E) key[i] = 0;
    }
    int chosen = 0;
    double weight = 0., total = 0.;
    for (int j = 0; j < p.k; ++j) {
        u64 k = 0;
        int e = E;
        double w = 0.;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (key[i] > k || (key[i] == k && at[i] < e)) k = key[i], e = at[i], w = s[i];
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) {
            const u64 ok = __shfl_xor(k, off, 64);
            const int oe = __shfl_xor(e, off, 64);
            const double ow = __shfl_xor(w, off, 64);
            if (ok > k || (ok == k && oe < e)) k = ok, e = oe, w = ow;
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (at[i] == e) at[i] = E, key[i] = 0;
        total += w;
        if (lane == j) chosen = e, weight = w;
    }
    if (live && lane < p.k) {
        if (p.renorm) weight = total > 0. ? weight / total : 0.;
        p.idx[t * p.k + lane] = chosen;
        p.w[t * p.k + lane] = (float)(weight * (double)p.scale);
    }
}

// V: experts of a lane, e = lane + 64 i
template <bool BF16, int V>
__global__ __launch_bounds__(kThreads) void select_kernel(SelectParams p)
{
    __shared__ double keys[kWaves][V * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t t0 = (int64_t)blockIdx.x * kWaves; t0 < p.T; t0 += (int64_t)gridDim.x * kWaves) {
        const int64_t t = t0 + wave;
        const bool live = t < p.T;
        const void *row = static_cast<const char *>(p.logits) + (live ? t : 0) * p.stride * (BF16 ? 2 : 4);
        float l[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = lane + 64 * i;
            l[i] = e < p.E ? logit<BF16>(row, e) : -INFINITY;
            if (!BF16 && p.n_parts > 0 && e < p.E && live) {
                for (int j = 0; j < p.n_parts; ++j) l[i] += p.parts[j * p.part_stride + t * p.E + e];
                p.sum_out[t * p.E + e] = l[i];
            }
            if (l[i] != l[i]) l[i] = -INFINITY;
        }
        select_token<V>(p, l, keys[wave], t, live);
    }
}

// n rows of logits from row t0 to LDS, N elements a load; NaN as -infinity.  Unrolled: so many loads are on their way at once.
template <bool BF16, int N>
__device__ __forceinline__ void load_rows(const SelectParams &p, int64_t t0, int n, int ld, float *rows)
{
    constexpr int U = N == 1 ? 16 : 8;
    const int lane = threadIdx.x, per = p.E / N, total = n * per;
    int row = lane / per, col = lane - row * per;  // of vector lane, lane + 64, ...
    const int step_row = 64 / per, step_col = 64 - step_row * per;
    for (int i = lane; i < total;) {
        uint32_t x[U][N == 1 ? 1 : 4];
        int at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            at[u] = i < total ? row * ld + col * N : -1;
            const char *from = static_cast<const char *>(p.logits) + ((t0 + (i < total ? row : 0)) * p.stride + col * N) * (BF16 ? 2 : 4);
            if constexpr (N == 1) {
                x[u][0] = BF16 ? (uint32_t)*reinterpret_cast<const uint16_t *>(from) << 16 : *reinterpret_cast<const uint32_t *>(from);
            } else {
                const uint4 v = *reinterpret_cast<const uint4 *>(from);
                x[u][0] = v.x, x[u][1] = v.y, x[u][2] = v.z, x[u][3] = v.w;
            }
            i += 64;
            row += step_row;
            col += step_col;
            if (col >= per) col -= per, ++row;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (at[u] >= 0) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const uint32_t w = x[u][BF16 ? j / 2 : j];
                    const float f = __uint_as_float(!BF16 || N == 1 ? w : j & 1 ? w & 0xffff0000u : w << 16);
                    rows[at[u] + j] = f == f ? f : -INFINITY;
                }
            }
    }
}

// The value of the lane 1 or 2 over, of the four lanes of a token.
template <int BY>
__device__ __forceinline__ uint32_t over(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, BY == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true); }
template <int BY>
__device__ __forceinline__ float over(float x) { return __uint_as_float(over<BY>(__float_as_uint(x))); }
template <int BY>
__device__ __forceinline__ u64 over(u64 x) { return (u64)over<BY>((uint32_t)(x >> 32)) << 32 | over<BY>((uint32_t)x); }

// V: experts of a lane where a token is done again, E / 64 at least; KL: entries of a token's list, k + 2 at least
template <bool BF16, int V, int KL>
__global__ __launch_bounds__(64) void select_many_kernel(SelectParams p)
{
    constexpr int R = kManyTokens, S = 64 / R, OWN = (KL + S - 1) / S;  // tokens, lanes of one, and entries of the list that a lane settles
    extern __shared__ __align__(16) float smem[];
    const int lane = threadIdx.x, r = lane / S, q = lane % S, E = p.E, size = E / p.groups;
    const int ld = many_row(E);
    float *const rows = smem;                                         // [R][ld]
    double *const keys = reinterpret_cast<double *>(rows + R * ld);   // [E], for a token done again, behind the use of
    float *const of_group = rows + R * ld;                            // [G][R]; both only with groups
    float *const bias = rows + R * ld + many_groups(p);               // [E]
    const bool grouped = p.kept < p.groups;
    const bool by_logit = !p.bias && !grouped;  // without a bias keys are ordered as logits are, where they differ at all
    const bool wide = E % (BF16 ? 8 : 4) == 0 && p.stride % (BF16 ? 8 : 4) == 0 && reinterpret_cast<uintptr_t>(p.logits) % 16 == 0;
    for (int e = lane; e < E; e += 64) bias[e] = p.bias ? p.bias[e] : 0.f;
    for (int64_t t0 = (int64_t)blockIdx.x * R; t0 < p.T; t0 += (int64_t)gridDim.x * R) {
        const int n = (int)min((int64_t)R, p.T - t0);
        __syncthreads();
        if (wide) load_rows<BF16, BF16 ? 8 : 4>(p, t0, n, ld, rows);
        else load_rows<BF16, 1>(p, t0, n, ld, rows);
        __syncthreads();
        const bool live = r < n;
        const float *const mine = rows + (live ? r : 0) * ld;
        float top = 0.f;
        double sum = 1.;
        if (p.softmax) {
            top = -INFINITY;
            for (int e = q; e < E; e += S) top = fmaxf(top, mine[e]);
            top = fmaxf(top, over<1>(top));
            top = fmaxf(top, over<2>(top));
            if (p.bias || grouped || !p.renorm) {
                sum = 0.;
#pragma unroll 2
                for (int e = q; e < E; e += S) sum += mine[e] == -INFINITY ? 0. : exp((double)mine[e] - (double)top);
                sum += __longlong_as_double((long long)over<1>((u64)__double_as_longlong(sum)));
                sum += __longlong_as_double((long long)over<2>((u64)__double_as_longlong(sum)));
            }
        }
        bool again = p.softmax && !(fabsf(top) < INFINITY);
        const float inverse = (float)(1. / sum);
        // in 32 bits: an exponential and a reciprocal of a number of at least 1 are off by less than 4e-7 together
        auto near_key = [&](int e) __attribute__((always_inline)) -> float {
            const float l = mine[e];
            if (by_logit) return l;
            const float s = p.softmax ? __expf(l - top) * inverse : __builtin_amdgcn_rcpf(1.f + __expf(-l));
            const float k = s + bias[e];
            return l > -INFINITY && k > -INFINITY ? k : -INFINITY;
        };
        // keys of this lane's experts first + q, first + q + S, ..., four at a time, so that their LDS reads and exponentials overlap
        auto walk = [&](int first, int count, auto each) __attribute__((always_inline)) {
            int j = q;
            for (; j + 3 * S < count; j += 4 * S) {
                float k[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) k[u] = near_key(first + j + u * S);
#pragma unroll
                for (int u = 0; u < 4; ++u) each(k[u], first + j + u * S);
            }
            for (; j < count; j += S) each(near_key(first + j), first + j);
        };
        auto score_of = [&](float l) __attribute__((always_inline)) -> double { return p.softmax ? exp((double)l - (double)top) / sum : sigmoid(l); };
        float largest = 0.f;  // |key|, for the error of the 32-bit sum
        u64 groups = 1;
        if (grouped) {
            for (int g = 0; g < p.groups; ++g) {
                float best = -INFINITY, second = -INFINITY;
                walk(g * size, size, [&](float k, int) __attribute__((always_inline)) {
                    second = fmaxf(second, fminf(best, k));
                    best = fmaxf(best, k);
                });
                float ob = over<1>(best), os = over<1>(second);
                second = fmaxf(fmaxf(second, os), fminf(best, ob));
                best = fmaxf(best, ob);
                ob = over<2>(best), os = over<2>(second);
                second = fmaxf(fmaxf(second, os), fminf(best, ob));
                best = fmaxf(best, ob);
                if (best > -INFINITY) largest = fmaxf(largest, fabsf(best));
                if (p.group_top == 2 && second > -INFINITY) {
                    largest = fmaxf(largest, fabsf(second));
                    best += second;
                }
                if (q == 0) of_group[g * R + r] = best;
            }
            __syncthreads();
            // a lane ranks every fourth group
            groups = 0;
            float last = INFINITY, next = -INFINITY;
            for (int g = q; g < p.groups; g += S) {
                const float x = of_group[g * R + r];
                int before = 0;
                for (int h = 0; h < p.groups; ++h) {
                    const float y = of_group[h * R + r];
                    before += y > x || (y == x && h < g);
                }
                if (before < p.kept) groups |= 1ull << g, last = fminf(last, x);
                else next = fmaxf(next, x);
            }
            groups |= over<1>(groups);
            groups |= over<2>(groups);
            last = fminf(last, over<1>(last)), next = fmaxf(next, over<1>(next));
            last = fminf(last, over<2>(last)), next = fmaxf(next, over<2>(next));
            // two keys to a sum, on either side
            if (!(last - next > 4.f * (5e-7f + 2.4e-7f * largest))) again = true;
        }
        float a[KL];
        int idx[KL];
#pragma unroll
        for (int i = 0; i < KL; ++i) a[i] = -INFINITY, idx[i] = -1;
        auto offer = [&](float x, int e) __attribute__((always_inline)) {
            if (!__any(x > a[KL - 1])) return;
#pragma unroll
            for (int i = 0; i < KL; ++i) {
                const bool up = x > a[i];
                const float ax = a[i];
                const int ex = idx[i];
                a[i] = up ? x : ax;
                idx[i] = up ? e : ex;
                x = up ? ax : x;
                e = up ? ex : e;
            }
        };
        if (grouped) {
            u64 left = groups;
            for (int i = 0; i < p.kept; ++i) {  // every token its own groups, in ascending order
                const int g = __builtin_ctzll(left);
                left &= left - 1;
                walk(g * size, size, offer);
            }
        } else {
            walk(0, E, offer);
        }
        // The lists of four lanes become one.  Of two sorted lists the larger of entry i and entry KL - 1 - i are the KL largest; between the two joins they
        // are sorted again.
        auto join = [&](auto by) __attribute__((always_inline)) {
            constexpr int BY = decltype(by)::value;
            float ob[KL];
            int oi[KL];
#pragma unroll
            for (int i = 0; i < KL; ++i) ob[i] = over<BY>(a[i]), oi[i] = (int)over<BY>((uint32_t)idx[i]);
            // either lane of a pair puts together the same list, in the same order
            float la[KL];
            int li[KL];
#pragma unroll
            for (int i = 0; i < KL; ++i) {
                const bool upper = (q & BY) != 0;
                const float low = upper ? ob[i] : a[i], high = upper ? a[KL - 1 - i] : ob[KL - 1 - i];
                const int low_i = upper ? oi[i] : idx[i], high_i = upper ? idx[KL - 1 - i] : oi[KL - 1 - i];
                la[i] = high > low ? high : low;
                li[i] = high > low ? high_i : low_i;
            }
#pragma unroll
            for (int i = 0; i < KL; ++i) a[i] = la[i], idx[i] = li[i];
        };
        join(std::integral_constant<int, 1>{});
#pragma unroll
        for (int i = 1; i < KL; ++i)
#pragma unroll
            for (int j = i; j > 0; --j) {
                const bool up = a[j] > a[j - 1];
                const float ax = a[j];
                const int ex = idx[j];
                a[j] = up ? a[j - 1] : ax, idx[j] = up ? idx[j - 1] : ex;
                a[j - 1] = up ? ax : a[j - 1], idx[j - 1] = up ? ex : idx[j - 1];
            }
        join(std::integral_constant<int, 2>{});
        float least = a[0], most = a[0];
#pragma unroll
        for (int i = 1; i < KL; ++i) least = fminf(least, a[i]), most = fmaxf(most, a[i]);
        // a lane settles entries q, q + S, ... of the list
        double key[OWN], score[OWN];
        int at[OWN], rank[OWN];
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            at[o] = -1;
#pragma unroll
            for (int i = 0; i < S && o * S + i < KL; ++i)
                if (q == i) at[o] = idx[o * S + i];
            score[o] = at[o] >= 0 ? score_of(mine[at[o]]) : 0.;
            key[o] = at[o] >= 0 ? score[o] + (double)bias[at[o]] : -INFINITY;
            rank[o] = 0;
        }
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            // against each lane's entry o
#pragma unroll
            for (int i = 0; i < S; ++i) {
                double other = key[o];
                int oi = at[o];
                if (i & 1) other = __longlong_as_double((long long)over<1>((u64)__double_as_longlong(other))), oi = (int)over<1>((uint32_t)oi);
                if (i & 2) other = __longlong_as_double((long long)over<2>((u64)__double_as_longlong(other))), oi = (int)over<2>((uint32_t)oi);
#pragma unroll
                for (int m = 0; m < OWN; ++m)
                    rank[m] += (other > key[m] || (other == key[m] && (unsigned)oi < (unsigned)at[m])) && !(i == 0 && m == o);
            }
        }
        // what fell off the lists has a key of no more than this; an empty place in them: nothing has
        const double rest = least == -INFINITY ? -INFINITY : by_logit ? score_of(least) * (1. + 1e-14) : (double)least + 5e-7 + 1.2e-7 * (double)fmaxf(fabsf(most), fabsf(least));
        double total = 0.;
#pragma unroll
        for (int o = 0; o < OWN; ++o)
            if (rank[o] < p.k && o * S + q < KL) {
                if (!(key[o] > rest)) again = true;
                total += score[o];
            }
        total += __longlong_as_double((long long)over<1>((u64)__double_as_longlong(total)));
        total += __longlong_as_double((long long)over<2>((u64)__double_as_longlong(total)));
        uint32_t failed = again;
        failed |= over<1>(failed);
        failed |= over<2>(failed);
        if (live && !failed) {
#pragma unroll
            for (int o = 0; o < OWN; ++o)
                if (rank[o] < p.k && o * S + q < KL) {
                    double w = score[o];
                    if (p.renorm) w = total > 0. ? w / total : 0.;
                    p.idx[(t0 + r) * p.k + rank[o]] = at[o];
                    p.w[(t0 + r) * p.k + rank[o]] = (float)(w * (double)p.scale);
                }
        }
        u64 todo = __ballot(live && failed && q == 0);
        __syncthreads();
        while (todo) {
            const int row = __builtin_ctzll(todo) / S;
            todo &= todo - 1;
            float l[V];
#pragma unroll
            for (int i = 0; i < V; ++i) l[i] = lane + 64 * i < E ? rows[row * ld + lane + 64 * i] : -INFINITY;
            select_token<V>(p, l, keys, t0 + row, true);
        }
    }
}

template <bool BF16, int V, int KL>
int launch_many_as(const SelectParams &p, hipStream_t s)
{
    const size_t smem = (kManyTokens * many_row(p.E) + many_groups(p) + p.E) * 4;
    auto kern = select_many_kernel<BF16, V, KL>;
    static std::once_flag once;  // per instantiation
    static hipError_t setup_rc = hipSuccess;
    std::call_once(once, [&]() { setup_rc = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 96 * 1024); });
    MOE_HIP_CHECK(setup_rc);
    const int64_t blocks = ((int64_t)p.T + kManyTokens - 1) / kManyTokens;
    hipLaunchKernelGGL(kern, dim3((unsigned)(blocks < 1 << 16 ? blocks : 1 << 16)), dim3(64), smem, s, p);
    MOE_LAUNCH_CHECK("select_many_kernel");
    return MOE_OK;
}

template <bool BF16, int V>
int launch_many(const SelectParams &p, hipStream_t s)
{
    if (p.k <= 2) return launch_many_as<BF16, V, 4>(p, s);
    if (p.k <= 6) return launch_many_as<BF16, V, 8>(p, s);
    return launch_many_as<BF16, V, 10>(p, s);
}

template <bool BF16>
int launch_as(const SelectParams &p, hipStream_t s)
{
    if (p.T >= kManyFrom && p.n_parts == 0) return p.E <= 256 ? launch_many<BF16, 4>(p, s) : launch_many<BF16, 16>(p, s);
    const int64_t blocks = ((int64_t)p.T + kWaves - 1) / kWaves;
    const dim3 grid((unsigned)(blocks < 1 << 16 ? blocks : 1 << 16));
    if (p.E <= 64) hipLaunchKernelGGL((select_kernel<BF16, 1>), grid, dim3(kThreads), 0, s, p);
    else if (p.E <= 128) hipLaunchKernelGGL((select_kernel<BF16, 2>), grid, dim3(kThreads), 0, s, p);
    else if (p.E <= 256) hipLaunchKernelGGL((select_kernel<BF16, 4>), grid, dim3(kThreads), 0, s, p);
    else if (p.E <= 512) hipLaunchKernelGGL((select_kernel<BF16, 8>), grid, dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((select_kernel<BF16, 16>), grid, dim3(kThreads), 0, s, p);
    MOE_LAUNCH_CHECK("select_kernel");
    return MOE_OK;
}

}  // namespace

int launch_select(const SelectParams &p, int dtype, hipStream_t s)
{
    return dtype == MOE_DTYPE_BF16 ? launch_as<true>(p, s) : launch_as<false>(p, s);
}

}  // namespace moe355
