// The next token of every row of logits: temperature, top-k, top-p, min-p, and a draw from given random numbers.
//
// All filters keep a beginning of one order (descending logit, ascending index), so a row's kept set is a threshold: a key (the
// logit's bits, made to order like the logit) and how many of the tokens with just that key stay.  It is found by radix
// selection on the keys, over counts for top-k and over weights for top-p, without sorting the row.
//
// Weights are exp in 64 bits, summed as whole numbers of 2^-f (f = 62 - ceil(log2 V)): sums of whole numbers do not depend on
// their order, so the parallel sums give one result, and an error of V 2^-(f+1) at most, under 1e-11 of the sum for the usual V.
// The token at the border of a cumulative sum then is the one that sums in 64 bits choose.
#include "moe_internal.h"

namespace moe355 {

namespace {

typedef unsigned long long u64;

struct SampleParams {
    const void *logits;
    int64_t stride;
    int B, V, bits;  // bits: f
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *token;
    float *logprob;
};

static constexpr uint32_t kLowest = 0x007fffffu;  // key of -infinity

template <bool BF16>
__device__ __forceinline__ float logit_at(const void *row, int i)
{
    float v = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(row)[i] << 16) : static_cast<const float *>(row)[i];
    v += 0.f;  // -0 is 0
    return v != v ? -INFINITY : v;
}
// orders like the logit
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t u = __float_as_uint(v);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

struct Row {
    double top, temperature;
    double unit;  // 2^f
};
__device__ __forceinline__ double weight(const Row &r, float v)
{
    return (double)v == r.top ? 1.0 : exp(((double)v - r.top) / r.temperature);
}
__device__ __forceinline__ u64 whole(const Row &r, double w) { return (u64)rint(w * r.unit); }

static constexpr int kThreads = 1024;

struct Shared {
    u64 mass[256];
    uint32_t count[256];
    u64 sum[kThreads / 64];
    uint32_t ties[kThreads / 64];
    uint32_t best_key;
    int best_index;
    u64 before;
    uint32_t digit, before_count;
    int token;
    u64 token_mass;
};

__device__ __forceinline__ u64 shfl_xor_u64(u64 v, int off) { return __shfl_xor(v, off, 64); }

__device__ u64 block_sum(u64 v, Shared &sh)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += shfl_xor_u64(v, off);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.sum[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 all = 0;
    for (int w = 0; w < kThreads / 64; ++w) all += sh.sum[w];
    return all;
}

// exclusive prefix over the block of (ties, mass), and their totals
__device__ void block_scan(uint32_t &ties, u64 &mass, uint32_t &all_ties, u64 &all_mass, Shared &sh)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t t = ties;
    u64 m = mass;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t ot = __shfl_up(t, off, 64);
        const u64 om = __shfl_up(m, off, 64);
        if (lane >= off) {
            t += ot;
            m += om;
        }
    }
    __syncthreads();
    if (lane == 63) {
        sh.ties[w] = t;
        sh.sum[w] = m;
    }
    __syncthreads();
    uint32_t bt = 0;
    u64 bm = 0;
    all_ties = 0;
    all_mass = 0;
    for (int i = 0; i < kThreads / 64; ++i) {
        if (i < w) {
            bt += sh.ties[i];
            bm += sh.sum[i];
        }
        all_ties += sh.ties[i];
        all_mass += sh.sum[i];
    }
    ties = bt + t - ties;
    mass = bm + m - mass;
}

// A beginning of the order: all tokens with a greater key, and the first `ties` with this one.
struct Cut {
    uint32_t key;
    uint32_t ties;
};

// Radix walk from the top digit down: the key at which the running count (or mass) of the tokens within `in`, in descending order of
// keys, reaches `target`; `before`: the running value in front of that key.
template <bool BF16, bool MASS>
__device__ void walk(const void *row, int V, const Row &r, const Cut &in, u64 in_tie_mass, double target, uint32_t &key, u64 &before, Shared &sh)
{
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    before = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) sh.mass[tid] = 0;
        __syncthreads();
        for (int i = tid; i < V; i += kThreads) {
            const float v = logit_at<BF16>(row, i);
            const uint32_t k = key_of(v);
            if (k <= kLowest || k <= in.key || (shift < 24 && (k >> (shift + 8)) != prefix)) continue;
            atomicAdd(&sh.mass[(k >> shift) & 255], MASS ? whole(r, weight(r, v)) : 1ull);
        }
        __syncthreads();
        if (tid == 0) {
            // tokens with the border key of `in`, which are not all within it
            if (in.key > kLowest && (shift == 24 || (in.key >> (shift + 8)) == prefix))
                sh.mass[(in.key >> shift) & 255] += MASS ? in_tie_mass * in.ties : in.ties;
            u64 run = before;
            int digit = -1, last = 0;
            u64 last_run = run;
            for (int d = 255; d >= 0; --d) {
                if (!sh.mass[d]) continue;
                // the first digit at which the running value reaches the target
                if ((double)(run + sh.mass[d]) >= target) {
                    digit = d;
                    break;
                }
                last = d;
                last_run = run;
                run += sh.mass[d];
            }
            sh.digit = digit < 0 ? last : digit;
            sh.before = digit < 0 ? last_run : run;
        }
        __syncthreads();
        prefix = prefix << 8 | sh.digit;
        before = sh.before;
    }
    key = prefix;
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleParams p)
{
    __shared__ Shared sh;
    const int b = blockIdx.x, tid = threadIdx.x;
    const char *row = static_cast<const char *>(p.logits) + (int64_t)b * p.stride * (BF16 ? 2 : 4);
    // the first of the order
    u64 best = 0;
    for (int i = tid; i < p.V; i += kThreads) {
        const u64 c = (u64)key_of(logit_at<BF16>(row, i)) << 32 | (uint32_t)~i;
        best = c > best ? c : best;
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        const u64 o = shfl_xor_u64(best, off);
        best = o > best ? o : best;
    }
    if ((tid & 63) == 0) sh.sum[tid >> 6] = best;
    __syncthreads();
    for (int w = 0; w < kThreads / 64; ++w) best = sh.sum[w] > best ? sh.sum[w] : best;
    const uint32_t top_key = (uint32_t)(best >> 32);
    const int first = (int)~(uint32_t)best;
    const float temperature = p.temperature ? p.temperature[b] : 1.f;
    if (top_key <= kLowest || !(temperature > 0.f)) {
        if (tid == 0) {
            p.token[b] = top_key <= kLowest ? -1 : first;
            if (p.logprob) p.logprob[b] = top_key <= kLowest ? -INFINITY : 0.f;
        }
        return;
    }
    const Row r = {(double)logit_of(top_key), (double)temperature, (double)(1ull << p.bits)};
    const int top_k = p.top_k ? p.top_k[b] : 0;
    const double top_p = p.top_p ? p.top_p[b] : 1.f, min_p = p.min_p ? p.min_p[b] : 0.f;

    Cut cut = {kLowest, 0};
    u64 tie_mass = 0;
    if (top_k > 0 && top_k < p.V) {
        uint32_t key;
        u64 before;
        walk<BF16, false>(row, p.V, r, cut, 0, (double)top_k, key, before, sh);
        cut = {key, (uint32_t)(top_k - (int64_t)before)};
        tie_mass = whole(r, weight(r, logit_of(key)));
        // fewer tokens than top_k: the last key found has fewer ties than asked for, which the pass below counts out
    }
    if (top_p < 1.0) {
        u64 mass = 0;
        uint32_t ties = 0;
        for (int i = tid; i < p.V; i += kThreads) {
            const float v = logit_at<BF16>(row, i);
            const uint32_t k = key_of(v);
            if (k > cut.key && k > kLowest) mass += whole(r, weight(r, v));
            ties += cut.key > kLowest && k == cut.key;
        }
        mass = block_sum(mass, sh);
        const u64 all_ties = block_sum(ties, sh);
        if (cut.key > kLowest && cut.ties > all_ties) cut.ties = (uint32_t)all_ties;
        const double target = top_p * (double)(mass + tie_mass * cut.ties);
        uint32_t key;
        u64 before;
        walk<BF16, true>(row, p.V, r, cut, tie_mass, target, key, before, sh);
        const u64 one = whole(r, weight(r, logit_of(key)));
        // ties stay while the sum in front of them is below the target
        double n = one ? ceil((target - (double)before) / (double)one) : 1.0;
        n = n < 1.0 ? 1.0 : n;
        uint32_t keep = n > 4e9 ? 0xffffffffu : (uint32_t)n;
        if (key == cut.key) keep = keep < cut.ties ? keep : cut.ties;
        cut = {key, keep};
        tie_mass = one;
    }
    // the kept tokens in ascending index: their sum, then the one at which the running sum passes u times it
    const int last_tile = ceil_div(p.V, kThreads);
    u64 total = 0;
    double goal = 0.0;
    for (int pass = 0; pass < 2; ++pass) {
        u64 run = 0;
        uint32_t run_ties = 0;
        if (pass) goal = (double)p.u[b] * (double)total;
        if (tid == 0) sh.token = 0x7fffffff;
        for (int tile = 0; tile < last_tile; ++tile) {
            const int i = tile * kThreads + tid;
            const float v = i < p.V ? logit_at<BF16>(row, i) : -INFINITY;
            const uint32_t k = key_of(v);
            const bool tie = cut.key > kLowest && k == cut.key;
            const double w = k > kLowest && (tie || k > cut.key) ? weight(r, v) : 0.0;
            const bool big = w > 0.0 && (w >= min_p || i == first);
            uint32_t ties = tie, all_ties;
            u64 none = 0, all;
            block_scan(ties, none, all_ties, all, sh);
            const bool keep = big && (!tie || run_ties + ties < cut.ties);
            const u64 mine = keep ? whole(r, w) : 0;
            u64 before = mine;
            uint32_t zero = 0, zeros;
            block_scan(zero, before, zeros, all, sh);
            if (pass && keep && (double)(run + before + mine) > goal) atomicMin(&sh.token, i);
            run += all;
            run_ties += all_ties;
            __syncthreads();
            if (pass && sh.token != 0x7fffffff) break;
        }
        total = pass ? total : run;
    }
    __syncthreads();
    if (tid == 0) {
        // u < 1 in fp32 and whole numbers below 2^63: the sum passes u times itself, unless rounding of the product lifts it there
        const int token = sh.token == 0x7fffffff ? first : sh.token;
        p.token[b] = token;
        if (p.logprob) p.logprob[b] = (float)log(weight(r, logit_at<BF16>(row, token)) / ((double)total / r.unit));
    }
}

}  // namespace

int launch_sample(const void *logits, int dtype, int64_t stride, int B, int V, const float *u, const float *temperature, const int32_t *top_k,
                  const float *top_p, const float *min_p, int32_t *token, float *logprob, void *ws, hipStream_t s)
{
    int bits = 62;
    while ((1ll << (62 - bits)) < V) --bits;
    const SampleParams p = {logits, stride, B, V, bits, u, temperature, top_p, min_p, top_k, token, logprob};
    (void)ws;
    if (dtype == MOE_DTYPE_BF16) hipLaunchKernelGGL(sample_kernel<true>, dim3(B), dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL(sample_kernel<false>, dim3(B), dim3(kThreads), 0, s, p);
    MOE_LAUNCH_CHECK("sample_kernel");
    return MOE_OK;
}

int64_t sample_workspace(int B, int V) { return 256 + 0 * (int64_t)B * V; }

}  // namespace moe355
