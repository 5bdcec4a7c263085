// The next token of every row of logits: temperature, top-k, top-p, min-p, and a draw from given random numbers.
//
// All filters keep a beginning of one order (descending logit, ascending index), so a row's kept set is one threshold on the pair
// (key: the logit's bits, made to order like the logit; index).  It is found without sorting the row: a histogram over 2048 steps of
// 1/64 in (largest - logit) / temperature, of counts for top-k and of weights for top-p, says which step holds the border.  Where the
// tokens down to that step are few (kCandidates), they alone are sorted, and all that is left happens on them; where they are many, the
// ones of the border step alone; where these are too many as well (a flat or a very wide row), a radix walk over the pairs settles
// it, 8 bits a pass over the row.
//
// Weights are exp in 64 bits, summed as whole numbers of 2^-f (f = 62 - ceil(log2 V), at most 50): sums of whole numbers do not depend on
// their order, so atomic sums give one result.  The largest weight is 1, so a sum is off by V 2^-(f+1) of itself at most, 1.1e-10 for 32000 tokens,
// 1.8e-9 for 128000, 3e-8 for 2^19; roundings of either sign make some 1e-12 of it.  Only a border nearer than that to u, top_p or the sum
// before a token can fall on another token than in exact sums.  A token that weighs less than 2^-(f+1) (2^-46 for 128000) counts as nothing.
//
// Bound by the 64-bit weights and by the passes over the row, for few rows by latency.  Measured, all filters mixed, the four kernels: 256 rows of
// 128000 fp32 logits (131 MB) 22 + 34 + 41 + 31 us; 64 rows of 51201 in bf16 6 + 9 + 15 + 29; one row of 128000 by top-p 3 + 10 + 8 + 17.
#include <stddef.h>

#include <mutex>

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
    int chunks, chunk;   // blocks of a row and tokens of each; 1: sample_kernel alone
    uint8_t *work;       // with more: a RowWork a row
};

// NaN is -infinity (the larger of a number and a NaN is the number)
__device__ __forceinline__ float clean(float v) { return fmaxf(v, -INFINITY); }
template <bool BF16>
__device__ __forceinline__ float logit_at(const void *row, int i)
{
    return clean(BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(row)[i] << 16) : static_cast<const float *>(row)[i]);
}
// 16 bytes of a row at a time.  Rows lie at any element, so the load is told nothing about its alignment (the hardware needs none).
template <bool BF16>
struct Vec {
    static constexpr int kN = BF16 ? 8 : 4;
    uint32_t w[4];
    __device__ __forceinline__ float raw(int j) const
    {
        return BF16 ? __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16) : __uint_as_float(w[j & 3]);
    }
    __device__ __forceinline__ float operator[](int j) const { return clean(raw(j)); }
    __device__ __forceinline__ float largest() const
    {
        float most = raw(0);
#pragma unroll
        for (int j = 1; j < kN; ++j) most = fmaxf(most, raw(j));
        return most;
    }
};
template <bool BF16>
__device__ __forceinline__ Vec<BF16> load_vec(const char *row, int i, int V)
{
    Vec<BF16> v;
    if (i + Vec<BF16>::kN <= V) {
        __builtin_memcpy(v.w, row + (int64_t)i * (BF16 ? 2 : 4), 16);
    } else {  // past the end: -infinity
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (BF16) {
                const uint32_t lo = i + 2 * j < V ? reinterpret_cast<const uint16_t *>(row)[i + 2 * j] : 0xff80u;
                const uint32_t hi = i + 2 * j + 1 < V ? reinterpret_cast<const uint16_t *>(row)[i + 2 * j + 1] : 0xff80u;
                v.w[j] = lo | hi << 16;
            } else {
                v.w[j] = i + j < V ? reinterpret_cast<const uint32_t *>(row)[i + j] : 0xff800000u;
            }
        }
    }
    return v;
}
// orders like the logit; -0 is 0
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t u = __float_as_uint(v + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

struct Row {
    float largest, steps;  // steps of the histogram in one unit of the logit
    double top, rate;      // log2(e) / temperature
    double unit;           // 2^f
};

// 2^(i / 32)
__constant__ static const double kRoots[32] = {
    1.0, 1.0218971486541166, 1.0442737824274138, 1.0671404006768237,
    1.0905077326652577, 1.1143867425958924, 1.1387886347566916, 1.1637248587775775,
    1.189207115002721, 1.215247359980469, 1.241857812073484, 1.2690509571917332,
    1.2968395546510096, 1.3252366431597413, 1.3542555469368927, 1.383909881963832,
    1.4142135623730951, 1.4451808069770467, 1.4768261459394993, 1.5091644275934228,
    1.5422108254079407, 1.5759808451078865, 1.6104903319492543, 1.645755478153965,
    1.681792830507429, 1.718619298122478, 1.7562521603732995, 1.7947090750031072,
    1.8340080864093424, 1.8741676341103, 1.9152065613971474, 1.9571441241754002,
};

// exp((v - largest) / temperature) = 2^y, y <= 0: y = n / 32 + rest, |rest| <= 1/64, 2^(n/32) from the table and the exponent, 2^rest by
// its series (the first term left out is (ln 2 / 64)^6 / 720 = 2e-15 of it).  17 operations in 64 bits with whole(), a third of what exp() and a
// division by the temperature take, and the kernel is bound by them. 
// Without a branch: -infinity gives 2^-1000, and where the largest logit is infinite, top is 1e300 and infinity gives 1.
__device__ __forceinline__ double weight(const Row &r, float v, const double *roots)
{
    const double y = fmin(fmax(((double)v - r.top) * r.rate, -1000.0), 0.0);
    const double magic = 6755399441055744.0;  // 1.5 * 2^52: a sum with it is rounded to a whole number, held in its low word
    const double t = fma(y, 32.0, magic);
    const int n = (int)(uint32_t)__double_as_longlong(t);
    const double rest = fma(t - magic, -0.03125, y);
    double e = 0.0013333558146428443;
    e = fma(e, rest, 0.009618129107628477);
    e = fma(e, rest, 0.05550410866482158);
    e = fma(e, rest, 0.24022650695910072);
    e = fma(e, rest, 0.6931471805599453);
    e = fma(e, rest, 1.0);
    e *= roots[n & 31];
    // y > -1000: the exponent stays that of a normal number
    return __longlong_as_double(__double_as_longlong(e) + ((long long)(n >> 5) << 52));
}
// w * 2^f to the nearest whole number; f <= 50 and w <= 1, so that the sum with 2^52 holds it in its low bits
__device__ __forceinline__ u64 whole(const Row &r, double w)
{
    return (u64)__double_as_longlong(fma(w, r.unit, 4503599627370496.0)) - 0x4330000000000000ull;
}

static constexpr int kThreads = 1024, kWaves = kThreads / 64, kSteps = 2048, kCandidates = 4096, kSegments = MOE_SAMPLE_MAX_V / 256;
// Copies of the histogram, a lane's by its number: the logits of a wave crowd into few steps, and atomic sums on one address queue
// (131072 sums of 64 bits over 8 steps by one block: 32 us with one copy, 16 with four, 13 with eight; 12 over 64 steps and more.  fp32 sums
// would take 164 us wherever they go: the LDS adds fp32 a lane at a time.)
static constexpr int kCopies = 4;

struct Shared {
    u64 sum[kWaves];
    double roots[32];                     // kRoots: lanes ask for different ones
    uint32_t n, digit;
    u64 before;
    int token;
    alignas(16) union {
        u64 histogram[kSteps * kCopies];  // counts or weights; then
        u64 segment[kSegments];           // the kept weights of every 64 vectors of the row
        u64 list[kCandidates];            // or, in a kernel that has only them, candidates
    };
    u64 candidate[kCandidates];
};

// The block's LDS.  Every function is inlined and asks for it itself: behind a reference the compiler may not know that it is LDS and
// go through flat instructions, which are slower and not kept in order.
extern __shared__ __align__(16) uint8_t lds[];
__device__ __forceinline__ Shared &shared() { return *reinterpret_cast<Shared *>(lds); }

__device__ __forceinline__ u64 pack(uint32_t key, int i) { return (u64)key << 32 | (uint32_t)~i; }  // orders like (logit, -index)

// Step of the histogram, ascending as the logit descends, equal for equal logits.
__device__ __forceinline__ int step_of(const Row &r, float v)
{
    const float d = r.largest - v;
    return d > 0.f ? (int)fminf(d * r.steps, (float)(kSteps - 1)) : 0;
}

__device__ __forceinline__ u64 block_sum(u64 v)
{
    Shared &sh = shared();
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.sum[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all += sh.sum[w];
    return all;
}

// Exclusive prefix over the block's threads.
__device__ __forceinline__ u64 block_scan(u64 mine)
{
    Shared &sh = shared();
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    u64 x = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const u64 o = __shfl_up(x, off, 64);
        if (lane >= off) x += o;
    }
    __syncthreads();
    if (lane == 63) sh.sum[w] = x;
    __syncthreads();
    u64 front = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) front += i < w ? sh.sum[i] : 0;
    return front + x - mine;
}

// f(vector, its number) for the vectors of the tokens from `from` (a multiple of 64 vectors) to `to`, -infinity for places past it.  A thread
// has the next two vectors in flight.  f is called by whole waves.
template <bool BF16, typename F>
__device__ __forceinline__ void over_vectors(const char *row, int from, int to, F f)
{
    static constexpr int kN = Vec<BF16>::kN, kFlight = 2;
    const int vectors = (to + kN - 1) / kN, mine = from / kN + (int)threadIdx.x;
    Vec<BF16> x[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) x[u] = load_vec<BF16>(row, min(mine + u * kThreads, vectors) * kN, to);
#pragma unroll 1
    for (int base = 0; from / kN + base < vectors; base += kFlight * kThreads) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const int at = mine + base + u * kThreads;
            const Vec<BF16> now = x[u];
            x[u] = load_vec<BF16>(row, min(at + kFlight * kThreads, vectors) * kN, to);
            f(now, at);
        }
    }
}

// f(v, index) for every token; skip(largest logit of a vector): whether f need not see the vector; after each vector done(its number).  The work
// of four tokens at most is mixed by the compiler: with more of it in registers the 64-bit arithmetic spills.
template <bool BF16, typename S, typename F, typename G>
__device__ __forceinline__ void over_row(const char *row, int from, int to, S skip, F f, G done)
{
    static constexpr int kN = Vec<BF16>::kN;
    over_vectors<BF16>(row, from, to, [&](const Vec<BF16> &now, int at) {
        if (!skip(now.largest())) {
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                f(now[j], at * kN + j);
                if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        }
        done(at);
    });
}

// The border of a step that holds too many tokens to sort, `before` in front of the step: walks the step's pairs from the cut on, 8 bits
// a pass from the top, to the one at which the running value reaches the target; that pair is the last that stays.
template <bool BF16>
__device__ __forceinline__ u64 walk(const char *row, int V, const Row &r, bool by_mass, int step, u64 cut, u64 before, double target)
{
    Shared &sh = shared();
    const int tid = threadIdx.x;
    u64 prefix = 0;
#pragma unroll 1
    for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 512) sh.candidate[tid] = 0;
        __syncthreads();
        over_row<BF16>(row, 0, V, [](float) { return false; }, [&](float v, int i) {
            if (v == -INFINITY || step_of(r, v) != step) return;
            const u64 c = pack(key_of(v), i);
            if (c < cut || (shift < 56 && (c >> (shift + 8)) != prefix)) return;
            const int digit = (int)(c >> shift) & 255;
            atomicAdd(&sh.candidate[digit], by_mass ? whole(r, weight(r, v, sh.roots)) : 1ull);
            atomicAdd(&sh.candidate[256 + digit], 1ull);  // a digit whose tokens weigh nothing is a digit all the same
        }, [](int) {});
        __syncthreads();
        if (tid == 0) {
            u64 run = before, last_run = run;
            int digit = -1, last = 0;
            for (int d = 255; d >= 0; --d) {
                if (!sh.candidate[256 + d]) continue;
                last = d;
                last_run = run;
                if ((double)(run + sh.candidate[d]) >= target) {
                    digit = d;
                    break;
                }
                run += sh.candidate[d];
            }
            sh.digit = digit < 0 ? last : digit;
            sh.before = digit < 0 ? last_run : run;
        }
        __syncthreads();
        prefix = prefix << 8 | sh.digit;
        before = sh.before;
    }
    return prefix;
}

// The candidates, descending (bitonic over the next power of two; the places behind them are 0, below every pair).  Exchanges over
// less than 128 places stay inside a wave's own 128, without a barrier.
__device__ __forceinline__ void sort_candidates(int n)
{
    Shared &sh = shared();
    int m = 128;
    while (m < n) m <<= 1;
    for (int i = n + threadIdx.x; i < m; i += kThreads) sh.candidate[i] = 0;
    const auto exchange = [&](int i, int gap, int size) {
        const int lo = 2 * i - (i & (gap - 1)), hi = lo + gap;
        const u64 a = sh.candidate[lo], b = sh.candidate[hi];
        if ((a < b) == ((lo & size) == 0)) {
            sh.candidate[lo] = b;
            sh.candidate[hi] = a;
        }
    };
    __syncthreads();
    for (int size = 2; size <= m; size <<= 1) {
        int gap = size >> 1;
        for (; gap >= 128; gap >>= 1) {
            for (int i = threadIdx.x; i < m / 2; i += kThreads) exchange(i, gap, size);
            __syncthreads();
        }
        for (; gap > 0; gap >>= 1) {
            // threads 64 k .. 64 k + 63 exchange inside places 128 k .. 128 k + 127
            for (int i = threadIdx.x; i < m / 2; i += kThreads) exchange(i, gap, size);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");  // waits for the wave's own accesses
            __builtin_amdgcn_wave_barrier();
        }
        if (size >= 128) __syncthreads();
    }
    __syncthreads();
}

static constexpr int kEach = kSteps / kThreads;  // steps a thread

// The step in which the running value of the histogram reaches the target, which is top_k, or top_p of the whole; kSteps where it never does.
// own: the thread's steps.  before: the running value in front of the step.  upto: how many tokens the steps up to it hold, by weight only
// about: a token of step i weighs 2^f exp(-(i + 1/2) / 64), a per cent more or less.
__device__ __forceinline__ int border_step(const Row &r, bool by_mass, const u64 (&own)[kEach], double &target, u64 &before, float &upto)
{
    Shared &sh = shared();
    const int at = threadIdx.x * kEach;
    u64 mine = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) mine += own[i];
    u64 run = block_scan(mine);
    if (threadIdx.x == 0) sh.digit = kSteps;
    if (threadIdx.x == kThreads - 1) sh.before = run + mine;
    __syncthreads();
    if (by_mass) target *= (double)sh.before;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if ((double)run < target && (double)(run + own[i]) >= target) {  // one place at most
            sh.digit = at + i;
            sh.before = run;
        }
        run += own[i];
    }
    __syncthreads();
    const int s = sh.digit;
    before = sh.before;
    float tokens = 0.f;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (at + i <= s) tokens += by_mass ? (float)own[i] / (float)r.unit * __expf(fminf((float)(at + i) * 0.015625f + 0.0078125f, 80.f)) : (float)own[i];
    tokens = fminf(tokens, 1e9f);
    upto = (float)block_sum((u64)tokens);
    return s;
}

// The last of the n sorted candidates in front of which the running value, `before` in front of the first, is below the target.
__device__ __forceinline__ u64 border_candidate(const Row &r, bool by_mass, int n, double target, u64 before)
{
    Shared &sh = shared();
    if (!by_mass) return sh.candidate[min(n, (int)((u64)target - before)) - 1];
    int last = 0;
    for (int base = 0; base < n; base += kThreads) {
        const int i = base + threadIdx.x;
        const u64 mine = i >= n ? 0 : whole(r, weight(r, logit_of((uint32_t)(sh.candidate[i] >> 32)), sh.roots));
        const u64 at = before + block_scan(mine);
        const int stay = (int)block_sum(i < n && (double)at < target ? 1 : 0);
        if (stay > 0) last = base + stay - 1;
        if (stay < min(n - base, kThreads)) break;
        before += block_sum(mine);
    }
    return sh.candidate[last];
}

// Whether the tokens up to the border step are few enough to sort.  By weight, what is not sorted costs little (it is summed while the border
// step's tokens are gathered); by count it costs top-p a histogram of its own.  (512 candidates to sort: 5 us, 4096: 18.)
__device__ __forceinline__ bool few(bool by_mass, float upto) { return upto <= (by_mass ? 512.f : 0.95f * kCandidates); }

// A row's settings.
struct Plan {
    Row r;
    int top_k;
    double top_p, min_p;
    bool none, only_first;   // nothing can be drawn; the first of the order alone stays
    bool by_count, by_mass;  // top-k, top-p leave something out
};
__device__ __forceinline__ Plan plan_of(const SampleParams &p, int b, float largest)
{
    Plan q;
    const float temperature = p.temperature ? p.temperature[b] : 1.f;
    q.top_k = p.top_k ? p.top_k[b] : 0;
    q.top_p = p.top_p ? p.top_p[b] : 1.f;
    q.min_p = p.min_p ? p.min_p[b] : 0.f;
    q.none = largest == -INFINITY;
    q.only_first = !(temperature > 0.f) || !(q.min_p <= 1.0) || q.top_k == 1 || !(q.top_p > 0.0);  // NaN: no weight is at least that
    q.by_count = q.top_k > 0 && q.top_k < p.V;
    q.by_mass = q.top_p < 1.0;
    // an infinite logit's share is the same at every temperature, an infinite one among them
    const bool finite = largest < INFINITY;
    q.r = {largest, fminf(64.f / temperature, 3e38f), finite ? (double)largest : 1e300, 1.44269504088896340736 / (finite ? (double)temperature : 1.0),
           (double)(1ull << p.bits)};
    return q;
}

// The largest logit of the tokens from .. to: four vectors of a thread in flight, an instruction a token.
template <bool BF16>
__device__ __forceinline__ float largest_of(const char *row, int from, int to)
{
    static constexpr int kN = Vec<BF16>::kN, kFlight = 4;
    const int vectors = (to + kN - 1) / kN, tid = threadIdx.x;
    float largest = -INFINITY;
    for (int base = from / kN + tid; base < vectors; base += kThreads * kFlight) {
        Vec<BF16> x[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) x[u] = load_vec<BF16>(row, min(base + u * kThreads, vectors) * kN, to);
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
#pragma unroll
            for (int j = 0; j < kN; ++j) largest = fmaxf(largest, x[u].raw(j));  // of a number and a NaN the number
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) largest = fmaxf(largest, __shfl_xor(largest, off, 64));
    float *wave_top = reinterpret_cast<float *>(shared().sum);
    if ((tid & 63) == 0) wave_top[tid >> 6] = largest;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) largest = fmaxf(largest, wave_top[w]);
    __syncthreads();
    return largest + 0.f;  // -0 is 0
}

// Adds the tokens from .. to that are not below the cut to a cleared histogram.
template <bool BF16>
__device__ __forceinline__ void fill_histogram(const char *row, int from, int to, const Row &r, bool by_mass, u64 cut)
{
    Shared &sh = shared();
    __syncthreads();
    for (int i = threadIdx.x; i < kSteps * kCopies; i += kThreads) sh.histogram[i] = 0;
    __syncthreads();
    u64 *const own = sh.histogram + (threadIdx.x & (kCopies - 1));
    const auto below = [&](float most) { return !(most > -INFINITY) || (cut && most < logit_of((uint32_t)(cut >> 32))); };
    if (by_mass)
        over_row<BF16>(row, from, to, below, [&](float v, int i) {
            u64 w = whole(r, weight(r, v, sh.roots));
            w = pack(key_of(v), i) < cut ? 0 : w;
            atomicAdd(own + step_of(r, v) * kCopies, w);
        }, [](int) {});
    else
        // -infinity counts in the last step: where that makes it the border, it holds fewer candidates, and all stay
        over_row<BF16>(row, from, to, below, [&](float v, int) { atomicAdd(own + step_of(r, v) * kCopies, 1ull); }, [](int) {});
    __syncthreads();
}

// Of the tokens from .. to, those of step hi, or of all up to it, from the cut on become candidates (sh.n of them; it may be more than there is
// room for).  sum_up: what is not a candidate and surely stays by weight is summed by segments of the row.
template <bool BF16>
__device__ __forceinline__ int gather(const char *row, int from, int to, const Plan &q, u64 cut, int hi, bool only_hi, bool sum_up, u64 *segment, u64 *list)
{
    static constexpr int kN = Vec<BF16>::kN;
    Shared &sh = shared();
    const Row &r = q.r;
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    u64 kept = 0;
    over_vectors<BF16>(row, from, to, [&](const Vec<BF16> &now, int at) {
        // in a step after hi, as most are
        const bool beyond = hi < kSteps - 1 && (r.largest - now.largest()) * r.steps >= (float)(hi + 1);
        if (!beyond) {
            u64 c[kN];
            uint32_t picked = 0;
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                const float v = now[j];
                const int s = step_of(r, v);
                c[j] = pack(key_of(v), at * kN + j);
                const bool in = v > -INFINITY && s <= hi && c[j] >= cut, pick = in && (s == hi || !only_hi);
                picked |= pick ? 1u << j : 0u;
                if (sum_up) {
                    const double w = weight(r, v, sh.roots);
                    kept += in && !pick && w >= q.min_p ? whole(r, w) : 0;
                    if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (picked) {  // one sum for the vector: its result is waited for
                uint32_t place = atomicAdd(&sh.n, (uint32_t)__popc(picked));
#pragma unroll
                for (int j = 0; j < kN; ++j)
                    if (picked >> j & 1) {
                        if (place < (uint32_t)kCandidates) list[place] = c[j];
                        ++place;
                    }
            }
        }
        if (!sum_up) return;
        u64 sum = kept;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
        if ((threadIdx.x & 63) == 0 && at * kN < to) segment[at / 64] = sum;
        kept = 0;
    });
    __syncthreads();
    return (int)sh.n;
}

// What stays of the tokens from .. to, summed by segments of the row.
template <bool BF16>
__device__ __forceinline__ void sum_segments(const char *row, int from, int to, const Plan &q, u64 cut, u64 *segment)
{
    u64 kept = 0;
    const auto below = [&](float most) { return !(most > -INFINITY) || (cut && most < logit_of((uint32_t)(cut >> 32))); };
    over_row<BF16>(row, from, to, below, [&](float v, int i) {
        if (pack(key_of(v), i) < cut) return;
        const double w = weight(q.r, v, shared().roots);
        kept += w >= q.min_p ? whole(q.r, w) : 0;
    }, [&](int at) {
        u64 sum = kept;
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
        if ((threadIdx.x & 63) == 0 && at * Vec<BF16>::kN < to) segment[at / 64] = sum;
        kept = 0;
    });
}

// Where there are few rows, several blocks share one: three kernels fill a row's RowWork, a chunk of the row a block, before sample_kernel
// goes on with what is left of it.  (One row of 128000 tokens: 75 us by one block, 42 of them the histogram.)
static constexpr int kMaxChunks = 64;
// The border step of the first filter.  What is gathered, and what is summed, goes by it, so it is settled once: two kernels need not round the same.
struct Border {
    double target;
    u64 before;
    int step, all;  // all: the tokens of all steps up to it are the candidates, not those of the step alone
};
struct RowWork {
    float largest[kMaxChunks];       // of every chunk
    Border border;
    uint32_t n, pad[57];             // candidates
    u64 histogram[kSteps];
    u64 candidate[kCandidates];
    u64 segment[kSegments];
};

__device__ __forceinline__ RowWork &work_of(const SampleParams &p, int b) { return reinterpret_cast<RowWork *>(p.work)[b]; }
__device__ __forceinline__ float largest_of_row(const SampleParams &p, int b)
{
    float largest = -INFINITY;
    for (int c = 0; c < p.chunks; ++c) largest = fmaxf(largest, work_of(p, b).largest[c]);
    return largest;
}
template <bool BF16>
__device__ __forceinline__ const char *row_of(const SampleParams &p, int b)
{
    return static_cast<const char *>(p.logits) + (int64_t)b * p.stride * (BF16 ? 2 : 4);
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void sample_largest_kernel(SampleParams p)
{
    const int c = blockIdx.x, b = blockIdx.y, from = c * p.chunk;
    RowWork &work = work_of(p, b);
    for (int i = c * kThreads + threadIdx.x; i < kSteps; i += p.chunks * kThreads) work.histogram[i] = 0;
    if (c == 0 && threadIdx.x == 0) work.n = 0;
    const float largest = largest_of<BF16>(row_of<BF16>(p, b), from, min(p.V, from + p.chunk));
    if (threadIdx.x == 0) work.largest[c] = largest;
}

template <bool BF16>
__global__ __launch_bounds__(kThreads, 8) void sample_histogram_kernel(SampleParams p)
{
    Shared &sh = shared();
    const int c = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, from = c * p.chunk, to = min(p.V, from + p.chunk);
    RowWork &work = work_of(p, b);
    const Plan q = plan_of(p, b, largest_of_row(p, b));
    if (q.none || q.only_first) return;
    if (tid < 32) sh.roots[tid] = kRoots[tid];
    __syncthreads();
    if (!q.by_count && !q.by_mass) {
        sum_segments<BF16>(row_of<BF16>(p, b), from, to, q, 0, work.segment);
        return;
    }
    fill_histogram<BF16>(row_of<BF16>(p, b), from, to, q.r, !q.by_count, 0);
    for (int i = tid; i < kSteps; i += kThreads) {
        u64 sum = 0;
#pragma unroll
        for (int k = 0; k < kCopies; ++k) sum += sh.histogram[i * kCopies + k];
        if (sum) atomicAdd(&work.histogram[i], sum);
    }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads, 8) void sample_gather_kernel(SampleParams p)
{
    Shared &sh = shared();
    const int c = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, from = c * p.chunk, to = min(p.V, from + p.chunk);
    RowWork &work = work_of(p, b);
    const Plan q = plan_of(p, b, largest_of_row(p, b));
    if (q.none || q.only_first || (!q.by_count && !q.by_mass)) return;
    if (tid < 32) sh.roots[tid] = kRoots[tid];
    // every block of the row finds the same border, by the same instructions from the same whole numbers
    u64 own[kEach], before;
#pragma unroll
    for (int i = 0; i < kEach; ++i) own[i] = work.histogram[tid * kEach + i];
    float upto;
    double target = q.by_count ? (double)q.top_k : q.top_p;
    const int s = border_step(q.r, !q.by_count, own, target, before, upto);
    const bool all = few(!q.by_count, upto);
    if (c == 0 && tid == 0) work.border = {target, before, s, all};
    if (s == kSteps) return;
    const int n = gather<BF16>(row_of<BF16>(p, b), from, to, q, 0, s, !all, !all && !q.by_count, work.segment, sh.list);
    if (tid == 0) sh.digit = atomicAdd(&work.n, (uint32_t)n);
    __syncthreads();
    const uint32_t first = sh.digit;
    for (int i = tid; i < min(n, kCandidates); i += kThreads)
        if (first + i < (uint32_t)kCandidates) work.candidate[first + i] = sh.list[i];
}

// A block a row.
template <bool BF16, bool SHARED_ROW>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleParams p)
{
    Shared &sh = shared();
    const int64_t index = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (index >= p.B) return;
    const int b = (int)index, tid = threadIdx.x, lane = tid & 63;
    const char *row = row_of<BF16>(p, b);
    if (tid < 32) sh.roots[tid] = kRoots[tid];
    if (tid == 0) sh.token = 0x7fffffff;
    __syncthreads();
    const float largest = SHARED_ROW ? largest_of_row(p, b) : largest_of<BF16>(row, 0, p.V);
    const Plan q = plan_of(p, b, largest);
    const Row &r = q.r;
    const double min_p = q.min_p;
    if (q.none || q.only_first) {
        if (!q.none) {
            int first = 0x7fffffff, from = 0, to = p.V;
            if (SHARED_ROW) {  // in the first chunk that has it
                while (work_of(p, b).largest[from] != largest) ++from;
                from *= p.chunk;
                to = min(p.V, from + p.chunk);
            }
            over_row<BF16>(row, from, to, [&](float most) { return most < largest; }, [&](float v, int i) { first = v == largest && i < first ? i : first; }, [](int) {});
            if (first != 0x7fffffff) atomicMin(&sh.token, first);
        }
        __syncthreads();
        if (tid == 0) {
            p.token[b] = q.none ? -1 : sh.token;
            if (p.logprob) p.logprob[b] = q.none ? -INFINITY : 0.f;
        }
        return;
    }
    const int segments = ceil_div(p.V, 64 * Vec<BF16>::kN);
    u64 cut = 0;          // tokens from this pair on stay
    int n = 0;            // candidates
    bool all = false;     // they are all that may stay
    bool summed = false;  // the segments hold what stays in front of the border step
    const auto weigh = [&](u64 c) { return weight(r, logit_of((uint32_t)(c >> 32)), sh.roots); };

    // first by count, then by weight; in one loop, so that there is one copy of what they share
#pragma unroll 1
    for (int stage = 0; stage < 2; ++stage) {
        const bool by_mass = stage == 1;
        if (by_mass ? !q.by_mass : !q.by_count) continue;
        double target = by_mass ? q.top_p : (double)q.top_k;
        u64 before = 0;
        int s = 0;
        if (all) {  // by weight, of the candidates that top-k left
            u64 mine = 0;
            for (int i = tid; i < n; i += kThreads) mine += sh.candidate[i] >= cut ? whole(r, weigh(sh.candidate[i])) : 0;
            target = q.top_p * (double)block_sum(mine);
        } else {
            const bool done = SHARED_ROW && !(by_mass && q.by_count);  // the first filter: other blocks have gathered the candidates
            if (done) {
                const Border &border = work_of(p, b).border;
                target = border.target;
                before = border.before;
                s = border.step;
                all = border.all;
            } else {
                fill_histogram<BF16>(row, 0, p.V, r, by_mass, cut);
                u64 own[kEach];
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    own[i] = 0;
#pragma unroll
                    for (int c = 0; c < kCopies; ++c) own[i] += sh.histogram[(tid * kEach + i) * kCopies + c];
                }
                float upto;
                s = border_step(r, by_mass, own, target, before, upto);
                all = few(by_mass, upto);
            }
            if (s == kSteps) {  // fewer tokens than top_k
                all = false;
                continue;
            }
            summed = !all && by_mass;
            if (done) {
                const RowWork &work = work_of(p, b);
                n = (int)work.n;
                for (int i = tid; i < min(n, kCandidates); i += kThreads) sh.candidate[i] = work.candidate[i];
                __syncthreads();
                if (summed)
                    for (int i = tid; i < segments; i += kThreads) sh.segment[i] = work.segment[i];
                __syncthreads();
            }
            if (!done || (all && n > kCandidates)) {
                if (done) {  // the estimate was wrong
                    all = false;
                    summed = by_mass;
                }
                n = gather<BF16>(row, 0, p.V, q, cut, s, !all, summed, sh.segment, sh.candidate);
                if (all && n > kCandidates) {  // as above
                    all = false;
                    summed = by_mass;
                    n = gather<BF16>(row, 0, p.V, q, cut, s, true, summed, sh.segment, sh.candidate);
                }
            }
            if (all) before = 0;
            if (n == 0) continue;
            if (n <= kCandidates) sort_candidates(n);
        }
        cut = n <= kCandidates ? border_candidate(r, by_mass, n, target, before) : walk<BF16>(row, p.V, r, by_mass, s, cut, before, target);
    }

    // what stays, by segments of the row
    __syncthreads();
    if (all || (summed && n <= kCandidates)) {
        if (all) {
            for (int i = tid; i < segments; i += kThreads) sh.segment[i] = 0;
            __syncthreads();
        }
        for (int i = tid; i < n; i += kThreads) {
            const u64 c = sh.candidate[i];
            const double w = weigh(c);
            if (c >= cut && w >= min_p) atomicAdd(&sh.segment[(int)~(uint32_t)c / (64 * Vec<BF16>::kN)], whole(r, w));
        }
    } else if (SHARED_ROW && !q.by_count && !q.by_mass) {
        for (int i = tid; i < segments; i += kThreads) sh.segment[i] = work_of(p, b).segment[i];
    } else {
        sum_segments<BF16>(row, 0, p.V, q, cut, sh.segment);
    }
    __syncthreads();
    // the segment, and in it the token, at which the running sum passes u times the sum
    static_assert(kSegments == kSteps, "as many segments a thread as steps");
    u64 mine = 0;
    u64 own[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int at = tid * kEach + i;
        own[i] = at < segments ? sh.segment[at] : 0;
        mine += own[i];
    }
    const u64 total = block_sum(mine);
    const double goal = (double)fminf(fmaxf(p.u[b], 0.f), 0.99999994f) * (double)total;  // below the total
    u64 run = block_scan(mine);
    if (tid == 0) sh.digit = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const u64 next = run + own[i];
        if ((double)run <= goal && (double)next > goal) {
            sh.digit = tid * kEach + i;
            sh.before = run;
        }
        run = next;
    }
    __syncthreads();
    if (tid < 64) {
        const int base = ((int)sh.digit * 64 + lane) * Vec<BF16>::kN;
        const Vec<BF16> x = load_vec<BF16>(row, min(base, p.V), p.V);
        u64 each[Vec<BF16>::kN], sum = 0;
#pragma unroll
        for (int j = 0; j < Vec<BF16>::kN; ++j) {
            const float v = x[j];
            each[j] = 0;
            if (v != -INFINITY && pack(key_of(v), base + j) >= cut) {
                const double w = weight(r, v, sh.roots);
                if (w >= min_p) each[j] = whole(r, w);
            }
            sum += each[j];
        }
        u64 at = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const u64 o = __shfl_up(at, off, 64);
            if (lane >= off) at += o;
        }
        at += sh.before - sum;
#pragma unroll
        for (int j = 0; j < Vec<BF16>::kN; ++j) {
            if ((double)at <= goal && (double)(at + each[j]) > goal) sh.token = base + j;
            at += each[j];
        }
    }
    __syncthreads();
    if (tid == 0) {
        const int token = min(sh.token, p.V - 1);  // the running sum passes a part of the total for some token; an index in any case
        p.token[b] = token;
        if (p.logprob) p.logprob[b] = (float)log(weight(r, logit_at<BF16>(row, token), sh.roots) / ((double)total / r.unit));
    }
}

// LDS of the kernels that share a row: a histogram or a list, so that a CU holds two blocks.
constexpr size_t kHistogramLds = offsetof(Shared, candidate), kListLds = offsetof(Shared, list) + kCandidates * 8;

int set_lds(const void *kernel)
{
    MOE_HIP_CHECK(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared)));
    return MOE_OK;
}

template <bool BF16>
int launch_as(const SampleParams &p, hipStream_t s)
{
    static std::once_flag once;
    static int setup_rc = MOE_OK;
    std::call_once(once, [&]() {
        for (const void *kernel : {reinterpret_cast<const void *>(sample_kernel<BF16, false>), reinterpret_cast<const void *>(sample_kernel<BF16, true>),
                                   reinterpret_cast<const void *>(sample_largest_kernel<BF16>), reinterpret_cast<const void *>(sample_histogram_kernel<BF16>),
                                   reinterpret_cast<const void *>(sample_gather_kernel<BF16>)})
            if (setup_rc == MOE_OK) setup_rc = set_lds(kernel);
    });
    if (setup_rc != MOE_OK) {
        set_error("moe_sample: the device refuses %d bytes of LDS", (int)sizeof(Shared));
        return setup_rc;
    }
    if (p.chunks > 1) {
        const dim3 grid(p.chunks, p.B);
        hipLaunchKernelGGL(sample_largest_kernel<BF16>, grid, dim3(kThreads), offsetof(Shared, list), s, p);
        MOE_LAUNCH_CHECK("sample_largest_kernel");
        hipLaunchKernelGGL(sample_histogram_kernel<BF16>, grid, dim3(kThreads), kHistogramLds, s, p);
        MOE_LAUNCH_CHECK("sample_histogram_kernel");
        hipLaunchKernelGGL(sample_gather_kernel<BF16>, grid, dim3(kThreads), kListLds, s, p);
        MOE_LAUNCH_CHECK("sample_gather_kernel");
    }
    // rows of the grid of 2^21 blocks: a launch of 2^32 threads in one dimension starts fewer and says nothing
    const int across = p.B < 1 << 21 ? p.B : 1 << 21;
    const dim3 rows(across, (p.B - 1) / across + 1);
    if (p.chunks > 1) hipLaunchKernelGGL((sample_kernel<BF16, true>), rows, dim3(kThreads), sizeof(Shared), s, p);
    else hipLaunchKernelGGL((sample_kernel<BF16, false>), rows, dim3(kThreads), sizeof(Shared), s, p);
    MOE_LAUNCH_CHECK("sample_kernel");
    return MOE_OK;
}

// Blocks of a row: so many that the rows together give 1024 (a CU holds two), of 8192 tokens and more, which is a row's fixed cost in each.
int chunks_for(int B, int V)
{
    int chunks = 1024 / (B > 0 ? B : 1);
    if (chunks > V / 8192) chunks = V / 8192;
    return chunks < 1 ? 1 : chunks > kMaxChunks ? kMaxChunks : chunks;
}

}  // namespace

int launch_sample(const void *logits, int dtype, int64_t stride, int B, int V, const float *u, const float *temperature, const int32_t *top_k,
                  const float *top_p, const float *min_p, int32_t *token, float *logprob, void *ws, hipStream_t s)
{
    int bits = 62;
    while ((1ll << (62 - bits)) < V) --bits;
    bits = bits < 50 ? bits : 50;
    // chunks begin at whole vectors of all threads
    const int chunk = (int)align_up(ceil_div(V, chunks_for(B, V)), 8192);
    const SampleParams p = {logits, stride, B, V, bits, u, temperature, top_p, min_p, top_k, token, logprob, ceil_div(V, chunk), chunk, static_cast<uint8_t *>(ws)};
    return dtype == MOE_DTYPE_BF16 ? launch_as<true>(p, s) : launch_as<false>(p, s);
}

int64_t sample_workspace(int B, int V) { return 256 + (chunks_for(B, V) > 1 ? (int64_t)B * (int64_t)sizeof(RowWork) : 0); }

}  // namespace moe355
