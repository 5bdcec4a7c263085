// Selection of experts from logits: scores, a bias that moves the selection and not the weights, groups, top-k, weights.
//
//   s_e = 1 / (1 + exp(-l_e))  or  exp(l_e - max l) / sum exp(l - max l);   key_e = s_e + b_e
// in 64 bits: two keys that differ are then told apart as any other 64-bit program tells them (in 32 bits a large part of the
// scores near 1 would be equal), and equal ones go to the lower index.  An expert without a key (logit -infinity or NaN, or bias
// -infinity or NaN) is ordered behind all others and has weight 0.
//
// One wave a token.
#include "b128_internal.h"

namespace moe355 {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
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

// V: experts of a lane, e = lane + 64 i
template <bool BF16, int V>
__global__ __launch_bounds__(kThreads) void select_kernel(SelectParams p)
{
    __shared__ double keys[kWaves][V * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int E = p.E, size = E / p.groups;
    for (int64_t t0 = (int64_t)blockIdx.x * kWaves; t0 < p.T; t0 += (int64_t)gridDim.x * kWaves) {
        const int64_t t = t0 + wave;
        const bool live = t < p.T;
        const void *row = static_cast<const char *>(p.logits) + (live ? t : 0) * p.stride * (BF16 ? 2 : 4);
        float l[V];
        double s[V];
        u64 key[V];
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = lane + 64 * i;
            l[i] = e < E ? logit<BF16>(row, e) : -INFINITY;
            if (!BF16 && p.n_parts > 0 && e < E && live) {
                for (int j = 0; j < p.n_parts; ++j) l[i] += p.parts[j * p.part_stride + t * E + e];
                p.sum_out[t * E + e] = l[i];
            }
            if (l[i] != l[i]) l[i] = -INFINITY;
            top = fmaxf(top, l[i]);
        }
        if (p.softmax) {
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
            for (int i = 0; i < V; ++i) s[i] = 1. / (1. + exp(-(double)l[i]));
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = lane + 64 * i;
            const double k = e < E && l[i] != -INFINITY ? s[i] + (p.bias ? (double)p.bias[e] : 0.) : -INFINITY;
            key[i] = ordered(k);
            if (key[i] == 0) s[i] = 0.;
            keys[wave][e] = key[i] ? k : -INFINITY;
        }
        __syncthreads();
        u64 groups = ~0ull;
        if (p.kept < p.groups) {
            // a lane a group
            double best = -INFINITY, second = -INFINITY;
            if (lane < p.groups)
                for (int j = 0; j < size; ++j) {
                    const double k = keys[wave][lane * size + j];
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
        __syncthreads();
    }
}

template <bool BF16>
int launch_as(const SelectParams &p, hipStream_t s)
{
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
