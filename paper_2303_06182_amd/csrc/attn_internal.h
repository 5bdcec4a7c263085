// Internal declarations of the attention half of a decoder step (attn_api.hip, kv_append.hip, attn_decode.hip, attn_prefill.hip).
#pragma once

#include "moe_internal.h"

struct moe_attn_handle {
    moe_attn_config_t cfg;
    int device;
    int num_cus;
};

namespace moe355 {

// Everything the kernels know of a call.  Pointers are device pointers; see include/moe.h for their meaning.
struct AttnParams {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    const int32_t *q_offsets, *kv_len, *page_table;
    int B, T, n_heads, n_kv_heads, group;  // group: query heads of a key head
    int page_shift, num_pages, max_pages;
    int max_q, max_kv, room;               // clamped to what the handle can hold; room: the most keys of a sequence
    // attention
    const void *q;
    int64_t q_stride;
    float scale_log2e;                     // scale * log2(e): scores are kept as powers of two
    int causal, window;
    void *out;
    float *lse;
    // partial results of units that several blocks share, and where the sequences begin in the tile space
    float *part;
    int64_t *seq_tiles;
    int n_blocks;
    int units;                             // of a sequence at most: pieces of 16 rows times key heads
    int few_rows;                          // sequences of up to so many rows (new tokens times group) are the decode kernel's
};

// A sequence's new tokens and keys, clamped to what can exist, so that no index derived from them leaves its array.  The bounds max_q and max_kv
// say what is worked on, not where it is: positions come from the whole lengths.
struct Seq {
    int first, n;  // new tokens that are worked on, and the first of them
    int kv;        // keys in front of this one may be seen
    int begin;     // position of the first new token; negative where there are more of them than the length says
};
__device__ __forceinline__ Seq load_seq(const AttnParams &p, int b)
{
    int lo = p.q_offsets[b], hi = p.q_offsets[b + 1], kv = p.kv_len[b];
    lo = min(max(lo, 0), p.T);
    hi = min(max(hi, lo), p.T);
    kv = min(max(kv, 0), p.room);
    const int begin = kv - (hi - lo), n = min(hi - lo, p.max_q);
    if (p.causal) kv = max(begin + n, 0);  // without the keys of new tokens past max_q, which may not have been written
    return {lo, n, min(kv, p.max_kv), begin};
}

struct AppendParams {
    AttnParams a;
    const void *k_new, *v_new;
    int64_t k_stride, v_stride;
    const double *inv_freq;
    int rot_dim, interleaved;
    void *q_out;
};

int launch_kv_append(int dtype, int head_dim, const AppendParams &p, hipStream_t s);
int launch_attn_decode(int dtype, int head_dim, const AttnParams &p, int num_cus, hipStream_t s);
int64_t attn_decode_workspace(int head_dim, int num_cus);
int launch_attn_prefill(int dtype, int head_dim, const AttnParams &p, int num_cus, hipStream_t s);
int64_t attn_prefill_workspace(int head_dim, int num_cus);

}  // namespace moe355
