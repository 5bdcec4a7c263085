// C-ABI entry points of the attention half of a decoder step and of sampling (declared in include/moe.h): argument
// validation on the host, then the launches.
#include <new>

#include "attn_internal.h"

namespace moe355 {

int launch_sample(const void *logits, int dtype, int64_t stride, int B, int V, const float *u, const float *temperature, const int32_t *top_k,
                  const float *top_p, const float *min_p, int32_t *token, float *logprob, void *ws, hipStream_t s);
int64_t sample_workspace(int B, int V);

namespace {

// Rows (new tokens times heads of a group) up to which a sequence is the decode kernel's, 16 at a time: it reads the cache once for each 16, the
// prefill kernel once for 128 or 256, which it computes whether they are there or not.  64 sequences of 2048 keys, decode / prefill, us:
//   4 key heads of 128, bf16   16 rows 33 / 88    48 rows 64 / 90     64 rows 69 / 90     96 rows 98 / 91
//   16 key heads of 64, bf16   16 rows 58 / 168   48 rows 118 / 171   64 rows 156 / 171   96 rows 225 / 176
//   4 key heads of 128, fp32   16 rows 39 / 167   48 rows 107 / 169   64 rows 139 / 170   96 rows 202 / 172
//   16 key heads of 64, fp32   16 rows 68 / 171   48 rows 182 / 212   64 rows 238 / 213   96 rows 338 / 223
// 64 is right for three of the four; fp32 over 16 heads of 64 loses 25 us at it, and the border is one for all, whatever the lengths.
constexpr int kFewRows = 64;

bool bad_ptr(const void *p, const char *name, int align, bool nullable = false)
{
    if (!p && nullable) return false;
    if (!p) {
        set_error("%s is NULL", name);
        return true;
    }
    if (reinterpret_cast<uintptr_t>(p) % align != 0) {
        set_error("%s is not %d-byte aligned", name, align);
        return true;
    }
    return false;
}

int unsupported(const char *what, long long v)
{
    set_error("%s = %lld is not supported", what, v);
    return MOE_ERR_UNSUPPORTED;
}

int validate(const moe_attn_config_t *c)
{
    if (!c) {
        set_error("config is NULL");
        return MOE_ERR_INVALID_ARG;
    }
    if (c->dtype != MOE_DTYPE_F32 && c->dtype != MOE_DTYPE_BF16) return unsupported("dtype", c->dtype);
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return unsupported("head_dim", c->head_dim);
    if (c->n_kv_heads < 1) return unsupported("n_kv_heads", c->n_kv_heads);
    if (c->n_heads < 1 || c->n_heads > MOE_ATTN_MAX_HEADS || c->n_heads % c->n_kv_heads != 0) return unsupported("n_heads", c->n_heads);
    if (c->page_size < 16 || c->page_size > 128 || (c->page_size & (c->page_size - 1)) != 0) return unsupported("page_size", c->page_size);
    if (c->rot_dim < 0 || c->rot_dim > c->head_dim || c->rot_dim % 16 != 0) return unsupported("rot_dim", c->rot_dim);
    if (c->B_max < 1 || c->B_max > MOE_ATTN_MAX_B) return unsupported("B_max", c->B_max);
    if (c->T_max < 0 || c->T_max >= 1 << 24) {
        set_error("T_max = %d outside [0, 2^24)", c->T_max);
        return MOE_ERR_INVALID_ARG;
    }
    if (c->num_pages < 1 || c->max_pages < 1 || (int64_t)c->max_pages * c->page_size >= 1 << 30) {
        set_error("num_pages = %d and max_pages = %d have to be positive, max_pages * page_size below 2^30", c->num_pages, c->max_pages);
        return MOE_ERR_INVALID_ARG;
    }
    if (c->rot_interleaved != 0 && c->rot_interleaved != 1) {
        set_error("rot_interleaved must be 0 or 1");
        return MOE_ERR_INVALID_ARG;
    }
    return MOE_OK;
}

// What append and attention have in common; fills p.  MOE_OK with p.B = 0: nothing to do.
int check_batch(const moe_attn_handle_t *h, const moe_kv_cache_t *cache, const int32_t *q_offsets, const int32_t *kv_len, const int32_t *page_table,
                int32_t B, int32_t T, int32_t max_q, int32_t max_kv, AttnParams &p)
{
    if (!h) {
        set_error("handle is NULL");
        return MOE_ERR_INVALID_ARG;
    }
    const moe_attn_config_t &c = h->cfg;
    if (B < 0 || B > c.B_max || T < 0 || T > c.T_max || max_q < 0 || max_kv < 0) {
        set_error("B = %d, T = %d, max_q = %d, max_kv = %d: B outside [0, B_max = %d], T outside [0, T_max = %d], or a negative bound", B, T, max_q, max_kv,
                  c.B_max, c.T_max);
        return MOE_ERR_INVALID_ARG;
    }
    p = AttnParams{};
    if (B == 0 || T == 0 || max_q == 0) return MOE_OK;
    int dev = -1;
    MOE_HIP_CHECK(hipGetDevice(&dev));
    if (dev != h->device) {
        set_error("current device %d is not the handle's device %d", dev, h->device);
        return MOE_ERR_INVALID_ARG;
    }
    if (!cache) {
        set_error("cache is NULL");
        return MOE_ERR_INVALID_ARG;
    }
    if (bad_ptr(cache->k, "cache->k", 16) || bad_ptr(cache->v, "cache->v", 16) || bad_ptr(cache->k_scale, "cache->k_scale", 16) ||
        bad_ptr(cache->v_scale, "cache->v_scale", 16) || bad_ptr(q_offsets, "q_offsets", 16) || bad_ptr(kv_len, "kv_len", 16) ||
        bad_ptr(page_table, "page_table", 16))
        return MOE_ERR_INVALID_ARG;
    int shift = 4;
    while (1 << shift < c.page_size) ++shift;
    p.k = static_cast<uint8_t *>(cache->k);
    p.v = static_cast<uint8_t *>(cache->v);
    p.k_scale = cache->k_scale;
    p.v_scale = cache->v_scale;
    p.q_offsets = q_offsets;
    p.kv_len = kv_len;
    p.page_table = page_table;
    p.B = B;
    p.T = T;
    p.n_heads = c.n_heads;
    p.n_kv_heads = c.n_kv_heads;
    p.group = c.n_heads / c.n_kv_heads;
    p.page_shift = shift;
    p.num_pages = c.num_pages;
    p.max_pages = c.max_pages;
    p.max_q = max_q < T ? max_q : T;
    p.room = c.max_pages * c.page_size;
    p.max_kv = max_kv < p.room ? max_kv : p.room;
    return MOE_OK;
}

bool bad_stride(int64_t stride, int64_t least, int dtype, const char *name)
{
    const int per16 = dtype == MOE_DTYPE_BF16 ? 8 : 4;
    if (stride >= least && stride % per16 == 0) return false;
    set_error("%s = %lld: at least %lld elements and a multiple of 16 bytes", name, (long long)stride, (long long)least);
    return true;
}

}  // namespace
}  // namespace moe355

using namespace moe355;

extern "C" {

int moe_attn_create(const moe_attn_config_t *cfg, moe_attn_handle_t **out)
{
    if (!out) {
        set_error("out is NULL");
        return MOE_ERR_INVALID_ARG;
    }
    *out = nullptr;
    const int rc = validate(cfg);
    if (rc != MOE_OK) return rc;
    int dev = 0, cus = 0;
    MOE_HIP_CHECK(hipGetDevice(&dev));
    MOE_HIP_CHECK(hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev));
    moe_attn_handle_t *h = new (std::nothrow) moe_attn_handle_t;
    if (!h) {
        set_error("out of host memory");
        return MOE_ERR_INVALID_ARG;
    }
    h->cfg = *cfg;
    h->device = dev;
    h->num_cus = cus;
    *out = h;
    set_error("%s", "");
    return MOE_OK;
}

int moe_attn_destroy(moe_attn_handle_t *h)
{
    delete h;
    return MOE_OK;
}

int64_t moe_attn_workspace_bytes(const moe_attn_handle_t *h)
{
    if (!h) {
        set_error("handle is NULL");
        return MOE_ERR_INVALID_ARG;
    }
    // partial results, of one kernel at a time, and where the sequences begin among the tiles
    const int64_t decode = attn_decode_workspace(h->cfg.head_dim, h->num_cus), prefill = attn_prefill_workspace(h->cfg.head_dim, h->num_cus);
    return (decode > prefill ? decode : prefill) + align_up((int64_t)(h->cfg.B_max + 1) * 8, 256);
}

int moe_kv_append(moe_attn_handle_t *h, const moe_kv_cache_t *cache, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                  const void *v, int64_t v_stride, const double *inv_freq, const int32_t *q_offsets, const int32_t *kv_len,
                  const int32_t *page_table, int32_t B, int32_t T, int32_t max_q, void *q_out, void *stream)
{
    set_error("%s", "");
    AppendParams p = {};
    const int rc = check_batch(h, cache, q_offsets, kv_len, page_table, B, T, max_q, 0x7fffffff, p.a);
    if (rc != MOE_OK || p.a.B == 0) return rc;
    const moe_attn_config_t &c = h->cfg;
    if (bad_ptr(k, "k", 16) || bad_ptr(v, "v", 16) || bad_ptr(q, "q", 16, true) || bad_ptr(q_out, "q_out", 16, !q) ||
        bad_ptr(inv_freq, "inv_freq", 16, c.rot_dim == 0))
        return MOE_ERR_INVALID_ARG;
    if (!q && q_out) {
        set_error("q_out without q");
        return MOE_ERR_INVALID_ARG;
    }
    const int64_t kv_row = (int64_t)c.n_kv_heads * c.head_dim;
    if (bad_stride(k_stride, kv_row, c.dtype, "k_stride") || bad_stride(v_stride, kv_row, c.dtype, "v_stride") ||
        (q && bad_stride(q_stride, (int64_t)c.n_heads * c.head_dim, c.dtype, "q_stride")))
        return MOE_ERR_INVALID_ARG;
    p.a.q = q;
    p.a.q_stride = q_stride;
    p.k_new = k;
    p.v_new = v;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.inv_freq = inv_freq;
    p.rot_dim = c.rot_dim;
    p.interleaved = c.rot_interleaved;
    p.q_out = q_out;
    return launch_kv_append(c.dtype, c.head_dim, p, (hipStream_t)stream);
}

int moe_attn_forward(moe_attn_handle_t *h, const moe_kv_cache_t *cache, const void *q, int64_t q_stride, const int32_t *q_offsets,
                     const int32_t *kv_len, const int32_t *page_table, int32_t B, int32_t T, int32_t max_q, int32_t max_kv, float scale,
                     int32_t causal, int32_t window, void *out, float *lse, void *workspace, int64_t workspace_bytes, void *stream)
{
    set_error("%s", "");
    AttnParams p;
    const int rc = check_batch(h, cache, q_offsets, kv_len, page_table, B, T, max_q, max_kv, p);
    if (rc != MOE_OK) return rc;
    const float scale_log2e = scale * 1.44269504088896340736f;
    if ((causal != 0 && causal != 1) || window < 0 || !(scale_log2e - scale_log2e == 0.f)) {
        set_error("causal = %d (0 or 1), window = %d (0 or more), scale = %g (finite, and times log2(e))", causal, window, (double)scale);
        return MOE_ERR_INVALID_ARG;
    }
    if (p.B == 0) return MOE_OK;
    const moe_attn_config_t &c = h->cfg;
    if (bad_ptr(q, "q", 16) || bad_ptr(out, "out", 16) || bad_ptr(lse, "lse", 16, true)) return MOE_ERR_INVALID_ARG;
    if (bad_stride(q_stride, (int64_t)c.n_heads * c.head_dim, c.dtype, "q_stride")) return MOE_ERR_INVALID_ARG;
    const int64_t need = moe_attn_workspace_bytes(h);
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < need) {
        set_error("workspace: %lld bytes at a multiple of 256 are needed", (long long)need);
        return MOE_ERR_WORKSPACE;
    }
    p.q = q;
    p.q_stride = q_stride;
    p.scale_log2e = scale_log2e;
    p.causal = causal;
    p.window = window < 1 << 30 ? window : 1 << 30;  // positions lie in (-2^24, 2^30): a difference of one and a window stays in 32 bits
    p.out = out;
    p.lse = lse;
    p.part = static_cast<float *>(workspace);
    p.seq_tiles = reinterpret_cast<int64_t *>(static_cast<uint8_t *>(workspace) + need - align_up((int64_t)(c.B_max + 1) * 8, 256));
    p.few_rows = kFewRows;
    const bool many = (int64_t)p.max_q * p.group > kFewRows;
    // Sequences of few rows: none where all sequences have max_q new tokens, and these are many.  That is so where there are max_q a sequence, unless one
    // has more; the prefill kernel then takes sequences of any number of rows, so that each is computed whatever the offsets say.
    if (!many || (int64_t)p.max_q * B > T) {
        const int failed = launch_attn_decode(c.dtype, c.head_dim, p, h->num_cus, (hipStream_t)stream);
        if (failed != MOE_OK) return failed;
    } else {
        p.few_rows = 0;
    }
    return many ? launch_attn_prefill(c.dtype, c.head_dim, p, h->num_cus, (hipStream_t)stream) : MOE_OK;
}

int64_t moe_sample_workspace_bytes(int32_t B, int32_t V)
{
    if (B < 0 || V < 1 || V > MOE_SAMPLE_MAX_V) {
        set_error("moe_sample: B = %d, V = %d: 1 <= V <= %d", B, V, MOE_SAMPLE_MAX_V);
        return MOE_ERR_INVALID_ARG;
    }
    return sample_workspace(B, V);
}

int moe_sample(const void *logits, int32_t dtype, int64_t row_stride, int32_t B, int32_t V, const float *u, const float *temperature,
               const int32_t *top_k, const float *top_p, const float *min_p, int32_t *token, float *logprob, void *workspace,
               int64_t workspace_bytes, void *stream)
{
    set_error("%s", "");
    const int64_t need = moe_sample_workspace_bytes(B, V);
    if (need < 0) return (int)need;
    if (dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16) return unsupported("dtype", dtype);
    if (B == 0) return MOE_OK;
    if (bad_ptr(logits, "logits", dtype == MOE_DTYPE_BF16 ? 2 : 4) || bad_ptr(u, "u", 4) || bad_ptr(temperature, "temperature", 4, true) || bad_ptr(top_k, "top_k", 4, true) ||
        bad_ptr(top_p, "top_p", 4, true) || bad_ptr(min_p, "min_p", 4, true) || bad_ptr(token, "token", 4) || bad_ptr(logprob, "logprob", 4, true))
        return MOE_ERR_INVALID_ARG;
    if (B > 1 && row_stride < V) {
        set_error("row_stride = %lld is less than V = %d", (long long)row_stride, V);
        return MOE_ERR_INVALID_ARG;
    }
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < need) {
        set_error("workspace: %lld bytes at a multiple of 256 are needed", (long long)need);
        return MOE_ERR_WORKSPACE;
    }
    return launch_sample(logits, dtype, row_stride, B, V, u, temperature, top_k, top_p, min_p, token, logprob, workspace, (hipStream_t)stream);
}

}  // extern "C"
