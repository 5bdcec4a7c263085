// C-ABI entry points of the selection of experts and of e4m3 operands with a scale per block of 128 (declared in include/moe.h):
// argument validation on the host, then the launches.  The experts' feed-forward and the layer on them are in moe_api.hip.
#include "b128_internal.h"

namespace moe355 {

namespace {

constexpr int kMostColumns = 1 << 24;  // 16 rows of them have 32-bit offsets

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

}  // namespace

int check_select(const moe_select_config_t *c)
{
    if (!c) {
        set_error("select config is NULL");
        return MOE_ERR_INVALID_ARG;
    }
    if (c->E < 1 || c->E > MOE_MAX_E) return unsupported("E", c->E);
    if (c->k < 1 || c->k > MOE_MAX_K || c->k > c->E) return unsupported("k", c->k);
    if (c->score != MOE_SCORE_SOFTMAX && c->score != MOE_SCORE_SIGMOID) return unsupported("score", c->score);
    if (c->n_groups < 1 || c->n_groups > MOE_MAX_GROUPS || c->E % c->n_groups != 0) return unsupported("n_groups", c->n_groups);
    if (c->groups_kept < 1 || c->groups_kept > c->n_groups || c->groups_kept * (c->E / c->n_groups) < c->k) return unsupported("groups_kept", c->groups_kept);
    if (c->group_top != 1 && c->group_top != 2) return unsupported("group_top", c->group_top);
    if (c->renormalize != 0 && c->renormalize != 1) {
        set_error("renormalize must be 0 or 1");
        return MOE_ERR_INVALID_ARG;
    }
    if (!(c->scale - c->scale == 0.f)) {
        set_error("scale = %g is not finite", (double)c->scale);
        return MOE_ERR_INVALID_ARG;
    }
    return MOE_OK;
}

SelectParams select_params(const moe_select_config_t &c)
{
    SelectParams p = {};
    p.E = c.E;
    p.k = c.k;
    p.softmax = c.score == MOE_SCORE_SOFTMAX;
    p.groups = c.n_groups;
    p.kept = c.groups_kept;
    p.group_top = c.group_top;
    p.renorm = c.renormalize;
    p.scale = c.scale;
    return p;
}

}  // namespace moe355

using namespace moe355;

extern "C" {

int moe_select_experts(const moe_select_config_t *cfg, const void *logits, int32_t dtype, int64_t row_stride, const float *bias, int32_t T,
                       int32_t *topk_idx, float *topk_w, void *stream)
{
    set_error("%s", "");
    const int rc = check_select(cfg);
    if (rc != MOE_OK) return rc;
    if (dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16) return unsupported("dtype", dtype);
    if (T < 0 || (int64_t)T * cfg->k > 0x3fffffff) {
        set_error("T = %d is negative, or its assignments do not fit the int32 row indices", T);
        return MOE_ERR_INVALID_ARG;
    }
    if (T == 0) return MOE_OK;
    if (bad_ptr(logits, "logits", dtype == MOE_DTYPE_BF16 ? 2 : 4) || bad_ptr(bias, "bias", 4, true) || bad_ptr(topk_idx, "topk_idx", 4) ||
        bad_ptr(topk_w, "topk_w", 4))
        return MOE_ERR_INVALID_ARG;
    if (T > 1 && row_stride < cfg->E) {
        set_error("row_stride = %lld is less than E = %d", (long long)row_stride, cfg->E);
        return MOE_ERR_INVALID_ARG;
    }
    SelectParams p = select_params(*cfg);
    p.logits = logits;
    p.stride = row_stride;
    p.bias = bias;
    p.T = T;
    p.idx = topk_idx;
    p.w = topk_w;
    return launch_select(p, dtype, (hipStream_t)stream);
}

int64_t moe_b128_scale_cols(int32_t cols)
{
    if (cols < 1) {
        set_error("cols = %d is not positive", cols);
        return MOE_ERR_INVALID_ARG;
    }
    return b128_scale_cols(cols);
}

int moe_quantize_b128(const void *x, int32_t dtype, int64_t row_stride, int32_t matrices, int32_t rows, int32_t cols, int32_t block_rows, void *q_out,
                      void *scale_out, void *stream)
{
    set_error("%s", "");
    if (dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16) return unsupported("dtype", dtype);
    if (block_rows != 1 && block_rows != kBlock) return unsupported("block_rows", block_rows);
    if (cols < 16 || cols % 16 != 0 || cols > kMostColumns) return unsupported("cols", cols);
    if (matrices < 0 || rows < 0) {
        set_error("matrices = %d, rows = %d: 0 or more", matrices, rows);
        return MOE_ERR_INVALID_ARG;
    }
    if (matrices == 0 || rows == 0) return MOE_OK;
    if (bad_ptr(x, "x", 16) || bad_ptr(q_out, "q_out", 16) || bad_ptr(scale_out, "scale_out", 4)) return MOE_ERR_INVALID_ARG;
    if ((int64_t)matrices * rows > 1 && (row_stride < cols || row_stride % (dtype == MOE_DTYPE_BF16 ? 8 : 4) != 0)) {
        set_error("row_stride = %lld: at least cols = %d elements and a multiple of 16 bytes", (long long)row_stride, cols);
        return MOE_ERR_INVALID_ARG;
    }
    return launch_quantize_b128(x, dtype, row_stride, matrices, rows, cols, block_rows, static_cast<uint8_t *>(q_out), static_cast<uint8_t *>(scale_out),
                                (hipStream_t)stream);
}

int moe_gemm_b128(const void *a_q, const void *a_scale, int32_t a_count, const int32_t *a_rows, const void *w_q, const void *w_scale,
                  const int32_t *offsets, int32_t E, int32_t n_rows, int32_t N, int32_t K, void *c, int32_t c_dtype, void *stream)
{
    set_error("%s", "");
    if (c_dtype != MOE_DTYPE_F32 && c_dtype != MOE_DTYPE_BF16) return unsupported("c_dtype", c_dtype);
    if (E < 1 || E > MOE_MAX_E || (E > 1 && !offsets)) {
        set_error("E = %d outside [1, %d], or more than one expert without offsets", E, MOE_MAX_E);
        return MOE_ERR_INVALID_ARG;
    }
    if (N < 8 || N % 8 != 0 || N > kMostColumns) return unsupported("N", N);
    if (K < 16 || K % 16 != 0 || K > kMostColumns) return unsupported("K", K);
    if (n_rows < 0 || n_rows > 0x3fffffff || a_count < 0 || (!a_rows && a_count < n_rows) || (n_rows > 0 && a_count == 0)) {
        set_error("n_rows = %d, a_count = %d: rows in [0, 2^30), each of them a row of a_q", n_rows, a_count);
        return MOE_ERR_INVALID_ARG;
    }
    if (n_rows == 0) return MOE_OK;
    if (bad_ptr(a_q, "a_q", 16) || bad_ptr(a_scale, "a_scale", 4) || bad_ptr(a_rows, "a_rows", 4, true) || bad_ptr(w_q, "w_q", 16) ||
        bad_ptr(w_scale, "w_scale", 4) || bad_ptr(offsets, "offsets", 4, true) || bad_ptr(c, "c", 16))
        return MOE_ERR_INVALID_ARG;
    GemmB128 g = {};
    g.a = static_cast<const uint8_t *>(a_q);
    g.a_scale = static_cast<const uint8_t *>(a_scale);
    g.a_count = a_count;
    g.a_rows = a_rows;
    g.w = static_cast<const uint8_t *>(w_q);
    g.w_scale = static_cast<const uint8_t *>(w_scale);
    g.offsets = offsets;
    g.E = E;
    g.n_rows = n_rows;
    g.N = g.Nh = N;
    g.K = K;
    g.c = c;
    g.c_dtype = c_dtype;
    g.precise = c_dtype == MOE_DTYPE_F32;
    return launch_gemm_b128(g, (hipStream_t)stream);
}

}  // extern "C"
