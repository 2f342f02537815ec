// C ABI of the attention half of a layer (RMS norm, rotary positions, KV cache, attention) and of sampling: argument validation and dispatch only.  See
// include/qarl.h.
#include <math.h>

#include "common.hpp"

namespace qarl {

static int bad_arg(const char *who, const char *what)
{
    set_error("%s: %s", who, what);
    return QARL_ERR_INVALID_ARG;
}

static int check_dtype(const char *who, const char *name, int dt)
{
    if (dt == QARL_OUT_BF16 || dt == QARL_OUT_F32) return QARL_OK;
    set_error("%s: %s must be QARL_OUT_BF16 or QARL_OUT_F32 (got %d)", who, name, dt);
    return QARL_ERR_INVALID_ARG;
}

static int check_norm_sizes(const char *who, int64_t rows, int K, float eps)
{
    if (rows < 0 || K <= 0) {
        set_error("%s: rows >= 0 and K > 0 required (got %lld, %d)", who, (long long)rows, K);
        return QARL_ERR_INVALID_ARG;
    }
    if (!(eps >= 0.f) || eps > 3.0e38f) {
        set_error("%s: eps must be finite and not negative (got %g)", who, (double)eps);
        return QARL_ERR_INVALID_ARG;
    }
    if (K % 8 != 0 || K > 16384) {
        set_error("%s: K %% 8 == 0 and K <= 16384 required (got %d)", who, K);
        return QARL_ERR_UNSUPPORTED;
    }
    return QARL_OK;
}

// A matrix of rows, or null: 16-byte aligned, its rows at a stride of at least K elements, a multiple of 8
static int check_rows(const char *who, const char *name, const void *p, int64_t stride, int K)
{
    if (!p) return QARL_OK;
    if (stride < K) {
        set_error("%s: rows of %s overlap (stride %lld, K %d)", who, name, (long long)stride, K);
        return QARL_ERR_INVALID_ARG;
    }
    if (!aligned16(p) || stride % 8 != 0) {
        set_error("%s: %s must be 16-byte aligned and its stride a multiple of 8 elements (got %lld)", who, name, (long long)stride);
        return QARL_ERR_ALIGNMENT;
    }
    return QARL_OK;
}

static int check_cache(const qarl_kv_cache *c, const char *who, KvArgs &kv)
{
    if (!c) return bad_arg(who, "null cache descriptor");
    if (c->fmt != QARL_KV_BF16 && c->fmt != QARL_KV_E4M3 && c->fmt != QARL_KV_E2M1) {
        set_error("%s: unknown cache format %d", who, c->fmt);
        return QARL_ERR_UNSUPPORTED;
    }
    if (c->num_pages <= 0 || c->page_size <= 0 || c->kv_heads <= 0 || c->head_dim <= 0) {
        set_error("%s: num_pages, page_size, kv_heads, head_dim must be positive (got %d, %d, %d, %d)", who, c->num_pages, c->page_size,
                  c->kv_heads, c->head_dim);
        return QARL_ERR_INVALID_ARG;
    }
    if ((c->head_dim != 64 && c->head_dim != 128) || c->page_size < 8 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) ||
        c->kv_heads > 1024) {
        set_error("%s: need head_dim 64 or 128, page_size a power of two from 8 to 1024, kv_heads <= 1024 (got %d, %d, %d)", who, c->head_dim,
                  c->page_size, c->kv_heads);
        return QARL_ERR_UNSUPPORTED;
    }
    const bool scaled = c->fmt != QARL_KV_BF16;
    if (!c->k || !c->v || (scaled && (!c->k_scales || !c->v_scales))) return bad_arg(who, "null cache buffer");
    if (!aligned16(c->k) || !aligned16(c->v) || (scaled && (!aligned16(c->k_scales) || !aligned16(c->v_scales)))) {
        set_error("%s: cache buffers must be 16-byte aligned", who);
        return QARL_ERR_ALIGNMENT;
    }
    kv = KvArgs{c->fmt, c->num_pages, __builtin_ctz((unsigned)c->page_size), c->kv_heads, c->head_dim, c->k, c->v, (float *)c->k_scales, (float *)c->v_scales};
    return QARL_OK;
}

}  // namespace qarl

using namespace qarl;

extern "C" {

int qarl_add_rmsnorm(const void *x_bf16, int64_t x_stride, const void *residual, int64_t residual_stride, const void *weight_bf16,
                     int64_t rows, int K, float eps, int stream_dtype, void *residual_out, int64_t residual_out_stride, void *y_bf16,
                     int64_t y_stride, void *codes, float *scales, int via_bf16, void *stream)
{
    const char *who = "qarl_add_rmsnorm";
    int rc = check_norm_sizes(who, rows, K, eps);
    if (rc || (rc = check_dtype(who, "stream_dtype", stream_dtype))) return rc;
    if (rows == 0) return QARL_OK;
    if (!x_bf16 || !weight_bf16) return bad_arg(who, "null x or weight");
    if (!y_bf16 && !codes && !residual_out) return bad_arg(who, "no output");
    if ((codes == nullptr) != (scales == nullptr)) return bad_arg(who, "codes and scales go together");
    if ((rc = check_rows(who, "x", x_bf16, x_stride, K)) || (rc = check_rows(who, "residual", residual, residual_stride, K)) ||
        (rc = check_rows(who, "residual_out", residual_out, residual_out_stride, K)) || (rc = check_rows(who, "y", y_bf16, y_stride, K)))
        return rc;
    if (!aligned16(weight_bf16) || ((uintptr_t)codes & 7u) || ((uintptr_t)scales & 3u)) {
        set_error("%s: weight must be 16-byte, codes 8-byte, scales 4-byte aligned", who);
        return QARL_ERR_ALIGNMENT;
    }
    NormArgs a = {x_bf16, residual, weight_bf16, x_stride, residual_stride, residual_out_stride, y_stride, rows, K, eps,
                  stream_dtype == QARL_OUT_F32, residual_out, y_bf16, codes, scales, via_bf16};
    return launch_rmsnorm(a, (hipStream_t)stream);
}

size_t qarl_add_rmsnorm_backward_workspace_bytes(int64_t rows, int K)
{
    if (rows <= 0 || K <= 0) return 0;
    return (size_t)rmsnorm_backward_groups(rows, K) * (size_t)K * sizeof(float);
}

int qarl_add_rmsnorm_backward(const void *dy_bf16, int64_t dy_stride, const void *h, int64_t h_stride, const void *dh, int64_t dh_stride,
                              const void *weight_bf16, int64_t rows, int K, float eps, int stream_dtype, void *dx, int64_t dx_stride,
                              void *dw, int dw_dtype, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "qarl_add_rmsnorm_backward";
    int rc = check_norm_sizes(who, rows, K, eps);
    if (rc || (rc = check_dtype(who, "stream_dtype", stream_dtype)) || (rc = check_dtype(who, "dw_dtype", dw_dtype))) return rc;
    if (dw && ((uintptr_t)dw & (dw_dtype == QARL_OUT_F32 ? 3u : 1u))) {
        set_error("%s: dw is not aligned to its type", who);
        return QARL_ERR_ALIGNMENT;
    }
    if (rows > 0) {
        if (!dy_bf16 || !h || !weight_bf16 || !dx) return bad_arg(who, "null dy, h, weight or dx");
        if ((rc = check_rows(who, "dy", dy_bf16, dy_stride, K)) || (rc = check_rows(who, "h", h, h_stride, K)) ||
            (rc = check_rows(who, "dh", dh, dh_stride, K)) || (rc = check_rows(who, "dx", dx, dx_stride, K)))
            return rc;
        if (!aligned16(weight_bf16)) {
            set_error("%s: weight must be 16-byte aligned", who);
            return QARL_ERR_ALIGNMENT;
        }
        const size_t need = dw ? qarl_add_rmsnorm_backward_workspace_bytes(rows, K) : 0;
        if (need && (!ws || ws_bytes < need || !aligned16(ws))) {
            set_error("%s: needs %zu bytes of 16-byte aligned workspace (got %zu)", who, need, ws_bytes);
            return QARL_ERR_WORKSPACE;
        }
    } else if (!dw) {
        return QARL_OK;
    }
    NormGradArgs a = {dy_bf16, h, dh, weight_bf16, dy_stride, h_stride, dh_stride, dx_stride, rows, K, eps,
                      stream_dtype == QARL_OUT_F32, dx, dw, dw_dtype == QARL_OUT_F32, (float *)ws};
    return launch_rmsnorm_backward(a, (hipStream_t)stream);
}

size_t qarl_kv_cache_bytes(int fmt, int num_pages, int page_size, int kv_heads, int head_dim)
{
    if ((fmt != QARL_KV_BF16 && fmt != QARL_KV_E4M3 && fmt != QARL_KV_E2M1) || num_pages <= 0 || page_size <= 0 || kv_heads <= 0 || head_dim <= 0) return 0;
    const size_t n = (size_t)num_pages * page_size * kv_heads * head_dim;
    return fmt == QARL_KV_BF16 ? 2 * n : fmt == QARL_KV_E4M3 ? n : n / 2;
}

size_t qarl_kv_scales_bytes(int fmt, int num_pages, int page_size, int kv_heads, int head_dim)
{
    if ((fmt != QARL_KV_E4M3 && fmt != QARL_KV_E2M1) || num_pages <= 0 || page_size <= 0 || kv_heads <= 0 || head_dim <= 0) return 0;
    return (size_t)num_pages * page_size * kv_heads * sizeof(float);
}

int qarl_kv_cache_write(const qarl_kv_cache *cache, const void *k_bf16, int64_t k_token_stride, int64_t k_head_stride, const void *v_bf16,
                        int64_t v_token_stride, int64_t v_head_stride, int64_t T, const int64_t *slots, void *stream)
{
    const char *who = "qarl_kv_cache_write";
    KvArgs kv;
    int rc = check_cache(cache, who, kv);
    if (rc) return rc;
    if (T < 0) return bad_arg(who, "T >= 0 required");
    if (T == 0) return QARL_OK;
    if (!k_bf16 || !v_bf16 || !slots) return bad_arg(who, "null k, v or slots");
    if (!aligned16(k_bf16) || !aligned16(v_bf16) || k_token_stride % 8 || k_head_stride % 8 || v_token_stride % 8 || v_head_stride % 8 ||
        ((uintptr_t)slots & 7u)) {
        set_error("%s: k and v must be 16-byte aligned, their strides multiples of 8 elements, slots 8-byte aligned", who);
        return QARL_ERR_ALIGNMENT;
    }
    return launch_kv_write(kv, k_bf16, k_token_stride, k_head_stride, v_bf16, v_token_stride, v_head_stride, T, slots, (hipStream_t)stream);
}

static double pair_at(int rotary_dim, double base, double original_len, double turns)
{
    return rotary_dim * log(original_len / (turns * 6.283185307179586)) / (2.0 * log(base));
}

int qarl_rope_frequencies(int rotary_dim, double base, int scaling, double factor, double original_len, double low, double high,
                          double *inv_freq, float *amplitude)
{
    const char *who = "qarl_rope_frequencies";
    if (!inv_freq || !amplitude) return bad_arg(who, "null output");
    if (rotary_dim <= 0 || !(base > 1.0) || !(base < 1e30)) return bad_arg(who, "rotary_dim > 0 and 1 < base < 1e30 required");
    if (scaling != QARL_ROPE_PLAIN && scaling != QARL_ROPE_LINEAR && scaling != QARL_ROPE_YARN && scaling != QARL_ROPE_BANDS) {
        set_error("%s: unknown scaling %d", who, scaling);
        return QARL_ERR_UNSUPPORTED;
    }
    if (rotary_dim % 16 != 0 || rotary_dim > 2 * QARL_ROPE_MAX_PAIRS) {
        set_error("%s: rotary_dim must be a multiple of 16 and at most %d (got %d)", who, 2 * QARL_ROPE_MAX_PAIRS, rotary_dim);
        return QARL_ERR_UNSUPPORTED;
    }
    const bool ramps = scaling == QARL_ROPE_YARN || scaling == QARL_ROPE_BANDS;
    if (scaling != QARL_ROPE_PLAIN && !(factor >= 1.0 && factor < 1e9)) return bad_arg(who, "factor must be at least 1 and finite");
    if (ramps && (!(original_len >= 1.0 && original_len < 1e18) || !(low > 0.0 && low < high && high < 1e9)))
        return bad_arg(who, "original_len >= 1 and 0 < low < high required");
    double first = 0.0, last = 0.0;
    if (scaling == QARL_ROPE_YARN) {
        first = fmax(floor(pair_at(rotary_dim, base, original_len, high)), 0.0);
        last = fmin(ceil(pair_at(rotary_dim, base, original_len, low)), rotary_dim - 1.0);
    }
    for (int i = 0; i < rotary_dim / 2; ++i) {
        const double f = pow(base, -2.0 * i / rotary_dim);
        double keep = 1.0;      // share of the pair's own frequency, beside the stretched one
        if (scaling == QARL_ROPE_LINEAR) keep = 0.0;
        else if (scaling == QARL_ROPE_YARN) keep = last <= 0.0 ? 0.0 : 1.0 - fmin(fmax((i - first) / fmax(last - first, 0.001), 0.0), 1.0);      // (last <= 0: no pair makes `low` turns)
        else if (scaling == QARL_ROPE_BANDS) keep = fmin(fmax((original_len * f / 6.283185307179586 - low) / (high - low), 0.0), 1.0);
        inv_freq[i] = scaling == QARL_ROPE_PLAIN ? f : f * keep + f / factor * (1.0 - keep);
    }
    *amplitude = scaling == QARL_ROPE_YARN ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
    return QARL_OK;
}

int qarl_rope_init(qarl_rope *rope, int rotary_dim, int layout, const double *inv_freq, float amplitude)
{
    const char *who = "qarl_rope_init";
    if (!rope || !inv_freq) return bad_arg(who, "null pointer");
    if (layout != QARL_ROPE_HALF && layout != QARL_ROPE_PAIRS) {
        set_error("%s: unknown layout %d", who, layout);
        return QARL_ERR_UNSUPPORTED;
    }
    if (rotary_dim <= 0 || rotary_dim % 16 != 0 || rotary_dim > 2 * QARL_ROPE_MAX_PAIRS) {
        set_error("%s: rotary_dim must be a positive multiple of 16 and at most %d (got %d)", who, 2 * QARL_ROPE_MAX_PAIRS, rotary_dim);
        return QARL_ERR_UNSUPPORTED;
    }
    if (!(amplitude > 0.f && amplitude < 1e30f)) return bad_arg(who, "amplitude must be positive and finite");
    for (int i = 0; i < rotary_dim / 2; ++i)
        if (!(inv_freq[i] >= 0.0 && inv_freq[i] < 3.1415926535897931)) return bad_arg(who, "frequencies must lie in [0, pi) radians a position");
    *rope = qarl_rope{};
    rope->rotary_dim = rotary_dim;
    rope->layout = layout;
    rope->amplitude = amplitude;
    // f / 2 pi in units of 2^-64 turns: the long double has 64 bits
    for (int i = 0; i < rotary_dim / 2; ++i)
        rope->turns[i] = (uint64_t)roundl((long double)inv_freq[i] / 6.283185307179586476925286766559L * 18446744073709551616.0L);
    return QARL_OK;
}

static int check_rope(const char *who, const qarl_rope *rope, int head_dim)
{
    if (!rope) return bad_arg(who, "null rope descriptor");
    if ((rope->layout != QARL_ROPE_HALF && rope->layout != QARL_ROPE_PAIRS) || rope->rotary_dim <= 0 || rope->rotary_dim % 16 != 0 ||
        rope->rotary_dim > 2 * QARL_ROPE_MAX_PAIRS)
        return bad_arg(who, "the rope descriptor was not made by qarl_rope_init");
    if (rope->rotary_dim > head_dim) {
        set_error("%s: rotary_dim %d exceeds head_dim %d", who, rope->rotary_dim, head_dim);
        return QARL_ERR_INVALID_ARG;
    }
    return QARL_OK;
}

// One side (queries, or keys) of a rotation: 16-byte aligned, strides of whole 16 bytes, outputs whose heads do not meet
static int check_heads(const char *who, const char *name, const RotHeads &x, int64_t T, int head_dim, int unit)
{
    if (x.heads == 0) return QARL_OK;
    if (!x.in || !x.out) {
        set_error("%s: null %s", who, name);
        return QARL_ERR_INVALID_ARG;
    }
    if (!aligned16(x.in) || !aligned16(x.out) || x.token_stride % unit || x.head_stride % unit || x.out_token_stride % unit || x.out_head_stride % unit) {
        set_error("%s: %s must be 16-byte aligned, its strides multiples of %d elements", who, name, unit);
        return QARL_ERR_ALIGNMENT;
    }
    // one of the two strides steps over all that the other spans
    const int64_t heads = x.heads, ts = x.out_token_stride < 0 ? -x.out_token_stride : x.out_token_stride,
                  hs = x.out_head_stride < 0 ? -x.out_head_stride : x.out_head_stride;
    const bool heads_apart = heads == 1 || hs >= head_dim, tokens_apart = T == 1 || ts >= head_dim;
    const bool nested = heads == 1 || T == 1 || ts >= (heads - 1) * hs + head_dim || hs >= (T - 1) * ts + head_dim;
    if (!heads_apart || !tokens_apart || !nested) {
        set_error("%s: heads of %s_out overlap (strides %lld, %lld)", who, name, (long long)x.out_token_stride, (long long)x.out_head_stride);
        return QARL_ERR_INVALID_ARG;
    }
    return QARL_OK;
}

int qarl_rotary(const qarl_rope *rope, const int64_t *positions, int64_t T, int head_dim, int dtype, const void *q, int64_t q_token_stride,
                int64_t q_head_stride, int q_heads, void *q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, const void *k,
                int64_t k_token_stride, int64_t k_head_stride, int k_heads, void *k_out, int64_t k_out_token_stride, int64_t k_out_head_stride,
                int inverse, void *stream)
{
    const char *who = "qarl_rotary";
    int rc = check_dtype(who, "dtype", dtype);
    if (rc) return rc;
    if (T < 0 || q_heads < 0 || k_heads < 0 || head_dim <= 0) return bad_arg(who, "T, q_heads, k_heads must not be negative, head_dim must be positive");
    if ((rc = check_rope(who, rope, head_dim))) return rc;
    if (head_dim % 16 != 0 || head_dim > 1024 || q_heads > 65536 || k_heads > 65536) {
        set_error("%s: need head_dim %% 16 == 0, head_dim <= 1024, heads <= 65536 (got %d, %d, %d)", who, head_dim, q_heads, k_heads);
        return QARL_ERR_UNSUPPORTED;
    }
    if (T == 0 || q_heads + k_heads == 0) return QARL_OK;
    if (!positions) return bad_arg(who, "null positions");
    const int unit = dtype == QARL_OUT_F32 ? 4 : 8;
    RotaryArgs a = {*rope, positions, T, head_dim, dtype == QARL_OUT_F32, inverse != 0,
                    {q, q_token_stride, q_head_stride, q_out, q_out_token_stride, q_out_head_stride, q_heads},
                    {k, k_token_stride, k_head_stride, k_out, k_out_token_stride, k_out_head_stride, k_heads}};
    if ((rc = check_heads(who, "q", a.q, T, head_dim, unit)) || (rc = check_heads(who, "k", a.k, T, head_dim, unit))) return rc;
    if ((uintptr_t)positions & 7u) {
        set_error("%s: positions must be 8-byte aligned", who);
        return QARL_ERR_ALIGNMENT;
    }
    return launch_rotary(a, (hipStream_t)stream);
}

int qarl_rotary_kv_write(const qarl_kv_cache *cache, const qarl_rope *rope, const int64_t *positions, int64_t T, const void *q_bf16, int64_t q_token_stride,
                         int64_t q_head_stride, int q_heads, void *q_out_bf16, int64_t q_out_token_stride, int64_t q_out_head_stride, const void *k_bf16,
                         int64_t k_token_stride, int64_t k_head_stride, const void *v_bf16, int64_t v_token_stride, int64_t v_head_stride,
                         const int64_t *slots, void *stream)
{
    const char *who = "qarl_rotary_kv_write";
    RotaryWriteArgs a = {};
    int rc = check_cache(cache, who, a.kv);
    if (rc || (rc = check_rope(who, rope, cache->head_dim))) return rc;
    if (T < 0 || q_heads < 0 || q_heads > 65536) return bad_arg(who, "T >= 0 and 0 <= q_heads <= 65536 required");
    if (T == 0) return QARL_OK;
    if (!positions || !k_bf16 || !v_bf16 || !slots) return bad_arg(who, "null positions, k, v or slots");
    a.q = RotHeads{q_bf16, q_token_stride, q_head_stride, q_out_bf16, q_out_token_stride, q_out_head_stride, q_heads};
    if ((rc = check_heads(who, "q", a.q, T, cache->head_dim, 8))) return rc;
    if (!aligned16(k_bf16) || !aligned16(v_bf16) || k_token_stride % 8 || k_head_stride % 8 || v_token_stride % 8 || v_head_stride % 8 ||
        ((uintptr_t)slots & 7u) || ((uintptr_t)positions & 7u)) {
        set_error("%s: k and v must be 16-byte aligned, their strides multiples of 8 elements, positions and slots 8-byte aligned", who);
        return QARL_ERR_ALIGNMENT;
    }
    a.rope = *rope;
    a.positions = positions;
    a.slots = slots;
    a.T = T;
    a.k = k_bf16;
    a.v = v_bf16;
    a.k_token_stride = k_token_stride;
    a.k_head_stride = k_head_stride;
    a.v_token_stride = v_token_stride;
    a.v_head_stride = v_head_stride;
    return launch_rotary_write(a, (hipStream_t)stream);
}

size_t qarl_sample_workspace_bytes(int T, int V)
{
    if (T <= 0 || V <= 0) return 0;
    return sample_ws_bytes(T, V);
}

int qarl_sample(const void *logits, int dtype, int64_t row_stride, int T, int V, const float *u, const float *temperature, const int32_t *top_k,
                const float *top_p, const float *min_p, int32_t *token, float *logprob, float *kept_logprob, void *ws, size_t ws_bytes, void *stream)
{
    const char *who = "qarl_sample";
    int rc = check_dtype(who, "dtype", dtype);
    if (rc) return rc;
    if (T < 0 || V <= 0) return bad_arg(who, "T >= 0 and V > 0 required");
    if (V > 1 << 20) {
        set_error("%s: V is at most 2^20 (got %d)", who, V);
        return QARL_ERR_UNSUPPORTED;
    }
    if (T == 0) return QARL_OK;
    if (!logits || !u || !token) return bad_arg(who, "null logits, u or token");
    if (T > 1 && row_stride < V) return bad_arg(who, "rows of logits overlap");
    if (((uintptr_t)logits & (dtype == QARL_OUT_F32 ? 3u : 1u)) ||
        (((uintptr_t)u | (uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p | (uintptr_t)token | (uintptr_t)logprob | (uintptr_t)kept_logprob) & 3u)) {
        set_error("%s: logits must be aligned to their type, the arrays of a value a row to 4 bytes", who);
        return QARL_ERR_ALIGNMENT;
    }
    const size_t need = sample_ws_bytes(T, V);
    if (need && (!ws || ws_bytes < need || !aligned16(ws))) {
        set_error("%s: needs %zu bytes of 16-byte aligned workspace (got %zu)", who, need, ws_bytes);
        return QARL_ERR_WORKSPACE;
    }
    SampleArgs a = {logits, dtype == QARL_OUT_F32, row_stride, T, V, u, temperature, top_p, min_p, top_k, token, logprob, kept_logprob, ws};
    return launch_sample(a, (hipStream_t)stream);
}

int qarl_kv_cache_read(const qarl_kv_cache *cache, const int32_t *block_table, int64_t table_stride, int table_width, const int32_t *offsets,
                       int S, int64_t total, void *k_out_bf16, void *v_out_bf16, void *stream)
{
    const char *who = "qarl_kv_cache_read";
    KvArgs kv;
    int rc = check_cache(cache, who, kv);
    if (rc) return rc;
    if (S < 0 || total < 0 || table_width < 0) return bad_arg(who, "S, total and table_width must not be negative");
    if (total == 0) return QARL_OK;
    if (S > 0 && (!offsets || (!block_table && table_width > 0))) return bad_arg(who, "null block_table or offsets");
    if (S > 1 && table_stride < table_width) return bad_arg(who, "rows of block_table overlap");
    if (!k_out_bf16 || !v_out_bf16) return bad_arg(who, "null output");
    if (!aligned16(k_out_bf16) || !aligned16(v_out_bf16) || ((uintptr_t)block_table & 3u) || ((uintptr_t)offsets & 3u)) {
        set_error("%s: outputs must be 16-byte aligned, index arrays 4-byte aligned", who);
        return QARL_ERR_ALIGNMENT;
    }
    return launch_kv_read(kv, block_table, table_stride, table_width, offsets, S, total, k_out_bf16, v_out_bf16, (hipStream_t)stream);
}

size_t qarl_paged_attention_workspace_bytes(const qarl_kv_cache *cache, int T, int q_heads, int S, int max_q_len, int max_kv_len)
{
    if (!cache || T <= 0 || q_heads <= 0 || S <= 0 || max_q_len <= 0 || max_kv_len <= 0 || cache->kv_heads <= 0 || q_heads % cache->kv_heads)
        return 0;
    return attention_ws_bytes(T, q_heads, cache->kv_heads, cache->head_dim, S, max_q_len, max_kv_len);
}

int qarl_paged_attention(const void *q_bf16, int64_t q_token_stride, int64_t q_head_stride, int T, int q_heads, const qarl_kv_cache *cache,
                         const int32_t *block_table, int64_t table_stride, int table_width, const int32_t *kv_lens, const int32_t *q_offsets,
                         int S, int max_q_len, int max_kv_len, float scale, int window, void *out, int out_dtype, float *lse, void *ws,
                         size_t ws_bytes, void *stream)
{
    const char *who = "qarl_paged_attention";
    AttnArgs a;
    int rc = check_cache(cache, who, a.kv);
    if (rc || (rc = check_dtype(who, "out_dtype", out_dtype))) return rc;
    if (T < 0 || S < 0 || q_heads <= 0 || max_q_len < 0 || max_kv_len < 0 || table_width < 0 || window < 0)
        return bad_arg(who, "T, S, max_q_len, max_kv_len, table_width and window must not be negative, q_heads must be positive");
    if (!(scale >= -1.0e38f && scale <= 1.0e38f)) return bad_arg(who, "scale must be finite, at most 1e38 in size");     // (times log2 e it is still finite)
    if (q_heads % a.kv.kv_heads != 0 || q_heads > 1024) {
        set_error("%s: q_heads must be a multiple of kv_heads and at most 1024 (got %d, %d)", who, q_heads, a.kv.kv_heads);
        return QARL_ERR_UNSUPPORTED;
    }
    if ((int64_t)T * (q_heads / a.kv.kv_heads) > 0x7fff0000LL) {
        set_error("%s: %d tokens of %d query heads per cached one exceed the row index", who, T, q_heads / a.kv.kv_heads);
        return QARL_ERR_UNSUPPORTED;
    }
    if (max_kv_len > 1 << 28) {
        set_error("%s: max_kv_len is at most 2^28 (got %d)", who, max_kv_len);
        return QARL_ERR_UNSUPPORTED;
    }
    if (T == 0 || S == 0) return QARL_OK;
    if (!q_bf16 || !out || !kv_lens || !q_offsets || (!block_table && table_width > 0)) return bad_arg(who, "null pointer");
    if (max_q_len == 0) return bad_arg(who, "max_q_len must be positive where there are tokens");
    if (S > 1 && table_stride < table_width) return bad_arg(who, "rows of block_table overlap");
    if (!aligned16(q_bf16) || !aligned16(out) || q_token_stride % 8 || q_head_stride % 8 || ((uintptr_t)block_table & 3u) ||
        ((uintptr_t)kv_lens & 3u) || ((uintptr_t)q_offsets & 3u) || ((uintptr_t)lse & 3u)) {
        set_error("%s: q and out must be 16-byte aligned, q's strides multiples of 8 elements, index arrays and lse 4-byte aligned", who);
        return QARL_ERR_ALIGNMENT;
    }
    const size_t need = qarl_paged_attention_workspace_bytes(cache, T, q_heads, S, max_q_len, max_kv_len);
    if (need && (!ws || ws_bytes < need || !aligned16(ws))) {
        set_error("%s: needs %zu bytes of 16-byte aligned workspace (got %zu)", who, need, ws_bytes);
        return QARL_ERR_WORKSPACE;
    }
    a.q = q_bf16;
    a.q_token_stride = q_token_stride;
    a.q_head_stride = q_head_stride;
    a.T = T;
    a.q_heads = q_heads;
    a.table = block_table;
    a.table_stride = table_stride;
    a.table_width = table_width;
    a.kv_lens = kv_lens;
    a.q_offsets = q_offsets;
    a.S = S;
    a.max_q_len = max_q_len;
    a.max_kv_len = max_kv_len;
    a.scale = scale;
    a.window = window;
    a.out = out;
    a.out_f32 = out_dtype == QARL_OUT_F32;
    a.lse = lse;
    a.ws = ws;
    return launch_attention(a, (hipStream_t)stream);
}

}  // extern "C"
