// api_lowbit.hip -- the extern "C" boundary of the 8-bit KV cache and the
// 4-bit weights: argument validation on the host, workspace queries and
// dispatch.  Nothing is enqueued unless every check passes.
#include <climits>
#include <cmath>

#include "wf_api_internal.h"

namespace {

using wf::aligned16;
using wf::head_dim_ok;
using wf::kMaxGamma;
using wf::kMaxLayers;
using wf::kMaxQHeads;

constexpr int kMaxW4Rows = 64;
constexpr int kMaxW4Inputs = 1 << 20;

wf_status_t check_cache(const wf_kv8_cache_t *c) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !aligned16(c->k) ||
        !aligned16(c->v) || c->n_kv_heads < 1 || c->n_kv_heads > kMaxQHeads || c->cap < 1 ||
        c->cap > INT32_MAX / 2)
        return WF_ERR_INVALID_ARG;
    return head_dim_ok(c->head_dim) ? WF_OK : WF_ERR_UNSUPPORTED;
}

inline bool dtype_ok(wf_dtype_t dt) { return dt == WF_F32 || dt == WF_BF16; }
inline wf_dtype_t storage(wf_dtype_t dt) { return dt == WF_BF16_TILED ? WF_BF16 : dt; }
inline size_t elem_bytes(wf_dtype_t dt) { return dt == WF_F32 ? 4 : 2; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Workspace of the 8-bit prefill: the prefill's own (bf16: the zero block; fp32:
// nothing), then the K rows and the V rows, [n_kv_heads][n_tok][head_dim] each; this is
// where the K rows start.
size_t kv8_prefill_rows_at(wf_dtype_t dt, int n_tok, int d_in, const wf_kv8_cache_t &c) {
    return align256(wf::prefill_workspace_bytes(storage(dt), n_tok, d_in, c.n_kv_heads,
                                                c.head_dim));
}

wf_status_t kv8_attn_common(wf_dtype_t dt, const void *q, const wf_kv8_cache_t *c, void *out,
                            const uint64_t *tree_mask, int gamma, int ctx_len, int n_q_heads,
                            float softmax_scale, int num_splits, void *workspace,
                            size_t workspace_bytes, void *stream) {
    wf_status_t st = check_cache(c);
    if (st != WF_OK)
        return st;
    st = wf::check_attn(dt, gamma, ctx_len, n_q_heads, c->n_kv_heads, c->head_dim, num_splits);
    if (st != WF_OK)
        return st;
    if (!q || !out || !aligned16(q) || !aligned16(out))
        return WF_ERR_INVALID_ARG;
    if ((long long)ctx_len + gamma > c->cap)
        return WF_ERR_INVALID_ARG;
    if (!std::isfinite(softmax_scale) || softmax_scale <= 0.f)
        return WF_ERR_INVALID_ARG;
    const wf::AttnPlan p = wf::plan_attn8(dt, gamma, ctx_len, n_q_heads, c->n_kv_heads,
                                          c->head_dim, num_splits);
    const size_t need = wf::attn_workspace_bytes(p, gamma, n_q_heads, c->head_dim);
    if (!workspace || workspace_bytes < need || !aligned16(workspace))
        return WF_ERR_WORKSPACE;
    return wf::launch_attn8(dt, q, *c, out, gamma, ctx_len, n_q_heads, softmax_scale, tree_mask,
                            p, workspace, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" {

size_t wf_kv8_code_bytes(int32_t n_kv_heads, int32_t cap, int32_t head_dim) {
    if (n_kv_heads < 1 || n_kv_heads > kMaxQHeads || cap < 1 || cap > INT32_MAX / 2 ||
        !head_dim_ok(head_dim))
        return 0;
    return (size_t)n_kv_heads * wf::kv8_blocks(cap) * WF_KV8_BLOCK * head_dim;
}

size_t wf_kv8_scale_bytes(int32_t n_kv_heads, int32_t cap) {
    if (n_kv_heads < 1 || n_kv_heads > kMaxQHeads || cap < 1 || cap > INT32_MAX / 2)
        return 0;
    return (size_t)n_kv_heads * wf::kv8_blocks(cap);
}

wf_status_t wf_kv8_append(wf_dtype_t dt, const wf_kv8_cache_t *cache, const void *k,
                          const void *v, int32_t n_tok, int32_t start_pos, size_t tok_stride,
                          size_t head_stride, void *stream) {
    const wf_status_t st = check_cache(cache);
    if (st != WF_OK)
        return st;
    if (!dtype_ok(dt) || n_tok < 0 || start_pos < 0 ||
        (long long)start_pos + n_tok > cache->cap)
        return WF_ERR_INVALID_ARG;
    if (n_tok == 0)
        return WF_OK;
    const size_t unit = 16 / elem_bytes(dt);
    if (!k || !v || !aligned16(k) || !aligned16(v) || tok_stride % unit || head_stride % unit)
        return WF_ERR_INVALID_ARG;
    return wf::launch_kv8_append(dt, *cache, k, v, n_tok, start_pos, tok_stride, head_stride,
                                 nullptr, static_cast<hipStream_t>(stream));
}

size_t wf_kv8_only_prefill_workspace_bytes(wf_dtype_t dt, int32_t n_tok, int32_t d_in,
                                           int32_t n_kv_heads, int32_t head_dim) {
    if (n_tok < 1 || wf::check_prefill(dt, n_tok, 0, n_tok, d_in, n_kv_heads, head_dim, 1.0) !=
                         WF_OK)
        return 0;
    const wf_kv8_cache_t c{nullptr, nullptr, nullptr, nullptr, n_kv_heads, n_tok, head_dim};
    return kv8_prefill_rows_at(dt, n_tok, d_in, c) +
           2 * align256((size_t)n_kv_heads * n_tok * head_dim * elem_bytes(dt));
}

wf_status_t wf_kv8_only_prefill(wf_dtype_t dt, const void *x, const void *w_k, const void *w_v,
                                const wf_kv8_cache_t *cache, int32_t n_tok, int32_t start_pos,
                                int32_t d_in, double rope_base, void *workspace,
                                size_t workspace_bytes, void *stream) {
    wf_status_t st = check_cache(cache);
    if (st != WF_OK)
        return st;
    st = wf::check_prefill(dt, n_tok, start_pos, cache->cap, d_in, cache->n_kv_heads,
                           cache->head_dim, rope_base);
    if (st != WF_OK)
        return st;
    if (n_tok == 0)
        return WF_OK;
    if (!x || !w_k || !w_v || !aligned16(x) || !aligned16(w_k) || !aligned16(w_v))
        return WF_ERR_INVALID_ARG;
    const size_t need = wf_kv8_only_prefill_workspace_bytes(dt, n_tok, d_in, cache->n_kv_heads,
                                                            cache->head_dim);
    if (!workspace || workspace_bytes < need || !aligned16(workspace))
        return WF_ERR_WORKSPACE;
    const int dh = cache->head_dim;
    const size_t eb = elem_bytes(dt);
    char *kr = static_cast<char *>(workspace) + kv8_prefill_rows_at(dt, n_tok, d_in, *cache);
    char *vr = kr + align256((size_t)cache->n_kv_heads * n_tok * dh * eb);
    // The prefill writes row start_pos + t of a head's cache rows; handed a
    // cache of n_tok rows per head that begins start_pos rows earlier, it
    // writes row t of the workspace's [n_kv_heads][n_tok][head_dim].
    const uintptr_t back = (uintptr_t)start_pos * dh * eb;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    st = wf::launch_prefill(dt, x, w_k, w_v,
                            reinterpret_cast<void *>(reinterpret_cast<uintptr_t>(kr) - back),
                            reinterpret_cast<void *>(reinterpret_cast<uintptr_t>(vr) - back),
                            n_tok, start_pos, n_tok, d_in, cache->n_kv_heads, dh, rope_base,
                            workspace, s);
    if (st != WF_OK)
        return st;
    // The fp32 prefill has no zero block, so its rows lie where other calls have
    // theirs: the append leaves zeros there.
    const char *zero_end =
        dt == WF_F32 ? static_cast<const char *>(workspace) + wf::kCounterBytes : nullptr;
    return wf::launch_kv8_append(storage(dt), *cache, kr, vr, n_tok, start_pos, dh,
                                 (size_t)n_tok * dh, zero_end, s);
}

size_t wf_kv8_verify_attn_workspace_bytes(wf_dtype_t dt, int32_t gamma, int32_t ctx_len,
                                          int32_t n_q_heads, int32_t n_kv_heads,
                                          int32_t head_dim, int32_t num_splits) {
    if (wf::check_attn(dt, gamma, ctx_len, n_q_heads, n_kv_heads, head_dim, num_splits) != WF_OK)
        return 0;
    const wf::AttnPlan p = wf::plan_attn8(dt, gamma, ctx_len, n_q_heads, n_kv_heads, head_dim,
                                          num_splits);
    return wf::attn_workspace_bytes(p, gamma, n_q_heads, head_dim);
}

wf_status_t wf_kv8_verify_attn(wf_dtype_t dt, const void *q, const wf_kv8_cache_t *cache,
                               void *out, int32_t gamma, int32_t ctx_len, int32_t n_q_heads,
                               float softmax_scale, int32_t num_splits, void *workspace,
                               size_t workspace_bytes, void *stream) {
    return kv8_attn_common(dt, q, cache, out, nullptr, gamma, ctx_len, n_q_heads, softmax_scale,
                           num_splits, workspace, workspace_bytes, stream);
}

wf_status_t wf_kv8_verify_attn_tree(wf_dtype_t dt, const void *q, const wf_kv8_cache_t *cache,
                                    void *out, const uint64_t *tree_mask, int32_t gamma,
                                    int32_t ctx_len, int32_t n_q_heads, float softmax_scale,
                                    int32_t num_splits, void *workspace,
                                    size_t workspace_bytes, void *stream) {
    if (!tree_mask || !aligned16(tree_mask))
        return WF_ERR_INVALID_ARG;
    return kv8_attn_common(dt, q, cache, out, tree_mask, gamma, ctx_len, n_q_heads,
                           softmax_scale, num_splits, workspace, workspace_bytes, stream);
}

wf_status_t wf_kv8_compact_path(const wf_kv8_cache_t *cache, const int32_t *accept,
                                const int32_t *path, int32_t gamma, int32_t ctx_len,
                                int32_t n_layers, size_t code_layer_stride,
                                size_t scale_layer_stride, void *stream) {
    const wf_status_t st = check_cache(cache);
    if (st != WF_OK)
        return st;
    if (!accept || !path || gamma < 1 || gamma > kMaxGamma || ctx_len < 0 ||
        (long long)ctx_len + gamma > cache->cap || n_layers < 1 || n_layers > kMaxLayers)
        return WF_ERR_INVALID_ARG;
    if (n_layers > 1 &&
        (code_layer_stride < wf_kv8_code_bytes(cache->n_kv_heads, cache->cap, cache->head_dim) ||
         scale_layer_stride < wf_kv8_scale_bytes(cache->n_kv_heads, cache->cap) ||
         code_layer_stride % 16))
        return WF_ERR_INVALID_ARG;
    return wf::launch_kv8_compact(*cache, accept, path, gamma, ctx_len, n_layers,
                                  n_layers > 1 ? code_layer_stride : 0,
                                  n_layers > 1 ? scale_layer_stride : 0,
                                  static_cast<hipStream_t>(stream));
}

namespace {
// a weight's shape: fewer than 2^26 tiles of 16 x 128 (the grid of the packing)
bool w4_weight_ok(int rows, int cols) {
    return rows >= 1 && rows <= (1 << 30) && cols >= 32 && cols % 32 == 0 &&
           cols <= kMaxW4Inputs &&
           (long long)((rows + 15) / 16) * ((cols + 127) / 128) < (1 << 26);
}
}  // namespace

wf_status_t wf_w4_quantize(const void *w, int32_t rows, int32_t cols, void *codes,
                           uint8_t *scales, void *stream) {
    if (!w || !codes || !scales || !aligned16(w) || !aligned16(codes) || !w4_weight_ok(rows, cols))
        return WF_ERR_INVALID_ARG;
    return wf::launch_w4_quantize(w, rows, cols, codes, scales, static_cast<hipStream_t>(stream));
}

size_t wf_w4_packed_bytes(int32_t rows, int32_t cols) {
    return w4_weight_ok(rows, cols) ? wf::w4_packed_bytes(rows, cols) : 0;
}

wf_status_t wf_w4_pack(const void *codes, const uint8_t *scales, int32_t rows, int32_t cols,
                       void *packed, size_t packed_bytes, void *stream) {
    if (!codes || !scales || !packed || !aligned16(codes) || !aligned16(packed) ||
        !w4_weight_ok(rows, cols))
        return WF_ERR_INVALID_ARG;
    if (packed_bytes < wf::w4_packed_bytes(rows, cols))
        return WF_ERR_WORKSPACE;
    return wf::launch_w4_pack(codes, scales, rows, cols, packed, static_cast<hipStream_t>(stream));
}

namespace {
bool linear_w4_shape_ok(int n_rows, int n_out, int k_in) {
    return n_rows >= 1 && n_rows <= kMaxW4Rows && w4_weight_ok(n_out, k_in);
}
}  // namespace

size_t wf_linear_w4_workspace_bytes(int32_t n_rows, int32_t n_out, int32_t k_in) {
    return linear_w4_shape_ok(n_rows, n_out, k_in)
               ? wf::linear_w4_workspace_bytes(n_rows, n_out, k_in)
               : 0;
}

wf_status_t wf_linear_w4(const void *x, const void *packed, const void *res, wf_dtype_t out_dt,
                         void *y, int32_t n_rows, int32_t n_out, int32_t k_in, void *workspace,
                         size_t workspace_bytes, void *stream) {
    if (!dtype_ok(out_dt) || !x || !packed || !y || !aligned16(x) || !aligned16(packed) ||
        !linear_w4_shape_ok(n_rows, n_out, k_in))
        return WF_ERR_INVALID_ARG;
    const size_t need = wf::linear_w4_workspace_bytes(n_rows, n_out, k_in);
    if (need && (!workspace || workspace_bytes < need || !aligned16(workspace)))
        return WF_ERR_WORKSPACE;
    return wf::launch_linear_w4(static_cast<const uint16_t *>(x),
                                static_cast<const uint8_t *>(packed),
                                static_cast<const uint16_t *>(res), out_dt == WF_F32, y, n_rows,
                                n_out, k_in, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
