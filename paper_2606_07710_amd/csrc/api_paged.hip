// api_paged.hip -- the extern "C" boundary of the paged cache and of the token
// log probabilities: argument validation on the host, workspace queries and
// dispatch.  Nothing is enqueued unless every check passes.
#include <climits>
#include <cmath>

#include "wf_api_internal.h"

namespace {

using wf::aligned16;
using wf::head_dim_ok;
using wf::kMaxGamma;
using wf::kMaxQHeads;

constexpr int kMaxSeqs = 1024;
constexpr int kMaxSelected = 1024;
constexpr int kMaxCallRows = 1 << 20;
constexpr long long kMaxPositions = 1ll << 26;

inline bool dtype_ok(wf_dtype_t dt) { return dt == WF_F32 || dt == WF_BF16; }
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

wf_status_t check_cache(wf_dtype_t dt, const wf_paged_cache_t *c) {
    if (!dtype_ok(dt) || !c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v) ||
        !aligned16(c->bounds) || c->n_pages < 1 || c->n_kv_heads < 1 ||
        c->n_kv_heads > kMaxQHeads)
        return WF_ERR_INVALID_ARG;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
        return WF_ERR_INVALID_ARG;
    return head_dim_ok(c->head_dim) ? WF_OK : WF_ERR_UNSUPPORTED;
}

bool batch_ok(const wf_paged_cache_t &c, const wf_paged_batch_t *b, int n_rows, bool limit_rows) {
    return b && b->page_table && b->row_start && b->ctx_len && aligned4(b->page_table) &&
           aligned4(b->row_start) && aligned4(b->ctx_len) && b->n_seqs >= 1 &&
           b->n_seqs <= kMaxSeqs && b->max_pages >= 1 &&
           (long long)b->max_pages * c.page_size <= kMaxPositions && n_rows >= 0 &&
           n_rows <= kMaxCallRows &&
           (!limit_rows || (b->max_rows >= 1 && b->max_rows <= kMaxGamma));
}

bool q_heads_ok(int n_q_heads, int n_kv_heads) {
    return n_q_heads >= 1 && n_q_heads <= kMaxQHeads && n_kv_heads >= 1 &&
           n_q_heads % n_kv_heads == 0;
}

bool attn_sizes_ok(int n_rows, int n_q_heads, int n_kv_heads) {
    return q_heads_ok(n_q_heads, n_kv_heads) && n_rows >= 0 &&
           (long long)n_rows * n_q_heads <= (1 << 22);
}

bool select_sizes_ok(int n_rows, int n_kv_heads, int max_pages) {
    return n_rows >= 0 && n_kv_heads >= 1 && n_kv_heads <= kMaxQHeads &&
           (long long)n_rows * n_kv_heads <= (1 << 19) && max_pages >= 1 && max_pages <= 65536;
}

wf_status_t attn_common(wf_dtype_t dt, const void *q, const wf_paged_cache_t *c,
                        const wf_paged_batch_t *b, bool sparse, const int32_t *sel, int n_sel,
                        void *out, const uint64_t *tree_mask, int n_rows, int n_q_heads,
                        float softmax_scale, void *workspace, size_t workspace_bytes,
                        void *stream) {
    const wf_status_t st = check_cache(dt, c);
    if (st != WF_OK)
        return st;
    if (!batch_ok(*c, b, n_rows, true) || !attn_sizes_ok(n_rows, n_q_heads, c->n_kv_heads) ||
        !std::isfinite(softmax_scale) || softmax_scale <= 0.f)
        return WF_ERR_INVALID_ARG;
    if (n_rows == 0)
        return WF_OK;
    if (!q || !out || !aligned16(q) || !aligned16(out) || !aligned16(tree_mask) ||
        (sparse && (!sel || !aligned4(sel))))
        return WF_ERR_INVALID_ARG;
    const wf::PagedPlan p = wf::plan_paged(dt, b->max_rows, n_q_heads, c->n_kv_heads, sparse);
    if (!workspace || !aligned16(workspace) ||
        workspace_bytes < wf::paged_attn_workspace_bytes(p, c->head_dim))
        return WF_ERR_WORKSPACE;
    return wf::launch_paged_attn(dt, q, *c, *b, sel, n_sel, out, tree_mask, n_rows, n_q_heads,
                                 softmax_scale, p, workspace, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" {

wf_status_t wf_paged_append(wf_dtype_t dt, const wf_paged_cache_t *cache,
                            const wf_paged_batch_t *batch, const void *k, const void *v,
                            size_t kv_row_stride, const void *q, size_t q_row_stride, void *q_out,
                            int32_t n_q_heads, const int32_t *positions, double rope_base,
                            int32_t n_rows, void *stream) {
    const wf_status_t st = check_cache(dt, cache);
    if (st != WF_OK)
        return st;
    if (!batch_ok(*cache, batch, n_rows, false) || !std::isfinite(rope_base) || rope_base <= 0.0 ||
        !aligned4(positions))
        return WF_ERR_INVALID_ARG;
    if (q && !q_heads_ok(n_q_heads, cache->n_kv_heads))
        return WF_ERR_INVALID_ARG;
    if (n_rows == 0)
        return WF_OK;
    const size_t unit = dt == WF_F32 ? 4 : 8;
    const size_t most = (size_t)1 << 40;             // strides whose offsets fit 64 bits
    if (!k || !v || !aligned16(k) || !aligned16(v) || kv_row_stride % unit ||
        kv_row_stride < (size_t)cache->n_kv_heads * cache->head_dim || kv_row_stride > most)
        return WF_ERR_INVALID_ARG;
    if (q && (!q_out || !aligned16(q) || !aligned16(q_out) || q_row_stride % unit ||
              q_row_stride < (size_t)n_q_heads * cache->head_dim || q_row_stride > most))
        return WF_ERR_INVALID_ARG;
    return wf::launch_paged_append(dt, *cache, *batch, k, v, kv_row_stride, q, q_row_stride, q_out,
                                   n_q_heads, positions, rope_base, n_rows,
                                   static_cast<hipStream_t>(stream));
}

size_t wf_paged_verify_attn_workspace_bytes(wf_dtype_t dt, int32_t n_rows, int32_t n_seqs,
                                            int32_t max_rows, int32_t n_q_heads,
                                            int32_t n_kv_heads, int32_t head_dim) {
    if (!dtype_ok(dt) || !attn_sizes_ok(n_rows, n_q_heads, n_kv_heads) || !head_dim_ok(head_dim) ||
        n_seqs < 1 || n_seqs > kMaxSeqs || max_rows < 1 || max_rows > kMaxGamma)
        return 0;
    return wf::paged_attn_workspace_bytes(
        wf::plan_paged(dt, max_rows, n_q_heads, n_kv_heads, false), head_dim);
}

wf_status_t wf_paged_verify_attn(wf_dtype_t dt, const void *q, const wf_paged_cache_t *cache,
                                 const wf_paged_batch_t *batch, void *out,
                                 const uint64_t *tree_mask, int32_t n_rows, int32_t n_q_heads,
                                 float softmax_scale, void *workspace, size_t workspace_bytes,
                                 void *stream) {
    return attn_common(dt, q, cache, batch, false, nullptr, 0, out, tree_mask, n_rows, n_q_heads,
                       softmax_scale, workspace, workspace_bytes, stream);
}

size_t wf_paged_select_workspace_bytes(int32_t n_rows, int32_t n_kv_heads, int32_t max_pages) {
    return select_sizes_ok(n_rows, n_kv_heads, max_pages)
               ? wf::paged_select_workspace_bytes(n_rows, n_kv_heads, max_pages)
               : 0;
}

wf_status_t wf_paged_select(wf_dtype_t dt, const void *q, const wf_paged_cache_t *cache,
                            const wf_paged_batch_t *batch, int32_t *sel, int32_t n_sel,
                            int32_t n_recent, int32_t n_rows, int32_t n_q_heads, void *workspace,
                            size_t workspace_bytes, void *stream) {
    const wf_status_t st = check_cache(dt, cache);
    if (st != WF_OK)
        return st;
    if (!cache->bounds || !batch_ok(*cache, batch, n_rows, true) ||
        !select_sizes_ok(n_rows, cache->n_kv_heads, batch->max_pages) ||
        !q_heads_ok(n_q_heads, cache->n_kv_heads) || n_recent < 1 || n_sel < n_recent ||
        n_sel > kMaxSelected)
        return WF_ERR_INVALID_ARG;
    if (n_rows == 0)
        return WF_OK;
    if (!q || !sel || !aligned16(q) || !aligned4(sel))
        return WF_ERR_INVALID_ARG;
    if (!workspace || !aligned16(workspace) ||
        workspace_bytes <
            wf::paged_select_workspace_bytes(n_rows, cache->n_kv_heads, batch->max_pages))
        return WF_ERR_WORKSPACE;
    return wf::launch_paged_select(dt, q, *cache, *batch, sel, n_sel, n_recent, n_rows, n_q_heads,
                                   workspace, static_cast<hipStream_t>(stream));
}

size_t wf_paged_sparse_attn_workspace_bytes(wf_dtype_t dt, int32_t n_rows, int32_t n_q_heads,
                                            int32_t n_kv_heads, int32_t head_dim,
                                            int32_t page_size, int32_t n_sel) {
    if (!dtype_ok(dt) || !attn_sizes_ok(n_rows, n_q_heads, n_kv_heads) || !head_dim_ok(head_dim) ||
        (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128) || n_sel < 1 ||
        n_sel > kMaxSelected)
        return 0;
    return wf::paged_attn_workspace_bytes(wf::plan_paged(dt, 1, n_q_heads, n_kv_heads, true),
                                          head_dim);
}

wf_status_t wf_paged_sparse_attn(wf_dtype_t dt, const void *q, const wf_paged_cache_t *cache,
                                 const wf_paged_batch_t *batch, const int32_t *sel, int32_t n_sel,
                                 void *out, const uint64_t *tree_mask, int32_t n_rows,
                                 int32_t n_q_heads, float softmax_scale, void *workspace,
                                 size_t workspace_bytes, void *stream) {
    if (n_sel < 1 || n_sel > kMaxSelected)
        return WF_ERR_INVALID_ARG;
    // (chunks of 128 listed keys are counted in 32 bits)
    if (cache && attn_sizes_ok(n_rows, n_q_heads, cache->n_kv_heads) &&
        (long long)n_rows * cache->n_kv_heads *
                ((n_q_heads / cache->n_kv_heads + 15) / 16) *
                (((long long)n_sel * cache->page_size + 127) / 128) > INT32_MAX)
        return WF_ERR_INVALID_ARG;
    return attn_common(dt, q, cache, batch, true, sel, n_sel, out, tree_mask, n_rows, n_q_heads,
                       softmax_scale, workspace, workspace_bytes, stream);
}

namespace {
bool logprob_sizes_ok(wf_dtype_t dt, int n_rows, int vocab, int n_top) {
    return dtype_ok(dt) && n_rows >= 0 && n_rows <= kMaxCallRows && vocab >= 1 &&
           vocab <= (1 << 30) && n_top >= 0 && n_top <= 64 && n_top <= vocab;
}
}  // namespace

size_t wf_token_logprobs_workspace_bytes(wf_dtype_t dt, int32_t n_rows, int32_t vocab,
                                         int32_t n_top) {
    return logprob_sizes_ok(dt, n_rows, vocab, n_top)
               ? wf::token_logprobs_workspace_bytes(dt, n_rows, vocab, n_top)
               : 0;
}

wf_status_t wf_token_logprobs(wf_dtype_t dt, const void *logits, size_t row_stride,
                              const int32_t *tokens, int32_t n_rows, int32_t vocab, int32_t n_top,
                              float *logprob_out, float *entropy_out, int32_t *rank_out,
                              int32_t *top_ids, float *top_logprobs, void *workspace,
                              size_t workspace_bytes, void *stream) {
    if (!logprob_sizes_ok(dt, n_rows, vocab, n_top) || row_stride < (size_t)vocab ||
        row_stride > ((size_t)1 << 40))
        return WF_ERR_INVALID_ARG;
    if (n_rows == 0)
        return WF_OK;
    const uintptr_t elem = dt == WF_F32 ? 4 : 2;
    if (!logits || reinterpret_cast<uintptr_t>(logits) % elem || !aligned4(tokens) ||
        !aligned4(logprob_out) || !aligned4(entropy_out) || !aligned4(rank_out) ||
        !aligned4(top_ids) || !aligned4(top_logprobs))
        return WF_ERR_INVALID_ARG;
    // tokens and what is said of them come together, as do the alternatives
    if (tokens ? !logprob_out : logprob_out || rank_out)
        return WF_ERR_INVALID_ARG;
    if ((n_top > 0) != (top_ids != nullptr) || (n_top > 0) != (top_logprobs != nullptr))
        return WF_ERR_INVALID_ARG;
    if (!workspace || !aligned16(workspace) ||
        workspace_bytes < wf::token_logprobs_workspace_bytes(dt, n_rows, vocab, n_top))
        return WF_ERR_WORKSPACE;
    return wf::launch_token_logprobs(dt, logits, row_stride, tokens, n_rows, vocab, n_top,
                                     logprob_out, entropy_out, rank_out, top_ids, top_logprobs,
                                     workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
