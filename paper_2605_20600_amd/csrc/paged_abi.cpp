// C ABI of the paged cache, its attention and the token scores: every argument
// is checked here before anything is launched.  No entry point throws.
#include <cmath>
#include <cstdint>

#include "../../include/headkv.h"
#include "paged.h"
#include "paged_check.h"

using namespace headkv;

extern "C" {

headkv_status headkv_paged_plan(const headkv_paged_config* cfg, size_t* page_bytes,
                                size_t* pool_bytes) {
    PagedDims c;
    if (headkv_status st = make_dims(cfg, &c)) return st;
    if (page_bytes) *page_bytes = (size_t)c.page_bytes;
    if (pool_bytes) *pool_bytes = (size_t)c.page_bytes * (size_t)c.num_pages;
    return HEADKV_OK;
}

headkv_status headkv_paged_write(const headkv_paged_config* cfg, void* pool,
                                 const headkv_paged_lists* lists, const uint16_t* k,
                                 const uint16_t* v, int64_t list_stride, int64_t token_stride,
                                 int64_t head_stride, int32_t tokens, const int32_t* counts,
                                 void* stream) {
    PagedDims c;
    PagedLists l;
    if (headkv_status st = make_dims(cfg, &c)) return st;
    if (headkv_status st = make_lists(c, lists, true, &l)) return st;
    if (tokens < 0) return bad("tokens must be >= 0");
    if (tokens == 0) return HEADKV_OK;  // rows of no tokens may have no address
    if (headkv_status st = check_rows(k, v, list_stride, token_stride, head_stride)) return st;
    if (!pool || !aligned(pool, 256)) return bad("pool is NULL or not 256-byte aligned");
    if (!aligned(counts, 4)) return bad("counts not aligned");
    const PagedRows r{list_stride, token_stride, head_stride};
    return hip_status(launch_paged_write(c, static_cast<char*>(pool), l, k, v, r, tokens, counts,
                                         stream),
                      "paged write launch");
}

headkv_status headkv_paged_read(const headkv_paged_config* cfg, const void* pool,
                                const headkv_paged_lists* lists, int32_t begin, int32_t tokens,
                                uint16_t* k, uint16_t* v, int64_t list_stride,
                                int64_t token_stride, int64_t head_stride, void* stream) {
    PagedDims c;
    PagedLists l;
    if (headkv_status st = make_dims(cfg, &c)) return st;
    if (headkv_status st = make_lists(c, lists, true, &l)) return st;
    if (tokens < 0) return bad("tokens must be >= 0");
    if (tokens == 0) return HEADKV_OK;
    if (headkv_status st = check_rows(k, v, list_stride, token_stride, head_stride)) return st;
    if (!pool || !aligned(pool, 256)) return bad("pool is NULL or not 256-byte aligned");
    if ((l.lists > 1 && list_stride < c.d) || (tokens > 1 && token_stride < c.d) ||
        (c.heads > 1 && head_stride < c.d))
        return bad("output rows overlap: a stride is smaller than head_dim");
    const PagedRows r{list_stride, token_stride, head_stride};
    return hip_status(launch_paged_read(c, static_cast<const char*>(pool), l, begin, tokens, k, v,
                                        r, stream),
                      "paged read launch");
}

headkv_status headkv_paged_attn_plan(const headkv_paged_config* cfg,
                                     const headkv_paged_lists* own,
                                     const headkv_paged_lists* shared, size_t* workspace_bytes) {
    PagedDims c;
    PagedLists o, s;
    if (headkv_status st = make_dims(cfg, &c)) return st;
    if (headkv_status st = make_lists(c, own, false, &o)) return st;
    if (shared)
        if (headkv_status st = make_lists(c, shared, false, &s)) return st;
    if (!workspace_bytes) return bad("workspace_bytes is NULL");
    *workspace_bytes = paged_attn_workspace(c, o, shared ? &s : nullptr);
    return HEADKV_OK;
}

headkv_status headkv_paged_attn(const headkv_paged_config* cfg, const void* pool,
                                const headkv_paged_lists* own, const headkv_paged_lists* shared,
                                const int32_t* share, const uint16_t* q, int64_t q_stride,
                                float* out, float* lse, void* workspace, size_t workspace_bytes,
                                void* stream) {
    PagedDims c;
    PagedLists o, s;
    if (headkv_status st = make_dims(cfg, &c)) return st;
    if (headkv_status st = make_lists(c, own, true, &o)) return st;
    if ((shared != nullptr) != (share != nullptr))
        return bad("shared and share must both be given or both be NULL");
    if (shared)
        if (headkv_status st = make_lists(c, shared, true, &s)) return st;
    if (!pool || !aligned(pool, 256)) return bad("pool is NULL or not 256-byte aligned");
    if (!q || !out) return bad("q / out is NULL");
    if (!aligned(q, 16) || !aligned(out, 16)) return bad("q / out not 16-byte aligned");
    if (!aligned(lse, 4) || !aligned(share, 4)) return bad("lse / share not aligned");
    if (q_stride < 0 || q_stride % 8) return bad("q_stride must be >= 0 and a multiple of 8");
    const size_t need = paged_attn_workspace(c, o, shared ? &s : nullptr);
    if (headkv_status st = check_workspace(workspace, workspace_bytes, need)) return st;
    return hip_status(launch_paged_attn(c, static_cast<const char*>(pool), o,
                                        shared ? &s : nullptr, share, q, q_stride, out, lse,
                                        workspace, stream),
                      "paged attention launch");
}

static constexpr int kMostTokens = 1 << 24;  // of a row: sums with lengths are 32-bit numbers

headkv_status headkv_paged_attn_tokens_plan(const headkv_paged_config* cfg,
                                            const headkv_paged_lists* own,
                                            const headkv_paged_lists* shared, int32_t tokens,
                                            size_t* workspace_bytes) {
    PagedDims c;
    PagedLists o, s;
    if (headkv_status st = make_dims(cfg, &c)) return st;
    if (headkv_status st = make_lists(c, own, false, &o)) return st;
    if (shared)
        if (headkv_status st = make_lists(c, shared, false, &s)) return st;
    if (tokens < 0) return bad("tokens must be >= 0");
    if (tokens > kMostTokens) return hip_status(kTooLarge, "");
    if (!workspace_bytes) return bad("workspace_bytes is NULL");
    const size_t need = paged_attn_tokens_workspace(c, o, shared ? &s : nullptr, tokens);
    if (!need) return hip_status(kTooLarge, "");
    *workspace_bytes = need;
    return HEADKV_OK;
}

headkv_status headkv_paged_attn_tokens(const headkv_paged_config* cfg, const void* pool,
                                       const headkv_paged_lists* own,
                                       const headkv_paged_lists* shared, const int32_t* share,
                                       int32_t tokens, const int32_t* counts,
                                       const int32_t* window, const uint16_t* q,
                                       int64_t q_row_stride, int64_t q_token_stride, float* out,
                                       float* lse, void* workspace, size_t workspace_bytes,
                                       void* stream) {
    PagedDims c;
    PagedLists o, s;
    if (headkv_status st = make_dims(cfg, &c)) return st;
    if (headkv_status st = make_lists(c, own, true, &o)) return st;
    if ((shared != nullptr) != (share != nullptr))
        return bad("shared and share must both be given or both be NULL");
    if (shared)
        if (headkv_status st = make_lists(c, shared, true, &s)) return st;
    if (tokens < 0) return bad("tokens must be >= 0");
    if (tokens == 0) return HEADKV_OK;  // rows of no tokens may have no address
    if (tokens > kMostTokens) return hip_status(kTooLarge, "");
    if (!pool || !aligned(pool, 256)) return bad("pool is NULL or not 256-byte aligned");
    if (!q || !out) return bad("q / out is NULL");
    if (!aligned(q, 16) || !aligned(out, 16)) return bad("q / out not 16-byte aligned");
    if (!aligned(lse, 4) || !aligned(share, 4) || !aligned(counts, 4) || !aligned(window, 4))
        return bad("lse / share / counts / window not aligned");
    if (q_row_stride < 0 || q_row_stride % 8 || q_token_stride < 0 || q_token_stride % 8)
        return bad("strides of q must be >= 0 and multiples of 8");
    const size_t need = paged_attn_tokens_workspace(c, o, shared ? &s : nullptr, tokens);
    if (!need) return hip_status(kTooLarge, "");
    if (headkv_status st = check_workspace(workspace, workspace_bytes, need)) return st;
    const PagedTokens t{tokens, counts, window, q, q_row_stride, q_token_stride};
    return hip_status(launch_paged_attn_tokens(t, c, static_cast<const char*>(pool), o,
                                               shared ? &s : nullptr, share, out, lse, workspace,
                                               stream),
                      "paged attention launch");
}

static headkv_status check_scores(int32_t rows, int32_t vocab, int32_t top) {
    if (rows < 0 || vocab < 1) return bad("rows must be >= 0 and vocab >= 1");
    if (vocab > (1 << 24)) return unsupported("vocab > 2^24");
    if (top < 0 || top > HEADKV_MAX_TOP || top > vocab)
        return bad("top out of [0, min(HEADKV_MAX_TOP, vocab)]");
    return HEADKV_OK;
}

headkv_status headkv_logprobs_plan(int32_t rows, int32_t vocab, int32_t top,
                                   size_t* workspace_bytes) {
    if (headkv_status st = check_scores(rows, vocab, top)) return st;
    if (!workspace_bytes) return bad("workspace_bytes is NULL");
    *workspace_bytes = logprobs_workspace(rows, vocab, top);
    return HEADKV_OK;
}

headkv_status headkv_token_logprobs(const void* logits, int32_t logits_type, int32_t rows,
                                    int32_t vocab, int64_t row_stride, const int32_t* tokens,
                                    float temperature, int32_t top, float* logprob,
                                    float* entropy, int32_t* rank, float* top_logprob,
                                    int32_t* top_index, void* workspace, size_t workspace_bytes,
                                    void* stream) {
    if (headkv_status st = check_scores(rows, vocab, top)) return st;
    if (logits_type != HEADKV_LOGITS_BF16 && logits_type != HEADKV_LOGITS_F32)
        return bad("unknown logits_type");
    if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.f / temperature))
        return bad("temperature must be > 0");
    if (row_stride < vocab) return bad("row_stride < vocab");
    if (rows == 0) return HEADKV_OK;
    if (!logits || !tokens || !logprob) return bad("logits / tokens / logprob is NULL");
    if (top && (!top_logprob || !top_index)) return bad("top_logprob / top_index is NULL");
    if (!aligned(logits, logits_type == HEADKV_LOGITS_BF16 ? 2 : 4) || !aligned(tokens, 4) ||
        !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(rank, 4) ||
        !aligned(top_logprob, 4) || !aligned(top_index, 4))
        return bad("a pointer is not aligned");
    const size_t need = logprobs_workspace(rows, vocab, top);
    if (headkv_status st = check_workspace(workspace, workspace_bytes, need)) return st;
    const ScoreArgs a{logits,      tokens,    logprob,    entropy, rank,  top_logprob,
                      top_index,   row_stride, rows,      vocab,   top,   1.f / temperature};
    return hip_status(launch_token_logprobs(a, logits_type, workspace, stream),
                      "token scores launch");
}

}  // extern "C"
