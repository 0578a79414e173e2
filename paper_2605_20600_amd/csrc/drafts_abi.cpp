// C ABI of the page tables and of the verification of drafted tokens: every argument is
// checked here before anything is launched.  No entry point throws.
#include <cmath>
#include <cstdint>

#include "../../include/headkv.h"
#include "paged.h"
#include "paged_check.h"

using namespace headkv;

namespace {

headkv_status check_sizes(int32_t rows, int32_t drafts, int32_t vocab) {
    if (rows < 0 || vocab < 1) return bad("rows must be >= 0 and vocab >= 1");
    if (vocab > (1 << 24)) return unsupported("vocab > 2^24");
    if (drafts < 0 || drafts > HEADKV_MAX_DRAFTS)
        return unsupported("drafts out of [0, HEADKV_MAX_DRAFTS]");
    return HEADKV_OK;
}

headkv_status check_tables(const headkv_paged_tables* t) {
    if (!t) return bad("tables is NULL");
    if (t->kv_heads < 1 || t->kv_heads > 1024) return unsupported("kv_heads out of [1, 1024]");
    if (t->page_tokens != 32 && t->page_tokens != 64 && t->page_tokens != 128 &&
        t->page_tokens != 256)
        return unsupported("page_tokens must be 32, 64, 128 or 256");
    if (t->num_pages < 1 || t->lists < 1 || t->rows < 1 || t->max_pages < 1)
        return bad("num_pages, lists, rows and max_pages must be >= 1");
    if (t->lists % t->rows) return bad("lists must be a multiple of rows");
    if ((int64_t)t->lists * t->kv_heads > (1 << 24)) return unsupported("lists * kv_heads > 2^24");
    if (t->max_pages > (1 << 22)) return unsupported("max_pages > 2^22");
    if ((int64_t)t->lists * t->kv_heads * t->max_pages >= (1ll << 31))
        return unsupported("lists * kv_heads * max_pages >= 2^31");
    return HEADKV_OK;
}

}  // namespace

extern "C" {

headkv_status headkv_paged_extend_plan(const headkv_paged_tables* tables,
                                       size_t* workspace_bytes) {
    if (headkv_status st = check_tables(tables)) return st;
    if (!workspace_bytes) return bad("workspace_bytes is NULL");
    *workspace_bytes = extend_workspace();
    return HEADKV_OK;
}

headkv_status headkv_paged_extend(const headkv_paged_tables* tables, const int32_t* advance,
                                  const int32_t* counts, int32_t tokens, void* workspace,
                                  size_t workspace_bytes, void* stream) {
    if (headkv_status st = check_tables(tables)) return st;
    if (tokens < 0) return bad("tokens must be >= 0");
    if (tokens > (1 << 24)) return unsupported("tokens > 2^24");
    const headkv_paged_tables& t = *tables;
    if (!t.pages || !t.len || !t.first || !t.free_pages || !t.free_state)
        return bad("pages / len / first / free_pages / free_state is NULL");
    const void* all[] = {t.pages,      t.len,        t.first, t.order, t.window,
                         t.free_pages, t.free_state, advance, counts};
    for (const void* p : all)
        if (!aligned(p, 4)) return bad("a pointer is not aligned");
    if (headkv_status st = check_workspace(workspace, workspace_bytes, extend_workspace()))
        return st;
    return hip_status(launch_extend(t, advance, counts, tokens, workspace, stream),
                      "page tables launch");
}

headkv_status headkv_verify_plan(int32_t rows, int32_t drafts, int32_t vocab,
                                 size_t* workspace_bytes) {
    if (headkv_status st = check_sizes(rows, drafts, vocab)) return st;
    if (!workspace_bytes) return bad("workspace_bytes is NULL");
    *workspace_bytes = verify_workspace(rows, drafts, vocab);
    return HEADKV_OK;
}

headkv_status headkv_verify_drafts(const void* logits, const void* draft_logits,
                                   int32_t logits_type, int32_t rows, int32_t drafts,
                                   int32_t vocab, int64_t row_stride, int64_t token_stride,
                                   int64_t draft_row_stride, int64_t draft_token_stride,
                                   const int32_t* tokens, const int32_t* counts,
                                   const float* uniforms, double temperature, int32_t* out_tokens,
                                   int32_t* out_count, float* out_logprob, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    if (headkv_status st = check_sizes(rows, drafts, vocab)) return st;
    if (logits_type != HEADKV_LOGITS_BF16 && logits_type != HEADKV_LOGITS_F32)
        return bad("unknown logits_type");
    const double k = temperature == 0 ? 0.0 : 1.4426950408889634074 / temperature;
    if (!(temperature >= 0) || !std::isfinite(temperature) || !std::isfinite(k))
        return bad("temperature must be 0, or > 0 and finite with its inverse");
    if (row_stride < 0 || token_stride < 0 || draft_row_stride < 0 || draft_token_stride < 0)
        return bad("strides must be >= 0");
    if (rows == 0) return HEADKV_OK;
    if (!logits || !uniforms || !out_tokens || !out_count)
        return bad("logits / uniforms / out_tokens / out_count is NULL");
    if (drafts && !tokens) return bad("tokens is NULL");
    const size_t size = logits_type == HEADKV_LOGITS_BF16 ? 2 : 4;
    if (!aligned(logits, size) || !aligned(draft_logits, size) || !aligned(tokens, 4) ||
        !aligned(counts, 4) || !aligned(uniforms, 4) || !aligned(out_tokens, 4) ||
        !aligned(out_count, 4) || !aligned(out_logprob, 4))
        return bad("a pointer is not aligned");
    const size_t need = verify_workspace(rows, drafts, vocab);
    if (headkv_status st = check_workspace(workspace, workspace_bytes, need)) return st;
    const VerifyArgs a{logits,     draft_logits, tokens,       counts,
                       uniforms,   out_tokens,   out_count,    out_logprob,
                       row_stride, token_stride, draft_row_stride, draft_token_stride,
                       rows,       drafts,       vocab,
                       k};
    return hip_status(launch_verify(a, logits_type, workspace, stream), "verification launch");
}

}  // extern "C"
