// C ABI of the verification of drafted tokens: every argument is checked here before
// anything is launched.  No entry point throws.
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

}  // namespace

extern "C" {

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
