// C ABI of the paged cache, its attention and the token scores: every argument
// is checked here before anything is launched.  No entry point throws.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "../../include/headkv.h"
#include "abi_error.h"
#include "paged.h"

using namespace headkv;

namespace {

headkv_status bad(const char* msg) { return set_error(HEADKV_ERR_INVALID_ARG, msg); }
headkv_status unsupported(const char* msg) { return set_error(HEADKV_ERR_UNSUPPORTED, msg); }

headkv_status hip_status(int e, const char* what) {
    if (e == 0) return HEADKV_OK;
    if (e == kTooLarge) return unsupported("more tokens of all lists than one call takes");
    return set_error(HEADKV_ERR_HIP, std::string(what) + ": " + hipGetErrorString((hipError_t)e));
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

headkv_status make_dims(const headkv_paged_config* c, PagedDims* out) {
    if (!c) return bad("config is NULL");
    if (c->kv_type < HEADKV_KV_BF16 || c->kv_type > HEADKV_KV_FP4) return bad("unknown kv_type");
    if (c->head_dim != 64 && c->head_dim != 128) return unsupported("head_dim must be 64 or 128");
    if (c->kv_heads < 1 || c->kv_heads > 1024) return unsupported("kv_heads out of [1, 1024]");
    if (c->group < 1 || c->group > HEADKV_MAX_GROUP)
        return unsupported("group out of [1, HEADKV_MAX_GROUP]");
    int shift = 5;
    while (shift < 8 && (1 << shift) != c->page_tokens) ++shift;
    if ((1 << shift) != c->page_tokens) return unsupported("page_tokens must be 32, 64, 128 or 256");
    if (c->num_pages < 1) return bad("num_pages must be >= 1");
    PagedDims d{};
    d.type = c->kv_type;
    d.d = c->head_dim;
    d.heads = c->kv_heads;
    d.group = c->group;
    d.ptok = c->page_tokens;
    d.pshift = shift;
    d.num_pages = c->num_pages;
    const int row = d.type == HEADKV_KV_BF16 ? 2 * d.d : d.type == HEADKV_KV_INT8 ? d.d : d.d / 2;
    const int scale = d.type == HEADKV_KV_BF16 ? 0 : d.type == HEADKV_KV_INT8 ? 2 : d.d / 32;
    d.v_off = d.ptok * row;
    d.ks_off = 2 * d.v_off;
    d.vs_off = d.ks_off + d.ptok * scale;
    d.page_bytes = ((int64_t)d.vs_off + d.ptok * scale + 127) / 128 * 128;
    *out = d;
    return HEADKV_OK;
}

// pointers: whether the device arrays are needed (not for a plan)
headkv_status make_lists(const PagedDims& c, const headkv_paged_lists* l, bool pointers,
                         PagedLists* out) {
    if (!l) return bad("lists is NULL");
    if (l->lists < 1 || l->max_pages < 1) return bad("lists and max_pages must be >= 1");
    if ((int64_t)l->lists * c.heads > (1 << 24)) return unsupported("lists * kv_heads > 2^24");
    if (l->max_pages > (1 << 22)) return unsupported("max_pages > 2^22");
    if (l->extra < 0 || l->max_len < 0) return bad("extra and max_len must be >= 0");
    if (pointers && !l->pages) return bad("pages is NULL");
    if (!aligned(l->pages, 4) || !aligned(l->len, 4) || !aligned(l->first, 4) ||
        !aligned(l->order, 4))
        return bad("pages / len / first / order not aligned");
    *out = PagedLists{l->pages, l->len, l->first, l->order, l->lists, l->max_pages, l->extra,
                      (int)std::min<int64_t>(l->max_len, (int64_t)l->max_pages * c.ptok)};
    return HEADKV_OK;
}

headkv_status check_rows(const void* k, const void* v, int64_t list, int64_t token, int64_t head) {
    if (!k || !v) return bad("k / v is NULL");
    if (!aligned(k, 16) || !aligned(v, 16)) return bad("k / v not 16-byte aligned");
    if (list < 0 || token < 0 || head < 0 || list % 8 || token % 8 || head % 8)
        return bad("strides must be >= 0 and multiples of 8 elements");
    return HEADKV_OK;
}

headkv_status check_workspace(const void* ws, size_t have, size_t need) {
    if (have < need)
        return set_error(HEADKV_ERR_CAPACITY, "workspace of " + std::to_string(have) +
                                                  " bytes, " + std::to_string(need) + " needed");
    if (need && !ws) return bad("workspace is NULL");
    if (!aligned(ws, 256)) return bad("workspace not 256-byte aligned");
    return HEADKV_OK;
}

}  // namespace

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
