// Checks of arguments that the entry points of the paged calls share.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "abi_error.h"
#include "paged.h"

namespace headkv {

inline headkv_status bad(const char* msg) { return set_error(HEADKV_ERR_INVALID_ARG, msg); }
inline headkv_status unsupported(const char* msg) { return set_error(HEADKV_ERR_UNSUPPORTED, msg); }

inline headkv_status hip_status(int e, const char* what) {
    if (e == 0) return HEADKV_OK;
    if (e == kTooLarge) return unsupported("more tokens of all lists than one call takes");
    return set_error(HEADKV_ERR_HIP, std::string(what) + ": " + hipGetErrorString((hipError_t)e));
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline headkv_status make_dims(const headkv_paged_config* c, PagedDims* out) {
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
inline headkv_status make_lists(const PagedDims& c, const headkv_paged_lists* l, bool pointers,
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

inline headkv_status check_rows(const void* k, const void* v, int64_t list, int64_t token, int64_t head) {
    if (!k || !v) return bad("k / v is NULL");
    if (!aligned(k, 16) || !aligned(v, 16)) return bad("k / v not 16-byte aligned");
    if (list < 0 || token < 0 || head < 0 || list % 8 || token % 8 || head % 8)
        return bad("strides must be >= 0 and multiples of 8 elements");
    return HEADKV_OK;
}

inline headkv_status check_workspace(const void* ws, size_t have, size_t need) {
    if (have < need)
        return set_error(HEADKV_ERR_CAPACITY, "workspace of " + std::to_string(have) +
                                                  " bytes, " + std::to_string(need) + " needed");
    if (need && !ws) return bad("workspace is NULL");
    if (!aligned(ws, 256)) return bad("workspace not 256-byte aligned");
    return HEADKV_OK;
}

}  // namespace headkv
