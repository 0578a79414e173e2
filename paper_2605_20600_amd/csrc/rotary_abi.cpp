// C ABI of the norms with rotary positions: every argument is checked here before
// anything is launched.  No entry point throws.
#include <cmath>
#include <cstdint>

#include "../../include/headkv.h"
#include "paged.h"
#include "paged_check.h"

using namespace headkv;

namespace {

headkv_status check_config(const headkv_rotary_config* c) {
    if (!c) return bad("config is NULL");
    if (c->head_dim != 64 && c->head_dim != 128) return unsupported("head_dim must be 64 or 128");
    if (c->rotary_dims < 0 || c->rotary_dims > c->head_dim || c->rotary_dims % 16)
        return unsupported("rotary_dims must be a multiple of 16 in [0, head_dim]");
    if (c->layout != HEADKV_ROPE_HALF && c->layout != HEADKV_ROPE_PAIRS) return bad("unknown layout");
    if (c->axes != 1 && c->axes != 2) return unsupported("axes must be 1 or 2");
    if (c->norm < HEADKV_NORM_NONE || c->norm > HEADKV_NORM_LAYER) return bad("unknown norm");
    if (!(c->eps >= 0.f) || !std::isfinite(c->eps)) return bad("eps must be >= 0 and finite");
    if (!std::isfinite(c->scale)) return bad("scale must be finite");
    return HEADKV_OK;
}

// keys: whether rows come back, or go to a cache
headkv_status make_rows(const headkv_rotary_config& c, const headkv_rotary_rows* r, bool comes_back,
                        RotaryRows* out) {
    *out = RotaryRows{};
    if (!r) return HEADKV_OK;
    if (r->heads < 0 || r->heads > 65536) return unsupported("heads out of [0, 65536]");
    if (r->heads == 0) return HEADKV_OK;
    if (!r->in || (comes_back && !r->out)) return bad("in / out is NULL");
    if (!aligned(r->in, 16) || (comes_back && !aligned(r->out, 16)))
        return bad("in / out not 16-byte aligned");
    const int64_t strides[6] = {r->in_row,  r->in_token,  r->in_head,
                                r->out_row, r->out_token, r->out_head};
    for (int i = 0; i < (comes_back ? 6 : 3); ++i)
        if (strides[i] < 0 || strides[i] % 8)
            return bad("strides must be >= 0 and multiples of 8 elements");
    if (!aligned(r->weight, 16) || !aligned(r->bias, 16))
        return bad("weight / bias not 16-byte aligned");
    if (r->per_head != 0 && r->per_head != 1) return bad("per_head must be 0 or 1");
    out->in = r->in;
    out->out = r->out;
    out->from = PagedRows{r->in_row, r->in_token, r->in_head};
    out->to = PagedRows{r->out_row, r->out_token, r->out_head};
    out->weight = r->weight;
    out->bias = r->bias;
    out->heads = r->heads;
    out->step = r->per_head ? c.head_dim : 0;
    return HEADKV_OK;
}

// Rows that several threads would write in no order.
headkv_status check_out(const RotaryRows& r, int d, int rows, int tokens) {
    if ((r.heads > 1 && r.to.head < d) || (r.heads && tokens > 1 && r.to.token < d) ||
        (r.heads && rows > 1 && r.to.list < d))
        return bad("output rows overlap: a stride is smaller than head_dim");
    return HEADKV_OK;
}

headkv_status make_args(const headkv_rotary_config* c, const double* turns,
                        const int32_t* positions, int rows, int tokens, const int32_t* counts,
                        RotaryArgs* a) {
    if (c->rotary_dims && (!turns || !positions)) return bad("turns / positions is NULL");
    if (!aligned(turns, 8) || !aligned(positions, 4) || !aligned(counts, 4))
        return bad("turns / positions / counts not aligned");
    a->turns = turns;
    a->positions = positions;
    a->counts = counts;
    a->d = c->head_dim;
    a->rows = rows;
    a->tokens = tokens;
    a->r = c->rotary_dims;
    a->axes = c->axes;
    a->layout = c->layout;
    a->norm = c->norm;
    a->eps = c->eps;
    a->scale = c->scale;
    return HEADKV_OK;
}

}  // namespace

extern "C" {

headkv_status headkv_rotary_plan(const headkv_rotary_config* cfg, double* turns) {
    if (headkv_status st = check_config(cfg)) return st;
    const int n = cfg->rotary_dims / cfg->axes;
    if (cfg->scaling < HEADKV_SCALE_NONE || cfg->scaling > HEADKV_SCALE_BANDS)
        return bad("unknown scaling");
    if (!(cfg->base > 0) || !std::isfinite(cfg->base)) return bad("base must be > 0 and finite");
    if (cfg->scaling != HEADKV_SCALE_NONE && (!(cfg->factor > 0) || !std::isfinite(cfg->factor)))
        return bad("factor must be > 0 and finite");
    if (cfg->scaling == HEADKV_SCALE_BANDS &&
        (cfg->original_len < 1 || !(cfg->low >= 0) || !(cfg->high > cfg->low) ||
         !std::isfinite(cfg->high)))
        return bad("original_len must be >= 1 and 0 <= low < high, finite");
    if (!turns && n) return bad("turns is NULL");
    double base = cfg->base;
    if (cfg->scaling == HEADKV_SCALE_BASE && n > 2) base *= std::pow(cfg->factor, n / (n - 2.0));
    if (!std::isfinite(base) || !(base > 0)) return bad("base is not finite once scaled");
    for (int j = 0; j < cfg->rotary_dims / 2; ++j) {
        double omega = std::pow(base, -2.0 * (j % (n / 2)) / n);
        const double slow = omega / cfg->factor;
        if (cfg->scaling == HEADKV_SCALE_LINEAR) {
            omega = slow;
        } else if (cfg->scaling == HEADKV_SCALE_BANDS) {
            const double m = cfg->original_len * omega / (2 * M_PI);
            const double on = (m - cfg->low) / (cfg->high - cfg->low);
            omega = on >= 1 ? omega : on <= 0 ? slow : slow + on * (omega - slow);
        }
        turns[j] = omega / (2 * M_PI);
    }
    return HEADKV_OK;
}

headkv_status headkv_rotary(const headkv_rotary_config* cfg, const double* turns,
                            const int32_t* positions, int32_t rows, int32_t tokens,
                            const int32_t* counts, const headkv_rotary_rows* q,
                            const headkv_rotary_rows* k, void* stream) {
    if (headkv_status st = check_config(cfg)) return st;
    if (rows < 0 || tokens < 0) return bad("rows and tokens must be >= 0");
    if (rows == 0 || tokens == 0) return HEADKV_OK;  // rows of no tokens may have no address
    RotaryArgs a{};
    if (headkv_status st = make_rows(*cfg, q, true, &a.q)) return st;
    if (headkv_status st = make_rows(*cfg, k, true, &a.k)) return st;
    if (a.q.heads + a.k.heads == 0) return HEADKV_OK;
    if (headkv_status st = check_out(a.q, cfg->head_dim, rows, tokens)) return st;
    if (headkv_status st = check_out(a.k, cfg->head_dim, rows, tokens)) return st;
    if (headkv_status st = make_args(cfg, turns, positions, rows, tokens, counts, &a)) return st;
    return hip_status(launch_rotary(a, nullptr, stream), "rotary launch");
}

headkv_status headkv_paged_write_rotary(const headkv_paged_config* cfg, void* pool,
                                        const headkv_paged_lists* lists,
                                        const headkv_rotary_config* rotary, const double* turns,
                                        const int32_t* positions, int32_t tokens,
                                        const int32_t* counts, const headkv_rotary_rows* q,
                                        const headkv_rotary_rows* k, const uint16_t* v,
                                        int64_t v_list_stride, int64_t v_token_stride,
                                        int64_t v_head_stride, void* stream) {
    RotaryCache to{};
    if (headkv_status st = make_dims(cfg, &to.c)) return st;
    if (headkv_status st = make_lists(to.c, lists, true, &to.lists)) return st;
    if (headkv_status st = check_config(rotary)) return st;
    if (rotary->head_dim != to.c.d) return bad("head_dim of the rotation is not the cache's");
    if (tokens < 0) return bad("tokens must be >= 0");
    if (tokens == 0) return HEADKV_OK;
    RotaryArgs a{};
    if (headkv_status st = make_rows(*rotary, q, true, &a.q)) return st;
    if (headkv_status st = make_rows(*rotary, k, false, &a.k)) return st;
    if (a.k.heads != to.c.heads) return bad("keys of kv_heads heads are needed");
    if (headkv_status st = check_out(a.q, to.c.d, to.lists.lists, tokens)) return st;
    if (headkv_status st = check_rows(k->in, v, v_list_stride, v_token_stride, v_head_stride))
        return st;
    if (!pool || !aligned(pool, 256)) return bad("pool is NULL or not 256-byte aligned");
    if (headkv_status st = make_args(rotary, turns, positions, to.lists.lists, tokens, counts, &a))
        return st;
    to.pool = static_cast<char*>(pool);
    to.v = v;
    to.v_rows = PagedRows{v_list_stride, v_token_stride, v_head_stride};
    return hip_status(launch_rotary(a, &to, stream), "rotary write launch");
}

}  // extern "C"
