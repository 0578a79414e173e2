// Decode attention over a paged cache, with prefixes that several rows share.
// One wavefront per (batch row, query head): a lane scores one token at a time,
// 64 tokens share a running maximum, then every lane sums its own dims.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "paged.h"
#include "paged_device.h"

namespace headkv {
namespace {

using namespace dev;

// Value of dim i of token tp of a page: K rows (V false) or V cells.
template <int TYPE, int D, bool V>
__device__ __forceinline__ float element(const PagedDims& c, const char* page, int tp, int i) {
    const char* base = V ? page + c.v_off : page;
    if constexpr (TYPE == kBf16) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(base);
        return bf16_value(V ? p[((tp >> 3) * D + i) * 8 + (tp & 7)] : p[tp * D + i]);
    } else if constexpr (TYPE == kInt8) {
        const int8_t* p = reinterpret_cast<const int8_t*>(base);
        const float s = bf16_value(
            reinterpret_cast<const uint16_t*>(page + (V ? c.vs_off : c.ks_off))[tp]);
        return (float)(V ? p[((tp >> 3) * D + i) * 8 + (tp & 7)] : p[tp * D + i]) * s;
    } else {
        const uint8_t* p = reinterpret_cast<const uint8_t*>(base);
        const uint32_t b =
            V ? p[((tp >> 3) * (D / 2) + i / 2) * 8 + (tp & 7)] : p[tp * (D / 2) + i / 2];
        const uint32_t e = (uint8_t)(V ? page[c.vs_off + i / 32 * c.ptok + tp]
                                       : page[c.ks_off + tp * (D / 32) + i / 32]);
        const f32x2_t x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(b, 1.f, 0);
        return x[i & 1] * fp4_power(e);
    }
}

template <int TYPE, int D>
__global__ __launch_bounds__(64) void k_paged_attn(PagedDims c, const char* pool, PagedLists own,
                                                   PagedLists shared, const int32_t* share,
                                                   const uint16_t* q, int64_t q_stride, float* out,
                                                   float* lse) {
    const int hq = blockIdx.x % (c.heads * c.group), b = blockIdx.x / (c.heads * c.group);
    const int h = hq / c.group, lane = threadIdx.x;
    __shared__ float qs[D];
    const float scale = (float)(1.0 / __builtin_sqrt((double)D));
    for (int i = lane; i < D; i += 64) qs[i] = bf16_value(q[b * q_stride + hq * D + i]) * scale;
    __syncthreads();
    float m = -INFINITY, sum = 0.f, acc[D / 64] = {};
    auto visit = [&](const PagedLists& p, int64_t lh) {
        const int len = list_len(p, c.ptok, lh);
        const int first = p.first ? max(p.first[lh], 0) : 0;
        for (int t0 = first & ~31; t0 < len; t0 += 32) {  // 32 tokens lie in one page
            const char* page = list_page(c, p, pool, lh, t0);
            if (!page) continue;
            const int tp = t0 & (c.ptok - 1), t = t0 + lane;
            float s = -INFINITY;
            if (lane < 32 && t >= first && t < len) {
                s = 0.f;
                for (int i = 0; i < D; ++i)
                    s = fmaf(qs[i], element<TYPE, D, false>(c, page, tp + lane, i), s);
            }
            float mx = s;
            for (int o = 1; o < 64; o *= 2) mx = fmaxf(mx, __shfl_xor(mx, o));
            mx = fmaxf(mx, m);
            if (mx == -INFINITY) mx = 0.f;  // nothing seen yet: exp of -inf stays 0
            const float f = expf(m - mx), w = expf(s - mx);
            m = mx;
            sum = sum * f + w;
            for (float& a : acc) a *= f;
            for (int j = 0; j < 32; ++j) {
                if (t0 + j < first || t0 + j >= len) continue;
                const float wj = __shfl(w, j);
                for (int e = 0; e < D / 64; ++e)
                    acc[e] = fmaf(wj, element<TYPE, D, true>(c, page, tp + j, lane + 64 * e), acc[e]);
            }
        }
    };
    visit(own, (int64_t)b * c.heads + h);
    if (share) {
        const int l = share[b];
        if (l >= 0 && l < shared.lists) visit(shared, (int64_t)l * c.heads + h);
    }
    for (int o = 1; o < 64; o *= 2) sum += __shfl_xor(sum, o);
    const int64_t row = (int64_t)b * c.heads * c.group + hq;
    for (int e = 0; e < D / 64; ++e)
        out[row * D + lane + 64 * e] = sum == 0.f ? 0.f : acc[e] / sum;
    if (lse && lane == 0) lse[row] = sum == 0.f ? -INFINITY : m + logf(sum);
}

template <int TYPE, int D>
int attn_launch(const PagedDims& c, const char* pool, const PagedLists& own,
                const PagedLists* shared, const int32_t* share, const uint16_t* q,
                int64_t q_stride, float* out, float* lse, void* stream) {
    const unsigned grid = (unsigned)own.lists * c.heads * c.group;
    k_paged_attn<TYPE, D><<<grid, 64, 0, (hipStream_t)stream>>>(
        c, pool, own, shared ? *shared : PagedLists{}, share, q, q_stride, out, lse);
    return (int)hipGetLastError();
}

}  // namespace

size_t paged_attn_workspace(const PagedDims&, const PagedLists&, const PagedLists*) { return 0; }

int launch_paged_attn(const PagedDims& c, const char* pool, const PagedLists& own,
                      const PagedLists* shared, const int32_t* share, const uint16_t* q,
                      int64_t q_stride, float* out, float* lse, void*, void* stream) {
    auto run = [&](auto fn) {
        return fn(c, pool, own, shared, share, q, q_stride, out, lse, stream);
    };
    if (c.d == 128)
        return c.type == kBf16   ? run(attn_launch<kBf16, 128>)
               : c.type == kInt8 ? run(attn_launch<kInt8, 128>)
                                 : run(attn_launch<kFp4, 128>);
    return c.type == kBf16   ? run(attn_launch<kBf16, 64>)
           : c.type == kInt8 ? run(attn_launch<kInt8, 64>)
                             : run(attn_launch<kFp4, 64>);
}

}  // namespace headkv
