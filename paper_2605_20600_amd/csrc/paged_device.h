// Device side of the paged cache's layout and number formats (paged.h).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "paged.h"

namespace headkv {
namespace dev {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

constexpr int kBf16 = HEADKV_KV_BF16, kInt8 = HEADKV_KV_INT8, kFp4 = HEADKV_KV_FP4;
constexpr uint16_t kNan16 = 0x7fc0;

// Length of list l, head h as the calls see it: [0, max_len], and what the
// page table can hold.
__device__ __forceinline__ int list_len(const PagedLists& p, int ptok, int64_t lh) {
    if (!p.len) return min(p.extra, p.max_len);
    const int64_t n = (int64_t)max(p.len[lh], 0) + p.extra;
    return (int)min(min(n, (int64_t)p.max_len), (int64_t)p.max_pages * ptok);
}

// The page that holds token t of list l, head h, or NULL: dropped, or past the
// table.
__device__ __forceinline__ const char* list_page(const PagedDims& c, const PagedLists& p,
                                                 const char* pool, int64_t lh, int64_t t) {
    const int64_t i = t >> c.pshift;
    if (t < 0 || i >= p.max_pages) return nullptr;
    const int page = p.pages[lh * p.max_pages + i];
    if (page < 0 || page >= c.num_pages) return nullptr;
    return pool + page * c.page_bytes;
}

__device__ __forceinline__ float bf16_value(uint32_t b) { return __uint_as_float(b << 16); }
__device__ __forceinline__ uint16_t bf16_round(float x) {
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// Scale of a row of INT8 whose largest absolute value has the bf16 bits `top`:
// top / 127 rounded to bf16.  A product that is off by 2^-22 of it does as well: m / 127
// with m of 8 bits is no nearer to a bf16 tie than 2^-16 of it, but for half the least
// subnormal number, which comes out as it is.
__device__ __forceinline__ uint16_t int8_scale(uint32_t top) {
    return top >= 0x7f80 ? kNan16 : bf16_round(bf16_value(top) * (1.f / 127.f));
}
// Codes x / scale of a row, rounded.  x and scale have 8 bits each, so a quotient is
// a tie n + 1/2 exactly or 2^-10 and more away from one.  From the inverse scale
// it comes within 2^-22 of itself, less than 2^-15; rounded to 2^-13 first, which
// brings ties back to where they are, it then rounds as the quotient itself does.
// (A division costs 20 instructions: writing whole images of INT8 was bound by them.)
struct Int8Row {
    float scale, inverse;
    __device__ __forceinline__ explicit Int8Row(uint16_t s) : scale(bf16_value(s)), inverse(1.f / scale) {}
    __device__ __forceinline__ Int8Row(float s, float i) : scale(s), inverse(i) {}
    // where the inverse may not be a normal number: no scale to speak of, 0 or NaN
    __device__ __forceinline__ bool small() const { return !(scale >= 0x1p-100f); }
    __device__ __forceinline__ float slow(float x) const {
        return scale > 0.f ? fminf(fmaxf(rintf(x / scale), -127.f), 127.f) + 128.f : 128.f;
    }
    // the codes of the bf16 in the halves of a and b, first to last
    __device__ __forceinline__ uint32_t codes(uint32_t a, uint32_t b) const {
        constexpr float kRound = 1536.f;  // 2^-13 is the last bit of what lies about it
        const float x[4] = {bf16_value(a & 0xffffu), bf16_value(a >> 16), bf16_value(b & 0xffffu),
                            bf16_value(b >> 16)};
        float n[4];  // and 128
#pragma unroll
        for (int i = 0; i < 4; ++i)
            n[i] = __builtin_rintf(fmaf(x[i], inverse, kRound) - (kRound - 128.f));
        if (__builtin_expect(small(), 0)) {
            asm volatile("");  // a branch: the divisions are what is saved
#pragma unroll
            for (int i = 0; i < 4; ++i) n[i] = slow(x[i]);
        }
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_pk_u8_f32(n[0], 0, w);
        w = __builtin_amdgcn_cvt_pk_u8_f32(n[1], 1, w);
        w = __builtin_amdgcn_cvt_pk_u8_f32(n[2], 2, w);
        w = __builtin_amdgcn_cvt_pk_u8_f32(n[3], 3, w);
        return w ^ 0x80808080u;
    }
};

// Exponent byte of 32 FP4 values whose largest absolute value has the bf16 bits
// `top` = m 2^a: the smallest power with top <= 6 s is 2^(a - 2) up to m = 1.5
// (64 / 128 of mantissa), else 2^(a - 1).
__device__ __forceinline__ uint32_t fp4_scale(uint32_t top) {
    return top >= 0x7f80 ? 255u : (uint32_t)max((int)((top + 63) >> 7) - 2, 1);
}
__device__ __forceinline__ float fp4_power(uint32_t e) {
    return __uint_as_float(e == 255 ? 0x7fc00000u : e << 23);
}

}  // namespace dev
}  // namespace headkv
