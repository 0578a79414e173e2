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
// top / 127 rounded to bf16.  Rounding the quotient to fp32 first changes
// nothing: m / 127 with m of 8 bits is no nearer to a bf16 tie than 2^-16 of it.
__device__ __forceinline__ uint16_t int8_scale(uint32_t top) {
    return top >= 0x7f80 ? kNan16 : bf16_round(bf16_value(top) / 127.f);
}
// x / scale rounded: both have 8 bits, so the quotient is a tie exactly or 2^-12
// away from one, and rounding it to fp32 first changes nothing.
__device__ __forceinline__ int int8_code(uint32_t x, uint16_t scale) {
    const float s = bf16_value(scale);
    if (!(s > 0.f)) return 0;  // an empty row, or NaN
    return (int)fminf(fmaxf(rintf(bf16_value(x) / s), -127.f), 127.f);
}

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
