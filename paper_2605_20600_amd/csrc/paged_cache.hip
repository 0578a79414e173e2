// Writing keys and values into a paged cache, quantised on the way, and reading
// them back (formats and layout: headkv.h, paged.h).
// What a task is: paged_write.h.
// One MI355X: 16 images of up to 2352 tokens, 32 heads of 128, INT8: read back (with
// zeros past their ends) 113 us, 6.0 TB/s, bound by the bytes; written 59 us for 166 MB,
// 2.8 TB/s, the vector ALU busy for 46 % of the time and four of five wavefronts there
// for tokens that a short image does not have (BF16 64 us, FP4 53; images that are all
// whole 191 us for 930 MB, 4.9 TB/s).  One token for 8 x 32 lists: 3.0 and 3.4 us, a
// launch's time.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "paged.h"
#include "paged_device.h"
#include "paged_write.h"

namespace headkv {
namespace {

using namespace dev;

constexpr int kThreads = kWriteThreads;

template <int TYPE, int D>
__global__ __launch_bounds__(kThreads) void k_paged_write(PagedDims c, char* pool, PagedLists ls,
                                                          const uint16_t* __restrict__ k,
                                                          const uint16_t* __restrict__ v,
                                                          PagedRows r, int tokens, int blocks,
                                                          const int32_t* __restrict__ counts) {
    write_eights<TYPE, D, true>(blockIdx.x, c, pool, ls, k, v, r, tokens, blocks, counts);
}

template <int TYPE, int D>
__global__ __launch_bounds__(kThreads) void k_paged_write_few(PagedDims c, char* pool, PagedLists ls,
                                                              const uint16_t* __restrict__ k,
                                                              const uint16_t* __restrict__ v,
                                                              PagedRows r, int tokens,
                                                              const int32_t* __restrict__ counts) {
    write_singles<TYPE, D, true>(blockIdx.x, c, pool, ls, k, v, r, tokens, counts);
}

template <int TYPE, int D>
__global__ __launch_bounds__(kThreads) void k_paged_read(PagedDims c, const char* pool,
                                                         PagedLists ls, int begin, int tokens,
                                                         int blocks, uint16_t* __restrict__ k,
                                                         uint16_t* __restrict__ v, PagedRows r) {
    int blk;
    const Task<D> task(blockIdx.x, ls.lists, c.heads, blocks, &blk);
    if (!task.any) return;
    const int len = list_len(ls, c.ptok, task.lh);
    const int64_t from = begin >= 0 ? begin : (int64_t)len + begin;  // position of output row 0
    const int64_t p0 = ((from >> 3) + blk) * 8;
    if (p0 >= from + tokens) return;
    const char* page = p0 < len ? list_page(c, ls, pool, task.lh, p0) : nullptr;
    const int tp = (int)(p0 & (c.ptok - 1)), lane = task.lane;
    const int64_t row0 = task.l * r.list + task.h * r.head + (p0 - from) * r.token;

    {  // K: 16 dims of one token
        const int t = lane / (D / 16), piece = lane % (D / 16);
        const bool out = p0 + t >= from && p0 + t < from + tokens;
        uint32_t w[8] = {};
        if (page && p0 + t < len) {
            if constexpr (TYPE == kBf16) {
                const uint4* src =
                    reinterpret_cast<const uint4*>(page + (tp + t) * (2 * D) + piece * 32);
                const uint4 a = src[0], b = src[1];
                w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
                w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
            } else if constexpr (TYPE == kInt8) {
                const uint4 a = *reinterpret_cast<const uint4*>(page + (tp + t) * D + piece * 16);
                const uint32_t in[4] = {a.x, a.y, a.z, a.w};
                const float s =
                    bf16_value(reinterpret_cast<const uint16_t*>(page + c.ks_off)[tp + t]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t u = in[i / 2] >> (16 * (i & 1));
                    w[i] = bf16_round((float)(int8_t)u * s) |
                           (uint32_t)bf16_round((float)(int8_t)(u >> 8) * s) << 16;
                }
            } else {
                const uint2 a = *reinterpret_cast<const uint2*>(page + (tp + t) * (D / 2) + piece * 8);
                const uint32_t in[2] = {a.x, a.y};
                const float s =
                    fp4_power((uint8_t)page[c.ks_off + (tp + t) * (D / 32) + piece / 2]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const f32x2_t x =
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[i / 4] >> (8 * (i % 4)), 1.f, 0);
                    w[i] = bf16_round(x[0] * s) | (uint32_t)bf16_round(x[1] * s) << 16;
                }
            }
        }
        if (out) {
            uint4* dst = reinterpret_cast<uint4*>(k + row0 + t * r.token + piece * 16);
            dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
            dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }

    // V: two dims of eight tokens
    uint32_t w[8] = {};
    if (page) {
        const char* cells = page + c.v_off + (tp >> 3) * 8 * (c.v_off / c.ptok);
        if constexpr (TYPE == kBf16) {
            const uint4 a = reinterpret_cast<const uint4*>(cells + lane * 32)[0];
            const uint4 b = reinterpret_cast<const uint4*>(cells + lane * 32)[1];
            const uint32_t lo[4] = {a.x, a.y, a.z, a.w}, hi[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int t = 0; t < 8; t += 2) {
                w[t] = (lo[t / 2] & 0xffffu) | hi[t / 2] << 16;
                w[t + 1] = lo[t / 2] >> 16 | (hi[t / 2] & 0xffff0000u);
            }
        } else if constexpr (TYPE == kInt8) {
            const uint4 a = *reinterpret_cast<const uint4*>(cells + lane * 16);
            const uint32_t lo[2] = {a.x, a.y}, hi[2] = {a.z, a.w};
            const uint4 sc =
                *reinterpret_cast<const uint4*>(page + c.vs_off + 2 * tp);  // tp: a multiple of 8
            const uint32_t ss[4] = {sc.x, sc.y, sc.z, sc.w};
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const float s = bf16_value(ss[t / 2] >> (16 * (t & 1)) & 0xffffu);
                w[t] = bf16_round((float)(int8_t)(lo[t / 4] >> (8 * (t % 4))) * s) |
                       (uint32_t)bf16_round((float)(int8_t)(hi[t / 4] >> (8 * (t % 4))) * s) << 16;
            }
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(cells + lane * 8);
            const uint32_t in[2] = {a.x, a.y};
            const uint2 sc =
                *reinterpret_cast<const uint2*>(page + c.vs_off + lane / 16 * c.ptok + tp);
            const uint32_t ss[2] = {sc.x, sc.y};
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const float s = fp4_power(ss[t / 4] >> (8 * (t % 4)) & 0xffu);
                const f32x2_t x =
                    __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[t / 4] >> (8 * (t % 4)), 1.f, 0);
                w[t] = bf16_round(x[0] * s) | (uint32_t)bf16_round(x[1] * s) << 16;
            }
        }
    }
#pragma unroll
    for (int t = 0; t < 8; ++t)
        if (p0 + t >= from && p0 + t < from + tokens)
            *reinterpret_cast<uint32_t*>(v + row0 + t * r.token + 2 * lane) =
                p0 + t < len ? w[t] : 0u;
}

// Tokens of a list up to which they are written one by one (alone in a graph, one
// by one and as blocks of eight, 8 x 32 lists INT8: 1 token 3.2 and 5.9 us, 4 3.3
// and 5.8, 16 4.0 and 6.2; 64 x 32: 1 3.7 and 6.5, 4 6.0 and 9.5, 16 15.0 and 14.1;
// 256 x 20 of 64 dims FP4: 1 3.5 and 5.1, 4 6.6 and 6.5, 8 9.7 and 6.9).
constexpr int kFew = 4;

// Blocks of eight positions that `tokens` tokens starting anywhere can touch.
int token_blocks(int tokens) { return (int)(((int64_t)tokens + 14) / 8); }

template <int D>
int grid_of(const PagedLists& l, int heads, int blocks, unsigned* grid) {
    const int64_t n = (int64_t)l.lists * heads * blocks;
    const int64_t g = (n + kThreads / (D / 2) - 1) / (kThreads / (D / 2));
    if (g >= 1 << 24) return kTooLarge;  // 2^32 threads: more than a launch has
    *grid = (unsigned)g;
    return 0;
}

template <int TYPE, int D>
int write_launch(const PagedDims& c, char* pool, const PagedLists& l, const uint16_t* k,
                 const uint16_t* v, const PagedRows& r, int tokens, const int32_t* counts,
                 void* stream) {
    unsigned grid;
    if (tokens <= kFew && grid_of<D>(l, c.heads, tokens, &grid) == 0) {
        k_paged_write_few<TYPE, D><<<grid, kThreads, 0, (hipStream_t)stream>>>(c, pool, l, k, v, r,
                                                                               tokens, counts);
        return (int)hipGetLastError();
    }
    const int blocks = token_blocks(tokens);
    if (int e = grid_of<D>(l, c.heads, blocks, &grid)) return e;
    k_paged_write<TYPE, D><<<grid, kThreads, 0, (hipStream_t)stream>>>(c, pool, l, k, v, r, tokens,
                                                                       blocks, counts);
    return (int)hipGetLastError();
}

template <int TYPE, int D>
int read_launch(const PagedDims& c, const char* pool, const PagedLists& l, int begin, int tokens,
                uint16_t* k, uint16_t* v, const PagedRows& r, void* stream) {
    unsigned grid;
    const int blocks = token_blocks(tokens);
    if (int e = grid_of<D>(l, c.heads, blocks, &grid)) return e;
    k_paged_read<TYPE, D><<<grid, kThreads, 0, (hipStream_t)stream>>>(c, pool, l, begin, tokens,
                                                                      blocks, k, v, r);
    return (int)hipGetLastError();
}

}  // namespace

#define PAGED_DISPATCH(fn, ...)                                              \
    (c.d == 128 ? (c.type == kBf16   ? fn<kBf16, 128>(__VA_ARGS__)           \
                   : c.type == kInt8 ? fn<kInt8, 128>(__VA_ARGS__)           \
                                     : fn<kFp4, 128>(__VA_ARGS__))           \
                : (c.type == kBf16   ? fn<kBf16, 64>(__VA_ARGS__)            \
                   : c.type == kInt8 ? fn<kInt8, 64>(__VA_ARGS__)            \
                                     : fn<kFp4, 64>(__VA_ARGS__)))

int launch_paged_write(const PagedDims& c, char* pool, const PagedLists& l, const uint16_t* k,
                       const uint16_t* v, const PagedRows& r, int tokens, const int32_t* counts,
                       void* stream) {
    return PAGED_DISPATCH(write_launch, c, pool, l, k, v, r, tokens, counts, stream);
}

int launch_paged_read(const PagedDims& c, const char* pool, const PagedLists& l, int begin,
                      int tokens, uint16_t* k, uint16_t* v, const PagedRows& r, void* stream) {
    return PAGED_DISPATCH(read_launch, c, pool, l, begin, tokens, k, v, r, stream);
}

}  // namespace headkv
