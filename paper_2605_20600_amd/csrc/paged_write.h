// Appending keys and values to a paged cache: what a block of the writing kernels does
// (paged_cache.hip; with KEYS = false, for values alone, rotary.hip).
//
// A task is the up to eight tokens of one aligned block of eight (one row of V
// cells) of one list and head, taken by d / 2 lanes.  For K a lane holds 16 dims
// of one token and stores them contiguously; for V it holds two dims of the
// eight tokens, which are its two cells (FP4: its cell), so that a full block's
// cells leave as whole 16-byte pieces without any exchange between lanes.  The
// largest value of a row (FP4: of 32 dims) is found with lane exchanges, for V
// on two tokens' bits at a time.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "paged.h"
#include "paged_device.h"

namespace headkv {
namespace dev {

typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

constexpr int kWriteThreads = 256;

__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t,
                              __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a),
                                                        __builtin_bit_cast(u16x2_t, b)));
}

// Maximum of each half over groups of LANES adjacent lanes.
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
    if (LANES > 1) v = pk_max(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false));
    if (LANES > 2) v = pk_max(v, __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, false));
    if (LANES > 4) v = pk_max(v, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, false));
    if (LANES > 8) v = pk_max(v, __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, false));
    if (LANES > 16) v = pk_max(v, (uint32_t)__shfl_xor((int)v, 16));
    if (LANES > 32) v = pk_max(v, (uint32_t)__shfl_xor((int)v, 32));
    return v;
}

// The eight-token block of a task: its list and head, first position and page.
template <int D>
struct Task {
    static constexpr int LANES = D / 2;
    int lane;        // of the task
    int l, h;
    int64_t lh;
    bool any;        // a task at all
    __device__ Task(int block, int lists, int heads, int blocks, int* blk) {
        // (32 bits: a grid has fewer than 2^24 blocks)
        uint32_t i = (uint32_t)block * (kWriteThreads / LANES) + threadIdx.x / LANES;
        if constexpr (LANES == 64) i = __builtin_amdgcn_readfirstlane(i);
        lane = threadIdx.x % LANES;
        const uint32_t token = i / (uint32_t)heads;
        h = (int)(i - token * heads);  // heads of a token are neighbours in memory
        l = (int)(token / (uint32_t)blocks);
        *blk = (int)(token - (uint32_t)l * blocks);
        any = l < lists;
        lh = (int64_t)l * heads + h;
    }
};

template <int TYPE, int D, bool KEYS>
__device__ __forceinline__ void write_eights(int block, const PagedDims& c, char* pool, const PagedLists& ls,
                                            const uint16_t* __restrict__ k,
                                            const uint16_t* __restrict__ v, const PagedRows& r,
                                            int tokens, int blocks, const int32_t* __restrict__ counts) {
    int blk;
    const Task<D> task(block, ls.lists, c.heads, blocks, &blk);
    if (!task.any) return;
    const int64_t base = (int64_t)(ls.len ? max(ls.len[task.lh], 0) : 0) + ls.extra;
    const int64_t end = base + (counts ? min(max(counts[task.l], 0), tokens) : tokens);
    const int64_t p0 = ((base >> 3) + blk) * 8;
    if (p0 >= end) return;
    // every load is on its way before the first is waited for
    char* page = const_cast<char*>(list_page(c, ls, pool, task.lh, p0));
    const int tp = (int)(p0 & (c.ptok - 1)), lane = task.lane;
    const int64_t row0 = task.l * r.list + task.h * r.head + (p0 - base) * r.token;
    const int key_t = lane / (D / 16), piece = lane % (D / 16);
    const bool key_there = p0 + key_t >= base && p0 + key_t < end;
    uint32_t key[8] = {};
    if (KEYS && key_there) {
        const uint4* src = reinterpret_cast<const uint4*>(k + row0 + key_t * r.token + piece * 16);
        const uint4 a = src[0], b = src[1];
        key[0] = a.x, key[1] = a.y, key[2] = a.z, key[3] = a.w;
        key[4] = b.x, key[5] = b.y, key[6] = b.z, key[7] = b.w;
    }
    uint32_t w[8];
    bool there[8], full = true;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        there[t] = p0 + t >= base && p0 + t < end;
        full = full && there[t];
    }
    if (full) {  // (no branch for each)
#pragma unroll
        for (int t = 0; t < 8; ++t)
            w[t] = *reinterpret_cast<const uint32_t*>(v + row0 + t * r.token + 2 * lane);
    } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
            w[t] = there[t] ? *reinterpret_cast<const uint32_t*>(v + row0 + t * r.token + 2 * lane) : 0u;
    }
    if (!page) return;

    if constexpr (KEYS) {  // 16 dims of one token
        const int t = key_t;
        const bool there = key_there;
        const uint32_t* w = key;
        if constexpr (TYPE == kBf16) {
            if (there) {
                uint4* dst = reinterpret_cast<uint4*>(page + (tp + t) * (2 * D) + piece * 32);
                dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
                dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
        } else {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = pk_max(m, w[i] & 0x7fff7fffu);
            m = lanes_max<TYPE == kInt8 ? D / 16 : 2>(m);
            const uint32_t top = max(m & 0xffffu, m >> 16);
            if constexpr (TYPE == kInt8) {
                const uint16_t s = int8_scale(top);
                const Int8Row row(s);
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = row.codes(w[2 * i], w[2 * i + 1]);
                if (there) {
                    *reinterpret_cast<uint4*>(page + (tp + t) * D + piece * 16) =
                        make_uint4(o[0], o[1], o[2], o[3]);
                    if (piece == 0) reinterpret_cast<uint16_t*>(page + c.ks_off)[tp + t] = s;
                }
            } else {
                const uint32_t e = fp4_scale(top);
                const float s = fp4_power(e);
                uint32_t o[2] = {};
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t* p = w + 4 * i;
                    auto lo = [](uint32_t u) { return __uint_as_float(u << 16); };
                    auto hi = [](uint32_t u) { return __uint_as_float(u & 0xffff0000u); };
                    o[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o[i], lo(p[0]), hi(p[0]), s, 0);
                    o[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o[i], lo(p[1]), hi(p[1]), s, 1);
                    o[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o[i], lo(p[2]), hi(p[2]), s, 2);
                    o[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o[i], lo(p[3]), hi(p[3]), s, 3);
                }
                if (there) {
                    *reinterpret_cast<uint2*>(page + (tp + t) * (D / 2) + piece * 8) =
                        make_uint2(o[0], o[1]);
                    if (piece % 2 == 0)
                        page[c.ks_off + (tp + t) * (D / 32) + piece / 2] = (char)e;
                }
            }
        }
    }

    // V: two dims of eight tokens
    char* cells = page + c.v_off + (tp >> 3) * 8 * (c.v_off / c.ptok);
    if constexpr (TYPE == kBf16) {
        char* dst = cells + lane * 32;
        if (full) {
            uint32_t o[8];
#pragma unroll
            for (int t = 0; t < 8; t += 2) {
                o[t / 2] = (w[t] & 0xffffu) | w[t + 1] << 16;
                o[4 + t / 2] = w[t] >> 16 | (w[t + 1] & 0xffff0000u);
            }
            reinterpret_cast<uint4*>(dst)[0] = make_uint4(o[0], o[1], o[2], o[3]);
            reinterpret_cast<uint4*>(dst)[1] = make_uint4(o[4], o[5], o[6], o[7]);
        } else {
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (there[t]) {
                    reinterpret_cast<uint16_t*>(dst)[t] = (uint16_t)w[t];
                    reinterpret_cast<uint16_t*>(dst)[8 + t] = (uint16_t)(w[t] >> 16);
                }
        }
        return;
    }
    uint32_t m[4];  // largest bits of tokens t (low half) and t + 4
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint32_t a = w[t] & 0x7fff7fffu, b = w[t + 4] & 0x7fff7fffu;
        m[t] = pk_max((a & 0xffffu) | b << 16, a >> 16 | (b & 0xffff0000u));
        m[t] = lanes_max<TYPE == kInt8 ? D / 2 : 16>(m[t]);
    }
    if constexpr (TYPE == kInt8) {
        // lane t works out token t's scale and its inverse for all lanes
        uint32_t top = 0;
#pragma unroll
        for (int t = 0; t < 8; ++t)
            if ((lane & 7) == t) top = t < 4 ? m[t] & 0xffffu : m[t - 4] >> 16;
        const uint16_t mine = int8_scale(top);
        const Int8Row own(mine);
        uint32_t o[4] = {};
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const Int8Row row(__shfl(own.scale, t, 8), __shfl(own.inverse, t, 8));
            // both dims of the token, into byte t % 4 of a word each
            const uint32_t codes = row.codes(w[t], 0);
            o[t / 4] |= (codes & 0xffu) << (8 * (t % 4));
            o[2 + t / 4] |= (codes >> 8 & 0xffu) << (8 * (t % 4));
        }
        char* dst = cells + lane * 16;
        if (full) {
            *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
        } else {
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (there[t]) {
                    dst[t] = (char)(o[t / 4] >> (8 * (t % 4)));
                    dst[8 + t] = (char)(o[2 + t / 4] >> (8 * (t % 4)));
                }
        }
        if (lane < 8 && p0 + lane >= base && p0 + lane < end)
            reinterpret_cast<uint16_t*>(page + c.vs_off)[tp + lane] = mine;
    } else {
        uint32_t o[2] = {};
        uint32_t mine = 0;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const uint32_t e = fp4_scale(t < 4 ? m[t] & 0xffffu : m[t - 4] >> 16);
            if (lane % 16 == t) mine = e;
            const uint32_t b =
                __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, __uint_as_float(w[t] << 16),
                                                         __uint_as_float(w[t] & 0xffff0000u),
                                                         fp4_power(e), 0) & 0xffu;
            o[t / 4] |= b << (8 * (t % 4));
        }
        char* dst = cells + lane * 8;
        if (full) {
            *reinterpret_cast<uint2*>(dst) = make_uint2(o[0], o[1]);
        } else {
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (there[t]) dst[t] = (char)(o[t / 4] >> (8 * (t % 4)));
        }
        const int t = lane % 16;
        if (t < 8 && p0 + t >= base && p0 + t < end)
            page[c.vs_off + lane / 16 * c.ptok + tp + t] = (char)mine;
    }
}

// A token or a few for every list: d / 2 lanes take one token of one head, two dims
// of its key and value each, whose loads do not wait for the list's length and page.
template <int TYPE, int D, bool KEYS>
__device__ __forceinline__ void write_singles(int block, const PagedDims& c, char* pool, const PagedLists& ls,
                                            const uint16_t* __restrict__ k,
                                            const uint16_t* __restrict__ v, const PagedRows& r,
                                            int tokens, const int32_t* __restrict__ counts) {
    int i;  // the token
    const Task<D> task(block, ls.lists, c.heads, tokens, &i);
    if (!task.any) return;
    if (counts && i >= counts[task.l]) return;
    const int lane = task.lane;
    const int64_t row = task.l * r.list + task.h * r.head + i * r.token + 2 * lane;
    const uint32_t wk = KEYS ? *reinterpret_cast<const uint32_t*>(k + row) : 0u;
    const uint32_t wv = *reinterpret_cast<const uint32_t*>(v + row);
    const int64_t at = (int64_t)(ls.len ? max(ls.len[task.lh], 0) : 0) + ls.extra + i;
    char* page = const_cast<char*>(list_page(c, ls, pool, task.lh, at));
    const int tp = (int)(at & (c.ptok - 1));
    // the largest bits of the key (low half) and the value
    const uint32_t a = wk & 0x7fff7fffu, b = wv & 0x7fff7fffu;
    uint32_t m = pk_max((a & 0xffffu) | b << 16, a >> 16 | (b & 0xffff0000u));
    if (TYPE != kBf16) m = lanes_max<TYPE == kInt8 ? D / 2 : 16>(m);
    if (!page) return;
    char* cells = page + c.v_off + (tp >> 3) * 8 * (c.v_off / c.ptok);
    const int t = tp & 7;
    if constexpr (TYPE == kBf16) {
        if (KEYS) reinterpret_cast<uint32_t*>(page + tp * (2 * D))[lane] = wk;
        uint16_t* to = reinterpret_cast<uint16_t*>(cells) + lane * 16 + t;
        to[0] = (uint16_t)wv;
        to[8] = (uint16_t)(wv >> 16);
    } else if constexpr (TYPE == kInt8) {
        const uint16_t sk = int8_scale(m & 0xffffu), sv = int8_scale(m >> 16);
        const Int8Row key(sk), value(sv);
        const uint32_t codes = (key.codes(wk, 0) & 0xffffu) | value.codes(wv, 0) << 16;
        if (KEYS) reinterpret_cast<uint16_t*>(page + tp * D)[lane] = (uint16_t)codes;
        char* to = cells + lane * 16 + t;
        to[0] = (char)(codes >> 16);
        to[8] = (char)(codes >> 24);
        if (KEYS && lane == 0) reinterpret_cast<uint16_t*>(page + c.ks_off)[tp] = sk;
        if (lane == 1) reinterpret_cast<uint16_t*>(page + c.vs_off)[tp] = sv;
    } else {
        const uint32_t ek = fp4_scale(m & 0xffffu), ev = fp4_scale(m >> 16);
        auto code = [](uint32_t w, uint32_t e) {
            return (char)__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(
                0, __uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u), fp4_power(e), 0);
        };
        if (KEYS) page[tp * (D / 2) + lane] = code(wk, ek);
        cells[lane * 8 + t] = code(wv, ev);
        if (KEYS && lane % 16 == 0) page[c.ks_off + tp * (D / 32) + lane / 16] = (char)ek;
        if (lane % 16 == 1) page[c.vs_off + lane / 16 * c.ptok + tp] = (char)ev;
    }
}

}  // namespace dev
}  // namespace headkv
