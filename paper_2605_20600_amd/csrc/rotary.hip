// Norms of queries and keys with rotary positions (formulas: headkv.h), rows to rows or
// straight into a paged cache, values with them.
//
// A row of d values is held by d / 16 lanes, 16 values each: for a pair's two values to
// lie in one lane, eight values 8 u .. of the turned part's first half and the eight r / 2
// further on (HALF), or 16 consecutive ones (PAIRS, and what does not turn).  Either way
// lane u has the pairs 8 u .. 8 u + 7, whatever the head, so a wavefront takes 8 (d = 64:
// 16) heads of one token at a time, works the token's angles out once and goes on to its
// other heads.  Queries and keys are one sequence of heads; a token's heads are shared by
// as many wavefronts as it takes to fill the card.
// Angles: turns = position * (omega / 2 pi) in 64 bits, of which the nearest quarter is taken
// off before what is left is rounded to 32.  The rest is fp32, the one rounding to bf16 at the
// end; a cache quantises the bf16 values, as it would those of a call of its own, so that both
// ways give the same bits.
// One MI355X: 32768 tokens of 40 heads of 128, half of a head turned, RMS norms: 160 us, 4.2
// TB/s, of the 5.2 that a copy reaches, the vector ALU's norm and conversions beside it; 16
// prompts of up to 2352 tokens, 32 heads of 128, queries back, keys and values into INT8: 88
// us; five tokens of 256 rows, 20 heads of 64 into FP4: 11 us; one token of 8 rows 5.5 us, the
// loads that wait for each other.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "paged.h"
#include "paged_device.h"
#include "paged_write.h"

namespace headkv {
namespace {

using namespace dev;

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kNoCache = -1;
constexpr int kThreads = kWriteThreads, kWaves = kThreads / 64;

// Sum over groups of N = 4 or 8 adjacent lanes.
template <int N>
__device__ __forceinline__ float lanes_add(float v) {
    auto moved = [](float x, auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value,
                                                          0xF, 0xF, false));
    };
    v += moved(v, std::integral_constant<int, 0xB1>{});
    v += moved(v, std::integral_constant<int, 0x4E>{});
    if (N == 8) v += moved(v, std::integral_constant<int, 0x141>{});
    return v;
}

__device__ __forceinline__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)a, (__bf16)b});
}

// Sine and cosine of t turns: what is left of the nearest quarter, in 32 bits, by their Taylor
// series, whose next terms are below 2^-29, and the quarter by which is which and its sign.
// (The hardware's own, of a rest of up to half a turn, are off by 2^-22.9, and a token of 8 rows
// takes 4.9 us with them: more of what is quantised after them comes out a step away.)
__device__ __forceinline__ void sine_of_turns(double t, float* sine, float* cosine) {
    const double quarters = __builtin_rint(4 * t);
    const float x = 6.2831853071795865f * (float)(t - 0.25 * quarters), y = x * x;
    const int n = (int)(quarters - 4 * __builtin_floor(0.25 * quarters));
    float s = fmaf(y, 1.f / 362880, -1.f / 5040);
    s = fmaf(y, s, 1.f / 120);
    s = fmaf(y, s, -1.f / 6);
    s = fmaf(x * y, s, x);
    float c = fmaf(y, -1.f / 3628800, 1.f / 40320);
    c = fmaf(y, c, -1.f / 720);
    c = fmaf(y, c, 1.f / 24);
    c = fmaf(y, c, -0.5f);
    c = fmaf(y, c, 1.f);
    const float u = n & 1 ? c : s, v = n & 1 ? s : c;
    *sine = n & 2 ? -u : u;
    *cosine = (n + 1) & 2 ? -v : v;
}

struct Call {
    RotaryArgs a;
    RotaryCache to;
    int split;   // wavefronts of a token
    int blocks;  // of the queries and keys; the values' come behind them
    int eights;  // blocks of eight tokens that a list's values may touch, 0: taken one by one
};

// The 16 values of a lane: where its two halves start in a row, and the first values of
// the half's group of 32 (FP4).
struct Place {
    int off[2];
    bool turns;
};

// A key row into its page: eight values at each of the two places.
template <int TYPE, int D>
__device__ __forceinline__ void store_key(const PagedDims& c, char* page, int tp, const Place& p,
                                          const uint32_t* w, int u, uint16_t* tops) {
    if constexpr (TYPE == kBf16) {
        uint16_t* row = reinterpret_cast<uint16_t*>(page + tp * (2 * D));
        *reinterpret_cast<uint4*>(row + p.off[0]) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(row + p.off[1]) = make_uint4(w[4], w[5], w[6], w[7]);
        return;
    }
    uint32_t m[2];  // largest bits of each half's eight values
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        m[x] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m[x] = pk_max(m[x], w[4 * x + i] & 0x7fff7fffu);
    }
    if constexpr (TYPE == kInt8) {
        const uint32_t both = lanes_max<D / 16>(pk_max(m[0], m[1]));
        const uint16_t s = int8_scale(max(both & 0xffffu, both >> 16));
        const Int8Row row(s);
#pragma unroll
        for (int x = 0; x < 2; ++x)
            *reinterpret_cast<uint2*>(page + tp * D + p.off[x]) =
                make_uint2(row.codes(w[4 * x], w[4 * x + 1]), row.codes(w[4 * x + 2], w[4 * x + 3]));
        if (u == 0) reinterpret_cast<uint16_t*>(page + c.ks_off)[tp] = s;
    } else {
        // the eights of a group of 32 lie in lanes that depend on r: through LDS, which a
        // wavefront reads and writes in order
#pragma unroll
        for (int x = 0; x < 2; ++x) tops[p.off[x] / 8] = (uint16_t)max(m[x] & 0xffffu, m[x] >> 16);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const uint2 t = *reinterpret_cast<const uint2*>(tops + p.off[x] / 32 * 4);
            const uint32_t four = pk_max(t.x, t.y);
            const uint32_t e = fp4_scale(max(four & 0xffffu, four >> 16));
            const float s = fp4_power(e);
            uint32_t o = 0;
            auto lo = [](uint32_t v) { return __uint_as_float(v << 16); };
            auto hi = [](uint32_t v) { return __uint_as_float(v & 0xffff0000u); };
            const uint32_t* v = w + 4 * x;
            o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, lo(v[0]), hi(v[0]), s, 0);
            o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, lo(v[1]), hi(v[1]), s, 1);
            o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, lo(v[2]), hi(v[2]), s, 2);
            o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, lo(v[3]), hi(v[3]), s, 3);
            *reinterpret_cast<uint32_t*>(page + tp * (D / 2) + p.off[x] / 2) = o;
            if (p.off[x] % 32 == 0) page[c.ks_off + tp * (D / 32) + p.off[x] / 32] = (char)e;
        }
        // before the next row's are written
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

// How a row lies in its lanes: pairs beside each other, or halves; kWhole: halves of 128 bytes,
// lines that each load reads whole, and nobody again.  (Keys and queries of 16 prompts, 32
// heads of 128: 102 us, loaded past the caches so 88; lines that two loads share, past the
// caches, 173 instead of 160 for 32768 tokens of 40 heads.)
enum { kPairs, kHalves, kWhole };

template <int TYPE, int D, int ORDER>
__device__ __forceinline__ void turn_rows(const Call& call, uint16_t* tops) {
    constexpr int LANES = D / 16, HEADS = 64 / LANES;  // of a row, of a wavefront's step
    constexpr bool HALF = ORDER != kPairs;
    const RotaryArgs& a = call.a;
    const int lane = threadIdx.x & 63;
    const uint32_t job = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t token = job / (uint32_t)call.split, part = job - token * call.split;
    const uint32_t b = token / (uint32_t)a.tokens;
    const int i = (int)(token - b * a.tokens);
    if (b >= (uint32_t)a.rows || (a.counts && i >= a.counts[b])) return;
    const int u = lane % LANES, sub = lane / LANES;
    tops += sub * (D / 8);

    Place p;
    p.turns = u < a.r / 16;
    p.off[0] = HALF && p.turns ? 8 * u : 16 * u;
    p.off[1] = HALF && p.turns ? a.r / 2 + 8 * u : 16 * u + 8;
    float cs[8], sn[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) cs[j] = 1.f, sn[j] = 0.f;
    if (p.turns) {
        const int32_t* at = a.positions + (int64_t)token * a.axes;
        const int first = at[0], second = at[a.axes - 1];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int pair = 8 * u + j;
            const double t = (double)(pair < a.r / 2 / a.axes ? first : second) * a.turns[pair];
            float s, c;
            sine_of_turns(t, &s, &c);
            cs[j] = a.scale * c;
            sn[j] = a.scale * s;
        }
    }

    const int heads = a.q.heads + a.k.heads;
    for (int f = (int)part * HEADS + sub; f < heads; f += call.split * HEADS) {
        const bool key = f >= a.q.heads;
        const RotaryRows& rows = key ? a.k : a.q;
        const int h = key ? f - a.q.heads : f;
        const uint16_t* in = rows.in + b * rows.from.list + i * rows.from.token + h * rows.from.head;
        u32x4_t in_x[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const u32x4_t* from = reinterpret_cast<const u32x4_t*>(in + p.off[x]);
            if constexpr (ORDER == kWhole) in_x[x] = __builtin_nontemporal_load(from);
            else in_x[x] = *from;
        }
        uint32_t w[8];
        float y[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t v = in_x[j / 4][j % 4];
            y[2 * j] = __uint_as_float(v << 16);
            y[2 * j + 1] = __uint_as_float(v & 0xffff0000u);
        }
        if (a.norm != HEADKV_NORM_NONE) {
            if (a.norm == HEADKV_NORM_LAYER) {
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 16; ++j) sum += y[j];
                const float mean = lanes_add<LANES>(sum) * (1.f / D);
#pragma unroll
                for (int j = 0; j < 16; ++j) y[j] -= mean;
            }
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) sum = fmaf(y[j], y[j], sum);
            const float f = rsqrtf(lanes_add<LANES>(sum) * (1.f / D) + a.eps);
#pragma unroll
            for (int j = 0; j < 16; ++j) y[j] *= f;
            if (rows.weight) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(
                        rows.weight + h * rows.step + p.off[x / 2] + 4 * (x & 1));
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[4 * x + e] *= v[e];
                }
            }
            if (rows.bias) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(
                        rows.bias + h * rows.step + p.off[x / 2] + 4 * (x & 1));
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[4 * x + e] += v[e];
                }
            }
        }
        if (p.turns) {  // (what does not turn keeps its bits: a product with 0 may be NaN)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float& m = y[HALF ? j : 2 * j];
                float& n = y[HALF ? 8 + j : 2 * j + 1];
                const float x = m, z = n;
                m = x * cs[j] - z * sn[j];
                n = x * sn[j] + z * cs[j];
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = pack(y[2 * j], y[2 * j + 1]);
        if (TYPE == kNoCache || !key) {
            uint16_t* out = rows.out + b * rows.to.list + i * rows.to.token + h * rows.to.head;
#pragma unroll
            for (int x = 0; x < 2; ++x)
                __builtin_nontemporal_store(
                    u32x4_t{w[4 * x], w[4 * x + 1], w[4 * x + 2], w[4 * x + 3]},
                    reinterpret_cast<u32x4_t*>(out + p.off[x]));
        } else {
            const PagedDims& c = call.to.c;
            const PagedLists& ls = call.to.lists;
            const int64_t lh = (int64_t)b * c.heads + h;
            const int64_t to = (int64_t)(ls.len ? max(ls.len[lh], 0) : 0) + ls.extra + i;
            char* page = const_cast<char*>(list_page(c, ls, call.to.pool, lh, to));
            if (page)
                store_key<TYPE == kNoCache ? kBf16 : TYPE, D>(c, page, (int)(to & (c.ptok - 1)), p, w,
                                                              u, tops);
        }
    }
}

template <int TYPE, int D, int ORDER>
__global__ __launch_bounds__(kThreads) void k_rotary(Call call) {
    constexpr int kTops = TYPE == kFp4 ? 64 / (D / 16) * (D / 8) : 1;  // of a wavefront
    __shared__ __align__(16) uint16_t tops[kWaves][kTops];
    if constexpr (TYPE != kNoCache) {
        if (blockIdx.x >= (unsigned)call.blocks) {
            const int block = blockIdx.x - call.blocks;
            const RotaryCache& t = call.to;
            if (call.eights)
                write_eights<TYPE, D, false>(block, t.c, t.pool, t.lists, nullptr, t.v, t.v_rows,
                                             call.a.tokens, call.eights, call.a.counts);
            else
                write_singles<TYPE, D, false>(block, t.c, t.pool, t.lists, nullptr, t.v, t.v_rows,
                                              call.a.tokens, call.a.counts);
            return;
        }
    }
    turn_rows<TYPE, D, ORDER>(call, tops[threadIdx.x >> 6]);
}

// Wavefronts of a call: below so many, a token's heads are shared among more.
constexpr int kFill = 4096;
// Values are written token by token up to so many tokens, as headkv_paged_write does.
constexpr int kFew = 4;

template <int TYPE, int D>
int launch(Call call, hipStream_t st) {
    const RotaryArgs& a = call.a;
    constexpr int HEADS = 64 / (D / 16);
    const int64_t tokens = (int64_t)a.rows * a.tokens;
    const int steps = std::max(1, (a.q.heads + a.k.heads + HEADS - 1) / HEADS);
    call.split = (int)std::min<int64_t>(steps, std::max<int64_t>(1, kFill / tokens));
    const int64_t blocks = (tokens * call.split + kWaves - 1) / kWaves;
    int64_t more = 0;
    if (TYPE != kNoCache) {
        constexpr int kTasks = kThreads / (D / 2);
        auto tasks = [&](int64_t of_list) {
            return ((int64_t)a.rows * call.to.c.heads * of_list + kTasks - 1) / kTasks;
        };
        more = tasks(a.tokens);
        if (a.tokens > kFew || blocks + more >= 1 << 24) {
            call.eights = (int)(((int64_t)a.tokens + 14) / 8);
            more = tasks(call.eights);
        }
    }
    if (blocks + more >= 1 << 24) return kTooLarge;  // 2^32 threads: more than a launch has
    call.blocks = (int)blocks;
    const unsigned grid = (unsigned)(blocks + more);
    if (a.layout == HEADKV_ROPE_PAIRS)
        k_rotary<TYPE, D, kPairs><<<grid, kThreads, 0, st>>>(call);
    else if (D == 128 && a.r == D)
        k_rotary<TYPE, D, D == 128 ? kWhole : kHalves><<<grid, kThreads, 0, st>>>(call);
    else
        k_rotary<TYPE, D, kHalves><<<grid, kThreads, 0, st>>>(call);
    return (int)hipGetLastError();
}

template <int D>
int launch_type(const Call& call, int type, hipStream_t st) {
    return type == kNoCache ? launch<kNoCache, D>(call, st)
           : type == kBf16  ? launch<kBf16, D>(call, st)
           : type == kInt8  ? launch<kInt8, D>(call, st)
                            : launch<kFp4, D>(call, st);
}

}  // namespace

int launch_rotary(const RotaryArgs& a, const RotaryCache* cache, void* stream) {
    Call call{};
    call.a = a;
    if (cache) call.to = *cache;
    const int type = cache ? cache->c.type : kNoCache;
    return a.d == 128 ? launch_type<128>(call, type, (hipStream_t)stream)
                      : launch_type<64>(call, type, (hipStream_t)stream);
}

}  // namespace headkv
