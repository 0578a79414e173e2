// Decode attention over a paged cache, with prefixes that several rows share
// (formulas and formats: headkv.h; page layout: paged.h).
//
// All query vectors that read one list of keys and values are the columns of one
// small matrix: the group's query heads for a row's own list, those of every row
// that shares it for a prefix.  A wavefront takes NB * 16 columns and steps of 32
// tokens (a step lies in one page); per step, on 16x16x32 bf16 matrix
// instructions,
//   S^T = K Q^T   A = the keys as they lie in the page: lane l holds 16 bytes of
//                 one token's row at a time.  Which dims a lane's part of the
//                 contraction stands for is free as long as Q^T agrees, so a
//                 load is contiguous; which token a row of A stands for is free
//                 too, and is chosen so that the eight scores a lane gets are
//                 those of the eight tokens of one V cell.
//   softmax       online, per column in fp32 (exp2), a running maximum per
//                 wavefront
//   O^T += V^T P^T  A = V cells (eight tokens of a dim) as they lie in the page,
//                 B = the lane's eight weights as they are.  A weight enters as
//                 three bf16 numbers that sum to it exactly (24 bits), so P keeps
//                 fp32's precision.
// Nothing goes through LDS or between lanes but the maximum.  Codes of 8 and 4
// bits are exact in bf16; an INT8 scale multiplies its token's score or weight,
// an FP4 scale enters with the conversion.
// The wavefronts of a block split its tokens and meet in LDS; blocks split a list
// into chunks, whose parts (maximum, sum, unnormalised output) the block that brings
// the last part of a row's list joins in their order, those of the row's prefix
// among them.
// One MI355X, d = 128: 64 x 32 lists of 2000 INT8 tokens 187 us, 5.7 TB/s of codes and
// scales (a copy reads and writes 5.1), BF16 334, 6.3 TB/s, bound by the bytes, FP4 116; of
// 64 to 1024 INT8 tokens 38 us, 4.9 TB/s, and 1 x 32 lists of up to 2480 8.8 us, by the four
// loads that wait for each other before the first tokens are there and the join; 32 x 8
// FP4 lists of up to 16384 for 4 heads each 56 us, 3.9 TB/s, the vector ALU busy for 46 % and
// the matrix cores for 18 % of the time, 2.4 of the 4 wavefronts of a SIMD there on
// average.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "paged.h"
#include "paged_device.h"

namespace headkv {
namespace {

using namespace dev;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kStep = 32;                          // tokens of a wavefront's step
constexpr int kUnit = kStep * kWaves;              // and of a block's
constexpr int kSharedMost = 64 * kStep;            // tokens of a chunk at most: pages in the lanes
constexpr int kWideWaves = 8, kWideThreads = 64 * kWideWaves;
constexpr int kCutBlocks = 256;                 // that few cuts of many columns are made into
constexpr int kWideCols = 2 * 16 * kWideWaves;  // columns of a block of k_attn_shared_wide
constexpr int kCutCols = 16 * kWideWaves;       // and of k_attn_cut_wide

// One attention call as the kernels see it.
struct AttnCall {
    PagedDims c;
    const char* pool;
    PagedLists own, shared;
    const int32_t* share;
    const uint16_t* q;
    int64_t q_stride;
    float* out;
    float* lse;
    int* arrived;  // [kCounters] chunks that are done, of the launch's lists in their order
    f32x2_t* ml;   // [batch][query heads][own parts] maximum (log2) and sum
    float* part;   // [batch][query heads][own parts][d]
    f32x2_t* shared_ml;  // [batch][query heads][shared parts]
    float* shared_part;  // [batch][query heads][shared parts][d]
    int list0, lists;                // own lists of this launch, in their order
    int own_chunk, own_parts;        // tokens of a chunk, chunks at most
    int shared_chunk, shared_parts;  // (0: no shared lists)
    int tiles;                       // column tiles in the grid, per shared list
    int shared_block0, shared_blocks;  // of this launch, before those of own lists
    // Several tokens of each row (TOK): a row's tokens are cut into `cuts` of `cut` each,
    // and a cut takes the place of a row: own.lists counts cuts, c.group is the columns of
    // one, `cut` tokens of `heads` query heads.
    int tokens, cuts, cut, heads, reach;  // reach: no list has more tokens, new ones too
    int64_t q_token, row0;
    int* chunk_of_all;  // the chunk that few cuts of many columns have got
    const int32_t* counts;
    const int32_t* window;
};

// The tokens of a cut: n from token0 of row b on; n <= 0: none.
struct Cut {
    int b, token0, n;
    __device__ __forceinline__ Cut(const AttnCall& a, int v) {
        b = v / a.cuts;
        token0 = (v - b * a.cuts) * a.cut;
        n = min(a.cut, (a.counts ? min(a.counts[b], a.tokens) : a.tokens) - token0);
    }
};

__device__ __forceinline__ u32x4_t nt16(const char* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
}

// What a step reads of a page: lane l has i = l % 16 and quarter = l / 16.
template <int TYPE, int D>
struct Tile {
    static constexpr int KN = TYPE == kBf16 ? D / 32 : TYPE == kInt8 ? D / 64 : 1;
    static constexpr int VN = TYPE == kBf16 ? D / 16 : TYPE == kInt8 ? D / 32 : D / 64;
    static constexpr int kRow = TYPE == kBf16 ? 2 * D : TYPE == kInt8 ? D : D / 2;  // of a token
    u32x4_t k[2][KN];
    u32x4_t v[VN];
    u32x4_t ks, vs;     // INT8: scales of the quarter's eight tokens
    uint32_t ke[2];     // FP4: exponents of the lane's key rows
    u32x2_t ve[D / 64]; // and of its eight tokens of each V load

    // Where a lane's loads are, from the step's place in the page: 32 bits beside an
    // address that the wavefront has in scalar registers.
    struct Place {
        uint32_t key, value, scales, key_powers, value_powers;
        __device__ __forceinline__ Place(const PagedDims& c, int lane) {
            const uint32_t i = lane & 15, quarter = lane >> 4, row = 8 * (i >> 2) + (i & 3);
            key = row * kRow + quarter * (TYPE == kFp4 && D == 64 ? 8 : 16);
            value = quarter * (8 * kRow) + i * 16;
            scales = 16 * quarter;
            key_powers = row * (D / 32) + (D == 128 ? quarter : quarter >> 1);
            value_powers = (i >> 3) * c.ptok + 8 * quarter;
        }
    };

    // ONCE: nobody else reads it.
    template <bool ONCE, typename T>
    static __device__ __forceinline__ T get(const char* p) {
        const T* t = reinterpret_cast<const T*>(p);
        return ONCE ? __builtin_nontemporal_load(t) : *t;
    }
    template <bool ONCE>
    __device__ __forceinline__ void load(const PagedDims& c, const char* page, int tp, const Place& o) {
        const char* at = page + tp * kRow;
        if constexpr (TYPE == kInt8) {
            ks = *reinterpret_cast<const u32x4_t*>(page + c.ks_off + 2 * tp + o.scales);
            vs = *reinterpret_cast<const u32x4_t*>(page + c.vs_off + 2 * tp + o.scales);
        }
        // 16 bytes (FP4, d = 64: 8) of the rows of the two key blocks
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (TYPE == kFp4)
                ke[u] = (uint8_t)(page + c.ks_off + tp * (D / 32) + o.key_powers)[4 * u * (D / 32)];
#pragma unroll
            for (int j = 0; j < KN; ++j) {
                const char* from = at + o.key + (4 * u * kRow + 64 * j);
                if constexpr (TYPE == kFp4 && D == 64) {
                    const u32x2_t w = get<ONCE, u32x2_t>(from);
                    k[u][j][0] = w[0], k[u][j][1] = w[1];
                } else {
                    k[u][j] = get<ONCE, u32x4_t>(from);
                }
            }
        }
        // the quarter's eight tokens of 1, 2 or 4 dims
        if constexpr (TYPE == kFp4) {
#pragma unroll
            for (int j = 0; j < VN; ++j)
                ve[j] = *reinterpret_cast<const u32x2_t*>(page + c.vs_off + 2 * j * c.ptok + tp +
                                                          o.value_powers);
        }
#pragma unroll
        for (int j = 0; j < VN; ++j) v[j] = get<ONCE, u32x4_t>(at + c.v_off + o.value + 256 * j);
    }

    // Nothing that times a zero weight is not zero, for the lane's tokens n whose
    // bit n of `seen` is 0 (never written, perhaps): pairs of 16 bits, or bytes.
    static __device__ __forceinline__ u32x4_t blank16(u32x4_t w, uint32_t seen) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] &= (seen >> (2 * e) & 1 ? 0xffffu : 0u) | (seen >> (2 * e + 1) & 1 ? 0xffff0000u : 0u);
        return w;
    }
    static __device__ __forceinline__ u32x2_t blank8(u32x2_t w, uint32_t seen) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) m |= seen >> (4 * h + e) & 1 ? 0xffu << (8 * e) : 0u;
            w[h] &= m;
        }
        return w;
    }
    __device__ __forceinline__ void blank(uint32_t seen) {
        if constexpr (TYPE == kInt8) vs = blank16(vs, seen);
#pragma unroll
        for (int j = 0; j < VN; ++j) {
            if constexpr (TYPE == kFp4) ve[j] = blank8(ve[j], seen);
            if constexpr (TYPE == kBf16) v[j] = blank16(v[j], seen);
        }
    }
};

// First of the eight dims of key step s that a lane of `quarter` holds.
template <int TYPE, int D>
__device__ __forceinline__ int key_dim(int s, int quarter) {
    if (TYPE == kBf16) return 32 * s + 8 * quarter;
    if (TYPE == kInt8) return 64 * (s >> 1) + 16 * quarter + 8 * (s & 1);
    return D / 4 * quarter + 8 * s;
}

__device__ __forceinline__ uint32_t pack_high(uint32_t lo, uint32_t hi) {  // bits 31:16 of each
    return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
}
__device__ __forceinline__ uint32_t pack_low(uint32_t lo, uint32_t hi) {
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}
// A loaded word as it is: without this the compiler keeps the bytes that are used
// later apart from the load on, in a register each (INT8, d = 128: 347 instead of
// 155 registers).
__device__ __forceinline__ uint32_t whole(uint32_t w) {
    asm("" : "+v"(w));
    return w;
}
// four int8 codes as bf16 (exact)
__device__ __forceinline__ void int8_pack(uint32_t in, uint32_t* o) {
    const uint32_t w = whole(in);
    const uint32_t a = __float_as_uint((float)(int8_t)w), b = __float_as_uint((float)(int8_t)(w >> 8));
    const uint32_t c = __float_as_uint((float)(int8_t)(w >> 16)), d = __float_as_uint((float)(int8_t)(w >> 24));
    o[0] = pack_high(a, b);
    o[1] = pack_high(c, d);
}
// The conversion takes its scale from the exponent; that of byte 255 gives NaN.
__device__ __forceinline__ float fp4_exponent(uint32_t e) { return __uint_as_float(e << 23); }
template <int SEL>
__device__ __forceinline__ uint32_t fp4_pack(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}
__device__ __forceinline__ bf16x8_t operand(const uint32_t* w) {
    return __builtin_bit_cast(bf16x8_t, u32x4_t{w[0], w[1], w[2], w[3]});
}

// K operand n of a load of keys (it has 1, 2 or d / 32 of them).
template <int TYPE>
__device__ __forceinline__ bf16x8_t key_operand(const u32x4_t& k, uint32_t ke, int n) {
    if constexpr (TYPE == kBf16) return __builtin_bit_cast(bf16x8_t, k);
    uint32_t o[4];
    if constexpr (TYPE == kInt8) {
        int8_pack(k[2 * n], o);
        int8_pack(k[2 * n + 1], o + 2);
    } else {
        const float e = fp4_exponent(ke);
        const uint32_t w = k[n];
        o[0] = fp4_pack<0>(w, e);
        o[1] = fp4_pack<1>(w, e);
        o[2] = fp4_pack<2>(w, e);
        o[3] = fp4_pack<3>(w, e);
    }
    return operand(o);
}

// The two V^T operands of eight FP4 bytes: two dims of the lane's eight tokens.
__device__ __forceinline__ void fp4_pair(uint32_t v0, uint32_t v1, const u32x2_t& ve, bf16x8_t* a) {
    uint32_t w[8], lo[4], hi[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t b = h ? v1 : v0, x = whole(ve[h]);
        w[4 * h] = fp4_pack<0>(b, fp4_exponent(x & 0xffu));
        w[4 * h + 1] = fp4_pack<1>(b, fp4_exponent(x >> 8 & 0xffu));
        w[4 * h + 2] = fp4_pack<2>(b, fp4_exponent(x >> 16 & 0xffu));
        w[4 * h + 3] = fp4_pack<3>(b, fp4_exponent(x >> 24));
    }
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        lo[n] = pack_low(w[2 * n], w[2 * n + 1]);
        hi[n] = pack_high(w[2 * n], w[2 * n + 1]);
    }
    a[0] = operand(lo);
    a[1] = operand(hi);
}
// V^T operands of a load of values: one for each of the dims it holds (1, 2 or 4).
template <int TYPE>
__device__ __forceinline__ void value_operands(const u32x4_t& v, const u32x2_t& ve, bf16x8_t* a) {
    if constexpr (TYPE == kBf16) {
        a[0] = __builtin_bit_cast(bf16x8_t, v);
    } else if constexpr (TYPE == kInt8) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            uint32_t o[4];
            int8_pack(v[2 * x], o);
            int8_pack(v[2 * x + 1], o + 2);
            a[x] = operand(o);
        }
    } else {
        const u32x2_t e{whole(ve[0]), whole(ve[1])};
        fp4_pair(v[0], v[1], e, a);
        fp4_pair(v[2], v[3], e, a + 2);
    }
}

// Bit n: token n of the lane's eight, of the step at `at`, lies in [first, end).
__device__ __forceinline__ uint32_t seen_of(int at, int first, int end, int lane) {
    const int tk = at + 8 * (lane >> 4);
    const int lo = min(max(first - tk, 0), 8), hi = min(max(end - tk, 0), 8);
    return 0xffu >> (8 - hi) & 0xffu << lo;
}

// f over the four lanes of a column (lanes i, i + 16, i + 32, i + 48).
template <typename F>
__device__ __forceinline__ float over_quarters(float v, F f) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(x[0]), __uint_as_float(x[1]));
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

__device__ __forceinline__ float rounded(float a, float b) {  // the product, not fused
#pragma clang fp contract(off)
    return a * b;
}

// Without the instructions that fmaxf adds where an argument might be a signalling
// NaN.  (Not for what a matrix instruction has just written: the compiler keeps no
// distance from it for an asm.)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The reference before any score: below all, and finite, so that nothing is NaN.
constexpr float kLow = -3.402823466e38f;

// All ones in each half of w that is no finite bf16.
__device__ __forceinline__ u32x4_t odd_of(const u32x4_t& w) {
    u32x4_t odd;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        odd[e] = ((w[e] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) |
                 ((w[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
    return odd;
}
// The largest bits so far of each half, without signs; and whether any lane has one of those.
__device__ __forceinline__ uint32_t top_of(uint32_t top, const u32x4_t& w) {
    typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < 4; ++e)
        top = __builtin_bit_cast(
            uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, top),
                                                __builtin_bit_cast(u16x2_t, w[e] & 0x7fff7fffu)));
    return top;
}
__device__ __forceinline__ bool any_odd(uint32_t top) {
    return __builtin_amdgcn_ballot_w64((top & 0xffffu) >= 0x7f80u || top >= 0x7f800000u) != 0;
}

// State of a wavefront: column i = lane % 16 of each of its NB tiles.
template <int TYPE, int D, int NB>
struct Wave {
    static constexpr int KS = D / 32;  // key steps
    static constexpr int DB = D / 16;  // blocks of 16 output rows
    static constexpr int VX = DB / Tile<TYPE, D>::VN;  // dims of a V load
    bf16x8_t q[NB][KS];
    f32x4_t acc[NB][DB];  // block VX j + x: rows 16 of load j, dim x of each
    float m[NB], sum[NB];  // reference (log2) and sum of 2^(score - reference)
    // A reference is a rounded product; scores less it, computed with one rounding, are
    // off by that, half a unit in its last place: 1/2 at 2^24, 128 and so past exp2's
    // range at 2^31.  From 2^24 on the scores are rounded like it too.
    bool far;

    __device__ __forceinline__ void clear() {
        far = false;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            m[b] = kLow;
            sum[b] = 0.f;
#pragma unroll
            for (int j = 0; j < DB; ++j) acc[b][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    }

    // One step: operands from key(u, s) and value(j, a), INT8 scales.  partial: not
    // all tokens are attended, bit n of seen_by(b) is set if token n of the lane's eight is
    // by its column of tile b.
    template <typename Key, typename Value, typename SeenBy>
    __device__ __forceinline__ void step(Key key, Value value, const u32x4_t& key_scales,
                                         const u32x4_t& value_scales, bool partial, SeenBy seen_by) {
        constexpr float kScale = (float)(1.4426950408889634 / (D == 128 ? 11.313708498984761 : 8.0));
        f32x4_t st[NB][2];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8_t a = key(u, s);
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    st[b][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        a, q[b][s], s == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : st[b][u], 0, 0, 0);
            }
        }
        float ks[8], vs[8];  // INT8: scales of the lane's tokens
#pragma unroll
        for (int n = 0; n < 8; ++n) ks[n] = kScale;
        if constexpr (TYPE == kInt8) {
#pragma unroll
            for (int n = 0; n < 8; n += 2) {
                const uint32_t k = whole(key_scales[n / 2]), v = whole(value_scales[n / 2]);
                ks[n] *= __uint_as_float(k << 16);
                ks[n + 1] *= __uint_as_float(k & 0xffff0000u);
                vs[n] = __uint_as_float(v << 16);
                vs[n + 1] = __uint_as_float(v & 0xffff0000u);
            }
        }
        // pieces of the weights: B operands, three for each column tile
        bf16x8_t p[NB][3];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            // scores less the reference, log2
            const uint32_t seen = seen_by(b);
            float x[8];
            auto less = [&](bool twice) {
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    const float s = st[b][n / 4][n % 4];
                    if (twice) x[n] = rounded(s, ks[n]) - m[b];
                    else x[n] = fmaf(s, ks[n], -m[b]);
                }
                if (__builtin_expect(partial, 0)) {
                    asm volatile("");  // a branch: its selects cost as much as the products
#pragma unroll
                    for (int n = 0; n < 8; ++n) x[n] = seen >> n & 1 ? x[n] : -INFINITY;
                }
            };
            if (__builtin_expect(far, 0)) less(true);
            else less(false);
            // A reference up to 2^8 below the largest score does as well, and has to
            // follow it far less often.
            const float most = max3(max3(max3(x[0], x[1], x[2]), x[3], x[4]), max3(x[5], x[6], x[7]), 0.f);
            if (__builtin_amdgcn_ballot_w64(most > 8.f) != 0) {
                float mx = kLow;
#pragma unroll
                for (int n = 0; n < 8; ++n)
                    if (!partial || (seen >> n & 1)) mx = fmaxf(mx, rounded(st[b][n / 4][n % 4], ks[n]));
                mx = over_quarters(mx, [](float x, float y) { return fmaxf(x, y); });
                const float now = fmaxf(mx, m[b]), f = __builtin_amdgcn_exp2f(m[b] - now);
                m[b] = now;
                far = far || __builtin_amdgcn_ballot_w64(now > kLow && !(fabsf(now) < 0x1p24f)) != 0;
                sum[b] *= f;
#pragma unroll
                for (int j = 0; j < DB; ++j) acc[b][j] *= f;
                less(far);
            }
            uint32_t w[3][4];
#pragma unroll
            for (int n = 0; n < 8; n += 2) {
                uint32_t hi[2], mid[2], lo[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float y = __builtin_amdgcn_exp2f(x[n + e]);
                    sum[b] += y;
                    if constexpr (TYPE == kInt8) y *= vs[n + e];
                    hi[e] = __float_as_uint(y);
                    const float r = y - __uint_as_float(hi[e] & 0xffff0000u);
                    mid[e] = __float_as_uint(r);
                    lo[e] = __float_as_uint(r - __uint_as_float(mid[e] & 0xffff0000u));
                }
                w[0][n / 2] = pack_high(hi[0], hi[1]);
                w[1][n / 2] = pack_high(mid[0], mid[1]);
                w[2][n / 2] = pack_high(lo[0], lo[1]);
            }
#pragma unroll
            for (int e = 0; e < 3; ++e) p[b][e] = operand(w[e]);
        }
        // four products that do not wait for each other, at a time
        constexpr int J = VX * NB >= 4 ? 1 : 4 / (VX * NB);
#pragma unroll
        for (int j0 = 0; j0 < Tile<TYPE, D>::VN; j0 += J) {
            bf16x8_t a[J][VX];
#pragma unroll
            for (int j = 0; j < J; ++j) value(j0 + j, a[j]);
#pragma unroll
            for (int e = 0; e < 3; ++e)
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int x = 0; x < VX; ++x)
#pragma unroll
                        for (int b = 0; b < NB; ++b) {
                            f32x4_t& o = acc[b][VX * (j0 + j) + x];
                            o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[j][x], p[b][e], o, 0, 0, 0);
                        }
        }
    }

    // What the lane has of its column in tile b, dims in order (row: d floats).
    __device__ __forceinline__ void to_row(int b, int quarter, float* row) const {
#pragma unroll
        for (int j = 0; j < Tile<TYPE, D>::VN; ++j) {
            const f32x4_t* a = acc[b] + VX * j;
            if constexpr (VX == 1) {
                *reinterpret_cast<f32x4_t*>(row + 16 * j + 4 * quarter) = a[0];
            } else if constexpr (VX == 2) {
                f32x4_t* p = reinterpret_cast<f32x4_t*>(row + 32 * j + 8 * quarter);
                p[0] = f32x4_t{a[0][0], a[1][0], a[0][1], a[1][1]};
                p[1] = f32x4_t{a[0][2], a[1][2], a[0][3], a[1][3]};
            } else {
                f32x4_t* p = reinterpret_cast<f32x4_t*>(row + 64 * j + 16 * quarter);
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] = f32x4_t{a[0][r], a[1][r], a[2][r], a[3][r]};
            }
        }
    }

    // The tokens of the step at token `at` that lie in [first, end).
    __device__ __forceinline__ void step_at(Tile<TYPE, D>& t, int at, int first, int end, int lane) {
        const bool partial = at < first || at + kStep > end;
        uint32_t seen = 0xffu;
        if (partial) {
            seen = seen_of(at, first, end, lane);
            t.blank(seen);
        }
        constexpr int kPer = KS / Tile<TYPE, D>::KN;  // operands of a load of keys
        step([&](int u, int s) { return key_operand<TYPE>(t.k[u][s / kPer], t.ke[u], s % kPer); },
             [&](int j, bf16x8_t* a) { value_operands<TYPE>(t.v[j], t.ve[TYPE == kFp4 ? j : 0], a); },
             t.ks, t.vs, partial, [&](int) { return seen; });
    }

    // Where columns differ in what they attend, a value that is no finite number must not
    // reach those that do not attend it, whose weight is 0.  It is taken out of the operand,
    // and the outputs of the columns that do attend one are NaN from here on: ones in the places
    // of such values (odd: all ones there) times ones for what the lane's column attends count
    // them, for output block `block`.
    __device__ __forceinline__ void spoil(const u32x4_t& odd, uint32_t seen, int block) {
        constexpr uint32_t kOnes = 0x3f803f80u;
        const u32x4_t there{odd[0] & kOnes, odd[1] & kOnes, odd[2] & kOnes, odd[3] & kOnes};
        const u32x4_t mine = Tile<TYPE, D>::blank16(u32x4_t{kOnes, kOnes, kOnes, kOnes}, seen);
        const f32x4_t count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8_t, there), __builtin_bit_cast(bf16x8_t, mine),
            f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[0][block][r] = count[r] > 0.f ? NAN : acc[0][block][r];
    }
    // The same for a tile, of which the lane's column attends `seen`.  (A look at each value of
    // the steps that columns differ in, one or two a list: 64 x 32 lists of 64 to 1024 tokens
    // FP4 32.6 us, with it 33.5, BF16 79.7 and 79.8, INT8 no change; cuts of 128 columns, where
    // whoever converts a value looks at it, 24 rows of 256 tokens FP4 121.2 and 123.1, BF16
    // 116.3 and 119.3.)
    __device__ __forceinline__ void keep_apart(Tile<TYPE, D>& t, uint32_t seen) {
        using T = Tile<TYPE, D>;
        if constexpr (TYPE == kInt8) {  // scales, which the lane gives its column's weights
            t.vs = T::blank16(t.vs, seen);
        } else if constexpr (TYPE == kBf16) {
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < T::VN; ++j) top = top_of(top, t.v[j]);
            if (__builtin_expect(!any_odd(top), 1)) return;
#pragma unroll
            for (int j = 0; j < T::VN; ++j) {
                __builtin_amdgcn_sched_barrier(0);  // (in the registers of one at a time)
                const u32x4_t odd = odd_of(t.v[j]);
                spoil(odd, seen, j);
                t.v[j] &= ~odd;
            }
        } else {
            // exponents from 253 on, of which 4 and 6 are infinite (and all of 255): a lane has
            // those of its quarter's tokens for dims of the first or the second half of a load's
            // 16 rows, and its outputs' rows lie in the first or the second half by its quarter
            auto full = [](uint32_t e) { return ((e & 0x7f7f7f7fu) + 0x03030303u) & e & 0x80808080u; };
            uint32_t some = 0;
#pragma unroll
            for (int j = 0; j < T::VN; ++j) some |= full(t.ve[j][0]) | full(t.ve[j][1]);
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(some != 0) == 0, 1)) return;
            // (worked out here: no register holds it from step to step)
            const int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));
#pragma unroll
            for (int j = 0; j < T::VN; ++j) {
                uint32_t tokens = 0;  // bit n: the lane's token n
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t m = full(t.ve[j][h]) >> 7;
                    t.ve[j][h] &= ~(m * 255u);
                    tokens |= ((m | m >> 7 | m >> 14 | m >> 21) & 15u) << (4 * h);
                }
                bool mine = false;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t of_half = (uint32_t)__shfl((int)tokens, (lane & 48) + 8 * half);
                    const uint64_t hit = __builtin_amdgcn_ballot_w64((of_half & seen) != 0);
                    const uint32_t columns = (uint32_t)(hit | hit >> 16 | hit >> 32 | hit >> 48);
                    if (lane >> 5 == half) mine = columns >> (lane & 15) & 1;
                }
#pragma unroll
                for (int x = 0; x < VX; ++x)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        acc[0][VX * j + x][r] = mine ? NAN : acc[0][VX * j + x][r];
            }
        }
    }

    // A step where columns differ in what they attend: the lane's own is [first, end); all
    // of them attend [all_first, all_end), none outside [any_first, any_end).
    struct Seen {
        int first, end, all_first, all_end, any_first, any_end;
    };
    __device__ __forceinline__ void step_at(Tile<TYPE, D>& t, int at, const Seen& s, int lane) {
        const bool partial = at < s.all_first || at + kStep > s.all_end;
        uint32_t seen = 0xffu;
        if (partial) {
            t.blank(seen_of(at, s.any_first, s.any_end, lane));
            seen = seen_of(at, s.first, s.end, lane);
            keep_apart(t, seen);
        }
        constexpr int kPer = KS / Tile<TYPE, D>::KN;
        step([&](int u, int s) { return key_operand<TYPE>(t.k[u][s / kPer], t.ke[u], s % kPer); },
             [&](int j, bf16x8_t* a) { value_operands<TYPE>(t.v[j], t.ve[TYPE == kFp4 ? j : 0], a); },
             t.ks, t.vs, partial, [&](int) { return seen; });
    }

    // Lane n: the page of the wavefront's n-th step of the tokens [t0, t1).
    template <int W>
    static __device__ __forceinline__ int pages_of(const PagedDims& c, const int32_t* pages, int t0,
                                                   int t1, int wave, int lane) {
        const int mine = t0 + (wave + W * lane) * kStep;
        return mine < t1 ? pages[mine >> c.pshift] : -1;
    }

    // Tokens [t0, t1) of a list, t0 a multiple of 32, those before `first` not
    // attended; this wavefront takes every W-th step, on pages_of()'s page.
    template <bool ONCE, int W>
    __device__ __forceinline__ void run(const PagedDims& c, const char* pool, int page, int t0, int t1,
                                        int first, int wave, int lane) {
        run_steps<ONCE, W>(c, pool, page, t0, t1, wave, lane, [&](Tile<TYPE, D>& t, int at) {
            step_at(t, at, first, t1, lane);
        });
    }
    template <bool ONCE, int W, typename Step>
    __device__ __forceinline__ void run_steps(const PagedDims& c, const char* pool, int page, int t0,
                                              int t1, int wave, int lane, Step step) {
        if (t0 + (wave + W * lane) * kStep >= t1) page = -1;
        uint64_t todo = __builtin_amdgcn_ballot_w64(page >= 0 && page < c.num_pages);
        if (!todo) return;
        const typename Tile<TYPE, D>::Place place(c, lane);
        auto fetch = [&](Tile<TYPE, D>& t, int n) {
            const int at = t0 + (wave + W * n) * kStep;
            t.template load<ONCE>(c, pool + __builtin_amdgcn_readlane(page, n) * c.page_bytes, at & (c.ptok - 1), place);
        };
        Tile<TYPE, D> now, next;
        int n = __builtin_ctzll(todo);
        fetch(now, n);
        for (;;) {
            todo &= todo - 1;
            const int after = todo ? __builtin_ctzll(todo) : -1;
            if (after >= 0) fetch(next, after);
            step(now, t0 + (wave + W * n) * kStep);
            if (after < 0) break;
            // Two tiles in turn, without the copy, take 12 to 30 more registers: 64 x 32
            // lists of 1000 INT8 tokens 42 us instead of 39.
            now = next;
            n = after;
        }
    }
};

// A barrier of the W wavefronts that work together: all of a block, or one alone.
template <int W>
__device__ __forceinline__ void together() {
    if constexpr (W == kWaves) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

// Joins W wavefronts and gives the maximum, sum and output of their first `cols`
// columns to `store(column, d, four outputs, m, sum)`.
template <int W, int TYPE, int D, typename Store>
__device__ __forceinline__ void join_waves(Wave<TYPE, D, 1>& w, float* lds, int cols, int wave,
                                           int lane, Store store) {
    constexpr int ROW = D + 4;  // floats of a column in LDS: 16-byte writes of 16 columns do not meet
    float* ms = lds;                     // [wave][16] maximum, then sum
    float* o = lds + 2 * W * 16;         // [wave][cols][ROW]
    const int i = lane & 15, quarter = lane >> 4;
    const float sum = over_quarters(w.sum[0], [](float x, float y) { return x + y; });
    if (lane < 16) {
        ms[wave * 16 + lane] = w.m[0];
        ms[(W + wave) * 16 + lane] = sum;
    }
    if (i < cols) w.to_row(0, quarter, o + (wave * cols + i) * ROW);
    together<W>();
    for (int k = wave * 64 + lane; k < cols * (D / 4); k += 64 * W) {
        const int col = k / (D / 4), d = k % (D / 4) * 4;
        float m = kLow;
#pragma unroll
        for (int x = 0; x < W; ++x) m = fmaxf(m, ms[x * 16 + col]);
        f32x4_t v{0.f, 0.f, 0.f, 0.f};
        float s = 0.f;
#pragma unroll
        for (int x = 0; x < W; ++x) {
            const float mx = ms[x * 16 + col];
            const float f = __builtin_amdgcn_exp2f(mx - m);
            s += f * ms[(W + x) * 16 + col];
            v += f * *reinterpret_cast<const f32x4_t*>(o + (x * cols + col) * ROW + d);
        }
        store(col, d, v, m, s);
    }
    together<W>();
}

// LDS that W wavefronts need for `cols` columns.
constexpr size_t join_bytes(int d, int cols, int W = kWaves) {
    return (2 * W * 16 + W * cols * (d + 4)) * sizeof(float);
}

__device__ __forceinline__ void write_out(const AttnCall& a, int64_t row, int d, int D, f32x4_t v,
                                          float m, float sum) {
    if (row < 0) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    *reinterpret_cast<f32x4_t*>(a.out + row * D + d) = v * inv;
    if (a.lse && d == 0)
        a.lse[row] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// The chunks of a list: its tokens from the step of `first` on.
struct Span {
    int len, first, start, chunks;
};
__device__ __forceinline__ Span span_of(const PagedLists& p, int ptok, int64_t lh, int chunk) {
    Span s;
    s.len = list_len(p, ptok, lh);
    s.first = p.first ? max(p.first[lh], 0) : 0;
    s.start = s.first & ~(kStep - 1);
    s.chunks = s.len > s.first ? (s.len - s.start + chunk - 1) / chunk : 0;
    return s;
}

// The same of a cut, whose first token sees least of what is behind a window.
__device__ __forceinline__ Span span_of_cut(const AttnCall& a, int64_t real, const Cut& cut, int chunk,
                                            int* base, int* window) {
    Span s;
    *base = list_len(a.own, a.c.ptok, real);
    *window = a.window ? a.window[real] : 0;
    s.first = a.own.first ? max(a.own.first[real], 0) : 0;
    if (*window > 0) s.first = max(s.first, *base + cut.token0 + 1 - *window);
    s.len = min(*base + cut.token0 + cut.n, a.own.max_pages * a.c.ptok);
    s.start = s.first & ~(kStep - 1);
    s.chunks = s.len > s.first ? (s.len - s.start + chunk - 1) / chunk : 0;
    return s;
}
// Chunks of the own list of row (TOK: cut) v, kv head h.
template <bool TOK>
__device__ __forceinline__ int own_chunks(const AttnCall& a, int v, int h) {
    if constexpr (TOK) {
        const Cut cut(a, v);
        int base, window;
        return span_of_cut(a, (int64_t)cut.b * a.c.heads + h, cut, a.own_chunk, &base, &window).chunks;
    }
    return span_of(a.own, a.c.ptok, (int64_t)v * a.c.heads + h, a.own_chunk).chunks;
}
// Row of q, of kv head h: column `col` of row (TOK: cut) v.
template <int D, bool TOK>
__device__ __forceinline__ const uint16_t* query(const AttnCall& a, int v, int h, int col) {
    if constexpr (TOK) {
        const Cut cut(a, v);
        const int token = min(col / a.heads, max(cut.n, 1) - 1), head = col % a.heads;
        return a.q + cut.b * a.q_stride + (cut.token0 + token) * a.q_token + (h * a.heads + head) * D;
    }
    return a.q + v * a.q_stride + (h * a.c.group + col) * D;
}
// Its row of the output; -1: none, a token behind the row's last.
template <bool TOK>
__device__ __forceinline__ int64_t out_row(const AttnCall& a, int lh, int col) {
    if constexpr (TOK) {
        const int v = lh / a.c.heads, h = lh - v * a.c.heads;
        const Cut cut(a, v);
        const int token = col / a.heads;
        if (token >= cut.n) return -1;
        return (((int64_t)cut.b * a.tokens + cut.token0 + token) * a.c.heads + h) * a.heads +
               col % a.heads;
    }
    return (int64_t)lh * a.c.group + col;
}

// Parts that a block of another XCD reads in the same launch: written through,
// and read past, the L2s.
__device__ __forceinline__ void publish(void* p, uint32_t lo, uint32_t hi) {
    __hip_atomic_store(static_cast<uint64_t*>(p), (uint64_t)hi << 32 | lo, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2_t published(const void* p) {
    return __builtin_bit_cast(f32x2_t, __hip_atomic_load(static_cast<const uint64_t*>(p),
                                                         __ATOMIC_RELAXED,
                                                         __HIP_MEMORY_SCOPE_AGENT));
}

__device__ __forceinline__ void publish4(float* p, f32x4_t v) {
    publish(p, __float_as_uint(v[0]), __float_as_uint(v[1]));
    publish(p + 2, __float_as_uint(v[2]), __float_as_uint(v[3]));
}

// The sum of parts, one after the other.
struct Sum {
    f32x4_t v{0.f, 0.f, 0.f, 0.f};
    float m = kLow, s = 0.f;
    __device__ __forceinline__ void add(f32x4_t pv, float pm, float ps) {
        const float now = fmaxf(m, pm);
        const float f = __builtin_amdgcn_exp2f(m - now), g = __builtin_amdgcn_exp2f(pm - now);
        v = f * v + g * pv;
        s = f * s + g * ps;
        m = now;
    }
    // n parts, the loads of eight at a time in flight
    template <typename V, typename M>
    __device__ __forceinline__ void add_parts(int n, V value, M ml) {
        for (int i0 = 0; i0 < n; i0 += 8) {
            f32x4_t v[8];
            f32x2_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = min(i0 + i, n - 1);
                v[i] = value(at);
                w[i] = ml(at);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i0 + i < n) add(v[i], w[i][0], w[i][1]);
        }
    }
};

// The rows whose columns a block of a shared list has: `members` of its rows, counted
// up to rank1, those of ranks [rank0, rank1) in row_of.  W wavefronts.
template <int W, bool TOK>
__device__ __forceinline__ int find_members(const AttnCall& a, int list, int rank0, int rank1,
                                            int* row_of, int* found, int tid) {
    const int lane = tid & 63, wave = tid >> 6;
    int members = 0;
    for (int b0 = 0; b0 < a.own.lists && members < rank1; b0 += 64 * W) {
        const int b = b0 + tid;
        bool is = b < a.own.lists;
        if constexpr (TOK) {
            if (is) {
                const Cut cut(a, b);
                is = cut.n > 0 && a.share[cut.b] == list;
            }
        } else {
            is = is && a.share[b] == list;
        }
        const uint64_t mask = __builtin_amdgcn_ballot_w64(is);
        if (lane == 0) found[wave] = __builtin_popcountll(mask);
        __syncthreads();
        int rank = members + __builtin_popcountll(mask & ((1ull << lane) - 1));
        for (int x = 0; x < W; ++x) {
            if (x < wave) rank += found[x];
            members += found[x];
        }
        if (is && rank >= rank0 && rank < rank1) row_of[rank - rank0] = b;
        __syncthreads();
    }
    return members;
}

// Column `col` of a shared list is a query head of the member of rank col / group.
template <int TYPE, int D, bool TOK>
__device__ __forceinline__ void load_queries(const AttnCall& a, int h, int col, int rank0,
                                             const int* row_of, int lane, bf16x8_t* q) {
    const int group = a.c.group;
    const uint16_t* from = query<D, TOK>(a, row_of[col / group - rank0], h, col % group);
#pragma unroll
    for (int k = 0; k < D / 32; ++k)
        q[k] = *reinterpret_cast<const bf16x8_t*>(from + key_dim<TYPE, D>(k, lane >> 4));
}
// Where its part of a chunk lies.
__device__ __forceinline__ int64_t shared_slot(const AttnCall& a, int h, int col, int rank0,
                                               const int* row_of, int chunk) {
    const int group = a.c.group;
    const int64_t row = ((int64_t)row_of[col / group - rank0] * a.c.heads + h) * group + col % group;
    return row * a.shared_parts + chunk;
}

// Parts of the prefix that row (of a cut: its row) b shares, for kv head h.
__device__ __forceinline__ int prefix_parts(const AttnCall& a, int b, int h) {
    if (!a.shared_parts) return 0;
    const int l = a.share[b];
    if (l < 0 || l >= a.shared.lists) return 0;
    return span_of(a.shared, a.c.ptok, (int64_t)l * a.c.heads + h, a.shared_chunk).chunks;
}

// Output `col`, dims d .. d + 3 of a list whose `chunks` parts and `prefix` parts are
// all there.  WITH: the prefix's come from the same launch too.
template <int D, bool WITH>
__device__ __forceinline__ void add_prefix(const AttnCall& a, Sum& all, int64_t row, int prefix, int d) {
    const int64_t at = row * a.shared_parts;
    all.add_parts(
        prefix,
        [&](int j) {
            const float* p = a.shared_part + (at + j) * D + d;
            if constexpr (!WITH) return *reinterpret_cast<const f32x4_t*>(p);
            const f32x2_t x = published(p), y = published(p + 2);
            return f32x4_t{x[0], x[1], y[0], y[1]};
        },
        [&](int j) { return WITH ? published(a.shared_ml + at + j) : a.shared_ml[at + j]; });
}
template <int D, bool WITH, bool TOK>
__device__ __forceinline__ void finish(const AttnCall& a, int lh, int chunks, int prefix, int col, int d) {
    const int64_t row = (int64_t)lh * a.c.group + col, slot = row * a.own_parts;
    Sum all;
    all.add_parts(
        chunks,
        [&](int j) {
            const float* p = a.part + (slot + j) * D + d;
            const f32x2_t x = published(p), y = published(p + 2);
            return f32x4_t{x[0], x[1], y[0], y[1]};
        },
        [&](int j) { return published(a.ml + slot + j); });
    add_prefix<D, WITH>(a, all, row, prefix, d);
    write_out(a, out_row<TOK>(a, lh, col), d, D, all.v, all.m, all.s);
}

// `columns` of a list's part have arrived; true for the last of `total`.
__device__ __forceinline__ bool arrive(int* counter, int columns, int total) {
    const bool last = __hip_atomic_fetch_add(counter, columns, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT) + columns == total;
    if (last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return last;
}

// A row's own list: one block, or with W = 1 one wavefront, per (row, kv head, chunk),
// the first also for an empty list.
template <int TYPE, int D, bool WITH, int W, bool TOK>
__device__ __forceinline__ void own_block(const AttnCall& a, int block, float* lds, int* flags) {
    const int lane = threadIdx.x & 63;
    int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int unit = block;
    if constexpr (W == 1) {
        unit = block * kWaves + wave;
        if (unit >= a.lists * a.own_parts) return;
        lds += wave * (join_bytes(D, a.c.group, 1) / sizeof(float));
        flags += wave;
        wave = 0;
    }
    const int tid = wave * 64 + lane;
    const int group = a.c.group;
    const int rank = unit % a.lists, chunk = unit / a.lists;
    int at = a.list0 + rank, last = a.own.lists * a.c.heads - 1, cut_at = 0;
    if constexpr (TOK) {  // the last cut of every row first, which attends most
        const int lists = a.own.lists / a.cuts * a.c.heads;
        cut_at = at / lists;
        at -= cut_at * lists;
        cut_at = a.cuts - 1 - cut_at;
        last = lists - 1;
    }
    int lh = a.own.order ? min(max(a.own.order[at], 0), last) : at;
    const int b = lh / a.c.heads, h = lh % a.c.heads;
    // the pages as they are without a window, before the length is known
    const int32_t* pages = a.own.pages + (int64_t)lh * a.own.max_pages;
    const int g0 = chunk * a.own_chunk, g1 = min(g0 + a.own_chunk, TOK ? a.reach : a.own.max_len);
    int page = Wave<TYPE, D, 1>::template pages_of<W>(a.c, pages, g0, g1, wave, lane);
    Span s;
    int base = 0, window = 0, v = b, token0 = 0;
    if constexpr (TOK) {
        v = b * a.cuts + cut_at;
        const Cut cut(a, v);
        if (cut.n <= 0) return;
        token0 = cut.token0;
        s = span_of_cut(a, lh, cut, a.own_chunk, &base, &window);
        lh = v * a.c.heads + h;
    } else {
        s = span_of(a.own, a.c.ptok, lh, a.own_chunk);
    }
    const int chunks = max(s.chunks, 1);
    if (chunk >= chunks) return;
    const int t0 = s.start + chunk * a.own_chunk, t1 = min(s.len, t0 + a.own_chunk);
    const int64_t row0 = (int64_t)lh * group;
    const int prefix = prefix_parts(a, b, h);

    Wave<TYPE, D, 1> w;
    w.clear();
    const uint16_t* q = query<D, TOK>(a, v, h, min(lane & 15, group - 1));
#pragma unroll
    for (int k = 0; k < D / 32; ++k)
        w.q[0][k] = *reinterpret_cast<const bf16x8_t*>(q + key_dim<TYPE, D>(k, lane >> 4));
    if (s.chunks > 0) {  // (else t0 may be past what an int holds)
        if (s.start > 0) page = Wave<TYPE, D, 1>::template pages_of<W>(a.c, pages, t0, t1, wave, lane);
        if constexpr (TOK) {
            // the lane's column, the first and the last
            const int list_first = a.own.first ? max(a.own.first[(int64_t)b * a.c.heads + h], 0) : 0;
            const int token = min((lane & 15) / a.heads, a.cut - 1);
            auto first_of = [&](int token) {
                return window > 0 ? max(list_first, base + token0 + token + 1 - window) : list_first;
            };
            const typename Wave<TYPE, D, 1>::Seen seen{
                first_of(token), min(base + token0 + token + 1, t1), first_of(a.cut - 1),
                min(base + token0 + 1, t1), s.first, t1};
            w.template run_steps<false, W>(a.c, a.pool, page, t0, t1, wave, lane,
                                           [&](Tile<TYPE, D>& t, int at) { w.step_at(t, at, seen, lane); });
        } else {
            w.template run<true, W>(a.c, a.pool, page, t0, t1, s.first, wave, lane);
        }
    }

    int* counter = a.arrived + (WITH ? lh : rank);
    // the only part that is still missing, or the only one at all
    if (WITH && tid == 0)
        *flags = chunks == 1 && (prefix == 0 || __hip_atomic_load(counter, __ATOMIC_RELAXED,
                                                                  __HIP_MEMORY_SCOPE_AGENT) ==
                                                    group * prefix);
    bool alone = chunks == 1;
    join_waves<W>(w, lds, group, wave, lane, [&](int col, int d, f32x4_t v, float m, float sum) {
        if (WITH) alone = *flags;  // (there is a barrier before)
        if (alone) {
            Sum all{v, m, sum};
            add_prefix<D, WITH>(a, all, row0 + col, prefix, d);
            write_out(a, out_row<TOK>(a, lh, col), d, D, all.v, all.m, all.s);
        } else {
            const int64_t slot = (row0 + col) * a.own_parts + chunk;
            publish4(a.part + slot * D + d, v);
            if (d == 0) publish(a.ml + slot, __float_as_uint(m), __float_as_uint(sum));
        }
    });
    if (WITH) alone = *flags;
    if (alone) {
        if (WITH && prefix > 0 && tid == 0)
            __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return;
    }
    // every published word has left before the list's part counts as arrived
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    together<W>();
    if (tid == 0) *flags = arrive(counter, group, group * (chunks + (WITH ? prefix : 0)));
    together<W>();
    if (!*flags) return;
    for (int i = tid; i < group * (D / 4); i += 64 * W)
        finish<D, WITH, TOK>(a, lh, chunks, prefix, i / (D / 4), i % (D / 4) * 4);
}

// A shared list of few columns (members * group of them): one block per (list, kv
// head, chunk) and tile of 16 columns; a block goes on to every `tiles`-th tile.
struct SharedLds {
    int row_of[17], found[kWaves];
    int chunks[16];       // of the members' own lists
    int done[16], count;  // members (of the tile) whose parts are all there
};
template <int TYPE, int D, bool TOK>
__device__ __forceinline__ void shared_block(const AttnCall& a, int block, float* lds, SharedLds& ints) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lists = a.shared.lists * a.c.heads;
    const int per_tile = lists * a.shared_parts;
    const int tile0 = block / per_tile, item = block % per_tile;
    const int lh = item % lists, chunk = item / lists;
    const int list = lh / a.c.heads, h = lh % a.c.heads, group = a.c.group;
    const Span s = span_of(a.shared, a.c.ptok, lh, a.shared_chunk);
    const int32_t* pages = a.shared.pages + (int64_t)lh * a.shared.max_pages;
    int* row_of = ints.row_of;

    for (int tile = tile0;; tile += a.tiles) {
        const int c0 = tile * 16, rank0 = c0 / group, rank1 = (c0 + 15) / group + 1;
        const int members = find_members<kWaves, TOK>(a, list, rank0, rank1, row_of, ints.found, tid);
        const int cols = min(16, members * group - c0);
        if (cols <= 0 || chunk >= s.chunks) return;  // (the length is not waited for alone)
        const int t0 = s.start + chunk * a.shared_chunk, t1 = min(s.len, t0 + a.shared_chunk);
        // lane i: the member of rank rank0 + i, its columns in the tile
        auto columns = [&] {
            return min(c0 + cols, (rank0 + lane + 1) * group) - max(c0, (rank0 + lane) * group);
        };
        Wave<TYPE, D, 1> w;
        w.clear();
        load_queries<TYPE, D, TOK>(a, h, c0 + min(lane & 15, cols - 1), rank0, row_of, lane, w.q[0]);
        if (wave == 0 && columns() > 0)
            ints.chunks[lane] = max(own_chunks<TOK>(a, row_of[lane], h), 1);
        const int page = Wave<TYPE, D, 1>::template pages_of<kWaves>(a.c, pages, t0, t1, wave, lane);
        w.template run<false, kWaves>(a.c, a.pool, page, t0, t1, s.first, wave, lane);
        join_waves<kWaves>(w, lds, cols, wave, lane, [&](int n, int d, f32x4_t v, float m, float sum) {
            const int64_t slot = shared_slot(a, h, c0 + n, rank0, row_of, chunk);
            publish4(a.shared_part + slot * D + d, v);
            if (d == 0) publish(a.shared_ml + slot, __float_as_uint(m), __float_as_uint(sum));
        });
        if (a.lists == 0) continue;  // a later launch joins
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (wave == 0) {
            const int mine = columns();
            const bool last = mine > 0 && arrive(a.arrived + row_of[lane] * a.c.heads + h, mine,
                                                 group * (ints.chunks[lane] + s.chunks));
            const uint64_t mask = __builtin_amdgcn_ballot_w64(last);
            if (last) ints.done[__builtin_popcountll(mask & ((1ull << lane) - 1))] = lane;
            if (lane == 0) ints.count = __builtin_popcountll(mask);
        }
        __syncthreads();
        const int per = group * (D / 4);
        for (int i = tid; i < ints.count * per; i += kThreads) {
            const int n = ints.done[i / per], k = i % per;
            finish<D, true, TOK>(a, row_of[n] * a.c.heads + h, ints.chunks[n], s.chunks, k / (D / 4),
                            k % (D / 4) * 4);
        }
        __syncthreads();  // row_of and done are written again
    }
}

// Wavefronts of a SIMD that the kernels' registers allow; the compiler passes the
// limits by a few registers if it isn't held to them.
template <int TYPE, int D>
constexpr int own_waves() { return D == 64 || TYPE == kFp4 ? 4 : TYPE == kInt8 ? 3 : 2; }
template <int TYPE, int D>
constexpr int with_shared_waves() { return D == 64 ? 4 : TYPE == kBf16 ? 2 : 3; }

template <int TYPE, int D, int W, bool TOK>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(own_waves<TYPE, D>())))
void k_attn_own(AttnCall a) {
    extern __shared__ __align__(16) float lds[];  // join_bytes(D, group)
    __shared__ int flags[kWaves];
    own_block<TYPE, D, false, W, TOK>(a, blockIdx.x, lds, flags);
}

// Shared lists of few columns and the rows' own ones in one launch: the shared ones'
// blocks, which have more to compute, start first, and the rows' fill the CUs beside
// them.  Whichever brings the last part of a row's list joins them all.  (64 rows on a
// prefix of 2048 INT8 tokens with own lists of 64 to 1024, 32 heads: 55 us; in two
// launches, with the prefix's parts read by the second, 62.)
template <int TYPE, int D, int W, bool TOK>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(with_shared_waves<TYPE, D>())))
void k_attn_with_shared(AttnCall a) {
    extern __shared__ __align__(16) float lds[];  // join_bytes(D, 16)
    __shared__ SharedLds ints;
    const int block = blockIdx.x;
    if (block < a.shared_blocks) shared_block<TYPE, D, TOK>(a, a.shared_block0 + block, lds, ints);
    else own_block<TYPE, D, true, W, TOK>(a, block - a.shared_blocks, lds, ints.found);
}

// Which values of a step's operands are no finite numbers: any, of each of the four wavefronts
// that convert them, and where (of a wavefront that has none nothing is written).
template <int TYPE, int D>
struct Odd {
    __align__(16) uint32_t any[4];
    u32x4_t of[TYPE == kInt8 ? 1 : D / 16][64];
};

// What a wavefront of k_attn_shared_wide does of a step's operands: the first four
// wavefronts convert those of the keys, the others those of the values, D / 64 each
// (FP4 values: two), which lie together in the page.  One load for all of them, at
// an address that follows from the token and a number per lane, so that it needs no
// branch: a load that only some wavefronts do is waited for where the branch ends.
template <int TYPE, int D>
struct Share {
    using T = Tile<TYPE, D>;
    static constexpr int KS = D / 32, N = D / 64, kRow = T::kRow;
    static constexpr int kWords = TYPE == kBf16 ? 4 * N : TYPE == kInt8 ? 2 * N : 2;
    u32x4_t raw[(kWords + 3) / 4];
    u32x4_t scales;  // INT8: of the lane's eight tokens
    u32x2_t powers;  // FP4: exponents
    int off, more, scale_off, scale_step;
    int slot;     // of its first operand
    bool values;

    __device__ __forceinline__ Share(const PagedDims& c, int wave, int lane) {
        const int i = lane & 15, quarter = lane >> 4, w = wave & 3;
        values = wave >= 4;
        more = 0;
        scale_step = 2;
        if (!values) {
            const int row = 8 * (i >> 2) + 4 * (w >> 1) + (i & 3), part = w & 1;
            slot = (w >> 1) * KS + part * N;
            off = row * kRow;
            if constexpr (TYPE == kBf16) {
                off += (4 * N * part + quarter) * 16;
                more = 64;
            }
            if constexpr (TYPE == kInt8) {
                off += N == 2 ? (4 * part + quarter) * 16 : quarter * 16 + part * 8;
                scale_off = c.ks_off + 16 * quarter;
            }
            if constexpr (TYPE == kFp4) {  // eight bytes that hold the row's exponents
                off += N == 2 ? quarter * 16 + part * 8 : quarter * 8;
                scale_step = D / 32;
                scale_off = c.ks_off + (row * scale_step & ~7);
                more = (row * scale_step & 7) + (N == 2 ? quarter : quarter >> 1);
            }
        } else {
            const int pair = N == 2 ? w : w & 1;
            slot = 2 * KS + (TYPE == kFp4 ? 2 * pair : w * N);
            off = c.v_off + quarter * (8 * kRow);
            if constexpr (TYPE == kBf16) {
                off += (16 * N * w + i) * 16;
                more = 256;
            }
            if constexpr (TYPE == kInt8) {
                off += N == 2 ? (16 * w + i) * 16 : (16 * (w >> 1) + i) * 16 + (w & 1) * 8;
                scale_off = c.vs_off + 16 * quarter;
            }
            if constexpr (TYPE == kFp4) {
                const int load = pair >> 1;
                off += (16 * load + i) * 16 + (pair & 1) * 8;
                scale_step = 1;
                scale_off = c.vs_off + (2 * load + (i >> 3)) * c.ptok + 8 * quarter;
            }
        }
    }

    __device__ __forceinline__ void fetch(const char* page, int tp) {
        const char* from = page + tp * kRow + off;
        if constexpr (kWords == 2) {
            const u32x2_t w = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(from));
            raw[0][0] = w[0], raw[0][1] = w[1];
        } else {
            raw[0] = nt16(from);
            if constexpr (kWords == 8) raw[1] = nt16(from + more);
        }
        const char* s = page + tp * scale_step + scale_off;
        if constexpr (TYPE == kInt8) scales = *reinterpret_cast<const u32x4_t*>(s);
        if constexpr (TYPE == kFp4) powers = *reinterpret_cast<const u32x2_t*>(s);
    }

    // Its operands, into the lane's places of the slots; values that are not seen as
    // zeros (INT8: with scales of zero, which go to slot `at_scales` and the next).
    // odd, if given: values that are no finite numbers are taken out, all ones in their places
    // go to odd's slots, and odd->any says whether there are some.
    __device__ __forceinline__ void convert(u32x4_t (*to)[64], int at_scales, bool partial,
                                            uint32_t seen, int wave, int lane,
                                            Odd<TYPE, D>* odd = nullptr) {
        if (values && partial) {
            if constexpr (TYPE == kBf16) {
#pragma unroll
                for (u32x4_t& w : raw) w = T::blank16(w, seen);
            }
            if constexpr (TYPE == kInt8) scales = T::blank16(scales, seen);
            if constexpr (TYPE == kFp4) powers = T::blank8(powers, seen);
        }
        if constexpr (TYPE == kBf16) {
            if (odd && values) take_out<N>(raw, *odd, wave, lane);
#pragma unroll
            for (int x = 0; x < N; ++x) to[slot + x][lane] = raw[x];
        } else if constexpr (TYPE == kInt8) {
#pragma unroll
            for (int x = 0; x < N; ++x) {
                uint32_t o[4];
                int8_pack(raw[0][2 * x], o);
                int8_pack(raw[0][2 * x + 1], o + 2);
                to[slot + x][lane] = u32x4_t{o[0], o[1], o[2], o[3]};
            }
            if ((wave & 3) == 0) to[at_scales + values][lane] = scales;
        } else if (values) {
            bf16x8_t o[2];
            fp4_pair(raw[0][0], raw[0][1], powers, o);
            u32x4_t w[2]{__builtin_bit_cast(u32x4_t, o[0]), __builtin_bit_cast(u32x4_t, o[1])};
            if (odd) take_out<2>(w, *odd, wave, lane);
            to[slot][lane] = w[0];
            to[slot + 1][lane] = w[1];
        } else {
            const uint64_t all = (uint64_t)whole(powers[1]) << 32 | whole(powers[0]);
            const uint32_t e = (uint32_t)(all >> (8 * more)) & 0xffu;
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const uint32_t w = N == 2 ? raw[0][x] : (wave & 1) ? raw[0][1] : raw[0][0];
                to[slot + x][lane] = __builtin_bit_cast(u32x4_t, key_operand<kFp4>(u32x4_t{w, 0, 0, 0}, e, 0));
            }
        }
    }

    template <int M>
    __device__ __forceinline__ void take_out(u32x4_t* w, Odd<TYPE, D>& odd, int wave, int lane) {
        uint32_t top = 0;
#pragma unroll
        for (int x = 0; x < M; ++x) top = top_of(top, w[x]);
        const bool any = any_odd(top);
        if (lane == 0) odd.any[wave & 3] = any;
        if (__builtin_expect(!any, 1)) return;
#pragma unroll
        for (int x = 0; x < M; ++x) {
            const u32x4_t none = odd_of(w[x]);
            odd.of[slot - 2 * KS + x][lane] = none;
            w[x] &= ~none;
        }
    }
};

// A shared list of many columns: the W wavefronts of a block take NB * 16 columns
// each and the same tokens, whose operands they convert once for all, a share each,
// into LDS in the order in which the lanes read them: those of the next step while
// one is computed, from loads of the step before it.  256 columns of 2 x 8 lists of
// 16384 FP4 tokens: 83 us, 0.83 PFLOP/s on the matrix cores (K once, V with three
// pieces), which are busy for a third of the time; the vector ALU's share, the
// exponentials and the weights' pieces, is 40 %, and the two meet at a step's barrier.
template <int TYPE, int D, bool TOK>
__global__ __launch_bounds__(kWideThreads) void k_attn_shared_wide(AttnCall a) {
    using T = Tile<TYPE, D>;
    constexpr int W = kWideWaves, COLS = kWideCols, NB = COLS / (16 * W);
    constexpr int KS = D / 32, DB = D / 16, VX = DB / T::VN;
    constexpr int kScales = 2 * KS + DB;  // INT8: scales lie behind the operands
    constexpr int kSlots = kScales + (TYPE == kInt8 ? 2 : 0);
    __shared__ u32x4_t operands[2][kSlots][64];  // of two steps in turn
    __shared__ int row_of[COLS + 1];
    __shared__ int found[W];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lists = a.shared.lists * a.c.heads;
    const int per_tile = lists * a.shared_parts;
    const int block = a.shared_block0 + blockIdx.x;
    const int tile0 = block / per_tile, item = block % per_tile;
    const int lh = item % lists, chunk = item / lists;
    const int list = lh / a.c.heads, h = lh % a.c.heads, group = a.c.group;
    const Span s = span_of(a.shared, a.c.ptok, lh, a.shared_chunk);
    if (chunk >= s.chunks) return;
    const int t0 = s.start + chunk * a.shared_chunk, t1 = min(s.len, t0 + a.shared_chunk);
    // lane n: page of step n of the chunk, which has 64 at most
    int page = -1;
    if (t0 + lane * kStep < t1)
        page = a.shared.pages[(int64_t)lh * a.shared.max_pages + ((t0 + lane * kStep) >> a.c.pshift)];
    const uint64_t steps = __builtin_amdgcn_ballot_w64(page >= 0 && page < a.c.num_pages);
    Share<TYPE, D> share(a.c, wave, lane);

    for (int tile = tile0;; tile += a.tiles) {
        // the members that the tile's columns belong to: ranks [rank0, rank1)
        const int c0 = tile * COLS, rank0 = c0 / group, rank1 = (c0 + COLS - 1) / group + 1;
        const int members = find_members<W, TOK>(a, list, rank0, rank1, row_of, found, tid);
        const int cols = min(COLS, members * group - c0);  // of this tile
        if (cols <= 0) return;
        const int w0 = wave * 16 * NB;  // the wavefront's first column
        Wave<TYPE, D, NB> w;
        w.clear();
#pragma unroll
        for (int n = 0; n < NB; ++n)
            load_queries<TYPE, D, TOK>(a, h, c0 + min(w0 + 16 * n + (lane & 15), cols - 1), rank0, row_of,
                                  lane, w.q[n]);
        auto part_of = [&](int n, uint32_t* seen) {  // step n: is it attended in part
            const int at = t0 + n * kStep;
            const bool partial = at < s.first || at + kStep > t1;
            *seen = partial ? seen_of(at, s.first, t1, lane) : 0xffu;
            return partial;
        };
        if (steps) {
            uint64_t to_fetch = steps;
            int held = 0;  // the step whose loads are held
            auto fetch = [&] {  // past the last step, that one again
                if (to_fetch) held = __builtin_ctzll(to_fetch);
                to_fetch &= to_fetch - 1;
                share.fetch(a.pool + __builtin_amdgcn_readlane(page, held) * a.c.page_bytes,
                            (t0 + held * kStep) & (a.c.ptok - 1));
            };
            auto produce = [&](int into) {
                uint32_t seen;
                const bool partial = part_of(held, &seen);
                share.convert(operands[into], kScales, partial, seen, wave, lane);
                fetch();
            };
            fetch();
            produce(0);
            __syncthreads();
            int buf = 0;
            for (uint64_t todo = steps; todo; todo &= todo - 1, buf ^= 1) {
                produce(buf ^ 1);
                if (w0 < cols) {
                    uint32_t seen;
                    const bool partial = part_of(__builtin_ctzll(todo), &seen);
                    u32x4_t ks{}, vs{};
                    if constexpr (TYPE == kInt8) {
                        ks = operands[buf][kScales][lane];
                        vs = operands[buf][kScales + 1][lane];
                    }
                    w.step([&](int u, int k) {
                               return __builtin_bit_cast(bf16x8_t, operands[buf][u * KS + k][lane]);
                           },
                           [&](int j, bf16x8_t* v) {
#pragma unroll
                               for (int x = 0; x < VX; ++x)
                                   v[x] = __builtin_bit_cast(
                                       bf16x8_t, operands[buf][2 * KS + j * VX + x][lane]);
                           },
                           ks, vs, partial, [&](int) { return seen; });
                }
                __syncthreads();
            }
        }

        // the columns' parts, from where they are
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const int at = w0 + 16 * n + (lane & 15);
            const float sum = over_quarters(w.sum[n], [](float x, float y) { return x + y; });
            if (at < cols) {
                const int64_t slot = shared_slot(a, h, c0 + at, rank0, row_of, chunk);
                w.to_row(n, lane >> 4, a.shared_part + slot * D);
                if (lane < 16) a.shared_ml[slot] = f32x2_t{w.m[n], sum};
            }
        }
        __syncthreads();  // row_of is written again
    }
}

// Cuts of many columns (the pieces of a prompt): a block takes a cut's, up to 128, and the
// tokens of a chunk of its list, as k_attn_shared_wide does; what a column sees ends with
// its own token, so a wavefront leaves out the steps that none of its columns sees.
// Outputs of a list that has one chunk and shares nothing are written here, the others'
// parts are added up by k_attn_join.
//
// Few lists, whose lengths only the device knows: every block counts the tokens of all,
// cuts them into chunks of a length that leaves each CU about one, and takes every
// gridDim-th of these.  (A grid of every chunk that there might be instead, most of them
// none: the others lie two on a CU beside CUs that have none, 28 us instead of 20 when both
// were there; by a trace of the present build 24.5.)
constexpr int kFewCuts = kWideThreads;

// A cut and what is known of its list.
struct CutItem {
    int real, b, h, token0, n;    // n tokens from token0 of row b on, the list's number
    int base, window, list_first; // tokens before row b's new ones, the window, the list's `first`
    __device__ __forceinline__ CutItem() {}
    // Cut number t: the last ones of all rows first, of lists in their order.
    __device__ __forceinline__ CutItem(const AttnCall& a, int t) {
        const int at = place(a, t);
        real = a.own.order ? min(max(a.own.order[at], 0), a.own.lists / a.cuts * a.c.heads - 1) : at;
        base = list_len(a.own, a.c.ptok, real);
        window = a.window ? a.window[real] : 0;
        list_first = a.own.first ? max(a.own.first[real], 0) : 0;
        row(a);
        n = Cut(a, b * a.cuts + token0 / a.cut).n;
    }
    __device__ __forceinline__ int place(const AttnCall& a, int t) {
        const int lists = a.own.lists / a.cuts * a.c.heads, from_last = t / lists;
        token0 = (a.cuts - 1 - from_last) * a.cut;
        return t - from_last * lists;
    }
    __device__ __forceinline__ void row(const AttnCall& a) {
        b = real / a.c.heads;
        h = real - b * a.c.heads;
    }
    __device__ __forceinline__ int first_of(int token) const {
        return window > 0 ? max(list_first, base + token0 + token + 1 - window) : list_first;
    }
    // Its span, in as many chunks as `most` tokens make, of about equal length: *chunk tokens.
    __device__ __forceinline__ Span span(const AttnCall& a, int most, int* chunk) const {
        Span s;
        s.first = first_of(0);
        s.len = min(base + token0 + n, a.own.max_pages * a.c.ptok);
        s.start = s.first & ~(kStep - 1);
        s.chunks = 0;
        *chunk = kStep;
        if (s.len > s.first) {
            const int tokens = s.len - s.start, chunks = (tokens + most - 1) / most;
            *chunk = ((tokens + chunks - 1) / chunks + kStep - 1) / kStep * kStep;
            s.chunks = (tokens + *chunk - 1) / *chunk;
        }
        return s;
    }
};

struct Plan {
    int ends[kFewCuts];  // chunks of the cuts up to this one
    int sums[kWideWaves];
    int real[kFewCuts], n[kFewCuts], base[kFewCuts], window[kFewCuts], first[kFewCuts];
    __device__ __forceinline__ CutItem item(const AttnCall& a, int t) const {
        CutItem c;
        c.place(a, t);
        c.real = real[t];
        c.n = n[t];
        c.base = base[t];
        c.window = window[t];
        c.list_first = first[t];
        c.row(a);
        return c;
    }
};

// Fills p; the number of chunks of all cuts, and the tokens of one.
__device__ __forceinline__ int plan_chunks(const AttnCall& a, Plan& p, int* chunk) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool is = tid < a.own.lists * a.c.heads;
    const CutItem c(a, is ? tid : 0);
    int even;
    const Span s = c.span(a, kSharedMost, &even);
    // (a sum that 32 bits hold; longer lists are cut into as many parts as there may be)
    uint32_t sum = is && c.n > 0 && s.chunks > 0 ? min((uint32_t)(s.len - s.start), 1u << 22) : 0;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) sum += __shfl_xor(sum, o);
    if (lane == 0) p.sums[wave] = (int)sum;
    p.real[tid] = c.real;
    p.n[tid] = c.n;
    p.base[tid] = c.base;
    p.window[tid] = c.window;
    p.first[tid] = c.list_first;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < kWideWaves; ++w) sum += (uint32_t)p.sums[w];
    // a quarter more than each CU's share, so that lists of about equal length stay whole
    const uint32_t want = (sum + sum / 4) / kCutBlocks;
    *chunk = max((int)((want + kUnit - 1) / kUnit * kUnit), a.own_chunk);
    int up = is && c.n > 0 ? max(1, c.span(a, *chunk, &even).chunks) : 0;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int y = __shfl_up(up, o);
        if (lane >= o) up += y;
    }
    __syncthreads();
    if (lane == 63) p.sums[wave] = up;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWideWaves; ++w)
        if (w < wave) up += p.sums[w];
    p.ends[tid] = up;
    __syncthreads();
    return p.ends[kFewCuts - 1];
}

// Operands of two steps in turn; INT8: the scales lie behind them.
template <int TYPE, int D>
using CutOperands = u32x4_t[2][2 * (D / 32) + D / 16 + (TYPE == kInt8 ? 2 : 0)][64];

template <int TYPE, int D>
__device__ __forceinline__ void cut_block(const AttnCall& a, const CutItem& c, int chunk,
                                          CutOperands<TYPE, D>& operands, Odd<TYPE, D>* odd) {
    using T = Tile<TYPE, D>;
    constexpr int W = kWideWaves, NB = kCutCols / (16 * W);
    constexpr int KS = D / 32, DB = D / 16, VX = DB / T::VN;
    constexpr int kScales = 2 * KS + DB;  // INT8: scales lie behind the operands
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (c.n <= 0) return;
    int most;
    const Span s = c.span(a, a.own_chunk, &most);
    if (chunk >= max(s.chunks, 1)) return;
    const int t0 = s.start + chunk * most, t1 = min(s.len, t0 + most);
    // lane n: page of step n of a piece of the chunk, which has 64
    auto pages_of = [&](int begin) {
        const int at = begin + lane * kStep;
        return s.chunks > 0 && at < t1
                   ? a.own.pages[(int64_t)c.real * a.own.max_pages + (at >> a.c.pshift)] : -1;
    };
    int page = pages_of(t0);

    const int cols = c.n * a.heads;
    const int w0 = wave * 16 * NB;  // the wavefront's first column
    auto end_of = [&](int token) { return min(c.base + c.token0 + token + 1, t1); };
    auto token_of = [&](int col) { return min(col, cols - 1) / a.heads; };
    const int low = token_of(w0), high = token_of(w0 + 16 * NB - 1);
    const int any_first = c.first_of(low), any_end = end_of(high);
    const int all_first = c.first_of(high), all_end = end_of(low);
    // steps that some columns of the cut may attend and others not: those that end past this
    const int all_see = c.window > 0 ? 0 : end_of(0);
    Wave<TYPE, D, NB> w;
    w.clear();
    int first[NB], end[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int col = min(w0 + 16 * n + (lane & 15), cols - 1);
        const int token = token_of(col);
        first[n] = c.first_of(token);
        end[n] = end_of(token);
        const uint16_t* q = a.q + c.b * a.q_stride + (c.token0 + token) * a.q_token +
                            (c.h * a.heads + col - token * a.heads) * D;
#pragma unroll
        for (int k = 0; k < KS; ++k)
            w.q[n][k] = *reinterpret_cast<const bf16x8_t*>(q + key_dim<TYPE, D>(k, lane >> 4));
    }
    Share<TYPE, D> share(a.c, wave, lane);
    for (int begin = t0;;) {
        const uint64_t steps = __builtin_amdgcn_ballot_w64(page >= 0 && page < a.c.num_pages);
        uint64_t to_fetch = steps;
        int held = 0;  // the step whose loads are held
        auto fetch = [&] {  // past the last step, that one again
            if (to_fetch) held = __builtin_ctzll(to_fetch);
            to_fetch &= to_fetch - 1;
            share.fetch(a.pool + __builtin_amdgcn_readlane(page, held) * a.c.page_bytes,
                        (begin + held * kStep) & (a.c.ptok - 1));
        };
        auto produce = [&](int into) {
            const int tk = begin + held * kStep;
            const bool partial = tk < s.first || tk + kStep > t1;
            const uint32_t seen = partial ? seen_of(tk, s.first, t1, lane) : 0xffu;
            share.convert(operands[into], kScales, partial, seen, wave, lane,
                          tk + kStep > all_see ? &odd[into] : nullptr);
            fetch();
        };
        auto consume = [&](int buf, int n) {
            const int tk = begin + n * kStep;
            if (w0 >= cols || tk >= any_end || tk + kStep <= any_first) return;
            const bool partial = tk < all_first || tk + kStep > all_end;
            uint32_t seen[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n)
                seen[n] = partial ? seen_of(tk, first[n], end[n], lane) : 0xffu;
            u32x4_t ks{}, vs{};
            if constexpr (TYPE == kInt8) {
                ks = operands[buf][kScales][lane];
                vs = operands[buf][kScales + 1][lane];
            }
            if constexpr (TYPE == kInt8) {
                static_assert(NB == 1, "one tile of columns a wavefront");
                if (partial) vs = T::blank16(vs, seen[0]);
            } else if (tk + kStep > all_see) {
                const u32x4_t any = *reinterpret_cast<const u32x4_t*>(odd[buf].any);
                if (__builtin_expect(__builtin_amdgcn_readfirstlane(any[0] | any[1] | any[2] | any[3]), 0)) {
                    constexpr int kOf = TYPE == kFp4 ? 2 : D / 64;  // operands of a wavefront
#pragma unroll
                    for (int j = 0; j < DB; ++j) {
                        __builtin_amdgcn_sched_barrier(0);  // (in the registers of one at a time)
                        if (__builtin_amdgcn_readfirstlane(any[j / kOf]))
                            w.spoil(odd[buf].of[j][lane], seen[0], j);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            w.step([&](int u, int k) {
                       return __builtin_bit_cast(bf16x8_t, operands[buf][u * KS + k][lane]);
                   },
                   [&](int j, bf16x8_t* v) {
#pragma unroll
                       for (int x = 0; x < VX; ++x)
                           v[x] = __builtin_bit_cast(bf16x8_t,
                                                     operands[buf][2 * KS + j * VX + x][lane]);
                   },
                   ks, vs, partial, [&](int n) { return seen[n]; });
        };
        if (steps) {
            fetch();
            produce(0);
            __syncthreads();
            int buf = 0;
            for (uint64_t todo = steps; todo; todo &= todo - 1, buf ^= 1) {
                produce(buf ^ 1);
                consume(buf, __builtin_ctzll(todo));
                __syncthreads();
            }
        }
        if (t1 - begin <= kSharedMost) break;
        begin += kSharedMost;
        page = pages_of(begin);
    }

    const bool direct = s.chunks <= 1 && prefix_parts(a, c.b, c.h) == 0;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int col = w0 + 16 * n + (lane & 15);
        const float sum = over_quarters(w.sum[n], [](float x, float y) { return x + y; });
        if (col >= cols) continue;
        const int token = col / a.heads;
        if (direct) {
            const int64_t row = (((int64_t)c.b * a.tokens + c.token0 + token) * a.c.heads + c.h) * a.heads +
                                col - token * a.heads;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int j = 0; j < DB; ++j) w.acc[n][j] *= inv;
            w.to_row(n, lane >> 4, a.out + row * D);
            if (a.lse && lane < 16)
                a.lse[row] = sum == 0.f ? -INFINITY
                                        : (w.m[n] + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
        } else {
            const int lh = (c.b * a.cuts + c.token0 / a.cut) * a.c.heads + c.h;
            const int64_t slot = ((int64_t)lh * a.c.group + col) * a.own_parts + chunk;
            w.to_row(n, lane >> 4, a.part + slot * D);
            if (lane < 16) a.ml[slot] = f32x2_t{w.m[n], sum};
        }
    }
}

template <int TYPE, int D, bool FEW>
__global__ __launch_bounds__(kWideThreads) void k_attn_cut_wide(AttnCall a, int* chunk_of_all) {
    __shared__ CutOperands<TYPE, D> operands;
    __shared__ __align__(16) Odd<TYPE, D> odd[2];
    if constexpr (FEW) {
        __shared__ Plan plan;
        int chunk;
        const int all = plan_chunks(a, plan, &chunk);
        a.own_chunk = chunk;
        if (blockIdx.x == 0 && threadIdx.x == 0) *chunk_of_all = chunk;
        for (int item = blockIdx.x; item < all; item += gridDim.x) {
            int t = 0;  // the first cut whose chunks end behind it
#pragma unroll
            for (int o = kFewCuts / 2; o > 0; o /= 2)
                if (plan.ends[t + o - 1] <= item) t += o;
            t = __builtin_amdgcn_readfirstlane(t);
            cut_block<TYPE, D>(a, plan.item(a, t), item - (t ? plan.ends[t - 1] : 0), operands, odd);
            __syncthreads();  // the operands are written again
        }
    } else {
        const int item = a.list0 + blockIdx.x, cuts = a.own.lists * a.c.heads;
        cut_block<TYPE, D>(a, CutItem(a, item % cuts), item / cuts, operands, odd);
    }
}

// Adds up the parts of cuts, of their own lists and of the prefixes that they share: a
// thread for each four dims of an output.
template <int D>
__global__ __launch_bounds__(kThreads) void k_attn_join(AttnCall a, const int* chunk_of_all) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t row = i / (D / 4) + a.row0;
    const int d = (int)(i % (D / 4)) * 4;
    const int lh = (int)(row / a.c.group), col = (int)(row - (int64_t)lh * a.c.group);
    if (chunk_of_all) a.own_chunk = *chunk_of_all;
    if (lh >= a.own.lists * a.c.heads) return;
    const int v = lh / a.c.heads, h = lh - v * a.c.heads;
    const Cut cut(a, v);
    if (col >= cut.n * a.heads) return;
    CutItem c;
    c.real = cut.b * a.c.heads + h;
    c.token0 = cut.token0;
    c.n = cut.n;
    c.base = list_len(a.own, a.c.ptok, c.real);
    c.window = a.window ? a.window[c.real] : 0;
    c.list_first = a.own.first ? max(a.own.first[c.real], 0) : 0;
    int most;
    const int chunks = max(c.span(a, a.own_chunk, &most).chunks, 1);
    const int prefix = prefix_parts(a, cut.b, h);
    if (chunks == 1 && prefix == 0) return;  // there already
    Sum all;
    const int64_t slot = row * a.own_parts;
    all.add_parts(
        chunks, [&](int j) { return *reinterpret_cast<const f32x4_t*>(a.part + (slot + j) * D + d); },
        [&](int j) { return a.ml[slot + j]; });
    add_prefix<D, false>(a, all, row, prefix, d);
    write_out(a, out_row<true>(a, lh, col), d, D, all.v, all.m, all.s);
}

// ------------------------------------------------------------------- launch
constexpr int kCus = 256;

// Tokens of a chunk of lists of up to max_len tokens, of which `want` chunks are wanted.
// Own lists: about two blocks per CU for few lists, else short enough that blocks
// that are done early find others (512 lists of 250-4000 INT8 tokens: at most 768 tokens
// 44.9 us, 1024 44.4, 1536 46, 2048 52; 256 of 1500-16384 for 4 heads 96, 93, 92, 96, FP4
// 59, 57, 58, 54; 32 lists of 98-2480 tokens: 256 tokens 8.5 us, 512 11; 128, a step of a
// wavefront, 15).
// Shared lists: as many blocks as there are CUs, beside which own lists find room (64
// rows on a prefix of 2048 INT8 tokens: 256 blocks 54.3 us, 384 53.4, 512 55.1; the own
// lists' blocks first 70).
constexpr int kLeastChunk = 2 * kUnit, kOwnMost = 8 * kUnit;
int chunk_of(int max_len, int64_t want, int most) {
    const int64_t chunk = ((max_len + want - 1) / want + kUnit - 1) / kUnit * kUnit;
    return (int)std::min<int64_t>(std::max<int64_t>(chunk, kLeastChunk), most);
}

int parts_of(int max_len, int chunk) { return (max_len + chunk - 1) / chunk; }

// Parts that no smaller max_len has more of, if chunks of `least` tokens are made
// longer only once there are `want` of them, up to `most` tokens: a workspace that is
// large enough for a length is so for all shorter ones.
int64_t most_parts(int max_len, int64_t want, int least, int most) {
    return std::max<int64_t>(1, std::max<int64_t>(std::min<int64_t>(parts_of(max_len, least), want),
                                                  parts_of(max_len, most)));
}

// Parts that the lists of few cuts of many columns have at most.
constexpr int kCutParts = 16;
// Tokens of a block's chunk at most, pages in the lanes of four wavefronts: where lists are
// so many that a CU has several blocks, however long, parts would only take space.
constexpr int kOwnLongest = 64 * kUnit, kManyLists = 16 * kCus;

struct Split {
    int own_chunk, own_parts, shared_chunk, shared_parts;
    // Shared lists: which kernel takes them, and the column tiles of one in the grid:
    // as many as its share of all columns takes; a list with more has its blocks go
    // round.  Tiles of 16 columns read and convert the tokens for each tile, but run
    // beside the own lists; the wide kernel does for 256 columns, with a barrier per
    // step, and takes 20 us and more however short the prefix is.  Which is faster
    // follows from the work, in blocks of 16 columns and 256 tokens.  Time of the wide
    // kernel over that of tiles of 16 by columns of a prefix, d = 128, 1 or 2 prefixes of
    // 512 to 16384 tokens, 2 to 32 heads in groups of 1 to 16, own lists of up to 64 or 576
    // tokens, all from memory:
    //         columns  blocks 3072   4096       6144       8192       12288      16384
    //   BF16     96     .81 - 1.14              .79 -  .96             .42 -  .66
    //           128                .80 -  .99              .63 -  .90             .33 - .61
    //           256                .85 - 1.11              .63 -  .83             .47 - .81
    //           384    1.04 - 1.18              .82 - 1.01             .67 -  .82
    //   INT8     96     .97 - 1.15             1.12 - 1.24             .89 -  .97
    //           128                .98 - 1.22              .91 - 1.06             .71 - .85
    //           256                .98 - 1.38              .83 -  .99             .68 - .87
    //           384    1.00 - 1.34             1.03 - 1.20             .87 -  .97
    //   FP4     128               1.21 - 1.36             1.04 - 1.18             .96 - 1.03
    //           256               1.09 - 1.72             1.06 - 1.12             .85 -  .93
    //           384    1.17 - 1.62             1.01 - 1.44            1.04 - 1.10
    // (FP4 of 96 columns 1.2 however many blocks, 192 of 24576 blocks .87 - .93; 256 columns of
    // FP4 over 2 x 8 lists of 16384: 109 us in tiles and 96 wide, over 8 lists 60 and 68.
    // BF16 of 3072 blocks may go either way: 96 columns of 8 heads over 16384 tokens 55 and
    // 50, of 16 heads over 8192 57 and 65.)
    bool wide;
    int tiles;
    // Own lists: a wavefront each, not a block, where they are many and short, so that
    // what a list costs however short it is (four loads that wait for each other) is paid
    // for four at a time.  A block and a wavefront, tokens from memory, lengths from an
    // eighth of the longest on, us: INT8, d = 128, 512 lists of up to 32 tokens 5.5 and
    // 5.5, 64 6.5 and 7.3; 1024 of 64 9.3 and 8.2, 96 9.8 and 9.8, 128 10.6 and 11.5; 2048
    // of 128 16.5 and 15.1, 256 22.2 and 21.2; 4096 of 512 61.5 and 61.6; 12288 of 128 77
    // and 55, 1536 481 and 455; FP4, d = 64, 1024 of 64 5.6 and 5.5, 96 6.0 and 6.6; 2048 of
    // 256 12.3 and 12.9; 4096 of 512 27.8 and 24.8; BF16, d = 128, 512 of 32 5.7 and 6.5, 1024
    // of 64 11.0 and 9.7; 2048 of 192 28.7 and 28.3, 256 33.4 and 35.2.
    bool single;
    bool own_wide;
    // offsets, and the total
    size_t ml, part, shared_ml, shared_part, chunk, bytes;
};

// cuts: own lists are those of cuts; wide ones go to k_attn_cut_wide.
Split split_of(const PagedDims& c, const PagedLists& own, const PagedLists* shared,
               bool cuts = false) {
    Split s{};
    const size_t lists = (size_t)own.lists * c.heads, rows = lists * c.group;
    auto wanted = [](int64_t blocks, int64_t items) { return std::max<int64_t>(1, blocks / items); };
    s.own_wide = cuts && c.group > 16;
    s.single = !s.own_wide && (int64_t)own.max_len * 6 + 640 <= (int64_t)lists &&
               (!cuts || own.max_len <= kSharedMost);
    int64_t own_want = wanted(cuts ? 4 * kCus : 2 * kCus, lists);
    int most_chunk = kOwnMost;
    if (s.own_wide) {
        own_want = lists <= kFewCuts ? kCutParts : 1;
        most_chunk = 1 << 30;
    } else if (cuts && s.single) {
        most_chunk = kSharedMost;  // one part
    } else if (cuts && lists >= kManyLists) {
        most_chunk = kOwnLongest;
    }
    s.own_chunk = chunk_of(own.max_len, own_want, most_chunk);
    s.own_parts = std::max(1, parts_of(own.max_len, s.own_chunk));
    const size_t own_most = most_parts(own.max_len, own_want, kLeastChunk, most_chunk);
    size_t shared_most = 0;
    if (shared) {
        const int64_t mean = ((int64_t)own.lists * c.group + shared->lists - 1) / shared->lists;
        const int64_t blocks = (mean + 15) / 16 * shared->lists * c.heads *
                               parts_of(shared->max_len, kLeastChunk);  // of 16 columns, 256 tokens
        s.wide = c.type == kBf16   ? mean >= 96 && blocks >= 3072
                 : c.type == kInt8 ? mean >= 96 && blocks >= (mean < 160 ? 12288 : 8192)
                                   : mean >= 192 && blocks >= 16384;
        const int cols = s.wide ? kWideCols : 16;
        s.tiles = (int)((mean + cols - 1) / cols);
        const int64_t want = wanted(kCus, (int64_t)shared->lists * c.heads * s.tiles);
        s.shared_chunk = chunk_of(shared->max_len, want, kSharedMost);
        s.shared_parts = std::max(1, parts_of(shared->max_len, s.shared_chunk));
        shared_most = most_parts(shared->max_len, want, kLeastChunk, kSharedMost);
    }
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t own_places = own_most > 1 || shared ? rows * own_most : 0;
    s.ml = kCounterBytes;
    s.part = s.ml + up(own_places * sizeof(f32x2_t));
    s.shared_ml = s.part + up(own_places * c.d * sizeof(float));
    s.shared_part = s.shared_ml + up(rows * shared_most * sizeof(f32x2_t));
    s.chunk = s.shared_part + rows * shared_most * c.d * sizeof(float);
    s.bytes = s.chunk + (cuts ? 256 : 0);
    return s;
}

template <int TYPE, int D, bool TOK>
int attn_launch(AttnCall a, bool wide, bool single, bool own_wide, hipStream_t st) {
    const int lists = a.own.lists * a.c.heads;
    // (a launch has fewer than 2^32 threads)
    constexpr int64_t kMost = (1ll << 31) / kThreads, kWideMost = (1ll << 31) / kWideThreads;
    const int most = (int)std::max<int64_t>(1, std::min<int64_t>(kCounters, kMost / a.own_parts));
    auto own_blocks = [&] {
        const int64_t units = (int64_t)a.lists * a.own_parts;
        return single ? (units + kWaves - 1) / kWaves : units;
    };
    if (a.shared_parts) {
        const int64_t blocks = (int64_t)a.shared.lists * a.c.heads * a.shared_parts * a.tiles;
        if (blocks >= 1ll << 31) return kTooLarge;
        if (!wide) {  // with the own lists, where one launch holds them all
            a.lists = lists <= most && !own_wide ? lists : 0;
            if (blocks + own_blocks() > kMost) a.lists = 0;
        }
        const int64_t part = wide ? kWideMost : kMost;
        for (int64_t b0 = 0; b0 < blocks; b0 += part) {
            a.shared_block0 = (int)b0;
            a.shared_blocks = (int)std::min(blocks - b0, part);
            if (wide) {
                k_attn_shared_wide<TYPE, D, TOK><<<a.shared_blocks, kWideThreads, 0, st>>>(a);
            } else {
                const unsigned grid = (unsigned)(a.shared_blocks + own_blocks());
                const size_t lds = join_bytes(D, 16);
                if (single) k_attn_with_shared<TYPE, D, 1, TOK><<<grid, kThreads, lds, st>>>(a);
                else k_attn_with_shared<TYPE, D, kWaves, TOK><<<grid, kThreads, lds, st>>>(a);
            }
            if (int e = (int)hipGetLastError()) return e;
        }
        if (a.lists) return 0;
    }
    if constexpr (TOK) {
        if (own_wide) {
            const int64_t blocks = (int64_t)lists * a.own_parts;
            if (blocks >= 1ll << 31) return kTooLarge;
            int* chunk = lists <= kFewCuts ? a.chunk_of_all : nullptr;
            if (chunk) {
                k_attn_cut_wide<TYPE, D, true><<<(unsigned)std::min<int64_t>(blocks, kCutBlocks),
                                                 kWideThreads, 0, st>>>(a, chunk);
                if (int e = (int)hipGetLastError()) return e;
            }
            for (int64_t b0 = 0; b0 < blocks && !chunk; b0 += kWideMost) {
                a.list0 = (int)b0;
                k_attn_cut_wide<TYPE, D, false><<<(unsigned)std::min(blocks - b0, kWideMost),
                                                  kWideThreads, 0, st>>>(a, nullptr);
                if (int e = (int)hipGetLastError()) return e;
            }
            const bool parts = a.own_parts > 1 || a.shared_parts;
            const int64_t rows = parts ? (int64_t)lists * a.c.group : 0;  // (below 2^32)
            constexpr int64_t kPer = 1 << 24;
            for (int64_t r0 = 0; r0 < rows; r0 += kPer) {
                a.row0 = r0;
                const int64_t n = std::min(rows - r0, kPer) * (D / 4);
                k_attn_join<D><<<(unsigned)((n + kThreads - 1) / kThreads), kThreads, 0, st>>>(a, chunk);
                if (int e = (int)hipGetLastError()) return e;
            }
            return 0;
        }
    }
    for (int l0 = 0; l0 < lists; l0 += most) {
        a.list0 = l0;
        a.lists = std::min(lists - l0, most);
        const unsigned grid = (unsigned)own_blocks();
        const size_t lds = join_bytes(D, a.c.group);
        if (single) k_attn_own<TYPE, D, 1, TOK><<<grid, kThreads, lds, st>>>(a);
        else k_attn_own<TYPE, D, kWaves, TOK><<<grid, kThreads, lds, st>>>(a);
        if (int e = (int)hipGetLastError()) return e;
    }
    return 0;
}

}  // namespace

size_t paged_attn_workspace(const PagedDims& c, const PagedLists& own, const PagedLists* shared) {
    return split_of(c, own, shared).bytes;
}

static int launch_call(AttnCall a, const Split& s, void* ws, bool tok, void* stream) {
    char* w = static_cast<char*>(ws);
    a.arrived = reinterpret_cast<int*>(w);
    a.ml = reinterpret_cast<f32x2_t*>(w + s.ml);
    a.part = reinterpret_cast<float*>(w + s.part);
    a.shared_ml = reinterpret_cast<f32x2_t*>(w + s.shared_ml);
    a.shared_part = reinterpret_cast<float*>(w + s.shared_part);
    a.chunk_of_all = reinterpret_cast<int*>(w + s.chunk);
    a.own_chunk = s.own_chunk;
    a.own_parts = s.own_parts;
    a.shared_chunk = s.shared_chunk;
    a.shared_parts = s.shared_parts;
    a.tiles = s.tiles;
    hipStream_t st = (hipStream_t)stream;
    auto run = [&](auto type, auto dim) {
        constexpr int TYPE = decltype(type)::value, D = decltype(dim)::value;
        return tok ? attn_launch<TYPE, D, true>(a, s.wide, s.single, s.own_wide, st)
                   : attn_launch<TYPE, D, false>(a, s.wide, s.single, false, st);
    };
    auto of_dim = [&](auto dim) {
        return a.c.type == kBf16   ? run(std::integral_constant<int, kBf16>{}, dim)
               : a.c.type == kInt8 ? run(std::integral_constant<int, kInt8>{}, dim)
                                   : run(std::integral_constant<int, kFp4>{}, dim);
    };
    return a.c.d == 128 ? of_dim(std::integral_constant<int, 128>{})
                        : of_dim(std::integral_constant<int, 64>{});
}

int launch_paged_attn(const PagedDims& c, const char* pool, const PagedLists& own,
                      const PagedLists* shared, const int32_t* share, const uint16_t* q,
                      int64_t q_stride, float* out, float* lse, void* ws, void* stream) {
    AttnCall a{};
    a.c = c;
    a.pool = pool;
    a.own = own;
    if (shared) a.shared = *shared;
    a.share = share;
    a.q = q;
    a.q_stride = q_stride;
    a.out = out;
    a.lse = lse;
    return launch_call(a, split_of(c, own, shared), ws, false, stream);
}

// Cuts in the place of rows.  Of up to 16 columns, for own_block, or up to kCutCols for
// k_attn_cut_wide, which converts a list's tokens for all of them once but takes some 4 to 8 us
// more however short the list is.  Times of the first over the second, tokens from memory,
// the longest list four times the shortest, one call after the other:
//   columns of a row and head     24    32    48    64    96   128
//   1024 lists of up to 2048 INT8 1.25  1.33  1.70  1.90  1.96  2.25
//                            FP4  .93   .96  1.28  1.19  1.32  1.49
//                            BF16 2.11  2.10  2.92  3.47  4.03  4.73
//   1024 of up to 256        INT8 1.03  1.03  1.18  1.16  1.30  1.45
//                            FP4  .84   .84  1.00  1.05   .95  1.05
//                            BF16 1.28  1.28  1.47  1.75  2.06  2.47
//   32 of up to 2048         INT8 .79   .78   .89   .83   .86   .97
//                            FP4  .71   .70   .74   .67   .68   .73
//                            BF16 .90   .91  1.00   .98  1.07  1.20
// so by the columns and by the work, in tiles of 16 columns and tokens of a list.
static bool is_wide(const PagedDims& c, int64_t lists, int64_t columns, int64_t reach) {
    const bool fp4 = c.type == kFp4;
    return columns >= (fp4 ? 33 : 17) &&
           lists * ((columns + 15) / 16) * reach >= (fp4 ? 1 << 20 : 1 << 19);
}
static bool cut_rows(PagedDims* c, PagedLists* own, int tokens, bool wide, int* cuts, int* cut) {
    *cut = std::max(1, std::min((wide ? kCutCols : 16) / c->group, tokens));
    *cuts = (tokens + *cut - 1) / *cut;
    if ((int64_t)own->lists * *cuts * c->heads > 1 << 24) return false;
    own->lists *= *cuts;
    c->group *= *cut;
    return true;
}
static int reach_of(const PagedDims& c, const PagedLists& own, int tokens) {
    return (int)std::min<int64_t>((int64_t)own.max_len + tokens, (int64_t)own.max_pages * c.ptok);
}

// Enough for every shorter length too: narrow cuts up to where wide ones take over.
size_t paged_attn_tokens_workspace(const PagedDims& c, const PagedLists& own, const PagedLists* shared,
                                   int tokens) {
    tokens = std::max(tokens, 1);
    const int64_t lists = (int64_t)own.lists * c.heads, columns = (int64_t)tokens * c.group;
    const int reach = reach_of(c, own, tokens);
    size_t bytes = 0;
    for (bool wide : {false, true}) {
        PagedDims d = c;
        PagedLists o = own;
        int cuts, cut;
        o.max_len = reach;
        if (is_wide(c, lists, columns, reach) != wide) {
            if (wide) continue;
            int64_t lo = 0, hi = reach;  // narrow at lo, wide at hi
            while (hi - lo > 1) {
                const int64_t mid = lo + (hi - lo) / 2;
                (is_wide(c, lists, columns, mid) ? hi : lo) = mid;
            }
            o.max_len = (int)lo;
        }
        if (!cut_rows(&d, &o, tokens, wide, &cuts, &cut)) return 0;
        bytes = std::max(bytes, split_of(d, o, shared, true).bytes);
    }
    return bytes;
}

int launch_paged_attn_tokens(const PagedTokens& t, const PagedDims& c, const char* pool,
                             const PagedLists& own, const PagedLists* shared, const int32_t* share,
                             float* out, float* lse, void* ws, void* stream) {
    AttnCall a{};
    a.c = c;
    a.own = own;
    a.reach = reach_of(c, own, t.tokens);
    const bool wide = is_wide(c, (int64_t)own.lists * c.heads, (int64_t)t.tokens * c.group, a.reach);
    if (!cut_rows(&a.c, &a.own, t.tokens, wide, &a.cuts, &a.cut)) return kTooLarge;
    a.own.max_len = a.reach;
    const Split s = split_of(a.c, a.own, shared, true);
    a.own.max_len = own.max_len;
    a.heads = c.group;
    a.pool = pool;
    if (shared) a.shared = *shared;
    a.share = share;
    a.tokens = t.tokens;
    a.counts = t.counts;
    a.window = t.window;
    a.q = t.q;
    a.q_stride = t.q_row;
    a.q_token = t.q_token;
    a.out = out;
    a.lse = lse;
    return launch_call(a, s, ws, true, stream);
}

}  // namespace headkv
