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
constexpr int kWideWaves = 8, kWideThreads = 64 * kWideWaves;
constexpr int kWideCols = 2 * 16 * kWideWaves;  // columns of a block of k_attn_shared_wide

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
    // all tokens are attended, bit n of `seen` is set if token n of the lane's eight is.
    template <typename Key, typename Value>
    __device__ __forceinline__ void step(Key key, Value value, const u32x4_t& key_scales,
                                         const u32x4_t& value_scales, bool partial, uint32_t seen) {
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
             t.ks, t.vs, partial, seen);
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
            step_at(now, t0 + (wave + W * n) * kStep, first, t1, lane);
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
template <int W>
__device__ __forceinline__ int find_members(const AttnCall& a, int list, int rank0, int rank1,
                                            int* row_of, int* found, int tid) {
    const int lane = tid & 63, wave = tid >> 6;
    int members = 0;
    for (int b0 = 0; b0 < a.own.lists && members < rank1; b0 += 64 * W) {
        const int b = b0 + tid;
        const bool is = b < a.own.lists && a.share[b] == list;
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
template <int TYPE, int D>
__device__ __forceinline__ void load_queries(const AttnCall& a, int h, int col, int rank0,
                                             const int* row_of, int lane, bf16x8_t* q) {
    const int group = a.c.group;
    const uint16_t* from = a.q + row_of[col / group - rank0] * a.q_stride +
                           (h * group + col % group) * D;
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

// Parts of the prefix that row b shares, for kv head h.
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
template <int D, bool WITH>
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
    write_out(a, row, d, D, all.v, all.m, all.s);
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
template <int TYPE, int D, bool WITH, int W>
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
    const int at = a.list0 + rank;
    const int lh = a.own.order ? min(max(a.own.order[at], 0), a.own.lists * a.c.heads - 1) : at;
    const int b = lh / a.c.heads, h = lh % a.c.heads;
    // the pages as they are without a window, before the length is known
    const int32_t* pages = a.own.pages + (int64_t)lh * a.own.max_pages;
    const int g0 = chunk * a.own_chunk, g1 = min(g0 + a.own_chunk, a.own.max_len);
    int page = Wave<TYPE, D, 1>::template pages_of<W>(a.c, pages, g0, g1, wave, lane);
    const Span s = span_of(a.own, a.c.ptok, lh, a.own_chunk);
    const int chunks = max(s.chunks, 1);
    if (chunk >= chunks) return;
    const int t0 = s.start + chunk * a.own_chunk, t1 = min(s.len, t0 + a.own_chunk);
    const int64_t row0 = (int64_t)lh * group;
    const int prefix = prefix_parts(a, b, h);

    Wave<TYPE, D, 1> w;
    w.clear();
    const uint16_t* q = a.q + b * a.q_stride + (h * group + min(lane & 15, group - 1)) * D;
#pragma unroll
    for (int k = 0; k < D / 32; ++k)
        w.q[0][k] = *reinterpret_cast<const bf16x8_t*>(q + key_dim<TYPE, D>(k, lane >> 4));
    if (s.chunks > 0) {  // (else t0 may be past what an int holds)
        if (s.start > 0) page = Wave<TYPE, D, 1>::template pages_of<W>(a.c, pages, t0, t1, wave, lane);
        w.template run<true, W>(a.c, a.pool, page, t0, t1, s.first, wave, lane);
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
            write_out(a, row0 + col, d, D, all.v, all.m, all.s);
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
        finish<D, WITH>(a, lh, chunks, prefix, i / (D / 4), i % (D / 4) * 4);
}

// A shared list of few columns (members * group of them): one block per (list, kv
// head, chunk) and tile of 16 columns; a block goes on to every `tiles`-th tile.
struct SharedLds {
    int row_of[17], found[kWaves];
    int chunks[16];       // of the members' own lists
    int done[16], count;  // members (of the tile) whose parts are all there
};
template <int TYPE, int D>
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
        const int members = find_members<kWaves>(a, list, rank0, rank1, row_of, ints.found, tid);
        const int cols = min(16, members * group - c0);
        if (cols <= 0 || chunk >= s.chunks) return;  // (the length is not waited for alone)
        const int t0 = s.start + chunk * a.shared_chunk, t1 = min(s.len, t0 + a.shared_chunk);
        // lane i: the member of rank rank0 + i, its columns in the tile
        auto columns = [&] {
            return min(c0 + cols, (rank0 + lane + 1) * group) - max(c0, (rank0 + lane) * group);
        };
        Wave<TYPE, D, 1> w;
        w.clear();
        load_queries<TYPE, D>(a, h, c0 + min(lane & 15, cols - 1), rank0, row_of, lane, w.q[0]);
        if (wave == 0 && columns() > 0)
            ints.chunks[lane] = max(span_of(a.own, a.c.ptok, (int64_t)row_of[lane] * a.c.heads + h,
                                            a.own_chunk).chunks, 1);
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
            finish<D, true>(a, row_of[n] * a.c.heads + h, ints.chunks[n], s.chunks, k / (D / 4),
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

template <int TYPE, int D, int W>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(own_waves<TYPE, D>())))
void k_attn_own(AttnCall a) {
    extern __shared__ __align__(16) float lds[];  // join_bytes(D, group)
    __shared__ int flags[kWaves];
    own_block<TYPE, D, false, W>(a, blockIdx.x, lds, flags);
}

// Shared lists of few columns and the rows' own ones in one launch: the shared ones'
// blocks, which have more to compute, start first, and the rows' fill the CUs beside
// them.  Whichever brings the last part of a row's list joins them all.  (64 rows on a
// prefix of 2048 INT8 tokens with own lists of 64 to 1024, 32 heads: 55 us; in two
// launches, with the prefix's parts read by the second, 62.)
template <int TYPE, int D, int W>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(with_shared_waves<TYPE, D>())))
void k_attn_with_shared(AttnCall a) {
    extern __shared__ __align__(16) float lds[];  // join_bytes(D, 16)
    __shared__ SharedLds ints;
    const int block = blockIdx.x;
    if (block < a.shared_blocks) shared_block<TYPE, D>(a, a.shared_block0 + block, lds, ints);
    else own_block<TYPE, D, true, W>(a, block - a.shared_blocks, lds, ints.found);
}

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
    __device__ __forceinline__ void convert(u32x4_t (*to)[64], int at_scales, bool partial,
                                            uint32_t seen, int wave, int lane) {
        if (values && partial) {
            if constexpr (TYPE == kBf16) {
#pragma unroll
                for (u32x4_t& w : raw) w = T::blank16(w, seen);
            }
            if constexpr (TYPE == kInt8) scales = T::blank16(scales, seen);
            if constexpr (TYPE == kFp4) powers = T::blank8(powers, seen);
        }
        if constexpr (TYPE == kBf16) {
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
            to[slot][lane] = __builtin_bit_cast(u32x4_t, o[0]);
            to[slot + 1][lane] = __builtin_bit_cast(u32x4_t, o[1]);
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
};

// A shared list of many columns: the W wavefronts of a block take NB * 16 columns
// each and the same tokens, whose operands they convert once for all, a share each,
// into LDS in the order in which the lanes read them: those of the next step while
// one is computed, from loads of the step before it.  256 columns of 2 x 8 lists of
// 16384 FP4 tokens: 83 us, 0.83 PFLOP/s on the matrix cores (K once, V with three
// pieces), which are busy for a third of the time; the vector ALU's share, the
// exponentials and the weights' pieces, is 40 %, and the two meet at a step's barrier.
template <int TYPE, int D>
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
        const int members = find_members<W>(a, list, rank0, rank1, row_of, found, tid);
        const int cols = min(COLS, members * group - c0);  // of this tile
        if (cols <= 0) return;
        const int w0 = wave * 16 * NB;  // the wavefront's first column
        Wave<TYPE, D, NB> w;
        w.clear();
#pragma unroll
        for (int n = 0; n < NB; ++n)
            load_queries<TYPE, D>(a, h, c0 + min(w0 + 16 * n + (lane & 15), cols - 1), rank0, row_of,
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
                           ks, vs, partial, seen);
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
constexpr int kLeastChunk = 2 * kUnit, kOwnMost = 8 * kUnit, kSharedMost = 64 * kStep;
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
    // offsets, and the total
    size_t ml, part, shared_ml, shared_part, bytes;
};

Split split_of(const PagedDims& c, const PagedLists& own, const PagedLists* shared) {
    Split s{};
    const size_t lists = (size_t)own.lists * c.heads, rows = lists * c.group;
    auto wanted = [](int64_t blocks, int64_t items) { return std::max<int64_t>(1, blocks / items); };
    const int64_t own_want = wanted(2 * kCus, lists);
    s.own_chunk = chunk_of(own.max_len, own_want, kOwnMost);
    s.own_parts = std::max(1, parts_of(own.max_len, s.own_chunk));
    s.single = (int64_t)own.max_len * 6 + 640 <= (int64_t)lists;
    const size_t own_most = most_parts(own.max_len, own_want, kLeastChunk, kOwnMost);
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
    s.bytes = s.shared_part + rows * shared_most * c.d * sizeof(float);
    return s;
}

template <int TYPE, int D>
int attn_launch(AttnCall a, bool wide, bool single, hipStream_t st) {
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
            a.lists = lists <= most ? lists : 0;
            if (blocks + own_blocks() > kMost) a.lists = 0;
        }
        const int64_t part = wide ? kWideMost : kMost;
        for (int64_t b0 = 0; b0 < blocks; b0 += part) {
            a.shared_block0 = (int)b0;
            a.shared_blocks = (int)std::min(blocks - b0, part);
            if (wide) {
                k_attn_shared_wide<TYPE, D><<<a.shared_blocks, kWideThreads, 0, st>>>(a);
            } else {
                const unsigned grid = (unsigned)(a.shared_blocks + own_blocks());
                const size_t lds = join_bytes(D, 16);
                if (single) k_attn_with_shared<TYPE, D, 1><<<grid, kThreads, lds, st>>>(a);
                else k_attn_with_shared<TYPE, D, kWaves><<<grid, kThreads, lds, st>>>(a);
            }
            if (int e = (int)hipGetLastError()) return e;
        }
        if (a.lists) return 0;
    }
    for (int l0 = 0; l0 < lists; l0 += most) {
        a.list0 = l0;
        a.lists = std::min(lists - l0, most);
        const unsigned grid = (unsigned)own_blocks();
        const size_t lds = join_bytes(D, a.c.group);
        if (single) k_attn_own<TYPE, D, 1><<<grid, kThreads, lds, st>>>(a);
        else k_attn_own<TYPE, D, kWaves><<<grid, kThreads, lds, st>>>(a);
        if (int e = (int)hipGetLastError()) return e;
    }
    return 0;
}

}  // namespace

size_t paged_attn_workspace(const PagedDims& c, const PagedLists& own, const PagedLists* shared) {
    return split_of(c, own, shared).bytes;
}

int launch_paged_attn(const PagedDims& c, const char* pool, const PagedLists& own,
                      const PagedLists* shared, const int32_t* share, const uint16_t* q,
                      int64_t q_stride, float* out, float* lse, void* ws, void* stream) {
    const Split s = split_of(c, own, shared);
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
    char* w = static_cast<char*>(ws);
    a.arrived = reinterpret_cast<int*>(w);
    a.ml = reinterpret_cast<f32x2_t*>(w + s.ml);
    a.part = reinterpret_cast<float*>(w + s.part);
    a.shared_ml = reinterpret_cast<f32x2_t*>(w + s.shared_ml);
    a.shared_part = reinterpret_cast<float*>(w + s.shared_part);
    a.own_chunk = s.own_chunk;
    a.own_parts = s.own_parts;
    a.shared_chunk = s.shared_chunk;
    a.shared_parts = s.shared_parts;
    a.tiles = s.tiles;
    hipStream_t st = (hipStream_t)stream;
    if (c.d == 128)
        return c.type == kBf16   ? attn_launch<kBf16, 128>(a, s.wide, s.single, st)
               : c.type == kInt8 ? attn_launch<kInt8, 128>(a, s.wide, s.single, st)
                                 : attn_launch<kFp4, 128>(a, s.wide, s.single, st);
    return c.type == kBf16   ? attn_launch<kBf16, 64>(a, s.wide, s.single, st)
           : c.type == kInt8 ? attn_launch<kInt8, 64>(a, s.wide, s.single, st)
                             : attn_launch<kFp4, 64>(a, s.wide, s.single, st);
}

}  // namespace headkv
