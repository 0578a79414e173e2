// Verification of drafted tokens (formulas: headkv.h): sums of every position's exponentials,
// the decisions, and the next token by a running sum over one position.
//
// Decisions next to a border must not depend on the order of a sum, so exponentials and
// sums have 64 bits.  (The vector ALU does a product and sum of 64 bits in the time of one
// of 32.)
// k_verify_sums: a block takes a segment of one position's target or draft logits into
// registers and leaves its maximum and its sum relative to that; the block that brings the
// last part of a row adds them up, decides on the drafts and writes all results but the next
// token.  k_verify_next: a wavefront for each piece of the one position that the next token
// is drawn from leaves its sum of r; one of the row's last block finds the piece, takes its
// logits again and finds the token in it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "logits_device.h"
#include "paged.h"

namespace headkv {
namespace {

using namespace dev;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxSlots = 2 * HEADKV_MAX_DRAFTS + 1;  // positions of a row, target's and draft's
constexpr double kLn2 = 0.69314718055994530942;

// What a block knows of its segment: the bits of the sum of 2^y, y = (x - m) k, and the
// maximum m, a NaN if the segment has one or +inf.  (T = 0: the key of the largest logit.)
struct Part {
    uint64_t w[2];
};

// What the next token is drawn from: r(x) = max(e_p / sum_p - e_q / sum_q, 0).
struct Next {
    int pos;   // -1: no next token
    int gone;  // the certain draft that was not kept, or -1
    float p_max, q_max;
    double p_inv, q_inv;  // 1 / sum; q_inv = 0: no draft to subtract
};

// 2^(j / 32), rounded.
__constant__ const double kPowers[32] = {
    1.0, 1.0218971486541166, 1.0442737824274138, 1.0671404006768237,
    1.0905077326652577, 1.1143867425958924, 1.1387886347566916, 1.1637248587775775,
    1.189207115002721, 1.215247359980469, 1.241857812073484, 1.2690509571917332,
    1.2968395546510096, 1.3252366431597413, 1.3542555469368927, 1.383909881963832,
    1.4142135623730951, 1.4451808069770467, 1.4768261459394993, 1.5091644275934228,
    1.5422108254079407, 1.5759808451078865, 1.6104903319492543, 1.645755478153965,
    1.681792830507429, 1.718619298122478, 1.7562521603732995, 1.7947090750031072,
    1.8340080864093424, 1.8741676341103, 1.9152065613971474, 1.9571441241754002,
};
struct Powers {
    double of[32];
    __device__ __forceinline__ void fill() {  // before a barrier
        if (threadIdx.x < 32) of[threadIdx.x] = kPowers[threadIdx.x];
    }
    // e^((x - m) / temperature), m the largest logit (not -inf): 2^y, y = k times the difference
    // with k = log2(e) / T, in 32nds.  A sum with 1.5 2^52 leaves the nearest whole number of
    // them in its low bits; what is left, at most half a 32nd, has a Taylor series whose sixth
    // term is below 2^-48; 32nds come from a table, whose entries lie in different banks
    // each, and whole powers are added to the exponent.  Below 2^-1020 it is that, which no
    // sum with the largest logit's 1 in it sees.
    __device__ __forceinline__ double share(float x, float m, double k) const {
        constexpr double kMagic = 0x1.8p52, c = 0.69314718055994530942 / 32;
        // (32nds after the product: 32 k may pass what 64 bits hold where k does not)
        const double y = fmax(((double)x - (double)m) * k, -1020.0);
        const double t = fma(32.0, y, kMagic), f = fma(32.0, y, kMagic - t);
        const int n = (int)__builtin_bit_cast(uint64_t, t);
        double p = c * c * c * c * c / 120;
        p = fma(p, f, c * c * c * c / 24);
        p = fma(p, f, c * c * c / 6);
        p = fma(p, f, c * c / 2);
        p = fma(p, f, c);
        p = fma(p, f, 1.0);
        p *= of[n & 31];
        const uint64_t bits = __builtin_bit_cast(uint64_t, p);
        const uint32_t high = (uint32_t)(bits >> 32) + ((uint32_t)(n >> 5) << 20);
        return __builtin_bit_cast(double, (uint64_t)high << 32 | (uint32_t)bits);
    }
};
// The same where what is 0 matters: 0 from 2^-1020 on.
__device__ __forceinline__ double share_of(const Powers& p, float x, float m, double k) {
    return ((double)x - (double)m) * k > -1020.0 ? p.share(x, m, k) : 0.0;
}

__device__ __forceinline__ double wave_add(double v) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
    return v;
}

// Drafts of row r that count: up to its counts and the first token that is none; -1 for a
// row that is left out.  Every lane of a wavefront calls it.
__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int r) {
    const int lane = threadIdx.x & 63;
    const int t = lane < a.drafts ? a.tokens[(int64_t)r * a.drafts + lane] : -1;
    const uint64_t none = __builtin_amdgcn_ballot_w64(t < 0 || t >= a.vocab);
    const int n = __builtin_ctzll(none);  // (lane 63 never has a draft)
    return a.counts ? min(n, max(a.counts[r], -1)) : n;
}

// Segment `seg` of a row of logits: where its vectors start, and which of their values
// belong to the row.
template <typename T>
struct Place {
    const T* p;
    int first;   // index of value 0
    int lo, hi;  // values that belong to the row
    __device__ __forceinline__ Place(const T* row, int vocab, int seg, int size) {
        const int lead = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
        first = seg * size - lead;
        p = row + first;
        lo = max(-first, 0);
        hi = min(vocab - first, size);
    }
};

template <typename T>
__device__ __forceinline__ float value_at(const T* row, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(row[i]);
    else return __uint_as_float((uint32_t)row[i] << 16);
}

template <typename T>
__device__ __forceinline__ const T* target_row(const VerifyArgs& a, int r, int pos) {
    return static_cast<const T*>(a.logits) + r * a.row + pos * a.token;
}
template <typename T>
__device__ __forceinline__ const T* draft_row(const VerifyArgs& a, int r, int pos) {
    return static_cast<const T*>(a.draft) + r * a.draft_row + pos * a.draft_token;
}

// True for the last block of `total` to come here; the counter is then as it was found.
__device__ __forceinline__ bool last_of(int* counter, int total, int* flag) {
    // every published word has left before the block counts as arrived
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        *flag = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                total - 1;
        if (*flag) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return *flag;
}

template <typename T, int EPT, bool GREEDY>
__global__ __launch_bounds__(kThreads) void k_verify_sums(VerifyArgs a, int segments, Part* parts,
                                                          Next* nexts, int* arrived) {
    constexpr int SEG = kThreads * EPT;
    using Values = Logits<T, kThreads, EPT>;
    __shared__ float tops[kWaves];
    __shared__ double sums[kWaves];
    __shared__ uint64_t keys[kWaves];
    __shared__ float row_top[kMaxSlots];
    __shared__ double row_sum[kMaxSlots];
    __shared__ uint64_t row_key[HEADKV_MAX_DRAFTS + 1];
    __shared__ int flag;
    __shared__ Powers powers;
    powers.fill();
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool model = !GREEDY && a.draft;
    // (blocks go to the XCDs in turn: the same segments of all rows, which may be the only ones
    // that are not masked, must not all go to the same)
    const int rest = blockIdx.x / segments, seg = (blockIdx.x - rest * segments + rest) % segments;
    const int r = rest % a.rows, slot = rest / a.rows;
    // target and draft of a position beside each other
    const int pos = model ? slot >> 1 : slot;
    const bool draft = model && slot & 1;
    const int given = drafts_of(a, r);
    int32_t* out_tokens = a.out_tokens + (int64_t)r * (a.drafts + 1);
    float* out_logprob = a.out_logprob ? a.out_logprob + (int64_t)r * (a.drafts + 1) : nullptr;
    if (given < 0) {
        if (slot == 0 && seg == 0) {
            if (tid <= a.drafts) {
                out_tokens[tid] = -1;
                if (out_logprob) out_logprob[tid] = 0.f;
            }
            if (tid == 0) {
                a.out_count[r] = 0;
                nexts[r].pos = -1;
            }
        }
        return;
    }
    if (pos > given || (draft && pos >= given)) return;

    Values x;
    const Place<T> at(draft ? draft_row<T>(a, r, pos) : target_row<T>(a, r, pos), a.vocab, seg, SEG);
    x.load(at.p, at.lo, at.hi, tid);
    float m = -INFINITY;
    bool none = false;  // no number, or +inf
#pragma unroll
    for (int v = 0; v < Values::NV; ++v)
#pragma unroll
        for (int e = 0; e < Values::N; ++e) {
            m = fmaxf(m, x.at(v, e));
            none |= !(x.at(v, e) < INFINITY);
        }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) m = fmaxf(m, __shfl_xor(m, o));
    if (__builtin_amdgcn_ballot_w64(none)) m = NAN;
    if (lane == 0) tops[wave] = m;
    __syncthreads();
    m = tops[0];
    none = m != m;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        none |= tops[w] != tops[w];
        m = fmaxf(m, tops[w]);
    }
    const int slots = given + 1 + (model ? given : 0);
    Part* part = parts + ((int64_t)r * (2 * a.drafts + 1) + slot) * segments + seg;
    if constexpr (GREEDY) {
        uint64_t key = 0;
#pragma unroll
        for (int v = 0; v < Values::NV; ++v)
#pragma unroll
            for (int e = 0; e < Values::N; ++e) {
                const int j = (v * kThreads + tid) * Values::N + e;
                if (x.at(v, e) == m && j >= at.lo && j < at.hi)
                    key = max(key, key_of(order_of(m), at.first + j));
            }
#pragma unroll
        for (int o = 1; o < 64; o *= 2) key = max(key, (uint64_t)__shfl_xor((long long)key, o));
        if (lane == 0) keys[wave] = key;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) key = max(key, keys[w]);
        if (tid == 0) publish(part->w, none ? ~0ull : m == -INFINITY ? 0 : key);
    } else {
        double s = 0;
        if (m > -INFINITY) {
#pragma unroll
            for (int v = 0; v < Values::NV; ++v)
#pragma unroll
                for (int e = 0; e < Values::N; ++e) s += powers.share(x.at(v, e), m, a.k);
        }
        s = wave_add(s);
        if (lane == 0) sums[wave] = s;
        __syncthreads();
        if (tid == 0) {
            s = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s += sums[w];
            publish(part->w, __builtin_bit_cast(uint64_t, s));
            publish(part->w + 1, __float_as_uint(none ? NAN : m));
        }
    }
    if (!last_of(arrived + r, slots * segments, &flag)) return;

    // the row's parts, a wavefront for each position
    for (int i = wave; i < slots; i += kWaves) {
        const Part* p = parts + ((int64_t)r * (2 * a.drafts + 1) + i) * segments;
        if constexpr (GREEDY) {
            uint64_t key = 0;
            for (int j = lane; j < segments; j += 64) key = max(key, read(p[j].w));
#pragma unroll
            for (int o = 1; o < 64; o *= 2) key = max(key, (uint64_t)__shfl_xor((long long)key, o));
            if (lane == 0) row_key[i] = key;
        } else {
            float top = -INFINITY;
            bool none = false;
            for (int j = lane; j < segments; j += 64) {
                const float t = __uint_as_float((uint32_t)read(p[j].w + 1));
                none |= t != t;
                top = fmaxf(top, t);
            }
#pragma unroll
            for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
            double s = 0;
            for (int j = lane; j < segments; j += 64) {
                const float t = __uint_as_float((uint32_t)read(p[j].w + 1));
                if (t > -INFINITY)
                    s += __builtin_bit_cast(double, read(p[j].w)) * share_of(powers, t, top, a.k);
            }
            s = wave_add(s);
            none = __builtin_amdgcn_ballot_w64(none) != 0;
            if (lane == 0) {
                row_top[i] = none ? NAN : top;
                row_sum[i] = s;
            }
        }
    }
    __syncthreads();
    if (wave > 0) return;
    // lane i: draft i, or what follows the last of them
    const bool there = lane <= given;
    const int token = lane < given ? a.tokens[(int64_t)r * a.drafts + lane] : -1;
    bool fails = false, keeps = false;
    float logprob = 0.f;
    int largest = -1;
    Next next{};
    if (there && GREEDY) {
        const uint64_t key = row_key[lane];
        fails = key == 0 || key == ~0ull;
        largest = (int)~(uint32_t)key;
        keeps = lane < given && !fails && token == largest;
    }
    if (there && !GREEDY) {
        const int p = model ? 2 * lane : lane;
        next.gone = -1;
        next.p_max = row_top[p];
        next.p_inv = 1.0 / row_sum[p];
        fails = next.p_max != next.p_max || !(row_sum[p] > 0);
        if (lane < given) {
            double q = 1.0;
            if (model) {
                const float m = row_top[p + 1];
                fails |= m != m;
                next.q_max = m;
                next.q_inv = row_sum[p + 1] > 0 ? 1.0 / row_sum[p + 1] : 0.0;
                q = 0.0;
                if (!fails && next.q_inv > 0)
                    q = share_of(powers, value_at(draft_row<T>(a, r, lane), token), m, a.k) * next.q_inv;
            } else {
                next.gone = token;
            }
            if (!fails) {
                const float x = value_at(target_row<T>(a, r, lane), token);
                const double share = share_of(powers, x, next.p_max, a.k) * next.p_inv;
                const double u = a.uniforms[(int64_t)r * (a.drafts + 1) + lane];
                keeps = u < 1.0 && fmax(u, 0.0) * q < share;
                logprob = (float)((((double)x - (double)next.p_max) * a.k + log2(next.p_inv)) * kLn2);
            }
        }
    }
    const int stop = __builtin_ctzll(__builtin_amdgcn_ballot_w64(there && !keeps));
    const bool ends = __builtin_amdgcn_ballot_w64(fails) >> stop & 1;  // without a next token
    if (lane <= a.drafts) {
        if (GREEDY || lane != stop || ends) {
            out_tokens[lane] = lane < stop ? token : GREEDY && lane == stop && !ends ? largest : -1;
            if (out_logprob) out_logprob[lane] = lane < stop ? logprob : 0.f;
        }
    }
    if (lane == stop) {
        a.out_count[r] = stop + !ends;
        next.pos = ends ? -1 : stop;
        if (!GREEDY) nexts[r] = next;
    }
}

// The first of 64 lanes, or the last with any, at which the running sum from `before` on
// passes `want`; *passed: it does.  -1: no lane has any.
__device__ __forceinline__ int find_lane(double t, double before, double want, bool* passed,
                                         double* at, double* total) {
    const int lane = threadIdx.x & 63;
    double up = t;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const double y = __shfl_up(up, o);
        if (lane >= o) up += y;
    }
    const uint64_t over = __builtin_amdgcn_ballot_w64(t > 0 && before + up > want);
    const uint64_t some = __builtin_amdgcn_ballot_w64(t > 0);
    const int pick = over ? __builtin_ctzll(over) : some ? 63 - __builtin_clzll(some) : -1;
    *passed = over != 0;
    *at = before + __shfl(up - t, max(pick, 0));
    *total = __shfl(up, 63);
    return pick;
}

// A wavefront for `per` pieces of a row one after the other, kPiece values each: a block
// costs some 9 us, most of them for its sums to arrive, so there are no more than a few for each
// CU (128 rows of 65536: 38 us with 4096 blocks, 30 with 1024).  There is one place that computes a
// piece's r: with one for each of its uses the code does not stay in the instruction cache.
constexpr int kPieceEpt = 8, kPiece = 64 * kPieceEpt;

template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_next(VerifyArgs a, int blocks, int per,
                                                          uint64_t* sums, const Next* nexts,
                                                          int* arrived) {
    using Values = Logits<T, 64, kPieceEpt>;
    constexpr int NV = Values::NV, N = Values::N;
    __shared__ int flag;
    __shared__ Powers powers;
    __shared__ double values[kWaves][kPiece];  // r of a wavefront's piece
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = blockIdx.x / blocks, pieces = blocks * kWaves * per;
    Next n = nexts[r];
    if (n.pos < 0) return;
    powers.fill();
    __syncthreads();
    const T* row = target_row<T>(a, r, n.pos);
    const T* draft = n.q_inv > 0 ? draft_row<T>(a, r, n.pos) : nullptr;
    uint64_t* of_row = sums + (int64_t)r * pieces;
    auto sum_at = [&](int i) {
        return i < pieces ? __builtin_bit_cast(double, read(of_row + i)) : 0.0;
    };
    double u = a.uniforms[(int64_t)r * (a.drafts + 1) + a.drafts];
    u = u < 1.0 ? fmax(u, 0.0) : 0x1.fffffep-1;  // (NaN: the largest, too)

    // first every wavefront its own piece; then, by one, the piece that holds the token (and
    // where there is no r to speak of, one after the other with p in its place)
    enum { kOwn, kEach, kFound } now = kOwn;
    int piece = ((blockIdx.x - r * blocks) * kWaves + wave) * per, found = 0, first;
    const int end = piece + per;
    double before = 0, sum = 0, want = 0;
    for (;;) {
        const Place<T> at(row, a.vocab, piece, kPiece);
        first = at.first;
        Values p, q;
        p.load(at.p, at.lo, at.hi, lane);
        bool beside = false;  // the draft's vectors start at the same values
        if (draft) {
            const Place<T> other(draft, a.vocab, piece, kPiece);
            beside = other.first == at.first;
            if (beside) q.load(other.p, other.lo, other.hi, lane);
        }
        double mine = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int j = (v * 64 + lane) * N + e;
                const float x = p.at(v, e);
                double y = 0;
                if (x > -INFINITY && first + j != n.gone) {
                    y = share_of(powers, x, n.p_max, a.k) * n.p_inv;
                    if (draft) {
                        const float z = beside ? q.at(v, e) : value_at(draft, first + j);
                        y = fmax(y - share_of(powers, z, n.q_max, a.k) * n.q_inv, 0.0);
                    }
                }
                values[wave][j] = y;
                mine += y;
            }
        mine = wave_add(mine);
        if (now == kFound) break;
        if (now == kOwn) {
            if (lane == 0) publish(of_row + piece, __builtin_bit_cast(uint64_t, mine));
            if (++piece < end) continue;
            if (!last_of(arrived + r, blocks, &flag) || wave > 0) return;
            double total = 0;
            for (int i = 0; i < pieces; i += 64) total += wave_add(sum_at(i + lane));
            if (total < 0x1p-40) {
                n.gone = -1;
                draft = nullptr;
                want = u;
                now = kEach;
                piece = 0;
                continue;
            }
            want = u * total;
            for (int i = 0; i < pieces; i += 64) {
                bool passed;
                double at, all;
                const int pick = find_lane(sum_at(i + lane), sum, want, &passed, &at, &all);
                if (pick >= 0) found = i + pick, before = at;
                if (passed) break;
                sum += all;
            }
        } else {
            if (mine > 0) found = piece, before = sum;  // the last of them, if rounding leaves none
            sum += mine;
            if (!(sum > want) && piece + 1 < pieces) {
                ++piece;
                continue;
            }
        }
        piece = found;
        now = kFound;
    }
    // lane i: the vector's values i N to i N + N - 1
    int at_v = 0, at_lane = 0;
    sum = before;
#pragma unroll 1
    for (int v = 0; v < NV; ++v) {
        double t = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) t += values[0][(v * 64 + lane) * N + e];
        bool passed;
        double at, all;
        const int pick = find_lane(t, sum, want, &passed, &at, &all);
        if (pick >= 0) at_v = v, at_lane = pick, before = at;
        if (passed) break;
        sum += all;
    }
    if (lane != at_lane) return;
    int token = -1;
    bool done = false;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const int j = (at_v * 64 + lane) * N + e;
        const double y = values[0][j];
        if (done || !(y > 0)) continue;
        token = first + j;
        before += y;
        done = before > want;
    }
    const int64_t o = (int64_t)r * (a.drafts + 1) + n.pos;
    a.out_tokens[o] = token;
    if (a.out_logprob)
        a.out_logprob[o] = (float)((((double)value_at(row, token) - (double)n.p_max) * a.k +
                                    log2(n.p_inv)) * kLn2);
}

constexpr int kLeastSegment = kThreads * 8;
constexpr int kNextBlocks = 1024, kMostPieces = 16;

// Segments of a row that may start `lead` values into a vector.
int segments_of(int vocab, int size, int lead = 7) { return (vocab + lead + size - 1) / size; }

struct VerifyPlan {
    size_t nexts, sums, parts, bytes;  // offsets, and the total
};
VerifyPlan plan_of(int rows, int drafts, int vocab) {
    const size_t segments = segments_of(vocab, kLeastSegment), n = std::min(rows, kCounters);
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    VerifyPlan p;
    p.nexts = kCounterBytes;
    p.sums = p.nexts + up(n * sizeof(Next));
    p.parts = p.sums + up(n * (segments + kMostPieces) * kWaves * sizeof(uint64_t));
    p.bytes = p.parts + n * (2 * drafts + 1) * segments * sizeof(Part);
    return p;
}

template <typename T, int EPT>
int run(const VerifyArgs& a, const VerifyPlan& p, char* w, hipStream_t st) {
    auto* arrived = reinterpret_cast<int*>(w);
    auto* nexts = reinterpret_cast<Next*>(w + p.nexts);
    auto* sums = reinterpret_cast<uint64_t*>(w + p.sums);
    auto* parts = reinterpret_cast<Part*>(w + p.parts);
    const bool even = (reinterpret_cast<uintptr_t>(a.logits) | reinterpret_cast<uintptr_t>(a.draft) |
                       ((a.row | a.token | a.draft_row | a.draft_token) * sizeof(T))) % 16 == 0;
    const int lead = even ? 0 : 16 / (int)sizeof(T) - 1;
    const int segments = segments_of(a.vocab, kThreads * EPT, lead);
    const int64_t slots = a.drafts + 1 + (a.draft && a.k ? a.drafts : 0);
    const unsigned grid = (unsigned)(slots * a.rows * segments);
    if (a.k == 0) {
        k_verify_sums<T, EPT, true><<<grid, kThreads, 0, st>>>(a, segments, parts, nexts, arrived);
        return (int)hipGetLastError();
    }
    k_verify_sums<T, EPT, false><<<grid, kThreads, 0, st>>>(a, segments, parts, nexts, arrived);
    if (int e = (int)hipGetLastError()) return e;
    const int all = segments_of(a.vocab, kWaves * kPiece, lead);
    const int per = (int)std::min<int64_t>(kMostPieces, ((int64_t)a.rows * all + kNextBlocks - 1) / kNextBlocks);
    const int blocks = (all + per - 1) / per;
    k_verify_next<T><<<(unsigned)(a.rows * blocks), kThreads, 0, st>>>(a, blocks, per, sums, nexts,
                                                                      arrived);
    return (int)hipGetLastError();
}

}  // namespace

size_t verify_workspace(int rows, int drafts, int vocab) {
    return plan_of(rows, drafts, vocab).bytes;
}

int launch_verify(const VerifyArgs& all, int logits_type, void* ws, void* stream) {
    const VerifyPlan p = plan_of(all.rows, all.drafts, all.vocab);
    const int size = logits_type == HEADKV_LOGITS_BF16 ? 2 : 4;
    // (fewer than 2^32 threads in a launch)
    const int64_t per_row = (int64_t)(2 * all.drafts + 1) * segments_of(all.vocab, kLeastSegment);
    const int most = (int)std::max<int64_t>(1, std::min<int64_t>(kCounters, (1 << 24) / per_row));
    for (int r0 = 0; r0 < all.rows; r0 += most) {
        VerifyArgs a = all;
        a.rows = std::min(all.rows - r0, most);
        a.logits = static_cast<const char*>(all.logits) + r0 * all.row * size;
        if (a.draft) a.draft = static_cast<const char*>(all.draft) + r0 * all.draft_row * size;
        a.tokens += (int64_t)r0 * a.drafts;
        if (a.counts) a.counts += r0;
        const int64_t out = (int64_t)r0 * (a.drafts + 1);
        a.uniforms += out;
        a.out_tokens += out;
        a.out_count += r0;
        if (a.out_logprob) a.out_logprob += out;
        char* w = static_cast<char*>(ws);
        hipStream_t st = (hipStream_t)stream;
        // shorter segments where they are few
        const bool few = (int64_t)a.rows * (2 * a.drafts + 1) * segments_of(a.vocab, 8192) < 1024;
        int e;
        if (size == 2) e = few ? run<uint16_t, 8>(a, p, w, st) : run<uint16_t, 32>(a, p, w, st);
        else e = few ? run<uint32_t, 8>(a, p, w, st) : run<uint32_t, 32>(a, p, w, st);
        if (e) return e;
    }
    return 0;
}

}  // namespace headkv
