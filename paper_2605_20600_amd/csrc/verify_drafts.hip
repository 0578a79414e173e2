// Verification of drafted tokens (formulas: headkv.h): sums of every position's exponentials,
// the decisions, and the next token by a running sum over one position.
//
// Decisions next to a border must not depend on the order of a sum, so exponentials and
// sums have 64 bits: 2^y by its Taylor series about the nearest whole power, which is off
// by 2^-47 at most.  (The vector ALU does a product and sum of 64 bits in the time of one
// of 32.)
// k_verify_sums: a block takes a segment of one position's target or draft logits into
// registers and leaves its maximum and its sum relative to that; the block that brings the
// last part of a row adds them up, decides on the drafts and writes all results but the next
// token.  k_verify_next: a block for each segment of the one position that the next token
// is drawn from leaves its sum of r; the last one of a row finds the segment, takes its
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

// 2^y for y <= 0.
__device__ __forceinline__ double exp2_below(double y) {
    y = fmax(y, -1100.0);  // (0 from there on)
    const double n = __builtin_rint(y), f = (y - n) * kLn2;
    double p = 1.0 / 39916800;  // 1 / 11!
    p = fma(p, f, 1.0 / 3628800);
    p = fma(p, f, 1.0 / 362880);
    p = fma(p, f, 1.0 / 40320);
    p = fma(p, f, 1.0 / 5040);
    p = fma(p, f, 1.0 / 720);
    p = fma(p, f, 1.0 / 120);
    p = fma(p, f, 1.0 / 24);
    p = fma(p, f, 1.0 / 6);
    p = fma(p, f, 0.5);
    p = fma(p, f, 1.0);
    p = fma(p, f, 1.0);
    return __builtin_ldexp(p, (int)n);
}
// e^((x - m) / temperature), m the largest logit (not -inf)
__device__ __forceinline__ double share_of(float x, float m, double k) {
    return exp2_below(((double)x - (double)m) * k);
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
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool model = !GREEDY && a.draft;
    const int seg = blockIdx.x % segments, rest = blockIdx.x / segments;
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
                for (int e = 0; e < Values::N; ++e) s += share_of(x.at(v, e), m, a.k);
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
                    s += __builtin_bit_cast(double, read(p[j].w)) * share_of(t, top, a.k);
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
                    q = share_of(value_at(draft_row<T>(a, r, lane), token), m, a.k) * next.q_inv;
            } else {
                next.gone = token;
            }
            if (!fails) {
                const float x = value_at(target_row<T>(a, r, lane), token);
                const double share = share_of(x, next.p_max, a.k) * next.p_inv;
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

// r of a segment: the sum of each thread's vectors.
template <typename T, int EPT>
struct Rest {
    using Values = Logits<T, kThreads, EPT>;
    static constexpr int NV = Values::NV, N = Values::N, SEG = kThreads * EPT;
    Values p, q;
    int first, lo, hi;

    // one value's r; both rows' vectors may start at different values of the row
    __device__ __forceinline__ double at(const VerifyArgs& a, const Next& n, const T* draft, int v,
                                         int e, int tid) const {
        const int i = first + (v * kThreads + tid) * N + e;  // in the row
        double r = 0;
        const float x = p.at(v, e);
        if (x > -INFINITY && i != n.gone) r = share_of(x, n.p_max, a.k) * n.p_inv;
        if (n.q_inv > 0 && r > 0) {
            const float y = value_at(draft, i);
            if (y > -INFINITY) r = fmax(r - share_of(y, n.q_max, a.k) * n.q_inv, 0.0);
        }
        return r;
    }
};

template <typename T, int EPT>
__global__ __launch_bounds__(kThreads) void k_verify_next(VerifyArgs a, int segments,
                                                          uint64_t* segment_sums, const Next* nexts,
                                                          int* arrived) {
    using Values = Rest<T, EPT>;
    constexpr int NV = Values::NV, N = Values::N, SEG = Values::SEG;
    __shared__ double chunks[NV * kWaves];
    __shared__ int flag, where;
    __shared__ double before;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int seg = blockIdx.x % segments, r = blockIdx.x / segments;
    Next n = nexts[r];
    if (n.pos < 0) return;
    const T* row = target_row<T>(a, r, n.pos);
    const T* draft = n.q_inv > 0 ? draft_row<T>(a, r, n.pos) : nullptr;
    Values x;
    double s[NV];  // of the thread's vectors
    // the segment's sum, the same for all threads; chunks holds those of its parts
    auto sum_of = [&](int seg) {
        const Place<T> at(row, a.vocab, seg, SEG);
        x.first = at.first;
        x.p.load(at.p, at.lo, at.hi, tid);
        __syncthreads();  // chunks is read no more
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            s[v] = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) s[v] += x.at(a, n, draft, v, e, tid);
            const double t = wave_add(s[v]);
            if (lane == 0) chunks[v * kWaves + wave] = t;
        }
        __syncthreads();
        double all = 0;
        for (int i = 0; i < NV * kWaves; ++i) all += chunks[i];
        return all;
    };
    const double mine = sum_of(seg);
    uint64_t* of_row = segment_sums + (int64_t)r * segments;
    if (tid == 0) publish(of_row + seg, __builtin_bit_cast(uint64_t, mine));
    if (!last_of(arrived + r, segments, &flag)) return;

    // the segment that holds the token: every wavefront for itself
    double u = a.uniforms[(int64_t)r * (a.drafts + 1) + a.drafts];
    u = u < 1.0 ? fmax(u, 0.0) : 0x1.fffffep-1;  // (NaN: the largest, too)
    auto sum_at = [&](int i) {
        return i < segments ? __builtin_bit_cast(double, read(of_row + i)) : 0.0;
    };
    double total = 0;
    for (int i = 0; i < segments; i += 64) total += wave_add(sum_at(i + lane));
    int found = -1;
    double sum = 0, want = u * total;
    if (total < 0x1p-40) {  // nothing to speak of: p itself
        n.gone = -1;
        n.q_inv = 0;
        want = u;
        for (int i = 0; i < segments; ++i) {
            const double t = sum_of(i);
            if (t > 0) found = i, before = sum;  // the last of them, if rounding leaves none
            if (sum + t > want) break;
            sum += t;
        }
    } else {
        for (int i = 0; i < segments; i += 64) {
            const double t = sum_at(i + lane);
            double up = t;
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const double y = __shfl_up(up, o);
                if (lane >= o) up += y;
            }
            const uint64_t over = __builtin_amdgcn_ballot_w64(t > 0 && sum + up > want);
            const uint64_t some = __builtin_amdgcn_ballot_w64(t > 0);
            const int pick = over ? __builtin_ctzll(over) : some ? 63 - __builtin_clzll(some) : -1;
            if (pick >= 0) {
                found = i + pick;
                const double b = sum + __shfl(up - t, pick);
                if (tid == 0) before = b;
            }
            if (over) break;
            sum += __shfl(up, 63);
        }
    }
    __syncthreads();
    sum_of(found);
    // the vectors of a wavefront that hold it
    if (tid == 0) {
        double sum = before;
        int pick = 0;
        for (int i = 0; i < NV * kWaves; ++i) {
            const double t = chunks[i];
            if (t > 0) pick = i, before = sum;
            if (t > 0 && sum + t > want) break;
            sum += t;
        }
        where = pick;
    }
    __syncthreads();
    if (wave != where % kWaves) return;
    const int v = where / kWaves;
    double t = s[0];
#pragma unroll
    for (int i = 1; i < NV; ++i) t = v == i ? s[i] : t;
    double up = t;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const double y = __shfl_up(up, o);
        if (lane >= o) up += y;
    }
    const uint64_t over = __builtin_amdgcn_ballot_w64(t > 0 && before + up > want);
    const uint64_t some = __builtin_amdgcn_ballot_w64(t > 0);
    if (lane != (over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some))) return;
    double at = before + (up - t);
    int token = -1;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i != v) continue;
        bool done = false;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const double y = x.at(a, n, draft, i, e, tid);
            if (done || !(y > 0)) continue;
            token = x.first + (i * kThreads + tid) * N + e;
            at += y;
            done = at > want;
        }
    }
    const int64_t o = (int64_t)r * (a.drafts + 1) + n.pos;
    a.out_tokens[o] = token;
    if (a.out_logprob)
        a.out_logprob[o] = (float)((((double)value_at(row, token) - (double)n.p_max) * a.k +
                                    log2(n.p_inv)) * kLn2);
}

constexpr int kLeastSegment = kThreads * 8;

// Segments of a row, which may start up to seven values into a vector.
int segments_of(int vocab, int size) { return (vocab + 7 + size - 1) / size; }

struct VerifyPlan {
    size_t nexts, sums, parts, bytes;  // offsets, and the total
};
VerifyPlan plan_of(int rows, int drafts, int vocab) {
    const size_t segments = segments_of(vocab, kLeastSegment), n = std::min(rows, kCounters);
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    VerifyPlan p;
    p.nexts = kCounterBytes;
    p.sums = p.nexts + up(n * sizeof(Next));
    p.parts = p.sums + up(n * segments * sizeof(uint64_t));
    p.bytes = p.parts + n * (2 * drafts + 1) * segments * sizeof(Part);
    return p;
}

template <typename T, int EPT>
int run(const VerifyArgs& a, const VerifyPlan& p, char* w, hipStream_t st) {
    auto* arrived = reinterpret_cast<int*>(w);
    auto* nexts = reinterpret_cast<Next*>(w + p.nexts);
    auto* sums = reinterpret_cast<uint64_t*>(w + p.sums);
    auto* parts = reinterpret_cast<Part*>(w + p.parts);
    const int segments = segments_of(a.vocab, kThreads * EPT);
    const int64_t slots = a.drafts + 1 + (a.draft && a.k ? a.drafts : 0);
    const unsigned grid = (unsigned)(slots * a.rows * segments);
    if (a.k == 0) {
        k_verify_sums<T, EPT, true><<<grid, kThreads, 0, st>>>(a, segments, parts, nexts, arrived);
        return (int)hipGetLastError();
    }
    k_verify_sums<T, EPT, false><<<grid, kThreads, 0, st>>>(a, segments, parts, nexts, arrived);
    if (int e = (int)hipGetLastError()) return e;
    k_verify_next<T, EPT><<<(unsigned)(a.rows * segments), kThreads, 0, st>>>(a, segments, sums,
                                                                            nexts, arrived);
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
