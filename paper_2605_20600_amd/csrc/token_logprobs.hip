// Log probabilities of given tokens, entropy, rank and the most likely
// alternatives (formulas: headkv.h), in one pass over the logits.
//
// With y = (x - m) / temperature and m the largest logit,
//   log p_t = y_t - log S,  S = sum exp(y),  entropy = log S - sum exp(y) y / S.
// A block takes a segment of a row into registers (aligned 16-byte loads), finds
// its maximum, then the sums relative to it and the number of logits above the
// token's.  The segments of a row meet in the block that finishes last.
//
// Alternatives: a segment is 256 groups of up to 64 logits.  With T such that from
// `top` to kMaxTop groups have their maximum at T or above, at least `top` values
// are >= T and all of them belong to those groups, so few are left to rank
// whatever the distribution.  T is found by bisection on order-preserving
// integers, counting with ballots, from the least maximum of 32 sets of groups
// on; where equal maxima leave no such T, it is the one below which too few are
// left, and of the values equal to it the first in index order are taken.
//
// One MI355X: 18816 rows of 16384 fp32 logits 181 us, 6.8 TB/s, bound by the bytes; 256
// rows of 65536 bf16 logits with 20 alternatives 18 us, of which the bytes take 5: the
// load, the bisection, ranking the candidates and the join of a row's segments wait for
// each other (13 without alternatives); 20000 rows of 2000 bf16 logits with 5 52 us (33
// without), of which the bytes take 16: what a block costs for 4 KB; 1000 rows of 130000
// with 20 121 us (69); 8 rows of 16384 7 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "logits_device.h"
#include "paged.h"

namespace headkv {
namespace {

using namespace dev;

constexpr int kCus = 256;
constexpr int kMaxSegment = 16384;  // logits of a block
constexpr int kMaxTop = HEADKV_MAX_TOP;
constexpr int kGroups = 256;

// What a block knows of its segment: the maximum and the sum of 2^y, the sum of
// 2^y y (y in log2 units) and the number of logits above the token's.
struct Part {
    uint64_t w[2];
};

constexpr float kLog2e = 1.4426950408889634f;

// What exponents y = (x - m) / temperature, in log2 units, are computed from.  Near:
// y = x k - mk with mk = m k rounded once for all, which shifts every y by what it was
// rounded, left().  That is up to half a unit in the last place of mk: 1/2 at 2^24, where
// near ends, 128 and so past exp2's range at 2^31.  Far: (x - m) / temperature, shifted
// by nothing.  (Far if mk or k alone is no number, too.)
struct Reference {
    float m, mk;
    bool far;
    __device__ __forceinline__ Reference(float most, float k) : m(most) {
#pragma clang fp contract(off)
        mk = m == -INFINITY ? 0.f : m * k;  // (0 for an empty maximum)
        far = !(fabsf(mk) < 0x1p24f);
    }
    __device__ __forceinline__ float left(float k) const {
        return far || m == -INFINITY ? 0.f : fmaf(m, k, -mk);
    }
};

template <typename F>
__device__ __forceinline__ float wave_reduce(float v, F f) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v = f(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }

// The `top` largest of n keys in LDS, largest first, through out(rank, key): by
// counting the larger ones while few, else one after the other.  Every thread
// calls it; `scratch`: a key per wavefront.
template <int kThreads, typename Out>
__device__ __forceinline__ void select_top(const uint64_t* keys, int n, int top,
                                           uint64_t* scratch, int tid, Out out) {
    constexpr int kWaves = kThreads / 64;
    if (n <= kThreads) {
        if (tid < n) {
            const uint64_t mine = keys[tid];
            int rank = 0;
            for (int i = 0; i < n; ++i) rank += keys[i] > mine;
            if (rank < top) out(rank, mine);
        }
        return;
    }
    uint64_t last = ~0ull;
    for (int j = 0; j < top; ++j) {
        uint64_t best = 0;
        for (int i = tid; i < n; i += kThreads)
            if (keys[i] < last && keys[i] > best) best = keys[i];
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const uint64_t other = __shfl_xor((unsigned long long)best, o);
            best = other > best ? other : best;
        }
        __syncthreads();
        if ((tid & 63) == 0) scratch[tid >> 6] = best;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) best = scratch[w] > best ? scratch[w] : best;
        if (tid == 0) out(j, best);
        last = best;
    }
}

// (32 bf16 logits a thread: in as few registers as four blocks of a CU may have; with
// three, 256 rows of 65536 with 20 alternatives took 23 us instead of 18.5, 1000 of 130000
// 145 instead of 121, without alternatives 78 instead of 69.)
template <typename T, int kThreads, int kEpt>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kEpt == 32 && sizeof(T) == 2 ? 8 : 4)))
void k_token_logprobs(ScoreArgs a, int segments, Part* parts, uint64_t* part_keys, int* arrived) {
    using Values = Logits<T, kThreads, kEpt>;
    constexpr int N = Values::N, NV = Values::NV, kSegment = kThreads * kEpt;
    constexpr int kGroupMost = kMaxTop * (kSegment / kGroups);  // logits of kMaxTop groups
    constexpr int kCandidates = kGroupMost + kMaxTop > 512 ? kGroupMost + kMaxTop : 512;
    constexpr int kWaves = kThreads / 64;
    constexpr int kPerGroup = kThreads / kGroups, kPerSet = kThreads / kMaxTop;  // threads
    __shared__ float red[3][kWaves];
    __shared__ int ired[2][kWaves];
    __shared__ uint32_t maxima[kGroups], sets[kMaxTop];
    __shared__ uint64_t keys[kCandidates];
    __shared__ uint64_t scratch[kWaves], kept[kMaxTop];
    __shared__ int count;
    __shared__ uint32_t threshold[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = blockIdx.x / segments, seg = blockIdx.x % segments;
    const T* row = static_cast<const T*>(a.logits) + r * a.row_stride;
    // element j of the row's segments is logit j - lead: vectors are aligned
    const int lead = (int)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
    const int begin = seg * kSegment;
    const int lo = max(lead - begin, 0), hi = min(a.vocab + lead - begin, kSegment);
    Values x;
    x.load(row - lead + begin, lo, hi, tid);

    const int token = a.tokens[r];
    const bool has = token >= 0 && token < a.vocab;
    float xt = 0.f;
    if (has) {
        const T w = row[token];
        xt = sizeof(T) == 4 ? __uint_as_float((uint32_t)w) : __uint_as_float((uint32_t)w << 16);
    }
    const float k = a.scale * kLog2e;  // to log2 units

    float mine = -INFINITY;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < N; ++e) mine = fmaxf(mine, x.at(v, e));
    // of the thread, its group and its set; 0: no logits
    uint32_t om = tid * N < hi ? order_of(mine) : 0u, group = om;
#pragma unroll
    for (int o = 1; o < kPerSet; o *= 2) {
        if (o == kPerGroup) group = om;
        om = max(om, (uint32_t)__shfl_xor((int)om, o));
    }
    if (tid % kPerGroup == 0) maxima[tid / kPerGroup] = group;
    if (tid % kPerSet == 0) sets[tid / kPerSet] = om;
    float m = wave_reduce(mine, fmaxf);
    if (lane == 0) red[0][wave] = m;
    if (tid == 0) count = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, red[0][w]);

    // NaN and +inf in the segment make s NaN.
    auto scaled = [&](float d) { return d * a.scale * kLog2e; };
    const Reference own(m, k);
    float s = 0.f, t = 0.f;
    int above = 0;  // of the wavefront
    auto sums = [&](auto far) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float xv = x.at(v, e);
                const float y = decltype(far)::value ? scaled(xv - m) : fmaf(xv, k, -own.mk);
                const float p = __builtin_amdgcn_exp2f(y);
                s += p;
                t = fmaf(p, fmaxf(y, -1e30f), t);
                above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(xv > xt));
            }
    };
    if (__builtin_amdgcn_readfirstlane(own.far)) sums(std::true_type{});
    else sums(std::false_type{});
    s = wave_reduce(s, add);
    t = wave_reduce(t, add);
    if (lane == 0) {
        red[1][wave] = s;
        red[2][wave] = t;
        ired[0][wave] = above;
    }

    int n = 0;  // candidates
    if (a.top) {
        if (wave == 0) {
            uint32_t mx[kGroups / 64];
#pragma unroll
            for (int w = 0; w < kGroups / 64; ++w) mx[w] = maxima[64 * w + lane];
            // every set has a group at or above the least of them
            uint32_t low = sets[lane % kMaxTop];
#pragma unroll
            for (int o = 1; o < kMaxTop; o *= 2) low = min(low, (uint32_t)__shfl_xor((int)low, o));
            low = __builtin_amdgcn_readfirstlane(a.top == 1 ? order_of(m) : low);
            uint32_t high = order_of(m) + 1;  // groups at or above: >= top, < top
            auto groups = [&](uint32_t at) {
                int c = 0;
#pragma unroll
                for (int w = 0; w < kGroups / 64; ++w)
                    c += __builtin_popcountll(__builtin_amdgcn_ballot_w64(mx[w] >= at));
                return c;
            };
            bool few = low > 0 && groups(low) <= kMaxTop;
            while (!few && high - low > 1) {
                const uint32_t mid = low + (high - low) / 2;
                const int c = groups(mid);
                if (c < a.top) {
                    high = mid;
                } else {
                    low = mid;
                    few = c <= kMaxTop;
                }
            }
            if (lane == 0) {
                threshold[0] = few ? low - 1 : low;  // candidates are above this
                threshold[1] = few ? 0 : low;        // and of these the first, if any
            }
        }
        __syncthreads();
        const uint32_t over = threshold[0], equal = threshold[1];
        if (group > over) {
            const float least = value_of(max(over + 1, order_of(-INFINITY)));
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (!(x.at(v, e) >= least)) continue;
                    const int j = (v * kThreads + tid) * N + e;
                    if (j < lo || j >= hi) continue;
                    const int at = atomicAdd(&count, 1);
                    if (at < kGroupMost)
                        keys[at] = key_of(order_of(x.at(v, e)), begin + j - lead);
                }
        }
        __syncthreads();
        n = min(count, kGroupMost);
        if (equal > 0 && n < a.top) {  // the first values equal to T
            int want = a.top - n;
#pragma unroll 1
            for (int v = 0; v < NV && want > 0; ++v) {
                u32x4_t w = x.w[0];
#pragma unroll
                for (int i = 1; i < NV; ++i) w = v == i ? x.w[i] : w;
                const int j0 = (v * kThreads + tid) * N;
                uint32_t ties = 0;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float f = sizeof(T) == 4 ? __uint_as_float(w[e % 4])
                                    : __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
                    ties |= (uint32_t)(order_of(f) == equal && j0 + e >= lo && j0 + e < hi) << e;
                }
                int sum = __builtin_popcount(ties);
#pragma unroll
                for (int o = 1; o < 64; o *= 2) {
                    const int up = __shfl_up(sum, o);
                    if (lane >= o) sum += up;
                }
                if (lane == 63) ired[1][wave] = sum;
                __syncthreads();
                int before = sum - __builtin_popcount(ties), total = 0;
#pragma unroll
                for (int i = 0; i < kWaves; ++i) {
                    if (i < wave) before += ired[1][i];
                    total += ired[1][i];
                }
                for (int e = 0; e < N; ++e) {
                    if (!(ties >> e & 1)) continue;
                    if (before < want) keys[n + before] = key_of(equal, begin + j0 + e - lead);
                    ++before;
                }
                total = min(total, want);
                n += total;
                want -= total;
                __syncthreads();
            }
        }
    }
    __syncthreads();
    s = t = 0.f;
    above = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        s += red[1][w];
        t += red[2][w];
        above += ired[0][w];
    }

    if (segments > 1) {
        // the segment's part, then the last block of the row goes on with all
        const int64_t at = (int64_t)r * segments + seg;
        if (a.top) {
            uint64_t* mine_keys = part_keys + at * a.top;
            if (tid < a.top && tid >= n) publish(mine_keys + tid, 0);  // fewer logits than asked
            select_top<kThreads>(keys, n, a.top, scratch, tid, [&](int i, uint64_t key) {
                if (i < a.top) publish(mine_keys + i, key);
            });
        }
        if (tid == 0) {
            publish(parts[at].w, pair(__float_as_uint(m), __float_as_uint(s)));
            publish(parts[at].w + 1, pair(__float_as_uint(t), (uint32_t)above));
        }
        // every published word has left before the block counts as arrived
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) {
            const int got = __hip_atomic_fetch_add(arrived + r, 1, __ATOMIC_RELAXED,
                                                   __HIP_MEMORY_SCOPE_AGENT);
            count = got == segments - 1;
            if (count)  // as it was found
                __hip_atomic_store(arrived + r, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!count) return;
        const Part* p = parts + (int64_t)r * segments;
        // each wavefront for itself, 64 segments at a time
        m = -INFINITY;
        for (int i = lane; i < segments; i += 64) m = fmaxf(m, __uint_as_float(first_of(read(p[i].w))));
        m = wave_reduce(m, fmaxf);
        const Reference all(m, k);
        s = t = 0.f;
        above = 0;
        for (int i = lane; i < segments; i += 64) {
            const uint64_t u = read(p[i].w), v = read(p[i].w + 1);
            const float pm = __uint_as_float(first_of(u)), ps = __uint_as_float(second_of(u));
            const float pt = __uint_as_float(first_of(v));
            above += (int)second_of(v);
            // from the segment's reference, which may be the other kind, to the row's
            const Reference part(pm, k);
            float shift = part.mk - all.mk;
            if (__builtin_expect(part.far || all.far, 0)) {
                asm volatile("");  // a branch, which ordinary rows do not take
                shift = scaled(pm - m) + (all.left(k) - part.left(k));
            }
            if (pm == -INFINITY) shift = 0.f;  // nothing but -inf: ps is 0, or NaN
            const float f = __builtin_amdgcn_exp2f(shift);
            s = fmaf(f, ps, s);
            t = fmaf(f, fmaf(fmaxf(shift, -1e30f), ps, pt), t);
        }
        s = wave_reduce(s, add);
        t = wave_reduce(t, add);
#pragma unroll
        for (int o = 1; o < 64; o *= 2) above += __shfl_xor(above, o);
        if (a.top) {
            n = 0;
            const uint64_t* in = part_keys + (int64_t)r * segments * a.top;
            const int all = segments * a.top;
            __syncthreads();
            if (all <= kCandidates) {
                for (int i = tid; i < all; i += kThreads) keys[i] = read(in + i);
                n = all;
            } else {  // too many for LDS at once: segment after segment into the best so far
                for (int i = 0; i < segments; ++i) {
                    if (tid < a.top) keys[n + tid] = read(in + (int64_t)i * a.top + tid);
                    n += a.top;
                    __syncthreads();
                    if (n + a.top > kCandidates || i == segments - 1) {
                        if (tid < a.top) kept[tid] = 0;
                        __syncthreads();
                        select_top<kThreads>(keys, n, a.top, scratch, tid, [&](int j, uint64_t key) {
                            if (key) kept[j] = key;
                        });
                        __syncthreads();
                        if (tid < a.top) keys[tid] = kept[tid];
                        n = a.top;
                        __syncthreads();
                    }
                }
            }
            __syncthreads();
        }
    }

    const bool ok = s == s && m < INFINITY;
    constexpr float kLn2 = 0.6931471805599453f;
    const float log_s = __builtin_amdgcn_logf(s);  // log2
    const float log_true = log_s - Reference(m, k).left(k);
    auto logprob = [&](float v) {
        if (v == -INFINITY) return v;
        float y = (v - m) * a.scale;
        if (v - m == -INFINITY) y = (0.5f * v - 0.5f * m) * a.scale * 2.f;  // its half is a number
        return y - log_true * kLn2;
    };
    if (tid == 0) {
        a.logprob[r] = !ok ? NAN : has ? logprob(xt) : -INFINITY;
        if (a.entropy) a.entropy[r] = !ok ? NAN : s > 0.f ? (log_s - t / s) * kLn2 : 0.f;
        if (a.rank) a.rank[r] = ok && has ? above : -1;
    }
    if (a.top && !ok) {
        if (tid < a.top) {
            a.top_logprob[(int64_t)r * a.top + tid] = NAN;
            a.top_index[(int64_t)r * a.top + tid] = -1;
        }
    } else if (a.top) {
        select_top<kThreads>(keys, n, a.top, scratch, tid, [&](int i, uint64_t key) {
            const int64_t o = (int64_t)r * a.top + i;
            a.top_logprob[o] = logprob(value_of((uint32_t)(key >> 32)));
            a.top_index[o] = (int)~(uint32_t)key;
        });
    }
}

// Segments of a row that starts up to `lead` logits into a vector.
int segments_of(int vocab, int lead) { return (vocab + lead + kMaxSegment - 1) / kMaxSegment; }

struct ScorePlan {
    size_t parts, keys, bytes;  // offsets, and the total
};

ScorePlan plan_of(int rows, int vocab, int top) {
    const size_t segments = segments_of(vocab, 7);
    ScorePlan p{};
    if (segments > 1) {
        const size_t n = std::min(rows, kCounters) * segments;
        p.parts = kCounterBytes;
        p.keys = p.parts + n * sizeof(Part);
        p.bytes = p.keys + n * top * sizeof(uint64_t);
    }
    return p;
}

}  // namespace

size_t logprobs_workspace(int rows, int vocab, int top) { return plan_of(rows, vocab, top).bytes; }

int launch_token_logprobs(const ScoreArgs& all, int logits_type, void* ws, void* stream) {
    const ScorePlan p = plan_of(all.rows, all.vocab, all.top);
    const int size = logits_type == HEADKV_LOGITS_BF16 ? 2 : 4;
    const bool even = reinterpret_cast<uintptr_t>(all.logits) % 16 == 0 &&
                      (all.rows == 1 || all.row_stride * size % 16 == 0);
    const int lead = even ? 0 : 16 / size - 1;
    const int segments = segments_of(all.vocab, lead);
    char* w = static_cast<char*>(ws);
    auto* parts = reinterpret_cast<Part*>(w + p.parts);
    auto* keys = reinterpret_cast<uint64_t*>(w + p.keys);
    auto* arrived = reinterpret_cast<int*>(w);
    hipStream_t st = (hipStream_t)stream;
    // (fewer than 2^32 threads in a launch)
    const int most = std::min(segments > 1 ? kCounters : 1 << 22, (1 << 22) / segments);
    for (int r0 = 0; r0 < all.rows; r0 += most) {
        ScoreArgs a = all;
        a.rows = std::min(all.rows - r0, most);
        a.logits = static_cast<const char*>(all.logits) + r0 * all.row_stride * size;
        a.tokens += r0;
        a.logprob += r0;
        if (a.entropy) a.entropy += r0;
        if (a.rank) a.rank += r0;
        if (a.top) {
            a.top_logprob += (int64_t)r0 * a.top;
            a.top_index += (int64_t)r0 * a.top;
        }
        const int64_t grid = (int64_t)a.rows * segments;
        auto run = [&](auto kernel, int threads) {
            kernel<<<(unsigned)grid, threads, 0, st>>>(a, segments, parts, keys, arrived);
        };
        // The smallest segment that holds a row, so that no lane is idle; few blocks
        // have as many threads as possible, for latency.
        const int least = a.vocab + lead;
        auto pick = [&](auto type) {
            using T = decltype(type);
            if (least <= 2048) run(k_token_logprobs<T, 256, 8>, 256);
            else if (least <= 4096) run(k_token_logprobs<T, 256, 16>, 256);
            else if (least <= 8192) run(k_token_logprobs<T, 512, 16>, 512);
            else if (grid <= 2 * kCus) run(k_token_logprobs<T, 1024, 16>, 1024);
            else run(k_token_logprobs<T, 512, 32>, 512);
        };
        if (logits_type == HEADKV_LOGITS_BF16) pick(uint16_t{});
        else pick(uint32_t{});
        if (int e = (int)hipGetLastError()) return e;
    }
    return 0;
}

}  // namespace headkv
