// Log probabilities of given tokens, entropy, rank and the most likely
// alternatives.  One block per row, with y = x / temperature and m its largest:
//   log p_t = (y_t - m) - log S,  S = sum exp(y - m),
//   entropy = log S - sum exp(y - m) (y - m) / S,
// then the alternatives one after the other: the largest of the keys (value,
// lowest index first) below the one before.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "paged.h"

namespace headkv {
namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ float value(T x);
template <>
__device__ __forceinline__ float value<uint16_t>(uint16_t x) {
    return __uint_as_float((uint32_t)x << 16);
}
template <>
__device__ __forceinline__ float value<float>(float x) {
    return x;
}

// Order of logits and indices: larger keys first (value down, index up).
__device__ __forceinline__ uint64_t key_of(float x, int index) {
    uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);  // -0 equals 0
    u = u >> 31 ? ~u : u | 0x80000000u;
    return (uint64_t)u << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(uint64_t k) {
    uint32_t u = (uint32_t)(k >> 32);
    u = u >> 31 ? u & 0x7fffffffu : ~u;
    return __uint_as_float(u);
}

template <typename V, typename F>
__device__ V block_reduce(V v, F f) {
    __shared__ V part[kThreads];
    __syncthreads();
    part[threadIdx.x] = v;
    __syncthreads();
    for (int n = kThreads / 2; n > 0; n /= 2) {
        if ((int)threadIdx.x < n) part[threadIdx.x] = f(part[threadIdx.x], part[threadIdx.x + n]);
        __syncthreads();
    }
    return part[0];
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_token_logprobs(ScoreArgs a) {
    const int r = blockIdx.x;
    const T* x = static_cast<const T*>(a.logits) + r * a.row_stride;
    const int token = a.tokens[r];
    const bool has = token >= 0 && token < a.vocab;
    const float xt = has ? value(x[token]) : 0.f;
    float m = -INFINITY;
    bool ok = true;
    for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
        const float v = value(x[i]);
        m = fmaxf(m, v);
        ok = ok && v < INFINITY;
    }
    m = block_reduce(m, [](float p, float q) { return fmaxf(p, q); });
    ok = block_reduce((int)ok, [](int p, int q) { return p & q; });
    const float m0 = m == -INFINITY ? 0.f : m;
    float s = 0.f, t = 0.f;
    int above = 0;
    for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
        const float v = value(x[i]), y = (v - m0) * a.scale, e = expf(y);
        s += e;
        if (e > 0.f) t = fmaf(e, y, t);
        above += v > xt;
    }
    auto add = [](auto p, auto q) { return p + q; };
    s = block_reduce(s, add);
    t = block_reduce(t, add);
    above = block_reduce(above, add);
    const float ls = logf(s);
    auto logprob = [&](float v) { return v == -INFINITY ? v : (v - m0) * a.scale - ls; };
    if (threadIdx.x == 0) {
        a.logprob[r] = !ok ? NAN : has ? logprob(xt) : -INFINITY;
        if (a.entropy) a.entropy[r] = !ok ? NAN : s > 0.f ? ls - t / s : 0.f;
        if (a.rank) a.rank[r] = ok && has ? above : -1;
    }
    uint64_t last = ~0ull;
    for (int j = 0; j < a.top; ++j) {
        uint64_t best = 0;
        for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
            const uint64_t k = key_of(value(x[i]), i);
            if (k < last && k > best) best = k;
        }
        best = block_reduce(best, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
        if (threadIdx.x == 0) {
            a.top_logprob[(int64_t)r * a.top + j] = ok ? logprob(key_value(best)) : NAN;
            a.top_index[(int64_t)r * a.top + j] = ok ? (int)~(uint32_t)best : -1;
        }
        last = best;
    }
}

}  // namespace

size_t logprobs_workspace(int, int, int) { return 0; }

int launch_token_logprobs(const ScoreArgs& a, int logits_type, void*, void* stream) {
    if (logits_type == HEADKV_LOGITS_BF16)
        k_token_logprobs<uint16_t><<<a.rows, kThreads, 0, (hipStream_t)stream>>>(a);
    else
        k_token_logprobs<float><<<a.rows, kThreads, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

}  // namespace headkv
