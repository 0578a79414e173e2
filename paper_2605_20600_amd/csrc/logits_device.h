// Rows of logits in registers, their order, and words that the blocks of a launch leave for
// each other (token_logprobs.hip, verify_drafts.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

namespace headkv {
namespace dev {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// Words that a block of another XCD reads: written through, and read past, the
// L2s, which are not coherent with each other.  (Fences instead, which write the
// whole L2 back: 256 rows of 65536 logits 133 us, of 1024 threads a block 489.)
__device__ __forceinline__ void publish(uint64_t* p, uint64_t v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t read(const uint64_t* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t pair(uint32_t a, uint32_t b) { return (uint64_t)b << 32 | a; }
__device__ __forceinline__ uint32_t first_of(uint64_t v) { return (uint32_t)v; }
__device__ __forceinline__ uint32_t second_of(uint64_t v) { return (uint32_t)(v >> 32); }

// Order of logits: larger keys first; 0 is below every logit.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);  // -0 equals 0
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t key_of(uint32_t order, int index) {
    return (uint64_t)order << 32 | (uint32_t)~index;
}

template <typename T, int kThreads, int kEpt>
struct Logits {
    static constexpr int N = 16 / sizeof(T);  // of a vector
    static constexpr int NV = kEpt / N;       // vectors of a thread
    u32x4_t w[NV];

    __device__ __forceinline__ float at(int v, int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[v][e]);
        else return __uint_as_float(e & 1 ? w[v][e / 2] & 0xffff0000u : w[v][e / 2] << 16);
    }
    // Vector v of thread tid: elements j0 = (v kThreads + tid) N .. of the
    // segment, which starts at the 16-byte boundary p; those outside [lo, hi)
    // are -inf.
    __device__ __forceinline__ void load(const T* p, int lo, int hi, int tid) {
        constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int j0 = (v * kThreads + tid) * N;
            w[v] = u32x4_t{kNone, kNone, kNone, kNone};
            if (j0 >= lo && j0 + N <= hi) {
                w[v] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p + j0));
            } else if (j0 + N > lo && j0 < hi) {  // an end of the row
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (j0 + e < lo || j0 + e >= hi) continue;
                    const uint32_t x = p[j0 + e];
                    if constexpr (sizeof(T) == 4) w[v][e] = x;
                    else w[v][e / 2] = e & 1 ? (w[v][e / 2] & 0xffffu) | x << 16
                                             : (w[v][e / 2] & 0xffff0000u) | x;
                }
            }
        }
    }
};

}  // namespace dev
}  // namespace headkv
