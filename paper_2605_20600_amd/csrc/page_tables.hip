// Page tables brought from one step to the next (what is done: headkv.h).
//
// A list's places are looked at by four threads, a quarter each: one that ends has many.  A
// prefix sum over the threads says where each puts the pages that it frees, and after all of
// them are in the ring a second one which ones it takes.  Few lists are one block's work, in
// one launch; many are cut among blocks, which count in a first launch, free in a second and
// take in a third.  The start order is a stable counting sort by a key of 8 bits, a block for
// each layer, beside the last part.  Bound by the loads that wait for each other, and the
// launches: a few words are read and written for a list.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "paged.h"

namespace headkv {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kParts = 4, kLists = kThreads / kParts;  // threads of a list, lists of a block's turn
constexpr int kBlocks = 512;  // at most, of many lists
constexpr int kMostSorts = 4096;  // blocks that sort layers
constexpr int kKeys = 256;

struct Call {
    headkv_paged_tables t;
    const int32_t* advance;
    const int32_t* counts;
    int tokens, shift;  // log2 of page_tokens
    int lists;          // lists * kv_heads
    int per_layer;      // of those, of a layer
    int blocks, chunk;  // that the lists are cut among, and lists of each
};

// What the launches leave for each other.
struct Shared {
    uint32_t head, count;        // the ring as it was
    uint32_t frees[kBlocks], needs[kBlocks];
};

// A list before and after the step.
struct List {
    int len, first, before, n;
    bool ends;
};

__device__ __forceinline__ List list_at(const Call& c, int i) {
    const headkv_paged_tables& t = c.t;
    const int row = i / t.kv_heads % t.rows;
    List l;
    const int gained = c.advance ? c.advance[row] : 0;
    l.n = c.counts ? min(max(c.counts[row], 0), c.tokens) : c.tokens;
    l.ends = gained < 0;
    const int64_t len = (int64_t)max(t.len[i], 0) + gained;
    l.len = l.ends ? 0 : (int)min(len, (int64_t)t.max_pages << c.shift);
    l.before = l.ends ? 0 : max(t.first[i], 0);
    l.first = l.before;
    const int w = t.window ? t.window[i] : 0;
    if (w > 0) l.first = max(l.first, l.len + 1 - w);
    return l;
}

__device__ __forceinline__ bool held(const Call& c, int page) {
    return (uint32_t)page < (uint32_t)c.t.num_pages;
}

// f(place, page number) for the thread's part of places [p0, p1) of list i's table, the
// loads of eight at a time in flight.
template <typename F>
__device__ __forceinline__ void places(const Call& c, int i, int p0, int p1, F f) {
    const int32_t* table = c.t.pages + (int64_t)i * c.t.max_pages;
    p1 = min(p1, c.t.max_pages);
    if (p0 >= p1) return;
    const int n = p1 - p0, part = threadIdx.x % kParts;  // the thread's part of them
    p1 = p0 + (int)((int64_t)n * (part + 1) / kParts);
    p0 += (int)((int64_t)n * part / kParts);
    for (int p = p0; p < p1; p += 8) {
        int page[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) page[x] = table[min(p + x, p1 - 1)];
#pragma unroll
        for (int x = 0; x < 8; ++x)
            if (p + x < p1) f(p + x, page[x]);
    }
}
// The places whose pages list i frees.
template <typename F>
__device__ __forceinline__ void freed_places(const Call& c, int i, const List& l, F f) {
    if (l.ends) places(c, i, 0, c.t.max_pages, f);
    else places(c, i, l.before >> c.shift, l.first >> c.shift, f);
}
// The places that the next tokens of a list of `len` start on.
template <typename F>
__device__ __forceinline__ void next_places(const Call& c, int i, int len, int n, F f) {
    const int up = (1 << c.shift) - 1;
    places(c, i, (len + up) >> c.shift, (len + n + up) >> c.shift, f);
}

__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
    return v;
}

// Sum over the block of v's below the thread's own; *total: of all.
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* total, uint32_t* scratch) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t up = v;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t y = __shfl_up(up, o);
        if (lane >= o) up += y;
    }
    if (lane == 63) scratch[wave] = up;
    __syncthreads();
    uint32_t below = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) below += scratch[w];
        all += scratch[w];
    }
    __syncthreads();
    *total = all;
    return below + up - v;
}

// Sum of the counts of blocks before `block`, and of all.
__device__ __forceinline__ void blocks_before(const uint32_t* counts, int blocks, int block,
                                              uint32_t* before, uint32_t* all, uint32_t* scratch) {
    const int i = threadIdx.x;
    const uint32_t v = i < blocks ? counts[i] : 0;
    const uint32_t below = block_before(v, all, scratch);
    __shared__ uint32_t found;
    if (i == block) found = below;
    __syncthreads();
    *before = found;
    __syncthreads();
}

// Lists [i0, i1) free their pages, the first of which is number `before` of all; lengths and
// windows become the new ones.  Returns the pages freed.
__device__ __forceinline__ uint32_t free_pages(const Call& c, int i0, int i1, uint32_t head,
                                               uint32_t count, uint32_t before, uint32_t* scratch) {
    const uint32_t size = c.t.num_pages, end = (uint32_t)(((uint64_t)head + count) % size);
    uint32_t all = 0;
    for (int base = i0; base < i1; base += kLists) {
        const int i = base + threadIdx.x / kParts;
        uint32_t mine = 0, total;
        List l;
        if (i < i1) {
            l = list_at(c, i);
            freed_places(c, i, l, [&](int, int page) { mine += held(c, page); });
        }
        uint32_t k = before + all + block_before(mine, &total, scratch);
        all += total;
        if (i >= i1) continue;
        int32_t* table = c.t.pages + (int64_t)i * c.t.max_pages;
        if (l.ends || mine)
            freed_places(c, i, l, [&](int p, int page) {
                if (held(c, page)) {
                    if (k < size - count) c.t.free_pages[((uint64_t)end + k) % size] = page;
                    ++k;
                    table[p] = -1;
                } else if (l.ends) {
                    table[p] = -1;
                }
            });
        if (threadIdx.x % kParts == 0) {  // (all have read them before the sum)
            c.t.len[i] = l.len;
            c.t.first[i] = l.first;
        }
    }
    return all;
}

__device__ __forceinline__ int tokens_next(const Call& c, int i) {
    const int row = i / c.t.kv_heads % c.t.rows;
    return c.counts ? min(max(c.counts[row], 0), c.tokens) : c.tokens;
}

// Lists [i0, i1), their lengths the new ones, take pages of a ring of `count`, the first of
// which is number `before` of all that are taken.  Returns the pages asked for.
__device__ __forceinline__ uint32_t take_pages(const Call& c, int i0, int i1, uint32_t head,
                                               uint32_t count, uint32_t before, uint32_t* scratch) {
    const uint32_t size = c.t.num_pages;
    uint32_t all = 0;
    for (int base = i0; base < i1; base += kLists) {
        const int i = base + threadIdx.x / kParts;
        uint32_t mine = 0, total;
        int len = 0, n = 0;
        if (i < i1) {
            len = c.t.len[i];
            n = tokens_next(c, i);
            next_places(c, i, len, n, [&](int, int page) { mine += !held(c, page); });
        }
        uint32_t k = before + all + block_before(mine, &total, scratch);
        all += total;
        if (mine == 0) continue;
        int32_t* table = c.t.pages + (int64_t)i * c.t.max_pages;
        next_places(c, i, len, n, [&](int p, int page) {
            if (held(c, page)) return;
            if (k < count) table[p] = c.t.free_pages[((uint64_t)head + k) % size];
            ++k;
        });
    }
    return all;
}

__device__ __forceinline__ void write_state(const Call& c, uint32_t head, uint32_t count,
                                            uint32_t asked) {
    const uint32_t given = min(count, asked);
    c.t.free_state[0] = (int)(((uint64_t)head + given) % c.t.num_pages);
    c.t.free_state[1] = (int)(count - given);
    c.t.free_state[2] = (int)(asked - given);
    c.t.free_state[3] = 0;
}

__device__ __forceinline__ void read_state(const Call& c, uint32_t* head, uint32_t* count) {
    *head = (uint32_t)c.t.free_state[0] % (uint32_t)c.t.num_pages;
    *count = (uint32_t)min(max(c.t.free_state[1], 0), c.t.num_pages);
}

// Tokens in eighths of an octave, 8 bits.
__device__ __forceinline__ int key_of(int n) {
    const int e = 31 - __builtin_clz(max(n, 8));
    return n < 8 ? max(n, 0) : (e - 2) * 8 + ((n >> (e - 3)) & 7);
}

struct Sort {
    int next[kKeys];           // where the next list of a key goes
    int found[kWaves][kKeys];  // lists of each key that a wavefront has
};

// The start order of a layer, lengths and windows being the new ones.
__device__ __forceinline__ void sort_layer(const Call& c, int layer, Sort& s, uint32_t* scratch) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int i0 = layer * c.per_layer;
    auto key_at = [&](int j) {
        const int i = i0 + j;
        return kKeys - 1 - key_of(c.t.len[i] + tokens_next(c, i) - c.t.first[i]);  // most first
    };
    if (tid < kKeys) s.next[tid] = 0;
    __syncthreads();
    for (int j = tid; j < c.per_layer; j += kThreads) atomicAdd(&s.next[key_at(j)], 1);
    __syncthreads();
    uint32_t total;
    const uint32_t below = block_before(tid < kKeys ? s.next[tid] : 0, &total, scratch);
    if (tid < kKeys) s.next[tid] = (int)below;
    for (int base = 0; base < c.per_layer; base += kThreads) {
        const int j = base + tid;
        const bool is = j < c.per_layer;
        const int key = is ? key_at(j) : 0;
        for (int x = tid; x < kWaves * kKeys; x += kThreads) (&s.found[0][0])[x] = 0;
        __syncthreads();
        uint64_t same = __builtin_amdgcn_ballot_w64(is);  // lanes of the same key
#pragma unroll
        for (int bit = 0; bit < 8; ++bit) {
            const uint64_t set = __builtin_amdgcn_ballot_w64(key >> bit & 1);
            same &= key >> bit & 1 ? set : ~set;
        }
        const int rank = __builtin_popcountll(same & ((1ull << lane) - 1));
        if (is && rank == 0) s.found[wave][key] = __builtin_popcountll(same);
        __syncthreads();
        if (is) {
            int at = s.next[key] + rank;
            for (int w = 0; w < wave; ++w) at += s.found[w][key];
            c.t.order[i0 + at] = j;
        }
        __syncthreads();
        if (tid < kKeys) {
            int n = s.next[tid];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) n += s.found[w][tid];
            s.next[tid] = n;
        }
        __syncthreads();
    }
}

// All of it, for few lists.
__global__ __launch_bounds__(kThreads) void k_extend(Call c) {
    __shared__ uint32_t scratch[kWaves];
    __shared__ Sort sort;
    uint32_t head, count;
    read_state(c, &head, &count);
    const uint32_t freed = free_pages(c, 0, c.lists, head, count, 0, scratch);
    __syncthreads();
    count = (uint32_t)min((uint64_t)count + freed, (uint64_t)c.t.num_pages);
    const uint32_t asked = take_pages(c, 0, c.lists, head, count, 0, scratch);
    if (threadIdx.x == 0) write_state(c, head, count, asked);
    if (c.t.order)
        for (int layer = 0; layer * c.per_layer < c.lists; ++layer) sort_layer(c, layer, sort, scratch);
}

// Many lists: what each block's free and ask for.
__global__ __launch_bounds__(kThreads) void k_extend_count(Call c, Shared* sh) {
    __shared__ int sums[2][kWaves];
    const int i0 = blockIdx.x * c.chunk, i1 = min(i0 + c.chunk, c.lists);
    int frees = 0, needs = 0;
    for (int i = i0 + threadIdx.x / kParts; i < i1; i += kLists) {
        const List l = list_at(c, i);
        freed_places(c, i, l, [&](int, int page) { frees += held(c, page); });
        next_places(c, i, l.len, l.n, [&](int, int page) { needs += l.ends || !held(c, page); });
    }
    frees = wave_sum(frees);
    needs = wave_sum(needs);
    if ((threadIdx.x & 63) == 0) {
        sums[0][threadIdx.x >> 6] = frees;
        sums[1][threadIdx.x >> 6] = needs;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        frees = needs = 0;
        for (int w = 0; w < kWaves; ++w) frees += sums[0][w], needs += sums[1][w];
        sh->frees[blockIdx.x] = frees;
        sh->needs[blockIdx.x] = needs;
        if (blockIdx.x == 0) read_state(c, &sh->head, &sh->count);
    }
}

__global__ __launch_bounds__(kThreads) void k_extend_free(Call c, const Shared* sh) {
    __shared__ uint32_t scratch[kWaves];
    uint32_t before, all;
    blocks_before(sh->frees, c.blocks, blockIdx.x, &before, &all, scratch);
    const int i0 = blockIdx.x * c.chunk;
    free_pages(c, i0, min(i0 + c.chunk, c.lists), sh->head, sh->count, before, scratch);
}

__global__ __launch_bounds__(kThreads) void k_extend_take(Call c, const Shared* sh) {
    __shared__ uint32_t scratch[kWaves];
    __shared__ Sort sort;
    if (blockIdx.x >= (unsigned)c.blocks) {
        const int step = gridDim.x - c.blocks;
        for (int layer = blockIdx.x - c.blocks; layer < c.lists / c.per_layer; layer += step)
            sort_layer(c, layer, sort, scratch);
        return;
    }
    uint32_t before, all, freed;
    blocks_before(sh->frees, c.blocks, 0, &before, &freed, scratch);
    const uint32_t count = (uint32_t)min((uint64_t)sh->count + freed, (uint64_t)c.t.num_pages);
    blocks_before(sh->needs, c.blocks, blockIdx.x, &before, &all, scratch);
    const int i0 = blockIdx.x * c.chunk;
    take_pages(c, i0, min(i0 + c.chunk, c.lists), sh->head, count, before, scratch);
    if (blockIdx.x == 0 && threadIdx.x == 0) write_state(c, sh->head, count, all);
}

// Lists up to which one block does all, in one turn (one block and three launches, every
// eighth list of 2480 tokens ending, in a graph: 512 lists 21 and 18 us, 1024 36 and 17, 2048
// 69 and 19, 65536 - and 25; 256 of which none ends 8 in one block).
constexpr int kFew = kLists;

}  // namespace

size_t extend_workspace() { return (sizeof(Shared) + 255) / 256 * 256; }

int launch_extend(const headkv_paged_tables& t, const int32_t* advance, const int32_t* counts,
                  int tokens, void* ws, void* stream) {
    Call c{};
    c.t = t;
    c.advance = advance;
    c.counts = counts;
    c.tokens = tokens;
    while ((1 << c.shift) < t.page_tokens) ++c.shift;
    c.lists = t.lists * t.kv_heads;
    c.per_layer = t.rows * t.kv_heads;
    hipStream_t st = (hipStream_t)stream;
    if (c.lists <= kFew) {
        k_extend<<<1, kThreads, 0, st>>>(c);
        return (int)hipGetLastError();
    }
    c.chunk = std::max(kLists, (c.lists + kBlocks - 1) / kBlocks);
    c.blocks = (c.lists + c.chunk - 1) / c.chunk;
    auto* sh = static_cast<Shared*>(ws);
    k_extend_count<<<c.blocks, kThreads, 0, st>>>(c, sh);
    if (int e = (int)hipGetLastError()) return e;
    k_extend_free<<<c.blocks, kThreads, 0, st>>>(c, sh);
    if (int e = (int)hipGetLastError()) return e;
    const int layers = t.order ? std::min(t.lists / t.rows, kMostSorts) : 0;
    k_extend_take<<<c.blocks + layers, kThreads, 0, st>>>(c, sh);
    return (int)hipGetLastError();
}

}  // namespace headkv
