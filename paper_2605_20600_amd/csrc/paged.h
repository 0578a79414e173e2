// Layout of a paged cache and the launchers of its kernels (paged_cache.hip,
// paged_attn.hip) and of the token scores (token_logprobs.hip).  Launchers
// return a hipError_t as an int, or kTooLarge; paged_abi.cpp has validated what they
// get.
//
// A page holds page_tokens tokens of one key/value head:
//   K rows     [token][d]: a token's key, contiguous (FP4: dim 2 i in the low
//              half of byte i, 2 i + 1 in the high half)
//   V cells    [token / 8][cell][token % 8]: eight consecutive tokens of one dim
//              (FP4: of two dims, as in a K byte) are contiguous, which is how a
//              matrix instruction takes V^T (a lane holds eight tokens of a dim)
//   K scales   INT8 [token] bf16; FP4 [token][d / 32] exponent bytes
//   V scales   INT8 [token] bf16; FP4 [d / 32][token] exponent bytes
// An exponent byte e stands for 2^(e - 127), 255 for NaN.
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/headkv.h"

namespace headkv {

constexpr int kTooLarge = -1;  // more blocks than a call may launch

struct PagedDims {
    int type, d, heads, group;
    int ptok, pshift;  // tokens of a page, and their log2
    int num_pages;
    int v_off, ks_off, vs_off;  // bytes from the page's start
    int64_t page_bytes;
};

struct PagedLists {
    const int32_t* pages;
    const int32_t* len;
    const int32_t* first;
    const int32_t* order;
    int lists, max_pages, extra, max_len;
};

// Counters at the start of a workspace, zero between launches.  Their number does
// not depend on a call's sizes, so calls of any sizes can share a workspace: what
// lies behind them, which no launch expects to find in any state, never comes to
// lie on them.  A call with more than so many lists or rows runs in several
// launches.
constexpr int kCounters = 1 << 16;
constexpr size_t kCounterBytes = kCounters * sizeof(int32_t);

struct PagedRows {  // bf16 rows of the caller: element strides
    int64_t list, token, head;
};

int launch_paged_write(const PagedDims& c, char* pool, const PagedLists& l, const uint16_t* k,
                       const uint16_t* v, const PagedRows& r, int tokens, const int32_t* counts,
                       void* stream);
int launch_paged_read(const PagedDims& c, const char* pool, const PagedLists& l, int begin,
                      int tokens, uint16_t* k, uint16_t* v, const PagedRows& r, void* stream);

size_t paged_attn_workspace(const PagedDims& c, const PagedLists& own, const PagedLists* shared);
int launch_paged_attn(const PagedDims& c, const char* pool, const PagedLists& own,
                      const PagedLists* shared, const int32_t* share, const uint16_t* q,
                      int64_t q_stride, float* out, float* lse, void* ws, void* stream);

struct ScoreArgs {
    const void* logits;
    const int32_t* tokens;
    float *logprob, *entropy;
    int32_t* rank;
    float* top_logprob;
    int32_t* top_index;
    int64_t row_stride;
    int rows, vocab, top;
    float scale;  // 1 / temperature
};
size_t logprobs_workspace(int rows, int vocab, int top);
int launch_token_logprobs(const ScoreArgs& a, int logits_type, void* ws, void* stream);

}  // namespace headkv
