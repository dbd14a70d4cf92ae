// Page selection for sparse decode attention: what sparse.cu offers to decode.cu.
#pragma once
#include <cuda_runtime.h>

#include "layout.cuh"
#include "prologue.cuh"

namespace wushkv {

constexpr int MAX_SELECT_PAGES = 16384;      // candidate pages of a sequence (1 048 576 tokens): their keys are ranked in one CTA's shared memory

struct SelectParams {
    CacheView c;
    int batch;
    const int* slot;
    const int* seq_len;
    const unsigned short* Q;
    Prologue pro;                            // pro.rope != nullptr: Q holds projected queries
    const signed char* bounds;               // [n_pages][n_kv][2][D]: lower, upper
    const signed char* exponents;            // [n_pages][n_kv]
    int n_select;
    int* selected;                           // [batch][n_kv][n_select]
    int max_candidates;                      // bound of the candidate pages, from the bound of the lengths
    int early;                               // 1: a kernel ahead has waited for everything that this one reads
};

// Upper bound of the packed pages of a sequence of at most max_seq_len tokens.
inline long long candidate_bound(const CacheView& c, int max_seq_len) {
    const int nq = n_quantized(max_seq_len - c.lag, c.s_sink, c.s_keep, c.s_flush);
    return nq > 0 ? (c.s_sink + nq - 1) / PAGE_TOKENS - c.s_sink / PAGE_TOKENS + 1 : 0;
}

// Enqueues the selection; WUSHKV_OK, WUSHKV_ECAPACITY (too many candidates) or WUSHKV_ECUDA.
int launch_select(SelectParams P, int max_seq_len, cudaStream_t stream);

}  // namespace wushkv
