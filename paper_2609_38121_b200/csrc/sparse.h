// Arguments of the sparse decode kernel, and its launches by code width (a source file each: sparse_2bit.cu and so on).
#pragma once
#include <cuda_runtime.h>

#include "layout.cuh"
#include "prologue.cuh"

namespace wushkv {

constexpr int MAX_SELECT_PAGES = 16384;      // candidate pages of a sequence (1 048 576 tokens): their keys are ranked in one CTA's shared memory

struct SparseParams {
    CacheView c;
    int batch;
    const int* slot;
    const int* seq_len;
    const unsigned short* Q;
    Prologue pro;                            // pro.rope != nullptr: Q holds projected queries
    const signed char* bounds;               // [n_pages][n_kv][2][D]: lower, upper; nullptr: the list is an input
    const signed char* exponents;            // [n_pages][n_kv]
    int n_select;
    int* selected;                           // [batch][n_kv][n_select]
    unsigned short* O;                       // bf16 [batch][n_q][D]; nullptr: selection alone
    int max_candidates;                      // bound of the candidate pages, from the bound of the lengths
    int stream_pages;                        // 1: the packed pages of a step cannot stay in L2 anyway: copy them with an evict-first hint
    int ring_offset;                         // where the staging rings begin behind the shared structure: 0 (they follow the scores in time) or behind the scores
};

int launch_sparse_2bit(const SparseParams& P, cudaStream_t st);
int launch_sparse_3bit(const SparseParams& P, cudaStream_t st);
int launch_sparse_4bit(const SparseParams& P, cudaStream_t st);

}  // namespace wushkv
