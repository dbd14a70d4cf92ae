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
    // The selection of wushkv_decode_attn_sparse is also the query preparation of the attention: it writes what
    // decode_prep_kernel writes (see DecodeParams in decode.cu).  nullptr: selection alone.
    uint4* qfrag;
    uint4* qwfrag;
    float* qscal;
    long long* plan;                         // written if the main kernel does not make the plan itself; else nullptr
};

// Arrival counters of a (sequence, KV head)'s 8 query head slots for the main kernel's merge, zeroed by the kernel that prepares
// the queries: in the unused half of the head's integer fragments.
__device__ __forceinline__ int* arrival_counters(uint4* qfrag, long long bh) { return reinterpret_cast<int*>(qfrag + bh * 256 + 128); }

// How one sequence decomposes into work units (identical for all of its KV heads).
constexpr int WIN_TOKENS = 8;                // window tokens per work unit
struct SeqInfo {
    int slot;
    int q_lo, q_hi;          // positions read from the packed codes: [q_lo, q_hi)
    int first_page, qp;      // packed pages covering them
    int n_sink, recent_lo;   // window tokens: positions [0, n_sink) and [recent_lo, S)
    int n_win;               // window tokens
    int U;                   // qp + ceil(n_win / WIN_TOKENS)
};

__device__ __forceinline__ SeqInfo seq_info(const CacheView& c, int S, int slot) {
    SeqInfo si;
    si.slot = slot;
    if (S <= 0 || slot < 0 || slot >= c.n_slots) {
        si.q_lo = si.q_hi = 0; si.first_page = si.qp = 0; si.n_sink = si.recent_lo = si.n_win = si.U = 0;
        return si;
    }
    const int nq = n_quantized(S - c.lag, c.s_sink, c.s_keep, c.s_flush);
    si.q_lo = c.s_sink; si.q_hi = c.s_sink + nq;
    si.first_page = si.q_lo / PAGE_TOKENS;
    si.qp = nq > 0 ? (si.q_hi - 1) / PAGE_TOKENS - si.first_page + 1 : 0;
    si.n_sink = min(S, c.s_sink);
    si.recent_lo = c.s_sink + nq;
    si.n_win = si.n_sink + max(0, S - si.recent_lo);
    si.U = si.qp + (si.n_win + WIN_TOKENS - 1) / WIN_TOKENS;
    return si;
}

// Sparse attention reads at most n_select of the packed pages, the first min(n_select, qp) entries of the (sequence, KV head)'s list.
__device__ __forceinline__ SeqInfo sparse_info(SeqInfo si, int n_select) {
    if (si.qp > n_select) { si.U -= si.qp - n_select; si.qp = n_select; }
    return si;
}

// Work plan for the main kernel: exclusive prefix of work units per sequence, by one CTA of at least 128 threads (all of them call).
// n_select > 0: sparse attention.
__device__ inline void write_plan(const CacheView& c, int batch, const int* seq_len, const int* slot, int n_select, long long* plan) {
    __shared__ long long plan_scan_s[4];
    const int i = threadIdx.x, lane = i & 31, warp = i >> 5;
    long long carry = 0;
    for (int base = 0; base < batch; base += 128) {
        const int bb = base + i;
        long long u = 0;
        if (i < 128 && bb < batch) {
            const SeqInfo si = seq_info(c, __ldcg(seq_len + bb), __ldg(slot + bb));
            u = n_select > 0 ? sparse_info(si, n_select).U : si.U;
        }
        long long incl = u;
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31 && warp < 4) plan_scan_s[warp] = incl;
        __syncthreads();
        long long before = 0;
        for (int w = 0; w < warp && w < 4; ++w) before += plan_scan_s[w];
        if (i < 128 && bb < batch) plan[bb + 1] = carry + before + incl;
        carry += plan_scan_s[0] + plan_scan_s[1] + plan_scan_s[2] + plan_scan_s[3];
        __syncthreads();
    }
    if (i == 0) plan[0] = 0;
}

// Upper bound of the packed pages of a sequence of at most max_seq_len tokens.
inline long long candidate_bound(const CacheView& c, int max_seq_len) {
    const int nq = n_quantized(max_seq_len - c.lag, c.s_sink, c.s_keep, c.s_flush);
    return nq > 0 ? (c.s_sink + nq - 1) / PAGE_TOKENS - c.s_sink / PAGE_TOKENS + 1 : 0;
}

// Enqueues the selection; WUSHKV_OK, WUSHKV_ECAPACITY (too many candidates) or WUSHKV_ECUDA.
int launch_select(SelectParams P, int max_seq_len, cudaStream_t stream);

}  // namespace wushkv
