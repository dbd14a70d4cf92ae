// Sparse decode attention: the bounds of packed pages, and the entry points (the kernel that selects and attends is in sparse_kernel.cuh).
//
// A page and head keeps, beside its packed record, 257 bytes: for every channel the smallest and the largest dequantized key
// of the page's tokens, rounded outwards to multiples of a power of two that is common to the page and head,
//     e = least integer >= -31 with max |khat| <= 127 * 2^e,  lower = floor(min khat / 2^e),  upper = ceil(max khat / 2^e).
#include <cuda_fp16.h>

#include <algorithm>

#include "host_common.h"
#include "prologue.cuh"
#include "sparse.h"

namespace wushkv {

constexpr unsigned FULL = 0xffffffffu;
constexpr int MIN_EXPONENT = -31, MAX_EXPONENT = 14;      // of 2^e: fp16 steps and offsets reach from 2^-24 to 2^20

// ------------------------------------------------------------------------------------------------
// bounds
// ------------------------------------------------------------------------------------------------
struct BoundsParams {
    CacheView c;
    const int* slot;
    const int* seq_len;
    const int* cu_new;
    signed char* bounds;
    signed char* exponents;
};

// Halves the live values of a butterfly over one lane bit: afterwards v[0 .. N) hold the lane's half, combined.
template <int N, bool MAX>
__device__ __forceinline__ void halve(float* v, int lane, int bit) {
    const bool upper = (lane & bit) != 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float send = upper ? v[i] : v[i + N], keep = upper ? v[i + N] : v[i];
        const float got = __shfl_xor_sync(FULL, send, bit);
        v[i] = MAX ? fmaxf(keep, got) : fminf(keep, got);
    }
}

// Minima and maxima of three; a * b + c of two halves and a float, rounded once.
__device__ __forceinline__ float min3(float a, float b, float c) { float d; asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }
__device__ __forceinline__ float max3(float a, float b, float c) { float d; asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }
__device__ __forceinline__ float fma_half(unsigned short a, unsigned short b, float c) {
    float d;
    asm("fma.rn.f32.f16 %0, %1, %2, %3;" : "=f"(d) : "h"(a), "h"(b), "f"(c));
    return d;
}
__device__ __forceinline__ void halves(unsigned w, unsigned short& lo, unsigned short& hi) { asm("mov.b32 {%0, %1}, %2;" : "=h"(lo), "=h"(hi) : "r"(w)); }

// A warp per (page, head).  Lane (g, t) reads the code words of token rows g and g + 8 of every 16-token block, which hold the
// channels 32 s + 16 hh + 8 u + 2 t + v of all s, hh, u, v: 32 running minima and maxima per lane, combined over g at the end.
// What bounds it is the integer pipe (256 codes per lane).  A code masked out of a 16-bit half at bit F is, read as fp16, the number
// code * 2^(F - 24); one multiply-add of halves gives 2^(F - 24) khat from it and the stored step, so that a code costs half a mask,
// one multiply-add and a half each of a three-input minimum and maximum.  8 x 8192 tokens of 4 heads at 2 bits: 11.1 us with the codes
// turned into floats by byte permutes (2.25 integer instructions per code instead of 1.6).
constexpr int BOUNDS_WARPS = 2;      // per CTA: few, so that the last wave of CTAs is short
template <int BITS>
__global__ void __launch_bounds__(BOUNDS_WARPS * 32) page_bounds_kernel(BoundsParams P) {
    constexpr int REC = record_bytes(BITS), CB = code_block_bytes(BITS);
    pdl_wait();
    pdl_launch_dependents();
    const CacheView& c = P.c;
    const int b = blockIdx.y, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int unit = blockIdx.x * BOUNDS_WARPS + (threadIdx.x >> 5);
    const int len = P.seq_len[b], n = P.cu_new[b + 1] - P.cu_new[b], slot = P.slot[b];
    if (n <= 0 || len <= 0) return;
    if (slot < 0 || slot >= c.n_slots) { if (unit == 0 && lane == 0) atomicOr(c.dev_status, WUSHKV_DEV_BAD_SLOT); return; }
    const int index = max(len - n, 0) / PAGE_TOKENS + unit / c.n_kv, h = unit % c.n_kv;
    if (index > (len - 1) / PAGE_TOKENS) return;
    if (index >= c.max_pages) { if (lane == 0) atomicOr(c.dev_status, WUSHKV_DEV_PAGE_TABLE_FULL); return; }
    const int page = c.page_table[static_cast<long long>(slot) * c.max_pages + index];
    if (page < 0 || page >= c.n_pages) { if (lane == 0) atomicOr(c.dev_status, WUSHKV_DEV_BAD_PAGE_ID); return; }
    const long long ph = static_cast<long long>(page) * c.n_kv + h;
    const unsigned char* rec = c.pages + ph * REC;

    uint4 words[4][BITS == 4 ? 2 : 1], meta[4];
    uint2 high[4];
#pragma unroll
    for (int bi = 0; bi < 4; ++bi) {
#pragma unroll
        for (int p = 0; p < (BITS == 4 ? 2 : 1); ++p) words[bi][p] = ld_in(reinterpret_cast<const uint4*>(rec + bi * CB + 512 * p) + lane);
        if (BITS == 3) high[bi] = ld_in(reinterpret_cast<const uint2*>(rec + k_hi_offset(3) + bi * 256) + lane);
        meta[bi] = ld_in(reinterpret_cast<const uint4*>(rec + meta_offset(BITS) + 128 * bi) + g);
    }
    float lo[32], hi[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) { lo[j] = INFINITY; hi[j] = -INFINITY; }
#pragma unroll
    for (int bi = 0; bi < 4; ++bi) {
        unsigned short step[2];
        float low[2];
#pragma unroll
        for (int rs = 0; rs < 2; ++rs) {
            unsigned short offset;
            halves(rs == 0 ? meta[bi].x : meta[bi].z, step[rs], offset);
            // minimum and maximum pass over a NaN: a token that is not there, or a damaged one
            low[rs] = index * PAGE_TOKENS + 16 * bi + 8 * rs + g < len ? __half2float(__ushort_as_half(offset)) : NAN;
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int at = BITS == 4 ? 4 * (s & 1) : 2 * s;               // bit of the field in its byte
            const float unit = 1.f / static_cast<float>(1 << (24 - at));
            const float low_unit[2] = {low[0] * unit, low[1] * unit};
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const uint4& q = words[bi][BITS == 4 ? s >> 1 : 0];
#pragma unroll
                for (int odd = 0; odd < 2; ++odd) {                        // bytes 0 and 2, or 1 and 3 of the words
                    float v[2][2];                                         // [byte][row half]
#pragma unroll
                    for (int rs = 0; rs < 2; ++rs) {
                        const unsigned w = (hh == 0 ? (rs == 0 ? q.x : q.y) : (rs == 0 ? q.z : q.w)) >> (8 * odd);
                        unsigned code = w & ((BITS == 4 ? 0x000F000Fu : 0x00030003u) << at);
                        if (BITS == 3) {
                            const unsigned hw = rs == 0 ? high[bi].x : high[bi].y;
                            const int shift = at + 2 - (8 * odd + 2 * s + hh);     // the third bit: from bit 2 s + hh of its byte to two above the field
                            code |= (shift >= 0 ? hw << shift : hw >> -shift) & (0x00010001u << (at + 2));
                        }
                        unsigned short c0, c1;
                        halves(code, c0, c1);
                        // the product has at most 15 bits: the multiply-add rounds once, as the sum alone does
                        v[0][rs] = fma_half(c0, step[rs], low_unit[rs]);
                        v[1][rs] = fma_half(c1, step[rs], low_unit[rs]);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int j = 8 * s + 4 * hh + 2 * k + odd;
                        lo[j] = min3(lo[j], v[k][0], v[k][1]);
                        hi[j] = max3(hi[j], v[k][0], v[k][1]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const float up = static_cast<float>(1 << (24 - (BITS == 4 ? 4 * ((j >> 3) & 1) : 2 * (j >> 3))));
        lo[j] *= up;
        hi[j] *= up;
    }
    halve<16, false>(lo, lane, 16); halve<16, true>(hi, lane, 16);
    halve<8, false>(lo, lane, 8);   halve<8, true>(hi, lane, 8);
    halve<4, false>(lo, lane, 4);   halve<4, true>(hi, lane, 4);
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = fmaxf(most, fmaxf(fabsf(lo[i]), fabsf(hi[i])));
    const unsigned bits = __reduce_max_sync(FULL, __float_as_uint(most));          // magnitudes compare like their bits
    int e = static_cast<int>(bits >> 23) - 126;                                       // most = f * 2^e, 1/2 <= f < 1
    e -= (bits & 0x7fffffu) <= 0x7e0000u ? 7 : 6;                                     // f <= 127/128 or not
    e = min(max(e, MIN_EXPONENT), MAX_EXPONENT);
    const float scale = __uint_as_float(static_cast<unsigned>(127 - e) << 23);
    int ql[4], qh[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        ql[i] = min(max(__float2int_rd(lo[i] * scale), -127), 127);
        qh[i] = min(max(__float2int_ru(hi[i] * scale), -127), 127);
    }
    // lane bits 4, 3, 2 chose j's bits 4, 3, 2, i is by = 2 u + v: channels ch, ch + 1, ch + 8, ch + 9
    const int j0 = 16 * (lane >> 4) + 8 * ((lane >> 3) & 1) + 4 * ((lane >> 2) & 1);
    const int ch = 32 * (j0 >> 3) + 16 * ((j0 >> 2) & 1) + 2 * t;
    unsigned short* out = reinterpret_cast<unsigned short*>(P.bounds + ph * 2 * D);
    const auto pair = [](int a, int b2) { return static_cast<unsigned short>((a & 255) | ((b2 & 255) << 8)); };
    out[ch / 2] = pair(ql[0], ql[1]);
    out[ch / 2 + 4] = pair(ql[2], ql[3]);
    out[D / 2 + ch / 2] = pair(qh[0], qh[1]);
    out[D / 2 + ch / 2 + 4] = pair(qh[2], qh[3]);
    if (lane == 0) P.exponents[ph] = static_cast<signed char>(e);
}

// ------------------------------------------------------------------------------------------------
// entry points
// ------------------------------------------------------------------------------------------------
// Upper bound of the packed pages of a sequence of at most max_seq_len tokens.
static long long candidate_bound(const CacheView& c, int max_seq_len) {
    const int nq = n_quantized(max_seq_len - c.lag, c.s_sink, c.s_keep, c.s_flush);
    return nq > 0 ? (c.s_sink + nq - 1) / PAGE_TOKENS - c.s_sink / PAGE_TOKENS + 1 : 0;
}

constexpr int MAX_LIST = 1 << 30;      // the kernel's walk over a list ends up to a step behind it, in 32 bits

// Checks and launches all three calls: bounds == nullptr: the list is an input; O == nullptr: the list is all that is asked for.
static int sparse_impl(const wushkv_cache* cache, int32_t batch, const int32_t* slot, const int32_t* seq_len, int32_t max_seq_len, const uint16_t* Q,
                       const wushkv_prologue* prologue, const int8_t* bounds, const int8_t* exponents, int32_t n_select, int32_t* selected, uint16_t* O, void* stream) {
    SparseParams P;
    const int rc = make_view(cache, P.c);
    if (rc != WUSHKV_OK) return rc;
    if (batch <= 0 || batch > 65535 || P.c.n_kv > 65535 || max_seq_len <= 0 || n_select <= 0 || n_select > MAX_LIST) return WUSHKV_EINVAL;
    if (!slot || !seq_len || !Q || !selected || !int_arrays(slot, seq_len, selected) || !aligned(Q, 16) || !aligned(bounds, 16) || !aligned(O, 16)) return WUSHKV_EINVAL;
    P.pro = Prologue{nullptr, 0, 0, nullptr, 0.f};
    if (prologue && !make_prologue(prologue, prologue->q_norm_weight, P.pro)) return WUSHKV_EINVAL;
    const long long candidates = std::max<long long>(candidate_bound(P.c, max_seq_len), 1);
    if (bounds && candidates > MAX_SELECT_PAGES) return WUSHKV_ECAPACITY;
    P.batch = batch; P.slot = slot; P.seq_len = seq_len; P.Q = Q;
    P.bounds = reinterpret_cast<const signed char*>(bounds); P.exponents = reinterpret_cast<const signed char*>(exponents);
    P.n_select = n_select; P.selected = selected; P.O = O;
    P.max_candidates = bounds ? static_cast<int>(candidates) : 0;      // a list that is given: nothing is scored
    P.ring_offset = 0;
    // upper bound of the packed bytes one step reads against the L2 size (126 MB)
    P.stream_pages = static_cast<double>(batch) * P.c.n_kv * std::min<double>(n_select, static_cast<double>(candidates)) * record_bytes(P.c.bits) > 126e6 ? 1 : 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return P.c.bits == 2 ? launch_sparse_2bit(P, st) : P.c.bits == 3 ? launch_sparse_3bit(P, st) : launch_sparse_4bit(P, st);
}

}  // namespace wushkv

using namespace wushkv;

extern "C" int wushkv_update_page_bounds(const wushkv_cache* cache, int32_t batch, const int32_t* slot, const int32_t* seq_len, const int32_t* cu_new,
                                         int32_t max_new, int8_t* bounds, int8_t* exponents, void* stream) {
    BoundsParams P;
    const int rc = make_view(cache, P.c);
    if (rc != WUSHKV_OK) return rc;
    if (batch <= 0 || batch > 65535 || max_new < 0 || !slot || !seq_len || !cu_new || !int_arrays(slot, seq_len, cu_new) || !bounds || !exponents || !aligned(bounds, 16)) return WUSHKV_EINVAL;
    if (max_new == 0) return WUSHKV_OK;
    P.slot = slot; P.seq_len = seq_len; P.cu_new = cu_new; P.bounds = bounds; P.exponents = exponents;
    // pages that max_new consecutive tokens can touch, and of those behind the table's end one, for the flag
    const long long pages = std::min<long long>((static_cast<long long>(max_new) + PAGE_TOKENS - 2) / PAGE_TOKENS, P.c.max_pages) + 1;
    const long long units = pages * P.c.n_kv;
    if (units > 0x7fffffff - BOUNDS_WARPS) return WUSHKV_ECAPACITY;
    const dim3 grid(static_cast<unsigned>((units + BOUNDS_WARPS - 1) / BOUNDS_WARPS), batch);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return launch_pdl(P.c.bits == 2 ? page_bounds_kernel<2> : P.c.bits == 3 ? page_bounds_kernel<3> : page_bounds_kernel<4>, grid, dim3(BOUNDS_WARPS * 32), 0, st, P) == cudaSuccess
        ? WUSHKV_OK : WUSHKV_ECUDA;
}
extern "C" int wushkv_select_pages(const wushkv_cache* cache, int32_t batch, const int32_t* slot, const int32_t* seq_len, int32_t max_seq_len,
                                   const uint16_t* Q, const wushkv_prologue* prologue, const int8_t* bounds, const int8_t* exponents,
                                   int32_t n_select, int32_t* selected, void* stream) {
    if (!bounds || !exponents) return WUSHKV_EINVAL;
    return sparse_impl(cache, batch, slot, seq_len, max_seq_len, Q, prologue, bounds, exponents, n_select, selected, nullptr, stream);
}

extern "C" int wushkv_decode_attn_selected(const wushkv_cache* cache, int32_t batch, const int32_t* slot, const int32_t* seq_len, int32_t max_seq_len,
                                           const uint16_t* Q, const wushkv_prologue* prologue, const int32_t* selected, int32_t n_select, uint16_t* O,
                                           void* stream) {
    if (!O) return WUSHKV_EINVAL;
    return sparse_impl(cache, batch, slot, seq_len, max_seq_len, Q, prologue, nullptr, nullptr, n_select, const_cast<int32_t*>(selected), O, stream);
}

extern "C" size_t wushkv_sparse_workspace_bytes(const wushkv_cache* cache, int32_t batch, int32_t max_seq_len, int32_t n_select) {
    CacheView v;
    if (make_view(cache, v) != WUSHKV_OK || batch <= 0 || max_seq_len <= 0 || n_select <= 0 || n_select > MAX_LIST) return 0;
    return (static_cast<size_t>(batch) * v.n_kv * n_select * sizeof(int32_t) + 255) / 256 * 256;
}

extern "C" int wushkv_decode_attn_sparse(const wushkv_cache* cache, int32_t batch, const int32_t* slot, const int32_t* seq_len, int32_t max_seq_len,
                                         const uint16_t* Q, const wushkv_prologue* prologue, const int8_t* bounds, const int8_t* exponents,
                                         int32_t n_select, int32_t* selected, uint16_t* O, void* workspace, size_t workspace_bytes, void* stream) {
    if (!bounds || !exponents || !O) return WUSHKV_EINVAL;
    if (!selected) {                                              // the caller does not want the list: it is kept in the workspace
        if (!cache || batch <= 0 || max_seq_len <= 0 || n_select <= 0 || !workspace || !aligned(workspace, 256)) return WUSHKV_EINVAL;
        const size_t need = wushkv_sparse_workspace_bytes(cache, batch, max_seq_len, n_select);
        if (need == 0) return WUSHKV_EINVAL;
        if (workspace_bytes < need) return WUSHKV_ECAPACITY;
        selected = static_cast<int32_t*>(workspace);
    }
    return sparse_impl(cache, batch, slot, seq_len, max_seq_len, Q, prologue, bounds, exponents, n_select, selected, O, stream);
}
