// Sparse decode attention: bounds of packed pages, the selection of pages by them, and the attention over the selected pages.
//
// A page and head keeps, beside its packed record, 257 bytes: for every channel the smallest and the largest dequantized key
// of the page's tokens, rounded outwards to multiples of a power of two that is common to the page and head,
//     e = least integer >= -31 with max |khat| <= 127 * 2^e,  lower = floor(min khat / 2^e),  upper = ceil(max khat / 2^e).
// With them the largest score that any token of the page can reach against a query q' is
//     2^e * sum_c ( max(q'_c, 0) upper_c + min(q'_c, 0) lower_c ),
// a dot product of 256 terms.  The query enters as 16-bit fixed point (two signed bytes per channel), so that the sum is an
// exact integer from mma.sync.m16n8k32 (s8 x s8): scores, and with them the selected pages, do not depend on the order of any
// summation.  q' itself is formed in 64 bits for the same reason: its rounding to 16 bits then is the same wherever it is done.
//
// Selection and attention are ONE kernel, a cluster of CTAs per (sequence, KV head).  As two kernels (the selection ahead of the
// dense decode kernel with a list) a step of 16 sequences x 8 heads with 64 of 510 pages took 36.4 us, of them 12 us selection:
// the second kernel's CTAs need the registers that the first one's hold, so its set-up (work plan, first list entries, first
// copies: 8 us) began only when the selection had ended, and many sequences' selections ran in waves of idle latency.  In one
// kernel the attention of a head follows its selection at once, and the selections of later CTAs overlap with it.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "decode_core.cuh"
#include "host_common.h"
#include "prologue.cuh"

namespace wushkv {

namespace cg = cooperative_groups;

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

// Two numbers per instruction, and minima and maxima of three.
__device__ __forceinline__ unsigned long long pack2(float a, float b) {
    unsigned long long d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ void unpack2(unsigned long long d, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(d)); }
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ float min3(float a, float b, float c) { float d; asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }
__device__ __forceinline__ float max3(float a, float b, float c) { float d; asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }

// A warp per (page, head).  Lane (g, t) reads the code words of token rows g and g + 8 of every 16-token block, which hold the
// channels 32 s + 16 hh + 8 u + 2 t + v of all s, hh, u, v: 32 running minima and maxima per lane, combined over g at the end.
// What bounds it is instructions (256 codes per lane): a code becomes a float by a byte permute that puts its byte, masked to one
// field, under the exponent of 2^23, the rest is done for the two token rows at once.
template <int BITS>
__global__ void __launch_bounds__(256) page_bounds_kernel(BoundsParams P) {
    constexpr int REC = record_bytes(BITS), CB = code_block_bytes(BITS);
    const CacheView& c = P.c;
    const int b = blockIdx.y, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int unit = blockIdx.x * 8 + (threadIdx.x >> 5);
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
        for (int p = 0; p < (BITS == 4 ? 2 : 1); ++p) words[bi][p] = __ldg(reinterpret_cast<const uint4*>(rec + bi * CB + 512 * p) + lane);
        if (BITS == 3) high[bi] = __ldg(reinterpret_cast<const uint2*>(rec + k_hi_offset(3) + bi * 256) + lane);
        meta[bi] = __ldg(reinterpret_cast<const uint4*>(rec + meta_offset(BITS) + 128 * bi) + g);
    }
    constexpr float MAGIC = 8388608.f;                       // 2^23
    const unsigned long long unmagic = pack2(-MAGIC, -MAGIC);
    float lo[32], hi[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) { lo[j] = INFINITY; hi[j] = -INFINITY; }
#pragma unroll
    for (int bi = 0; bi < 4; ++bi) {
        float step[2], low[2];
#pragma unroll
        for (int rs = 0; rs < 2; ++rs) {
            const unsigned m = rs == 0 ? meta[bi].x : meta[bi].z;
            __half2 h2;
            *reinterpret_cast<unsigned*>(&h2) = m;
            const float2 f = __half22float2(h2);
            const bool there = index * PAGE_TOKENS + 16 * bi + 8 * rs + g < len;
            step[rs] = there ? f.x : 0.f;
            low[rs] = there ? f.y : NAN;                 // minimum and maximum pass over a NaN: a token that is not there, or a damaged one
        }
        const unsigned long long low2 = pack2(low[0], low[1]);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            // a code in bits F .. of its byte is code * 2^F; the step takes the 2^-F, both exact
            constexpr unsigned FIELD = BITS == 4 ? 0x0F0F0F0Fu : 0x03030303u;
            const int shift = BITS == 4 ? 4 * (s & 1) : 2 * s;
            const float down = 1.f / static_cast<float>(1 << shift);
            const unsigned long long step2 = pack2(step[0] * down, step[1] * down);
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const uint4& q = words[bi][BITS == 4 ? s >> 1 : 0];
                unsigned w[2] = {hh == 0 ? q.x : q.z, hh == 0 ? q.y : q.w};
#pragma unroll
                for (int rs = 0; rs < 2; ++rs) {
                    w[rs] &= FIELD << shift;
                    if (BITS == 3) {
                        // the third bit, 4 * 2^F: for the uppermost field it would leave its byte, so that one is moved down
                        const unsigned hb = ((rs == 0 ? high[bi].x : high[bi].y) >> (2 * s + hh)) & 0x01010101u;
                        w[rs] = s < 3 ? w[rs] | (hb << (shift + 2)) : (w[rs] >> 2) | (hb << 6);
                    }
                }
                const unsigned long long step_here = BITS == 3 && s == 3 ? pack2(step[0] * (1.f / 16.f), step[1] * (1.f / 16.f)) : step2;
#pragma unroll
                for (int by = 0; by < 4; ++by) {
                    const float x0 = __uint_as_float(__byte_perm(w[0], 0x4B000000u, 0x7440u + by)), x1 = __uint_as_float(__byte_perm(w[1], 0x4B000000u, 0x7440u + by));
                    // step * code has at most 15 bits: the multiply-add rounds once, as the sum alone does
                    float v0, v1;
                    unpack2(fma2(step_here, add2(pack2(x0, x1), unmagic), low2), v0, v1);
                    const int j = 8 * s + 4 * hh + by;
                    lo[j] = min3(lo[j], v0, v1);
                    hi[j] = max3(hi[j], v0, v1);
                }
            }
        }
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
// selection and attention
// ------------------------------------------------------------------------------------------------
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

__device__ __forceinline__ void mma_s8(int (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int SPARSE_THREADS = 256, SPARSE_WARPS = SPARSE_THREADS / 32;
constexpr int SELECT_BINS = 4 * SPARSE_THREADS;

// Shared memory of a CTA: this, then a region for the selection (the page ids and the scores of the CTA's pages [per], [heads][per],
// CTA 0: key and page id of all pages) and the warps' staging rings.  Where the sizes allow it the rings are apart from the selection's
// region, so that window tokens can be staged from the start; else the rings begin where the selection's region began.
constexpr int LISTED = 512;               // listed pages that are handed over in shared memory, with their ids
template <int MODE>
struct SparseShared {
    static constexpr int GP = MODE == 0 ? 4 : 8, SETS = MODE == 0 ? 1 : 2;
    static constexpr int QF = MODE == 0 ? 64 : 128, QW = MODE == 0 ? 128 : 256;     // uint4 of the attention's integer / bf16 fragments
    union {
        double q[GP][D];                  // the queries, in 64 bits
        uint4 frag[SETS * 4 * 32];        // then the selection's query fragments: [digit set][64 bytes of bounds][lane]
        uint4 bins[SPARSE_THREADS];       // then this CTA's pages per bin of the range of keys
        float merged[GP][PART_STRIDE];    // at last the CTA's partial result of every head
    };
    union {
        double qc[GP][D];                 // q' of this CTA's rows
        uint2 listed[LISTED];             // then, CTA 0: the listed pages, index and id
    };
    uint4 attn[QF + QW];                  // the attention's query fragments
    float2 scal[8];                       // score multiplier (log2 domain) and x_min multiplier of the heads
    float unit[8];                        // score of one unit of 2^e dot
    float2 warp_best[SPARSE_WARPS][8];
    float2 best[8][8];                    // per CTA of the cluster: largest and smallest finite score of its pages, per head
    int scan[SPARSE_WARPS], below[SPARSE_WARPS], equal[SPARSE_WARPS];
    int bin, inside, wanted;              // CTA 0: the bin of the n_select-th key, keys in it, its rank among them
    unsigned kth;
    int n_list;
    unsigned list[SPARSE_THREADS];        // keys of that bin
};

// One window unit of this kernel: up to 16 bf16 tokens, key rows staged at rows, value rows behind them, 256 bytes each, the 16-byte
// piece i of row r at place i ^ (r & 7) (so that eight rows of a column of pieces lie in different banks).  Rows from n_valid on hold
// copies of valid ones.  (The dense kernel's units have 8 tokens; here a warp gets one unit or none, and 16 tokens cost it little more.)
constexpr int WIDE_TOKENS = 16;
template <int BITS, int MODE>
__device__ __forceinline__ void wide_window_unit(WarpState<MODE>& st, unsigned rows, int n_valid, const uint4* query, int lane) {
    constexpr int NH = WarpState<MODE>::NH;
    const int g = lane >> 2, mat = lane >> 3, r7 = lane & 7;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    {
        const unsigned row = rows + (r7 + 8 * (mat & 1)) * (2 * D);
#pragma unroll
        for (int s2 = 0; s2 < 4; ++s2) {
            unsigned a[2][4];
#pragma unroll
            for (int k = 0; k < 2; ++k) ldmatrix_x4(row + (((4 * s2 + 2 * k + (mat >> 1)) ^ r7) << 4), a[k][0], a[k][1], a[k][2], a[k][3]);
#pragma unroll
            for (int pass = 0; pass < (MODE == 0 ? 1 : 2); ++pass) {
                const uint4 bq = query[pass * 128 + s2 * 32 + lane];
                mma_bf16(acc, a[0][0], a[0][1], a[0][2], a[0][3], bq.x, bq.y);
                mma_bf16(acc, a[1][0], a[1][1], a[1][2], a[1][3], bq.z, bq.w);
            }
        }
    }
    float sc[2][NH], mx[NH];                              // rows g, g + 8
#pragma unroll
    for (int rs = 0; rs < 2; ++rs)
#pragma unroll
        for (int k = 0; k < NH; ++k) sc[rs][k] = g + 8 * rs < n_valid ? (MODE == 0 ? acc[2 * rs] + acc[2 * rs + 1] : acc[2 * rs + k]) : -INFINITY;
#pragma unroll
    for (int k = 0; k < NH; ++k) mx[k] = fmaxf(sc[0][k], sc[1][k]);
    st.raise_max(mx);
    float p[2][NH];
#pragma unroll
    for (int rs = 0; rs < 2; ++rs)
#pragma unroll
        for (int k = 0; k < NH; ++k) { p[rs][k] = ex2(sc[rs][k] - st.mr[k]); st.l[k] += p[rs][k]; }
    unsigned b01[MODE == 0 ? 1 : 2][2];                   // the probabilities as B fragments, tokens 2 t, 2 t + 1 (+ 8) of column g
#pragma unroll
    for (int rs = 0; rs < 2; ++rs)
#pragma unroll
        for (int pass = 0; pass < (MODE == 0 ? 1 : 2); ++pass) {
            unsigned pr;                                  // value column, remainder column; or two heads' values, then their remainders
            if (MODE == 0) pr = pack_bf2(p[rs][0], (p[rs][0] - bf16_round(p[rs][0])) * LO_SCALE);
            else if (pass == 0) pr = pack_bf2(p[rs][0], p[rs][NH - 1]);
            else pr = pack_bf2(p[rs][0] - bf16_round(p[rs][0]), p[rs][NH - 1] - bf16_round(p[rs][NH - 1]));
            b01[pass][rs] = movmatrix_trans(pr);
        }
    const unsigned row = rows + WIDE_TOKENS * 2 * D + (r7 + 8 * (mat >> 1)) * (2 * D);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        unsigned a0, a1, a2, a3;                          // channels 16 i .. + 7 and + 8 .. + 15 of tokens 0 .. 7, the same of tokens 8 .. 15
        ldmatrix_x4_trans(row + (((2 * i + (mat & 1)) ^ r7) << 4), a0, a1, a2, a3);
        const unsigned unit = bf16x2_pow2(field_shift<BITS>(i) - 24);      // the block's accumulator unit
#pragma unroll
        for (int pass = 0; pass < (MODE == 0 ? 1 : 2); ++pass) mma_bf16(st.o[i], a0, a1, a2, a3, mul_bf2(b01[pass][0], unit), mul_bf2(b01[pass][1], unit));
    }
}

// Staging ring of a warp: slots for the key side (codes, steps and offsets) and for the value side, filled and freed on their own,
// so that the next page's keys are on their way while this one's values are used.  Two CTAs fit on an SM.  The warp's lanes fill it
// with 16-byte asynchronous copies: a bulk copy costs the lane that requests it some 440 cycles, and requests of several lanes are
// served one after the other (three per page and eight rows per window unit made the staging slower than the work on it).
// Copies are waited for in the order of their groups: K_PENDING / V_PENDING groups may be outstanding behind the one that is needed
// next, where the order is  K0 V0  (K0 V0 K1 V1  with two slots each,  K0 K1 V0  with two and one), then, per unit,  K(i + NK)  after
// its scores and  V(i + NV)  after its values.
template <int BITS>
struct Ring {
    static constexpr int NK = BITS == 4 ? 1 : 2, NV = BITS == 2 ? 2 : 1;
    static constexpr int K_PENDING = NK + NV - 1, V_PENDING = NV == 2 ? 3 : 1;
    static constexpr int META = PAGE_TOKENS * 8;                                     // bytes of steps and offsets
    static constexpr int K_SLOT = side_bytes(BITS) + META, V_SLOT = side_bytes(BITS);
    static constexpr int BYTES = NK * K_SLOT + NV * V_SLOT;
    static_assert(K_SLOT % 16 == 0 && V_SLOT % 16 == 0, "copies are aligned");
    static_assert(BYTES >= 8 * PART_STRIDE * 4 && BYTES >= 2 * WIDE_TOKENS * D * 2, "the partials of 8 query heads fit, and a window unit");
};

__host__ __device__ inline int pages_per_cta(int pages, int cl) { return ((pages + cl - 1) / cl + 15) / 16 * 16; }

// Loads that stay where they are written: ahead of the work that their latency is to hide behind.
__device__ __forceinline__ uint4 ld_early(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ int ld_early_s8(const signed char* p) {
    int v;
    asm volatile("ld.global.nc.s8 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}

// Asynchronous copy of 16 bytes into shared memory, also with an L2 eviction policy.
__device__ __forceinline__ void copy16(unsigned dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16_hint(unsigned dst, const void* src, unsigned long long policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void copies_wait() {              // of this lane's copies; then of the whole warp's
    asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory");
    __syncwarp();
}

// Sums NV numbers per lane over groups of LANES lanes.  While there are several, each step hands half of them to the other side;
// afterwards lane l of the group holds the totals of first(l) .. first(l) + LEFT - 1, and REPLICAS lanes hold the same.
template <int NV, int LANES>
struct GroupSum {
    static constexpr int LEFT = NV > LANES ? NV / LANES : 1, REPLICAS = LANES > NV ? LANES / NV : 1;
    template <int N, int O>
    static __device__ __forceinline__ void step(double* v, int l) {
        if constexpr (O >= 1) {
            if constexpr (N > 1) {
                const bool upper = (l & O) != 0;
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    const double send = upper ? v[i] : v[i + N / 2], keep = upper ? v[i + N / 2] : v[i];
                    v[i] = keep + __shfl_xor_sync(FULL, send, O);
                }
                step<N / 2, O / 2>(v, l);
            } else {
                v[0] += __shfl_xor_sync(FULL, v[0], O);
                step<1, O / 2>(v, l);
            }
        }
    }
    static __device__ __forceinline__ void sum(double* v, int l) { step<NV, LANES / 2>(v, l); }
    static __device__ __forceinline__ int first(int l) { return l / REPLICAS * LEFT; }
    static __device__ __forceinline__ int replica(int l) { return l % REPLICAS; }
};

// One tile of 16 pages as a lane reads it: 64 bytes of the bounds of rows g and g + 8 and the rows' exponents.  ids: the page ids of
// the CTA's n pages, -1 where the table names none.
struct BoundsTile {
    uint4 a[2][4];
    int ex[2];
    bool good[2];
    __device__ __forceinline__ void load(const SparseParams& P, const int* ids, int h, int p0, int n, int g, int t) {
#pragma unroll
        for (int rs = 0; rs < 2; ++rs) {
            const int p = p0 + g + 8 * rs, page = p < n ? ids[p] : -1;
            good[rs] = page >= 0;
            const long long ph = static_cast<long long>(good[rs] ? page : 0) * P.c.n_kv + h;
            const uint4* src = reinterpret_cast<const uint4*>(P.bounds + ph * 2 * D) + t;
#pragma unroll
            for (int k = 0; k < 4; ++k) a[rs][k] = ld_early(src + 4 * k);
            ex[rs] = ld_early_s8(P.exponents + ph);
        }
    }
};
__device__ __forceinline__ void prefetch_bounds(const SparseParams& P, int page, int h) {
    const long long ph = static_cast<long long>(page) * P.c.n_kv + h;
    asm volatile("prefetch.global.L2 [%0];" ::"l"(P.bounds + ph * 2 * D));
    asm volatile("prefetch.global.L2 [%0];" ::"l"(P.bounds + ph * 2 * D + D));
    asm volatile("prefetch.global.L2 [%0];" ::"l"(P.exponents + ph));
}

// Bins of equal width; the product is monotonic in the key, so bins are in the keys' order.
__device__ __forceinline__ int bin_of(unsigned key, float per_bin) { return min(static_cast<int>(__uint_as_float(key) * per_bin), SELECT_BINS - 1); }

// The n_select smallest of the keys (.x; .y is the page's id), ties to the lower page, in ascending order of the pages, by one CTA.
// counted: this thread's four of the bins of equal width in which the cluster has counted the keys; the bin of the n_select-th smallest
// is found by a prefix sum and its few keys are compared with each other.
// The code is kept short: a CTA runs through it once, so that every instruction is fetched for one use (with the keys in registers
// and its loops unrolled it took 30 KB and was no faster).
template <class Shared>
__device__ __forceinline__ void list_pages(Shared& sh, const uint4& counted, float per_bin, const uint2* keys, int pages, int first, int n_select, int* out) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int c0 = static_cast<int>(counted.x), c1 = static_cast<int>(counted.y), c2 = static_cast<int>(counted.z), here = c0 + c1 + c2 + static_cast<int>(counted.w);
    int before = here;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(FULL, before, o);
        if (lane >= o) before += y;
    }
    if (lane == 31) sh.scan[warp] = before;
    __syncthreads();
    before -= here;
#pragma unroll
    for (int w = 0; w < SPARSE_WARPS; ++w) before += w < warp ? sh.scan[w] : 0;
    const int rest = n_select - before;                     // the rank, from 1, of the n_select-th key among this thread's bins
    if (rest >= 1 && rest <= here) {
        const int e = (rest > c0) + (rest > c0 + c1) + (rest > c0 + c1 + c2);
        const int skipped = e == 0 ? 0 : e == 1 ? c0 : e == 2 ? c0 + c1 : c0 + c1 + c2;
        sh.bin = 4 * tid + e;
        sh.wanted = rest - skipped - 1;
        sh.inside = e == 0 ? c0 : e == 1 ? c1 : e == 2 ? c2 : here - c0 - c1 - c2;
    }
    __syncthreads();
    const int bin = sh.bin, inside = sh.inside, wanted = sh.wanted;      // the bin of the n_select-th key, keys in it, its rank there from 0
    unsigned kth = 0u;
    if (inside <= SPARSE_THREADS) {
#pragma unroll 2
        for (int p = tid; p < pages; p += SPARSE_THREADS) {
            const unsigned u = keys[p].x;
            if (bin_of(u, per_bin) == bin) sh.list[atomicAdd(&sh.n_list, 1)] = u;
        }
        __syncthreads();
        if (tid < inside) {
            const unsigned u = sh.list[tid];
            int less = 0, same = 0;
#pragma unroll 2
            for (int k = 0; k < inside; ++k) { less += sh.list[k] < u; same += sh.list[k] == u; }
            if (less <= wanted && wanted < less + same) sh.kth = u;      // equal keys write the same
        }
        __syncthreads();
        kth = sh.kth;
    } else {
        // many keys that are (almost) the same: bit by bit, the largest v with fewer than n_select keys below it
#pragma unroll 1
        for (int bit = 30; bit >= 0; --bit) {
            const unsigned cand = kth | (1u << bit);
            int n = 0;
#pragma unroll 1
            for (int p = tid; p < pages; p += SPARSE_THREADS) n += keys[p].x < cand;
            __syncthreads();                                // the readers of the round before
            n = __reduce_add_sync(FULL, n);
            if (lane == 0) sh.scan[warp] = n;
            __syncthreads();
            int total = 0;
#pragma unroll
            for (int w = 0; w < SPARSE_WARPS; ++w) total += sh.scan[w];
            if (total < n_select) kth = cand;
        }
    }
    // all below it, and of those equal to it the first ones; every warp lists a run of consecutive pages
    const int run = (pages + SPARSE_THREADS - 1) / SPARSE_THREADS * 32, r_lo = min(warp * run, pages), r_hi = min(r_lo + run, pages);
    int below = 0, equal = 0;
#pragma unroll 2
    for (int p = r_lo + lane; p < r_hi; p += 32) { const unsigned u = keys[p].x; below += u < kth; equal += u == kth; }
    below = __reduce_add_sync(FULL, below);
    equal = __reduce_add_sync(FULL, equal);
    if (lane == 0) { sh.below[warp] = below; sh.equal[warp] = equal; }
    __syncthreads();
    int all_below = 0, below_before = 0, equal_before = 0;
#pragma unroll
    for (int w = 0; w < SPARSE_WARPS; ++w) {
        const int y = sh.below[w];
        all_below += y;
        if (w < warp) { below_before += y; equal_before += sh.equal[w]; }
    }
    const int room = n_select - all_below;                  // places for keys equal to the n_select-th
    const unsigned lower = (1u << lane) - 1u;
#pragma unroll 1
    for (int p0 = r_lo; p0 < r_hi; p0 += 32) {
        const int p = p0 + lane;
        const uint2 k = p < r_hi ? keys[p] : make_uint2(0xffffffffu, 0u);
        const unsigned is_below = __ballot_sync(FULL, k.x < kth), is_equal = __ballot_sync(FULL, k.x == kth);
        const int e = equal_before + __popc(is_equal & lower);
        if (k.x < kth || (k.x == kth && e < room)) {
            const int at = below_before + __popc(is_below & lower) + min(e, room);
            out[at] = first + p;
            if (at < LISTED) sh.listed[at] = make_uint2(first + p, k.y);
        }
        below_before += __popc(is_below);
        equal_before += __popc(is_equal);
    }
}

// One cluster of CL CTAs per (sequence, KV head).
//   1. q' = T_K^{-T} q: each CTA forms 128 / CL rows of it and hands them to the others through distributed shared memory.
//   2. Each CTA scores its share of the pages, 16 pages per warp and step: bounds straight from global memory into the A
//      fragments (their bytes are consecutive in k, so that one 16-byte load per lane and row is two registers of two k-steps).
//      The first step's loads are in flight during 1, the next step's during each step.
//   3. The largest score per head of all CTAs, the key of every page (how far it is below the best page of the head that it
//      matters most to), sent to CTA 0, which lists the pages; the other CTAs take the window tokens meanwhile.
//   4. The listed pages are dealt out to the cluster's warps; each keeps a running softmax (decode_core.cuh), and the states are
//      merged first within the CTAs, then, a CTA per head, over the cluster.
// Steps 1 to 3 are latency (the bounds of 16 sequences x 8 heads x 510 pages are 17 MB, 2.6 us at the copy rate), step 4 is the
// work of the dense kernel on fewer pages.
template <int BITS, int MODE, int CL>
__global__ void __launch_bounds__(SPARSE_THREADS, 2) sparse_decode_kernel(SparseParams P) {
    using Shared = SparseShared<MODE>;
    using R = Ring<BITS>;
    constexpr int GP = Shared::GP, SETS = Shared::SETS, NH = WarpState<MODE>::NH;
    extern __shared__ __align__(16) unsigned char sparse_smem[];
    Shared& sh = *reinterpret_cast<Shared*>(sparse_smem);
    unsigned char* region = sparse_smem + sizeof(Shared);
    unsigned char* rings = region + P.ring_offset;
    cg::cluster_group cluster = cg::this_cluster();
    const CacheView& c = P.c;
    const int rank = CL > 1 ? static_cast<int>(cluster.block_rank()) : 0, h = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, G = c.G;
    pdl_wait();
    pdl_launch_dependents();
    if (tid == 0) sh.n_list = 0;
    // ---- q': this thread's two rows of T_K^{-T} and its share of the queries are requested ahead of everything else
    constexpr int ROWS = D / CL, PAIRS = ROWS / 2, TPP = SPARSE_THREADS / PAIRS, QUADS = D / 4 / TPP;      // threads per pair of rows, float4 per thread and row
    constexpr int PART = QUADS > 4 ? 4 : QUADS;                                              // of them in flight together
    const int t_row = rank * ROWS + tid / TPP, seg = tid % TPP;
    const uint4* T = reinterpret_cast<const uint4*>(c.T_K_invT + (static_cast<long long>(h) * D + t_row) * D);
    uint4 tr[2][PART];
    const auto load_T = [&](int k0) {
#pragma unroll
        for (int k = 0; k < PART; ++k) { tr[0][k] = ld_early(T + seg + TPP * (k0 + k)); tr[1][k] = ld_early(T + PAIRS * (D / 4) + seg + TPP * (k0 + k)); }
    };
    load_T(0);
    uint2 q_bits = make_uint2(0u, 0u);                  // slots without a head are zero
    if (warp < G) q_bits = __ldg(reinterpret_cast<const uint2*>(P.Q + (static_cast<long long>(b) * c.n_q + h * G + warp) * D + 4 * lane));

    // ---- candidates
    const int S = __ldcg(P.seq_len + b), slot = P.slot[b];
    const bool attend = P.O != nullptr, given = P.bounds == nullptr;
    int* list = P.selected + (static_cast<long long>(b) * c.n_kv + h) * P.n_select;
    const SeqInfo si = seq_info(c, S, slot);
    int pages = si.qp;
    const int first = si.first_page;
    const bool reporter = rank == 0 && h == 0 && tid == 0;
    if ((slot < 0 || slot >= c.n_slots) && reporter) atomicOr(c.dev_status, WUSHKV_DEV_BAD_SLOT);
    if (first + pages > c.max_pages) {
        if (reporter) atomicOr(c.dev_status, WUSHKV_DEV_PAGE_TABLE_FULL);
        pages = max(c.max_pages - first, 0);
    }
    if (!given && pages > P.max_candidates) {           // a sequence longer than promised
        if (reporter) atomicOr(c.dev_status, WUSHKV_DEV_BAD_COUNT);
        pages = P.max_candidates;
    }
    const bool score = !given && pages > P.n_select;     // the same for the whole cluster, like all that depends on it
    const int n_listed = min(pages, P.n_select);
    if (!given && !score && rank == 0)
        for (int i = tid; i < P.n_select; i += SPARSE_THREADS) list[i] = i < pages ? first + i : -1;
    if (!attend && !score) return;
    const int per_max = pages_per_cta(P.max_candidates, CL);
    int* ids = reinterpret_cast<int*>(region);                                               // [per_max]
    float* scores = reinterpret_cast<float*>(ids + per_max);                                 // [G][per_max]
    uint2* keys = reinterpret_cast<uint2*>(scores + static_cast<size_t>(G) * per_max);       // CTA 0: [max_candidates]
    const int per = pages_per_cta(pages, CL), p_lo = min(rank * per, pages), n_here = min(p_lo + per, pages) - p_lo;      // this CTA's candidates
    const int* row = c.page_table + static_cast<long long>(slot) * c.max_pages;              // read only if there are pages
    if (score) {
        for (int p = tid; p < n_here; p += SPARSE_THREADS) {
            const int page = __ldg(row + first + p_lo + p);
            const bool good = page >= 0 && page < c.n_pages;
            if (good) prefetch_bounds(P, page, h);
            else atomicOr(c.dev_status, WUSHKV_DEV_BAD_PAGE_ID);
            ids[p] = good ? page : -1;
        }
    }

    // ---- window tokens: by all warps, or by those of the CTAs that will not be listing pages.  Staged early if the rings are apart.
    unsigned char* ring = rings + warp * R::BYTES;
    const unsigned k_slot0 = smem_u32(ring), v_slot0 = k_slot0 + R::NK * R::K_SLOT;
    const bool spared = score && CL > 1;
    const int win_first = (spared ? rank - 1 : rank) * SPARSE_WARPS + warp, win_stride = (spared ? CL - 1 : CL) * SPARSE_WARPS;
    const int n_window = (si.n_win + WIDE_TOKENS - 1) / WIDE_TOKENS;
    const int my_windows = !attend || (spared && rank == 0) || win_first >= n_window ? 0 : (n_window - win_first + win_stride - 1) / win_stride;
    // the rows of the k-th of them into the ring, two rows (lanes 0 - 15, 16 - 31) per instruction
    const auto stage_window = [&](int k) {
        if (k < my_windows) {
            const int w0 = (win_first + k * win_stride) * WIDE_TOKENS, last = si.n_win - 1, half = lane >> 4, piece = lane & 15;
            const long long plane = (static_cast<long long>(slot) * c.n_kv + h) * 2;
            const unsigned short* sink = c.sink_kv + plane * c.s_sink * D + piece * 8;
            const unsigned short* recent = c.ring_kv + plane * c.ring_cap * D + piece * 8;
            const int at0 = (si.recent_lo + max(w0 - si.n_sink, 0)) % c.ring_cap - max(w0, si.n_sink);      // ring row of window token w: at0 + w, or ring_cap less
#pragma unroll 2
            for (int j = 0; j < WIDE_TOKENS / 2; ++j) {
                const int r = 2 * j + half, w = min(w0 + r, last);
                const bool in_sink = w < si.n_sink;
                const int at = at0 + w;
                const unsigned short* src = in_sink ? sink + w * D : recent + (at < c.ring_cap ? at : at - c.ring_cap) * D;
                const unsigned dst = k_slot0 + r * (2 * D) + ((piece ^ (r & 7)) << 4);
                copy16(dst, src);
                copy16(dst + WIDE_TOKENS * 2 * D, src + static_cast<long long>(in_sink ? c.s_sink : c.ring_cap) * D);
            }
        }
        copies_commit();
    };

    if (warp < GP) {
        float x[4] = {bf16_bits_to_float(q_bits.x & 0xffff), bf16_bits_to_float(q_bits.x >> 16), bf16_bits_to_float(q_bits.y & 0xffff), bf16_bits_to_float(q_bits.y >> 16)};
        if (warp < G && P.pro.rope)
            norm_rope_warp(x, lane, P.pro, h * G + warp, prologue_position(P.pro, max(S - 1, 0), c.dev_status, lane == 0 && rank == 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) sh.q[warp][4 * lane + e] = static_cast<double>(x[e]);
    }
    __syncthreads();
    BoundsTile tile;
    if (score) tile.load(P, ids, h, 16 * warp, n_here, g, t);
    if (P.ring_offset > 0) stage_window(0);
    double acc[2 * GP];                                 // [row][head]
#pragma unroll
    for (int j = 0; j < 2 * GP; ++j) acc[j] = 0.0;
#pragma unroll
    for (int k0 = 0; k0 < QUADS; k0 += PART) {
        if (k0 > 0) load_T(k0);
#pragma unroll
        for (int k = 0; k < PART; ++k) {
            double tv[2][4];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                tv[r][0] = __uint_as_float(tr[r][k].x); tv[r][1] = __uint_as_float(tr[r][k].y);
                tv[r][2] = __uint_as_float(tr[r][k].z); tv[r][3] = __uint_as_float(tr[r][k].w);
            }
#pragma unroll
            for (int j = 0; j < GP; ++j) {
                const double2* q = reinterpret_cast<const double2*>(&sh.q[j][4 * (seg + TPP * (k0 + k))]);
                const double2 lo = q[0], hi = q[1];
#pragma unroll
                for (int r = 0; r < 2; ++r) acc[r * GP + j] = fma(tv[r][0], lo.x, fma(tv[r][1], lo.y, fma(tv[r][2], hi.x, fma(tv[r][3], hi.y, acc[r * GP + j]))));
            }
        }
    }
    using Sum = GroupSum<2 * GP, TPP>;
    Sum::sum(acc, seg);
    if (Sum::replica(seg) == 0)
#pragma unroll
        for (int i = 0; i < Sum::LEFT; ++i) {
            const int k = Sum::first(seg) + i;
            sh.qc[k % GP][t_row + (k / GP) * PAIRS] = acc[i];
        }
    if (CL > 1) cluster.sync(); else __syncthreads();   // sh.q has been read, too

    // ---- the query as two signed bytes per channel: q' ~ (max|q'| / 32512) (256 hi + lo), in B fragments.  A warp per column pair (or
    // column) of a head; the queries of head slots without a head are zero, and so are their columns.
    if (warp < GP) {
        double x[4], most = 0.0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {                            // from the CTA whose rows they are
            const double2* from = reinterpret_cast<const double2*>(&sh.qc[warp][4 * lane + 2 * e]);
            const double2 v = *(CL > 1 ? cluster.map_shared_rank(from, 4 * lane / ROWS) : from);
            x[2 * e] = v.x; x[2 * e + 1] = v.y;
            most = fmax(most, fmax(fabs(v.x), fabs(v.y)));
        }
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) most = fmax(most, __shfl_xor_sync(FULL, most, o));
        const bool usable = most > 0.0 && most < 3e38;          // otherwise all scores are 0: the lowest pages (NaN compares false)
        constexpr double QM = Q_MAX;
        const double per_unit = usable ? QM / most : 0.0;
        // selection: row byte o of the bounds (lower 0 .. 127, upper 128 .. 255) is word (o % 16) / 4 of lane t = (o % 64) / 16 in group o / 64
        unsigned word[2][2] = {{0u, 0u}, {0u, 0u}};             // [lower, upper][high, low digit]
        unsigned digits[2] = {0u, 0u};                          // attention: [high, low], a byte per channel
        int sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int v = usable ? min(max(__double2int_rn(x[e] * per_unit), -32512), 32512) : 0;
            const int hi_digit = (v + 128) >> 8, lo_digit = v - 256 * hi_digit;
            const unsigned wh = static_cast<unsigned>(hi_digit & 255) << (8 * e), wl = static_cast<unsigned>(lo_digit & 255) << (8 * e);
            digits[0] |= wh; digits[1] |= wl;
            if (v > 0) { word[1][0] |= wh; word[1][1] |= wl; } else { word[0][0] |= wh; word[0][1] |= wl; }
            sum += v;
        }
        unsigned* frag = reinterpret_cast<unsigned*>(sh.frag);
#pragma unroll
        for (int side = 0; side < 2; ++side)
#pragma unroll
            for (int digit = 0; digit < 2; ++digit) {
                const int set = MODE == 0 ? 0 : digit, column = MODE == 0 ? 2 * warp + digit : warp;
                const int group = 2 * side + lane / 16, tl = (lane % 16) / 4;
                frag[((set * 4 + group) * 32 + 4 * column + tl) * 4 + lane % 4] = word[side][digit];
            }
        if (lane == 0) sh.unit[warp] = usable ? static_cast<float>(__dmul_rn(most / QM, static_cast<double>(c.sm_scale))) : 0.f;
        if (attend) {
            // what decode_prep_kernel makes of q' (there from fp32 sums): digits in integer fragments, q' in the scale of the scores'
            // base-2 exponent as bf16 value and remainder, two scalars per head
            const float k2 = c.sm_scale * LOG2E, lam = usable ? static_cast<float>(most / QM) : 1.f;
            unsigned short* ifrag = reinterpret_cast<unsigned short*>(sh.attn);
            unsigned* wfrag = reinterpret_cast<unsigned*>(sh.attn + Shared::QF);
#pragma unroll
            for (int k = 0; k < 2; ++k) {                       // channels ch, ch + 1
                const int ch = 4 * lane + 2 * k, s = ch >> 5, hh = (ch >> 4) & 1, u = (ch >> 3) & 1, tq = (ch >> 1) & 3;
#pragma unroll
                for (int digit = 0; digit < 2; ++digit) {
                    const int set = MODE == 0 ? 0 : digit, column = MODE == 0 ? 2 * warp + digit : warp;
                    ifrag[set * 512 + (((s >> 1) * 32 + 4 * column + tq) * 16 + ((s & 1) * 2 + hh) * 4 + 2 * u) / 2] = static_cast<unsigned short>(digits[digit] >> (16 * k));
                }
                const int s16 = ch >> 4, r = (ch >> 3) & 1;
                float y[2], rest[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    y[e] = static_cast<float>(x[2 * k + e]) * k2;
                    rest[e] = y[e] - bf16_bits_to_float(float_to_bf16_bits(y[e]));
                }
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const int set = MODE == 0 ? 0 : part, column = MODE == 0 ? 2 * warp + part : warp;
                    const float a = part == 0 ? y[0] : rest[0], d = part == 0 ? y[1] : rest[1];
                    wfrag[set * 512 + ((s16 >> 1) * 32 + 4 * column + tq) * 4 + (s16 & 1) * 2 + r] = float_to_bf16_bits(a) | (static_cast<unsigned>(float_to_bf16_bits(d)) << 16);
                }
            }
            sum = __reduce_add_sync(FULL, sum);
            constexpr float FS = BITS != 4 ? 4.f : 16.f;        // the integer score carries this factor (page_scores)
            if (lane == 0) sh.scal[warp] = make_float2(k2 * lam * (1.f / FS), FS * static_cast<float>(sum));
        }
    }
    __syncthreads();

    if (score) {
        // ---- scores of this CTA's pages
        uint4 bq[SETS][4];
#pragma unroll
        for (int k = 0; k < SETS * 4; ++k) bq[k / 4][k % 4] = sh.frag[k * 32 + lane];
        float unit[NH], best[NH], worst[NH];                    // heads per lane: t, or 2 t and 2 t + 1
#pragma unroll
        for (int k = 0; k < NH; ++k) { const int head = MODE == 0 ? t : 2 * t + k; unit[k] = head < G ? sh.unit[head] : 0.f; best[k] = -INFINITY; worst[k] = INFINITY; }
        for (int p0 = 16 * warp; p0 < n_here; p0 += 16 * SPARSE_WARPS) {
            const BoundsTile now = tile;
            if (p0 + 16 * SPARSE_WARPS < n_here) tile.load(P, ids, h, p0 + 16 * SPARSE_WARPS, n_here, g, t);
            int acc_i[SETS][4] = {};
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int st = 0; st < SETS; ++st) {
                    mma_s8(acc_i[st], now.a[0][k].x, now.a[1][k].x, now.a[0][k].y, now.a[1][k].y, bq[st][k].x, bq[st][k].y);
                    mma_s8(acc_i[st], now.a[0][k].z, now.a[1][k].z, now.a[0][k].w, now.a[1][k].w, bq[st][k].z, bq[st][k].w);
                }
#pragma unroll
            for (int rs = 0; rs < 2; ++rs) {
                const int p = p0 + g + 8 * rs;
                if (p >= n_here) continue;
                const float grid = __uint_as_float(static_cast<unsigned>(127 + now.ex[rs]) << 23);
#pragma unroll
                for (int k = 0; k < NH; ++k) {
                    const int head = MODE == 0 ? t : 2 * t + k;
                    if (head >= G) continue;
                    const int dot = MODE == 0 ? 256 * acc_i[0][2 * rs] + acc_i[0][2 * rs + 1] : 256 * acc_i[0][2 * rs + k] + acc_i[SETS - 1][2 * rs + k];
                    // one rounding to 32 bits, one of the product: an order that a plain computation can repeat
                    const float s = now.good[rs] ? __fmul_rn(__int2float_rn(dot) * grid, unit[k]) : -INFINITY;
                    scores[head * per_max + p] = s;
                    best[k] = fmaxf(best[k], s);
                    if (now.good[rs]) worst[k] = fminf(worst[k], s);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < NH; ++k) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                best[k] = fmaxf(best[k], __shfl_xor_sync(FULL, best[k], o));
                worst[k] = fminf(worst[k], __shfl_xor_sync(FULL, worst[k], o));
            }
            const int head = MODE == 0 ? t : 2 * t + k;
            if (g == 0) sh.warp_best[warp][head] = make_float2(best[k], worst[k]);
        }
        __syncthreads();
        sh.bins[tid] = make_uint4(0u, 0u, 0u, 0u);              // in the place of the fragments, which every warp has read
        if (tid < 8 * CL) {
            const int head = tid & 7, peer = tid >> 3;
            float2 m = make_float2(-INFINITY, INFINITY);
            if (head < G)
#pragma unroll
                for (int w = 0; w < SPARSE_WARPS; ++w) { const float2 x = sh.warp_best[w][head]; m.x = fmaxf(m.x, x.x); m.y = fminf(m.y, x.y); }
            float2* to = CL > 1 ? cluster.map_shared_rank(&sh.best[0][0], peer) : &sh.best[0][0];
            to[rank * 8 + head] = m;
        }
        if (CL > 1) cluster.sync(); else __syncthreads();

        // ---- keys: bits of the distance below the best page (smaller is better), counted in bins between 0 and the least range of a
        // head's scores, which no finite key exceeds
        uint2* keys0 = CL > 1 ? cluster.map_shared_rank(keys, 0) : keys;
        float top[GP], width = INFINITY;
#pragma unroll
        for (int j = 0; j < GP; ++j) {
            float2 m = make_float2(-INFINITY, INFINITY);
#pragma unroll
            for (int r = 0; r < CL; ++r) { const float2 x = sh.best[r][j]; m.x = fmaxf(m.x, x.x); m.y = fminf(m.y, x.y); }
            top[j] = m.x == -INFINITY ? 0.f : m.x;
            if (j < G) width = fminf(width, m.x - m.y);
        }
        const float per_bin = width > 0.f && width < INFINITY ? (SELECT_BINS - 1) / width : 0.f;
        for (int p = tid; p < n_here; p += SPARSE_THREADS) {
            float key = -INFINITY;
#pragma unroll
            for (int j = 0; j < GP; ++j) if (j < G) key = fmaxf(key, __fsub_rn(scores[j * per_max + p], top[j]));
            const unsigned u = __float_as_uint(key) & 0x7fffffffu;
            keys0[p_lo + p] = make_uint2(u, static_cast<unsigned>(ids[p]));
            atomicAdd(reinterpret_cast<unsigned*>(sh.bins) + bin_of(u, per_bin), 1u);
        }
        if (CL > 1) cluster.sync(); else __syncthreads();
        if (rank == 0) {
            uint4 counted = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int r = 0; r < CL; ++r) {
                const uint4 x = *(CL > 1 ? cluster.map_shared_rank(&sh.bins[tid], r) : &sh.bins[tid]);
                counted.x += x.x; counted.y += x.y; counted.z += x.z; counted.w += x.w;
            }
            list_pages(sh, counted, per_bin, keys, pages, first, P.n_select, list);
        }
        if (!attend) {
            if (CL > 1) cluster.sync();                         // no CTA leaves while its bins are read
            return;
        }
        if (CL > 1 && rank == 0) __syncthreads();               // the keys' place may become the staging ring
    }

    // ---- attention: this warp's query fragments and state
    unsigned qf[4][2], qfl[MODE == 1 ? 4 : 1][2];
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
        const uint4 v = sh.attn[s2 * 32 + lane];
        qf[2 * s2][0] = v.x; qf[2 * s2][1] = v.y; qf[2 * s2 + 1][0] = v.z; qf[2 * s2 + 1][1] = v.w;
        if (MODE == 1) {
            const uint4 w = sh.attn[64 + s2 * 32 + lane];
            qfl[2 * s2][0] = w.x; qfl[2 * s2][1] = w.y; qfl[2 * s2 + 1][0] = w.z; qfl[2 * s2 + 1][1] = w.w;
        }
    }
    float fmul[NH], gadd[NH];
#pragma unroll
    for (int k = 0; k < NH; ++k) { const float2 v = sh.scal[MODE == 0 ? t : 2 * t + k]; fmul[k] = v.x; gadd[k] = v.y; }
    WarpState<MODE> st;
    st.reset();
    unsigned long long policy;
    if (P.stream_pages) policy = l2_evict_first_policy();
    else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
    // ---- window tokens
    if (score && CL == 1) __syncthreads();                      // the list is complete
#pragma unroll 1
    for (int k = 0; k < my_windows; ++k) {
        if (k > 0 || P.ring_offset == 0) stage_window(k);
        copies_wait<0>();
        wide_window_unit<BITS, MODE>(st, k_slot0, min(WIDE_TOKENS, si.n_win - (win_first + k * win_stride) * WIDE_TOKENS), sh.attn + Shared::QF, lane);
        __syncwarp();
    }
    if (score && CL > 1) cluster.sync();                        // the list is complete

    // ---- the listed pages, 32 of this warp's at a time: lane k looks up the k-th
    const int wid = rank * SPARSE_WARPS + warp;
    constexpr int STRIDE = CL * SPARSE_WARPS;
    for (int base = wid; base < n_listed; base += 32 * STRIDE) {
        const int n = min(32, (n_listed - base + STRIDE - 1) / STRIDE);
        int my_entry = -1, my_page = -1;
        if (lane < n) {
            const int u = base + lane * STRIDE;
            if (score && u < LISTED) {
                const uint2 e = *(CL > 1 ? cluster.map_shared_rank(&sh.listed[u], 0) : &sh.listed[u]);
                my_entry = static_cast<int>(e.x);
                my_page = static_cast<int>(e.y);                // -1: flagged when it was scored
            } else if ((my_entry = given || score ? __ldcg(list + u) : first + u) != -1) {
                const bool inside = my_entry >= first && my_entry < first + pages;
                const int page = inside ? __ldg(row + my_entry) : -1;
                if (page >= 0 && page < c.n_pages) my_page = page;
                else atomicOr(c.dev_status, WUSHKV_DEV_BAD_PAGE_ID);
            }
        }
        const unsigned all_there = __ballot_sync(FULL, my_page >= 0);
        unsigned there = all_there, k_todo = there, v_todo = there;      // units of this warp, and those whose keys and values are not yet requested
        int ki = 0, vi = 0, k_slot = 0, v_slot = 0;             // slots of the next copies, of the unit at hand
        const auto copy_side = [&](unsigned dst, const unsigned char* src, int bytes) {
#pragma unroll
            for (int i = 0; i < (bytes + 511) / 512; ++i)
                if (bytes % 512 == 0 || 512 * i + 16 * lane < bytes) copy16_hint(dst + 512 * i + 16 * lane, src + 512 * i + 16 * lane, policy);
        };
        const auto copy_page = [&](bool value, unsigned& todo) {
            if (todo) {
                const int page = __shfl_sync(FULL, my_page, __ffs(todo) - 1);
                todo &= todo - 1;
                const unsigned char* rec = c.pages + (static_cast<long long>(page) * c.n_kv + h) * record_bytes(BITS);
                if (value) {
                    copy_side(v_slot0 + vi * R::V_SLOT, rec + v_codes_offset(BITS), side_bytes(BITS));
                    vi = vi + 1 == R::NV ? 0 : vi + 1;
                } else {
                    copy_side(k_slot0 + ki * R::K_SLOT, rec, side_bytes(BITS));
                    copy_side(k_slot0 + ki * R::K_SLOT + side_bytes(BITS), rec + meta_offset(BITS), R::META);
                    ki = ki + 1 == R::NK ? 0 : ki + 1;
                }
            }
            copies_commit();
        };
        // steps -2, -1 only request; every copy has one place in the code, which is executed once or twice per launch and fetched each time
        constexpr int AHEAD = R::NK > R::NV ? R::NK : R::NV;
#pragma unroll 1
        for (int step = -AHEAD; step < __popc(all_there); ++step) {
            float sc[4][2 * NH];          // [block][row g: heads..., row g+8: heads...]
            unsigned vmeta[4][2];         // fp16x2 (Delta_v, x_min_v) of rows g, g+8
            if (step >= 0) {
                const int pos0 = __shfl_sync(FULL, my_entry, __ffs(there) - 1) * PAGE_TOKENS;
                there &= there - 1;
                const unsigned ks = k_slot0 + k_slot * R::K_SLOT;
                k_slot = k_slot + 1 == R::NK ? 0 : k_slot + 1;
                copies_wait<R::K_PENDING>();
                page_scores<BITS, MODE>(ks, ks + side_bytes(BITS), qf, qfl, gadd, sc, vmeta, lane);
                __syncwarp();
                if (pos0 < si.q_lo || pos0 + PAGE_TOKENS > si.q_hi) {      // first / last page of the quantized range: mask the tokens outside it
#pragma unroll
                    for (int bi = 0; bi < 4; ++bi)
#pragma unroll
                        for (int rs = 0; rs < 2; ++rs) {
                            const int p = pos0 + bi * 16 + 8 * rs + g;
                            if (p < si.q_lo || p >= si.q_hi) {
                                vmeta[bi][rs] = 0u;
#pragma unroll
                                for (int j = 0; j < NH; ++j) sc[bi][rs * NH + j] = -INFINITY;
                            }
                        }
                }
            }
            if (step >= -R::NK) copy_page(false, k_todo);       // into the slot just read
            if (step >= 0) {
                float mx[NH];
#pragma unroll
                for (int j = 0; j < NH; ++j) {
                    const float v = fmaxf(fmaxf(fmaxf(sc[0][j], sc[0][NH + j]), fmaxf(sc[1][j], sc[1][NH + j])),
                                          fmaxf(fmaxf(sc[2][j], sc[2][NH + j]), fmaxf(sc[3][j], sc[3][NH + j])));
                    mx[j] = v * fmul[j];      // scores are kept divided by the head's multiplier (> 0)
                }
                st.raise_max(mx);
                const unsigned vs = v_slot0 + v_slot * R::V_SLOT;
                v_slot = v_slot + 1 == R::NV ? 0 : v_slot + 1;
                copies_wait<R::V_PENDING>();
                page_values<BITS, MODE>(st, vs, sc, vmeta, fmul, lane);
                __syncwarp();
            }
            if (step >= -R::NV) copy_page(true, v_todo);
        }
        copies_wait<0>();
    }

    // ---- merge: the CTA's eight states, then the cluster's
    __syncwarp();
    store_state<BITS, MODE, false>(st, reinterpret_cast<float*>(ring), lane, G);
    __syncthreads();                                             // sh.attn has been read, too
    if (warp < G) {
        MergedState ms;
        ms.reset();
        ms.add<false>(SPARSE_WARPS, lane, [&](int k) { return reinterpret_cast<const float*>(rings + k * R::BYTES) + warp * PART_STRIDE; });
        if (CL > 1) ms.store(sh.merged[warp], lane);
        else ms.finish(P.O + (static_cast<long long>(b) * c.n_q + h * G + warp) * D, lane);
    }
    if (CL > 1) {
        cluster.sync();
        const int head = warp * CL + rank;
        if (head < G) {
            MergedState ms;
            ms.reset();
            const unsigned long long from = lane < CL ? reinterpret_cast<unsigned long long>(cluster.map_shared_rank(&sh.merged[head][0], lane)) : 0ull;
            ms.add<false>(CL, lane, [&](int k) { return reinterpret_cast<const float*>(__shfl_sync(FULL, from, k)); });
            ms.finish(P.O + (static_cast<long long>(b) * c.n_q + h * G + head) * D, lane);
        }
        cluster.sync();                                          // no CTA leaves while another reads its results
    }
}

// Upper bound of the packed pages of a sequence of at most max_seq_len tokens.
static long long candidate_bound(const CacheView& c, int max_seq_len) {
    const int nq = n_quantized(max_seq_len - c.lag, c.s_sink, c.s_keep, c.s_flush);
    return nq > 0 ? (c.s_sink + nq - 1) / PAGE_TOKENS - c.s_sink / PAGE_TOKENS + 1 : 0;
}

constexpr int SPARSE_SMEM_MAX = 226 * 1024, SPARSE_SMEM_HALF = 113 * 1024;      // of a CTA; of one of two on an SM
__host__ __device__ constexpr size_t scored_bytes(size_t group, size_t per, size_t pages) { return (4 * (1 + group) * per + 8 * pages + 15) / 16 * 16; }
static_assert(sizeof(SparseShared<1>) + scored_bytes(8, MAX_SELECT_PAGES / 8, MAX_SELECT_PAGES) <= SPARSE_SMEM_MAX, "clusters of 8 hold every allowed number of pages");

// Shared memory of a CTA and where in it the rings begin.
template <int BITS, int MODE>
static size_t sparse_smem(const SparseParams& P, int cl, int& ring_offset) {
    const size_t scored = P.bounds ? scored_bytes(P.c.G, pages_per_cta(P.max_candidates, cl), P.max_candidates) : 0;
    const size_t ring = P.O ? SPARSE_WARPS * Ring<BITS>::BYTES : 0, apart = sizeof(SparseShared<MODE>) + scored + ring;
    // apart from the scores unless that costs the second CTA of an SM one that would come
    const bool alone = static_cast<long long>(P.batch) * P.c.n_kv * cl <= sm_count();
    ring_offset = 0;
    if (scored > 0 && ring > 0 && apart <= (alone ? SPARSE_SMEM_MAX : SPARSE_SMEM_HALF)) { ring_offset = static_cast<int>(scored); return apart; }
    return sizeof(SparseShared<MODE>) + std::max(scored, ring);
}

template <int BITS, int MODE, int CL>
static int launch_sparse_cl(SparseParams P, cudaStream_t st) {
    const auto kernel = sparse_decode_kernel<BITS, MODE, CL>;
    if (!opt_in_dynamic_smem(reinterpret_cast<const void*>(kernel), SPARSE_SMEM_MAX)) return WUSHKV_ECUDA;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CL; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CL, P.c.n_kv, P.batch);
    cfg.blockDim = dim3(SPARSE_THREADS);
    cfg.dynamicSmemBytes = sparse_smem<BITS, MODE>(P, CL, P.ring_offset);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = CL > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, P) == cudaSuccess ? WUSHKV_OK : WUSHKV_ECUDA;
}

template <int BITS, int MODE>
static int launch_sparse_mode(const SparseParams& P, cudaStream_t st) {
    // CTAs per (sequence, KV head): enough for every SM to have one, but no fewer than 16 pages to score per warp, or (where pages are
    // not scored) one unit of attention
    const long long clusters = static_cast<long long>(P.batch) * P.c.n_kv;
    const long long work = std::max<long long>(P.bounds ? P.max_candidates / 16 : 0, P.O ? P.n_select : 0);
    int cl = knobs().select_cluster;
    if (cl != 2 && cl != 4 && cl != 8) cl = 1;
    while (knobs().select_cluster == 0 && cl < 8 && clusters * cl < sm_count() && work > static_cast<long long>(cl) * SPARSE_WARPS) cl *= 2;
    int offset;
    while (cl < 8 && sparse_smem<BITS, MODE>(P, cl, offset) > SPARSE_SMEM_MAX) cl *= 2;
    switch (cl) {
        case 1: return launch_sparse_cl<BITS, MODE, 1>(P, st);
        case 2: return launch_sparse_cl<BITS, MODE, 2>(P, st);
        case 4: return launch_sparse_cl<BITS, MODE, 4>(P, st);
        default: return launch_sparse_cl<BITS, MODE, 8>(P, st);
    }
}

// Checks and launches all three calls: bounds == nullptr: the list is an input; O == nullptr: the list is all that is asked for.
static int sparse_impl(const wushkv_cache* cache, int32_t batch, const int32_t* slot, const int32_t* seq_len, int32_t max_seq_len, const uint16_t* Q,
                       const wushkv_prologue* prologue, const int8_t* bounds, const int8_t* exponents, int32_t n_select, int32_t* selected, uint16_t* O, void* stream) {
    SparseParams P;
    const int rc = make_view(cache, P.c);
    if (rc != WUSHKV_OK) return rc;
    if (batch <= 0 || batch > 65535 || P.c.n_kv > 65535 || max_seq_len <= 0 || n_select <= 0) return WUSHKV_EINVAL;
    if (!slot || !seq_len || !Q || !selected || !aligned(Q, 16) || !aligned(bounds, 16) || !aligned(O, 16)) return WUSHKV_EINVAL;
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
    const bool mode0 = P.c.G <= 4;
    if (P.c.bits == 2) return mode0 ? launch_sparse_mode<2, 0>(P, st) : launch_sparse_mode<2, 1>(P, st);
    if (P.c.bits == 3) return mode0 ? launch_sparse_mode<3, 0>(P, st) : launch_sparse_mode<3, 1>(P, st);
    return mode0 ? launch_sparse_mode<4, 0>(P, st) : launch_sparse_mode<4, 1>(P, st);
}

}  // namespace wushkv

using namespace wushkv;

extern "C" int wushkv_update_page_bounds(const wushkv_cache* cache, int32_t batch, const int32_t* slot, const int32_t* seq_len, const int32_t* cu_new,
                                         int32_t max_new, int8_t* bounds, int8_t* exponents, void* stream) {
    BoundsParams P;
    const int rc = make_view(cache, P.c);
    if (rc != WUSHKV_OK) return rc;
    if (batch <= 0 || batch > 65535 || max_new < 0 || !slot || !seq_len || !cu_new || !bounds || !exponents || !aligned(bounds, 16)) return WUSHKV_EINVAL;
    if (max_new == 0) return WUSHKV_OK;
    P.slot = slot; P.seq_len = seq_len; P.cu_new = cu_new; P.bounds = bounds; P.exponents = exponents;
    const long long pages = (static_cast<long long>(max_new) + PAGE_TOKENS - 2) / PAGE_TOKENS + 1;       // that max_new consecutive tokens can touch
    const dim3 grid(static_cast<unsigned>((pages * P.c.n_kv + 7) / 8), batch);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (P.c.bits == 2) page_bounds_kernel<2><<<grid, 256, 0, st>>>(P);
    else if (P.c.bits == 3) page_bounds_kernel<3><<<grid, 256, 0, st>>>(P);
    else page_bounds_kernel<4><<<grid, 256, 0, st>>>(P);
    return cudaPeekAtLastError() == cudaSuccess ? WUSHKV_OK : WUSHKV_ECUDA;
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
    if (make_view(cache, v) != WUSHKV_OK || batch <= 0 || max_seq_len <= 0 || n_select <= 0) return 0;
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
