// Bounds of packed pages and the selection of pages by them (the attention over the selected pages is in decode.cu).
//
// A page and head keeps, beside its packed record, 257 bytes: for every channel the smallest and the largest dequantized key
// of the page's tokens, rounded outwards to multiples of a power of two that is common to the page and head,
//     e = least integer >= -31 with max |khat| <= 127 * 2^e,  lower = floor(min khat / 2^e),  upper = ceil(max khat / 2^e).
// With them the largest score that any token of the page can reach against a query q' is
//     2^e * sum_c ( max(q'_c, 0) upper_c + min(q'_c, 0) lower_c ),
// a dot product of 256 terms.  The query enters as 16-bit fixed point (two signed bytes per channel), so that the sum is an
// exact integer from mma.sync.m16n8k32 (s8 x s8): scores, and with them the selected pages, do not depend on the order of any
// summation.  q' itself is formed in 64 bits for the same reason: its rounding to 16 bits then is the same wherever it is done.
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "host_common.h"
#include "sparse.cuh"

namespace wushkv {

namespace cg = cooperative_groups;

constexpr unsigned FULL = 0xffffffffu;
constexpr int MIN_EXPONENT = -31, MAX_EXPONENT = 14;      // of 2^e: fp16 steps and offsets reach from 2^-24 to 2^20
constexpr double Q_MAX = 32512.0;                         // 127 * 256: both digits of the fixed-point query fit a signed byte
constexpr float LOG2E = 1.4426950408889634f;

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
// selection
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_s8(int (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int SELECT_THREADS = 256, SELECT_WARPS = SELECT_THREADS / 32;
constexpr int SELECT_BINS = 4 * SELECT_THREADS;

// Shared memory of a CTA: fixed part, then the scores of its pages [heads][per], then (CTA 0) the keys of all pages.
struct SelectShared {
    double q[8][D];                   // the queries, in 64 bits
    double qc[8][D];                  // q' of all CTAs' rows
    uint4 frag[2 * 4 * 32];           // B fragments: [digit set][64 bytes of bounds][lane]
    uint4 attn[128 + 256];            // the attention's integer and bf16 fragments of the head
    uint4 bins[SELECT_THREADS];       // CTA 0: pages per bin of the range of keys
    float unit[8];                    // score of one unit of 2^e dot
    float warp_best[SELECT_WARPS][8];
    float best[8][8];                 // per CTA of the cluster: largest score of its pages, per head
    int scan[SELECT_WARPS];
    unsigned most;                    // CTA 0: largest finite key
    int bin, before, inside;          // CTA 0: the bin of the n_select-th key, keys in the bins ahead, keys in it
    unsigned kth;
    int n_list;
    unsigned list[SELECT_THREADS];    // keys of that bin
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

// Sums NV numbers per lane over groups of LANES lanes.  While there are several, each step hands half of them to the other side;
// afterwards lane l of the group holds the totals of FIRST(l) .. FIRST(l) + LEFT - 1, and REPLICAS lanes hold the same.
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

// One tile of 16 pages as a lane reads it: 64 bytes of the bounds of rows g and g + 8 and the rows' exponents.
struct BoundsTile {
    uint4 a[2][4];
    int ex[2];
    bool good[2];
    __device__ __forceinline__ void load(const SelectParams& P, const int* table, int h, int p0, int p_hi, int g, int t) {
#pragma unroll
        for (int rs = 0; rs < 2; ++rs) {
            const int p = p0 + g + 8 * rs;
            const int page = p < p_hi ? __ldg(table + p) : -1;
            good[rs] = page >= 0 && page < P.c.n_pages;
            if (p < p_hi && !good[rs] && t == 0) atomicOr(P.c.dev_status, WUSHKV_DEV_BAD_PAGE_ID);
            const long long ph = static_cast<long long>(good[rs] ? page : 0) * P.c.n_kv + h;
            const uint4* src = reinterpret_cast<const uint4*>(P.bounds + ph * 2 * D) + t;
#pragma unroll
            for (int k = 0; k < 4; ++k) a[rs][k] = ld_early(src + 4 * k);
            ex[rs] = ld_early_s8(P.exponents + ph);
        }
    }
};

// One cluster of CL CTAs per (sequence, KV head).
//   1. q' = T_K^{-T} q: each CTA forms 128 / CL rows of it and hands them to the others through distributed shared memory.
//   2. Each CTA scores its share of the pages, 16 pages per warp and step: bounds straight from global memory into the A
//      fragments (their bytes are consecutive in k, so that one 16-byte load per lane and row is two registers of two k-steps).
//      The first step's loads are in flight during 1, the next step's during each step.
//   3. The largest score per head of all CTAs, the key of every page (how far it is below the best page of the head that it
//      matters most to), sent to CTA 0.
//   4. CTA 0 counts the keys in bins of equal width, finds the bin of the n_select-th smallest and its rank there by comparing
//      the bin's few keys with each other, and lists the pages.
// All of it is latency: the bounds of 16 sequences x 8 heads x 510 pages are 17 MB, 2.6 us at the copy rate.
template <int MODE, int CL>
__global__ void __launch_bounds__(SELECT_THREADS) select_pages_kernel(SelectParams P) {
    constexpr int GP = MODE == 0 ? 4 : 8, SETS = MODE == 0 ? 1 : 2;
    extern __shared__ __align__(16) unsigned char select_smem[];
    SelectShared& sh = *reinterpret_cast<SelectShared*>(select_smem);
    cg::cluster_group cluster = cg::this_cluster();
    const CacheView& c = P.c;
    const int rank = static_cast<int>(cluster.block_rank()), h = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, G = c.G;
    pdl_wait();
    pdl_launch_dependents();
    // nobody writes into another CTA's shared memory before that CTA has come here and zeroed what the others add to
    if (tid == 0) { sh.most = 0u; sh.n_list = 0; }
    if (CL > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");

    // ---- candidates
    const int S = __ldcg(P.seq_len + b), slot = P.slot[b];
    int* out = P.selected + (static_cast<long long>(b) * c.n_kv + h) * P.n_select;
    int pages = 0, first = 0;
    if (slot < 0 || slot >= c.n_slots) {
        if (rank == 0 && h == 0 && tid == 0) atomicOr(c.dev_status, WUSHKV_DEV_BAD_SLOT);
    } else if (S > 0) {
        const int nq = n_quantized(S - c.lag, c.s_sink, c.s_keep, c.s_flush);
        first = c.s_sink / PAGE_TOKENS;
        pages = nq > 0 ? (c.s_sink + nq - 1) / PAGE_TOKENS - first + 1 : 0;
        if (first + pages > c.max_pages) {
            if (rank == 0 && h == 0 && tid == 0) atomicOr(c.dev_status, WUSHKV_DEV_PAGE_TABLE_FULL);
            pages = max(c.max_pages - first, 0);
        }
        if (pages > P.max_candidates) {                 // a sequence longer than promised
            if (rank == 0 && h == 0 && tid == 0) atomicOr(c.dev_status, WUSHKV_DEV_BAD_COUNT);
            pages = P.max_candidates;
        }
    }
    const bool all = pages <= P.n_select;               // the same for the whole cluster
    const bool prepare = P.qfrag != nullptr;
    if (all) {
        if (rank == 0)
            for (int i = tid; i < P.n_select; i += SELECT_THREADS) out[i] = i < pages ? first + i : -1;
        if (!prepare) {
            if (CL > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
            return;
        }
        pages = 0;                                      // nothing to score
    }
    const int per_max = pages_per_cta(P.max_candidates, CL);
    float* scores = reinterpret_cast<float*>(select_smem + sizeof(SelectShared));            // [G][per_max]
    unsigned* keys = reinterpret_cast<unsigned*>(scores + static_cast<size_t>(G) * per_max);
    const int per = pages_per_cta(pages, CL), p_lo = min(rank * per, pages), p_hi = min(p_lo + per, pages);
    const int* table = c.page_table + static_cast<long long>(slot) * c.max_pages + first;

    // ---- q', two rows per thread (a query element read from shared memory serves both)
    constexpr int ROWS = D / CL, PAIRS = ROWS / 2, TPP = SELECT_THREADS / PAIRS, QUADS = D / 4 / TPP;      // threads per pair of rows, float4 per thread and row
    const int row = rank * ROWS + tid / TPP, seg = tid % TPP;
    const uint4* T = reinterpret_cast<const uint4*>(c.T_K_invT + (static_cast<long long>(h) * D + row) * D);
    uint4 tr[2][QUADS];
#pragma unroll
    for (int k = 0; k < QUADS; ++k) { tr[0][k] = ld_early(T + seg + TPP * k); tr[1][k] = ld_early(T + PAIRS * (D / 4) + seg + TPP * k); }
    BoundsTile tile;
    if (!all) tile.load(P, table, h, p_lo + 16 * warp, p_hi, g, t);
    if (warp < GP) {
        float x[4] = {0.f, 0.f, 0.f, 0.f};              // slots without a head are zero
        if (warp < G) {
            const uint2 w = *reinterpret_cast<const uint2*>(P.Q + (static_cast<long long>(b) * c.n_q + h * G + warp) * D + 4 * lane);
            x[0] = bf16_bits_to_float(w.x & 0xffff); x[1] = bf16_bits_to_float(w.x >> 16);
            x[2] = bf16_bits_to_float(w.y & 0xffff); x[3] = bf16_bits_to_float(w.y >> 16);
            if (P.pro.rope)
                norm_rope_warp(x, lane, P.pro, h * G + warp, prologue_position(P.pro, max(S - 1, 0), c.dev_status, lane == 0 && rank == 0));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sh.q[warp][4 * lane + e] = static_cast<double>(x[e]);
    }
    sh.bins[tid] = make_uint4(0u, 0u, 0u, 0u);
    for (int i = tid; i < SETS * 4 * 32; i += SELECT_THREADS) sh.frag[i] = make_uint4(0u, 0u, 0u, 0u);      // columns without a head
    if (prepare)
        for (int i = tid; i < 128 + 256; i += SELECT_THREADS) sh.attn[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    double acc[2 * GP];                                 // [row][head]
#pragma unroll
    for (int j = 0; j < 2 * GP; ++j) acc[j] = 0.0;
#pragma unroll
    for (int k = 0; k < QUADS; ++k) {
        double tv[2][4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            tv[r][0] = __uint_as_float(tr[r][k].x); tv[r][1] = __uint_as_float(tr[r][k].y);
            tv[r][2] = __uint_as_float(tr[r][k].z); tv[r][3] = __uint_as_float(tr[r][k].w);
        }
#pragma unroll
        for (int j = 0; j < GP; ++j) {
            const double2* q = reinterpret_cast<const double2*>(&sh.q[j][4 * (seg + TPP * k)]);
            const double2 lo = q[0], hi = q[1];
#pragma unroll
            for (int r = 0; r < 2; ++r) acc[r * GP + j] = fma(tv[r][0], lo.x, fma(tv[r][1], lo.y, fma(tv[r][2], hi.x, fma(tv[r][3], hi.y, acc[r * GP + j]))));
        }
    }
    using Sum = GroupSum<2 * GP, TPP>;
    Sum::sum(acc, seg);
    if (CL > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
#pragma unroll
    for (int peer = 0; peer < CL; ++peer) {
        if (peer % Sum::REPLICAS != Sum::replica(seg)) continue;
        double* q_of = CL > 1 ? cluster.map_shared_rank(&sh.qc[0][0], peer) : &sh.qc[0][0];
#pragma unroll
        for (int i = 0; i < Sum::LEFT; ++i) {
            const int k = Sum::first(seg) + i;
            q_of[(k % GP) * D + row + (k / GP) * PAIRS] = acc[i];
        }
    }
    if (CL > 1) cluster.sync(); else __syncthreads();

    // ---- the query as two signed bytes per channel: q' ~ (max|q'| / 32512) (256 hi + lo), in B fragments.  Row byte o of the
    // bounds (lower 0 .. 127, upper 128 .. 255) is word (o % 16) / 4 of lane t = (o % 64) / 16 in group o / 64.
    if (warp < G) {
        double x[4], most = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = sh.qc[warp][4 * lane + e]; most = fmax(most, fabs(x[e])); }
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) most = fmax(most, __shfl_xor_sync(FULL, most, o));
        const bool usable = most > 0.0 && most < 3e38;          // otherwise all scores are 0: the lowest pages
        const double per_unit = usable ? Q_MAX / most : 0.0;
        unsigned word[2][2] = {{0u, 0u}, {0u, 0u}};             // [lower, upper][high, low digit]
        unsigned digits[2] = {0u, 0u};                          // the same of the attention: [high, low], a byte per channel
        int sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int v = usable ? min(max(__double2int_rn(x[e] * per_unit), -32512), 32512) : 0;
            const int hi_digit = (v + 128) >> 8, lo_digit = v - 256 * hi_digit;
            digits[0] |= static_cast<unsigned>(hi_digit & 255) << (8 * e);
            digits[1] |= static_cast<unsigned>(lo_digit & 255) << (8 * e);
            sum += v;
            const unsigned wh = static_cast<unsigned>(hi_digit & 255) << (8 * e), wl = static_cast<unsigned>(lo_digit & 255) << (8 * e);
            if (v > 0) { word[1][0] |= wh; word[1][1] |= wl; } else { word[0][0] |= wh; word[0][1] |= wl; }
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
        if (lane == 0) sh.unit[warp] = usable ? static_cast<float>(__dmul_rn(most / Q_MAX, static_cast<double>(c.sm_scale))) : 0.f;
        if (prepare && rank == CL - 1) {
            // what decode_prep_kernel makes of q' (there from fp32 sums): digits in integer fragments, q' in the scale of the scores'
            // base-2 exponent as bf16 value and remainder, two scalars per head
            const float k2 = c.sm_scale * LOG2E, lam = usable ? static_cast<float>(most / Q_MAX) : 1.f;
            unsigned short* ifrag = reinterpret_cast<unsigned short*>(sh.attn);
            unsigned* wfrag = reinterpret_cast<unsigned*>(sh.attn + (MODE == 0 ? 64 : 128));
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
            if (lane == 0) {
                const float fs = c.bits != 4 ? 4.f : 16.f;      // the integer score of the main kernel carries this factor
                reinterpret_cast<float2*>(P.qscal)[static_cast<long long>(b) * c.n_q + h * G + warp] = make_float2(k2 * lam / fs, fs * static_cast<float>(sum));
            }
        }
    }
    __syncthreads();
    if (prepare && rank == CL - 1) {
        constexpr int QF = MODE == 0 ? 64 : 128, QW = MODE == 0 ? 128 : 256;
        const long long bh = static_cast<long long>(b) * c.n_kv + h;
        if (tid < 8) arrival_counters(P.qfrag, bh)[tid] = 0;
        if (tid < QF) P.qfrag[bh * 256 + tid] = sh.attn[tid];
        if (tid < QW) P.qwfrag[bh * 256 + tid] = sh.attn[QF + tid];
        if (P.plan && h == 0 && b == 0) write_plan(c, P.batch, P.seq_len, P.slot, P.n_select, P.plan);
    }
    if (all) return;

    // ---- scores of this CTA's pages
    uint4 bq[SETS][4];
#pragma unroll
    for (int k = 0; k < SETS * 4; ++k) bq[k / 4][k % 4] = sh.frag[k * 32 + lane];
    constexpr int NH = MODE == 0 ? 1 : 2;                       // heads per lane: t, or 2 t and 2 t + 1
    float unit[NH], best[NH];
#pragma unroll
    for (int k = 0; k < NH; ++k) { const int head = MODE == 0 ? t : 2 * t + k; unit[k] = head < G ? sh.unit[head] : 0.f; best[k] = -INFINITY; }
    for (int p0 = p_lo + 16 * warp; p0 < p_hi; p0 += 16 * SELECT_WARPS) {
        const BoundsTile now = tile;
        if (p0 + 16 * SELECT_WARPS < p_hi) tile.load(P, table, h, p0 + 16 * SELECT_WARPS, p_hi, g, t);
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
            if (p >= p_hi) continue;
            const float grid = __uint_as_float(static_cast<unsigned>(127 + now.ex[rs]) << 23);
#pragma unroll
            for (int k = 0; k < NH; ++k) {
                const int head = MODE == 0 ? t : 2 * t + k;
                if (head >= G) continue;
                const int dot = MODE == 0 ? 256 * acc_i[0][2 * rs] + acc_i[0][2 * rs + 1] : 256 * acc_i[0][2 * rs + k] + acc_i[SETS - 1][2 * rs + k];
                // one rounding to 32 bits, one of the product: an order that a plain computation can repeat
                const float s = now.good[rs] ? __fmul_rn(__int2float_rn(dot) * grid, unit[k]) : -INFINITY;
                scores[head * per_max + p - p_lo] = s;
                best[k] = fmaxf(best[k], s);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < NH; ++k) {
        best[k] = fmaxf(best[k], __shfl_xor_sync(FULL, best[k], 4));
        best[k] = fmaxf(best[k], __shfl_xor_sync(FULL, best[k], 8));
        best[k] = fmaxf(best[k], __shfl_xor_sync(FULL, best[k], 16));
        const int head = MODE == 0 ? t : 2 * t + k;
        if (g == 0) sh.warp_best[warp][head] = best[k];
    }
    __syncthreads();
    if (tid < 8 * CL) {
        const int head = tid & 7, peer = tid >> 3;
        float m = -INFINITY;
        if (head < G)
#pragma unroll
            for (int w = 0; w < SELECT_WARPS; ++w) m = fmaxf(m, sh.warp_best[w][head]);
        float* to = CL > 1 ? cluster.map_shared_rank(&sh.best[0][0], peer) : &sh.best[0][0];
        to[rank * 8 + head] = m;
    }
    if (CL > 1) cluster.sync(); else __syncthreads();

    // ---- keys: bits of the distance below the best page (smaller is better)
    unsigned* keys0 = CL > 1 ? cluster.map_shared_rank(keys, 0) : keys;
    float top[GP];
#pragma unroll
    for (int j = 0; j < GP; ++j) {
        float m = -INFINITY;
#pragma unroll
        for (int r = 0; r < CL; ++r) m = fmaxf(m, sh.best[r][j]);
        top[j] = m == -INFINITY ? 0.f : m;
    }
    constexpr unsigned INF_BITS = 0x7f800000u;
    unsigned most = 0u;
    for (int p = p_lo + tid; p < p_hi; p += SELECT_THREADS) {
        float key = -INFINITY;
#pragma unroll
        for (int j = 0; j < GP; ++j) if (j < G) key = fmaxf(key, __fsub_rn(scores[j * per_max + p - p_lo], top[j]));
        const unsigned u = __float_as_uint(key) & 0x7fffffffu;
        keys0[p] = u;
        if (u < INF_BITS) most = max(most, u);
    }
    most = __reduce_max_sync(FULL, most);
    if (lane == 0 && most > 0u) atomicMax(CL > 1 ? cluster.map_shared_rank(&sh.most, 0) : &sh.most, most);
    if (CL > 1) cluster.sync(); else __syncthreads();
    if (rank == 0) {
        // ---- bins of equal width from 0 to the largest key; the product is monotonic in the key, so bins are in the keys' order
        const float width = __uint_as_float(sh.most), per_bin = width > 0.f ? (SELECT_BINS - 1) / width : 0.f;
        const auto bin_of = [&](unsigned u) {
            return u < INF_BITS ? min(static_cast<int>(__uint_as_float(u) * per_bin), SELECT_BINS - 1) : SELECT_BINS - 1;
        };
        unsigned* bins = reinterpret_cast<unsigned*>(sh.bins);
        for (int p = tid; p < pages; p += SELECT_THREADS) atomicAdd(bins + bin_of(keys[p]), 1u);
        const auto prefix = [&](int x) {                        // exclusive prefix sum over the CTA
            int incl = x;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(FULL, incl, o);
                if (lane >= o) incl += y;
            }
            if (lane == 31) sh.scan[warp] = incl;
            __syncthreads();
            int before = 0;
#pragma unroll
            for (int w = 0; w < SELECT_WARPS; ++w) before += w < warp ? sh.scan[w] : 0;
            return before + incl - x;
        };
        __syncthreads();
        const uint4 mine = sh.bins[tid];
        const int counts[4] = {static_cast<int>(mine.x), static_cast<int>(mine.y), static_cast<int>(mine.z), static_cast<int>(mine.w)};
        int before = prefix(counts[0] + counts[1] + counts[2] + counts[3]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (before < P.n_select && P.n_select <= before + counts[e]) { sh.bin = 4 * tid + e; sh.before = before; sh.inside = counts[e]; }
            before += counts[e];
        }
        __syncthreads();
        const int bin = sh.bin, inside = sh.inside, wanted = P.n_select - sh.before - 1;      // rank of the n_select-th key in its bin
        unsigned kth = 0u;
        if (inside <= SELECT_THREADS) {
            for (int p = tid; p < pages; p += SELECT_THREADS) {
                const unsigned u = keys[p];
                if (bin_of(u) == bin) sh.list[atomicAdd(&sh.n_list, 1)] = u;
            }
            __syncthreads();
            if (tid < inside) {
                const unsigned u = sh.list[tid];
                int less = 0, same = 0;
                for (int k = 0; k < inside; ++k) { less += sh.list[k] < u; same += sh.list[k] == u; }
                if (less <= wanted && wanted < less + same) sh.kth = u;      // equal keys write the same
            }
            __syncthreads();
            kth = sh.kth;
        } else {
            // many keys that are (almost) the same: bit by bit, the largest v with fewer than n_select keys below it
            for (int bit = 30; bit >= 0; --bit) {
                const unsigned cand = kth | (1u << bit);
                int n = 0;
                for (int p = tid; p < pages; p += SELECT_THREADS) n += keys[p] < cand;
                n = __reduce_add_sync(FULL, n);
                __syncthreads();
                if (lane == 0) sh.scan[warp] = n;
                __syncthreads();
                int total = 0;
#pragma unroll
                for (int w = 0; w < SELECT_WARPS; ++w) total += sh.scan[w];
                if (total < P.n_select) kth = cand;
            }
        }
        __syncthreads();                                        // the readers of sh.scan
        // ---- all below it, and of those equal to it the first ones; every thread lists a run of consecutive pages
        const int run = (pages + SELECT_THREADS - 1) / SELECT_THREADS, r_lo = min(tid * run, pages), r_hi = min(r_lo + run, pages);
        int below = 0, equal = 0;
        for (int p = r_lo; p < r_hi; ++p) { below += keys[p] < kth; equal += keys[p] == kth; }
        static_assert(MAX_SELECT_PAGES < (1 << 15), "two counts in one prefix sum");
        const int packed = prefix((below << 16) + equal);
        int all_below = 0;
#pragma unroll
        for (int w = 0; w < SELECT_WARPS; ++w) all_below += sh.scan[w] >> 16;
        int below_before = packed >> 16, equal_before = packed & 0xffff;
        const int room = P.n_select - all_below;          // places for keys equal to the n_select-th
        for (int p = r_lo; p < r_hi; ++p) {
            const unsigned k = keys[p];
            if (k < kth) { out[below_before + min(equal_before, room)] = first + p; ++below_before; }
            else if (k == kth) { if (equal_before < room) out[below_before + equal_before] = first + p; ++equal_before; }
        }
    }
}

constexpr int SELECT_SMEM_MAX = 200 * 1024;
static_assert(sizeof(SelectShared) + 4 * (8 * MAX_SELECT_PAGES / 8 + MAX_SELECT_PAGES) <= SELECT_SMEM_MAX, "clusters of 8 hold every allowed number of pages");

template <int MODE, int CL>
static int launch_select_cl(const SelectParams& P, cudaStream_t st) {
    const auto kernel = select_pages_kernel<MODE, CL>;
    const size_t smem = sizeof(SelectShared) + sizeof(float) * (static_cast<size_t>(P.c.G) * pages_per_cta(P.max_candidates, CL) + P.max_candidates);
    if (!opt_in_dynamic_smem(reinterpret_cast<const void*>(kernel), SELECT_SMEM_MAX)) return WUSHKV_ECUDA;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CL; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CL, P.c.n_kv, P.batch);
    cfg.blockDim = dim3(SELECT_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, P) == cudaSuccess ? WUSHKV_OK : WUSHKV_ECUDA;
}

int launch_select(SelectParams P, int max_seq_len, cudaStream_t stream) {
    const long long most = std::max<long long>(candidate_bound(P.c, max_seq_len), 1);
    if (most > MAX_SELECT_PAGES) return WUSHKV_ECAPACITY;
    P.max_candidates = static_cast<int>(most);
    // CTAs per (sequence, KV head): enough for every SM to have one, but no fewer than 16 pages per warp
    const long long clusters = static_cast<long long>(P.batch) * P.c.n_kv;
    int cl = knobs().select_cluster;
    if (cl != 2 && cl != 4 && cl != 8) cl = 1;
    while (knobs().select_cluster == 0 && cl < 8 && clusters * cl < sm_count() && most > static_cast<long long>(cl) * 16 * SELECT_WARPS) cl *= 2;
    // the scores and the keys have to fit in shared memory
    const auto smem = [&](int k) { return sizeof(SelectShared) + sizeof(float) * (static_cast<size_t>(P.c.G) * pages_per_cta(P.max_candidates, k) + most); };
    while (cl < 8 && smem(cl) > SELECT_SMEM_MAX) cl *= 2;
    const bool mode0 = P.c.G <= 4;
    switch (cl) {
        case 1: return mode0 ? launch_select_cl<0, 1>(P, stream) : launch_select_cl<1, 1>(P, stream);
        case 2: return mode0 ? launch_select_cl<0, 2>(P, stream) : launch_select_cl<1, 2>(P, stream);
        case 4: return mode0 ? launch_select_cl<0, 4>(P, stream) : launch_select_cl<1, 4>(P, stream);
        default: return mode0 ? launch_select_cl<0, 8>(P, stream) : launch_select_cl<1, 8>(P, stream);
    }
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
    SelectParams P;
    const int rc = make_view(cache, P.c);
    if (rc != WUSHKV_OK) return rc;
    if (batch <= 0 || batch > 65535 || P.c.n_kv > 65535 || max_seq_len <= 0 || n_select <= 0) return WUSHKV_EINVAL;
    if (!slot || !seq_len || !Q || !bounds || !exponents || !selected || !aligned(Q, 16) || !aligned(bounds, 16)) return WUSHKV_EINVAL;
    P.pro = Prologue{nullptr, 0, 0, nullptr, 0.f};
    if (prologue && !make_prologue(prologue, prologue->q_norm_weight, P.pro)) return WUSHKV_EINVAL;
    P.batch = batch; P.slot = slot; P.seq_len = seq_len; P.Q = Q;
    P.bounds = reinterpret_cast<const signed char*>(bounds); P.exponents = reinterpret_cast<const signed char*>(exponents);
    P.n_select = n_select; P.selected = selected;
    P.qfrag = P.qwfrag = nullptr; P.qscal = nullptr; P.plan = nullptr;
    return launch_select(P, max_seq_len, static_cast<cudaStream_t>(stream));
}
