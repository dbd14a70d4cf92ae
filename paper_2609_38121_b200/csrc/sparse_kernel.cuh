// Sparse decode attention: the selection of pages by their bounds and the attention over the selected pages, one kernel.
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
#pragma once
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "decode_core.cuh"
#include "host_common.h"
#include "prologue.cuh"
#include "sparse.h"

namespace wushkv {

namespace cg = cooperative_groups;

__device__ __forceinline__ void mma_s8(int (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}


// Shared memory of a CTA: this, then a region for the selection (the page ids and the scores of the CTA's pages [per], [heads][per],
// CTA 0: key and page id of all pages) and the warps' staging rings.  Where the sizes allow it the rings are apart from the selection's
// region, so that window tokens can be staged from the start; else the rings begin where the selection's region began.
constexpr int LISTED = 512;               // listed pages that are handed over in shared memory, with their ids
template <int MODE, int NT>                  // NT: threads of a CTA
struct SparseShared {
    static constexpr int GP = MODE == 0 ? 4 : 8, SETS = MODE == 0 ? 1 : 2;
    static constexpr int WARPS = NT / 32, BINS = 4 * NT;
    static constexpr int QF = MODE == 0 ? 64 : 128, QW = MODE == 0 ? 128 : 256;     // uint4 of the attention's integer / bf16 fragments
    union {
        double q[GP][D];                  // the queries, in 64 bits
        uint4 frag[SETS * 4 * 32];        // then the selection's query fragments: [digit set][64 bytes of bounds][lane]
        uint4 bins[NT];                   // then this CTA's pages per bin of the range of keys
        float merged[GP][PART_STRIDE];    // at last the CTA's partial result of every head
    };
    union {
        double qc[GP][D];                 // q' of this CTA's rows
        uint2 listed[LISTED];             // then, CTA 0: the listed pages, index and id
    };
    uint4 attn[QF + QW];                  // the attention's query fragments
    float2 scal[8];                       // score multiplier (log2 domain) and x_min multiplier of the heads
    float unit[8];                        // score of one unit of 2^e dot
    float2 warp_best[WARPS][8];
    float2 best[8][8];                    // per CTA of the cluster: largest and smallest finite score of its pages, per head
    int scan[WARPS], below[WARPS], equal[WARPS];
    int bin, inside, wanted;              // CTA 0: the bin of the n_select-th key, keys in it, its rank among them
    unsigned kth;
    int n_list;
    unsigned list[NT];        // keys of that bin
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

// Loads that stay where they are written: behind pdl_wait() (what they read may come from the kernel ahead, so they do not take the
// read-only path either) and ahead of the work that their latency is to hide behind.
__device__ __forceinline__ uint4 ld_early(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ int ld_early_s8(const signed char* p) {
    int v;
    asm volatile("ld.global.s8 %0, [%1];" : "=r"(v) : "l"(p));
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
__device__ __forceinline__ int bin_of(unsigned key, float per_bin, int n_bins) { return min(static_cast<int>(__uint_as_float(key) * per_bin), n_bins - 1); }

// The n_select smallest of the keys (.x; .y is the page's id), ties to the lower page, in ascending order of the pages, by one CTA.
// counted: this thread's four of the bins of equal width in which the cluster has counted the keys; the bin of the n_select-th smallest
// is found by a prefix sum and its few keys are compared with each other.
// The code is kept short: a CTA runs through it once, so that every instruction is fetched for one use (with the keys in registers
// and its loops unrolled it took 30 KB and was no faster).
template <int NT, class Shared>
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
    for (int w = 0; w < Shared::WARPS; ++w) before += w < warp ? sh.scan[w] : 0;
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
    if (inside <= NT) {
#pragma unroll 2
        for (int p = tid; p < pages; p += NT) {
            const unsigned u = keys[p].x;
            if (bin_of(u, per_bin, Shared::BINS) == bin) sh.list[atomicAdd(&sh.n_list, 1)] = u;
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
            for (int p = tid; p < pages; p += NT) n += keys[p].x < cand;
            __syncthreads();                                // the readers of the round before
            n = __reduce_add_sync(FULL, n);
            if (lane == 0) sh.scan[warp] = n;
            __syncthreads();
            int total = 0;
#pragma unroll
            for (int w = 0; w < Shared::WARPS; ++w) total += sh.scan[w];
            if (total < n_select) kth = cand;
        }
    }
    // all below it, and of those equal to it the first ones; every warp lists a run of consecutive pages
    const int run = (pages + NT - 1) / NT * 32, r_lo = min(warp * run, pages), r_hi = min(r_lo + run, pages);
    int below = 0, equal = 0;
#pragma unroll 2
    for (int p = r_lo + lane; p < r_hi; p += 32) { const unsigned u = keys[p].x; below += u < kth; equal += u == kth; }
    below = __reduce_add_sync(FULL, below);
    equal = __reduce_add_sync(FULL, equal);
    if (lane == 0) { sh.below[warp] = below; sh.equal[warp] = equal; }
    __syncthreads();
    int all_below = 0, below_before = 0, equal_before = 0;
#pragma unroll
    for (int w = 0; w < Shared::WARPS; ++w) {
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

// One cluster of CL CTAs per (sequence, KV head); a CTA of NT threads, 512 threads on an SM.
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
template <int BITS, int MODE, int CL, int NT>
__global__ void __launch_bounds__(NT, 512 / NT) sparse_decode_kernel(SparseParams P) {
    using Shared = SparseShared<MODE, NT>;
    constexpr int WARPS = Shared::WARPS, HPW = (Shared::GP + WARPS - 1) / WARPS;      // head slots per warp where the warps share them out
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
    // ---- q': this thread's rows of T_K^{-T} and its share of the queries are requested ahead of everything else
    // Rows per thread: a query element read from shared memory serves all of them.  Four with CTAs of four warps, whose SMs are busy with
    // other pairs meanwhile (64 ragged sequences x 8 heads, 4 bits, graphs of one state: 39.6 -> 37.4 us); two where the chain of one CTA
    // counts, to which four make no difference beyond 1 % either way (1 x 2k tokens 9.3 and 9.3 us, 16 x 32k 24.3 and 24.0, its selection
    // alone 9.4 and 9.5).
    constexpr int ROWS = D / CL, RPT = NT == 128 ? 4 : 2;
    constexpr int SPACING = ROWS / RPT, TPR = NT / SPACING, QUADS = D / 4 / TPR;              // rows apart, threads per row, float4 per thread and row
    constexpr int PART = QUADS * RPT > 8 ? 8 / RPT : QUADS;                                  // of them in flight together
    static_assert(TPR <= 32 && QUADS >= 1 && QUADS % PART == 0, "a row is summed within a warp");
    const int t_row = rank * ROWS + tid / TPR, seg = tid % TPR;
    const uint4* T = reinterpret_cast<const uint4*>(c.T_K_invT + (static_cast<long long>(h) * D + t_row) * D);
    uint4 tr[RPT][PART];
    const auto load_T = [&](int k0) {
#pragma unroll
        for (int k = 0; k < PART; ++k)
#pragma unroll
            for (int r = 0; r < RPT; ++r) tr[r][k] = ld_early(T + r * SPACING * (D / 4) + seg + TPR * (k0 + k));
    };
    load_T(0);
    uint2 q_bits[HPW];                                  // slots without a head are zero
#pragma unroll
    for (int k = 0; k < HPW; ++k) {
        const int head = warp + k * WARPS;
        q_bits[k] = head < G ? ld_in(reinterpret_cast<const uint2*>(P.Q + (static_cast<long long>(b) * c.n_q + h * G + head) * D + 4 * lane)) : make_uint2(0u, 0u);
    }

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
        for (int i = tid; i < P.n_select; i += NT) list[i] = i < pages ? first + i : -1;
    if (!attend && !score) return;
    const int per_max = pages_per_cta(P.max_candidates, CL);
    int* ids = reinterpret_cast<int*>(region);                                               // [per_max]
    float* scores = reinterpret_cast<float*>(ids + per_max);                                 // [G][per_max]
    uint2* keys = reinterpret_cast<uint2*>(scores + static_cast<size_t>(G) * per_max);       // CTA 0: [max_candidates]
    const int per = pages_per_cta(pages, CL), p_lo = min(rank * per, pages), n_here = min(p_lo + per, pages) - p_lo;      // this CTA's candidates
    const int* row = c.page_table + static_cast<long long>(slot) * c.max_pages;              // read only if there are pages
    if (score) {
        for (int p = tid; p < n_here; p += NT) {
            const int page = ld_in(row + first + p_lo + p);
            const bool good = page >= 0 && page < c.n_pages;
            if (good) prefetch_bounds(P, page, h);
            else atomicOr(c.dev_status, WUSHKV_DEV_BAD_PAGE_ID);
            ids[p] = good ? page : -1;
        }
    }

    // ---- window tokens: by all warps, or by those of the CTAs that will not be listing pages.  Staged early if the rings are apart.
    // A unit is up to 16 consecutive rows of the sink buffer or of the ring; the ring's rows in use are one range or, where it wraps, two
    // (a full ring is one range from row 0 on: the order of the tokens does not matter).
    unsigned char* ring = rings + warp * R::BYTES;
    const unsigned k_slot0 = smem_u32(ring), v_slot0 = k_slot0 + R::NK * R::K_SLOT;
    const bool spared = score && CL > 1;
    const int win_first = (spared ? rank - 1 : rank) * WARPS + warp, win_stride = (spared ? CL - 1 : CL) * WARPS;
    const int n_recent = si.n_win - si.n_sink, at0 = n_recent >= c.ring_cap ? 0 : si.recent_lo % c.ring_cap;
    const int range0 = min(n_recent, c.ring_cap - at0), range1 = n_recent - range0;
    const int units_sink = (si.n_sink + WIDE_TOKENS - 1) / WIDE_TOKENS, units0 = (range0 + WIDE_TOKENS - 1) / WIDE_TOKENS;
    const int n_window = units_sink + units0 + (range1 + WIDE_TOKENS - 1) / WIDE_TOKENS;
    const int my_windows = !attend || (spared && rank == 0) || win_first >= n_window ? 0 : (n_window - win_first + win_stride - 1) / win_stride;
    // rows of the k-th of this warp's units into the ring, two rows (lanes 0 - 15, 16 - 31) per instruction; returns their number
    const auto stage_window = [&](int k) {
        int u = win_first + k * win_stride, rows = 0;
        if (k < my_windows) {
            const long long plane = (static_cast<long long>(slot) * c.n_kv + h) * 2;
            const unsigned short* src;
            int per_plane = c.ring_cap;
            if (u < units_sink) {
                src = c.sink_kv + plane * c.s_sink * D;
                per_plane = c.s_sink;
                rows = si.n_sink;
            } else {
                u -= units_sink;
                const bool wrapped = u >= units0;
                u -= wrapped ? units0 : 0;
                src = c.ring_kv + (plane * c.ring_cap + (wrapped ? 0 : at0)) * D;
                rows = wrapped ? range1 : range0;
            }
            rows = min(rows - u * WIDE_TOKENS, WIDE_TOKENS);
            src += u * WIDE_TOKENS * D + (lane & 15) * 8;
            const long long to_values = static_cast<long long>(per_plane) * D;
            const int half = lane >> 4;
            const unsigned dst = k_slot0 + half * (2 * D), place = ((lane & 15) ^ half) << 4;
#pragma unroll
            for (int j = 0; j < WIDE_TOKENS / 2; ++j) {
                const unsigned short* row_src = src + min(2 * j + half, rows - 1) * D;
                const unsigned row_dst = dst + 2 * j * (2 * D) + (place ^ ((2 * j & 7) << 4));      // row r = 2 j + half, piece i at i ^ (r & 7)
                copy16(row_dst, row_src);
                copy16(row_dst + WIDE_TOKENS * 2 * D, row_src + to_values);
            }
        }
        copies_commit();
        return rows;
    };
    int staged_rows = 0;

#pragma unroll
    for (int k = 0; k < HPW; ++k) {
        const int head = warp + k * WARPS;
        if (head >= GP) break;
        float x[4] = {bf16_bits_to_float(q_bits[k].x & 0xffff), bf16_bits_to_float(q_bits[k].x >> 16), bf16_bits_to_float(q_bits[k].y & 0xffff), bf16_bits_to_float(q_bits[k].y >> 16)};
        if (head < G && P.pro.rope)
            norm_rope_warp(x, lane, P.pro, h * G + head, prologue_position(P.pro, max(S - 1, 0), c.dev_status, lane == 0 && rank == 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) sh.q[head][4 * lane + e] = static_cast<double>(x[e]);
    }
    __syncthreads();
    BoundsTile tile;
    if (score) tile.load(P, ids, h, 16 * warp, n_here, g, t);
    if (P.ring_offset > 0) staged_rows = stage_window(0);
    double acc[RPT * GP];                                 // [row][head]
#pragma unroll
    for (int j = 0; j < RPT * GP; ++j) acc[j] = 0.0;
#pragma unroll
    for (int k0 = 0; k0 < QUADS; k0 += PART) {
        if (k0 > 0) load_T(k0);
#pragma unroll
        for (int k = 0; k < PART; ++k) {
            double tv[RPT][4];
#pragma unroll
            for (int r = 0; r < RPT; ++r) {
                tv[r][0] = __uint_as_float(tr[r][k].x); tv[r][1] = __uint_as_float(tr[r][k].y);
                tv[r][2] = __uint_as_float(tr[r][k].z); tv[r][3] = __uint_as_float(tr[r][k].w);
            }
#pragma unroll
            for (int j = 0; j < GP; ++j) {
                const double2* q = reinterpret_cast<const double2*>(&sh.q[j][4 * (seg + TPR * (k0 + k))]);
                const double2 lo = q[0], hi = q[1];
#pragma unroll
                for (int r = 0; r < RPT; ++r) acc[r * GP + j] = fma(tv[r][0], lo.x, fma(tv[r][1], lo.y, fma(tv[r][2], hi.x, fma(tv[r][3], hi.y, acc[r * GP + j]))));
            }
        }
    }
    using Sum = GroupSum<RPT * GP, TPR>;
    Sum::sum(acc, seg);
    if (Sum::replica(seg) == 0)
#pragma unroll
        for (int i = 0; i < Sum::LEFT; ++i) {
            const int k = Sum::first(seg) + i;
            sh.qc[k % GP][t_row + (k / GP) * SPACING] = acc[i];
        }
    if (CL > 1) cluster.sync(); else __syncthreads();   // sh.q has been read, too

    // ---- the query as two signed bytes per channel: q' ~ (max|q'| / 32512) (256 hi + lo), in B fragments.  A warp per column pair (or
    // column) of a head; the queries of head slots without a head are zero, and so are their columns.
#pragma unroll 1
    for (int head = warp; head < GP; head += WARPS) {
        double x[4], most = 0.0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {                            // from the CTA whose rows they are
            const double2* from = reinterpret_cast<const double2*>(&sh.qc[head][4 * lane + 2 * e]);
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
                const int set = MODE == 0 ? 0 : digit, column = MODE == 0 ? 2 * head + digit : head;
                const int group = 2 * side + lane / 16, tl = (lane % 16) / 4;
                frag[((set * 4 + group) * 32 + 4 * column + tl) * 4 + lane % 4] = word[side][digit];
            }
        if (lane == 0) sh.unit[head] = usable ? static_cast<float>(__dmul_rn(most / QM, static_cast<double>(c.sm_scale))) : 0.f;
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
                    const int set = MODE == 0 ? 0 : digit, column = MODE == 0 ? 2 * head + digit : head;
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
                    const int set = MODE == 0 ? 0 : part, column = MODE == 0 ? 2 * head + part : head;
                    const float a = part == 0 ? y[0] : rest[0], d = part == 0 ? y[1] : rest[1];
                    wfrag[set * 512 + ((s16 >> 1) * 32 + 4 * column + tq) * 4 + (s16 & 1) * 2 + r] = float_to_bf16_bits(a) | (static_cast<unsigned>(float_to_bf16_bits(d)) << 16);
                }
            }
            sum = __reduce_add_sync(FULL, sum);
            constexpr float FS = BITS != 4 ? 4.f : 16.f;        // the integer score carries this factor (page_scores)
            if (lane == 0) sh.scal[head] = make_float2(k2 * lam * (1.f / FS), FS * static_cast<float>(sum));
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
        for (int p0 = 16 * warp; p0 < n_here; p0 += 16 * WARPS) {
            const BoundsTile now = tile;
            if (p0 + 16 * WARPS < n_here) tile.load(P, ids, h, p0 + 16 * WARPS, n_here, g, t);
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
                for (int w = 0; w < WARPS; ++w) { const float2 x = sh.warp_best[w][head]; m.x = fmaxf(m.x, x.x); m.y = fminf(m.y, x.y); }
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
        const float per_bin = width > 0.f && width < INFINITY ? (Shared::BINS - 1) / width : 0.f;
        for (int p = tid; p < n_here; p += NT) {
            float key = -INFINITY;
#pragma unroll
            for (int j = 0; j < GP; ++j) if (j < G) key = fmaxf(key, __fsub_rn(scores[j * per_max + p], top[j]));
            const unsigned u = __float_as_uint(key) & 0x7fffffffu;
            keys0[p_lo + p] = make_uint2(u, static_cast<unsigned>(ids[p]));
            atomicAdd(reinterpret_cast<unsigned*>(sh.bins) + bin_of(u, per_bin, Shared::BINS), 1u);
        }
        if (CL > 1) cluster.sync(); else __syncthreads();
        if (rank == 0) {
            uint4 counted = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int r = 0; r < CL; ++r) {
                const uint4 x = *(CL > 1 ? cluster.map_shared_rank(&sh.bins[tid], r) : &sh.bins[tid]);
                counted.x += x.x; counted.y += x.y; counted.z += x.z; counted.w += x.w;
            }
            list_pages<NT>(sh, counted, per_bin, keys, pages, first, P.n_select, list);
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
        if (k > 0 || P.ring_offset == 0) staged_rows = stage_window(k);
        copies_wait<0>();
        wide_window_unit<BITS, MODE>(st, k_slot0, staged_rows, sh.attn + Shared::QF, lane);
        __syncwarp();
    }
    if (score && CL > 1) cluster.sync();                        // the list is complete

    // ---- the listed pages, 32 of this warp's at a time: lane k looks up the k-th
    const int wid = rank * WARPS + warp;
    constexpr int STRIDE = CL * WARPS;
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
                const int page = inside ? ld_in(row + my_entry) : -1;
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

    // ---- merge: the states of the CTA's warps, then the cluster's
    __syncwarp();
    store_state<BITS, MODE, false>(st, reinterpret_cast<float*>(ring), lane, G);
    __syncthreads();                                             // sh.attn has been read, too
#pragma unroll 1
    for (int head = warp; head < G; head += WARPS) {
        MergedState ms;
        ms.reset();
        ms.add<false>(WARPS, lane, [&](int k) { return reinterpret_cast<const float*>(rings + k * R::BYTES) + head * PART_STRIDE; });
        if (CL > 1) ms.store(sh.merged[head], lane);
        else ms.finish(P.O + (static_cast<long long>(b) * c.n_q + h * G + head) * D, lane);
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

constexpr int SPARSE_SMEM_MAX = 226 * 1024;
__host__ __device__ constexpr size_t scored_bytes(size_t group, size_t per, size_t pages) { return (4 * (1 + group) * per + 8 * pages + 15) / 16 * 16; }

// Shared memory of a CTA and where in it the rings begin.
template <int BITS, int MODE, int NT>
static size_t sparse_smem(const SparseParams& P, int cl, int& ring_offset) {
    constexpr size_t shared = sizeof(SparseShared<MODE, NT>);
    static_assert(shared + scored_bytes(MODE == 0 ? 4 : 8, MAX_SELECT_PAGES / 8, MAX_SELECT_PAGES) <= SPARSE_SMEM_MAX, "clusters of 8 hold every allowed number of pages");
    const size_t scored = P.bounds ? scored_bytes(P.c.G, pages_per_cta(P.max_candidates, cl), P.max_candidates) : 0;
    const size_t ring = P.O ? NT / 32 * Ring<BITS>::BYTES : 0, apart = shared + scored + ring;
    // apart from the scores unless that costs an SM one of the CTAs that its registers hold and that would come
    const bool alone = static_cast<long long>(P.batch) * P.c.n_kv * cl <= sm_count();
    ring_offset = 0;
    if (scored > 0 && ring > 0 && apart <= (alone ? SPARSE_SMEM_MAX : SPARSE_SMEM_MAX / (512 / NT))) { ring_offset = static_cast<int>(scored); return apart; }
    return shared + std::max(scored, ring);
}

template <int BITS, int MODE, int CL, int NT>
static int launch_sparse_cl(SparseParams P, cudaStream_t st) {
    const auto kernel = sparse_decode_kernel<BITS, MODE, CL, NT>;
    if (!opt_in_dynamic_smem(reinterpret_cast<const void*>(kernel), SPARSE_SMEM_MAX)) return WUSHKV_ECUDA;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CL; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CL, P.c.n_kv, P.batch);
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = sparse_smem<BITS, MODE, NT>(P, CL, P.ring_offset);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = CL > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, P) == cudaSuccess ? WUSHKV_OK : WUSHKV_ECUDA;
}

template <int BITS, int MODE>
static int launch_sparse_mode(const SparseParams& P, cudaStream_t st) {
    // CTAs per (sequence, KV head): more than one only while they all find an SM and each warp still has more than a tile of pages to
    // score or more than two pages to attend to.  (Graphs of one state: 16 x 8 heads of 510 pages, 64 selected: one CTA 24.1 us, two 26.7,
    // four 39.3: a cluster's barriers and remote loads cost more than half of the scoring saves.  1 x 8 heads of 2045 pages, 128 selected:
    // 1, 2, 4, 8 CTAs take 51.2, 36.5, 25.8, 20.3 us.)
    const long long pairs = static_cast<long long>(P.batch) * P.c.n_kv;
    const long long work = std::max<long long>(P.bounds ? P.max_candidates / 16 : 0, P.O ? P.n_select / 2 : 0);
    int offset, cl = knobs().select_cluster;
    // More pairs than CTAs of 8 warps are resident: CTAs of 4 warps, so that pairs in different steps overlap (64 ragged sequences x 8
    // heads, 4 bits, graphs of one state: 48.8 -> 39.6 us, 37.4 with the four rows per thread that they take; 16 x 8 heads, for which they are
    // not taken, 24.1 -> 30.6; when they came, 352 to 1024 pairs of 4 query heads ran 2 to 8 % faster, one case 1 % slower, 128 to 288 pairs 8 to
    // 30 % slower).  With more than 4 query heads the fixed part of a pair is too long for 4 warps (512 pairs: 51.0 us with 8, 60.3 with 4).
    if constexpr (MODE == 0) {
        const bool small = cl == 0 ? pairs > 2 * sm_count() : cl == -1;
        if (small && sparse_smem<BITS, MODE, 128>(P, 1, offset) <= SPARSE_SMEM_MAX / 2) return launch_sparse_cl<BITS, MODE, 1, 128>(P, st);
    }
    if (cl != 2 && cl != 4 && cl != 8) cl = 1;
    while (knobs().select_cluster == 0 && cl < 8 && 2 * pairs * cl <= sm_count() && work > 8 * cl) cl *= 2;
    while (cl < 8 && sparse_smem<BITS, MODE, 256>(P, cl, offset) > SPARSE_SMEM_MAX) cl *= 2;      // the scores and keys have to fit
    switch (cl) {
        case 1: return launch_sparse_cl<BITS, MODE, 1, 256>(P, st);
        case 2: return launch_sparse_cl<BITS, MODE, 2, 256>(P, st);
        case 4: return launch_sparse_cl<BITS, MODE, 4, 256>(P, st);
        default: return launch_sparse_cl<BITS, MODE, 8, 256>(P, st);
    }
}

template <int BITS>
static int launch_sparse(const SparseParams& P, cudaStream_t st) { return P.c.G <= 4 ? launch_sparse_mode<BITS, 0>(P, st) : launch_sparse_mode<BITS, 1>(P, st); }

}  // namespace wushkv
