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
    int wait_limit;                          // poll limit of the copies' barriers
    int drop_unit;                           // testing aid: the key copy of this page of the first (sequence, head)'s list is never issued (-1: none)
    int stream_pages;                        // 1: the packed pages of a step cannot stay in L2 anyway: copy them with an evict-first hint
};

__device__ __forceinline__ void mma_s8(int (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int SPARSE_THREADS = 256, SPARSE_WARPS = SPARSE_THREADS / 32;
constexpr int SELECT_BINS = 4 * SPARSE_THREADS;

// Shared memory of a CTA: this, then a region that first holds the scores of its pages [heads][per] and (CTA 0) the keys of all
// pages, later the warps' staging rings.
template <int MODE>
struct SparseShared {
    static constexpr int GP = MODE == 0 ? 4 : 8, SETS = MODE == 0 ? 1 : 2;
    static constexpr int QF = MODE == 0 ? 64 : 128, QW = MODE == 0 ? 128 : 256;     // uint4 of the attention's integer / bf16 fragments
    union {
        double q[GP][D];                  // the queries, in 64 bits
        uint4 attn[QF + QW];              // then the attention's query fragments
        float merged[GP][PART_STRIDE];    // at last the CTA's partial result of every head
    };
    union {
        double qc[GP][D];                 // q' of all CTAs' rows
        uint4 bins[SPARSE_THREADS];       // then, CTA 0: pages per bin of the range of keys
    };
    uint4 frag[SETS * 4 * 32];            // B fragments of the selection: [digit set][64 bytes of bounds][lane]
    unsigned long long bars[SPARSE_WARPS][4];
    float2 scal[8];                       // score multiplier (log2 domain) and x_min multiplier of the heads
    float unit[8];                        // score of one unit of 2^e dot
    float warp_best[SPARSE_WARPS][8];
    float best[8][8];                     // per CTA of the cluster: largest score of its pages, per head
    int scan[SPARSE_WARPS];
    unsigned most;                        // CTA 0: largest finite key
    int bin, before, inside;              // CTA 0: the bin of the n_select-th key, keys in the bins ahead, keys in it
    unsigned kth;
    int n_list;
    unsigned list[SPARSE_THREADS];        // keys of that bin
};

// Staging ring of a warp: slots for the key side (codes, steps and offsets) and for the value side, filled and freed on their own,
// so that the next page's keys are on their way while this one's values are used.  Two CTAs fit on an SM.
template <int BITS>
struct Ring {
    static constexpr int NK = BITS == 4 ? 1 : 2, NV = BITS == 2 ? 2 : 1;
    static constexpr int META = PAGE_TOKENS * 8, WINDOW = WIN_TOKENS * WIN_ROW;      // bytes of steps and offsets; of a window unit's rows
    static constexpr int K_SLOT = side_bytes(BITS) + META, V_SLOT = side_bytes(BITS) > WINDOW ? side_bytes(BITS) : WINDOW;
    static constexpr int BYTES = NK * K_SLOT + NV * V_SLOT;
    static_assert(K_SLOT >= WINDOW && K_SLOT % 16 == 0 && V_SLOT % 16 == 0, "window rows fit, copies are aligned");
    static_assert(BYTES >= 8 * PART_STRIDE * 4, "the partials of 8 query heads fit");
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

// Ordinary accesses to shared memory so far come before bulk copies into it later (after a barrier).
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async;" ::: "memory"); }

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

// One tile of 16 pages as a lane reads it: 64 bytes of the bounds of rows g and g + 8 and the rows' exponents.
struct BoundsTile {
    uint4 a[2][4];
    int ex[2];
    bool good[2];
    __device__ __forceinline__ void load(const SparseParams& P, const int* table, int h, int p0, int p_hi, int g, int t) {
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

// The n_select smallest of the keys, ties to the lower page, in ascending order of the pages, by one CTA.  Keys are counted in bins
// of equal width; the bin of the n_select-th smallest is found by a prefix sum and its few keys are compared with each other.
template <class Shared>
__device__ __forceinline__ void list_pages(Shared& sh, const unsigned* keys, int pages, int first, int n_select, int* out) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr unsigned INF_BITS = 0x7f800000u;
    // bins of equal width from 0 to the largest key; the product is monotonic in the key, so bins are in the keys' order
    const float width = __uint_as_float(sh.most), per_bin = width > 0.f ? (SELECT_BINS - 1) / width : 0.f;
    const auto bin_of = [&](unsigned u) { return u < INF_BITS ? min(static_cast<int>(__uint_as_float(u) * per_bin), SELECT_BINS - 1) : SELECT_BINS - 1; };
    unsigned* bins = reinterpret_cast<unsigned*>(sh.bins);
    for (int p = tid; p < pages; p += SPARSE_THREADS) atomicAdd(bins + bin_of(keys[p]), 1u);
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
        for (int w = 0; w < SPARSE_WARPS; ++w) before += w < warp ? sh.scan[w] : 0;
        return before + incl - x;
    };
    __syncthreads();
    const uint4 mine = sh.bins[tid];
    const int counts[4] = {static_cast<int>(mine.x), static_cast<int>(mine.y), static_cast<int>(mine.z), static_cast<int>(mine.w)};
    int before = prefix(counts[0] + counts[1] + counts[2] + counts[3]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (before < n_select && n_select <= before + counts[e]) { sh.bin = 4 * tid + e; sh.before = before; sh.inside = counts[e]; }
        before += counts[e];
    }
    __syncthreads();
    const int bin = sh.bin, inside = sh.inside, wanted = n_select - sh.before - 1;      // rank of the n_select-th key in its bin
    unsigned kth = 0u;
    if (inside <= SPARSE_THREADS) {
        for (int p = tid; p < pages; p += SPARSE_THREADS) {
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
            for (int p = tid; p < pages; p += SPARSE_THREADS) n += keys[p] < cand;
            n = __reduce_add_sync(FULL, n);
            __syncthreads();
            if (lane == 0) sh.scan[warp] = n;
            __syncthreads();
            int total = 0;
#pragma unroll
            for (int w = 0; w < SPARSE_WARPS; ++w) total += sh.scan[w];
            if (total < n_select) kth = cand;
        }
    }
    __syncthreads();                                        // the readers of sh.scan
    // all below it, and of those equal to it the first ones; every thread lists a run of consecutive pages
    const int run = (pages + SPARSE_THREADS - 1) / SPARSE_THREADS, r_lo = min(tid * run, pages), r_hi = min(r_lo + run, pages);
    int below = 0, equal = 0;
    for (int p = r_lo; p < r_hi; ++p) { below += keys[p] < kth; equal += keys[p] == kth; }
    static_assert(MAX_SELECT_PAGES < (1 << 15), "two counts in one prefix sum");
    const int packed = prefix((below << 16) + equal);
    int all_below = 0;
#pragma unroll
    for (int w = 0; w < SPARSE_WARPS; ++w) all_below += sh.scan[w] >> 16;
    int below_before = packed >> 16, equal_before = packed & 0xffff;
    const int room = n_select - all_below;                  // places for keys equal to the n_select-th
    for (int p = r_lo; p < r_hi; ++p) {
        const unsigned k = keys[p];
        if (k < kth) { out[below_before + min(equal_before, room)] = first + p; ++below_before; }
        else if (k == kth) { if (equal_before < room) out[below_before + equal_before] = first + p; ++equal_before; }
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
    cg::cluster_group cluster = cg::this_cluster();
    const CacheView& c = P.c;
    const int rank = CL > 1 ? static_cast<int>(cluster.block_rank()) : 0, h = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, G = c.G;
    pdl_wait();
    pdl_launch_dependents();
    // nobody writes into another CTA's shared memory before that CTA has come here and zeroed what the others add to
    if (tid == 0) { sh.most = 0u; sh.n_list = 0; }
    if (CL > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    const unsigned bar0 = smem_u32(&sh.bars[warp][0]);             // key slots, then (2 further) value slots
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) mbar_init(bar0 + 8 * k, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
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
        for (int i = tid; i < P.n_select; i += SPARSE_THREADS) list[i] = i < pages ? first + i : -1;
    if (!attend && !score) {
        if (CL > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
        return;
    }
    const int per_max = pages_per_cta(P.max_candidates, CL);
    float* scores = reinterpret_cast<float*>(region);                                        // [G][per_max]
    unsigned* keys = reinterpret_cast<unsigned*>(scores + static_cast<size_t>(G) * per_max);
    const int per = pages_per_cta(pages, CL), p_lo = min(rank * per, pages), p_hi = min(p_lo + per, pages);
    const int* row = c.page_table + static_cast<long long>(slot) * c.max_pages;              // read only if there are pages
    const int* table = row + first;

    // ---- q', two rows per thread (a query element read from shared memory serves both)
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
    BoundsTile tile;
    if (score) tile.load(P, table, h, p_lo + 16 * warp, p_hi, g, t);
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
    for (int i = tid; i < SETS * 4 * 32; i += SPARSE_THREADS) sh.frag[i] = make_uint4(0u, 0u, 0u, 0u);      // columns without a head
    if (tid < 8) sh.scal[tid] = make_float2(1.f, 0.f);
    __syncthreads();
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
    if (CL > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
#pragma unroll
    for (int peer = 0; peer < CL; ++peer) {
        if (peer % Sum::REPLICAS != Sum::replica(seg)) continue;
        double* q_of = CL > 1 ? cluster.map_shared_rank(&sh.qc[0][0], peer) : &sh.qc[0][0];
#pragma unroll
        for (int i = 0; i < Sum::LEFT; ++i) {
            const int k = Sum::first(seg) + i;
            q_of[(k % GP) * D + t_row + (k / GP) * PAIRS] = acc[i];
        }
    }
    if (CL > 1) cluster.sync(); else __syncthreads();   // sh.q has been read, too
    if (attend) {                                        // columns without a head
        for (int i = tid; i < Shared::QF + Shared::QW; i += SPARSE_THREADS) sh.attn[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
    }

    // ---- the query as two signed bytes per channel: q' ~ (max|q'| / 32512) (256 hi + lo), in B fragments
    if (warp < G) {
        double x[4], most = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = sh.qc[warp][4 * lane + e]; most = fmax(most, fabs(x[e])); }
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) most = fmax(most, __shfl_xor_sync(FULL, most, o));
        const bool usable = most > 0.0 && most < 3e38;          // otherwise all scores are 0: the lowest pages
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
        sh.bins[tid] = make_uint4(0u, 0u, 0u, 0u);
        // ---- scores of this CTA's pages
        uint4 bq[SETS][4];
#pragma unroll
        for (int k = 0; k < SETS * 4; ++k) bq[k / 4][k % 4] = sh.frag[k * 32 + lane];
        float unit[NH], best[NH];                               // heads per lane: t, or 2 t and 2 t + 1
#pragma unroll
        for (int k = 0; k < NH; ++k) { const int head = MODE == 0 ? t : 2 * t + k; unit[k] = head < G ? sh.unit[head] : 0.f; best[k] = -INFINITY; }
        for (int p0 = p_lo + 16 * warp; p0 < p_hi; p0 += 16 * SPARSE_WARPS) {
            const BoundsTile now = tile;
            if (p0 + 16 * SPARSE_WARPS < p_hi) tile.load(P, table, h, p0 + 16 * SPARSE_WARPS, p_hi, g, t);
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
                for (int w = 0; w < SPARSE_WARPS; ++w) m = fmaxf(m, sh.warp_best[w][head]);
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
        unsigned most = 0u;
        for (int p = p_lo + tid; p < p_hi; p += SPARSE_THREADS) {
            float key = -INFINITY;
#pragma unroll
            for (int j = 0; j < GP; ++j) if (j < G) key = fmaxf(key, __fsub_rn(scores[j * per_max + p - p_lo], top[j]));
            const unsigned u = __float_as_uint(key) & 0x7fffffffu;
            keys0[p] = u;
            if (u < 0x7f800000u) most = max(most, u);
        }
        most = __reduce_max_sync(FULL, most);
        if (lane == 0 && most > 0u) atomicMax(CL > 1 ? cluster.map_shared_rank(&sh.most, 0) : &sh.most, most);
        fence_proxy_async();                                    // the scores' and keys' places are filled by bulk copies later
        if (CL > 1) cluster.sync(); else __syncthreads();
        if (rank == 0) list_pages(sh, keys, pages, first, P.n_select, list);
        if (!attend) return;
        if (rank == 0) { fence_proxy_async(); __syncthreads(); }      // the keys' place becomes the staging ring
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
    unsigned char* ring = region + warp * R::BYTES;
    const unsigned k_slot0 = smem_u32(ring), v_slot0 = k_slot0 + R::NK * R::K_SLOT;
    const unsigned long long policy = l2_evict_first_policy();
    const int wait_limit = P.wait_limit;
    int k_next = 0, v_next = 0;                                 // copies issued so far
    int k_done = 0, v_done = 0;                                 // and used
    bool timed_out = false;
    // The key side (V == false) or value side of the next unit is announced and copied; bytes == 0: the unit is skipped.
    const auto wait = [&](bool value) {
        const int done = value ? v_done : k_done, n = value ? R::NV : R::NK;
        const unsigned bar = bar0 + 8 * ((value ? 2 : 0) + done % n);
        // a phase that one lane saw complete is complete for all: keep the decision warp-uniform
        if (!__any_sync(FULL, mbar_wait_bounded(bar, (done / n) & 1, wait_limit))) {
            timed_out = true;
            if (lane == 0) atomicOr(c.dev_status, WUSHKV_DEV_COPY_TIMEOUT);
            // other copies of this warp may still be in flight: wait for each (bounded) before the ring is used for anything else
            for (int k = k_done; k < k_next; ++k) mbar_wait_bounded(bar0 + 8 * (k % R::NK), (k / R::NK) & 1, min(wait_limit, 1 << 9));
            for (int k = v_done; k < v_next; ++k) mbar_wait_bounded(bar0 + 8 * (2 + k % R::NV), (k / R::NV) & 1, min(wait_limit, 1 << 9));
        }
        if (value) ++v_done; else ++k_done;
        return !timed_out;
    };

    // ---- window tokens: by all warps, or by those of the CTAs that are not listing pages
    const int n_window = (si.n_win + WIN_TOKENS - 1) / WIN_TOKENS;
    {
        const bool spared = score && CL > 1;
        const int first_warp = spared ? (rank - 1) * SPARSE_WARPS + warp : rank * SPARSE_WARPS + warp, stride = (spared ? CL - 1 : CL) * SPARSE_WARPS;
        const int n = (spared && rank == 0) || first_warp >= n_window ? 0 : (n_window - first_warp + stride - 1) / stride;
        const auto copy_rows = [&](bool value, int k) {
            const int w0 = (first_warp + k * stride) * WIN_TOKENS, n_valid = min(WIN_TOKENS, si.n_win - w0);
            const int done = value ? v_next : k_next, nn = value ? R::NV : R::NK;
            const unsigned bar = bar0 + 8 * ((value ? 2 : 0) + done % nn), dst = value ? v_slot0 + (done % nn) * R::V_SLOT : k_slot0 + (done % nn) * R::K_SLOT;
            if (lane == 0) mbar_expect_tx(bar, n_valid * D * 2);
            __syncwarp();
            if (lane < n_valid) {
                const int w = w0 + lane;
                const long long plane = (static_cast<long long>(slot) * c.n_kv + h) * 2 + (value ? 1 : 0);
                const unsigned short* src = w < si.n_sink ? c.sink_kv + (plane * c.s_sink + w) * D
                                                          : c.ring_kv + (plane * c.ring_cap + (si.recent_lo + (w - si.n_sink)) % c.ring_cap) * D;
                bulk_copy_g2s(dst + lane * WIN_ROW, src, D * 2, bar);
            }
            if (value) ++v_next; else ++k_next;
        };
        const int k0 = k_next, v0 = v_next;
        for (int k = 0; k < min(n, R::NK); ++k) copy_rows(false, k);
        for (int k = 0; k < min(n, R::NV); ++k) copy_rows(true, k);
        for (int k = 0; k < n && !timed_out; ++k) {
            const unsigned ks = k_slot0 + (k_done % R::NK) * R::K_SLOT, vs = v_slot0 + (v_done % R::NV) * R::V_SLOT;
            if (!wait(false) || !wait(true)) break;
            const uint4* wq = sh.attn + Shared::QF;
            window_unit<BITS, MODE>(st, ks, vs, min(WIN_TOKENS, si.n_win - (first_warp + k * stride) * WIN_TOKENS), [wq](int i) { return wq[i]; }, lane);
            __syncwarp();
            if (k_next - k0 < n) copy_rows(false, k_next - k0);
            if (v_next - v0 < n) copy_rows(true, v_next - v0);
        }
    }
    if (score) { if (CL > 1) cluster.sync(); else __syncthreads(); }      // the list is complete

    // ---- the listed pages, 32 of this warp's at a time: lane k looks up the k-th
    const int wid = rank * SPARSE_WARPS + warp;
    constexpr int STRIDE = CL * SPARSE_WARPS;
    for (int base = wid; base < n_listed && !timed_out; base += 32 * STRIDE) {
        const int n = min(32, (n_listed - base + STRIDE - 1) / STRIDE);
        int my_entry = -1, my_page = -1;
        if (lane < n) {
            const int u = base + lane * STRIDE;
            my_entry = given || score ? __ldcg(list + u) : first + u;
            if (my_entry != -1) {
                const bool inside = my_entry >= first && my_entry < first + pages;
                const int page = inside ? __ldg(row + my_entry) : -1;
                if (page >= 0 && page < c.n_pages) my_page = page;
                else atomicOr(c.dev_status, WUSHKV_DEV_BAD_PAGE_ID);
            }
        }
        unsigned there = __ballot_sync(FULL, my_page >= 0), k_todo = there, v_todo = there;      // units of this warp, and those not yet requested
        const auto copy_page = [&](bool value, unsigned& todo) {
            const int k = __ffs(todo) - 1;
            todo &= todo - 1;
            const int page = __shfl_sync(FULL, my_page, k);
            const int done = value ? v_next : k_next, nn = value ? R::NV : R::NK;
            if (lane == 0) {
                const unsigned bar = bar0 + 8 * ((value ? 2 : 0) + done % nn), dst = value ? v_slot0 + (done % nn) * R::V_SLOT : k_slot0 + (done % nn) * R::K_SLOT;
                const unsigned char* rec = c.pages + (static_cast<long long>(page) * c.n_kv + h) * record_bytes(BITS);
                const bool drop = P.drop_unit >= 0 && !value && b == 0 && h == 0 && P.drop_unit == base + k * STRIDE;      // testing aid
                mbar_expect_tx(bar, value ? side_bytes(BITS) : R::K_SLOT);
                if (value) {
                    if (P.stream_pages) bulk_copy_g2s_stream(dst, rec + v_codes_offset(BITS), side_bytes(BITS), bar, policy);
                    else bulk_copy_g2s(dst, rec + v_codes_offset(BITS), side_bytes(BITS), bar);
                } else if (!drop) {
                    if (P.stream_pages) {
                        bulk_copy_g2s_stream(dst, rec, side_bytes(BITS), bar, policy);
                        bulk_copy_g2s_stream(dst + side_bytes(BITS), rec + meta_offset(BITS), R::META, bar, policy);
                    } else {
                        bulk_copy_g2s(dst, rec, side_bytes(BITS), bar);
                        bulk_copy_g2s(dst + side_bytes(BITS), rec + meta_offset(BITS), R::META, bar);
                    }
                }
            }
            if (value) ++v_next; else ++k_next;
        };
#pragma unroll
        for (int k = 0; k < R::NK; ++k) if (k_todo) copy_page(false, k_todo);
#pragma unroll
        for (int k = 0; k < R::NV; ++k) if (v_todo) copy_page(true, v_todo);
        while (there && !timed_out) {
            const int k = __ffs(there) - 1;
            there &= there - 1;
            const int pos0 = __shfl_sync(FULL, my_entry, k) * PAGE_TOKENS;
            const unsigned ks = k_slot0 + (k_done % R::NK) * R::K_SLOT, vs = v_slot0 + (v_done % R::NV) * R::V_SLOT;
            if (!wait(false)) break;
            float sc[4][2 * NH];          // [block][row g: heads..., row g+8: heads...]
            unsigned vmeta[4][2];         // fp16x2 (Delta_v, x_min_v) of rows g, g+8
            page_scores<BITS, MODE>(ks, ks + side_bytes(BITS), qf, qfl, gadd, sc, vmeta, lane);
            __syncwarp();
            if (k_todo) copy_page(false, k_todo);               // the slot just read
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
            float mx[NH];
#pragma unroll
            for (int j = 0; j < NH; ++j) {
                const float v = fmaxf(fmaxf(fmaxf(sc[0][j], sc[0][NH + j]), fmaxf(sc[1][j], sc[1][NH + j])),
                                      fmaxf(fmaxf(sc[2][j], sc[2][NH + j]), fmaxf(sc[3][j], sc[3][NH + j])));
                mx[j] = v * fmul[j];          // scores are kept divided by the head's multiplier (> 0)
            }
            st.raise_max(mx);
            if (!wait(true)) break;
            page_values<BITS, MODE>(st, vs, sc, vmeta, fmul, lane);
            __syncwarp();
            if (v_todo) copy_page(true, v_todo);
        }
    }

    // ---- merge: the CTA's eight states, then the cluster's
    __syncwarp();
    store_state<BITS, MODE, false>(st, reinterpret_cast<float*>(ring), lane, G);
    __syncthreads();                                             // sh.attn has been read, too
    if (warp < G) {
        MergedState ms;
        ms.reset();
        ms.add<false>(SPARSE_WARPS, lane, [&](int k) { return reinterpret_cast<const float*>(region + k * R::BYTES) + warp * PART_STRIDE; });
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

constexpr int SPARSE_SMEM_MAX = 200 * 1024;
static_assert(sizeof(SparseShared<1>) + 4 * (8 * MAX_SELECT_PAGES / 8 + MAX_SELECT_PAGES) <= SPARSE_SMEM_MAX, "clusters of 8 hold every allowed number of pages");

template <int BITS, int MODE>
static size_t sparse_smem(const SparseParams& P, int cl) {
    const size_t scored = P.bounds ? sizeof(float) * (static_cast<size_t>(P.c.G) * pages_per_cta(P.max_candidates, cl) + P.max_candidates) : 0;
    return sizeof(SparseShared<MODE>) + std::max<size_t>(scored, P.O ? SPARSE_WARPS * Ring<BITS>::BYTES : 0);
}

template <int BITS, int MODE, int CL>
static int launch_sparse_cl(const SparseParams& P, cudaStream_t st) {
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
    cfg.dynamicSmemBytes = sparse_smem<BITS, MODE>(P, CL);
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
    while (cl < 8 && sparse_smem<BITS, MODE>(P, cl) > SPARSE_SMEM_MAX) cl *= 2;
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
    P.max_candidates = static_cast<int>(candidates);
    P.wait_limit = static_cast<int>(std::min<long long>(std::max<long long>(knobs().wait_limit, 0), 1 << 30));
    if (P.wait_limit == 0) P.wait_limit = 1 << 19;                // polls that may sleep ~2 us each: about a second
    P.drop_unit = static_cast<int>(std::min<long long>(std::max<long long>(knobs().drop_copy_unit, -1), 1 << 30));
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
