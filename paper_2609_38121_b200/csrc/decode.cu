// Decode attention over the packed cache (Algorithm 2 lines 3 and 5; Eq. 2; Eq. 3; Section 4.4).
//
// Two launches on the caller's stream:
//   1. decode_prep_kernel   q' = T_K^{-T} q per query head (Algorithm 2 line 3), written as mma
//                           B-fragments: for the quantized positions a 16-bit fixed-point copy of q' split
//                           into two signed bytes per channel (the operand of the integer mma), for the
//                           bf16 windows a bf16 value + rounding remainder.  Block (0,0) also writes the
//                           work plan: the prefix sums of work units per sequence.
//   2. decode_main_kernel   ONE wave of CTAs; every WARP owns an equal, contiguous slice of the
//                           flattened list of work units (sequence, KV head, unit), a unit being a
//                           64-token packed page or up to 8 tokens of the bf16 sink / recent windows.
//                           A warp streams its units into shared memory with bulk async copies (mbarrier
//                           ring).  Scores: the packed key codes become unsigned bytes with one AND per four
//                           codes and go through mma.sync.m16n8k32 (u8 x s8, exact 32-bit sums); values:
//                           code words become fp16 A-fragments with one AND per two codes and go through
//                           mma.sync.m16n8k16 with fp32 accumulation.  The affine part of Eq. 6 is factored
//                           out of the contractions:
//                               q'.k_hat = Delta_k (q'.c_k) + x_min_k sum(q'),
//                               o        = sum_s (p_s Delta_v,s) c_v,s + (sum_s p_s x_min_v,s) 1.
//                           Window units use ldmatrix + bf16 mma on the staged rows and fold into the
//                           same accumulators.  Softmax is online (running max / sum) per warp; a warp
//                           writes the outputs of a (sequence, KV head) that lies inside its slice, and one
//                           partial (max, sum, o) of one that it shares; the CTA's partials are merged when
//                           its warps are done, the CTAs' by whichever of them arrives last.
//
// No CTA waits on another.  The only waits are on a warp's own copy barriers, bounded by an
// iteration limit after which the kernel records WUSHKV_DEV_COPY_TIMEOUT and drains.
//
// Data that an earlier kernel of the same step may still be writing while a later one is already
// resident (programmatic dependent launch: sequence lengths, plan, query fragments, partials) is read
// with ld.global.cg or plain loads after griddepcontrol.wait, never through the read-only path.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cstdlib>

#include "host_common.h"
#include "prologue.cuh"
#include "layout.cuh"
#include "decode_core.cuh"

namespace wushkv {

// Warps per CTA of the main kernel.  ONE CTA per SM (16 warps, or 12 where registers or the larger 4-bit records
// limit it) instead of several CTAs of 4: the hardware warp scheduler serves the warps of an older CTA first, so with
// several CTAs per SM equal slices finished up to 15 us apart.
__host__ __device__ constexpr int main_warps(int bits, int mode) { return (bits == 2 && mode == 0) ? 16 : 12; }

struct DecodeParams {
    CacheView c;
    int batch;
    const int* slot;
    const int* seq_len;
    const unsigned short* Q;
    float* O;
    uint4* qfrag;        // [batch*n_kv][256]: s8 B fragments of the 4 k-steps, 2 x 32 uint4 per digit set (MODE 0: one set
                         // whose columns alternate high / low digit; MODE 1: high-digit set, low-digit set)
    uint4* qwfrag;       // [batch*n_kv][2][128]: bf16 B fragments for the windows (MODE 1: value set, remainder set)
    float* qscal;        // [batch][n_q][2]: score multiplier (log2 domain, > 0), x_min multiplier divided by it
    long long* plan;     // [batch+1]: exclusive prefix of work units per sequence (per KV head)
    float* part;         // [n_warps + batch*n_kv][G][PART_STRIDE]
    int n_warps;         // warps of the main kernel
    int wait_limit;      // poll limit of the device-side barrier waits (0: default, about a second)
    long long drop_unit; // testing aid: flattened index of a unit whose copy is never issued (-1: none)
    int q_early;         // 1: Q was final before the kernel ahead of the preparation kernel started
    int stream_pages;    // 1: the packed pages of a step cannot stay in L2 anyway: copy them with an evict-first hint
    Prologue pro;        // pro.rope != nullptr: Q holds projected queries, normalised and rotated by the preparation kernel
};

// Arrival counters of a (sequence, KV head)'s 8 query head slots for the main kernel's merge, zeroed by the preparation kernel:
// in the unused half of the head's integer fragments.
__device__ __forceinline__ int* arrival_counters(const DecodeParams& P, long long bh) { return reinterpret_cast<int*>(P.qfrag + bh * 256 + 128); }


// ------------------------------------------------------------------------------------------------
// 1. query preparation
// ------------------------------------------------------------------------------------------------
constexpr int PREP_THREADS = 512;                   // 16 warps share the 128 rows of T_K^{-T}
constexpr int PREP_ROWS = D / (PREP_THREADS / 32);   // rows per warp
constexpr int MAX_LOCAL_PLAN = 8192;                 // sequences up to which every CTA of the main kernel computes the work plan itself
// One CTA per (KV head, sequence).  What bounds it is latency and, as 16 warps share the SM's schedulers, the number of
// instructions: the selections of a plain butterfly, shuffles for maxima that one reduction does, and byte stores of fragments
// to global memory (now put together in shared memory and stored as 16-byte words) made it 5.4 us for 2 heads x 1 sequence, 8.2 us
// for 8 x 16 and 10.4 us for 8 x 1 with 8 query heads each, now 3.7, 5.8 and 6.2 us.  Two or four sequences per CTA (which read
// the 64 KB of T_K^{-T} once) ran 8 x 64 in 10.3 and 13.2 us against 11.5 us, but the step no faster: the CTAs then wait longer
// for room beside the append's.
template <int BITS, int MODE>
__global__ void __launch_bounds__(PREP_THREADS) decode_prep_kernel(DecodeParams P) {
    constexpr int QF = MODE == 0 ? 64 : 128, QW = MODE == 0 ? 128 : 256;     // uint4 of a (sequence, head)'s integer / bf16 fragments
    __shared__ uint4 buf[QF + QW > 256 ? QF + QW : 256];                     // the queries, later the fragments
    __shared__ float qp_s[8][D];
    __shared__ float red_abs[8][4];
    __shared__ int red_isum[8][4];
    __shared__ long long scan_s[4];
    float (*q_s)[D] = reinterpret_cast<float (*)[D]>(buf);
    const int h = blockIdx.x, b = blockIdx.y, G = P.c.G;
    const int i = threadIdx.x, lane = i & 31, warp = i >> 5;
    // Normally everything this kernel reads may come from the kernel ahead of it.  In the fused step
    // (q_early) that kernel is the single-token append, which started only after all earlier work had
    // finished: Q is final already, so the transform of the queries runs beside the append; the main kernel, which
    // needs the lengths, waits for this kernel, whose first CTA in turn ends after the append.
    const bool first_cta = h == 0 && b == 0;
    if (!P.q_early) pdl_wait();
    pdl_launch_dependents();               // the main kernel may start (and, unless q_early, stage pages) while this one runs

    // q'[g][i] = sum_j T_invT[h][i][j] q[g][j].  Lane L holds columns 4L .. 4L+3; the 32 products of a pass are indexed
    // k = row * GP + head (GP = 4 or 8 head slots), and slot i of lane L holds product i ^ L: rows and heads are read in
    // that order, so that the butterfly over the lanes adds slot to slot without a selection and leaves total L in lane L.
    constexpr int GP = MODE == 0 ? 4 : 8, PASS_ROWS = 32 / GP;      // MODE 0 serves G <= 4, MODE 1 serves G <= 8
    const float4* Tbase = reinterpret_cast<const float4*>(P.c.T_K_invT + (static_cast<long long>(h) * D + warp * PREP_ROWS) * D) + lane;
    float4 trow[PREP_ROWS];
#pragma unroll
    for (int r = 0; r < PREP_ROWS; ++r) trow[r] = ld_in(Tbase + ((r / PASS_ROWS) * PASS_ROWS + ((r % PASS_ROWS) ^ (lane / GP))) * (D / 4));
    for (int k = i; k < GP * (D / 2); k += PREP_THREADS) {               // unused head slots are zero
        const int g = k / (D / 2), c2 = 2 * (k % (D / 2));
        const unsigned w = g < G ? *reinterpret_cast<const unsigned*>(P.Q + (static_cast<long long>(b) * P.c.n_q + h * G + g) * D + c2) : 0u;
        *reinterpret_cast<float2*>(&q_s[g][c2]) = make_float2(bf16_bits_to_float(w & 0xffff), bf16_bits_to_float(w >> 16));
    }
    __syncthreads();
    if (P.pro.rope) {                     // projected queries: Norm and RoPE at the newest position (Algorithm 2 lines 1-2)
        if (warp < G) {
            const int g = warp, S = __ldcg(P.seq_len + b);
            float4* qv = reinterpret_cast<float4*>(&q_s[g][0]) + lane;
            const float4 x4 = *qv;
            float x[4] = {x4.x, x4.y, x4.z, x4.w};
            norm_rope_warp(x, lane, P.pro, h * G + g, prologue_position(P.pro, max(S - 1, 0), P.c.dev_status, lane == 0 && S > P.pro.n_pos));
            *qv = make_float4(x[0], x[1], x[2], x[3]);
        }
        __syncthreads();
    }
    {
        float4 qv[GP];
#pragma unroll
        for (int g = 0; g < GP; ++g) qv[g] = *reinterpret_cast<const float4*>(&q_s[g ^ (lane % GP)][4 * lane]);
#pragma unroll
        for (int r0 = 0; r0 < PREP_ROWS; r0 += PASS_ROWS) {
            float part[32];
#pragma unroll
            for (int k = 0; k < 32; ++k) {
                const float4 t = trow[r0 + k / GP], q = qv[k % GP];
                part[k] = fmaf(t.x, q.x, fmaf(t.y, q.y, fmaf(t.z, q.z, t.w * q.w)));
            }
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1)
#pragma unroll
                for (int k = 0; k < off; ++k) part[k] += __shfl_xor_sync(FULL, part[k + off], off);
            if (lane % GP < G) qp_s[lane % GP][warp * PREP_ROWS + r0 + lane / GP] = part[0];
        }
    }
    if (P.batch > MAX_LOCAL_PLAN && first_cta) {       // work plan for the main kernel: exclusive prefix of units per sequence
        if (P.q_early) pdl_wait();                      // the lengths come from the append
        long long carry = 0;
        for (int base = 0; base < P.batch; base += 128) {
            const int bb = base + i;
            long long u = 0;
            if (i < 128 && bb < P.batch) u = seq_info(P.c, __ldcg(P.seq_len + bb), __ldg(P.slot + bb)).U;
            long long incl = u;
            for (int o = 1; o < 32; o <<= 1) {
                const long long v = __shfl_up_sync(FULL, incl, o);
                if (lane >= o) incl += v;
            }
            if (lane == 31 && warp < 4) scan_s[warp] = incl;
            __syncthreads();
            long long before = 0;
            for (int w = 0; w < warp && w < 4; ++w) before += scan_s[w];
            if (i < 128 && bb < P.batch) P.plan[bb + 1] = carry + before + incl;
            carry += scan_s[0] + scan_s[1] + scan_s[2] + scan_s[3];
            __syncthreads();
        }
        if (i == 0) P.plan[0] = 0;
    }
    __syncthreads();
    if (i >= D) return;                    // the fragment stage has one thread per channel
    const int ch = i;
    const long long bh = static_cast<long long>(b) * P.c.n_kv + h;
    if (ch < 8) arrival_counters(P, bh)[ch] = 0;
    float acc[GP];
#pragma unroll
    for (int g = 0; g < GP; ++g) acc[g] = g < G ? qp_s[g][ch] : 0.f;
    const float k2 = P.c.sm_scale * LOG2E;
    // ---- 16-bit fixed point of q' per head: q'[ch] ~ lam * qi[ch], |qi| <= Q_MAX, qi = 256 hi + lo with both
    // digits signed bytes.  The scores of the quantized positions use exactly this rounded query
    // (code part and x_min part alike), so they are the scores of a slightly perturbed query, the same
    // for every position.
#pragma unroll
    for (int g = 0; g < GP; ++g) {
        if (g < G) {
            const unsigned ab = __reduce_max_sync(FULL, __float_as_uint(acc[g]) & 0x7fffffffu);     // magnitudes compare like their bits
            if (lane == 0) red_abs[g][warp] = __uint_as_float(ab);
        }
    }
    asm volatile("bar.sync 1, 128;" ::: "memory");                       // the four remaining warps
    int qi[GP];
#pragma unroll
    for (int g = 0; g < GP; ++g) {
        qi[g] = 0;
        if (g < G) {
            const float* ra = red_abs[g];
            const float amax = fmaxf(fmaxf(ra[0], ra[1]), fmaxf(ra[2], ra[3]));
            if (amax > 0.f && amax < 3e38f)
                qi[g] = max(-static_cast<int>(Q_MAX), min(static_cast<int>(Q_MAX), __float2int_rn(acc[g] * (Q_MAX / amax))));
            const int sm = __reduce_add_sync(FULL, qi[g]);
            if (lane == 0) red_isum[g][warp] = sm;
        }
    }
    // ---- B fragments of the integer mma (m16n8k32, B = 32 channels x 8 columns of signed bytes).  Channel i sits in
    // k-step s = i >> 5 at k index 16 hh + 4 t + bb, i.e. register hh, lane 4 n + t, byte bb of column n.
    // MODE 0: column n holds head n >> 1, high digit (n even) or low digit (n odd).  MODE 1: column n holds
    // head n; the high digits form the first fragment set, the low digits the second.
    const int s = ch >> 5, hh = (ch >> 4) & 1, bb = 2 * ((ch >> 3) & 1) + (ch & 1), t = (ch >> 1) & 3;
    signed char* frag = reinterpret_cast<signed char*>(buf);
#pragma unroll
    for (int n = 0; n < 8; ++n) {
        const int head = (MODE == 0) ? (n >> 1) : n;
        const int v = qi[head];
        const int hi = (v + 128) >> 8, lo = v - 256 * hi;          // hi in [-127, 127], lo in [-128, 127]
        const int off = (((s >> 1) * 32 + 4 * n + t) * 16) + ((s & 1) * 2 + hh) * 4 + bb;
        if (MODE == 0) {
            frag[off] = static_cast<signed char>((n & 1) ? lo : hi);
        } else {
            frag[off] = static_cast<signed char>(hi);
            frag[1024 + off] = static_cast<signed char>(lo);
        }
    }
    // ---- bf16 B fragments for the windows (mma.m16n8k16).  Element (k-step s16, register r, lane 4n+t, half hf) is
    // channel 16 s16 + 8 r + 2 t + hf of mma column n.  MODE 0: column n holds head n>>1, its rounded value (n even)
    // or the rounding remainder (n odd).  MODE 1: column n holds head n; a second copy holds the remainders.
    const int s16 = ch >> 4, r16 = ch & 15, r = r16 >> 3, tw = (r16 & 7) >> 1, hf = r16 & 1;
    unsigned short* wfrag = reinterpret_cast<unsigned short*>(buf + QF);
#pragma unroll
    for (int n = 0; n < 8; ++n) {
        const int head = (MODE == 0) ? (n >> 1) : n;
        const float y = acc[head] * k2;                           // zero for unused head slots
        const float wrem = y - __bfloat162float(__float2bfloat16_rn(y));
        const float wval = (MODE == 0 && (n & 1)) ? wrem : y;
        const int idx = ((((s16 >> 1) * 32 + 4 * n + tw) * 4 + (s16 & 1) * 2 + r) << 1) + hf;
        wfrag[idx] = __bfloat16_as_ushort(__float2bfloat16_rn(wval));
        if (MODE == 1) wfrag[1024 + idx] = __bfloat16_as_ushort(__float2bfloat16_rn(wrem));
    }
    asm volatile("bar.sync 1, 128;" ::: "memory");
    if (ch < G) {
        const int* ri = red_isum[ch];
        const float* ra = red_abs[ch];
        const float amax = fmaxf(fmaxf(ra[0], ra[1]), fmaxf(ra[2], ra[3]));
        const float lam_h = (amax > 0.f && amax < 3e38f) ? amax * (1.f / Q_MAX) : 1.f;
        constexpr float FS = BITS != 4 ? 4.f : 16.f;      // the integer score carries this factor (see the main kernel)
        float* qs = P.qscal + (static_cast<long long>(b) * P.c.n_q + h * G + ch) * 2;
        qs[0] = k2 * lam_h * (1.f / FS);                  // score (log2 domain) = qs[0] * (Delta_k * sum_int + x_min_k * qs[1])
        qs[1] = FS * static_cast<float>(ri[0] + ri[1] + ri[2] + ri[3]);
    }
#pragma unroll
    for (int k = 0; k < (QF + 127) / 128; ++k)
        if (128 * k + ch < QF) P.qfrag[bh * 256 + 128 * k + ch] = buf[128 * k + ch];
#pragma unroll
    for (int k = 0; k < QW / 128; ++k) P.qwfrag[bh * 256 + 128 * k + ch] = buf[QF + 128 * k + ch];
    if (P.q_early && first_cta) pdl_wait();              // see above
}

// ------------------------------------------------------------------------------------------------
// 2. main kernel helpers
// ------------------------------------------------------------------------------------------------

// One (sequence, KV head) stretch of a warp's slice, kept in shared memory.  Units [u0, u1) of the
// head's unit list: units below qp are packed pages (page index first_page + u), the rest are window
// units of WIN_TOKENS tokens.
struct Segment {
    int b, h, slot, u0, u1, qp, first_page, q_lo, q_hi, n_win, n_sink, recent_lo;
    long long head_first;                 // flattened index of the head's unit 0
};
constexpr int MAX_SEGMENTS = 6;           // per warp and round; more segments take further rounds

// A (sequence, KV head) whose units are shared by several warps: its index, its first unit in the flattened list, its units.
struct SharedHead {
    int bh, n_units;
    long long first;
    const float* rec;                     // the warp's partials of the head's queries, in shared or global memory
};
// The warp whose slice [w total / ns, (w + 1) total / ns) holds unit u.
__device__ __noinline__ int wide_quotient(long long a, long long b) { return static_cast<int>(a / b); }
__device__ __forceinline__ int slice_owner(long long u, long long total, int ns) {
    const long long x = (u + 1) * ns - 1;
    if (x < (1LL << 32) && total < (1LL << 32)) return static_cast<int>(static_cast<unsigned>(x) / static_cast<unsigned>(total));
    return wide_quotient(x, total);
}

// Merge of the heads that several warps share, at the end of the main kernel.  First the shares of this CTA's warps (at most one
// per warp) are merged, one warp per (head, query head).  The first and the last of these heads may reach into other CTAs: of
// those, the CTA that arrives last at the query head's counter merges the CTAs' states, in CTA order, and writes the output: no
// CTA waits for another, and the result does not depend on which one is last.  What this costs is latency, most of it the
// release before the counters (1.3 us, 4.7 us when all CTAs get there together), so the CTA's counters are advanced together.
template <int MAIN_WARPS>
__device__ __forceinline__ void merge_shared_heads(const DecodeParams& P, const SharedHead* shared_s, const long long total) {
    const CacheView& c = P.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, G = c.G;
    __shared__ int leader_s[2], n_ctas_s[2], last_s[2][8];       // [0] the CTA's first shared head, [1] its last one if that is another
    const int my_bh = lane < 2 * MAIN_WARPS ? shared_s[lane].bh : -1;
    const unsigned slots_of = __match_any_sync(FULL, my_bh);
    const unsigned leaders = __ballot_sync(FULL, my_bh >= 0 && lane == __ffs(slots_of) - 1);
    if (leaders == 0) return;                                    // the same for every warp
    const int n_heads = __popc(leaders), cta_warp0 = blockIdx.x * MAIN_WARPS;
    const long long rec_step = static_cast<long long>(G) * PART_STRIDE;
    // The CTAs that share a head: all from the one that owns its first unit to the one that owns its last, or, when there are
    // more CTAs than units, the owner of each unit.  A CTA's state is at the warp that owns its first unit of the head.
    const bool every_cta = total >= gridDim.x, every_warp = total >= P.n_warps;
    for (int item = warp; item < n_heads * G; item += MAIN_WARPS) {
        const int k_head = item / G, head = item % G;
        unsigned rest = leaders;
        for (int k = k_head; k > 0; --k) rest &= rest - 1;
        const int leader = __ffs(rest) - 1;
        const unsigned slots = __shfl_sync(FULL, slots_of, leader);
        const SharedHead hd = shared_s[leader];
        const int n_shares = __popc(slots);
        unsigned from_k = slots;                                     // lane k: the k-th share's slot is its lowest bit
        for (int k = min(lane, n_shares - 1); k > 0; --k) from_k &= from_k - 1;
        const unsigned long long my_rec = reinterpret_cast<unsigned long long>(shared_s[__ffs(from_k) - 1].rec + head * PART_STRIDE);
        MergedState ms;
        ms.reset();
        ms.add<false>(n_shares, lane, [&](int k) { return reinterpret_cast<const float*>(__shfl_sync(FULL, my_rec, k)); });
        int n_ctas = 1;
        if (k_head == 0 || k_head == n_heads - 1) {
            n_ctas = hd.n_units;
            if (every_cta) n_ctas = slice_owner(hd.first + hd.n_units - 1, total, P.n_warps) / MAIN_WARPS - slice_owner(hd.first, total, P.n_warps) / MAIN_WARPS + 1;
            if (lane == 0) { leader_s[k_head == 0 ? 0 : 1] = leader; n_ctas_s[k_head == 0 ? 0 : 1] = n_ctas; }
        }
        if (n_ctas > 1) ms.store(P.part + (static_cast<long long>(hd.bh) * G + head) * PART_STRIDE + (cta_warp0 + (leader >> 1)) * rec_step, lane);
        else ms.finish(P.O + (static_cast<long long>(hd.bh / c.n_kv) * c.n_q + (hd.bh % c.n_kv) * G + head) * D, lane);
    }
    __syncthreads();
    const int n_ends = n_heads > 1 ? 2 : 1;
    if (threadIdx.x < n_ends * G) {
        const int e = threadIdx.x / G, head = threadIdx.x % G;
        int last = 0;
        if (n_ctas_s[e] > 1) {
            __threadfence();                                     // the CTA's states before its arrival (barrier above), the others' after it
            last = atomicAdd(arrival_counters(P, shared_s[leader_s[e]].bh) + head, 1) == n_ctas_s[e] - 1;
            __threadfence();
        }
        last_s[e][head] = last;
    }
    __syncthreads();
    for (int item = warp; item < n_ends * G; item += MAIN_WARPS) {
        const int e = item / G, head = item % G;
        if (!last_s[e][head]) continue;
        const SharedHead hd = shared_s[leader_s[e]];
        const float* rec0 = P.part + (static_cast<long long>(hd.bh) * G + head) * PART_STRIDE;     // the head's record of warp 0
        const int w_first = slice_owner(hd.first, total, P.n_warps), c_first = w_first / MAIN_WARPS;
        MergedState ms;
        ms.reset();
        if (every_warp)
            ms.add<true>(n_ctas_s[e], lane, [&](int k) { return rec0 + max(w_first, (c_first + k) * MAIN_WARPS) * rec_step; });
        else
            ms.add<true>(n_ctas_s[e], lane, [&](int k) {
                const long long u = every_cta ? max(hd.first, static_cast<long long>(c_first + k) * MAIN_WARPS * total / P.n_warps) : hd.first + k;
                return rec0 + slice_owner(u, total, P.n_warps) * rec_step;
            });
        ms.finish(P.O + (static_cast<long long>(hd.bh / c.n_kv) * c.n_q + (hd.bh % c.n_kv) * G + head) * D, lane);
    }
}

// ------------------------------------------------------------------------------------------------
// main kernel
// ------------------------------------------------------------------------------------------------
#if WUSHKV_ABL & 16
__device__ unsigned long long g_timeline[8192 * 4];
__device__ __forceinline__ unsigned long long gtime() { unsigned long long t; asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t)); return t; }
#define TL(slot) do { if (lane == 0) g_timeline[((blockIdx.x * 16 + warp) & 8191) * 4 + (slot)] = gtime(); } while (0)
#else
#define TL(slot) do { } while (0)
#endif

template <int BITS, int MODE, int STAGES>
__global__ void __launch_bounds__(main_warps(BITS, MODE) * 32, 1) decode_main_kernel(DecodeParams P) {
    constexpr int MAIN_WARPS = main_warps(BITS, MODE);
    constexpr int REC = record_bytes(BITS);
    constexpr int NH = WarpState<MODE>::NH;
    static_assert(2 * WIN_TOKENS * WIN_ROW <= REC, "a window unit must fit in one stage");
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(smem + MAIN_WARPS * STAGES * REC);
    Segment* seg_all = reinterpret_cast<Segment*>(smem + MAIN_WARPS * STAGES * REC + MAIN_WARPS * STAGES * 8);
    const CacheView& c = P.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int G = c.G;
    Segment* segs = seg_all + warp * MAX_SEGMENTS;
    TL(0);

    // ---- work plan: prefix sums of units per sequence.  Recomputed here from the inputs (into the still
    // unused staging area) so that nothing the preparation kernel writes is needed before the first copies.
    __shared__ long long scan_s[MAIN_WARPS];
    long long* plan_s = reinterpret_cast<long long*>(smem);
    static_assert((MAX_LOCAL_PLAN + 1) * sizeof(long long) <= static_cast<size_t>(MAIN_WARPS) * STAGES * REC, "the plan must fit in the staging area");
    const bool local_plan = P.batch <= MAX_LOCAL_PLAN;
    if (P.q_early || !local_plan) pdl_wait();           // lengths from the append / plan from the preparation kernel
    for (int b = blockIdx.x * MAIN_WARPS * 32 + threadIdx.x; b < P.batch; b += gridDim.x * MAIN_WARPS * 32) {
        const int slot = __ldg(P.slot + b);
        if (slot < 0 || slot >= c.n_slots) atomicOr(c.dev_status, WUSHKV_DEV_BAD_SLOT);
    }
    if (local_plan) {
        long long carry = 0;
        for (int base = 0; base < P.batch; base += MAIN_WARPS * 32) {
            const int bb = base + threadIdx.x;
            long long incl = 0;
            if (bb < P.batch) incl = seq_info(c, __ldcg(P.seq_len + bb), __ldg(P.slot + bb)).U;
            for (int o = 1; o < 32; o <<= 1) {
                const long long v = __shfl_up_sync(FULL, incl, o);
                if (lane >= o) incl += v;
            }
            if (lane == 31) scan_s[warp] = incl;
            __syncthreads();
            long long before = 0, all = 0;
            for (int w = 0; w < MAIN_WARPS; ++w) { if (w < warp) before += scan_s[w]; all += scan_s[w]; }
            if (bb < P.batch) plan_s[bb + 1] = carry + before + incl;
            carry += all;
            __syncthreads();
        }
        if (threadIdx.x == 0) plan_s[0] = 0;
        __syncthreads();
    }
    const long long* plan = local_plan ? plan_s : P.plan;

    // ---- this warp's slice of the flattened unit list
    const long long total = plan[P.batch] * c.n_kv;
    const long long wg = static_cast<long long>(blockIdx.x) * MAIN_WARPS + warp;
    long long L = total > 0 ? wg * total / P.n_warps : 0;
    const long long L1 = total > 0 ? (wg + 1) * total / P.n_warps : 0;

    // position of the slice start: sequence b, head h, unit u
    int sb = 0, sh = 0, su = 0;
    if (L < L1) {
        int lo = 0, hi = P.batch;           // largest b with n_kv * plan[b] <= L
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (plan[mid] * c.n_kv <= L) lo = mid; else hi = mid;
        }
        sb = lo;
        const long long U = max(plan[lo + 1] - plan[lo], 1LL);
        const long long rem = L - plan[lo] * c.n_kv;
        sh = static_cast<int>(rem / U);
        su = static_cast<int>(rem % U);
    }
    for (int b = blockIdx.x; b < P.batch; b += gridDim.x)      // a sequence without units gets zeros
        if (plan[b + 1] == plan[b])
            for (int k = threadIdx.x; k < c.n_q * D; k += MAIN_WARPS * 32) P.O[static_cast<long long>(b) * c.n_q * D + k] = 0.f;
    __shared__ SharedHead shared_s[2 * MAIN_WARPS];             // [2 warp]: head the warp entered in its middle, [2 warp + 1]: head it left unfinished
    __shared__ long long total_s;           // kept for the merge at the end
    if (threadIdx.x < 2 * MAIN_WARPS) shared_s[threadIdx.x].bh = -1;
    if (threadIdx.x == 0) total_s = total;
    __syncthreads();                        // the staging area stops being plan scratch here
    pdl_launch_dependents();

    // ---- barriers
    const unsigned bar0 = smem_u32(bars + warp * STAGES);
    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < STAGES; ++s) mbar_init(bar0 + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    const unsigned stage0 = smem_u32(smem + warp * STAGES * REC);
    const long long page_row_bytes = static_cast<long long>(c.n_kv) * REC;
    const unsigned long long stream_policy = l2_evict_first_policy();

    if (WUSHKV_ABL & 8) { for (int k = lane; k < STAGES * REC / 4; k += 32) reinterpret_cast<unsigned*>(smem + warp * STAGES * REC)[k] = 0u; __syncwarp(); }
    unsigned qf[4][2];                  // integer B fragments of the four k-steps (MODE 1: the high digits)
    unsigned qfl[MODE == 1 ? 4 : 1][2]; // MODE 1: the low digits
    float fmul[NH], gadd[NH];
    WarpState<MODE> st;
    int stage = 0;                      // ring position of the next unit to consume (and to refill)
    unsigned phase_bits = 0;            // parity of each stage's next completion
    unsigned bad_bits = 0;              // lane 0: stages whose unit could not be fetched
    bool timed_out = false;
    const int wait_limit = P.wait_limit > 0 ? P.wait_limit : (1 << 19);      // polls that may sleep ~2 us each: about a second

    while (L < L1) {
        // ================= round set-up: list the next segments of the slice =====================
        int n_seg = 0, round_units = 0;
        while (n_seg < MAX_SEGMENTS && L < L1) {
            const SeqInfo si = seq_info(c, __ldcg(P.seq_len + sb), __ldg(P.slot + sb));
            if (si.U > 0) {
                const int u1 = static_cast<int>(min(static_cast<long long>(si.U), su + (L1 - L)));
                if (lane == 0) {
                    Segment sg;
                    sg.b = sb; sg.h = sh; sg.slot = si.slot; sg.u0 = su; sg.u1 = u1; sg.qp = si.qp; sg.first_page = si.first_page;
                    sg.q_lo = si.q_lo; sg.q_hi = si.q_hi; sg.n_win = si.n_win; sg.n_sink = si.n_sink; sg.recent_lo = si.recent_lo;
                    sg.head_first = L - su;
                    segs[n_seg] = sg;
                }
                ++n_seg;
                round_units += u1 - su;
                L += u1 - su;
                su = u1;
            }
            if (si.U == 0 || su >= si.U) {              // next head, or next sequence
                su = 0;
                if (si.U == 0 || ++sh >= c.n_kv) { sh = 0; ++sb; }
                if (sb >= P.batch) break;
            }
        }
        __syncwarp();

        // ================= producer: stages the units of this round, in order =====================
        const long long round_L0 = L - round_units;      // flattened index of the round's first unit
        int p_seg = -1, p_u = 0, p_u1 = 0, p_qp = 0, p_head_off = 0, issued = 0;
        const int* p_ptab = nullptr;
        auto issue_next = [&](const int s) {            // whole warp; stages the round's next unit into ring slot s
            if (p_u == p_u1) {                          // next segment
                ++p_seg;
                const Segment& sg = segs[p_seg];
                p_u = sg.u0; p_u1 = sg.u1; p_qp = sg.qp; p_head_off = sg.h * REC;
                p_ptab = c.page_table + static_cast<long long>(sg.slot) * c.max_pages + sg.first_page;
                if (sg.first_page + sg.qp > c.max_pages) {      // the page table cannot hold this length
                    if (lane == 0) atomicOr(c.dev_status, WUSHKV_DEV_PAGE_TABLE_FULL);
                    p_qp = min(p_qp, max(c.max_pages - sg.first_page, 0));   // pages beyond it are treated as window-less gaps below
                }
            }
            const unsigned bar = bar0 + 8 * s, dst = stage0 + s * REC;
            const Segment& sg = segs[p_seg];
            if (p_u < sg.qp) {                          // a packed page: one bulk copy
                if (lane == 0) {
                    const int page = (p_u < p_qp) ? __ldg(p_ptab + p_u) : -1;
                    if (static_cast<unsigned>(page) >= static_cast<unsigned long long>(c.n_pages)) {
                        if (p_u < p_qp) atomicOr(c.dev_status, WUSHKV_DEV_BAD_PAGE_ID);
                        bad_bits |= 1u << s;
                        mbar_arrive(bar);
                    } else if (WUSHKV_ABL & 8) {        // timing experiment: no copy, the stage keeps its (zeroed) content
                        bad_bits &= ~(1u << s);
                        mbar_arrive(bar);
                    } else {
                        bad_bits &= ~(1u << s);
                        mbar_expect_tx(bar, REC);
                        if (P.drop_unit >= 0 && P.drop_unit == round_L0 + issued) {
                            // testing aid: the copy is announced but never issued, so the wait for it runs into its limit
                        } else if (P.stream_pages) bulk_copy_g2s_stream(dst, c.pages + page * page_row_bytes + p_head_off, REC, bar, stream_policy);
                        else bulk_copy_g2s(dst, c.pages + page * page_row_bytes + p_head_off, REC, bar);
                    }
                }
            } else {                                    // up to 8 window tokens: one 256-byte row copy per lane
                const int w0 = (p_u - sg.qp) * WIN_TOKENS;
                const int n_valid = min(WIN_TOKENS, sg.n_win - w0);
                if (lane == 0) { bad_bits &= ~(1u << s); mbar_expect_tx(bar, n_valid * 2 * D * 2); }
                __syncwarp();
                const int r = lane & 7, which = lane >> 3;      // lanes 0-7: key rows, 8-15: value rows
                if (lane < 16 && r < n_valid) {
                    const int w = w0 + r;
                    const long long plane = (static_cast<long long>(sg.slot) * c.n_kv + sg.h) * 2 + which;
                    const unsigned short* src;
                    if (w < sg.n_sink) src = c.sink_kv + (plane * c.s_sink + w) * D;
                    else src = c.ring_kv + (plane * c.ring_cap + (sg.recent_lo + (w - sg.n_sink)) % c.ring_cap) * D;
                    bulk_copy_g2s(dst + which * WIN_V_OFF + r * WIN_ROW, src, D * 2, bar);
                }
            }
            ++p_u;
            ++issued;
        };
        for (int k = 0; k < STAGES && k < round_units && !timed_out; ++k) issue_next((stage + k) % STAGES);
        TL(1);

        // ================= consumer ==============================================================
        pdl_wait();                                     // query fragments come from the preparation kernel
        for (int cs = 0; cs < n_seg; ++cs) {
            const Segment& sg = segs[cs];               // rarely used fields are re-read from shared memory
            const long long bh = static_cast<long long>(sg.b) * c.n_kv + sg.h;
            const int u1 = sg.u1, qp = sg.qp, q_lo = sg.q_lo, q_hi = sg.q_hi;
            int pos0 = (sg.first_page + sg.u0) * PAGE_TOKENS;
            {   // query fragments and per-head scalars of this (sequence, KV head)
                const uint4* src = P.qfrag + bh * 256;
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2) {
                    const uint4 v = __ldcg(src + s2 * 32 + lane);
                    qf[2 * s2][0] = v.x; qf[2 * s2][1] = v.y; qf[2 * s2 + 1][0] = v.z; qf[2 * s2 + 1][1] = v.w;
                    if (MODE == 1) {
                        const uint4 w = __ldcg(src + 64 + s2 * 32 + lane);
                        qfl[2 * s2][0] = w.x; qfl[2 * s2][1] = w.y; qfl[2 * s2 + 1][0] = w.z; qfl[2 * s2 + 1][1] = w.w;
                    }
                }
#pragma unroll
                for (int k = 0; k < NH; ++k) {
                    const int head = MODE == 0 ? t : 2 * t + k;
                    fmul[k] = 1.f; gadd[k] = 0.f;             // unused head slots stay finite
                    if (head < G) {
                        const float2 v = __ldcg(reinterpret_cast<const float2*>(P.qscal + (static_cast<long long>(sg.b) * c.n_q + sg.h * G + head) * 2));
                        fmul[k] = v.x; gadd[k] = v.y;
                    }
                }
                st.reset();
            }
            for (int u = sg.u0; u < u1 && !timed_out; ++u, pos0 += PAGE_TOKENS) {
                const int s = stage;
                // a phase that one lane saw complete is complete for all: keep the decision warp-uniform
                if (!__any_sync(FULL, mbar_wait_bounded(bar0 + 8 * s, (phase_bits >> s) & 1u, wait_limit))) {
                    timed_out = true;
                    if (lane == 0) atomicOr(c.dev_status, WUSHKV_DEV_COPY_TIMEOUT);
                    // Copies of this warp's other stages may still be in flight: wait for each (bounded; a stage with nothing
                    // pending simply runs the limit out) before its shared memory is used for anything else or released.
                    const int drain_limit = min(wait_limit, 1 << 9);
#pragma unroll
                    for (int k = 0; k < STAGES; ++k) mbar_wait_bounded(bar0 + 8 * k, (phase_bits >> k) & 1u, drain_limit);
                    break;
                }
                phase_bits ^= 1u << s;
#if WUSHKV_ABL & 16
                if (lane == 0 && g_timeline[((blockIdx.x * 16 + warp) & 8191) * 4 + 2] == 0) g_timeline[((blockIdx.x * 16 + warp) & 8191) * 4 + 2] = gtime();
#endif
                const unsigned rec = stage0 + s * REC;
                if (u >= qp) {
                    // ======================= window unit: up to 8 bf16 tokens ==========================
                    const int w0 = (u - qp) * WIN_TOKENS;
                    const uint4* wsrc = P.qwfrag + (static_cast<long long>(sg.b) * c.n_kv + sg.h) * 256;
                    window_unit<BITS, MODE>(st, rec, rec + WIN_V_OFF, min(WIN_TOKENS, sg.n_win - w0), [wsrc](int k) { return __ldcg(wsrc + k); }, lane);
                } else if (!__any_sync(FULL, (bad_bits >> s) & 1u)) {
                    // ======================= packed page: 64 quantized tokens ==========================
                    const bool full_page = (pos0 >= q_lo) && (pos0 + PAGE_TOKENS <= q_hi);
                    float sc[4][2 * NH];          // [block][row g: heads..., row g+8: heads...]
                    unsigned vmeta[4][2];         // fp16x2 (Delta_v, x_min_v) of rows g, g+8
                    page_scores<BITS, MODE>(rec, rec + meta_offset(BITS), qf, qfl, gadd, sc, vmeta, lane);
                    if (!full_page) {             // first / last page of the quantized range: mask the tokens outside it
#pragma unroll
                        for (int bi = 0; bi < 4; ++bi) {
                            const int p0 = pos0 + bi * 16 + g, p1 = p0 + 8;
                            if (p0 < q_lo || p0 >= q_hi) {
                                vmeta[bi][0] = 0u;
#pragma unroll
                                for (int k = 0; k < NH; ++k) sc[bi][k] = -INFINITY;
                            }
                            if (p1 < q_lo || p1 >= q_hi) {
                                vmeta[bi][1] = 0u;
#pragma unroll
                                for (int k = 0; k < NH; ++k) sc[bi][NH + k] = -INFINITY;
                            }
                        }
                    }
                    // ---------------- running maximum of the page, rescale if it grew
                    float mx[NH];
#pragma unroll
                    for (int k = 0; k < NH; ++k) {
                        const float v = fmaxf(fmaxf(fmaxf(sc[0][k], sc[0][NH + k]), fmaxf(sc[1][k], sc[1][NH + k])),
                                              fmaxf(fmaxf(sc[2][k], sc[2][NH + k]), fmaxf(sc[3][k], sc[3][NH + k])));
                        mx[k] = v * fmul[k];          // scores are kept divided by the head's multiplier (> 0)
                    }
                    st.raise_max(mx);
                    // ---------------- probabilities, value reduction
                    page_values<BITS, MODE>(st, rec + v_codes_offset(BITS), sc, vmeta, fmul, lane);
                }
                __syncwarp();
                if (issued < round_units) issue_next(s);         // refill the stage just consumed
                stage = (stage + 1 == STAGES) ? 0 : stage + 1;
            }
            // A head that lies inside this warp's slice is finished here.  One that is shared leaves a partial result (after a
            // wait that ran out: of what was read until then, so that whoever merges the head still finds every share): in
            // the warp's ring if that has served its last unit, else in global memory.
            const int U = qp + (sg.n_win + WIN_TOKENS - 1) / WIN_TOKENS;
            if (sg.u0 == 0 && u1 == U) {
                store_state<BITS, MODE, true>(st, P.O + (static_cast<long long>(sg.b) * c.n_q + sg.h * G) * D, lane, G);
            } else {
                static_assert(8 * PART_STRIDE * 4 <= STAGES * REC, "the partials of 8 query heads must fit in a warp's ring");
                const bool last = cs == n_seg - 1 && L >= L1;
                float* rec = last ? reinterpret_cast<float*>(smem + warp * STAGES * REC) : P.part + (wg + bh) * G * PART_STRIDE;
                if (last) __syncwarp();                      // every lane has read the last unit
                store_state<BITS, MODE, false>(st, rec, lane, G);
                if (lane == 0) {
                    SharedHead& hd = shared_s[2 * warp + (sg.u0 == 0 ? 1 : 0)];
                    hd.bh = static_cast<int>(bh); hd.n_units = U; hd.first = sg.head_first; hd.rec = rec;
                }
            }
        }
        __syncwarp();
    }
    TL(3);
    // ---- heads that several warps share
    pdl_wait();                             // warps without units: the counters were zeroed by the preparation kernel
    __syncthreads();
    merge_shared_heads<MAIN_WARPS>(P, shared_s, total_s);
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
struct DecodePlan {
    int n_ctas, n_warps;
    size_t off_qfrag, off_qwfrag, off_qscal, off_plan, off_part, total;
};

static size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

static bool make_plan(const CacheView& c, int batch, int max_seq_len, DecodePlan& pl) {
    if (batch <= 0 || max_seq_len <= 0) return false;
    const long long pages_max = (static_cast<long long>(max_seq_len) + PAGE_TOKENS - 1) / PAGE_TOKENS + 1;
    const long long win_max = std::min<long long>(max_seq_len, c.s_sink + c.s_keep + c.s_flush - 1 + c.lag);
    const long long units_max = (pages_max + (win_max + WIN_TOKENS - 1) / WIN_TOKENS + 1) * batch * c.n_kv;
    const int warps = main_warps(c.bits, c.G <= 4 ? 0 : 1);
    long long ctas = knobs().decode_ctas;
    if (ctas <= 0) {
        // one CTA per SM; small problems take fewer, so that every warp still gets about two units
        ctas = std::min<long long>(sm_count(), (units_max + 2 * warps - 1) / (2 * warps));
    }
    ctas = std::max<long long>(1, std::min<long long>(ctas, 1 << 20));
    pl.n_ctas = static_cast<int>(ctas);
    pl.n_warps = pl.n_ctas * warps;
    const size_t bh = static_cast<size_t>(batch) * c.n_kv;
    size_t off = 0;
    pl.off_qfrag = off;  off = align_up(off + bh * 256 * sizeof(uint4), 256);
    pl.off_qwfrag = off; off = align_up(off + bh * 256 * sizeof(uint4), 256);
    pl.off_qscal = off;  off = align_up(off + static_cast<size_t>(batch) * c.n_q * 2 * sizeof(float), 256);
    pl.off_plan = off;   off = align_up(off + (static_cast<size_t>(batch) + 1) * sizeof(long long), 256);
    pl.off_part = off;   off = align_up(off + (pl.n_warps + bh) * c.G * PART_STRIDE * sizeof(float), 256);
    pl.total = off;
    return true;
}

static cudaEvent_t g_prof_start = nullptr, g_prof_stop = nullptr;

template <int BITS, int MODE>
static int launch_decode(const DecodeParams& P, int n_ctas, cudaStream_t st) {
    constexpr int MAIN_WARPS = main_warps(BITS, MODE);
#ifndef WUSHKV_STAGES_2BIT
#define WUSHKV_STAGES_2BIT 2
#endif
    constexpr int STAGES = (BITS == 2 && MODE == 0) ? WUSHKV_STAGES_2BIT : 2;      // per-warp ring depth
    constexpr size_t SMEM = static_cast<size_t>(MAIN_WARPS) * STAGES * record_bytes(BITS) + MAIN_WARPS * STAGES * 8 +
                            MAIN_WARPS * MAX_SEGMENTS * sizeof(Segment);
    cudaLaunchAttribute pdl_attr[1];
    pdl_attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    pdl_attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = st;
    cfg.attrs = pdl_attr;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3(P.c.n_kv, P.batch);
    cfg.blockDim = dim3(PREP_THREADS);
    cfg.dynamicSmemBytes = 0;
    if (cudaLaunchKernelEx(&cfg, decode_prep_kernel<BITS, MODE>, P) != cudaSuccess) return WUSHKV_ECUDA;
    if (!opt_in_dynamic_smem(reinterpret_cast<const void*>(decode_main_kernel<BITS, MODE, STAGES>), static_cast<int>(SMEM))) return WUSHKV_ECUDA;
    if (g_prof_start) cudaEventRecord(g_prof_start, st);
    cfg.gridDim = dim3(n_ctas);
    cfg.blockDim = dim3(MAIN_WARPS * 32);
    cfg.dynamicSmemBytes = SMEM;
    if (cudaLaunchKernelEx(&cfg, decode_main_kernel<BITS, MODE, STAGES>, P) != cudaSuccess) return WUSHKV_ECUDA;
    if (g_prof_stop) cudaEventRecord(g_prof_stop, st);
    return WUSHKV_OK;
}

}  // namespace wushkv

using namespace wushkv;

extern "C" size_t wushkv_decode_workspace_bytes(const wushkv_cache* cache, int32_t batch, int32_t max_seq_len) {
    CacheView v;
    if (make_view(cache, v) != WUSHKV_OK) return 0;
    DecodePlan pl;
    if (!make_plan(v, batch, max_seq_len, pl)) return 0;
    return pl.total;
}

static int decode_attn_impl(const wushkv_cache* cache, int32_t batch, const int32_t* slot, const int32_t* seq_len,
                            int32_t max_seq_len, const uint16_t* Q, float* O,
                            void* workspace, size_t workspace_bytes, void* stream, int q_early,
                            const wushkv_prologue* prologue = nullptr) {
    DecodeParams P;
    P.q_early = q_early;
    const int rc = make_view(cache, P.c);
    if (rc != WUSHKV_OK) return rc;
    if (!slot || !seq_len || !int_arrays(slot, seq_len) || !Q || !O || !workspace || !aligned(Q, 16) || !aligned(O, 16) || !aligned(workspace, 256)) return WUSHKV_EINVAL;
    DecodePlan pl;
    if (!make_plan(P.c, batch, max_seq_len, pl)) return WUSHKV_EINVAL;
    if (batch > 65535) return WUSHKV_EINVAL;
    if (workspace_bytes < pl.total) return WUSHKV_ECAPACITY;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    P.batch = batch; P.slot = slot; P.seq_len = seq_len; P.Q = Q; P.O = O;
    P.qfrag = reinterpret_cast<uint4*>(ws + pl.off_qfrag);
    P.qwfrag = reinterpret_cast<uint4*>(ws + pl.off_qwfrag);
    P.qscal = reinterpret_cast<float*>(ws + pl.off_qscal);
    P.plan = reinterpret_cast<long long*>(ws + pl.off_plan);
    P.part = reinterpret_cast<float*>(ws + pl.off_part);
    P.n_warps = pl.n_warps;
    P.wait_limit = static_cast<int>(std::min<long long>(std::max<long long>(knobs().wait_limit, 0), 1 << 30));
    P.drop_unit = knobs().drop_copy_unit;
    P.pro = Prologue{nullptr, 0, 0, nullptr, 0.f};
    if (prologue && !make_prologue(prologue, prologue->q_norm_weight, P.pro)) return WUSHKV_EINVAL;
    {   // upper bound of the packed bytes one step reads against the L2 size
        static int l2_bytes[64] = {};
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess) return WUSHKV_ECUDA;
        int l2 = (dev >= 0 && dev < 64) ? l2_bytes[dev] : 0;
        if (l2 == 0) {
            if (cudaDeviceGetAttribute(&l2, cudaDevAttrL2CacheSize, dev) != cudaSuccess) return WUSHKV_ECUDA;
            if (dev >= 0 && dev < 64) l2_bytes[dev] = l2;
        }
        const double step_bytes = static_cast<double>(batch) * P.c.n_kv * ((max_seq_len + PAGE_TOKENS - 1) / PAGE_TOKENS) *
                                  record_bytes(P.c.bits);
        P.stream_pages = step_bytes > static_cast<double>(l2) ? 1 : 0;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool mode0 = P.c.G <= 4;
    if (P.c.bits == 2) return mode0 ? launch_decode<2, 0>(P, pl.n_ctas, st) : launch_decode<2, 1>(P, pl.n_ctas, st);
    if (P.c.bits == 3) return mode0 ? launch_decode<3, 0>(P, pl.n_ctas, st) : launch_decode<3, 1>(P, pl.n_ctas, st);
    return mode0 ? launch_decode<4, 0>(P, pl.n_ctas, st) : launch_decode<4, 1>(P, pl.n_ctas, st);
}

extern "C" int wushkv_decode_attn(const wushkv_cache* cache, int32_t batch, const int32_t* slot, const int32_t* seq_len,
                                  int32_t max_seq_len, const uint16_t* Q, float* O,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    return decode_attn_impl(cache, batch, slot, seq_len, max_seq_len, Q, O, workspace, workspace_bytes, stream, 0);
}

extern "C" int wushkv_decode_attn_projected(const wushkv_cache* cache, int32_t batch, const int32_t* slot, const int32_t* seq_len,
                                            int32_t max_seq_len, const uint16_t* Q_proj, const wushkv_prologue* prologue, float* O,
                                            void* workspace, size_t workspace_bytes, void* stream) {
    if (!prologue) return WUSHKV_EINVAL;
    // the query's position is the final length minus one: the preparation kernel waits for the kernel ahead of it
    return decode_attn_impl(cache, batch, slot, seq_len, max_seq_len, Q_proj, O, workspace, workspace_bytes, stream, 0, prologue);
}

extern "C" int wushkv_decode_step(const wushkv_cache* cache, int32_t batch, const int32_t* slot, int32_t* seq_len,
                                  const int32_t* cu_new, int32_t max_seq_len,
                                  const uint16_t* K_new, const uint16_t* V_new, const uint16_t* Q, float* O,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    if (batch <= 0 || !Q || !O || !workspace) return WUSHKV_EINVAL;
    // validate the decode half before anything is appended
    CacheView v;
    int r = make_view(cache, v);
    if (r != WUSHKV_OK) return r;
    DecodePlan pl;
    if (!make_plan(v, batch, max_seq_len, pl) || batch > 65535 || !aligned(Q, 16) || !aligned(O, 16) || !aligned(workspace, 256)) return WUSHKV_EINVAL;
    if (workspace_bytes < pl.total) return WUSHKV_ECAPACITY;
    r = wushkv_append(cache, batch, slot, seq_len, cu_new, batch, 1, K_new, V_new, stream);
    if (r != WUSHKV_OK) return r;
    // the single-token append kernel is now the kernel ahead of the query preparation, and it started
    // only after all earlier work in the stream: the preparation may read Q without waiting for it
    return decode_attn_impl(cache, batch, slot, seq_len, max_seq_len, Q, O, workspace, workspace_bytes, stream, 1);
}

#if WUSHKV_ABL & 16
extern "C" int wushkv_debug_timeline(unsigned long long* host_out, int clear) {
    if (cudaMemcpyFromSymbol(host_out, g_timeline, sizeof(g_timeline)) != cudaSuccess) return WUSHKV_ECUDA;
    if (clear) { void* p; cudaGetSymbolAddress(&p, g_timeline); cudaMemset(p, 0, sizeof(g_timeline)); }
    return WUSHKV_OK;
}
#endif

extern "C" int wushkv_set_profile_events(void* start, void* stop) {
    if ((start == nullptr) != (stop == nullptr)) return WUSHKV_EINVAL;
    g_prof_start = static_cast<cudaEvent_t>(start);
    g_prof_stop = static_cast<cudaEvent_t>(stop);
    return WUSHKV_OK;
}

extern "C" size_t wushkv_step_staging_bytes(const wushkv_cache* cache, int32_t batch) {
    CacheView v;
    if (make_view(cache, v) != WUSHKV_OK || batch <= 0) return 0;
    const size_t kv = align_up(static_cast<size_t>(batch) * v.n_kv * D * 2, 256);
    const size_t q = align_up(static_cast<size_t>(batch) * v.n_q * D * 2, 256);
    const size_t o = align_up(static_cast<size_t>(batch) * v.n_q * D * 4, 256);
    return 2 * kv + q + o;
}

// Device-side alias of a pinned, mapped host buffer (unified addressing), or nullptr.
static void* mapped_alias(const void* host_ptr) {
    cudaPointerAttributes a;
    if (cudaPointerGetAttributes(&a, host_ptr) != cudaSuccess) { cudaGetLastError(); return nullptr; }
    if (a.type != cudaMemoryTypeHost || a.devicePointer == nullptr) return nullptr;
    return aligned(a.devicePointer, 16) ? a.devicePointer : nullptr;
}

extern "C" int wushkv_decode_step_host(const wushkv_cache* cache, int32_t batch, const int32_t* slot, int32_t* seq_len,
                                       const int32_t* cu_new, int32_t max_seq_len,
                                       const uint16_t* K_new_host, const uint16_t* V_new_host, const uint16_t* Q_host,
                                       float* O_host, void* staging, size_t staging_bytes,
                                       void* workspace, size_t workspace_bytes, void* stream) {
    CacheView v;
    const int rc = make_view(cache, v);
    if (rc != WUSHKV_OK) return rc;
    if (batch <= 0 || !K_new_host || !V_new_host || !Q_host || !O_host || !staging || !aligned(staging, 256)) return WUSHKV_EINVAL;
    if (staging_bytes < wushkv_step_staging_bytes(cache, batch)) return WUSHKV_ECAPACITY;
    const size_t kv_bytes = static_cast<size_t>(batch) * v.n_kv * D * 2, kv = align_up(kv_bytes, 256);
    const size_t q_bytes = static_cast<size_t>(batch) * v.n_q * D * 2, q = align_up(q_bytes, 256);
    const size_t o_bytes = static_cast<size_t>(batch) * v.n_q * D * 4;
    unsigned char* sp = static_cast<unsigned char*>(staging);
    uint16_t* dK = reinterpret_cast<uint16_t*>(sp);
    uint16_t* dV = reinterpret_cast<uint16_t*>(sp + kv);
    uint16_t* dQ = reinterpret_cast<uint16_t*>(sp + 2 * kv);
    float* dO = reinterpret_cast<float*>(sp + 2 * kv + q);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // Pinned host buffers are visible to the device: the kernels then read the new token and the queries,
    // and write the outputs, in place over the bus, which saves four copy operations per step (about 320 KB
    // in config 1, where the copies' fixed costs dominate).  WUSHKV_HOST_IO=copy forces the staged copies.
    if (!knobs().host_io_copy) {
        void* aK = mapped_alias(K_new_host);
        void* aV = aK ? mapped_alias(V_new_host) : nullptr;
        void* aQ = aV ? mapped_alias(Q_host) : nullptr;
        void* aO = aQ ? mapped_alias(O_host) : nullptr;
        if (aO)
            return wushkv_decode_step(cache, batch, slot, seq_len, cu_new, max_seq_len, static_cast<const uint16_t*>(aK),
                                      static_cast<const uint16_t*>(aV), static_cast<const uint16_t*>(aQ), static_cast<float*>(aO),
                                      workspace, workspace_bytes, stream);
    }
    if (cudaMemcpyAsync(dK, K_new_host, kv_bytes, cudaMemcpyHostToDevice, st) != cudaSuccess) return WUSHKV_ECUDA;
    if (cudaMemcpyAsync(dV, V_new_host, kv_bytes, cudaMemcpyHostToDevice, st) != cudaSuccess) return WUSHKV_ECUDA;
    if (cudaMemcpyAsync(dQ, Q_host, q_bytes, cudaMemcpyHostToDevice, st) != cudaSuccess) return WUSHKV_ECUDA;
    const int r = wushkv_decode_step(cache, batch, slot, seq_len, cu_new, max_seq_len, dK, dV, dQ, dO, workspace, workspace_bytes, stream);
    if (r != WUSHKV_OK) return r;
    if (cudaMemcpyAsync(O_host, dO, o_bytes, cudaMemcpyDeviceToHost, st) != cudaSuccess) return WUSHKV_ECUDA;
    return WUSHKV_OK;
}
