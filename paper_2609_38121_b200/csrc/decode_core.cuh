// What the decode kernels share: work units of a sequence, staging copies, scores and values of a packed page or of window
// tokens, the running softmax state of a warp and the merge of such states.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "layout.cuh"

namespace wushkv {

constexpr unsigned FULL = 0xffffffffu;
constexpr int PART_STRIDE = 132;          // floats per partial: [0]=max (log2 domain) [1]=sum [4..131]=o
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LO_SCALE = 2048.f;        // a "remainder" column of a window unit carries (x - rounded(x)) * 2^11
constexpr float Q_MAX = 32512.f;          // largest magnitude of the 16-bit fixed-point query (127 * 256: both digits fit a signed byte)
// Exponentials are taken against (running reference - LOG2_PV): every probability, and with it l, z and
// o of a partial, carries the common factor 2^LOG2_PV, which cancels in the final ratio and keeps
// fp16(p Delta_v) out of the subnormals.  The reference is only raised (and the state rescaled) when
// a unit's maximum exceeds it by more than MAX_SLACK, so p <= 2^(LOG2_PV + MAX_SLACK) and
// p Delta_v stays finite in fp16 for Delta_v < 2^(16 - LOG2_PV - MAX_SLACK) = 1024.
constexpr float LOG2_PV = 3.f;
constexpr float MAX_SLACK = 3.f;
constexpr int WIN_TOKENS = 8;             // window tokens per work unit
constexpr int WIN_ROW = 272;              // padded bytes per staged bf16 row (conflict-free ldmatrix)
constexpr int WIN_V_OFF = WIN_TOKENS * WIN_ROW;

#ifndef WUSHKV_ABL
#define WUSHKV_ABL 0        // timing experiments only: 1 no value contraction, 2 no key contraction, 8 no page copies, 16 per-warp time stamps
#endif

// shift of the code field used by k-step / channel block idx (0..7) inside its 16-bit lane, after
// the optional whole-word shift: the fp16 value of the masked field is code * 2^(field_shift - 24)
template <int BITS>
__host__ __device__ constexpr int field_shift(int idx) {
    return BITS != 4 ? (idx < 5 ? 2 * idx : 2 * (idx - 5)) : 4 * (idx & 1);     // 3 bits: its 2-bit plane
}
// bf16x2 bit pattern of (2^e, 2^e)
__host__ __device__ constexpr unsigned bf16x2_pow2(int e) {
    return (static_cast<unsigned>(e + 127) << 7) | (static_cast<unsigned>(e + 127) << 23);
}

// How one sequence decomposes into work units (identical for all of its KV heads).
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

__device__ __forceinline__ unsigned smem_u32(const void* p) { return static_cast<unsigned>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void mbar_init(unsigned bar, unsigned count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(unsigned bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(unsigned bar, unsigned parity) {
    unsigned ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity), "r"(2000u) : "memory");      // may sleep up to ~2 us in hardware
    return ok != 0;
}
// Bounded wait: false if the phase did not complete within the limit (about a second of sleeping polls).
__device__ __forceinline__ bool mbar_wait_bounded(unsigned bar, unsigned parity, int limit) {
    for (int it = 0; it < limit; ++it)
        if (mbar_try_wait(bar, parity)) return true;
    return false;
}

__device__ __forceinline__ void bulk_copy_g2s(unsigned dst, const void* src, unsigned bytes, unsigned bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// The same copy for data that is read once per step (packed pages): evict-first in L2, so that the
// stream does not push out what the step's other kernels re-read (transforms, fragments, partials).
__device__ __forceinline__ unsigned long long l2_evict_first_policy() {
    unsigned long long pol;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}
__device__ __forceinline__ void bulk_copy_g2s_stream(unsigned dst, const void* src, unsigned bytes, unsigned bar, unsigned long long pol) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "l"(pol) : "memory");
}
__device__ __forceinline__ uint2 lds64(unsigned addr) {
    uint2 v;
    asm("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint4 lds128(unsigned addr) {
    uint4 v;
    asm("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void ldmatrix_x4(unsigned addr, unsigned& a, unsigned& b, unsigned& c, unsigned& d) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(addr));
}
__device__ __forceinline__ void ldmatrix_x4_trans(unsigned addr, unsigned& a, unsigned& b, unsigned& c, unsigned& d) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(addr));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// first MMA of a chain: D = A B (no accumulator registers to initialise)
__device__ __forceinline__ void mma_f16_zero(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// integer mma: A = 16 x 32 unsigned bytes (codes), B = 32 x 8 signed bytes (query digits), exact 32-bit sums
__device__ __forceinline__ void mma_u8s8(int (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_u8s8_zero(int (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(0));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ unsigned movmatrix_trans(unsigned a) {
    unsigned d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ unsigned pack_h2(float lo, float hi) {      // lo -> bits 0..15, hi -> bits 16..31, saturating
    unsigned d;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ unsigned pack_bf2(float lo, float hi) {
    unsigned d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ unsigned mul_bf2(unsigned a, unsigned b) {
    unsigned d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ float ex2(float x) {      // 2^x, -inf -> 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 h2f2(unsigned u) {     // both halves of an fp16x2 register as floats
    __half2 h;
    *reinterpret_cast<unsigned*>(&h) = u;
    return __half22float2(h);
}
__device__ __forceinline__ float bf16_round(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

// Field idx (0..7) of a code word as an fp16x2 A-fragment register.  `w` is the raw word, `ws` the
// same word shifted right so that the upper fields fall into the low bits of each 16-bit lane.
template <int BITS>
__device__ __forceinline__ unsigned field(unsigned w, unsigned ws, int idx) {
    if (BITS != 4) {
        constexpr unsigned M0 = 0x00030003u;
        return idx < 5 ? (w & (M0 << (2 * idx))) : (ws & (M0 << (2 * (idx - 5))));
    } else {
        constexpr unsigned M0 = 0x000F000Fu;
        return idx < 2 ? (w & (M0 << (4 * idx))) : (ws & (M0 << (4 * (idx - 2))));
    }
}
template <int BITS> __device__ __forceinline__ unsigned pre_shift(unsigned w) { return BITS != 4 ? (w >> 10) : (w >> 8); }

// Per-warp running softmax state of one (sequence, KV head).  MODE 0: one head per thread (head t,
// value and rounding-remainder columns).  MODE 1: two heads per thread (2t, 2t+1).
// o[i][.] accumulates channel block i in units of 2^(field_shift(i) - 24); l, z and o carry the
// common factor 2^LOG2_PV.  m is the reference of the partial, not necessarily its exact maximum.
template <int MODE>
struct WarpState {
    static constexpr int NH = MODE == 0 ? 1 : 2;
    float m[NH], mr[NH], l[NH], z[NH];
    float o[8][4];
    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int k = 0; k < NH; ++k) { m[k] = -INFINITY; mr[k] = 0.f; l[k] = 0.f; z[k] = 0.f; }
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    }
    // Make the running reference cover this unit's maxima to within MAX_SLACK.  mx holds each lane's
    // maximum over its own tokens; the warp-wide reduction is only needed when some lane is past the
    // slack, which after the first unit of a slice is rare.  mr is what the exponentials subtract.
    __device__ __forceinline__ void raise_max(float (&mx)[NH]) {
        bool grew = false;
#pragma unroll
        for (int k = 0; k < NH; ++k) grew |= mx[k] > m[k] + MAX_SLACK;      // reference -inf: any finite score
        if (__any_sync(FULL, grew)) {
            float scl[NH];
#pragma unroll
            for (int k = 0; k < NH; ++k) {
                mx[k] = fmaxf(mx[k], __shfl_xor_sync(FULL, mx[k], 4));       // over the 8 token rows of the fragment
                mx[k] = fmaxf(mx[k], __shfl_xor_sync(FULL, mx[k], 8));
                mx[k] = fmaxf(mx[k], __shfl_xor_sync(FULL, mx[k], 16));
                const float mnew = fmaxf(m[k], mx[k]);
                const float ref = (mnew == -INFINITY) ? 0.f : mnew;          // all masked so far: any finite reference works
                scl[k] = ex2(m[k] - ref);                                    // old reference -inf: state is all zero, factor 0
                l[k] *= scl[k]; z[k] *= scl[k];
                m[k] = mnew;
                mr[k] = ref - LOG2_PV;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                o[i][0] *= scl[0]; o[i][2] *= scl[0];
                o[i][1] *= scl[NH - 1]; o[i][3] *= scl[NH - 1];
            }
        }
    }
};

// Writes this warp's state of every query head of one (sequence, KV head) to global memory: a partial (max, sum, o[128]) in
// records PART_STRIDE floats apart, or, WHOLE, the head's outputs o / sum in rows of D floats.
template <int BITS, int MODE, bool WHOLE>
__device__ __forceinline__ void store_state(const WarpState<MODE>& st, float* dst0, int lane, int G) {
    const int g = lane >> 2, t = lane & 3;
    constexpr int NH = WarpState<MODE>::NH;
#pragma unroll
    for (int k = 0; k < NH; ++k) {
        float l = st.l[k], z = st.z[k];
        l += __shfl_xor_sync(FULL, l, 4);  z += __shfl_xor_sync(FULL, z, 4);
        l += __shfl_xor_sync(FULL, l, 8);  z += __shfl_xor_sync(FULL, z, 8);
        l += __shfl_xor_sync(FULL, l, 16); z += __shfl_xor_sync(FULL, z, 16);
        const int head = MODE == 0 ? t : 2 * t + k;
        if (head < G) {
            float* dst = dst0 + head * (WHOLE ? D : PART_STRIDE);
            if (!WHOLE) {
                if (g == 0) { dst[0] = st.m[k]; dst[1] = l; }
                dst += 4;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float osc = exp2f(static_cast<float>(24 - field_shift<BITS>(i)));
                float lo_ch, hi_ch;
                if (MODE == 0) {
                    lo_ch = (st.o[i][0] + st.o[i][1] * (1.f / LO_SCALE)) * osc + z;
                    hi_ch = (st.o[i][2] + st.o[i][3] * (1.f / LO_SCALE)) * osc + z;
                } else {
                    lo_ch = st.o[i][k] * osc + z;
                    hi_ch = st.o[i][2 + k] * osc + z;
                }
                if (WHOLE) {
                    lo_ch = l > 0.f ? lo_ch / l : 0.f;
                    hi_ch = l > 0.f ? hi_ch / l : 0.f;
                }
                dst[16 * i + g] = lo_ch;
                dst[16 * i + g + 8] = hi_ch;
            }
        }
    }
}

// One window unit: up to 8 bf16 tokens, key rows staged at shared-memory address rec_k, value rows at rec_v, WIN_ROW bytes apart;
// query(k) is the lane's k-th word of the (sequence, KV head)'s bf16 query fragments.
template <int BITS, int MODE, class Query>
__device__ __forceinline__ void window_unit(WarpState<MODE>& st, unsigned rec_k, unsigned rec_v, int n_valid, Query query, int lane) {
    constexpr int NH = WarpState<MODE>::NH;
    const int g = lane >> 2;
    const int r_eff = (lane & 7) < n_valid ? (lane & 7) : 0;      // rows beyond the valid ones alias row 0
    const int mat = lane >> 3;
    const unsigned frag_off = r_eff * WIN_ROW + ((mat >> 1) * 16 + (mat & 1) * 8) * 2;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int pass = 0; pass < (MODE == 0 ? 1 : 2); ++pass) {
#pragma unroll
        for (int s2 = 0; s2 < 4; ++s2) {
            const uint4 bq = query(pass * 128 + s2 * 32 + lane);
            unsigned k0, k1, k2, k3;                      // (step 2s2: ch lo, ch hi), (step 2s2+1: ch lo, ch hi)
            ldmatrix_x4(rec_k + frag_off + s2 * 64, k0, k1, k2, k3);
            mma_bf16(acc, k0, k0, k1, k1, bq.x, bq.y);    // token rows 8..15 alias rows 0..7
            mma_bf16(acc, k2, k2, k3, k3, bq.z, bq.w);
        }
    }
    const bool ok = g < n_valid;
    float sc[NH], mx[NH];
    if (MODE == 0) sc[0] = ok ? acc[0] + acc[1] : -INFINITY;
    else { sc[0] = ok ? acc[0] : -INFINITY; sc[NH - 1] = ok ? acc[1] : -INFINITY; }
#pragma unroll
    for (int k = 0; k < NH; ++k) mx[k] = sc[k];
    st.raise_max(mx);
    float p[NH];
#pragma unroll
    for (int k = 0; k < NH; ++k) { p[k] = ex2(sc[k] - st.mr[k]); st.l[k] += p[k]; }
#pragma unroll
    for (int pass = 0; pass < (MODE == 0 ? 1 : 2); ++pass) {
        unsigned pr;                                      // this token's probabilities in the score-fragment layout
        if (MODE == 0) pr = pack_bf2(p[0], (p[0] - bf16_round(p[0])) * LO_SCALE);   // value column, remainder column
        else if (pass == 0) pr = pack_bf2(p[0], p[NH - 1]);
        else pr = pack_bf2(p[0] - bf16_round(p[0]), p[NH - 1] - bf16_round(p[NH - 1]));
        const unsigned b01 = movmatrix_trans(pr);         // tokens 2t, 2t+1 of column g; tokens 8..15 get zero
#pragma unroll
        for (int i2 = 0; i2 < 4; ++i2) {
            unsigned v0, v1, v2, v3;                      // (block 2i2: ch lo, ch hi), (block 2i2+1: ch lo, ch hi)
            ldmatrix_x4_trans(rec_v + frag_off + i2 * 64, v0, v1, v2, v3);
            // fold the block's accumulator unit in: p * v * 2^(shift - 24)
            mma_bf16(st.o[2 * i2], v0, v1, v0, v1, mul_bf2(b01, bf16x2_pow2(field_shift<BITS>(2 * i2) - 24)), 0u);
            mma_bf16(st.o[2 * i2 + 1], v2, v3, v2, v3, mul_bf2(b01, bf16x2_pow2(field_shift<BITS>(2 * i2 + 1) - 24)), 0u);
        }
    }
}

// Scores of one packed page (64 tokens), key codes at shared-memory address rec_k, steps and offsets at rec_meta, divided by the
// heads' multipliers: sc[block][row g: heads..., row g + 8: heads...]; vmeta[block][row]: fp16x2 (Delta_v, x_min_v) of the rows.
// qf: integer B fragments of the four k-steps (MODE 1: of the high digits, qfl those of the low ones); gadd: see qscal.
template <int BITS, int MODE>
__device__ __forceinline__ void page_scores(unsigned rec_k, unsigned rec_meta, const unsigned (&qf)[4][2], const unsigned (&qfl)[MODE == 1 ? 4 : 1][2],
                                            const float (&gadd)[WarpState<MODE>::NH], float (&sc)[4][2 * WarpState<MODE>::NH], unsigned (&vmeta)[4][2], int lane) {
    constexpr int CB = code_block_bytes(BITS), NH = WarpState<MODE>::NH;
    const int g = lane >> 2;
#pragma unroll
    for (int bi = 0; bi < 4; ++bi) {
        // The four k-steps of a block take one field of every code byte each.  Fields at an even
        // position come out of the mask as the code itself, fields at an odd position as the code
        // times FS (4 at 2 bits, 16 at 4 bits): the two kinds are summed separately (X, Y) and
        // joined as FS * X + Y, which is FS times the exact integer dot product.
        constexpr int FS = BITS != 4 ? 4 : 16;
        unsigned a[4][4];             // [k-step][A register]
        if (BITS != 4) {
            const uint4 kw = lds128(rec_k + bi * CB + 16 * lane);      // (row g, ch half 0), (g+8, 0), (g, 1), (g+8, 1)
            const unsigned sx = kw.x >> 4, sy = kw.y >> 4, sz = kw.z >> 4, sw = kw.w >> 4;
            a[0][0] = kw.x & 0x03030303u; a[0][1] = kw.y & 0x03030303u; a[0][2] = kw.z & 0x03030303u; a[0][3] = kw.w & 0x03030303u;
            a[1][0] = kw.x & 0x0C0C0C0Cu; a[1][1] = kw.y & 0x0C0C0C0Cu; a[1][2] = kw.z & 0x0C0C0C0Cu; a[1][3] = kw.w & 0x0C0C0C0Cu;
            a[2][0] = sx & 0x03030303u;   a[2][1] = sy & 0x03030303u;   a[2][2] = sz & 0x03030303u;   a[2][3] = sw & 0x03030303u;
            a[3][0] = sx & 0x0C0C0C0Cu;   a[3][1] = sy & 0x0C0C0C0Cu;   a[3][2] = sz & 0x0C0C0C0Cu;   a[3][3] = sw & 0x0C0C0C0Cu;
        } else {
            const uint4 ka = lds128(rec_k + bi * CB + 16 * lane);          // k-steps 0 (low nibbles), 1 (high nibbles)
            const uint4 kb = lds128(rec_k + bi * CB + 512 + 16 * lane);    // k-steps 2, 3
            a[0][0] = ka.x & 0x0F0F0F0Fu; a[0][1] = ka.y & 0x0F0F0F0Fu; a[0][2] = ka.z & 0x0F0F0F0Fu; a[0][3] = ka.w & 0x0F0F0F0Fu;
            a[1][0] = ka.x & 0xF0F0F0F0u; a[1][1] = ka.y & 0xF0F0F0F0u; a[1][2] = ka.z & 0xF0F0F0F0u; a[1][3] = ka.w & 0xF0F0F0F0u;
            a[2][0] = kb.x & 0x0F0F0F0Fu; a[2][1] = kb.y & 0x0F0F0F0Fu; a[2][2] = kb.z & 0x0F0F0F0Fu; a[2][3] = kb.w & 0x0F0F0F0Fu;
            a[3][0] = kb.x & 0xF0F0F0F0u; a[3][1] = kb.y & 0xF0F0F0F0u; a[3][2] = kb.z & 0xF0F0F0F0u; a[3][3] = kb.w & 0xF0F0F0F0u;
        }
        int dot[4];                   // MODE 0: (row g, row g+8) x (high, low digit) joined below; MODE 1: rows x heads 2t, 2t+1
        if (WUSHKV_ABL & 2) { dot[0] = a[0][0] & 1; dot[1] = a[0][1] & 1; dot[2] = a[0][2] & 1; dot[3] = a[0][3] & 1; } else
        {
            int X[4], Y[4];
            mma_u8s8_zero(X, a[0][0], a[0][1], a[0][2], a[0][3], qf[0][0], qf[0][1]);
            mma_u8s8_zero(Y, a[1][0], a[1][1], a[1][2], a[1][3], qf[1][0], qf[1][1]);
            mma_u8s8(X, a[2][0], a[2][1], a[2][2], a[2][3], qf[2][0], qf[2][1]);
            mma_u8s8(Y, a[3][0], a[3][1], a[3][2], a[3][3], qf[3][0], qf[3][1]);
#pragma unroll
            for (int e = 0; e < 4; ++e) dot[e] = X[e] * FS + Y[e];
        }
        unsigned ah[4][4];            // 3 bits: A registers of the 1-bit plane (codes' high bits), one shift + mask each
        if (BITS == 3 && !(WUSHKV_ABL & 2)) {
            const uint2 kh = lds64(rec_k + k_hi_offset(3) + bi * 256 + 8 * lane);      // words of token rows g, g+8
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                ah[ks][0] = (kh.x >> (2 * ks)) & 0x01010101u;     ah[ks][1] = (kh.y >> (2 * ks)) & 0x01010101u;
                ah[ks][2] = (kh.x >> (2 * ks + 1)) & 0x01010101u; ah[ks][3] = (kh.y >> (2 * ks + 1)) & 0x01010101u;
            }
            int Z[4];
            mma_u8s8_zero(Z, ah[0][0], ah[0][1], ah[0][2], ah[0][3], qf[0][0], qf[0][1]);
#pragma unroll
            for (int ks = 1; ks < 4; ++ks) mma_u8s8(Z, ah[ks][0], ah[ks][1], ah[ks][2], ah[ks][3], qf[ks][0], qf[ks][1]);
#pragma unroll
            for (int e = 0; e < 4; ++e) dot[e] += 4 * FS * Z[e];       // code = low plane + 4 x high bit
        }
        if (MODE == 1 && !(WUSHKV_ABL & 2)) {              // second fragment set: the low digits of the eight heads
            int X[4], Y[4];
            mma_u8s8_zero(X, a[0][0], a[0][1], a[0][2], a[0][3], qfl[0][0], qfl[0][1]);
            mma_u8s8_zero(Y, a[1][0], a[1][1], a[1][2], a[1][3], qfl[1][0], qfl[1][1]);
            mma_u8s8(X, a[2][0], a[2][1], a[2][2], a[2][3], qfl[2][0], qfl[2][1]);
            mma_u8s8(Y, a[3][0], a[3][1], a[3][2], a[3][3], qfl[3][0], qfl[3][1]);
            if (BITS == 3) {
                int Z[4];
                mma_u8s8_zero(Z, ah[0][0], ah[0][1], ah[0][2], ah[0][3], qfl[0][0], qfl[0][1]);
#pragma unroll
                for (int ks = 1; ks < 4; ++ks) mma_u8s8(Z, ah[ks][0], ah[ks][1], ah[ks][2], ah[ks][3], qfl[ks][0], qfl[ks][1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) Y[e] += 4 * FS * Z[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) dot[e] = dot[e] * 256 + (X[e] * FS + Y[e]);
        }
        const uint4 mt = lds128(rec_meta + 128 * bi + 16 * g);   // rows g (x,y) and g+8 (z,w)
        const float2 km_a = h2f2(mt.x), km_b = h2f2(mt.z);
        const float kd0 = km_a.x, km0 = km_a.y, kd1 = km_b.x, km1 = km_b.y;
        vmeta[bi][0] = mt.y; vmeta[bi][1] = mt.w;
        if (MODE == 0) {
            const float d0 = static_cast<float>(dot[0] * 256 + dot[1]), d1 = static_cast<float>(dot[2] * 256 + dot[3]);
            sc[bi][0] = fmaf(km0, gadd[0], d0 * kd0);
            sc[bi][NH] = fmaf(km1, gadd[0], d1 * kd1);
        } else {
            sc[bi][0] = fmaf(km0, gadd[0], static_cast<float>(dot[0]) * kd0);
            sc[bi][NH - 1] = fmaf(km0, gadd[NH - 1], static_cast<float>(dot[1]) * kd0);
            sc[bi][NH] = fmaf(km1, gadd[0], static_cast<float>(dot[2]) * kd1);
            sc[bi][2 * NH - 1] = fmaf(km1, gadd[NH - 1], static_cast<float>(dot[3]) * kd1);
        }
    }
}

// The page's probabilities and its values' contribution (value codes at shared-memory address rec_v); fmul: the heads' multipliers.
// Probability times value step is rounded to one fp16 (half a step: 2^-11 of it, an eighth of what an output in bf16 loses, and the
// tokens' errors average out), so that one MMA serves a block; the sums l and z and the accumulators stay in 32 bits.  Window
// probabilities, whose values are not quantized, are taken as two bf16 terms.
template <int BITS, int MODE>
__device__ __forceinline__ void page_values(WarpState<MODE>& st, unsigned rec_v, const float (&sc)[4][2 * WarpState<MODE>::NH], const unsigned (&vmeta)[4][2],
                                            const float (&fmul)[WarpState<MODE>::NH], int lane) {
    constexpr int CB = code_block_bytes(BITS), NH = WarpState<MODE>::NH;
#pragma unroll
    for (int bi = 0; bi < 4; ++bi) {
        const float2 vm_a = h2f2(vmeta[bi][0]), vm_b = h2f2(vmeta[bi][1]);
        const float vd0 = vm_a.x, vn0 = vm_a.y, vd1 = vm_b.x, vn1 = vm_b.y;
        unsigned r0, r1;
        if (MODE == 0) {
            const float p0 = ex2(fmaf(sc[bi][0], fmul[0], -st.mr[0])), p1 = ex2(fmaf(sc[bi][NH], fmul[0], -st.mr[0]));
            st.l[0] += p0 + p1;
            st.z[0] = fmaf(p0, vn0, fmaf(p1, vn1, st.z[0]));
            r0 = pack_h2(p0 * vd0, 0.f);
            r1 = pack_h2(p1 * vd1, 0.f);
        } else {
            const float p00 = ex2(fmaf(sc[bi][0], fmul[0], -st.mr[0])), p01 = ex2(fmaf(sc[bi][NH - 1], fmul[NH - 1], -st.mr[NH - 1]));
            const float p10 = ex2(fmaf(sc[bi][NH], fmul[0], -st.mr[0])), p11 = ex2(fmaf(sc[bi][2 * NH - 1], fmul[NH - 1], -st.mr[NH - 1]));
            st.l[0] += p00 + p10; st.l[NH - 1] += p01 + p11;
            st.z[0] = fmaf(p00, vn0, fmaf(p10, vn1, st.z[0]));
            st.z[NH - 1] = fmaf(p01, vn0, fmaf(p11, vn1, st.z[NH - 1]));
            r0 = pack_h2(p00 * vd0, p01 * vd0);
            r1 = pack_h2(p10 * vd1, p11 * vd1);
        }
        const unsigned b01 = movmatrix_trans(r0), b23 = movmatrix_trans(r1);
        if (WUSHKV_ABL & 1) { st.o[bi][0] += __uint_as_float(b01 ^ b23); } else
        if (BITS != 4) {
            const uint4 vw = lds128(rec_v + bi * CB + 16 * lane);
            const unsigned sx = pre_shift<2>(vw.x), sy = pre_shift<2>(vw.y), sz = pre_shift<2>(vw.z), sw = pre_shift<2>(vw.w);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                mma_f16(st.o[i], field<2>(vw.x, sx, i), field<2>(vw.y, sy, i), field<2>(vw.z, sz, i), field<2>(vw.w, sw, i), b01, b23);
            if (BITS == 3) {
                // 1-bit plane: words of token halves ps = 0, 1; one of five shifts of a word puts the bit of
                // (row half, channel block i) two bits above the low plane's field of block i, so that it reads
                // as 4 x (high bit) in that field's unit and lands in the same accumulator
                const uint2 vh = lds64(rec_v + v_hi_offset(3) - v_codes_offset(3) + bi * 256 + 8 * lane);
                const unsigned xv[5] = {vh.x, vh.x << 1, vh.x >> 9, vh.x >> 10, vh.x << 6};
                const unsigned yv[5] = {vh.y, vh.y << 1, vh.y >> 9, vh.y >> 10, vh.y << 6};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const unsigned m = 0x00010001u << v1_target(i);
                    const int r0 = i < 5 ? 0 : 2, r1 = i < 5 ? 1 : (i < 7 ? 3 : 4);
                    mma_f16(st.o[i], xv[r0] & m, xv[r1] & m, yv[r0] & m, yv[r1] & m, b01, b23);
                }
            }
        } else {
            const uint4 va = lds128(rec_v + bi * CB + 16 * lane);         // tokens 2t,2t+1
            const uint4 vb = lds128(rec_v + bi * CB + 512 + 16 * lane);   // tokens 2t+8,2t+9
            const unsigned a0s = pre_shift<4>(va.x), a1s = pre_shift<4>(va.y), a2s = pre_shift<4>(va.z), a3s = pre_shift<4>(va.w);
            const unsigned b0s = pre_shift<4>(vb.x), b1s = pre_shift<4>(vb.y), b2s = pre_shift<4>(vb.z), b3s = pre_shift<4>(vb.w);
#pragma unroll
            for (int k = 0; k < 4; ++k)     // channel blocks 0..3: words (rsel, j=0)
                mma_f16(st.o[k], field<4>(va.x, a0s, k), field<4>(va.z, a2s, k), field<4>(vb.x, b0s, k), field<4>(vb.z, b2s, k), b01, b23);
#pragma unroll
            for (int k = 0; k < 4; ++k)     // channel blocks 4..7: words (rsel, j=1)
                mma_f16(st.o[4 + k], field<4>(va.y, a1s, k), field<4>(va.w, a3s, k), field<4>(vb.y, b1s, k), field<4>(vb.w, b3s, k), b01, b23);
        }
    }
}

// Merge of partial states (max, sum, o) of one query head by one warp: lane L holds channels 4L .. 4L+3.  The tail of the
// kernel is a chain of latencies, so the rows of a batch and their maxima and sums are all requested together.
constexpr int MERGE_BATCH = 8;
struct MergedState {
    float m, l;
    float4 o;
    __device__ __forceinline__ void reset() { m = -INFINITY; l = 0.f; o = make_float4(0.f, 0.f, 0.f, 0.f); }
    // Adds n >= 1 partials; record(k) is the address of partial k.  The loads are unconditional (past the end the last record
    // again): under a condition each would wait for the one before.
    template <bool GLOBAL, class Record>
    __device__ __forceinline__ void add(int n, int lane, Record record) {
        constexpr int NB = GLOBAL ? 2 * MERGE_BATCH : MERGE_BATCH;
        for (int k = 0; k < n; k += NB) {
            float4 v[NB];
            float2 ml[NB];
            float mn = m;
#pragma unroll
            for (int e = 0; e < NB; ++e) {
                const float* rec = record(min(k + e, n - 1));
                const float2* pm = reinterpret_cast<const float2*>(rec);
                const float4* po = reinterpret_cast<const float4*>(rec + 4) + lane;
                ml[e] = GLOBAL ? __ldcg(pm) : *pm;               // GLOBAL: another CTA's, never through the L1
                v[e] = GLOBAL ? __ldcg(po) : *po;
            }
#pragma unroll
            for (int e = 0; e < NB; ++e) if (k + e >= n) ml[e].x = -INFINITY;
#pragma unroll
            for (int e = 0; e < NB; ++e) mn = fmaxf(mn, ml[e].x);
            if (mn == -INFINITY) continue;                       // nothing but empty partials so far
            const float keep = ex2(m - mn);
            l *= keep;
            o.x *= keep; o.y *= keep; o.z *= keep; o.w *= keep;
            m = mn;
#pragma unroll
            for (int e = 0; e < NB; ++e) {
                const float f = ex2(ml[e].x - mn);                   // an empty partial holds zeros
                l = fmaf(ml[e].y, f, l);
                o.x = fmaf(v[e].x, f, o.x); o.y = fmaf(v[e].y, f, o.y);
                o.z = fmaf(v[e].z, f, o.z); o.w = fmaf(v[e].w, f, o.w);
            }
        }
    }
    __device__ __forceinline__ void store(float* rec, int lane) const {
        if (lane == 0) *reinterpret_cast<float2*>(rec) = make_float2(m, l);
        reinterpret_cast<float4*>(rec + 4)[lane] = o;
    }
    __device__ __forceinline__ void finish(float* out, int lane) const {
        const bool any = l > 0.f;
        reinterpret_cast<float4*>(out)[lane] = any ? make_float4(o.x / l, o.y / l, o.z / l, o.w / l) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    // rounded to bf16 (sparse attention: what a selection of pages leaves out is larger than that rounding)
    __device__ __forceinline__ void finish(unsigned short* out, int lane) const {
        const float r = l > 0.f ? 1.f / l : 0.f;
        reinterpret_cast<uint2*>(out)[lane] = make_uint2(pack_bf2(o.x * r, o.y * r), pack_bf2(o.z * r, o.w * r));
    }
};

}  // namespace wushkv
