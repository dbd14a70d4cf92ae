// Management of the cache's pages: reserving, forking, releasing and compacting the rows of a page table, and the copies of
// packed pages and bf16 windows that go with them.
//
// The bookkeeping is one count per page, refs[p] = number of table entries that name page p; a page is free exactly when its
// count is 0.  There is no list of free pages to keep consistent and no order of requests in it: the free pages of a call are
// the zeros of refs, handed out lowest first, so that results depend on the state and the arguments alone.  Counts change by
// integer atomics, whose order does not show.
//
// reserve and compact need ranks over the whole pool (the k-th free page).  They run as ONE cluster of eight CTAs: every CTA
// counts its eighth of the pool, the counts meet at a cluster barrier, and a second walk writes each page's rank, so that a
// call is one launch.  What bounds them is latency (the barriers and the dependent loads table entry -> count), not the 4 bytes
// per page and entry that they read: 7.2 us to compact 4700 live pages of 64 sequences into the room of 32 that ended, 8.6 us to
// reserve for 12 forked sequences.  (The first form took 7.9 and 8.1 us; one CTA of 1024 threads without cluster barriers 14.0 and
// 9.8 in its place.)
//
// The copies move whole records with 16-byte loads and stores, a warp per record with all of its loads in flight; they are
// bound by HBM.
#include <cooperative_groups.h>

#include <algorithm>

#include "host_common.h"

namespace wushkv {

namespace cg = cooperative_groups;

constexpr int POOL_CTAS = 8;                 // of the one cluster
constexpr int POOL_THREADS = 512;
constexpr int POOL_WARPS = POOL_THREADS / 32;

struct PoolView {
    int n_slots, max_pages, n_pages;
    int* table;
    int* refs;
    int* dev_status;
};

// The page that an entry names: itself, or the page of a locked entry (see wushkv_pages_reserve); -1: none.
__device__ __forceinline__ int entry_page(int e) { return e >= -1 ? e : -2 - e; }
__device__ __forceinline__ int locked_entry(int page) { return -2 - page; }

// Gives one reference back.
__device__ __forceinline__ void drop_page(const PoolView& v, int entry) {
    const int page = entry_page(entry);
    if (page < 0) return;
    if (page >= v.n_pages) { atomicOr(v.dev_status, WUSHKV_DEV_BAD_PAGE_ID); return; }
    if (atomicSub(v.refs + page, 1) <= 0) {
        atomicAdd(v.refs + page, 1);
        atomicOr(v.dev_status, WUSHKV_DEV_BAD_REFS);
    }
}

// ---- fork, release ------------------------------------------------------------------------------------------------------
// A CTA per sequence, a thread per table entry.  Entries are exchanged, not overwritten, so that the counts stay right even
// when a row is named twice in a call.
__global__ void __launch_bounds__(256) pages_fork_kernel(PoolView v, const int* src_slot, const int* dst_slot, const int* src_len) {
    pdl_wait();
    pdl_launch_dependents();
    const int k = blockIdx.x;
    const int src = src_slot[k], dst = dst_slot[k], len = src_len[k];
    if (src < 0 || src >= v.n_slots || dst < 0 || dst >= v.n_slots) {
        if (threadIdx.x == 0) atomicOr(v.dev_status, WUSHKV_DEV_BAD_SLOT);
        return;
    }
    int used = len > 0 ? (len - 1) / PAGE_TOKENS + 1 : 0;
    if (used > v.max_pages) {
        if (threadIdx.x == 0) atomicOr(v.dev_status, WUSHKV_DEV_PAGE_TABLE_FULL);
        used = v.max_pages;
    }
    const int* from = v.table + static_cast<long long>(src) * v.max_pages;
    int* to = v.table + static_cast<long long>(dst) * v.max_pages;
    for (int i = threadIdx.x; i < v.max_pages; i += blockDim.x) {
        int page = -1;
        if (i < used) {
            page = entry_page(from[i]);
            if (page < 0 || page >= v.n_pages) { page = -1; atomicOr(v.dev_status, WUSHKV_DEV_BAD_PAGE_ID); }
        }
        if (page >= 0) atomicAdd(v.refs + page, 1);
        drop_page(v, atomicExch(to + i, page));
    }
}

__global__ void __launch_bounds__(256) pages_release_kernel(PoolView v, const int* slot, const int* keep_len) {
    pdl_wait();
    pdl_launch_dependents();
    const int k = blockIdx.x, s = slot[k];
    if (s < 0 || s >= v.n_slots) {
        if (threadIdx.x == 0) atomicOr(v.dev_status, WUSHKV_DEV_BAD_SLOT);
        return;
    }
    const int keep = keep_len ? keep_len[k] : 0;
    const int first = keep > 0 ? (keep - 1) / PAGE_TOKENS + 1 : 0;
    int* row = v.table + static_cast<long long>(s) * v.max_pages;
    for (int i = first + threadIdx.x; i < v.max_pages; i += blockDim.x) drop_page(v, atomicExch(row + i, -1));
}

// The cluster barriers order all memory accesses, global ones too: what a CTA has written before one is what the others read after it.
// ---- walks over the pool --------------------------------------------------------------------------------------------------
// Exclusive prefix sum over the CTA of one number per thread; *total: their sum.
__device__ __forceinline__ int block_prefix(int x, int* total, int* scratch) {      // scratch: POOL_WARPS ints
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    __syncthreads();                         // the scratch's previous readers
    if (lane == 31) scratch[warp] = incl;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < POOL_WARPS; ++w) {
        const int y = scratch[w];
        if (w < warp) before += y;
        all += y;
    }
    *total = all;
    return before + incl - x;
}

// This CTA's part of the pool: [lo, hi), a multiple of four pages from its beginning.
__device__ __forceinline__ void pool_part(int n_pages, int rank, int& lo, int& hi) {
    const long long per = ((static_cast<long long>(n_pages) + 4 * POOL_CTAS - 1) / (4 * POOL_CTAS)) * 4;
    lo = static_cast<int>(min(per * rank, static_cast<long long>(n_pages)));
    hi = static_cast<int>(min(per * (rank + 1), static_cast<long long>(n_pages)));
}

// Number of pages in [lo, hi) that are in use; every thread of the CTA gets it.
__device__ __forceinline__ int count_live(const int* refs, int lo, int hi, int* scratch) {
    int n = 0;
#pragma unroll 8
    for (int p = lo + threadIdx.x; p < hi; p += POOL_THREADS) n += refs[p] > 0;
    int total;
    block_prefix(n, &total, scratch);
    return total;
}

// ---- reserve ---------------------------------------------------------------------------------------------------------------
struct ReserveParams {
    PoolView v;
    int batch;
    const int* slot;
    const int* seq_len;
    const int* cu_new;
    int* copy_src;
    int* copy_dst;
    int* n_copies;
    int* need;           // [batch]: new pages of the sequence (~ of them if it also has shared pages to be written as a whole), later their first rank
    int* shared;         // [batch]: its last page if that is shared and about to be written, else -1; later 1 + the index of its copy, or 0
    int* list;           // [n_pages]: the free pages, lowest first, as many as are needed
};

// What sequence b asks for: its first and last page index to be written, whether the first is partly filled; false: nothing.
// beyond: nothing, because its tokens pass the table's end (slot, first and tail are set).
struct Request { int slot, first, last; bool tail, beyond; };
__device__ __forceinline__ bool request_of(const ReserveParams& P, int b, Request& r, bool report) {
    const int s0 = P.seq_len[b], n = P.cu_new[b + 1] - P.cu_new[b];
    r.slot = P.slot[b];
    r.beyond = false;
    if (r.slot < 0 || r.slot >= P.v.n_slots) { if (report) atomicOr(P.v.dev_status, WUSHKV_DEV_BAD_SLOT); return false; }
    if (n <= 0 || s0 < 0) return false;
    r.first = s0 / PAGE_TOKENS;
    r.tail = s0 % PAGE_TOKENS != 0;
    const long long last = (static_cast<long long>(s0) + n - 1) / PAGE_TOKENS;
    if (last >= P.v.max_pages) {
        if (report) atomicOr(P.v.dev_status, WUSHKV_DEV_PAGE_TABLE_FULL);
        r.beyond = true;
        return false;
    }
    r.last = static_cast<int>(last);
    return true;
}

// Calls with shared pages that are written from their first row on (by sequences that went back without a release), by one CTA: they
// are rare, and the table is walked once per step.  Of k holders of a page that are all here the last one keeps it, the others leave
// it: with every entry that is to be written taken off its page's count, the pages that are left to nobody are those whose holders
// are all here, and their keeper is the last sequence that was seen.  Leaves need and shared as the first step does, with ~ taken off,
// the counts as they were, and a whole page that is to be left as a locked entry, one that is kept as an unlocked one.  (12 sequences
// that write a whole shared page each: 12.3 us for the call, with partly filled ones 8.6.)
__device__ __noinline__ void settle_shared_pages(const ReserveParams& P, int lane, int warp) {
    const PoolView& v = P.v;
    int* last = P.list;                                  // [n_pages]
    for (int step = 0; step < 4; ++step) {
        for (int b = warp; b < P.batch; b += POOL_WARPS) {
            Request r;
            int need = 0, shared = -1;
            if (request_of(P, b, r, false)) {
                int* row = v.table + static_cast<long long>(r.slot) * v.max_pages;
                for (int i = r.first + lane; i <= r.last; i += 32) {
                    const int e = row[i], page = entry_page(e);
                    if (e == -1) { need += step == 2; continue; }
                    if (page >= v.n_pages) continue;
                    if (step == 0) last[page] = -1;
                    else if (step == 1) { atomicSub(v.refs + page, 1); atomicMax(last + page, b); }
                    else if (step == 3) atomicAdd(v.refs + page, 1);
                    else {
                        const bool keep = __ldcg(v.refs + page) <= 0 && __ldcg(last + page) == b;
                        if (i == r.first && r.tail) shared = keep ? -1 : page;
                        else { row[i] = keep ? page : locked_entry(page); need += !keep; }
                    }
                }
            }
            if (step == 2) {
                need = __reduce_add_sync(0xffffffffu, need);
                shared = __shfl_sync(0xffffffffu, shared, 0);
                if (lane == 0) { P.need[b] = need; P.shared[b] = shared; }
            }
        }
        __syncthreads();
    }
}

__global__ void __cluster_dims__(POOL_CTAS, 1, 1) __launch_bounds__(POOL_THREADS) pages_reserve_kernel(const __grid_constant__ ReserveParams P) {
    pdl_wait();
    pdl_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const PoolView& v = P.v;
    const int rank = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __shared__ int scratch[POOL_WARPS];
    __shared__ int tile[POOL_THREADS];
    __shared__ int free_s, copies_s;                     // free pages of this CTA's part; CTA 0: copies asked for
    __shared__ long long total_s;                        // CTA 0: pages asked for
    __shared__ int settled_s;                            // CTA 0: whether shared pages are left that are written as a whole

    // 1. what every sequence needs: a warp per sequence, a lane per page index
    for (int b = rank * POOL_WARPS + warp; b < P.batch; b += POOL_CTAS * POOL_WARPS) {
        Request r;
        int missing = 0, shared = -1;
        bool whole = false;                              // an existing page that others name too, all of whose tokens are new
        if (request_of(P, b, r, lane == 0)) {
            const int* row = v.table + static_cast<long long>(r.slot) * v.max_pages;
            for (int i = r.first + lane; i <= r.last; i += 32) {
                const int e = row[i];
                if (e == -1) {
                    ++missing;
                    if (i == r.first && r.tail) atomicOr(v.dev_status, WUSHKV_DEV_BAD_PAGE_ID);      // its tokens are lost
                } else {
                    const int page = entry_page(e);
                    const bool tail = i == r.first && r.tail;
                    if (page >= v.n_pages) { if (tail) atomicOr(v.dev_status, WUSHKV_DEV_BAD_PAGE_ID); }
                    else if (v.refs[page] > 1) { if (tail) shared = page; else whole = true; }
                }
            }
            missing = __reduce_add_sync(0xffffffffu, missing);
            shared = __shfl_sync(0xffffffffu, shared, 0);
            whole = __any_sync(0xffffffffu, whole);
        } else if (r.beyond && r.tail && r.first < v.max_pages && lane == 0) {
            // The append refuses the sequence, and what follows an append (the page's bounds up to this sequence's length) must not
            // reach a page that others read further: locked, as where the pool is empty.
            int* entry = v.table + static_cast<long long>(r.slot) * v.max_pages + r.first;
            const int page = entry_page(*entry);
            if (page >= 0 && page < v.n_pages && v.refs[page] > 1) *entry = locked_entry(page);
        }
        if (lane == 0) { P.need[b] = whole ? ~missing : missing; P.shared[b] = shared; }
    }
    int lo, hi;
    pool_part(v.n_pages, rank, lo, hi);
    const int live = count_live(v.refs, lo, hi, scratch);
    if (threadIdx.x == 0) free_s = hi - lo - live;
    cluster.sync();

    // 2. CTA 0: which shared pages are copied, and the first rank of every sequence.  The sequences are taken in order: one that
    // finds its page still shared copies it and leaves it, so of k holders of a page that are all here the last one keeps it.  Where
    // shared pages are written as a whole, too, the same is found out for all pages together.
    if (rank == 0) {
        long long pages;
        int copies;
        bool settled = false;
        for (;; settled = true) {
            bool whole = false;
            pages = 0;
            copies = 0;
            for (int base = 0; base < P.batch; base += POOL_THREADS) {
                const int b = base + threadIdx.x;
                int need = 0, shared = -1;
                if (b < P.batch) { need = P.need[b]; shared = P.shared[b]; }
                if (need < 0) { need = ~need; whole = true; }
                bool copy = settled && shared >= 0;
                if (!settled && __syncthreads_or(shared >= 0)) {
                    int earlier = 0;
                    for (int t0 = 0; t0 <= base; t0 += POOL_THREADS) {
                        __syncthreads();
                        // the entries of earlier tiles say in `tile` only whether they name the same page, so the list must not be rewritten yet
                        const int o = t0 + threadIdx.x;
                        tile[threadIdx.x] = o < P.batch ? (t0 == base ? shared : P.list[o]) : -1;
                        __syncthreads();
                        const int n = t0 == base ? static_cast<int>(threadIdx.x) : POOL_THREADS;
                        if (shared >= 0)
                            for (int k = 0; k < n; ++k) earlier += tile[k] == shared;
                    }
                    copy = shared >= 0 && v.refs[shared] - earlier > 1;
                }
                if (b < P.batch) P.list[b] = shared;         // kept for the tiles to come (the list proper is written after the next barrier)
                int total_p, total_c;
                const int at = block_prefix(need + (copy ? 1 : 0), &total_p, scratch);
                const int at_copy = block_prefix(copy ? 1 : 0, &total_c, scratch);
                if (b < P.batch) { P.need[b] = static_cast<int>(pages) + at; P.shared[b] = copy ? 1 + copies + at_copy : 0; }
                pages += total_p;
                copies += total_c;
            }
            if (settled || !__syncthreads_or(whole)) break;
            settle_shared_pages(P, lane, warp);
        }
        if (threadIdx.x == 0) { total_s = pages; copies_s = copies; settled_s = settled; }
    }
    cluster.sync();
    const long long wanted = *cluster.map_shared_rank(&total_s, 0);
    const int copies = *cluster.map_shared_rank(&copies_s, 0);
    const bool settled = *cluster.map_shared_rank(&settled_s, 0) != 0;
    int free_before = 0, free_all = 0;
    for (int r = 0; r < POOL_CTAS; ++r) {
        const int f = *cluster.map_shared_rank(&free_s, r);
        if (r < rank) free_before += f;
        free_all += f;
    }
    const bool granted = wanted <= free_all;

    // 3. the lowest free pages
    if (granted) {
        for (int t0 = lo, at = free_before; t0 < hi && at < wanted; t0 += 4 * POOL_THREADS) {
            const int p = t0 + 4 * static_cast<int>(threadIdx.x);
            bool free_here[4];
            int n = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) { free_here[e] = p + e < hi && v.refs[p + e] <= 0; n += free_here[e]; }
            int total;
            int k = at + block_prefix(n, &total, scratch);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (free_here[e]) { if (k < wanted) P.list[k] = p + e; ++k; }
            at += total;
        }
    }
    cluster.sync();

    // 4. hand them out
    for (int b = rank * POOL_WARPS + warp; b < P.batch; b += POOL_CTAS * POOL_WARPS) {
        Request r;
        if (!request_of(P, b, r, false)) continue;
        int* row = v.table + static_cast<long long>(r.slot) * v.max_pages;
        int at = P.need[b];
        if (r.tail) {
            const int e = row[r.first], page = entry_page(e), copy = P.shared[b];
            if (page >= 0 && page < v.n_pages) {
                if (!granted) {
                    // the page stays shared: the entry is locked, so that an append of this sequence is refused and cannot write into it
                    if (lane == 0) row[r.first] = v.refs[page] > 1 ? locked_entry(page) : page;
                } else if (copy > 0) {
                    if (lane == 0) {
                        const int own = P.list[at];
                        row[r.first] = own;
                        v.refs[own] = 1;
                        atomicSub(v.refs + page, 1);
                        P.copy_src[copy - 1] = page;
                        P.copy_dst[copy - 1] = own;
                    }
                    ++at;
                } else if (lane == 0 && e != page) {
                    row[r.first] = page;                 // locked before, and its only holder now
                }
            }
        }
        for (int i0 = r.first; i0 <= r.last; i0 += 32) {
            const int i = i0 + lane;
            const int e = i <= r.last ? row[i] : 0;
            const bool here = i <= r.last && !(r.tail && i == r.first && e != -1);
            const int page = here && e != -1 ? entry_page(e) : v.n_pages;
            const bool known = page < v.n_pages;
            if (!granted) {                              // shared pages stay shared here as well
                if (known) row[i] = v.refs[page] > 1 ? locked_entry(page) : page;
                continue;
            }
            const bool leave = known && settled && e < -1, wants = leave || (here && e == -1);
            const unsigned m = __ballot_sync(0xffffffffu, wants);
            const int k = at + __popc(m & ((1u << lane) - 1u));
            if (wants && k < wanted) {                   // (always, unless a slot is named twice)
                const int own = P.list[k];
                row[i] = own;
                v.refs[own] = 1;
                if (leave) atomicSub(v.refs + page, 1);
            } else if (known && e < -1) row[i] = page;   // locked before, and its only holder now
            at += __popc(m);
        }
    }
    const int written = granted ? copies : 0;
    for (int k = written + rank * POOL_THREADS + threadIdx.x; k < P.batch; k += POOL_CTAS * POOL_THREADS) { P.copy_src[k] = -1; P.copy_dst[k] = -1; }
    if (rank == 0 && threadIdx.x == 0) {
        *P.n_copies = written;
        if (!granted) atomicOr(v.dev_status, WUSHKV_DEV_POOL_EMPTY);
    }
}

// ---- compact ---------------------------------------------------------------------------------------------------------------
struct CompactParams {
    PoolView v;
    int* copy_src;
    int* copy_dst;
    int* n_copies;
    int* n_live;
    int* holes;          // [n_pages]: free pages below the number of live ones, lowest first
    int* movers;         // [n_pages]: live pages from that number on, highest first
    int* moved;          // [n_pages]: place of a live page, -1 of a page that was free
    int n_list;          // capacity of the copy list
};

__global__ void __cluster_dims__(POOL_CTAS, 1, 1) __launch_bounds__(POOL_THREADS) pages_compact_kernel(CompactParams P) {
    pdl_wait();
    pdl_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const PoolView& v = P.v;
    const int rank = blockIdx.x;
    __shared__ int scratch[POOL_WARPS];
    __shared__ int live_s, holes_s;
    int lo, hi;
    pool_part(v.n_pages, rank, lo, hi);
    const int live_here = count_live(v.refs, lo, hi, scratch);
    if (threadIdx.x == 0) live_s = live_here;
    cluster.sync();
    int before = 0, live = 0;
    for (int r = 0; r < POOL_CTAS; ++r) {
        const int n = *cluster.map_shared_rank(&live_s, r);
        if (r < rank) before += n;
        live += n;
    }
    // A free page p < live is hole number p - (live pages below p); a live page p >= live is mover number live - 1 - (live pages below p)
    // counted from the last.  There are as many of one as of the other.
    int my_holes = 0;
    for (int t0 = lo; t0 < hi; t0 += 4 * POOL_THREADS) {
        const int p = t0 + 4 * static_cast<int>(threadIdx.x);
        bool used[4];
        int n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) { used[e] = p + e < hi && v.refs[p + e] > 0; n += used[e]; }
        int total;
        int below = before + block_prefix(n, &total, scratch);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (p + e < hi) {
                if (p + e < live) { if (!used[e]) { P.holes[p + e - below] = p + e; ++my_holes; } }
                else if (used[e]) P.movers[live - 1 - below] = p + e;
                P.moved[p + e] = used[e] ? p + e : -1;      // (of a mover written again behind the barrier)
            }
            below += used[e];
        }
        before += total;
    }
    int holes_here;
    block_prefix(my_holes, &holes_here, scratch);
    if (threadIdx.x == 0) holes_s = holes_here;
    cluster.sync();
    int n_moves = 0;
    for (int r = 0; r < POOL_CTAS; ++r) n_moves += *cluster.map_shared_rank(&holes_s, r);
    for (int k = rank * POOL_THREADS + threadIdx.x; k < P.n_list; k += POOL_CTAS * POOL_THREADS) {
        int src = -1, dst = -1;
        if (k < n_moves) {
            src = P.movers[n_moves - 1 - k];
            dst = P.holes[k];
            P.moved[src] = dst;
            v.refs[dst] = v.refs[src];
            v.refs[src] = 0;
        }
        P.copy_src[k] = src;
        P.copy_dst[k] = dst;
    }
    if (rank == 0 && threadIdx.x == 0) { *P.n_copies = n_moves; *P.n_live = live; }
    cluster.sync();
    const long long entries = static_cast<long long>(v.n_slots) * v.max_pages;
#pragma unroll 4
    for (long long i = rank * POOL_THREADS + threadIdx.x; i < entries; i += POOL_CTAS * POOL_THREADS) {
        const int e = v.table[i], page = entry_page(e);
        if (page < 0) continue;
        if (page >= v.n_pages) { atomicOr(v.dev_status, WUSHKV_DEV_BAD_PAGE_ID); continue; }
        const int to = P.moved[page];
        if (to < 0) { atomicOr(v.dev_status, WUSHKV_DEV_BAD_REFS); v.table[i] = -1; continue; }        // an entry that the counts do not know
        if (to != page) v.table[i] = e >= 0 ? to : locked_entry(to);
    }
}

// ---- copies of pages and windows ----------------------------------------------------------------------------------------
struct CopyPagesParams {
    unsigned char* pages;
    signed char* bounds;         // [n_pages][n_kv][2][D], or nullptr
    signed char* exponents;      // [n_pages][n_kv]
    int* dev_status;
    const int* src;
    const int* dst;
    const int* n_copies;
    long long n_pages;
    int n_kv, max_copies;
};

template <int BITS>
__global__ void __launch_bounds__(256) copy_pages_kernel(CopyPagesParams P) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int REC = record_bytes(BITS), VECS = REC / 16, PER_LANE = (VECS + 31) / 32;
    static_assert(REC % 16 == 0, "records are copied in 16-byte vectors");
    const int lane = threadIdx.x & 31;
    const long long n = static_cast<long long>(max(0, min(*P.n_copies, P.max_copies))) * P.n_kv;
    for (long long u = blockIdx.x * 8ll + (threadIdx.x >> 5); u < n; u += gridDim.x * 8ll) {
        const int k = static_cast<int>(u / P.n_kv), h = static_cast<int>(u % P.n_kv);
        const int src = P.src[k], dst = P.dst[k];
        if (src < 0 && dst < 0) continue;                // an unused place of the list
        if (src < 0 || dst < 0 || src >= P.n_pages || dst >= P.n_pages) {
            if (lane == 0) atomicOr(P.dev_status, WUSHKV_DEV_BAD_PAGE_ID);
            continue;
        }
        if (src == dst) continue;
        const long long a = static_cast<long long>(src) * P.n_kv + h, b = static_cast<long long>(dst) * P.n_kv + h;
        const uint4* from = reinterpret_cast<const uint4*>(P.pages + a * REC);
        uint4* to = reinterpret_cast<uint4*>(P.pages + b * REC);
        uint4 x[PER_LANE], y;
        signed char e = 0;
#pragma unroll
        for (int i = 0; i < PER_LANE; ++i) if (32 * i + lane < VECS) x[i] = __ldcs(from + 32 * i + lane);
        if (P.bounds) {
            if (lane < 2 * D / 16) y = __ldcs(reinterpret_cast<const uint4*>(P.bounds + a * 2 * D) + lane);
            if (lane == 0) e = P.exponents[a];
        }
#pragma unroll
        for (int i = 0; i < PER_LANE; ++i) if (32 * i + lane < VECS) __stcs(to + 32 * i + lane, x[i]);
        if (P.bounds) {
            if (lane < 2 * D / 16) reinterpret_cast<uint4*>(P.bounds + b * 2 * D)[lane] = y;
            if (lane == 0) P.exponents[b] = e;
        }
    }
}

struct CopyWindowsParams {
    unsigned short* sink;
    unsigned short* ring;
    int* dev_status;
    const int* src_slot;
    const int* dst_slot;
    const int* src_len;
    int n_slots, planes, s_sink, ring_cap;               // planes: keys and values of all heads
};
constexpr int WINDOW_VECS = 8;                           // 16-byte vectors per thread

// blockIdx.y: the copy; its rows are numbered (plane, sink rows then ring rows), 16 vectors each.
__global__ void __launch_bounds__(256) copy_windows_kernel(CopyWindowsParams P) {
    pdl_wait();
    pdl_launch_dependents();
    const int k = blockIdx.y, src = P.src_slot[k], dst = P.dst_slot[k], len = P.src_len[k];
    if (src < 0 || src >= P.n_slots || dst < 0 || dst >= P.n_slots) {
        if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(P.dev_status, WUSHKV_DEV_BAD_SLOT);
        return;
    }
    if (src == dst) return;
    const int rows = P.s_sink + P.ring_cap;
    const long long n = static_cast<long long>(P.planes) * rows * (D / 8);
    uint4 x[WINDOW_VECS];
    uint4* to[WINDOW_VECS];
#pragma unroll
    for (int e = 0; e < WINDOW_VECS; ++e) {
        const long long i = (static_cast<long long>(blockIdx.x) * WINDOW_VECS + e) * 256 + threadIdx.x;
        to[e] = nullptr;
        if (i < n) {
            const long long row_id = i / (D / 8);
            const int vec = static_cast<int>(i % (D / 8)), plane = static_cast<int>(row_id / rows), row = static_cast<int>(row_id % rows);
            const bool sink = row < P.s_sink;
            const int r = sink ? row : row - P.s_sink, per = sink ? P.s_sink : P.ring_cap;
            if (r < len) {                               // position p < ring_cap is in row p; a longer sequence has used all rows
                unsigned short* base = sink ? P.sink : P.ring;
                x[e] = reinterpret_cast<const uint4*>(base + ((static_cast<long long>(src) * P.planes + plane) * per + r) * D)[vec];
                to[e] = reinterpret_cast<uint4*>(base + ((static_cast<long long>(dst) * P.planes + plane) * per + r) * D) + vec;
            }
        }
    }
#pragma unroll
    for (int e = 0; e < WINDOW_VECS; ++e) if (to[e]) *to[e] = x[e];
}

// The kernels walk pages and requests with 32-bit indexes that run past the end by up to a step, and add up the pages that a tile
// of POOL_THREADS requests asks for in 32 bits.
constexpr long long MAX_POOL_PAGES = 1 << 30;
constexpr int MAX_POOL_BATCH = 1 << 30, MAX_TABLE_PAGES = 1 << 20;
static_assert(POOL_THREADS * (MAX_TABLE_PAGES + 1ll) < 0x7fffffffll, "a tile's pages are counted in 32 bits");

static int make_pool(const wushkv_page_pool* p, PoolView& v) {
    if (!p || p->n_slots <= 0 || p->max_pages <= 0 || p->n_pages <= 0) return WUSHKV_EINVAL;
    if (p->n_pages > MAX_POOL_PAGES || p->max_pages > MAX_TABLE_PAGES) return WUSHKV_EINVAL;
    if (!p->page_table || !p->refs || !p->dev_status) return WUSHKV_EINVAL;
    if (!aligned(p->page_table, 4) || !aligned(p->refs, 4) || !aligned(p->dev_status, 4)) return WUSHKV_EINVAL;
    v.n_slots = p->n_slots; v.max_pages = p->max_pages; v.n_pages = static_cast<int>(p->n_pages);
    v.table = p->page_table; v.refs = p->refs; v.dev_status = p->dev_status;
    return WUSHKV_OK;
}

// Integers of workspace: `list` of reserve shares its place with the page numbers of its second phase, hence the larger of the two.
static size_t pool_workspace_ints(const PoolView& v, int batch) {
    const size_t reserve = 2 * static_cast<size_t>(batch) + std::max<size_t>(static_cast<size_t>(v.n_pages), static_cast<size_t>(batch));
    return std::max(reserve, 3 * static_cast<size_t>(v.n_pages));
}

static int launched(cudaError_t e) { return e == cudaSuccess ? WUSHKV_OK : WUSHKV_ECUDA; }

}  // namespace wushkv

using namespace wushkv;

extern "C" size_t wushkv_pages_workspace_bytes(const wushkv_page_pool* pool, int32_t batch) {
    PoolView v;
    if (make_pool(pool, v) != WUSHKV_OK || batch <= 0 || batch > MAX_POOL_BATCH) return 0;
    return pool_workspace_ints(v, batch) * sizeof(int);
}

extern "C" int wushkv_pages_reserve(const wushkv_page_pool* pool, int32_t batch, const int32_t* slot, const int32_t* seq_len, const int32_t* cu_new,
                                    int32_t* copy_src, int32_t* copy_dst, int32_t* n_copies, void* workspace, size_t workspace_bytes, void* stream) {
    ReserveParams P;
    const int rc = make_pool(pool, P.v);
    if (rc != WUSHKV_OK) return rc;
    if (batch <= 0 || batch > MAX_POOL_BATCH || !slot || !seq_len || !cu_new || !copy_src || !copy_dst || !n_copies || !workspace || !int_arrays(slot, seq_len, cu_new, copy_src, copy_dst, n_copies, workspace))
        return WUSHKV_EINVAL;
    if (workspace_bytes < pool_workspace_ints(P.v, batch) * sizeof(int)) return WUSHKV_ECAPACITY;
    P.batch = batch; P.slot = slot; P.seq_len = seq_len; P.cu_new = cu_new;
    P.copy_src = copy_src; P.copy_dst = copy_dst; P.n_copies = n_copies;
    P.need = static_cast<int*>(workspace);
    P.shared = P.need + batch;
    P.list = P.shared + batch;
    return launched(launch_pdl(pages_reserve_kernel, dim3(POOL_CTAS), dim3(POOL_THREADS), 0, static_cast<cudaStream_t>(stream), P));
}

extern "C" int wushkv_pages_fork(const wushkv_page_pool* pool, int32_t n, const int32_t* src_slot, const int32_t* dst_slot, const int32_t* src_len, void* stream) {
    PoolView v;
    const int rc = make_pool(pool, v);
    if (rc != WUSHKV_OK) return rc;
    if (n < 0 || !src_slot || !dst_slot || !src_len || !int_arrays(src_slot, dst_slot, src_len)) return WUSHKV_EINVAL;
    if (n == 0) return WUSHKV_OK;
    return launched(launch_pdl(pages_fork_kernel, dim3(n), dim3(256), 0, static_cast<cudaStream_t>(stream), v, src_slot, dst_slot, src_len));
}

extern "C" int wushkv_pages_release(const wushkv_page_pool* pool, int32_t n, const int32_t* slot, const int32_t* keep_len, void* stream) {
    PoolView v;
    const int rc = make_pool(pool, v);
    if (rc != WUSHKV_OK) return rc;
    if (n < 0 || !slot || !int_arrays(slot, keep_len)) return WUSHKV_EINVAL;
    if (n == 0) return WUSHKV_OK;
    return launched(launch_pdl(pages_release_kernel, dim3(n), dim3(256), 0, static_cast<cudaStream_t>(stream), v, slot, keep_len));
}

extern "C" int wushkv_pages_compact(const wushkv_page_pool* pool, int32_t* copy_src, int32_t* copy_dst, int32_t* n_copies, int32_t* n_live,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    CompactParams P;
    const int rc = make_pool(pool, P.v);
    if (rc != WUSHKV_OK) return rc;
    if (!copy_src || !copy_dst || !n_copies || !n_live || !workspace || !int_arrays(copy_src, copy_dst, n_copies, n_live, workspace)) return WUSHKV_EINVAL;
    if (workspace_bytes < 3 * static_cast<size_t>(P.v.n_pages) * sizeof(int)) return WUSHKV_ECAPACITY;
    P.copy_src = copy_src; P.copy_dst = copy_dst; P.n_copies = n_copies; P.n_live = n_live;
    P.holes = static_cast<int*>(workspace);
    P.movers = P.holes + P.v.n_pages;
    P.moved = P.movers + P.v.n_pages;
    P.n_list = (P.v.n_pages + 1) / 2;
    return launched(launch_pdl(pages_compact_kernel, dim3(POOL_CTAS), dim3(POOL_THREADS), 0, static_cast<cudaStream_t>(stream), P));
}

extern "C" int wushkv_copy_pages(const wushkv_cache* cache, int32_t max_copies, const int32_t* copy_src, const int32_t* copy_dst, const int32_t* n_copies,
                                 int8_t* bounds, int8_t* exponents, void* stream) {
    CacheView c;
    const int rc = make_view(cache, c);
    if (rc != WUSHKV_OK) return rc;
    if (max_copies < 0 || !copy_src || !copy_dst || !n_copies || !int_arrays(copy_src, copy_dst, n_copies) || (bounds == nullptr) != (exponents == nullptr) || !aligned(bounds, 16)) return WUSHKV_EINVAL;
    if (max_copies == 0) return WUSHKV_OK;
    CopyPagesParams P;
    P.pages = c.pages; P.bounds = bounds; P.exponents = exponents; P.dev_status = c.dev_status;
    P.src = copy_src; P.dst = copy_dst; P.n_copies = n_copies;
    P.n_pages = c.n_pages; P.n_kv = c.n_kv; P.max_copies = max_copies;
    const long long ctas = std::min<long long>((static_cast<long long>(max_copies) * c.n_kv + 7) / 8, 6ll * sm_count());
    const dim3 grid(static_cast<unsigned>(ctas));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return launched(launch_pdl(c.bits == 2 ? copy_pages_kernel<2> : c.bits == 3 ? copy_pages_kernel<3> : copy_pages_kernel<4>, grid, dim3(256), 0, st, P));
}

extern "C" int wushkv_copy_windows(const wushkv_cache* cache, int32_t n, const int32_t* src_slot, const int32_t* dst_slot, const int32_t* src_len, void* stream) {
    CacheView c;
    const int rc = make_view(cache, c);
    if (rc != WUSHKV_OK) return rc;
    if (n < 0 || n > 65535 || !src_slot || !dst_slot || !src_len || !int_arrays(src_slot, dst_slot, src_len)) return WUSHKV_EINVAL;
    if (n == 0) return WUSHKV_OK;
    CopyWindowsParams P;
    P.sink = c.sink_kv; P.ring = c.ring_kv; P.dev_status = c.dev_status;
    P.src_slot = src_slot; P.dst_slot = dst_slot; P.src_len = src_len;
    P.n_slots = c.n_slots; P.planes = 2 * c.n_kv; P.s_sink = c.s_sink; P.ring_cap = c.ring_cap;
    const long long vecs = static_cast<long long>(P.planes) * (P.s_sink + P.ring_cap) * (D / 8);
    const dim3 grid(static_cast<unsigned>((vecs + 256 * WINDOW_VECS - 1) / (256 * WINDOW_VECS)), n);
    return launched(launch_pdl(copy_windows_kernel, grid, dim3(256), 0, static_cast<cudaStream_t>(stream), P));
}
