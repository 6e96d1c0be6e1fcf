// Pages of a paged cache: sharing them between sequences, giving writers pages of their own, handing back what a prune
// left behind, moving the live ones together, copying their rows, and appending new rows.
//
// The bookkeeping (fork, reserve, free, compact) works on small integer arrays and is bound by latency: one launch each,
// every rank that decides who gets which page comes from a prefix sum in a fixed order, atomics only count.  The data
// movement (copy, append) is bound by memory: 128-bit loads and stores, nothing else.
#include <limits.h>

#include "csp_internal.cuh"

namespace csp {
namespace {

constexpr int kTableThreads = 1024;
constexpr int kPerThread = 4;                            // neighbouring entries per thread and scan step

// Exclusive prefix sum over the block of one packed pair of 16-bit counts per thread; `total` is the block's sum.  A
// step covers kTableThreads * kPerThread = 4096 entries, so neither half can overflow.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* warp_sums, uint32_t& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();                                     // the previous step's sums have been read
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    uint32_t w = warp_sums[lane];                        // kTableThreads / 32 = 32 warps: one sum per lane
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, w, d);
        if (lane >= d) w += y;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const uint32_t before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
    return x - v + (warp > 0 ? before : 0u);
}

// The arrays are changed by the kernel that reads them (stores and atomics of other threads of the block): read them
// from L2, where atomics land.
__device__ __forceinline__ int32_t ld(const int32_t* p) { return __ldcg(p); }

// Table entries e = b * max_pages + i as csp_pages_reserve sees them.  A thread takes kPerThread neighbours at a time, so that
// the chains of dependent loads (sequence, entry, count) of all four are under way together.
struct Entry { int page; bool claim, fresh; };
constexpr int kNamed = INT_MAX;                          // in PageArgs::last: a table entry names the page, but it is counted free
__device__ __forceinline__ void reserve_entries(const PageArgs& a, uint32_t entries, uint32_t e0, bool flag, Entry (&x)[kPerThread],
                                                int (&refs)[kPerThread], int* named) {
    int held[kPerThread], need[kPerThread], first[kPerThread], i[kPerThread];
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
        const uint32_t e = e0 + j, b = e / uint32_t(a.max_pages);
        i[j] = int(e - b * uint32_t(a.max_pages));
        held[j] = need[j] = first[j] = 0;
        x[j] = Entry{-1, false, false};
        if (e < entries) { held[j] = ld(a.held + b); need[j] = ld(a.need + b); first[j] = ld(a.first + b); }
    }
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
        x[j].fresh = i[j] >= held[j] && i[j] < need[j];
        if (i[j] >= first[j] && i[j] < held[j] && i[j] < need[j]) {
            const int page = ld(a.table + e0 + j);
            if (page >= 0 && page < a.n_pages) x[j].page = page;
            else if (flag) atomicOr(a.status, CSP_DEV_BAD_LEN);
        }
    }
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) refs[j] = x[j].page >= 0 ? ld(a.refs + x[j].page) : 1;
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
        if (refs[j] <= 0) {
            if (flag) { atomicOr(a.status, CSP_DEV_BAD_LEN); a.last[x[j].page] = kNamed; *named = 1; }
            x[j].page = -1;
        }
        x[j].claim = refs[j] > 1;
    }
}

// A shared page is copied for whoever asks for it, except that the last one to ask keeps it when all who share it ask.  One
// that more ask for than it is counted for contradicts itself and stays as it is.
__device__ __forceinline__ void reserve_copies(const PageArgs& a, uint32_t e0, const Entry (&x)[kPerThread],
                                               const int (&refs)[kPerThread], bool (&copies)[kPerThread]) {
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) {
        const int claims = x[j].claim ? ld(a.claims + x[j].page) : 0;
        copies[j] = x[j].claim && claims <= refs[j] && !(claims == refs[j] && ld(a.last + x[j].page) == int32_t(e0 + j));
    }
}

// One block: bound by the latency of its chains of loads (9 us for 12 sequences), with thousands of entries by the scattered
// loads that one SM can have in flight (80 sequences, 5 K entries: 32 us).  Spread over the GPU it would be three launches.
__global__ void __launch_bounds__(kTableThreads) pages_reserve_kernel(const PageArgs a, const int32_t* n_new, int whole,
                                                                      int2* moves, int max_moves, int32_t* n_moves) {
    __shared__ uint32_t warp_sums[32];
    __shared__ int fail, named;                          // named: some page is counted free, but a table entry names it
    __shared__ uint32_t sum_want, sum_copy, sum_free;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) { fail = named = 0; sum_want = sum_copy = sum_free = 0; }
    __syncthreads();
    // how many pages every sequence needs, and from which on they have to be its own: one warp per sequence
    for (int b = warp; b < a.batch; b += kTableThreads / 32) {
        int lo = INT_MAX, hi = 0;
        for (int h = lane; h < a.n_heads; h += 32) {
            const int r = a.n_rows[int64_t(b) * a.n_heads + h];
            lo = min(lo, r);
            hi = max(hi, r);
        }
        lo = __reduce_min_sync(0xffffffffu, lo);
        hi = __reduce_max_sync(0xffffffffu, hi);
        const int more = n_new ? n_new[b] : 0, held = a.held[b];
        const int64_t need = (int64_t(hi) + more + a.page_rows - 1) / a.page_rows;
        if (lane == 0) {
            if (lo < 0 || more < 0 || held < 0 || held > a.max_pages) atomicOr(&fail, CSP_DEV_BAD_LEN);
            else if (need > a.max_pages) atomicOr(&fail, CSP_DEV_CAPACITY);
            else { a.first[b] = whole ? 0 : lo / a.page_rows; a.need[b] = int(need); }
        }
    }
    for (int p = tid; p < a.n_pages; p += kTableThreads) { a.claims[p] = 0; a.last[p] = -1; }
    __syncthreads();
    const uint32_t entries = uint32_t(a.batch) * uint32_t(a.max_pages);          // (31 bits)
    constexpr uint32_t kStep = kTableThreads * kPerThread;
    Entry x[kPerThread];
    int refs[kPerThread];
    bool copies[kPerThread];
    if (!fail) {
        for (uint32_t e0 = tid * kPerThread; e0 < entries; e0 += kStep) {
            reserve_entries(a, entries, e0, true, x, refs, &named);
#pragma unroll
            for (int j = 0; j < kPerThread; ++j)
                if (x[j].claim) { atomicAdd(a.claims + x[j].page, 1); atomicMax(a.last + x[j].page, int32_t(e0 + j)); }
        }
    }
    __syncthreads();
    const bool any_named = named != 0;                   // such pages are left alone
    if (!fail) {
        uint32_t want = 0, copy = 0, free_pages = 0;
        for (uint32_t e0 = tid * kPerThread; e0 < entries; e0 += kStep) {
            if (entries > kStep) reserve_entries(a, entries, e0, false, x, refs, &named);        // (else they are here still)
            reserve_copies(a, e0, x, refs, copies);
#pragma unroll
            for (int j = 0; j < kPerThread; ++j) { copy += copies[j]; want += copies[j] || x[j].fresh; }
        }
#pragma unroll 4
        for (int p = tid; p < a.n_pages; p += kTableThreads) free_pages += ld(a.refs + p) == 0;
        if (any_named)
            for (int p = tid; p < a.n_pages; p += kTableThreads) free_pages -= ld(a.refs + p) == 0 && ld(a.last + p) == kNamed;
        want = __reduce_add_sync(0xffffffffu, want);
        copy = __reduce_add_sync(0xffffffffu, copy);
        free_pages = __reduce_add_sync(0xffffffffu, free_pages);
        if (lane == 0) { atomicAdd(&sum_want, want); atomicAdd(&sum_copy, copy); atomicAdd(&sum_free, free_pages); }
    }
    __syncthreads();
    if (tid == 0) {
        if (!fail && (sum_want > sum_free || sum_copy > uint32_t(max_moves))) fail = CSP_DEV_CAPACITY;
        if (fail) atomicOr(a.status, fail);
        *n_moves = fail ? 0 : int(sum_copy);
    }
    __syncthreads();
    if (fail) return;                                    // all or nothing
    // the free pages, lowest first
    uint32_t base = 0;
    for (int p0 = 0; p0 < a.n_pages && base < sum_want; p0 += kTableThreads * kPerThread) {
        bool is_free[kPerThread];
        uint32_t n = 0, total;
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            const int p = p0 + tid * kPerThread + j;
            is_free[j] = p < a.n_pages && ld(a.refs + p) == 0;
            if (any_named) is_free[j] = is_free[j] && ld(a.last + p) != kNamed;
            n += is_free[j];
        }
        uint32_t rank = base + block_scan(n, warp_sums, total);
#pragma unroll
        for (int j = 0; j < kPerThread; ++j)
            if (is_free[j] && rank < sum_want) a.list[rank++] = p0 + tid * kPerThread + j;
        base += total;
    }
    __syncthreads();
    // hand them out in the order of sequence and table index
    uint32_t base_want = 0, base_copy = 0;
    for (uint32_t e_base = 0; e_base < entries; e_base += kStep) {
        const uint32_t e0 = e_base + tid * kPerThread;
        if (entries > kStep) {
            reserve_entries(a, entries, e0, false, x, refs, &named);
            reserve_copies(a, e0, x, refs, copies);
        }
        uint32_t n = 0, total;
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            if (e0 >= entries) { x[j].fresh = false; copies[j] = false; }
            n += (copies[j] || x[j].fresh ? 1u : 0u) + (copies[j] ? 0x10000u : 0u);
        }
        const uint32_t before = block_scan(n, warp_sums, total);
        uint32_t want = base_want + (before & 0xffffu), copy = base_copy + (before >> 16);
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            if (!copies[j] && !x[j].fresh) continue;
            const int to = ld(a.list + want++);
            if (copies[j]) moves[copy++] = make_int2(x[j].page, to);
            a.table[e0 + j] = to;
            a.refs[to] = 1;                              // it was free: nobody claims it
        }
        base_want += total & 0xffffu;
        base_copy += total >> 16;
    }
    __syncthreads();
    for (int p = tid; p < a.n_pages; p += kTableThreads) {
        const int c = ld(a.claims + p);
        if (c > 0) {
            const int r = ld(a.refs + p);
            if (c > r) atomicOr(a.status, CSP_DEV_BAD_LEN);
            else a.refs[p] = c == r ? 1 : r - c;
        }
    }
    for (int b = tid; b < a.batch; b += kTableThreads) a.held[b] = max(ld(a.held + b), ld(a.need + b));
}

__global__ void __launch_bounds__(kTableThreads) pages_compact_kernel(const PageArgs a, int2* moves, int max_moves,
                                                                      int32_t* n_moves) {
    __shared__ uint32_t warp_sums[32];
    __shared__ uint32_t sum_live, sum_movers;
    __shared__ int named;                                // some page is counted free, but a table entry names it
    const int tid = threadIdx.x, lane = tid & 31;
    if (tid == 0) { sum_live = sum_movers = 0; named = 0; }
    __syncthreads();
    const uint32_t entries = uint32_t(a.batch) * uint32_t(a.max_pages);          // (31 bits)
#pragma unroll 4
    for (uint32_t e = tid; e < entries; e += kTableThreads) {
        const uint32_t b = e / uint32_t(a.max_pages);
        const int p = a.table[e];
        if (int(e - b * uint32_t(a.max_pages)) < ld(a.held + b) && p >= 0 && p < a.n_pages && ld(a.refs + p) <= 0) named = 1;
    }
    uint32_t n = 0;
    for (int p = tid; p < a.n_pages; p += kTableThreads) n += ld(a.refs + p) > 0;
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) atomicAdd(&sum_live, n);
    __syncthreads();
    const int live = int(sum_live);
    n = 0;
    for (int p = live + tid; p < a.n_pages; p += kTableThreads) n += ld(a.refs + p) > 0;
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) atomicAdd(&sum_movers, n);
    __syncthreads();
    const bool fits = sum_movers <= uint32_t(max_moves);
    if (tid == 0) {
        if (!fits || named) atomicOr(a.status, (fits ? 0 : CSP_DEV_CAPACITY) | (named ? CSP_DEV_BAD_LEN : 0));
        *n_moves = fits && !named ? int(sum_movers) : 0;
    }
    if (!fits || named) return;                          // a page that moved into a hole would be named by others
    // as many holes in front of `live` as pages in use behind it; both lists ascending
    uint32_t base = 0;
    for (int p0 = 0; p0 < live; p0 += kTableThreads * kPerThread) {
        bool hole[kPerThread];
        uint32_t c = 0, total;
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            const int p = p0 + tid * kPerThread + j;
            hole[j] = p < live && ld(a.refs + p) <= 0;
            c += hole[j];
        }
        uint32_t rank = base + block_scan(c, warp_sums, total);
#pragma unroll
        for (int j = 0; j < kPerThread; ++j)
            if (hole[j]) a.list[rank++] = p0 + tid * kPerThread + j;
        base += total;
    }
    __syncthreads();
    base = 0;
    for (int p0 = live; p0 < a.n_pages; p0 += kTableThreads * kPerThread) {
        int refs[kPerThread];
        uint32_t c = 0, total;
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            const int p = p0 + tid * kPerThread + j;
            refs[j] = p < a.n_pages ? ld(a.refs + p) : 0;
            c += refs[j] > 0;
        }
        uint32_t rank = base + block_scan(c, warp_sums, total);
#pragma unroll
        for (int j = 0; j < kPerThread; ++j) {
            const int p = p0 + tid * kPerThread + j;
            if (p >= a.n_pages) continue;
            int to = -1;
            if (refs[j] > 0) {
                to = ld(a.list + rank);
                moves[rank++] = make_int2(p, to);
                a.refs[to] = refs[j];
                a.refs[p] = 0;
            }
            a.claims[p] = to;                            // where the page went
        }
        base += total;
    }
    __syncthreads();
    for (uint32_t e = tid; e < entries; e += kTableThreads) {
        const uint32_t b = e / uint32_t(a.max_pages);
        if (int(e - b * uint32_t(a.max_pages)) >= ld(a.held + b)) continue;
        const int p = a.table[e];
        if (p >= 0 && p < live) continue;
        const int to = p >= live && p < a.n_pages ? ld(a.claims + p) : -1;
        if (to >= 0) a.table[e] = to;
        else atomicOr(a.status, CSP_DEV_BAD_LEN);
    }
}

// one block per sequence
__global__ void pages_free_kernel(const PageArgs a) {
    __shared__ int lo, hi;
    const int b = blockIdx.x;
    if (threadIdx.x == 0) { lo = INT_MAX; hi = 0; }
    __syncthreads();
    int l = INT_MAX, u = 0;
    for (int h = threadIdx.x; h < a.n_heads; h += blockDim.x) {
        const int r = a.n_rows[int64_t(b) * a.n_heads + h];
        l = min(l, r);
        u = max(u, r);
    }
    atomicMin(&lo, l);
    atomicMax(&hi, u);
    __syncthreads();
    const int held = a.held[b];
    const int64_t need = (int64_t(hi) + a.page_rows - 1) / a.page_rows;
    if (lo < 0 || held < 0 || held > a.max_pages || need > held) {
        if (threadIdx.x == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
        return;
    }
    __syncthreads();                                     // everybody has read held[b]
    int32_t* const row = a.table + int64_t(b) * a.max_pages;
    for (int i = int(need) + threadIdx.x; i < held; i += blockDim.x) {
        const int p = row[i];
        if (p < 0 || p >= a.n_pages) { atomicOr(a.status, CSP_DEV_BAD_LEN); continue; }
        if (atomicSub(a.refs + p, 1) <= 0) { atomicAdd(a.refs + p, 1); atomicOr(a.status, CSP_DEV_BAD_LEN); continue; }
        row[i] = -1;
    }
    if (threadIdx.x == 0) a.held[b] = int(need);
}

__global__ void __launch_bounds__(kTableThreads) pages_fork_kernel(const PageArgs a, const int32_t* src, const int32_t* dst,
                                                                   int n) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t* const owner = a.first;                      // [batch]: the first fork that names the sequence as its dst
    for (int b = tid; b < a.batch; b += kTableThreads) { owner[b] = INT_MAX; a.need[b] = -1; }
    __syncthreads();
    for (int i = tid; i < n; i += kTableThreads) {
        const int d = dst[i];
        if (d >= 0 && d < a.batch) atomicMin(owner + d, i);
    }
    __syncthreads();
    // One warp per fork; a dst is written by its owner only, and no src is a dst: no order matters.  First all of them are
    // looked at, while the counts are those of the call's start (4.1 us for 8 forks instead of 3.1; need[d]: the fork that is done).
    for (int i = warp; i < n; i += kTableThreads / 32) {
        const int s = src[i], d = dst[i];
        bool ok = s >= 0 && s < a.batch && d >= 0 && d < a.batch;
        ok = ok && ld(owner + d) == i && ld(owner + s) == INT_MAX && ld(a.held + d) == 0;
        const int held = ok ? ld(a.held + s) : 0;
        ok = ok && held >= 0 && held <= a.max_pages;
        for (int j = lane; ok && j < held; j += 32) {
            const int p = a.table[int64_t(s) * a.max_pages + j];
            ok = p >= 0 && p < a.n_pages && ld(a.refs + p) > 0;
        }
        ok = __all_sync(0xffffffffu, ok);
        if (lane == 0) {
            if (ok) a.need[d] = i;
            else atomicOr(a.status, CSP_DEV_BAD_LEN);
        }
    }
    __syncthreads();
    for (int i = warp; i < n; i += kTableThreads / 32) {
        const int s = src[i], d = dst[i];
        if (d < 0 || d >= a.batch || ld(a.need + d) != i) continue;
        const int held = ld(a.held + s);
        for (int j = lane; j < held; j += 32) {
            const int p = a.table[int64_t(s) * a.max_pages + j];
            a.table[int64_t(d) * a.max_pages + j] = p;
            atomicAdd(a.refs + p, 1);
        }
        for (int h = lane; h < a.n_heads; h += 32)
            a.n_rows[int64_t(d) * a.n_heads + h] = a.n_rows[int64_t(s) * a.n_heads + h];
        if (lane == 0) a.held[d] = held;
    }
}

// ---- data movement -------------------------------------------------------------------------------------------------
constexpr int kCopyThreads = 256;
constexpr int kCopyDepth = 8;                            // 16-byte loads in flight per thread: a 128-row page of one head at d = 128

__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// Work item = (move, K or V, head): the rows of one head in one page.  Bound by memory: every byte is read and written
// once (1.3 GB of pages in 407 us, 6.4 TB/s, which is what a plain copy reaches; 117 MB in 38 us).
__global__ void __launch_bounds__(kCopyThreads) pages_copy_kernel(const PageCopyArgs a) {
    int n = *a.n_moves;
    if (n < 0 || n > a.max_moves) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
        n = n < 0 ? 0 : a.max_moves;
    }
    const int cpr = a.chunks_per_row, chunks = a.page_rows * cpr;
    const int64_t items = int64_t(n) * 2 * a.n_kv_heads;
    for (int64_t w = blockIdx.x; w < items; w += gridDim.x) {
        const int h = int(w % a.n_kv_heads), which = int(w / a.n_kv_heads % 2);
        const int2 m = a.moves[w / (2 * a.n_kv_heads)];
        if (m.x < 0 || m.x >= a.n_pages || m.y < 0 || m.y >= a.n_pages) {
            if (threadIdx.x == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
            continue;
        }
        const int64_t st = which ? a.v_st : a.k_st, head = int64_t(h) * (which ? a.v_sh : a.k_sh);
        const int64_t page = which ? a.v_sb : a.k_sb;
        uint4* const pool = static_cast<uint4*>(which ? a.v : a.k);
        const uint4* const from = pool + int64_t(m.x) * page + head;
        uint4* const to = pool + int64_t(m.y) * page + head;
        for (int c0 = threadIdx.x; c0 < chunks; c0 += kCopyThreads * kCopyDepth) {
            uint4 v[kCopyDepth];
            int64_t at[kCopyDepth];
#pragma unroll
            for (int j = 0; j < kCopyDepth; ++j) {
                const int c = c0 + j * kCopyThreads;
                at[j] = int64_t(c / cpr) * st + c % cpr;
                if (c < chunks) v[j] = ld_stream(from + at[j]);
            }
#pragma unroll
            for (int j = 0; j < kCopyDepth; ++j)
                if (c0 + j * kCopyThreads < chunks) to[at[j]] = v[j];
        }
    }
}

// What csp_append_paged does with unit u: its first new row and how many follow; flags what it refuses.
__device__ __forceinline__ int append_rows(const AppendArgs& a, int u, int b, int& first, bool flag) {
    first = a.n_rows[u];
    int more = a.n_new ? a.n_new[b] : a.max_new, bad = 0;
    if (more < 0 || more > a.max_new) { bad |= CSP_DEV_BAD_LEN; more = more < 0 ? 0 : a.max_new; }
    if (first < 0) { bad |= CSP_DEV_BAD_LEN; more = 0; }
    else if (int64_t(first) + more > a.capacity) { bad |= CSP_DEV_CAPACITY; more = 0; }
    if (flag && bad) atomicOr(a.status, bad);
    return more;
}

// Block (u, .) moves kAppendRows new rows of unit u at a time, K and V: 16 bytes per thread and step, four steps in flight.  Bound
// by memory: every byte is read and written once (3 K tokens of 32 heads at d = 128, 50 MB: 22.5 us, 4.5 TB/s; a block
// per row 46 us), one token by the launch (3 us).
constexpr int kAppendRows = 32;
__global__ void __launch_bounds__(kCopyThreads) append_kernel(const AppendArgs a, int log_chunks, int count_here) {
    const int u = blockIdx.x, b = u / a.n_kv_heads, h = u - b * a.n_kv_heads;
    int first;
    const bool lead = blockIdx.y == 0 && threadIdx.x == 0;
    const int more = append_rows(a, u, b, first, lead);
    if (lead && count_here) a.n_rows_out[u] = first + more;
    for (int i0 = blockIdx.y * kAppendRows; i0 < more; i0 += int(gridDim.y) * kAppendRows) {
        const int rows = min(more - i0, kAppendRows);
        const uint4* const from[2] = {static_cast<const uint4*>(a.k_new) + int64_t(b) * a.kn_sb + int64_t(h) * a.kn_sh + int64_t(i0) * a.kn_st,
                                      static_cast<const uint4*>(a.v_new) + int64_t(b) * a.vn_sb + int64_t(h) * a.vn_sh + int64_t(i0) * a.vn_st};
        const int total = rows << (log_chunks + 1);          // chunks of [row][K or V][16 bytes]
        const int32_t* const table = a.page_table + int64_t(b) * a.max_pages;
        for (int x0 = threadIdx.x; x0 < total; x0 += 4 * blockDim.x) {
            uint4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int x = x0 + j * int(blockDim.x), c = x & ((1 << log_chunks) - 1), which = (x >> log_chunks) & 1, i = x >> (log_chunks + 1);
                if (x < total) v[j] = ld_stream((which ? from[1] + i * a.vn_st : from[0] + i * a.kn_st) + c);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int x = x0 + j * int(blockDim.x), c = x & ((1 << log_chunks) - 1), which = (x >> log_chunks) & 1, i = x >> (log_chunks + 1);
                if (x >= total) continue;
                const uint32_t t = uint32_t(first + i0 + i), slot = t % uint32_t(a.page_rows);
                const int page = table[t / uint32_t(a.page_rows)];
                if (page < 0 || page >= a.n_pages) {
                    if (which == 0 && c == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
                    continue;
                }
                if (which) static_cast<uint4*>(a.v)[int64_t(page) * a.v_sb + int64_t(h) * a.v_sh + int64_t(slot) * a.v_st + c] = v[j];
                else static_cast<uint4*>(a.k)[int64_t(page) * a.k_sb + int64_t(h) * a.k_sh + int64_t(slot) * a.k_st + c] = v[j];
            }
        }
    }
}

// the row counts, where they are updated in place: only after every block of append_kernel has read them
__global__ void append_count_kernel(const AppendArgs a) {
    const int u = blockIdx.x * blockDim.x + threadIdx.x;
    if (u >= a.units) return;
    int first;
    const int more = append_rows(a, u, u / a.n_kv_heads, first, false);
    a.n_rows_out[u] = first + more;
}

inline csp_status launched() { return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA; }

}  // namespace

size_t pages_workspace_bytes(const csp_page_state& s) {
    return kStatusBytes + 3 * round256(size_t(s.n_pages) * 4) + 2 * round256(size_t(s.batch) * 4);
}

PageArgs page_args(const csp_page_state& s, void* ws) {
    PageArgs a;
    a.table = s.page_table; a.held = s.held; a.refs = s.refs; a.n_rows = s.n_rows;
    a.batch = s.batch; a.n_heads = s.n_heads; a.max_pages = s.max_pages; a.page_rows = s.page_rows; a.n_pages = s.n_pages;
    a.status = static_cast<int32_t*>(ws);
    const size_t pages = round256(size_t(s.n_pages) * 4) / 4;
    a.claims = a.status + kStatusBytes / 4;
    a.last = a.claims + pages;
    a.list = a.last + pages;
    a.first = a.list + pages;
    a.need = a.first + round256(size_t(s.batch) * 4) / 4;
    return a;
}

csp_status launch_pages_fork(const PageArgs& a, const int32_t* src, const int32_t* dst, int n, cudaStream_t s) {
    if (n == 0) return CSP_OK;
    pages_fork_kernel<<<1, kTableThreads, 0, s>>>(a, src, dst, n);
    return launched();
}

csp_status launch_pages_reserve(const PageArgs& a, const int32_t* n_new, int whole, int32_t* moves, int max_moves,
                                int32_t* n_moves, cudaStream_t s) {
    pages_reserve_kernel<<<1, kTableThreads, 0, s>>>(a, n_new, whole, reinterpret_cast<int2*>(moves), max_moves, n_moves);
    return launched();
}

csp_status launch_pages_free(const PageArgs& a, cudaStream_t s) {
    if (a.batch == 0) return CSP_OK;
    pages_free_kernel<<<a.batch, 128, 0, s>>>(a);
    return launched();
}

csp_status launch_pages_compact(const PageArgs& a, int32_t* moves, int max_moves, int32_t* n_moves, cudaStream_t s) {
    pages_compact_kernel<<<1, kTableThreads, 0, s>>>(a, reinterpret_cast<int2*>(moves), max_moves, n_moves);
    return launched();
}

csp_status launch_pages_copy(const PageCopyArgs& a, cudaStream_t s) {
    const int64_t most = int64_t(a.max_moves) * 2 * a.n_kv_heads;
    if (most == 0) return CSP_OK;
    const int64_t fill = 8 * int64_t(sm_count());        // blocks of 256 threads that the GPU holds at once
    pages_copy_kernel<<<int(most < fill ? most : fill), kCopyThreads, 0, s>>>(a);
    return launched();
}

csp_status launch_append(const AppendArgs& a, cudaStream_t s) {
    if (a.units == 0) return CSP_OK;
    const bool in_place = a.n_rows_out == a.n_rows;
    if (a.max_new > 0) {
        const int log_chunks = a.chunks_per_row == 8 ? 3 : a.chunks_per_row == 16 ? 4 : 5;
        // a single row needs one or two warps
        const int chunks = (a.max_new < kAppendRows ? a.max_new : kAppendRows) * 2 * a.chunks_per_row;
        const int threads = chunks < kCopyThreads ? (chunks + 31) / 32 * 32 : kCopyThreads;
        const int blocks = a.max_new / kAppendRows + (a.max_new % kAppendRows ? 1 : 0);
        append_kernel<<<dim3(a.units, blocks < 65535 ? blocks : 65535), threads, 0, s>>>(a, log_chunks, in_place ? 0 : 1);
        if (const csp_status st = launched()) return st;
    }
    if (in_place || a.max_new == 0) append_count_kernel<<<(a.units + 127) / 128, 128, 0, s>>>(a);
    return launched();
}

}  // namespace csp
