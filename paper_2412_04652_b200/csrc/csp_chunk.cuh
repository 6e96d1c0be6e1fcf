// Shared by the chunk attention kernels (csp_chunk.cu: many query rows per KV head, csp_chunk_few.cu: up to sixteen; over pages in 4
// bits csp_chunk_q4_many.cu and csp_chunk_q4.cu) and the kernel that joins the parts of a split cache.
#pragma once

#include "csp_device.cuh"
#include "csp_internal.cuh"

namespace csp {

struct ChunkPlan {                                       // sizes that host and device agree on
    int tok_tile, pair_tokens;                           // tokens in a row tile: 128 / G; in an item: a pair of these
    int n_pairs, row_slots;                              // items per unit, rows of a partial result
    int n_items;                                         // units x pairs
    int grid;                                            // resident blocks
    int key_tile, min_tiles;                             // keys per tile; tiles that a part of a cut item has at least
    int item_cost;                                       // what an item costs besides its key tiles, in key tiles
    bool drawn;                                          // items may be drawn whole from a counter instead of shared out
    int snap;                                            // tiles by which a share may differ from an equal one to avoid a cut
    Divider by_pairs, by_heads, by_group, by_tile;       // n_pairs, KV heads, query heads per KV head, key_tile
};

// What a block says about the items it was given only part of (see Share): the one that begins with it (-1: none), and whether
// the one it goes on with ends with it.
struct ChunkParts { int32_t first, last; };

// where a workspace keeps the partial results
struct PartialLayout { size_t parts, ml, o, total; };
PartialLayout partial_layout(const csp_params& p, const ChunkPlan& pl);
// joins them; few: up to sixteen rows per item
csp_status launch_chunk_join(const csp_params& p, const ChunkArgs& a, const ChunkPlan& pl, bool few, ChunkParts* parts,
                             float* partial, float2* ml, cudaStream_t s);

// how a chunk of bf16 queries is cut into items; for more than three items of sixteen query rows per KV head a cache in 4 bits is cut alike
ChunkPlan chunk_plan(const csp_params& p, int max_new);
inline void set_dividers(const csp_params& p, ChunkPlan& pl) {
    pl.by_pairs = divider(pl.n_pairs);
    pl.by_heads = divider(p.n_kv_heads);
    pl.by_group = divider(p.n_q_heads / p.n_kv_heads);
    pl.by_tile = divider(pl.key_tile);
}
csp_status launch_chunk_q4_many(const csp_params& p, const ChunkArgs& a, const ChunkPlan& pl, const csp_tensor& q, const Q4Args& c,
                                ChunkParts* parts, float* partial, float2* ml, cudaStream_t s);

csp_status launch_chunk_few(const csp_params& p, const ChunkArgs& a, const ChunkPlan& pl, const csp_tensor& q,
                            const CUtensorMap& tk, const CUtensorMap& tv, ChunkParts* parts, float* partial, float2* ml,
                            cudaStream_t s);

namespace dev {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kSeesAll = 1 << 30;

// Positions are held in fp32 relative to the last token's of the item.  A token's own is exact up to 2^24 from there; up to half
// of that, a key whose position is rounded (by 2^-24 of its distance from the last token) is at least half as far from the token,
// so that every distance keeps 23 bits.  A token farther off is flagged at the item's end.  (Integer distances would cost a conversion
// per logit.)
constexpr float kFarToken = 8388608.f;

// What the rows of a pair look at.
struct PairRange {
    int rows, n_new, tok0, count;                        // rows of the unit, tokens of the sequence, first token, tokens here
    int row0, prefix;                                    // row of the first token; clamped prefix
    int kv_end[2];                                       // keys that row tile 0 / the whole pair can see: [0, kv_end)
    int tiles;
};
// (rows, tokens and prefix as they stand in memory)
__device__ __forceinline__ PairRange pair_range_of(const ChunkArgs& a, const ChunkPlan& pl, int rows, int n_new, int prefix, int pair) {
    PairRange x;
    x.rows = min(max(rows, 0), a.capacity);
    x.n_new = min(max(n_new, 0), a.max_new);
    x.tok0 = pair * pl.pair_tokens;
    x.count = min(x.n_new - x.tok0, pl.pair_tokens);
    x.row0 = x.rows - x.n_new + x.tok0;
    x.prefix = min(max(prefix, 0), x.rows);
    const int last0 = x.row0 + min(x.count, pl.tok_tile) - 1, last1 = x.row0 + x.count - 1;
    x.kv_end[0] = last0 < 0 ? 0 : max(last0 + 1, x.prefix);
    x.kv_end[1] = last1 < 0 ? 0 : max(last1 + 1, x.prefix);
    x.tiles = pl.by_tile(x.kv_end[1] + pl.key_tile - 1);
    return x;
}
__device__ __forceinline__ PairRange pair_range(const ChunkArgs& a, const ChunkPlan& pl, int u, int pair) {
    const int b = pl.by_heads(u), h = u - b * a.n_kv_heads;
    return pair_range_of(a, pl, a.n_rows[u], a.n_new ? a.n_new[b] : a.max_new,
                         a.mods.prefix ? a.mods.prefix[int64_t(b) * a.mods.prefix_sb + int64_t(h) * a.mods.prefix_sh] : 0, pair);
}

// The resident blocks share the work evenly, whatever the lengths are: laid end to end, the items (a pair of row tiles of one
// unit, `tiles` key tiles and item_cost more) are cut into as many equal shares as there are blocks.  A cut inside an item
// divides its key tiles; the parts are joined afterwards.  Cuts that fall near an item's end go to the end (a share
// may be an eighth, but no more than `snap` tiles, larger or smaller), so that work that divides by itself is not cut at
// all, and no share is smaller than an item of min_tiles tiles.  Block c handles tiles [tile0, ...) of item0 up to [.., tile1) of item1: at most its
// first item is the rest of a cut one (partial result 2 c) and its last one the beginning (2 c + 1).
struct Share { int item0, tile0, item1, tile1; bool drawn; };
__device__ __forceinline__ int item_weight(const ChunkArgs& a, const ChunkPlan& pl, int item, bool flag, int& tiles) {
    const int u = pl.by_pairs(item), pair = item - u * pl.n_pairs;
    const PairRange x = pair_range(a, pl, u, pair);
    if (flag && pair == 0) {
        const int rows = a.n_rows[u], more = a.n_new ? a.n_new[pl.by_heads(u)] : a.max_new;
        if (rows != x.rows || more != x.n_new || x.n_new > x.rows) atomicOr(a.status, CSP_DEV_BAD_LEN);
    }
    tiles = x.count > 0 ? x.tiles : 0;
    return x.count > 0 ? x.tiles + pl.item_cost : 0;
}
// All threads of the block; scratch: 68 words of shared memory.  Every block goes over all items (a few per thread): that
// costs less than a launch of its own would.  (The launcher has made sure that the total fits 30 bits.)
// chains, if given: four words, of item0 where it is the rest of a cut item and of item1 where it is cut: the block that the item
// begins in, and in how many blocks its parts are.
template <int kThreads>
__device__ __forceinline__ Share find_share(const ChunkArgs& a, const ChunkPlan& pl, int* scratch, int* chains = nullptr) {
    static_assert(kThreads % 32 == 0 && kThreads <= 1024, "one partial sum per warp");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (pl.n_items + kThreads - 1) / kThreads;
    const int i0 = min(tid * per, pl.n_items), i1 = min(i0 + per, pl.n_items);
    int mine = 0, most = 0, tiles = 0;
#pragma unroll 4
    for (int i = i0; i < i1; ++i) {
        const int w = item_weight(a, pl, i, blockIdx.x == 0, tiles);
        mine += w;
        most = max(most, w);
    }
    most = __reduce_max_sync(0xffffffffu, most);
    int x = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) { scratch[warp] = x; scratch[36 + warp] = most; }
    int* const found = scratch + 32;                     // two (item, tile) pairs
    if (tid < 2) { found[2 * tid] = pl.n_items; found[2 * tid + 1] = 0; }
    __syncthreads();
    const int sums = lane < kThreads / 32 ? scratch[lane] : 0;
    const int total = __reduce_add_sync(0xffffffffu, sums);
    const int before = __reduce_add_sync(0xffffffffu, lane < warp ? sums : 0) + x - mine;
    const int share = max((total + int(gridDim.x) - 1) / int(gridDim.x), pl.item_cost + pl.min_tiles), snap = min(share / 8, pl.snap);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const long long cut = (long long)(share) * (blockIdx.x + k);
        if (cut < before || cut >= before + mine) continue;      // exactly one thread, or none behind the end
        const int at = int(cut);
        int s = before;
        for (int i = i0; i < i1; ++i) {
            const int w = per == 1 ? mine : item_weight(a, pl, i, false, tiles);
            if (at < s + w) {
                const int t = at - s - pl.item_cost;
                if (at - s <= snap || t < pl.min_tiles) { found[2 * k] = i; found[2 * k + 1] = 0; }
                else if (s + w - at <= snap || tiles - t < pl.min_tiles) { found[2 * k] = i + 1; found[2 * k + 1] = 0; }
                else {
                    found[2 * k] = i; found[2 * k + 1] = t;
                    if (chains) {                        // cuts number first to last fall into the item like this one
                        const int first = (s + max(snap, pl.item_cost + pl.min_tiles - 1)) / share + 1;
                        const int last = (s + w - max(snap, pl.min_tiles - 1) - 1) / share;
                        chains[2 * k] = first - 1; chains[2 * k + 1] = last - first + 2;
                    }
                }
                break;
            }
            s += w;
        }
    }
    __syncthreads();
    Share mine_now = {found[0], found[1], found[2], found[3], false};
    if (pl.drawn) {                                      // not where one item is more than a share
        most = __reduce_max_sync(0xffffffffu, lane < kThreads / 32 ? scratch[36 + lane] : 0);
        if (most <= share) mine_now = Share{-1, 0, pl.n_items, 0, true};
    }
    __syncthreads();                                     // the scratch is free again
    return mine_now;
}

// Draws of whole items from a counter in the status area: the first is the block's own number, later ones are looked at one
// item ahead.  The last block to finish leaves both counters at zero for the next call.
struct ItemDraw {
    int32_t* status; int n_items, ahead;
    __device__ __forceinline__ void init(int lane, int32_t* st, int n) {
        status = st; n_items = n; ahead = 0;
        if (lane == 0) ahead = int(gridDim.x) + atomicAdd(status + 8, 1);
    }
    __device__ __forceinline__ int next(int lane) {
        const int w = __shfl_sync(0xffffffffu, ahead, 0);
        if (w < n_items && lane == 0) ahead = int(gridDim.x) + atomicAdd(status + 8, 1);
        return w;
    }
    __device__ __forceinline__ void done() {             // one thread
        if (atomicAdd(status + 9, 1) == int(gridDim.x) - 1) { status[8] = 0; status[9] = 0; }
    }
};

__device__ __forceinline__ float rcpf(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 32 bytes at once (the address a multiple of 32)
__device__ __forceinline__ void st_global_32(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// two floats -> packed bf16 pair (lo in the low half), round to nearest even
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// whether the phase is complete, without waiting at all
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded wait like mbar_wait, for loops that wait several times per tile: the clock is looked at only now and then (the
// instruction itself suspends the thread for a while), and nothing is returned.  A wait that gives up raises the abort flag
// and lets the caller go on; the loops ask for the flag once per tile.
__device__ __forceinline__ void lean_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    if (mbar_try_wait(bar, parity)) return;
    unsigned long long t0 = 0;
    for (uint32_t i = 1;; ++i) {
        if (mbar_try_wait(bar, parity)) return;
        if (i % 16u == 0u) {
            if (*abort_flag) return;
            const unsigned long long now = global_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > kWaitLimitNs) { *abort_flag = 1; return; }
        }
    }
}
// the same for a whole warp, which goes on converged
__device__ __forceinline__ void warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    lean_wait(bar, parity, abort_flag);
    __syncwarp();
}
// whether the block has given up; the same answer in all lanes
__device__ __forceinline__ bool warp_aborted(volatile int* abort_flag) { return __any_sync(0xffffffffu, *abort_flag != 0); }

}  // namespace dev
}  // namespace csp
