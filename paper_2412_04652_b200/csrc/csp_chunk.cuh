// Shared by the two chunk attention kernels (csp_chunk.cu: many query rows per KV head, csp_chunk_few.cu: up to sixteen) and
// the kernel that joins the parts of a split cache.
#pragma once

#include "csp_device.cuh"
#include "csp_internal.cuh"

namespace csp {

struct ChunkPlan {                                       // sizes that host and device agree on
    int tok_tile;                                        // tokens in a row tile: 128 / G
    int n_pairs, splits, row_slots;                      // row pairs per unit, splits per pair, rows of a partial result
    int n_items;
    int key_tile, min_tiles;                             // keys per tile; tiles that a part of a split cache has at least
};

csp_status launch_chunk_few(const csp_params& p, const ChunkArgs& a, const ChunkPlan& pl, const csp_tensor& q,
                            const CUtensorMap& tk, const CUtensorMap& tv, float* partial, float2* ml, cudaStream_t s);

namespace dev {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kSeesAll = 1 << 30;

// What the rows of a pair look at.
struct PairRange {
    int rows, n_new, tok0, count;                        // rows of the unit, tokens of the sequence, first token, tokens here
    int row0, prefix;                                    // row of the first token; clamped prefix
    int kv_end[2];                                       // keys that row tile 0 / the whole pair can see: [0, kv_end)
    int tiles, per_split, active;
};
__device__ __forceinline__ PairRange pair_range(const ChunkArgs& a, const ChunkPlan& pl, int u, int pair) {
    PairRange x;
    const int b = u / a.n_kv_heads, h = u % a.n_kv_heads;
    x.rows = min(max(a.n_rows[u], 0), a.capacity);
    x.n_new = a.n_new ? min(max(a.n_new[b], 0), a.max_new) : a.max_new;
    x.tok0 = pair * 2 * pl.tok_tile;
    x.count = min(x.n_new - x.tok0, 2 * pl.tok_tile);
    x.row0 = x.rows - x.n_new + x.tok0;
    x.prefix = a.mods.prefix ? min(max(a.mods.prefix[int64_t(b) * a.mods.prefix_sb + int64_t(h) * a.mods.prefix_sh], 0), x.rows) : 0;
    const int last0 = x.row0 + min(x.count, pl.tok_tile) - 1, last1 = x.row0 + x.count - 1;
    x.kv_end[0] = last0 < 0 ? 0 : max(last0 + 1, x.prefix);
    x.kv_end[1] = last1 < 0 ? 0 : max(last1 + 1, x.prefix);
    x.tiles = (x.kv_end[1] + pl.key_tile - 1) / pl.key_tile;
    // a unit is divided by its own length, so that batches of any length below the capacity are spread evenly
    x.per_split = max(pl.min_tiles, (x.tiles + pl.splits - 1) / pl.splits);
    x.active = max(1, (x.tiles + x.per_split - 1) / x.per_split);
    return x;
}

// Draws of work items: the first is the block's own number, later ones come from a counter in the status area, looked at
// one item ahead.  The last block to finish leaves both counters at zero for the next call.
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
// two floats -> packed bf16 pair (lo in the low half), round to nearest even
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// bounded wait of a whole warp: all lanes come back with the same answer
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}

}  // namespace dev
}  // namespace csp
