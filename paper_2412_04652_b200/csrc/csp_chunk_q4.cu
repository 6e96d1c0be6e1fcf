// Attention of new tokens over pages held in 4 bits, up to sixteen query rows (token x head) per item.
//
// A row is base + scale code, so  <q, k_t> = scale_t <q, code_t> + base_t sum q  and
// sum_t p_t v_t = sum_t (p_t scale'_t) code'_t + sum_t p_t base'_t: the products see whole numbers, and what belongs to a row is
// applied to 32-bit sums.  The codes become operands without any arithmetic: four bits in the lowest places of a half are
// the number code 2^-24, in the next four places code 2^-20, both exactly (numbers below the smallest normal one), so a word
// of eight codes takes four ANDs and a shift.  The constant powers of two are put into the query (times 16 where the codes are the
// lower ones) and into the results.
//
// Keys are the M of the warp-level products and the query rows the N, so that eight rows cost one product where rows as M would
// pad them to sixteen:  S^T = K Q^T,  O^T = V^T P^T.  The transposed fragments fit each other up to one 8 x 8 transposition
// per eight keys and rows (movmatrix).  In the first product a lane takes 16 bytes of each of its keys, in whatever order the
// dimensions come (the query is laid out alike), in the second one 8 bytes, i.e. sixteen dimensions of four keys.
//
// Queries are scaled by a power of two, row by row, so that their largest value lies in [1, 2): a half holds every bf16
// value exactly from there down to 2^-14 of it.  A weight times its row's scale is rounded to a half (11 bits), relative to a power
// of two that follows the largest scale seen as the softmax's reference follows the largest logit.
//
// Organisation: one CTA per SM works off an equal share of all 64-key tiles.
//   producers    two warps stream tiles (codes and scales of K and V) with bulk copies into rings, one ring for each group of
//                two warps, and the items' queries and descriptions into a ring of their own
//   groups       take the tiles in turn, 32 keys per warp; at the end of an item every warp leaves its sums in shared memory
//   finisher     joins them in a fixed order
#include <limits.h>

#include "csp_chunk.cuh"

namespace csp {
namespace {
using namespace dev;

constexpr int kQ4Tile = 64;                              // keys per tile
constexpr int kItems = 3;                                // ring of items
constexpr int kItemWords = 8;
enum ItemWord { kwItem, kwRows, kwRow0, kwCount, kwPrefix, kwPart, kwPosRef, kwTok0 };
constexpr int kEndOfItem = 1;                            // in an entry's flags: the group has no more tiles of this item
constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;
constexpr float kTiny = 0x1p-126f, kHuge = 0x1p126f;     // bounds of the reference of the scales

struct FewQuery { const uint16_t* q; int64_t sb, sh, st; };

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ float lo_bf16(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

template <int NH, int RH>   // head_dim = 64 NH, 8 RH query rows
struct Q4Shape {
    static constexpr int D = 64 * NH, R = 8 * RH;
    static constexpr int NG = RH == 1 ? 8 : 4;           // groups of two warps
    static constexpr int NW = 2 * NG;
    static constexpr int kSlots = (RH == 1 ? 2 : 4) * (NH == 1 ? 2 : 1);               // tiles in flight per group
    static constexpr uint32_t kCodeBytes = kQ4Tile * D / 2, kScaleBytes = kQ4Tile * 4; // of K or of V
    static constexpr uint32_t kSlotBytes = 2 * kCodeBytes + 2 * kScaleBytes;
    static constexpr uint32_t kQRow = D * 2 + 16;                                      // padded: rows start in other banks
    static constexpr uint32_t kMerge = NG * kSlots * kSlotBytes;                       // [warp][R][D + 2] floats
    static constexpr uint32_t kMeta = kMerge + NW * R * (D + 2) * 4;                   // per slot: 64 positions, 64 documents
    static constexpr uint32_t kQ = kMeta + NG * kSlots * kQ4Tile * 8;                  // per item: R query rows,
    static constexpr uint32_t kRowConst = kQ + kItems * R * kQRow;                     //   [R] (factor of the logits, sum of q),
    static constexpr uint32_t kInfo = kRowConst + kItems * R * 8;                      //   words; then the item to finish
    static constexpr uint32_t kEntry = kInfo + (kItems + 1) * kItemWords * 4;          // [group][slot] int2: tile, flags
    static constexpr uint32_t kBars = kEntry + NG * kSlots * 8;
    static constexpr int kBarCount = 2 * NG * kSlots + 2 * kItems + 2;
    static constexpr uint32_t kFills = kBars + kBarCount * 8;
    static constexpr uint32_t kMisc = kFills + NG * 4;
    static constexpr uint32_t kTotal = kMisc + 16;
    static constexpr int kThreads = 32 * (NW + 3);
};

template <int NH, int RH>
__global__ void __launch_bounds__(Q4Shape<NH, RH>::kThreads, 1)
chunk_q4_few_kernel(const ChunkArgs a, const ChunkPlan pl, const FewQuery qy, const Q4Args cache, ChunkParts* const parts,
                    float* const partial, float2* const partial_ml) {
    using Shape = Q4Shape<NH, RH>;
    constexpr int D = Shape::D, R = Shape::R, NG = Shape::NG, NW = Shape::NW, NST = Shape::kSlots;
    constexpr int KW = D / 32;                           // words of a key that a lane has in the first product
    constexpr int VW = D / 64;                           // and in the second one
    constexpr int MT = D / 16;                           // 16-dimension tiles of the output

    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 127u) & ~127u;
    uint8_t* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    float* const merge = reinterpret_cast<float*>(base_ptr + Shape::kMerge);
    float2* const row_const = reinterpret_cast<float2*>(base_ptr + Shape::kRowConst);
    int32_t* const info = reinterpret_cast<int32_t*>(base_ptr + Shape::kInfo);
    int32_t* const finish = info + kItems * kItemWords;
    int2* const entry = reinterpret_cast<int2*>(base_ptr + Shape::kEntry);
    uint32_t* const fills = reinterpret_cast<uint32_t*>(base_ptr + Shape::kFills);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(base_ptr + Shape::kMisc);
    const uint32_t full_bar = base + Shape::kBars, empty_bar = full_bar + 8 * NG * NST;
    const uint32_t item_full = empty_bar + 8 * NG * NST, item_empty = item_full + 8 * kItems;
    const uint32_t done_bar = item_empty + 8 * kItems, read_bar = done_bar + 8;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = a.group;
    const ModArgs& md = a.mods;
    if (tid == 0) {
        *abort_flag = 0;
        for (int i = 0; i < NG * NST; ++i) { mbar_init(full_bar + 8 * i, 1); mbar_init(empty_bar + 8 * i, 2); }
        for (int i = 0; i < kItems; ++i) { mbar_init(item_full + 8 * i, 1); mbar_init(item_empty + 8 * i, NW); }
        mbar_init(done_bar, NW);
        mbar_init(read_bar, 1);
        for (int g = 0; g < NG; ++g) fills[g] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    const Share share = find_share<Shape::kThreads>(a, pl, reinterpret_cast<int*>(merge));      // (synchronises)

    if (warp >= NW + 1) {
        // =============================== producers ===============================
        // Both go over the same items; tile n of the block goes to group n % NG, and producer n & 1 brings it.
        const int me = warp - (NW + 1);
        bool ok = true;
        uint32_t n_tile = 0, n_item = 0;                 // tiles of all items before the current one; items
        // How many slots each group has been given, in 8 bits per group of this producer's.  Beyond 4 NST it goes on at 2 NST:
        // what tells the phases is the number modulo 2 NST.
        static_assert(NG <= 8 && 4 * NST < 256 && (NST & (NST - 1)) == 0, "counts in 8 bits");
        uint32_t given = 0;
        auto count_of = [&](int g) { return (given >> (8 * (g >> 1))) & 255u; };
        auto give = [&](int g) {
            const uint32_t n = count_of(g) + 1, sh = 8 * (g >> 1);
            given = (given & ~(255u << sh)) | ((n == 4 * NST ? 2 * NST : n) << sh);
        };
        auto slot_of = [&](int g) { return uint32_t(g) * NST + count_of(g) % NST; };
        auto phase_of = [&](int g) { return ((count_of(g) / NST) & 1u) ^ 1u; };
        auto wait = [&](uint32_t bar, uint32_t parity) {
            warp_wait(bar, parity, abort_flag);
            ok = ok && !warp_aborted(abort_flag);
        };
        auto marker = [&](int g, int tile, int flags) {  // a slot without data
            const uint32_t s = slot_of(g);
            wait(empty_bar + 8 * s, phase_of(g));
            if (!ok) return;
            if (lane == 0) { entry[s] = make_int2(tile, flags); mbar_arrive(full_bar + 8 * s); }
            give(g);
        };
        if (me == 0 && lane == 0) parts[blockIdx.x] = ChunkParts{-1, 0};
        const uint32_t tiles_per_page = uint32_t(a.page_rows) / uint32_t(kQ4Tile);
        auto page_of = [&](int b, int tile) {            // the page of a tile that lies inside the cache
            return a.page_table[int64_t(b) * a.max_pages + uint32_t(tile) / tiles_per_page];
        };
        constexpr int kRowLanes = D / 8;                 // lanes that hold a query row, eight values each
        constexpr int kQChunks = R * D / 8 / 32;
        uint4 next_q[kQChunks];
        PairRange next = {};
        int next_page = 0;                               // page of this producer's first tile of the next item
        auto my_first = [&](int tile0, uint32_t n0) { return tile0 + int((n0 ^ uint32_t(me)) & 1u); };
        auto look_up = [&](int item, uint32_t n0) {      // while the current item streams; n0: n_tile when it comes
            if (item > share.item1 || (item == share.item1 && share.tile1 == 0) || item >= pl.n_items) return;
            const int u = item / pl.n_pairs, b = u / a.n_kv_heads, h = u % a.n_kv_heads;
            next = pair_range(a, pl, u, item - u * pl.n_pairs);
            const int tile = my_first(item == share.item0 ? share.tile0 : 0, n0);
            if (next.count > 0 && tile < next.tiles) next_page = page_of(b, tile);
            if (me) return;
            // the query rows: 16-byte chunk `lane + 32 j` of [row][d]; rows that are none are zeros
#pragma unroll
            for (int j = 0; j < kQChunks; ++j) {
                const int c = lane + 32 * j, m = c / kRowLanes, tok = m / G;
                next_q[j] = tok < next.count ? *reinterpret_cast<const uint4*>(qy.q + int64_t(b) * qy.sb + int64_t(h * G + m % G) * qy.sh +
                                                                               int64_t(next.tok0 + tok) * qy.st + c % kRowLanes * 8)
                                             : make_uint4(0, 0, 0, 0);
            }
        };
        look_up(share.item0, 0);
        for (int item = share.item0; ok && item <= share.item1 && item < pl.n_items; ++item) {
            const int u = item / pl.n_pairs, b = u / a.n_kv_heads, h = u % a.n_kv_heads;
            const PairRange x = next;
            const int tile0 = item == share.item0 ? share.tile0 : 0, tile1 = item == share.item1 ? share.tile1 : x.tiles;
            if (x.count <= 0 || (item == share.item1 && tile1 == 0)) { look_up(item + 1, n_tile); continue; }
            const int32_t* const docs = md.documents ? md.documents + int64_t(b) * md.doc_sb + int64_t(h) * md.doc_sh : nullptr;
            const int32_t* const poss = md.slopes && md.positions ? md.positions + int64_t(b) * md.pos_sb + int64_t(h) * md.pos_sh : nullptr;
            // positions are staged relative to the last token's, so that near ones are exact in fp32
            const int row_last = max(x.row0 + x.count - 1, 0);
            const int pos_ref = md.slopes && x.rows > 0 ? (poss ? poss[row_last] : row_last) : 0;
            if (me == 0) {
                // ---- the item's description and queries, in halves and in the order of the codes
                if (lane == 0) {
                    if (tile0 > 0) parts[blockIdx.x].last = tile1 == x.tiles;
                    else if (tile1 < x.tiles) parts[blockIdx.x].first = item;
                }
                const uint32_t is = n_item % kItems;
                wait(item_empty + 8 * is, ((n_item / kItems) & 1u) ^ 1u);
                if (!ok) break;
                int32_t word = 0;
                switch (lane) {
                    case kwItem: word = item; break;
                    case kwRows: word = x.rows; break;
                    case kwRow0: word = x.row0; break;
                    case kwCount: word = x.count; break;
                    case kwPrefix: word = x.prefix; break;
                    case kwPart: word = tile0 > 0 ? 2 * int(blockIdx.x) : tile1 < x.tiles ? 2 * int(blockIdx.x) + 1 : -1; break;
                    case kwPosRef: word = pos_ref; break;
                    case kwTok0: word = x.tok0; break;
                }
                if (lane < kItemWords) info[is * kItemWords + lane] = word;
#pragma unroll
                for (int j = 0; j < kQChunks; ++j) {
                    const int c = lane + 32 * j, m = c / kRowLanes;
                    const uint32_t w[4] = {next_q[j].x, next_q[j].y, next_q[j].z, next_q[j].w};
                    float f[8];
                    uint32_t top = 0;                    // bits of the row's largest magnitude
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        f[2 * k] = lo_bf16(w[k]); f[2 * k + 1] = hi_bf16(w[k]);
                        top = max(top, max((w[k] << 16) & 0x7fffffffu, w[k] & 0x7fff0000u));
                    }
#pragma unroll
                    for (int d = 1; d < kRowLanes; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
                    const uint32_t ex = top >> 23;       // 255: an infinity or NaN, the row is no number
                    const float down = ex == 255u ? 0.f : __uint_as_float((254u - ex) << 23);        // 2^-e (0: 2^127)
                    float sum = 0.f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) { f[k] *= down; sum += f[k]; }
#pragma unroll
                    for (int d = 1; d < kRowLanes; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                    const float up = ex == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(ex << 23);
                    *reinterpret_cast<uint4*>(base_ptr + Shape::kQ + (is * R + m) * Shape::kQRow + (c % kRowLanes) * 16) =
                        make_uint4(pack_f16(16.f * f[0], 16.f * f[4]), pack_f16(f[1], f[5]), pack_f16(16.f * f[2], 16.f * f[6]), pack_f16(f[3], f[7]));
                    // logit = up 2^20 (scale S + base sum 2^-20), S the product with codes 2^-20
                    if (c % kRowLanes == 0) row_const[is * R + m] = make_float2(a.scale * kLog2e * 0x1p20f * up, sum * 0x1p-20f);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(item_full + 8 * is);
                ++n_item;
            }
            // ---- its tiles
            uint32_t ended = 0;                          // bit g: the group has been told that it has no more
            const uint8_t* const k_from = cache.k + h * cache.k_sh, * const v_from = cache.v + h * cache.v_sh;
            const uint8_t* const ks_from = cache.ks + h * cache.ks_sh, * const vs_from = cache.vs + h * cache.vs_sh;
            auto load = [&](uint32_t s, int64_t page, uint32_t tile) {       // one thread
                const int64_t row = int64_t(tile % tiles_per_page) * kQ4Tile;
                const uint32_t bar = full_bar + 8 * s, to = base + s * Shape::kSlotBytes;
                mbar_expect_tx(bar, Shape::kSlotBytes);
                bulk_load(to, k_from + page * cache.k_sb + row * (D / 2), Shape::kCodeBytes, bar);
                bulk_load(to + Shape::kCodeBytes, v_from + page * cache.v_sb + row * (D / 2), Shape::kCodeBytes, bar);
                bulk_load(to + 2 * Shape::kCodeBytes, ks_from + page * cache.ks_sb + row * 4, Shape::kScaleBytes, bar);
                bulk_load(to + 2 * Shape::kCodeBytes + Shape::kScaleBytes, vs_from + page * cache.vs_sb + row * 4, Shape::kScaleBytes, bar);
            };
            // a page outside the pool: rows of zeros, whatever their codes
            auto blank = [&](uint32_t s, int from, int step) {
                uint32_t* const sc = reinterpret_cast<uint32_t*>(base_ptr + s * Shape::kSlotBytes + 2 * Shape::kCodeBytes);
                for (int j = from; j < 2 * kQ4Tile; j += step) sc[j] = 0u;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            };
            const int first = my_first(tile0, n_tile);
            if (!docs && !md.slopes) {
                // Without positions and documents one lane does everything: at the full rate of HBM each producer has a tile to
                // bring every 750 clocks, and a whole warp takes longer for the steps below.
                const bool elected = elect_one();
                if (elected) {
                    int page = next_page;
                    for (int tile = first; tile < tile1; tile += 2) {
                        const int g = int((n_tile + uint32_t(tile - tile0)) % NG), now = page;
                        if (tile + 2 < tile1) page = page_of(b, tile + 2);        // in time for the next tile
                        const uint32_t s = slot_of(g);
                        lean_wait(empty_bar + 8 * s, phase_of(g), abort_flag);
                        if (*abort_flag) break;
                        const bool last = tile + NG >= tile1;
                        entry[s] = make_int2(tile, last ? kEndOfItem : 0);
                        if (uint32_t(now) < uint32_t(a.n_pages)) {
                            load(s, now, tile);
                        } else {
                            atomicOr(a.status, CSP_DEV_BAD_LEN);
                            blank(s, 0, 1);
                            mbar_arrive(full_bar + 8 * s);
                        }
                        give(g);
                        if (last) ended |= 1u << g;
                    }
                }
                const uint32_t who = __ballot_sync(0xffffffffu, elected), from = __ffs(who) - 1;
                given = __shfl_sync(0xffffffffu, given, from);
                ended = __shfl_sync(0xffffffffu, ended, from);
                ok = ok && !warp_aborted(abort_flag);
                n_tile += tile1 > tile0 ? tile1 - tile0 : 0;
                look_up(item + 1, n_tile);
            } else {
                int doc_lo = INT_MAX, doc_hi = INT_MIN;
                if (docs) {                              // sixteen rows at most
                    const int r = x.row0 + lane;
                    if (lane < x.count && r >= 0) doc_lo = doc_hi = docs[r];
                    doc_lo = __reduce_min_sync(0xffffffffu, doc_lo);
                    doc_hi = __reduce_max_sync(0xffffffffu, doc_hi);
                }
                int d_next[2] = {0, 0}, p_next[2] = {0, 0}, page_next = 0;
                auto fetch = [&](int tile) {             // a tile's page, documents and positions, one step ahead of their use
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int t = tile * kQ4Tile + lane + 32 * j;
                        d_next[j] = docs && t < x.rows ? docs[t] : 0;
                        p_next[j] = !md.slopes ? 0 : poss ? (t < x.rows ? poss[t] : pos_ref) : t;
                    }
                    page_next = page_of(b, tile);
                };
                // (with documents every tile is looked at, by both: who takes which depends on how many were skipped)
                const int step = docs ? 1 : 2;
                uint32_t n = n_tile;
                int tile = docs ? tile0 : first;
                if (tile < tile1) fetch(tile);
                for (; tile < tile1 && ok; tile += step) {
                    const int dd[2] = {d_next[0], d_next[1]}, pp[2] = {p_next[0], p_next[1]}, page = page_next;
                    if (tile + step < tile1) fetch(tile + step);
                    if (docs) {                          // a tile without any of the tokens' documents is skipped
                        bool hit = false;
#pragma unroll
                        for (int j = 0; j < 2; ++j) hit |= tile * kQ4Tile + lane + 32 * j < x.kv_end[1] && dd[j] >= doc_lo && dd[j] <= doc_hi;
                        if (!__any_sync(0xffffffffu, hit)) continue;
                        if ((n++ & 1u) != uint32_t(me)) continue;
                    }
                    const int g = int((docs ? n - 1 : n_tile + uint32_t(tile - tile0)) % NG);
                    // (with documents nobody knows yet which tile is the last)
                    const bool last = !docs && tile + NG >= tile1;
                    const uint32_t s = slot_of(g);
                    wait(empty_bar + 8 * s, phase_of(g));
                    if (!ok) break;
                    if (last) ended |= 1u << g;
                    float* const mp = reinterpret_cast<float*>(base_ptr + Shape::kMeta + s * kQ4Tile * 8);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        mp[lane + 32 * j] = float(pp[j] - pos_ref);
                        reinterpret_cast<int32_t*>(mp)[kQ4Tile + lane + 32 * j] = dd[j];
                    }
                    const bool there = uint32_t(page) < uint32_t(a.n_pages);
                    if (!there) blank(s, lane, 32);
                    __syncwarp();
                    if (elect_one()) {
                        entry[s] = make_int2(tile, last ? kEndOfItem : 0);
                        if (there) {
                            load(s, page, tile);
                        } else {
                            atomicOr(a.status, CSP_DEV_BAD_LEN);
                            mbar_arrive(full_bar + 8 * s);
                        }
                    }
                    __syncwarp();
                    give(g);
                }
                n_tile = docs ? n : n_tile + (tile1 > tile0 ? tile1 - tile0 : 0);
                look_up(item + 1, n_tile);
            }
            for (int g = me; g < NG && ok; g += 2)
                if (!(ended >> g & 1u)) marker(g, -1, kEndOfItem);
        }
        for (int g = me; g < NG && ok; g += 2) marker(g, -2, 0);       // no more items
        if (lane == 0)
            for (int g = me; g < NG; g += 2) fills[g] = count_of(g);
    } else if (warp == NW) {
        // =============================== finisher ===============================
        for (uint32_t n = 0;; ++n) {
            warp_wait(done_bar, n & 1u, abort_flag);
            if (warp_aborted(abort_flag)) break;
            const int item = finish[kwItem], count = finish[kwCount], part_slot = finish[kwPart], tok0 = finish[kwTok0];
            if (item < 0) break;
            const int u = item / pl.n_pairs, b = u / a.n_kv_heads, h = u % a.n_kv_heads;
            const bool final = part_slot < 0;
            constexpr int C = D / 32;                    // columns per lane
            for (int m = 0; m < count * G; ++m) {
                float2 st[NW];
                float mm = kNeg;
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    st[w] = *reinterpret_cast<const float2*>(merge + (w * R + m) * (D + 2) + D);
                    mm = fmaxf(mm, st[w].x);
                }
                float l = 0.f, o[C];
#pragma unroll
                for (int c = 0; c < C; ++c) o[c] = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const float wgt = ex2f(st[w].x - mm);
                    l += st[w].y * wgt;
#pragma unroll
                    for (int c = 0; c < C; c += 2) {
                        const float2 y = *reinterpret_cast<const float2*>(merge + (w * R + m) * (D + 2) + lane * C + c);
                        o[c] += y.x * wgt;
                        o[c + 1] += y.y * wgt;
                    }
                }
                const int tok = tok0 + m / G, head = h * G + m % G;
                if (final) {
                    const float inv = l == 0.f ? 0.f : 1.f / (n_term(a.n, mm) + l);      // l == 0: nothing was seen
                    uint32_t* const out = reinterpret_cast<uint32_t*>(a.out + int64_t(b) * a.o_sb + int64_t(head) * a.o_sh + int64_t(tok) * a.o_st + lane * C);
#pragma unroll
                    for (int c = 0; c < C; c += 2) out[c / 2] = l == 0.f ? 0u : pack_bf16(o[c] * inv, o[c + 1] * inv);
                    if (a.lse && lane == 0)
                        a.lse[(int64_t(b) * a.n_kv_heads * G + head) * a.max_new + tok] = l == 0.f ? -INFINITY : (mm + log2f(l)) * kLn2;
                } else {
                    const int64_t slot = int64_t(part_slot) * pl.row_slots;
#pragma unroll
                    for (int c = 0; c < C; c += 2) {     // laid out [column / 4][row][4]
                        const int col = lane * C + c;
                        *reinterpret_cast<float2*>(partial + (slot * (D / 4) + int64_t(col / 4) * pl.row_slots + m) * 4 + col % 4) =
                            make_float2(o[c], o[c + 1]);
                    }
                    if (lane == 0) partial_ml[slot + m] = make_float2(mm, l);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(read_bar);        // the area may be written again
        }
    } else {
        // =============================== groups ===============================
        const int group = warp >> 1, wi = warp & 1;
        const int gr = lane >> 2, qd = lane & 3;         // fragment row (a key, then dimensions) and column pair (query rows)
        // Which key of eight is fragment row i: i with the pairs (2, 3) and (6, 7) exchanged, so that the four keys that the
        // lanes of a half warp read together in the second product start in two halves of the banks, not in one.
        const int key_r = gr ^ ((gr >> 1) & 1);
        const int key_0 = 2 * qd + (qd & 1), key_1 = 2 * qd + 1 - (qd & 1);
        const bool capped = md.softcap > 0.f;
        // capped: x = c tanh(o / c) = c - 2 c / (1 + e^{2 o / c}), all in the base-2 domain
        const float cap2 = md.softcap * kLog2e, cap_in = capped ? 2.f / md.softcap : 0.f;
        uint32_t it = 0, n_item = 0;
        bool fresh = true;
        int rows = 0, live_rows = 0, lim_all = 0;
        uint32_t qb[RH][2 * KW][2];
        float acc[RH][MT][4];
        float factor[RH][2], q_sum[RH][2], m_run[RH][2], l_run[RH][2], b_run[RH][2], q_pos[RH][2], slope2[RH][2];
        int lim[RH][2], q_doc[RH][2];
        float v_ref = kTiny, v_inv = 1.f / kTiny;        // power of two that the scales of V are relative to
        for (;;) {
            const uint32_t s = group * NST + it % NST;
            warp_wait(full_bar + 8 * s, (it / NST) & 1u, abort_flag);
            if (warp_aborted(abort_flag)) break;
            ++it;
            const int2 en = entry[s];
            const int tile = en.x;
            if (tile == -2) {
                if (n_item > 0) warp_wait(read_bar, (n_item - 1u) & 1u, abort_flag);
                if (warp == 0 && lane == 0) finish[kwItem] = -1;
                __syncwarp();
                if (lane == 0) mbar_arrive(done_bar);
                break;
            }
            const uint32_t is = n_item % kItems;
            const int32_t* const in = info + is * kItemWords;
            if (fresh) {
                fresh = false;
                warp_wait(item_full + 8 * is, (n_item / kItems) & 1u, abort_flag);
                rows = in[kwRows];
                const int item = in[kwItem], row0 = in[kwRow0], count = in[kwCount], u = item / pl.n_pairs, b = u / a.n_kv_heads, h = u % a.n_kv_heads;
                live_rows = count * G;
                const int32_t* const docs = md.documents ? md.documents + int64_t(b) * md.doc_sb + int64_t(h) * md.doc_sh : nullptr;
                const int32_t* const poss = md.slopes && md.positions ? md.positions + int64_t(b) * md.pos_sb + int64_t(h) * md.pos_sh : nullptr;
                lim_all = kSeesAll;
#pragma unroll
                for (int n = 0; n < RH; ++n) {
                    const uint8_t* const qrow = base_ptr + Shape::kQ + (is * R + 8 * n + gr) * Shape::kQRow + qd * KW * 16;
#pragma unroll
                    for (int w = 0; w < KW; ++w) {
                        const uint4 y = *reinterpret_cast<const uint4*>(qrow + 16 * w);
                        qb[n][2 * w][0] = y.x; qb[n][2 * w][1] = y.y; qb[n][2 * w + 1][0] = y.z; qb[n][2 * w + 1][1] = y.w;
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int m = 8 * n + 2 * qd + c, tok = m / G, head = h * G + m % G, r = row0 + tok;
                        const bool valid = tok < count, sees = valid && r >= 0;
                        const float2 rc = row_const[is * R + m];
                        factor[n][c] = rc.x;
                        q_sum[n][c] = rc.y;
                        // rows that nobody asked for see everything: they must not send their warp through the masked path
                        lim[n][c] = !valid ? kSeesAll : sees ? max(r, in[kwPrefix] - 1) : -1;
                        lim_all = min(lim_all, lim[n][c]);
                        q_doc[n][c] = docs && sees ? docs[r] : 0;
                        q_pos[n][c] = md.slopes && sees ? float((poss ? poss[r] : r) - in[kwPosRef]) : 0.f;
                        slope2[n][c] = md.slopes && sees ? md.slopes[head] * kLog2e : 0.f;
                        m_run[n][c] = kNeg;
                        l_run[n][c] = b_run[n][c] = 0.f;
                    }
#pragma unroll
                    for (int t = 0; t < MT; ++t) acc[n][t][0] = acc[n][t][1] = acc[n][t][2] = acc[n][t][3] = 0.f;
                }
                lim_all = min(__reduce_min_sync(0xffffffffu, lim_all), rows - 1);
                v_ref = kTiny;
                v_inv = 1.f / kTiny;
            }
            if (tile >= 0) {
                const uint8_t* const k_s = base_ptr + s * Shape::kSlotBytes + wi * 32 * (D / 2);
                const uint8_t* const v_s = k_s + Shape::kCodeBytes;
                const uint32_t* const ks_s = reinterpret_cast<const uint32_t*>(base_ptr + s * Shape::kSlotBytes + 2 * Shape::kCodeBytes) + wi * 32;
                const uint32_t* const vs_s = ks_s + kQ4Tile;
                const int t0 = tile * kQ4Tile + wi * 32;
                // ---- S^T = K Q^T for 32 keys: two blocks of sixteen
                float x[2][RH][4];
                float k_scale[2][2], k_base[2][2], v_scale[2][2], v_base[2][2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    uint32_t kw[2][KW];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int key = 16 * k + 8 * i + key_r;
                        const uint32_t sk = t0 + key < rows ? ks_s[key] : 0u, sv = t0 + key < rows ? vs_s[key] : 0u;
                        k_scale[k][i] = lo_bf16(sk); k_base[k][i] = hi_bf16(sk);
                        v_scale[k][i] = lo_bf16(sv); v_base[k][i] = hi_bf16(sv);
                        const uint8_t* const from = k_s + key * (D / 2) + qd * KW * 4;
                        if (KW == 4) {
                            const uint4 y = *reinterpret_cast<const uint4*>(from);
                            kw[i][0] = y.x; kw[i][1] = y.y; kw[i][KW - 2] = y.z; kw[i][KW - 1] = y.w;
                        } else {
                            const uint2 y = *reinterpret_cast<const uint2*>(from);
                            kw[i][0] = y.x; kw[i][1] = y.y;
                        }
                    }
#pragma unroll
                    for (int n = 0; n < RH; ++n) x[k][n][0] = x[k][n][1] = x[k][n][2] = x[k][n][3] = 0.f;
#pragma unroll
                    for (int w = 0; w < KW; ++w) {
                        const uint32_t y0 = kw[0][w], y1 = kw[1][w], z0 = y0 >> 8, z1 = y1 >> 8;
#pragma unroll
                        for (int n = 0; n < RH; ++n) {
                            mma_f16(x[k][n], y0 & kLow, y1 & kLow, y0 & kHigh, y1 & kHigh, qb[n][2 * w][0], qb[n][2 * w][1]);
                            mma_f16(x[k][n], z0 & kLow, z1 & kLow, z0 & kHigh, z1 & kHigh, qb[n][2 * w + 1][0], qb[n][2 * w + 1][1]);
                        }
                    }
                }
                // ---- logits (base 2) of keys 8 i + key_r of block k and query rows 2 qd + c
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int n = 0; n < RH; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int i = j >> 1, c = j & 1;
                            x[k][n][j] = fmaf(k_scale[k][i], x[k][n][j], k_base[k][i] * q_sum[n][c]) * factor[n][c];
                        }
                if (capped || md.slopes) {
                    const float* const mp = reinterpret_cast<const float*>(base_ptr + Shape::kMeta + s * kQ4Tile * 8) + wi * 32;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float pos = md.slopes ? mp[16 * k + 8 * i + key_r] : 0.f;
#pragma unroll
                            for (int n = 0; n < RH; ++n)
#pragma unroll
                                for (int c = 0; c < 2; ++c) {
                                    float& y = x[k][n][2 * i + c];
                                    if (capped) y = fmaf(-2.f * cap2, rcpf(1.f + ex2f(y * cap_in)), cap2);
                                    if (md.slopes) y = fmaf(-slope2[n][c], fabsf(q_pos[n][c] - pos), y);
                                }
                        }
                }
                const bool masked = md.documents || t0 + 31 > lim_all;
                if (masked) {
                    const int32_t* const dp = reinterpret_cast<const int32_t*>(base_ptr + Shape::kMeta + s * kQ4Tile * 8) + kQ4Tile + wi * 32;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int key = 16 * k + 8 * i + key_r, t = t0 + key, doc = md.documents ? dp[key] : 0;
#pragma unroll
                            for (int n = 0; n < RH; ++n)
#pragma unroll
                                for (int c = 0; c < 2; ++c)
                                    if (t > lim[n][c] || t >= rows || (md.documents && doc != q_doc[n][c])) x[k][n][2 * i + c] = kNeg;
                        }
                }
                // ---- references: of the softmax per query row, of the scales per warp; raised when exceeded by 2^8 and 2^4
                const float v_top = fmaxf(fmaxf(v_scale[0][0], v_scale[0][1]), fmaxf(v_scale[1][0], v_scale[1][1]));
                float mx[RH][2];
                bool raise = v_top > 16.f * v_ref && v_ref < kHuge;
#pragma unroll
                for (int n = 0; n < RH; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        mx[n][c] = fmaxf(fmaxf(x[0][n][c], x[0][n][2 + c]), fmaxf(x[1][n][c], x[1][n][2 + c]));
                        raise = raise || mx[n][c] > m_run[n][c] + kLazy;
                    }
                if (__any_sync(0xffffffffu, raise)) {
                    // (the same power of two in all lanes; scales are not negative, so their bits are in order)
                    const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(fminf(fmaxf(v_top, v_ref), kHuge))) & 0x7f800000u;
                    const float v_new = __uint_as_float(top), shrink = v_ref * __uint_as_float((254u << 23) - top);
                    v_ref = v_new;
                    v_inv = __uint_as_float((254u << 23) - top);
#pragma unroll
                    for (int n = 0; n < RH; ++n)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float y = mx[n][c];
                            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 4));
                            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 8));
                            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 16));
                            float alpha = 1.f;
                            if (y > m_run[n][c] + kLazy) { alpha = ex2f(m_run[n][c] - y); m_run[n][c] = y; }
                            l_run[n][c] *= alpha;
                            b_run[n][c] *= alpha;
                            alpha *= shrink;
#pragma unroll
                            for (int t = 0; t < MT; ++t) { acc[n][t][c] *= alpha; acc[n][t][2 + c] *= alpha; }
                        }
                }
                // ---- weights
                uint32_t pb[2][RH][2];
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float sv = v_scale[k][i] * v_inv, bv = v_base[k][i];
#pragma unroll
                        for (int n = 0; n < RH; ++n) {
                            float w[2];
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                const float y = x[k][n][2 * i + c];
                                float p = ex2f(y - m_run[n][c]);
                                if (masked && y == kNeg) p = 0.f;
                                l_run[n][c] += p;
                                b_run[n][c] = fmaf(p, bv, b_run[n][c]);
                                w[c] = p * sv;
                            }
                            pb[k][n][i] = transpose8(pack_f16(w[0], w[1]));
                        }
                    }
                // ---- O^T += V^T P^T
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    uint32_t vw[4][VW];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = 16 * k + 8 * (i >> 1) + (i & 1 ? key_1 : key_0);
                        const uint8_t* const from = v_s + key * (D / 2) + gr * VW * 4;
                        if (VW == 2) {
                            const uint2 y = *reinterpret_cast<const uint2*>(from);
                            vw[i][0] = y.x; vw[i][VW - 1] = y.y;
                        } else {
                            vw[i][0] = *reinterpret_cast<const uint32_t*>(from);
                        }
                    }
#pragma unroll
                    for (int w = 0; w < VW; ++w)
#pragma unroll
                        for (int hf = 0; hf < 2; ++hf) {                 // values 0 - 3 and 4 - 7 of the word, of two keys each
                            const uint32_t y0 = __byte_perm(vw[0][w], vw[1][w], hf ? 0x7632 : 0x5410);
                            const uint32_t y1 = __byte_perm(vw[2][w], vw[3][w], hf ? 0x7632 : 0x5410);
                            const uint32_t z0 = y0 >> 8, z1 = y1 >> 8;
                            const int t = 4 * w + 2 * hf;
#pragma unroll
                            for (int n = 0; n < RH; ++n) {
                                mma_f16(acc[n][t], y0 & kLow, y0 & kHigh, y1 & kLow, y1 & kHigh, pb[k][n][0], pb[k][n][1]);
                                mma_f16(acc[n][t + 1], z0 & kLow, z0 & kHigh, z1 & kLow, z1 & kHigh, pb[k][n][0], pb[k][n][1]);
                            }
                        }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty_bar + 8 * s);
            if (!(en.y & kEndOfItem)) continue;
            // ---- end of the item: this warp's rows to shared memory, once the finisher has read the previous ones
            if (n_item > 0) warp_wait(read_bar, (n_item - 1u) & 1u, abort_flag);
#pragma unroll
            for (int n = 0; n < RH; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int m = 8 * n + 2 * qd + c;
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        l_run[n][c] += __shfl_xor_sync(0xffffffffu, l_run[n][c], d);
                        b_run[n][c] += __shfl_xor_sync(0xffffffffu, b_run[n][c], d);
                    }
                    if (md.slopes && fabsf(q_pos[n][c]) > kFarToken) atomicOr(a.status, CSP_DEV_BAD_LEN);
                    if (m >= live_rows) continue;
                    float* const mine = merge + (warp * R + m) * (D + 2);
#pragma unroll
                    for (int t = 0; t < MT; ++t)         // dimensions 2 t and 2 t + 1 of this lane's D / 8
                        *reinterpret_cast<float2*>(mine + gr * (D / 8) + 2 * t) =
                            make_float2(fmaf(acc[n][t][c] * 0x1p24f, v_ref, b_run[n][c]), fmaf(acc[n][t][2 + c] * 0x1p20f, v_ref, b_run[n][c]));
                    if (gr == 0) *reinterpret_cast<float2*>(mine + D) = make_float2(m_run[n][c], l_run[n][c]);
                }
            if (warp == 0 && lane < kItemWords) finish[lane] = in[lane];
            ++n_item;
            fresh = true;
            __syncwarp();
            if (lane == 0) { mbar_arrive(done_bar); mbar_arrive(item_empty + 8 * is); }
        }
    }
    __syncwarp();
    __syncthreads();
    if (*abort_flag && tid == 0) {
        atomicOr(a.status, CSP_DEV_TIMEOUT);
        for (int g = 0; g < NG; ++g) drain_ring(full_bar + 8 * NST * g, fills[g], NST);
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------

constexpr int kQ4Rows = 16;                              // query rows of an item at most

ChunkPlan chunk_q4_plan(const csp_params& p, int max_new) {
    ChunkPlan pl;
    const int G = p.n_q_heads / p.n_kv_heads;
    // (an item has 2 tok_tile tokens)
    pl.tok_tile = int64_t(max_new) * G <= kQ4Rows ? kQ4Rows : kQ4Rows / 2 / G;
    pl.drawn = false;
    pl.n_pairs = max_new / (2 * pl.tok_tile) + (max_new % (2 * pl.tok_tile) ? 1 : 0);
    if (pl.n_pairs < 1) pl.n_pairs = 1;
    pl.row_slots = (max_new < 2 * pl.tok_tile ? max_new : 2 * pl.tok_tile) * G;
    pl.key_tile = kQ4Tile;
    pl.min_tiles = 2;
    pl.item_cost = 2;
    pl.snap = 0x3fffffff;
    const int64_t items = int64_t(p.batch) * p.n_kv_heads * pl.n_pairs;
    const int64_t weight = (int64_t(p.out_capacity) + pl.key_tile - 1) / pl.key_tile + pl.item_cost;      // of an item, at most
    pl.n_items = items > 0x3fffffffLL / weight ? -1 : int(items);
    // no more blocks than there can be shares of the smallest size
    const int64_t most = (items > 65536 ? 65536 : items) * weight / (pl.item_cost + pl.min_tiles) + 1;
    pl.grid = most < sm_count() ? int(most) : sm_count();
    return pl;
}

template <int NH, int RH>
csp_status launch_few(const ChunkArgs& a, const ChunkPlan& pl, const FewQuery& q, const Q4Args& c, ChunkParts* parts, float* partial,
                      float2* ml, cudaStream_t s) {
    constexpr int smem = int(Q4Shape<NH, RH>::kTotal) + 128;
    static_assert(smem <= 227 * 1024, "shared memory of one CTA");
    auto kern = chunk_q4_few_kernel<NH, RH>;
    static std::atomic<bool> configured[kMaxDevices];
    if (!raise_smem_limit(kern, smem, configured)) return CSP_ERR_CUDA;
    kern<<<pl.grid, Q4Shape<NH, RH>::kThreads, smem, s>>>(a, pl, q, c, parts, partial, ml);
    return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA;
}

}  // namespace

size_t chunk_q4_workspace_bytes(const csp_params& p, int max_new) {
    if (p.dtype != CSP_BF16 || (p.head_dim != 64 && p.head_dim != 128)) return 0;
    if (p.out_capacity > (1 << 30)) return 0;                                    // a row index plus some tiles fits 32 bits
    if (int64_t(max_new) * (p.n_q_heads / p.n_kv_heads) > (1 << 24)) return 0;   // and so do a chunk's rows
    const ChunkPlan pl = chunk_q4_plan(p, max_new);
    if (pl.n_items < 0) return 0;                                                // key tiles are counted in 32 bits
    // enough for shorter chunks as well: the longest that is one item may have more rows in it
    const int few = kQ4Rows / (p.n_q_heads / p.n_kv_heads);
    const size_t mine = partial_layout(p, pl).total, shorter = partial_layout(p, chunk_q4_plan(p, max_new < few ? max_new : few)).total;
    return mine > shorter ? mine : shorter;
}

csp_status launch_chunk_q4(const csp_params& p, const ChunkArgs& a, const csp_tensor& q, const Q4Args& c, void* ws, cudaStream_t s) {
    const ChunkPlan pl = chunk_q4_plan(p, a.max_new);
    const PartialLayout lay = partial_layout(p, pl);
    ChunkParts* const parts = reinterpret_cast<ChunkParts*>(static_cast<char*>(ws) + lay.parts);
    float* const partial = reinterpret_cast<float*>(static_cast<char*>(ws) + lay.o);
    float2* const ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + lay.ml);
    const FewQuery qy = {static_cast<const uint16_t*>(q.ptr), q.stride_b, q.stride_h, q.stride_t};
    csp_status st;
    if (pl.row_slots <= 8)
        st = p.head_dim == 64 ? launch_few<1, 1>(a, pl, qy, c, parts, partial, ml, s) : launch_few<2, 1>(a, pl, qy, c, parts, partial, ml, s);
    else
        st = p.head_dim == 64 ? launch_few<1, 2>(a, pl, qy, c, parts, partial, ml, s) : launch_few<2, 2>(a, pl, qy, c, parts, partial, ml, s);
    // nothing is cut by a single block, and where two parts of min_tiles are more than a cache has
    if (st != CSP_OK || pl.grid == 1 || p.out_capacity <= (2 * pl.min_tiles - 1) * pl.key_tile) return st;
    return launch_chunk_join(p, a, pl, true, parts, partial, ml, s);
}

}  // namespace csp
