// Chunk attention with up to sixteen query rows (token x head) per KV head: single tokens, and a few tokens at once.
// One pass over K and V, bound by HBM (512 bytes per cached row and KV head at d = 128); the products are far too thin
// for a tcgen05 row tile of 128, whose softmax would run on a quarter of one warp group.  Here the rows are the M of a
// warp-level m16n8k16 product and the keys of a tile are spread over the warps, so every thread has a few logits.
//
// Same organisation as the decode kernel: one CTA per SM stays resident and works off an equal share of all
// 64-key tiles of all units.
//   warp 8      producer: streams tiles of K and V with TMA (128-byte swizzle, no multicast) through a ring of
//               stages, puts the keys' positions and documents beside them and says with each stage which tile it
//               holds; an item ends with a stage without data
//   warps 0-3, 4-7  two groups that take turns, so that one computes while the other one's tile arrives.  A warp owns
//               16 keys of its group's tiles: S = Q K^T, modifiers and mask, running softmax with a lazily raised
//               reference, then P V with the weights as a bf16 head plus a bf16 remainder (two products per fragment),
//               so that only the result is rounded to bf16.  At the end of an item they leave their results in
//               shared memory and go on with the next one
//   warp 9      joins the eight results of an item in a fixed order: a whole unit is finished here, a cut one leaves a
//               partial result.  The query rows and what else an item needs come with its first stage, so that nobody
//               waits for memory between items
// Measured for one token, d = 128: 32 sequences x 32 heads, 410 - 1640 rows (530 MB) 102 us, 5.2 TB/s over all and 5.6 behind the
// first 7 us, when the first tiles arrive (the last block ends 14 % later than the average); 4 sequences of 8 K - 32 K rows,
// 28 / 4 heads with a bias (169 MB) 41.5 us, 4.1 TB/s over all and 4.9 behind the start, and 6 us for joining; one short
// sequence 8 us.
#include <limits.h>

#include "csp_chunk.cuh"

namespace csp {
namespace {
using namespace dev;

constexpr int kFewTile = 64;                             // keys per stage
constexpr int kFewWarps = 4;                             // warps of a group, 16 keys of a tile each
constexpr int kFewConsumers = 2 * kFewWarps;
constexpr int kFewProducer = kFewConsumers, kFewFinisher = kFewConsumers + 1;
constexpr int kFewThreads = 32 * (kFewConsumers + 2);
constexpr int kItemWords = 8;                            // of a stage's info: see ItemWord
enum ItemWord { kwItem, kwTile, kwRows, kwRow0, kwCount, kwPrefix, kwPart, kwPosRef };
constexpr int kFewBlock = kFewTile * 128;                // bytes of one 64-column block of a tile

struct FewQuery { const uint16_t* q; int64_t sb, sh, st; };

__device__ __forceinline__ void ldsm_x4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}

template <int NH, int RH>
struct FewShape {
    static constexpr int D = 64 * NH, R = 8 * RH;
    static constexpr int kStages = NH == 2 ? (RH == 2 ? 4 : 5) : (RH == 2 ? 7 : 8);                    // 32 KB each at d = 128
    static constexpr uint32_t kTileBytes = NH * kFewBlock, kStageBytes = 2 * kTileBytes;
    static constexpr uint32_t kMerge = kStages * kStageBytes;                          // [warp][R][D + 2] floats
    static constexpr uint32_t kQ = kMerge + kFewConsumers * R * (D + 2) * 4;           // per stage: R query rows
    static constexpr uint32_t kMeta = kQ + kStages * R * D * 2;                        // per stage: 64 positions, 64 documents
    static constexpr uint32_t kInfo = kMeta + kStages * kFewTile * 8;                  // per stage: what it holds; then: the item to finish
    static constexpr uint32_t kBars = kInfo + (kStages + 1) * kItemWords * 4;          // full, empty, results there, results read
    static constexpr uint32_t kMisc = kBars + (2 * kStages + 2) * 8;
    static constexpr uint32_t kTotal = kMisc + 16;
};

template <int NH, int RH>   // head_dim = 64 NH, 8 RH query rows
__global__ void __launch_bounds__(kFewThreads, 1)
chunk_few_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const ChunkArgs a,
                 const ChunkPlan pl, const FewQuery qy, ChunkParts* const parts, float* const partial, float2* const partial_ml) {
    using Shape = FewShape<NH, RH>;
    constexpr int D = Shape::D, R = Shape::R, NST = Shape::kStages;
    constexpr int KS = D / 16;                           // k-steps of S = Q K^T
    constexpr int NT = D / 8;                            // 8-column tiles of the output
    constexpr uint32_t kTileBytes = Shape::kTileBytes, kStageBytes = Shape::kStageBytes;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    float* const merge = reinterpret_cast<float*>(base_ptr + Shape::kMerge);
    const uint32_t full_bar = base + Shape::kBars, empty_bar = full_bar + 8 * NST;
    const uint32_t done_bar = empty_bar + 8 * NST, read_bar = done_bar + 8;
    int32_t* const info = reinterpret_cast<int32_t*>(base_ptr + Shape::kInfo);
    int32_t* const finish = info + NST * kItemWords;
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(base_ptr + Shape::kMisc);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = a.group;
    const ModArgs& md = a.mods;
    if (tid == 0) {
        *abort_flag = 0;
        for (int s = 0; s < NST; ++s) { mbar_init(full_bar + 8 * s, 1); mbar_init(empty_bar + 8 * s, kFewConsumers); }
        mbar_init(done_bar, kFewConsumers);
        mbar_init(read_bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    const Share share = find_share<kFewThreads>(a, pl, reinterpret_cast<int*>(merge));      // (synchronises)

    uint32_t fills = 0;                                  // of the ring, by this thread
    if (warp == kFewProducer) {
        // =============================== producer ===============================
        uint32_t it = 0;
        bool ok = true;
        int32_t word = 0;                                // lane l: word l of the current item's info
        auto stage = [&](int item, int tile) {           // the next stage, free, with what it holds written beside it
            const uint32_t s = it % NST;
            warp_wait(empty_bar + 8 * s, ((it / NST) & 1u) ^ 1u, abort_flag);
            ok = ok && !warp_aborted(abort_flag);
            if (!ok) return s;
            if (lane < kItemWords) info[s * kItemWords + lane] = lane == kwItem ? item : lane == kwTile ? tile : word;
            ++it;
            return s;
        };
        auto marker = [&](int item) {                    // a stage without data: the item has no more tiles (-1: no more items)
            const uint32_t s = stage(item, -1);
            __syncwarp();
            if (ok && lane == 0) mbar_arrive(full_bar + 8 * s);
        };
        if (lane == 0) parts[blockIdx.x] = ChunkParts{-1, 0};
        const uint32_t tiles_per_page = uint32_t(a.page_rows) / uint32_t(kFewTile);      // (dense: not used)
        auto page_of = [&](int b, int tile) {            // the page of a tile that lies inside the cache
            return a.page_table[int64_t(b) * a.max_pages + uint32_t(tile) / tiles_per_page];
        };
        constexpr int kQChunks = R * D / 8 / 32;
        uint4 next_q[kQChunks];
        PairRange next = {};
        int next_page = 0;                               // lane l: page of the next item's tile l (of its first 32)
        auto look_up = [&](int u) {                      // while the current item streams
            if (u > share.item1 || (u == share.item1 && share.tile1 == 0) || u >= pl.n_items) return;
            next = pair_range(a, pl, u, 0);
            const int tile = (u == share.item0 ? share.tile0 : 0) + lane;
            if (a.page_table && next.count > 0 && tile < next.tiles) next_page = page_of(u / a.n_kv_heads, tile);
            // the query rows: 16-byte chunk `lane + 32 j` of [row][d]; rows that are none are zeros
            const int b = u / a.n_kv_heads, h = u % a.n_kv_heads;
#pragma unroll
            for (int j = 0; j < kQChunks; ++j) {
                const int c = lane + 32 * j, m = c / (D / 8), tok = m / G;
                next_q[j] = tok < next.count ? *reinterpret_cast<const uint4*>(qy.q + int64_t(b) * qy.sb + int64_t(h * G + m % G) * qy.sh +
                                                                               int64_t(tok) * qy.st + c % (D / 8) * 8)
                                             : make_uint4(0, 0, 0, 0);
            }
        };
        look_up(share.item0);
        for (int u = share.item0; ok && u <= share.item1 && u < pl.n_items; ++u) {
            const int b = u / a.n_kv_heads, h = u % a.n_kv_heads;
            const PairRange x = next;
            int pages = next_page;                       // lane l: the page of tile 32 j + l
            const int tile0 = u == share.item0 ? share.tile0 : 0, tile1 = u == share.item1 ? share.tile1 : x.tiles;
            if (x.count <= 0 || (u == share.item1 && tile1 == 0)) { look_up(u + 1); continue; }
            if (lane == 0) {
                if (tile0 > 0) parts[blockIdx.x].last = tile1 == x.tiles;
                else if (tile1 < x.tiles) parts[blockIdx.x].first = u;
            }
            const int32_t* const docs = md.documents ? md.documents + int64_t(b) * md.doc_sb + int64_t(h) * md.doc_sh : nullptr;
            const int32_t* const poss = md.slopes && md.positions ? md.positions + int64_t(b) * md.pos_sb + int64_t(h) * md.pos_sh : nullptr;
            const bool meta = docs || md.slopes;
            // positions are staged relative to the last token's, so that near ones are exact in fp32
            const int row_last = max(x.row0 + x.count - 1, 0);
            const int pos_ref = md.slopes && x.rows > 0 ? (poss ? poss[row_last] : row_last) : 0;
            int doc_lo = INT_MAX, doc_hi = INT_MIN;
            if (docs) {                                  // sixteen rows at most
                const int r = x.row0 + lane;
                if (lane < x.count && r >= 0) doc_lo = doc_hi = docs[r];
                doc_lo = __reduce_min_sync(0xffffffffu, doc_lo);
                doc_hi = __reduce_max_sync(0xffffffffu, doc_hi);
            }
            // documents and positions of four tiles' keys at once, fetched before the first of them is needed
            int d_now[8], p_now[8];
            auto fetch_meta = [&](int tile) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int t = tile * kFewTile + lane + 32 * j;
                    d_now[j] = docs && t < x.rows ? docs[t] : 0;
                    p_now[j] = !md.slopes ? 0 : poss ? (t < x.rows ? poss[t] : pos_ref) : t;
                }
            };
            const int part_slot = tile0 > 0 ? 2 * int(blockIdx.x) : tile1 < x.tiles ? 2 * int(blockIdx.x) + 1 : -1;
            switch (lane) {
                case kwRows: word = x.rows; break;
                case kwRow0: word = x.row0; break;
                case kwCount: word = x.count; break;
                case kwPrefix: word = x.prefix; break;
                case kwPart: word = part_slot; break;
                case kwPosRef: word = pos_ref; break;
            }
            auto put_q = [&](uint32_t s) {
#pragma unroll
                for (int j = 0; j < kQChunks; ++j) *reinterpret_cast<uint4*>(base_ptr + Shape::kQ + s * R * D * 2 + (lane + 32 * j) * 16) = next_q[j];
            };
            bool looked = false;
            if (!meta) {
                // Without positions and documents one lane does everything from the second tile on: at the full rate of HBM a
                // tile is due every 1400 clocks, and the steps below take a whole warp as long as that.
                auto load = [&](uint32_t s, int tile, int outer) {
                    mbar_expect_tx(full_bar + 8 * s, kStageBytes);
                    const int row = a.page_table ? int(uint32_t(tile) % tiles_per_page) * kFewTile : tile * kFewTile;
                    tma_load_5d(base + s * kStageBytes, &tmap_k, full_bar + 8 * s, 0, row, 0, h, outer);
                    tma_load_5d(base + s * kStageBytes + kTileBytes, &tmap_v, full_bar + 8 * s, 0, row, 0, h, outer);
                };
                auto checked = [&](int page) {           // outside the pool: an out-of-range coordinate, zeros arrive
                    if (uint32_t(page) < uint32_t(a.n_pages)) return page;
                    atomicOr(a.status, CSP_DEV_BAD_LEN);
                    return a.n_pages;
                };
                if (tile0 < tile1) {
                    const uint32_t s = stage(u, tile0);
                    put_q(s);
                    __syncwarp();
                    if (ok && lane == 0) load(s, tile0, a.page_table ? checked(pages) : b);
                    looked = true;
                }
                const bool elected = elect_one();
                uint32_t issued = 0;                     // (of the elected lane: fewer than there are tiles if a wait runs out)
                if (elected && ok) {
                    int page = a.page_table && tile0 + 1 < tile1 ? page_of(b, tile0 + 1) : 0;
                    for (int tile = tile0 + 1; tile < tile1; ++tile, ++issued) {
                        const uint32_t n = it + issued, s = n % NST;
                        const int outer = a.page_table ? checked(page) : b;
                        if (a.page_table && tile + 1 < tile1) page = page_of(b, tile + 1);        // in time for the next tile
                        lean_wait(empty_bar + 8 * s, ((n / NST) & 1u) ^ 1u, abort_flag);
                        if (*abort_flag) break;
                        *reinterpret_cast<int2*>(info + s * kItemWords) = make_int2(u, tile);
                        load(s, tile, outer);
                    }
                }
                it += __reduce_max_sync(0xffffffffu, issued);
                look_up(u + 1);
                __syncwarp();
                ok = ok && !warp_aborted(abort_flag);
                marker(u);
                continue;
            }
            for (int tile = tile0; tile < tile1 && ok; ++tile) {
                const int turn = (tile - tile0) & 3;
                if (meta && turn == 0) fetch_meta(tile);
                if (a.page_table && tile > tile0 && ((tile - tile0) & 31) == 0) pages = tile + lane < tile1 ? page_of(b, tile + lane) : 0;
                int dd[2] = {0, 0}, pp[2] = {0, 0};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (turn == j) { dd[0] = d_now[2 * j]; dd[1] = d_now[2 * j + 1]; pp[0] = p_now[2 * j]; pp[1] = p_now[2 * j + 1]; }
                if (docs) {                              // a tile without any of the tokens' documents is skipped
                    bool hit = false;
#pragma unroll
                    for (int j = 0; j < 2; ++j) hit |= tile * kFewTile + lane + 32 * j < x.kv_end[1] && dd[j] >= doc_lo && dd[j] <= doc_hi;
                    if (!__any_sync(0xffffffffu, hit)) continue;
                }
                int outer = b, row = tile * kFewTile;
                if (a.page_table) {
                    // a page number outside the pool becomes an out-of-range coordinate: zeros arrive, nothing faults
                    outer = __shfl_sync(0xffffffffu, pages, (tile - tile0) & 31);
                    if (outer < 0 || outer >= a.n_pages) {
                        if (lane == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
                        outer = a.n_pages;
                    }
                    row = int(uint32_t(tile) % tiles_per_page) * kFewTile;
                }
                const uint32_t s = stage(u, tile);
                if (!looked) put_q(s);
                if (meta) {
                    float* const mp = reinterpret_cast<float*>(base_ptr + Shape::kMeta + s * kFewTile * 8);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        mp[lane + 32 * j] = float(pp[j] - pos_ref);
                        reinterpret_cast<int32_t*>(mp)[kFewTile + lane + 32 * j] = dd[j];
                    }
                }
                __syncwarp();
                if (ok && lane == 0) {
                    mbar_expect_tx(full_bar + 8 * s, kStageBytes);
                    tma_load_5d(base + s * kStageBytes, &tmap_k, full_bar + 8 * s, 0, row, 0, h, outer);
                    tma_load_5d(base + s * kStageBytes + kTileBytes, &tmap_v, full_bar + 8 * s, 0, row, 0, h, outer);
                }
                if (!looked) { look_up(u + 1); looked = true; }
            }
            if (!looked) look_up(u + 1);
            marker(u);
        }
        if (ok) marker(-1);
        if (lane == 0) fills = it;
    } else if (warp == kFewFinisher) {
        // =============================== finisher ===============================
        for (uint32_t n = 0;; ++n) {
            warp_wait(done_bar, n & 1u, abort_flag);
            if (warp_aborted(abort_flag)) break;
            const int u = finish[kwItem], count = finish[kwCount], part_slot = finish[kwPart];
            if (u < 0) break;
            const int b = u / a.n_kv_heads, h = u % a.n_kv_heads;
            const bool final = part_slot < 0;
            constexpr int C = D / 32;                    // columns per lane
            for (int m = 0; m < count * G; ++m) {
                float2 st[kFewConsumers];
                float mm = kNeg;
#pragma unroll
                for (int ww = 0; ww < kFewConsumers; ++ww) {
                    st[ww] = *reinterpret_cast<const float2*>(merge + (ww * R + m) * (D + 2) + D);
                    mm = fmaxf(mm, st[ww].x);
                }
                float l = 0.f, o[C];
#pragma unroll
                for (int c = 0; c < C; ++c) o[c] = 0.f;
#pragma unroll
                for (int ww = 0; ww < kFewConsumers; ++ww) {
                    const float wgt = ex2f(st[ww].x - mm);
                    l += st[ww].y * wgt;
#pragma unroll
                    for (int c = 0; c < C; c += 2) {
                        const float2 y = *reinterpret_cast<const float2*>(merge + (ww * R + m) * (D + 2) + lane * C + c);
                        o[c] += y.x * wgt;
                        o[c + 1] += y.y * wgt;
                    }
                }
                const int tok = m / G, head = h * G + m % G;
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
        // =============================== consumer warps ===============================
        const int group = warp / kFewWarps, wi = warp % kFewWarps;
        const int gq = lane >> 2, qd = lane & 3;         // this thread's query row (and row + 8) and column pair
        // ldmatrix row addresses: lane l supplies row (l % 8) of matrix (l / 8)
        const int kr = wi * 16 + ((lane >> 4) << 3) + (lane & 7);      // K: matrices 2,3 are the second 8 rows
        const int kc = (lane >> 3) & 1;                                  //    matrices 1,3 the second 8 columns
        const int vr = wi * 16 + (((lane >> 3) & 1) << 3) + (lane & 7);  // V: matrices 1,3 are the second 8 rows
        const int vc = lane >> 4;                                        //    matrices 2,3 the next 8 columns
        const float scale2 = a.scale * kLog2e;
        const bool capped = md.softcap > 0.f;
        // capped: x = c tanh(o / c) = c - 2 c / (1 + e^{2 o / c}), all in the base-2 domain
        const float cap2 = md.softcap * kLog2e, cap_in = capped ? 2.f * kLog2e * a.scale / md.softcap : 0.f;
        uint32_t it = 0, n_tile = 0, n_done = 0;
        int item = -1, rows = 0;
        uint32_t qa[KS][4];
        float acc[NT][4];
        float m_run[RH], l_run[RH], q_pos[RH], slope2[RH];
        int lim[RH], q_doc[RH];
        for (;;) {
            const uint32_t s = it % NST;
            warp_wait(full_bar + 8 * s, (it / NST) & 1u, abort_flag);
            if (warp_aborted(abort_flag)) break;
            ++it;
            const int32_t* const in = info + s * kItemWords;
            const int w = in[kwItem], tile = in[kwTile];
            if (w != item && w >= 0) {
                item = w;
                rows = in[kwRows];
                const int row0 = in[kwRow0], count = in[kwCount], b = w / a.n_kv_heads, h = w % a.n_kv_heads;
                const int32_t* const docs = md.documents ? md.documents + int64_t(b) * md.doc_sb + int64_t(h) * md.doc_sh : nullptr;
                const int32_t* const poss = md.slopes && md.positions ? md.positions + int64_t(b) * md.pos_sb + int64_t(h) * md.pos_sh : nullptr;
#pragma unroll
                for (int rr = 0; rr < RH; ++rr) {
                    const int m = gq + 8 * rr, tok = m / G, head = h * G + m % G, r = row0 + tok;
                    const bool valid = tok < count, sees = valid && r >= 0;
                    const uint32_t* const qrow = reinterpret_cast<const uint32_t*>(base_ptr + Shape::kQ + s * R * D * 2 + m * D * 2);
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        qa[ks][rr] = qrow[ks * 8 + qd];
                        qa[ks][rr + 2] = qrow[ks * 8 + 4 + qd];
                    }
                    lim[rr] = !valid ? kSeesAll : sees ? max(r, in[kwPrefix] - 1) : -1;
                    q_doc[rr] = docs && sees ? docs[r] : 0;
                    q_pos[rr] = md.slopes && sees ? float((poss ? poss[r] : r) - in[kwPosRef]) : 0.f;
                    slope2[rr] = md.slopes && sees ? md.slopes[head] * kLog2e : 0.f;
                    m_run[rr] = kNeg;
                    l_run[rr] = 0.f;
                }
                if (RH == 1) {
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) qa[ks][1] = qa[ks][3] = 0u;
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.f;
            }
            if (tile >= 0) {
                if ((n_tile++ & 1u) != uint32_t(group)) {        // the other group's
                    __syncwarp();
                    if (lane == 0) mbar_arrive(empty_bar + 8 * s);
                    continue;
                }
                const uint32_t k_s = base + s * kStageBytes, v_s = k_s + kTileBytes;
                const int row_t = tile * kFewTile, row_w = row_t + wi * 16, r0 = row_w + 2 * qd;
                // what the modifiers need to know of this thread's four keys
                const float* const mp = reinterpret_cast<const float*>(base_ptr + Shape::kMeta + s * kFewTile * 8) + wi * 16 + 2 * qd;
                float2 pos[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                int2 doc[2] = {make_int2(0, 0), make_int2(0, 0)};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (md.slopes) pos[j] = *reinterpret_cast<const float2*>(mp + 8 * j);
                    if (md.documents) doc[j] = *reinterpret_cast<const int2*>(mp + kFewTile + 8 * j);
                }
                const float k_pos[4] = {pos[0].x, pos[0].y, pos[1].x, pos[1].y};
                const int k_doc[4] = {doc[0].x, doc[0].y, doc[1].x, doc[1].y};
                if (row_w + 16 > rows) {
                    // Rows past the end hold whatever the cache holds: their weights are zero, but zero times a
                    // non-finite value is not, so clear this warp's value rows beyond the end.
                    for (int j = lane; j < 16 * NH * 8; j += 32) {
                        const int r = wi * 16 + j / (NH * 8), c = j % (NH * 8);
                        if (row_t + r >= rows)
                            *reinterpret_cast<uint4*>(base_ptr + (v_s - base) + (c >> 3) * kFewBlock + r * 128 + (((c & 7) ^ (r & 7)) << 4)) =
                                make_uint4(0, 0, 0, 0);
                    }
                    __syncwarp();
                }
                // ---- S = Q K^T for 16 keys: two 8-key tiles
                float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int chunk = ks * 2 + kc;
                    uint32_t kb[4];
                    ldmatrix_x4(kb, k_s + (chunk >> 3) * kFewBlock + kr * 128 + (((chunk & 7) ^ (kr & 7)) << 4));
                    mma_bf16(s0, qa[ks], kb[0], kb[1]);
                    mma_bf16(s1, qa[ks], kb[2], kb[3]);
                }
                uint32_t ph[4] = {0u, 0u, 0u, 0u}, pr[4] = {0u, 0u, 0u, 0u};      // weights: bf16 head, bf16 remainder
#pragma unroll
                for (int rr = 0; rr < RH; ++rr) {
                    float xs[4] = {s0[2 * rr], s0[2 * rr + 1], s1[2 * rr], s1[2 * rr + 1]};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = r0 + (j & 1) + (j >> 1) * 8;
                        xs[j] = capped ? fmaf(-2.f * cap2, rcpf(1.f + ex2f(xs[j] * cap_in)), cap2) : xs[j] * scale2;
                        if (md.slopes) xs[j] = fmaf(-slope2[rr], fabsf(q_pos[rr] - k_pos[j]), xs[j]);
                        const bool sees = t <= lim[rr] && t < rows && (!md.documents || k_doc[j] == q_doc[rr]);
                        xs[j] = sees ? xs[j] : kNeg;
                    }
                    float mx = fmaxf(fmaxf(xs[0], xs[1]), fmaxf(xs[2], xs[3]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    if (mx > m_run[rr] + kLazy) {        // same decision in the four lanes of a row
                        const float alpha = ex2f(m_run[rr] - mx);
                        l_run[rr] *= alpha;
#pragma unroll
                        for (int t = 0; t < NT; ++t) { acc[t][2 * rr] *= alpha; acc[t][2 * rr + 1] *= alpha; }
                        m_run[rr] = mx;
                    }
                    float p[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) p[j] = xs[j] == kNeg ? 0.f : ex2f(xs[j] - m_run[rr]);
                    l_run[rr] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t hd = pack_bf16(p[2 * j], p[2 * j + 1]);
                        ph[rr + 2 * j] = hd;
                        pr[rr + 2 * j] = pack_bf16(p[2 * j] - __uint_as_float(hd << 16), p[2 * j + 1] - __uint_as_float(hd & 0xffff0000u));
                    }
                }
                // ---- acc += P V
#pragma unroll
                for (int t = 0; t < NT; t += 2) {
                    const int chunk = t + vc;
                    uint32_t vb[4];
                    ldsm_x4_t(vb, v_s + (chunk >> 3) * kFewBlock + vr * 128 + (((chunk & 7) ^ (vr & 7)) << 4));
                    mma_bf16(acc[t], ph, vb[0], vb[1]);
                    mma_bf16(acc[t], pr, vb[0], vb[1]);
                    mma_bf16(acc[t + 1], ph, vb[2], vb[3]);
                    mma_bf16(acc[t + 1], pr, vb[2], vb[3]);
                }
                if (row_w + 16 > rows) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(empty_bar + 8 * s);
                continue;
            }
            // ---- end of the item: this warp's rows to shared memory, once the finisher has read the previous ones
            if (n_done > 0) warp_wait(read_bar, (n_done - 1u) & 1u, abort_flag);
#pragma unroll
            for (int rr = 0; rr < RH; ++rr) {
                l_run[rr] += __shfl_xor_sync(0xffffffffu, l_run[rr], 1);
                l_run[rr] += __shfl_xor_sync(0xffffffffu, l_run[rr], 2);
                float* const mine = merge + (warp * R + gq + 8 * rr) * (D + 2);
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    *reinterpret_cast<float2*>(mine + t * 8 + 2 * qd) = make_float2(acc[t][2 * rr], acc[t][2 * rr + 1]);
                if (qd == 0) *reinterpret_cast<float2*>(mine + D) = make_float2(m_run[rr], l_run[rr]);
                if (md.slopes && w >= 0 && fabsf(q_pos[rr]) > kFarToken) atomicOr(a.status, CSP_DEV_BAD_LEN);
            }
            if (warp == 0 && lane < kItemWords) finish[lane] = in[lane];
            ++n_done;
            __syncwarp();
            if (lane == 0) { mbar_arrive(done_bar); mbar_arrive(empty_bar + 8 * s); }
            if (w < 0) break;                            // no more items: the finisher reads that too
        }
    }
    __syncwarp();
    __syncthreads();
    if (*abort_flag) {
        if (tid == 0) atomicOr(a.status, CSP_DEV_TIMEOUT);
        drain_ring(full_bar, fills, NST);
    }
}

template <int NH, int RH>
csp_status launch_few(const ChunkArgs& a, const ChunkPlan& pl, const FewQuery& q, const CUtensorMap& tk, const CUtensorMap& tv,
                      ChunkParts* parts, float* partial, float2* ml, cudaStream_t s) {
    constexpr int smem = int(FewShape<NH, RH>::kTotal) + 1024;
    static_assert(smem <= 227 * 1024, "shared memory of one CTA");
    auto kern = chunk_few_kernel<NH, RH>;
    static std::atomic<bool> configured[kMaxDevices];
    if (!raise_smem_limit(kern, smem, configured)) return CSP_ERR_CUDA;
    kern<<<pl.grid, kFewThreads, smem, s>>>(tk, tv, a, pl, q, parts, partial, ml);
    return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA;
}

}  // namespace

csp_status launch_chunk_few(const csp_params& p, const ChunkArgs& a, const ChunkPlan& pl, const csp_tensor& q,
                            const CUtensorMap& tk, const CUtensorMap& tv, ChunkParts* parts, float* partial, float2* ml,
                            cudaStream_t s) {
    const FewQuery qy = {static_cast<const uint16_t*>(q.ptr), q.stride_b, q.stride_h, q.stride_t};
    if (pl.row_slots <= 8)
        return p.head_dim == 64 ? launch_few<1, 1>(a, pl, qy, tk, tv, parts, partial, ml, s) : launch_few<2, 1>(a, pl, qy, tk, tv, parts, partial, ml, s);
    return p.head_dim == 64 ? launch_few<1, 2>(a, pl, qy, tk, tv, parts, partial, ml, s) : launch_few<2, 2>(a, pl, qy, tk, tv, parts, partial, ml, s);
}

}  // namespace csp
