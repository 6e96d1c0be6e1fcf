// Attention of a chunk of new tokens over a dense or paged cache with the n-softmax normaliser (Eq. 5-7):
//   out[b, hq, i, :] = sum_t e^{o_t} / (n + sum_j e^{o_j}) v_t,   o_t = modified(scale <q_i, k_t>),   t visible to token i.
//
// One pass over the keys with a running reference m (base-2 exponent) and sum l per query row.  The G query heads that
// share a KV head and the tokens of the chunk together are the rows of a tcgen05 tile of 128: row = token * G + head,
// so a tile of keys is fetched once for all of them.  A work item is a pair of such row tiles (up to 256 rows) of one
// (sequence, KV head) unit against a range of 128-key tiles; one CTA per SM stays resident and draws items from a
// counter.  Where there are few items (few heads, few tokens, a long cache) the keys of a unit are split over several
// items, which leave un-normalised partial results for a second small kernel.
//
// Inside a CTA
//   warp 8      producer: looks up pages, streams K and V tiles (128-byte swizzle, TMA, no multicast) through a ring of
//               shared-memory stages, stages positions and documents of the keys, and tells the other warps through a
//               small ring of entries which tile comes next (so that whatever it skips is skipped by everybody)
//   warp 9      one thread issues tcgen05.mma: S_g = Q K^T (128 x 128, fp32 in tensor memory) and O_g += P_g V
//   warps 0-3, 4-7  two softmax groups g = 0, 1, one query row per thread.  A group reads its S from tensor memory,
//               applies modifiers and mask, and writes the weights as bf16 back over S, where the second product
//               reads them as its A operand; O stays in tensor memory.  The reference is raised only when a logit
//               exceeds it by more than 2^8, which is rare after the first tile, so the O rows are rescaled (by the
//               softmax thread itself) hardly ever.
// With more than 128 rows in an item, group g takes row tile g and both see every key tile; with fewer, both take the
// same rows and alternate over the key tiles (their results are joined when the item ends): either way one group's
// softmax runs while the tensor cores work for the other.
#include <limits.h>

#include "csp_chunk.cuh"
#include "csp_tc.cuh"

namespace csp {
namespace {
using namespace dev;

constexpr int kGroupWarps = 4;
constexpr int kSoftmaxWarps = 2 * kGroupWarps;
constexpr int kChProducerWarp = kSoftmaxWarps, kChMmaWarp = kSoftmaxWarps + 1;
constexpr int kChThreads = 32 * (kSoftmaxWarps + 4);      // registers are shared out by groups of four warps: two stay idle
// Registers per thread.  The kernel is launched with 168 (what 384 threads may have); the softmax threads hold a whole
// row of S (128) and take 216, the other four warps make do with 72: 2 * 128 * 216 + 128 * 72 = 384 * 168.
constexpr int kSoftmaxRegs = 216, kOtherRegs = 72;
constexpr int kEntries = 8;                              // ring of tile entries
constexpr int kEntryWords = 16;
constexpr int kMinTiles = 2;                             // no item of a split cache is shorter than one tile per group
constexpr uint32_t kUnset = 0xBF800000u;                 // -1.0f: no sum of weights has these bits

// what an entry says
enum EntryWord { kKind, kTile0, kAct, kSeq, kHead, kTok0, kRows, kNew, kSplit, kActive, kQSlots, kFirst, kPair, kPrefix };
enum EntryKind { kEntryTile, kEntryEnd, kEntryStop };

struct ChunkSmem { uint32_t q, meta, entries, ml, bars, misc, total; };
template <int NH, bool kMeta>
struct ChunkShape {
    static constexpr int kStages = NH == 2 ? (kMeta ? 4 : 5) : 8;
    static constexpr uint32_t kStageBytes = NH * kBlockBytes;            // one tile of K or of V
    static constexpr uint32_t kQBytes = NH * kBlockBytes;                // one row tile of Q
    static constexpr int kBars = 2 * kStages + 2 * kEntries + 4 + 6 + 2;
    __host__ __device__ static constexpr ChunkSmem plan() {
        ChunkSmem s = {};
        uint32_t off = uint32_t(kStages) * kStageBytes;
        s.q = off;       off += 2 * kQBytes;
        s.meta = off;    off += kMeta ? kEntries * 1024 : 0;             // [entry][128] positions, then documents
        s.entries = off; off += kEntries * kEntryWords * 4;
        s.ml = off;      off += 2 * 128 * 4;                             // one value per row and group, exchanged twice
        s.bars = off;    off += kBars * 8;
        s.misc = off;    off += 16;
        s.total = off;
        return s;
    }
};

template <int NH, bool kCap, bool kBias, bool kDoc>
__global__ void __launch_bounds__(kChThreads, 1)
chunk_attn_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                  const __grid_constant__ CUtensorMap tmap_v, const ChunkArgs a, const ChunkPlan pl,
                  float* const partial, float2* const partial_ml) {
    constexpr int D = 64 * NH;
    constexpr bool kMeta = kBias || kDoc;
    using Shape = ChunkShape<NH, kMeta>;
    constexpr int NST = Shape::kStages;
    constexpr uint32_t kStageBytes = Shape::kStageBytes;
    // S: 128 x 128, both operands K-major.  O: 128 x D, B (V) with its rows along K
    constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t(128 >> 3) << 17) | (uint32_t(128 >> 4) << 24);
    constexpr uint32_t kIdescO = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (uint32_t(D >> 3) << 17) | (uint32_t(128 >> 4) << 24);

    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    constexpr ChunkSmem sp = Shape::plan();
    int32_t* const entries = reinterpret_cast<int32_t*>(base_ptr + sp.entries);
    float* const ml = reinterpret_cast<float*>(base_ptr + sp.ml);
    const uint32_t kv_full = base + sp.bars, kv_empty = kv_full + 8 * NST;
    const uint32_t ent_full = kv_empty + 8 * NST, ent_empty = ent_full + 8 * kEntries;
    const uint32_t q_full = ent_empty + 8 * kEntries, q_empty = q_full + 16;      // [2] each
    const uint32_t s_full = q_empty + 16, p_full = s_full + 16, pv_done = p_full + 16;   // [2] each
    const uint32_t join_bar = pv_done + 16, drain_bar = join_bar + 8;
    volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + sp.misc);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(base_ptr + sp.misc + 4);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        *abort_flag = 0;
        for (int s = 0; s < NST; ++s) { mbar_init(kv_full + 8 * s, 1); mbar_init(kv_empty + 8 * s, 1); }
        for (int e = 0; e < kEntries; ++e) { mbar_init(ent_full + 8 * e, 1); mbar_init(ent_empty + 8 * e, kSoftmaxWarps + 1); }
        for (int g = 0; g < 2; ++g) {
            mbar_init(q_full + 8 * g, 1); mbar_init(q_empty + 8 * g, 1);
            mbar_init(s_full + 8 * g, 1); mbar_init(p_full + 8 * g, kGroupWarps); mbar_init(pv_done + 8 * g, 1);
        }
        mbar_init(join_bar, kSoftmaxWarps);
        mbar_init(drain_bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kChMmaWarp) {
        tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512u);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t tmem_o[2] = {tmem, tmem + 128u}, tmem_s[2] = {tmem + 256u, tmem + 384u};

    if (warp >= kSoftmaxWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == kChProducerWarp) {
        // =============================== producer ===============================
        uint32_t n_entry = 0, n_stage = 0, q_uses[2] = {0, 0}, n_small = 0;
        bool ok = true;
        auto publish = [&](int32_t word) {               // lane l < kEntryWords brings word l
            const uint32_t e = n_entry % kEntries;
            ok = ok && warp_wait(ent_empty + 8 * e, ((n_entry / kEntries) & 1u) ^ 1u, abort_flag);
            if (lane < kEntryWords) entries[e * kEntryWords + lane] = word;
            return e;
        };
        auto announce = [&](uint32_t e) {
            __syncwarp();
            if (ok && lane == 0) mbar_arrive(ent_full + 8 * e);
            ++n_entry;
        };
        ItemDraw draw;
        draw.init(lane, a.status, pl.n_items);
        int w = blockIdx.x;
        while (ok && w < pl.n_items) {
            const int w_now = w;
            w = draw.next(lane);
            const int split = w_now % pl.splits, up = w_now / pl.splits, pair = up % pl.n_pairs, u = up / pl.n_pairs;
            const int b = u / a.n_kv_heads, h = u % a.n_kv_heads;
            const PairRange x = pair_range(a, pl, u, pair);
            if (pair == 0 && split == 0 && lane == 0) {
                const int rows = a.n_rows[u], more = a.n_new ? a.n_new[b] : a.max_new;
                if (rows != x.rows || more != x.n_new || x.n_new > x.rows) atomicOr(a.status, CSP_DEV_BAD_LEN);
            }
            if (x.count <= 0 || split >= x.active) continue;
            const bool big = x.count > pl.tok_tile;      // more than one row tile
            const int tile0 = split * x.per_split, tile1 = min(x.tiles, tile0 + x.per_split);
            const int q_slots = big ? 3 : 1 << (n_small++ & 1u);     // which of the two Q slots: slot g for group g, or one for both
            const int32_t* const docs = kDoc ? a.mods.documents + int64_t(b) * a.mods.doc_sb + int64_t(h) * a.mods.doc_sh : nullptr;
            const int32_t* const poss = kBias && a.mods.positions ? a.mods.positions + int64_t(b) * a.mods.pos_sb + int64_t(h) * a.mods.pos_sh : nullptr;
            // positions are staged relative to the last token's, so that near ones are exact in fp32
            const int row_last = max(x.row0 + x.count - 1, 0);
            const int pos_ref = kBias && x.tiles > 0 ? (poss ? poss[row_last] : row_last) : 0;
            int doc_lo[2] = {INT_MAX, INT_MAX}, doc_hi[2] = {INT_MIN, INT_MIN};
            if (kDoc) {                                  // the documents of each row tile's tokens
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int i_end = min(x.count, (g + 1) * pl.tok_tile);
                    for (int i = max(g * pl.tok_tile, -x.row0) + lane; i < i_end; i += 32) {
                        const int d = docs[x.row0 + i];
                        doc_lo[g] = min(doc_lo[g], d);
                        doc_hi[g] = max(doc_hi[g], d);
                    }
                    doc_lo[g] = __reduce_min_sync(0xffffffffu, doc_lo[g]);
                    doc_hi[g] = __reduce_max_sync(0xffffffffu, doc_hi[g]);
                }
            }
            int32_t word = 0;                            // this lane's word of the entries of this item
            switch (lane) {
                case kSeq: word = b; break;
                case kHead: word = h; break;
                case kTok0: word = x.tok0; break;
                case kRows: word = x.rows; break;
                case kNew: word = x.n_new; break;
                case kSplit: word = split; break;
                case kActive: word = x.active; break;
                case kQSlots: word = q_slots; break;
                case kFirst: word = 1; break;
                case kPair: word = pair; break;
                case kPrefix: word = x.prefix; break;
            }
            int n_done = 0;
            bool q_loaded = false;
            auto load_q = [&] {
                q_loaded = true;
#pragma unroll
                for (int slot = 0; slot < 2; ++slot) {
                    if (!(q_slots >> slot & 1)) continue;
                    ok = ok && warp_wait(q_empty + 8 * slot, (q_uses[slot] & 1u) ^ 1u, abort_flag);
                    ++q_uses[slot];
                    if (ok && lane == 0) {
                        mbar_expect_tx(q_full + 8 * slot, uint32_t(NH * a.group * min(pl.tok_tile, a.max_new)) * 128u);
#pragma unroll
                        for (int hb = 0; hb < NH; ++hb)
                            tma_load_4d(base + sp.q + slot * Shape::kQBytes + hb * kBlockBytes, &tmap_q, q_full + 8 * slot,
                                        hb * 64, h * a.group, x.tok0 + (big ? slot * pl.tok_tile : 0), b);
                    }
                }
            };
            int pages = 0;                               // lane l: the page of tile 32 j + l
            int d_next[4] = {0, 0, 0, 0}, p_next[4] = {0, 0, 0, 0};
            auto fetch_meta = [&](int tile) {            // documents and positions of one tile's keys, a tile ahead of their use
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int t = tile * kTileKeys + lane + 32 * j;
                    if (t >= x.rows) { d_next[j] = 0; p_next[j] = 0; continue; }
                    if (kDoc) d_next[j] = docs[t];
                    if (kBias) p_next[j] = poss ? poss[t] : t;
                }
            };
            if (kMeta && tile0 < tile1) fetch_meta(tile0);
            for (int tile = tile0; tile < tile1 && ok; ++tile) {
                const int t0 = tile * kTileKeys;
                if (a.page_table && ((tile - tile0) & 31) == 0) {
                    const int mine = tile + lane;
                    pages = mine < tile1 ? a.page_table[int64_t(b) * a.max_pages + int64_t(mine) * kTileKeys / a.page_rows] : 0;
                }
                int d_now[4], p_now[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) { d_now[j] = d_next[j]; p_now[j] = p_next[j]; }
                if (kMeta && tile + 1 < tile1) fetch_meta(tile + 1);
                int act = 0;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    if (g == 1 && !big) continue;
                    const int end = big && g == 0 ? x.kv_end[0] : x.kv_end[1];
                    bool any = t0 < end;
                    if (kDoc) {                          // a tile without any of the tokens' documents is skipped
                        bool hit = false;
#pragma unroll
                        for (int j = 0; j < 4; ++j) hit |= t0 + lane + 32 * j < end && d_now[j] >= doc_lo[g] && d_now[j] <= doc_hi[g];
                        any = __any_sync(0xffffffffu, hit);
                    }
                    act |= any ? 1 << g : 0;
                }
                if (act == 0) continue;
                if (!big) act = 1 << (n_done & 1);       // the groups take turns
                const uint32_t e = publish(lane == kTile0 ? t0 : lane == kAct ? act : lane == kKind ? int(kEntryTile) : word);
                if (lane == kFirst) word = 0;
                if (kMeta) {
                    float* const mp = reinterpret_cast<float*>(base_ptr + sp.meta + e * 1024);
                    int32_t* const md = reinterpret_cast<int32_t*>(base_ptr + sp.meta + e * 1024 + 512);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (kBias) mp[lane + 32 * j] = float(p_now[j] - pos_ref);
                        if (kDoc) md[lane + 32 * j] = d_now[j];
                    }
                }
                announce(e);
                int outer = b, row = t0;
                if (a.page_table) {
                    // a page number outside the pool becomes an out-of-range coordinate: zeros arrive, nothing faults
                    outer = __shfl_sync(0xffffffffu, pages, (tile - tile0) & 31);
                    if (outer < 0 || outer >= a.n_pages) {
                        if (lane == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
                        outer = a.n_pages;
                    }
                    row = t0 % a.page_rows;
                }
#pragma unroll
                for (int which = 0; which < 2; ++which, ++n_stage) {
                    const uint32_t s = n_stage % NST;
                    ok = ok && warp_wait(kv_empty + 8 * s, ((n_stage / NST) & 1u) ^ 1u, abort_flag);
                    if (ok && lane == 0) {
                        mbar_expect_tx(kv_full + 8 * s, kStageBytes);
#pragma unroll
                        for (int hb = 0; hb < NH; ++hb)
                            tma_load_4d(base + s * kStageBytes + hb * kBlockBytes, which ? &tmap_v : &tmap_k, kv_full + 8 * s, hb * 64,
                                        row, h, outer);
                    }
                }
                // Q goes behind the first two tiles (which need no more than four stages): its slot may still be in use
                if (++n_done == 2) load_q();
            }
            if (n_done == 1) load_q();
            announce(publish(lane == kKind ? int(kEntryEnd) : lane == kAct ? (q_loaded ? 1 : 0) : word));
        }
        if (ok) announce(publish(lane == kKind ? int(kEntryStop) : 0));
        if (lane == 0) {
            if (!ok) {
                // let copies that were issued land before the CTA's shared memory is given up
                for (int s = 0; s < NST; ++s) {
                    const unsigned long long t0 = global_ns();
                    while (!mbar_try_wait(kv_full + 8 * s, 0) && !mbar_try_wait(kv_full + 8 * s, 1) && global_ns() - t0 < kWaitLimitNs / 8) {}
                }
                atomicOr(a.status, CSP_DEV_TIMEOUT);
            }
            draw.done();
        }
        __syncwarp();
    } else if (warp == kChMmaWarp) {
        // =============================== MMA issuer ===============================
        if (lane == 0) {
            uint32_t n_entry = 0, q_uses[2] = {0, 0}, n_p[2] = {0, 0};
            int n_tile = 0, pend[2] = {-1, -1};          // tiles so far; tile whose P V product a group still owes
            bool started[2] = {false, false};            // the group has a product in this item (O holds something)
            bool ok = true;
            auto product = [&](int g) {                  // O_g += P_g V of the owed tile
                const uint32_t n = 2u * uint32_t(pend[g]) + 1u, s = n % NST;
                ok = ok && mbar_wait(p_full + 8 * g, n_p[g] & 1u, abort_flag) && mbar_wait(kv_full + 8 * s, (n / NST) & 1u, abort_flag);
                ++n_p[g];
                if (!ok) return;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < kTileKeys / 16; ++k)
                    tc_mma_bf16_ts(tmem_o[g], tmem_s[g] + 8u * k, sw128_desc_mn(base + s * kStageBytes + 2048u * k, kBlockBytes), kIdescO,
                                   (k > 0 || started[g]) ? 1u : 0u);
                started[g] = true;
                tc_commit(pv_done + 8 * g);
                if (pend[g ^ 1] != pend[g]) tc_commit(kv_empty + 8 * s);     // nobody else waits for this tile of V
                pend[g] = -1;
            };
            while (ok) {
                const uint32_t e = n_entry % kEntries;
                ok = mbar_wait(ent_full + 8 * e, (n_entry / kEntries) & 1u, abort_flag);
                if (!ok) break;
                const volatile int32_t* const en = entries + e * kEntryWords;
                const int kind = en[kKind], act = en[kAct], q_slots = en[kQSlots], first = en[kFirst];
                mbar_arrive(ent_empty + 8 * e);
                ++n_entry;
                if (kind == kEntryStop) break;
                if (kind == kEntryTile) {
                    if (first) {
                        started[0] = started[1] = false;
#pragma unroll
                        for (int slot = 0; slot < 2; ++slot) {
                            if (!(q_slots >> slot & 1)) continue;
                            ok = ok && mbar_wait(q_full + 8 * slot, q_uses[slot] & 1u, abort_flag);
                            ++q_uses[slot];
                        }
                    }
                    const uint32_t n = 2u * uint32_t(n_tile), s = n % NST;
                    ok = ok && mbar_wait(kv_full + 8 * s, (n / NST) & 1u, abort_flag);
                    if (!ok) break;
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        if (!(act >> g & 1)) continue;
                        if (pend[g] >= 0) product(g);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t q_s = base + sp.q + uint32_t(q_slots == 3 ? g : q_slots >> 1) * Shape::kQBytes;
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint32_t off = uint32_t(k >> 2) * kBlockBytes + uint32_t(k & 3) * 32u;
                            tc_mma_bf16(tmem_s[g], sw128_desc(q_s + off), sw128_desc(base + s * kStageBytes + off), kIdescS, k > 0 ? 1u : 0u);
                        }
                        tc_commit(s_full + 8 * g);
                        pend[g] = n_tile;
                    }
                    tc_commit(kv_empty + 8 * s);
                    // a group that sits this tile out pays what it owes now: its tile of V must not hold up the ring
#pragma unroll
                    for (int g = 0; g < 2; ++g)
                        if (!(act >> g & 1) && pend[g] >= 0) product(g);
                    ++n_tile;
                } else {
#pragma unroll
                    for (int g = 0; g < 2; ++g)
                        if (pend[g] >= 0) product(g);
#pragma unroll
                    for (int slot = 0; slot < 2; ++slot)
                        if (act && (q_slots >> slot & 1)) tc_commit(q_empty + 8 * slot);
                }
            }
            // nothing may be in flight when the tensor memory goes back
            tc_commit(drain_bar);
            const unsigned long long t0 = global_ns();
            while (!mbar_try_wait(drain_bar, 0) && global_ns() - t0 < kWaitLimitNs / 8) {}
        }
        __syncwarp();
    }
    } else {
        // =============================== softmax groups ===============================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int g = warp / kGroupWarps, m = tid & 127, G = a.group;
        const uint32_t lane_base = uint32_t((warp & 3) * 32) << 16;
        const uint32_t my_s = tmem_s[g] + lane_base, my_o = tmem_o[g] + lane_base;
        const float scale2 = a.scale * kLog2e;
        // capped: x = c tanh(o / c) = c - 2 c / (1 + e^{2 o / c}), all in the base-2 domain
        const float cap2 = kCap ? a.mods.softcap * kLog2e : 0.f, cap_in = kCap ? 2.f * kLog2e * a.scale / a.mods.softcap : 0.f;
        uint32_t n_entry = 0, n_tile = 0, n_mine = 0, n_join = 0;
        float m_run = kNeg, l_run = 0.f;
        int lim = -1, q_doc = 0, in_item = 0;
        float q_pos = 0.f, slope2 = 0.f;
        bool valid = false, live = false;
        int tok = 0, head = 0;
        for (;;) {
            const uint32_t e = n_entry % kEntries;
            if (!warp_wait(ent_full + 8 * e, (n_entry / kEntries) & 1u, abort_flag)) break;
            const int32_t* const en = entries + e * kEntryWords;
            const int kind = en[kKind];
            if (kind == kEntryStop) break;
            const int t0 = en[kTile0], act = en[kAct], rows = en[kRows], q_slots = en[kQSlots], b = en[kSeq], h = en[kHead];
            const bool big = q_slots == 3;
            if (en[kFirst]) {
                // this thread's query row: token m / G of its row tile, head m % G
                const int n_new = en[kNew], local = m / G;
                head = h * G + m - local * G;
                tok = en[kTok0] + (big ? g * pl.tok_tile : 0) + local;
                valid = local < pl.tok_tile && tok < n_new;
                const int r = rows - n_new + tok;
                const bool sees = valid && r >= 0;
                // rows that nobody asked for see everything: they must not send their warp through the masked path
                lim = !valid ? kSeesAll : r >= 0 ? max(r, en[kPrefix] - 1) : -1;
                live = __any_sync(0xffffffffu, valid);
                m_run = kNeg;
                l_run = 0.f;
                in_item = 0;
                if (kDoc) q_doc = sees ? a.mods.documents[int64_t(b) * a.mods.doc_sb + int64_t(h) * a.mods.doc_sh + r] : 0;
                if (kBias) {
                    const int32_t* const poss = a.mods.positions ? a.mods.positions + int64_t(b) * a.mods.pos_sb + int64_t(h) * a.mods.pos_sh : nullptr;
                    const int row_last = max(rows - n_new + en[kTok0] + min(n_new - en[kTok0], 2 * pl.tok_tile) - 1, 0);
                    const int ref = rows > 0 ? (poss ? poss[row_last] : row_last) : 0;
                    q_pos = sees ? float((poss ? poss[r] : r) - ref) : 0.f;
                    slope2 = sees ? a.mods.slopes[head] * kLog2e : 0.f;
                }
            }
            if (kind == kEntryTile) {
                const uint32_t v_stage = 2u * n_tile + 1u;
                ++n_tile;
                if (!(act >> g & 1)) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(ent_empty + 8 * e);
                    ++n_entry;
                    continue;
                }
                if (t0 + kTileKeys > rows) {
                    // Rows past the end hold whatever the cache holds: their weights are zero, but zero times a non-finite
                    // value is not, so clear these rows of V.  (Both groups may do it: they write the same zeros.)
                    const uint32_t s = v_stage % NST;
                    if (!warp_wait(kv_full + 8 * s, (v_stage / NST) & 1u, abort_flag)) break;
                    for (int j = m; j < (kTileKeys - (rows - t0)) * NH * 8; j += 128) {
                        const int r = rows - t0 + j / (NH * 8), c = j % (NH * 8);
                        *reinterpret_cast<uint4*>(base_ptr + s * kStageBytes + (c >> 3) * kBlockBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4)) =
                            make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                if (!warp_wait(s_full + 8 * g, n_mine & 1u, abort_flag)) break;
                tc_fence_after();
                if (live) {
                    uint32_t v[4][32];
#pragma unroll
                    for (int j = 0; j < 4; ++j) tc_ld_row32(v[j], my_s + 32u * j);
                    tc_wait_ld();
                    constexpr bool kScaled = kCap || kBias;           // v holds base-2 logits rather than raw products
                    if (kScaled) {
                        const float4* const mp = reinterpret_cast<const float4*>(base_ptr + sp.meta + e * 1024);
#pragma unroll
                        for (int c = 0; c < 128; c += 4) {
                            float4 pos = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (kBias) pos = mp[c >> 2];
                            const float pp[4] = {pos.x, pos.y, pos.z, pos.w};
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                uint32_t& r = v[c >> 5][(c & 31) + j];
                                float s = __uint_as_float(r);
                                s = kCap ? fmaf(-2.f * cap2, rcpf(1.f + ex2f(s * cap_in)), cap2) : s * scale2;
                                if (kBias) s = fmaf(-slope2, fabsf(q_pos - pp[j]), s);
                                r = __float_as_uint(s);
                            }
                        }
                    }
                    if (kDoc) {
                        const int4* const md = reinterpret_cast<const int4*>(base_ptr + sp.meta + e * 1024 + 512);
#pragma unroll
                        for (int c = 0; c < 128; c += 4) {
                            const int4 d4 = md[c >> 2];
                            const int dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (dd[j] != q_doc) v[c >> 5][(c & 31) + j] = __float_as_uint(-INFINITY);
                        }
                    }
                    if (__any_sync(0xffffffffu, t0 + kTileKeys - 1 > lim)) {
                        const int n_see = lim - t0 + 1;               // columns c < n_see are visible
#pragma unroll
                        for (int c = 0; c < 128; ++c)
                            if (c >= n_see) v[c >> 5][c & 31] = __float_as_uint(-INFINITY);
                    }
                    float mx = -INFINITY;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int c = 0; c < 32; c += 2) mx = fmax3(mx, __uint_as_float(v[j][c]), __uint_as_float(v[j][c + 1]));
                    if (!kScaled) mx *= scale2;
                    const bool raise = mx > m_run + (in_item ? kLazy : 0.f);
                    if (__any_sync(0xffffffffu, raise)) {
                        const float m_new = raise ? mx : m_run, alpha = ex2f(m_run - m_new);
                        if (in_item) {
                            // O holds products with weights relative to the old reference
                            if (!warp_wait(pv_done + 8 * g, (n_mine - 1u) & 1u, abort_flag)) break;
                            tc_fence_after();
#pragma unroll
                            for (int c = 0; c < D; c += 16) {         // sixteen at a time: the row of S is held meanwhile
                                uint32_t o[16];
                                tc_ld_row16(o, my_o + c);
                                tc_wait_ld();
#pragma unroll
                                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                                tc_st_row16(my_o + c, o);
                            }
                        }
                        l_run *= alpha;
                        m_run = m_new;
                    }
                    const float ref = m_run == kNeg ? 0.f : m_run;    // a row that has seen nothing yet: all weights zero
                    const float2 neg = make_float2(-ref, -ref), sc = kScaled ? make_float2(1.f, 1.f) : make_float2(scale2, scale2);
                    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t pk[16];
#pragma unroll
                        for (int c = 0; c < 32; c += 2) {
                            const float2 x = make_float2(__uint_as_float(v[j][c]), __uint_as_float(v[j][c + 1]));
                            const float2 p = ex2f2(kScaled ? __fadd2_rn(x, neg) : __ffma2_rn(x, sc, neg));
                            sum = __fadd2_rn(sum, p);
                            pk[c >> 1] = pack_bf16(p.x, p.y);
                        }
                        tc_st_row16(my_s + 16u * j, pk);
                    }
                    l_run += sum.x + sum.y;
                    tc_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) { mbar_arrive(p_full + 8 * g); mbar_arrive(ent_empty + 8 * e); }
                ++n_mine;
                ++in_item;
                ++n_entry;
                continue;
            }
            // ---------------------------------- end of the item ----------------------------------
            const int split = en[kSplit], active = en[kActive], pair = en[kPair];
            __syncwarp();
            if (lane == 0) mbar_arrive(ent_empty + 8 * e);
            ++n_entry;
            if (in_item) {
                if (!warp_wait(pv_done + 8 * g, (n_mine - 1u) & 1u, abort_flag)) break;
                tc_fence_after();
            }
            float m_all = m_run, l_all = l_run, w0 = in_item ? 1.f : 0.f, w1 = 0.f;
            bool has0 = in_item > 0, has1 = false;
            if (!big) {
                // both groups hold part of the same rows: exchange reference and sum, then each writes half the columns
                ml[g * 128 + m] = m_run;
                __syncwarp();
                if (lane == 0) mbar_arrive(join_bar);
                if (!warp_wait(join_bar, n_join++ & 1u, abort_flag)) break;
                const float m_other = ml[(g ^ 1) * 128 + m];
                m_all = fmaxf(m_run, m_other);
                const float mine = ex2f(m_run - m_all);
                __syncwarp();
                if (lane == 0) mbar_arrive(join_bar);
                if (!warp_wait(join_bar, n_join++ & 1u, abort_flag)) break;
                ml[g * 128 + m] = in_item ? l_run * mine : __uint_as_float(kUnset);     // the group had no tile: its O is not set
                __syncwarp();
                tc_fence_before();
                if (lane == 0) mbar_arrive(join_bar);
                if (!warp_wait(join_bar, n_join++ & 1u, abort_flag)) break;
                tc_fence_after();
                const float l0 = ml[m], l1 = ml[128 + m];
                has0 = __float_as_uint(l0) != kUnset;
                has1 = __float_as_uint(l1) != kUnset;
                l_all = (has0 ? l0 : 0.f) + (has1 ? l1 : 0.f);
                const float other = ex2f(m_other - m_all);
                w0 = g == 0 ? mine : other;
                w1 = g == 0 ? other : mine;
            }
            if (live) {
                const bool final = active == 1;
                const float denom = a.n * ex2f(-m_all) + l_all;
                const float inv = final ? 1.f / denom : 1.f;
                const uint32_t o0 = (big ? tmem_o[g] : tmem_o[0]) + lane_base, o1 = tmem_o[1] + lane_base;
                uint16_t* const out = a.out + int64_t(b) * a.o_sb + int64_t(head) * a.o_sh + int64_t(tok) * a.o_st;
                const int64_t slot = (int64_t(b * a.n_kv_heads + h) * pl.n_pairs + pair) * pl.splits + split;
                const int row = (tok - pair * 2 * pl.tok_tile) * G + (head - h * G);
                float* const part = partial + (slot * pl.row_slots + row) * D;
                const bool zero = l_all == 0.f;          // saw nothing; a NaN among what it saw comes out as NaN
                // a pair's columns all belong to its group; of shared rows each group writes half
                const int c_begin = big ? 0 : g * (D / 2), c_end = big ? D : c_begin + D / 2;
#pragma unroll 1
                for (int c = c_begin; c < c_end; c += 16) {
                    uint32_t x0[16], x1[16];
                    if (has0) tc_ld_row16(x0, o0 + c);
                    if (has1) tc_ld_row16(x1, o1 + c);
                    tc_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float y0 = has0 ? __uint_as_float(x0[j]) * w0 : 0.f, y1 = has1 ? __uint_as_float(x1[j]) * w1 : 0.f;
                        x0[j] = __float_as_uint(zero ? 0.f : (y0 + y1) * inv);
                    }
                    if (!valid) continue;
                    if (final) {
#pragma unroll
                        for (int j = 0; j < 16; j += 8) {
                            uint4 y;
                            y.x = pack_bf16(__uint_as_float(x0[j]), __uint_as_float(x0[j + 1]));
                            y.y = pack_bf16(__uint_as_float(x0[j + 2]), __uint_as_float(x0[j + 3]));
                            y.z = pack_bf16(__uint_as_float(x0[j + 4]), __uint_as_float(x0[j + 5]));
                            y.w = pack_bf16(__uint_as_float(x0[j + 6]), __uint_as_float(x0[j + 7]));
                            *reinterpret_cast<uint4*>(out + c + j) = y;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; j += 4)
                            *reinterpret_cast<uint4*>(part + c + j) = make_uint4(x0[j], x0[j + 1], x0[j + 2], x0[j + 3]);
                    }
                }
                if (valid && (big || g == 0)) {
                    if (!final) partial_ml[slot * pl.row_slots + row] = make_float2(m_all, l_all);
                    else if (a.lse)
                        a.lse[(int64_t(b) * a.n_kv_heads * G + head) * a.max_new + tok] = zero ? -INFINITY : (m_all + log2f(l_all)) * kLn2;
                }
            }
            if (!big) {
                // the other group has read this group's O, and the exchange area is free again
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(join_bar);
                if (!warp_wait(join_bar, n_join++ & 1u, abort_flag)) break;
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == kChMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 512u);
    }
}

// out = sum_s O_s 2^(m_s - m) / (n 2^-m + sum_s l_s 2^(m_s - m)) over the parts of a split pair; one warp per query row
template <int D>
__global__ void __launch_bounds__(256) chunk_merge_kernel(const ChunkArgs a, const ChunkPlan pl, const float* partial,
                                                          const float2* partial_ml) {
    constexpr int C = D / 32;                            // columns per lane
    const int lane = threadIdx.x & 31, G = a.group;
    const int64_t id = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5);
    const int row = int(id % pl.row_slots);
    const int64_t up = id / pl.row_slots;
    const int pair = int(up % pl.n_pairs), u = int(up / pl.n_pairs);
    if (u >= a.batch * a.n_kv_heads) return;
    const int b = u / a.n_kv_heads, h = u % a.n_kv_heads;
    const PairRange x = pair_range(a, pl, u, pair);
    const int tok = x.tok0 + row / G, head = h * G + row % G;
    if (x.active <= 1 || tok >= x.n_new) return;         // nothing was split; the item itself wrote the result
    const int64_t slot0 = up * pl.splits;
    float m = kNeg;
    for (int s = lane; s < x.active; s += 32) m = fmaxf(m, partial_ml[(slot0 + s) * pl.row_slots + row].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    float l = 0.f, o[C];
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = 0.f;
#pragma unroll 4
    for (int s = 0; s < x.active; ++s) {
        const float2 p = partial_ml[(slot0 + s) * pl.row_slots + row];
        const float w = ex2f(p.x - m);
        const float* const src = partial + ((slot0 + s) * pl.row_slots + row) * D + lane * C;
        float y[C];
        if (C == 4) *reinterpret_cast<float4*>(y) = *reinterpret_cast<const float4*>(src);
        else *reinterpret_cast<float2*>(y) = *reinterpret_cast<const float2*>(src);
        l += p.y * w;
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] += y[c] * w;
    }
    const float inv = l == 0.f ? 0.f : 1.f / (a.n * ex2f(-m) + l);
    uint32_t* const out = reinterpret_cast<uint32_t*>(a.out + int64_t(b) * a.o_sb + int64_t(head) * a.o_sh + int64_t(tok) * a.o_st + lane * C);
#pragma unroll
    for (int c = 0; c < C; c += 2) out[c / 2] = pack_bf16(o[c] * inv, o[c + 1] * inv);
    if (a.lse && lane == 0)
        a.lse[(int64_t(b) * a.n_kv_heads * G + head) * a.max_new + tok] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ---- host side -----------------------------------------------------------------------------------------------------

// How many parts the keys of a pair are divided into.  An estimate of the time in SM clocks, from the kernels' own
// figures: a key tile, what an item costs besides, what the joining kernel costs.  With fewer items than SMs the longest
// item counts, otherwise the waves plus half an item for the uneven end.
constexpr int kMaxSplits = 64;
int pick_splits(int64_t pairs, int64_t cap_tiles, int min_tiles, double tile, double item, int sms) {
    const double join = 6000.;
    int best = 1;
    double best_cost = 0;
    for (int s = 1; s <= kMaxSplits; ++s) {
        const int64_t per = (cap_tiles + s - 1) / s;
        if (s > 1 && per < min_tiles) break;
        const double one = double(per) * tile + item, items = double(pairs) * s;
        const double cost = one * (items <= sms ? 1. : items / sms + 0.5) + (s > 1 ? join : 0.);
        if (s == 1 || cost < best_cost * 0.98) { best = s; best_cost = cost; }
    }
    return best;
}

// Up to sixteen query rows per KV head (single tokens above all) go to the kernel that streams the cache through
// warp-level products: its rows are spread over all threads, where a tcgen05 row tile would leave most of them idle.
// Measured for one token, 32 sequences x 32 heads, 410 - 1640 rows each, d = 128: TODO us there, 173 us in row tiles.
constexpr int kFewRows = 16;

ChunkPlan chunk_plan(const csp_params& p, int max_new) {
    ChunkPlan pl;
    const int G = p.n_q_heads / p.n_kv_heads;
    pl.tok_tile = 128 / G;
    pl.n_pairs = (max_new + 2 * pl.tok_tile - 1) / (2 * pl.tok_tile);
    if (pl.n_pairs < 1) pl.n_pairs = 1;
    pl.row_slots = (max_new < 2 * pl.tok_tile ? max_new : 2 * pl.tok_tile) * G;
    const bool few = pl.row_slots <= kFewRows;
    pl.key_tile = few ? 64 : kTileKeys;
    pl.min_tiles = few ? 2 : kMinTiles;
    const int64_t pairs = int64_t(p.batch) * p.n_kv_heads * pl.n_pairs;
    // a tile of 64 or 128 keys as a share of the memory stream, or the products of two row tiles
    const double tile = few ? 1400. : pl.row_slots > 128 ? 2400. : 2800.;
    pl.splits = pick_splits(pairs, (int64_t(p.out_capacity) + pl.key_tile - 1) / pl.key_tile, pl.min_tiles, tile,
                            few ? 2500. : 4000., sm_count());
    const int64_t items = pairs * pl.splits;
    pl.n_items = items > 0x3fffffffLL ? -1 : int(items);
    return pl;
}

struct PartialLayout { size_t ml, o, total; };
PartialLayout partial_layout(const csp_params& p, const ChunkPlan& pl) {
    PartialLayout x;
    const size_t rows = pl.splits > 1 && pl.n_items > 0 ? size_t(pl.n_items) * size_t(pl.row_slots) : 0;
    x.ml = kStatusBytes;
    x.o = x.ml + round256(rows * sizeof(float2));
    x.total = x.o + round256(rows * size_t(p.head_dim) * 4);
    return x;
}

template <int NH, bool kCap, bool kBias, bool kDoc>
csp_status launch_variant(const ChunkArgs& a, const ChunkPlan& pl, const CUtensorMap& tq, const CUtensorMap& tk,
                          const CUtensorMap& tv, float* partial, float2* ml, cudaStream_t s) {
    constexpr int smem = int(ChunkShape<NH, kBias || kDoc>::plan().total) + 1024;
    static_assert(smem <= 227 * 1024, "shared memory of one CTA");
    auto kern = chunk_attn_kernel<NH, kCap, kBias, kDoc>;
    static std::atomic<bool> configured[kMaxDevices];
    if (!raise_smem_limit(kern, smem, configured)) return CSP_ERR_CUDA;
    const int sms = sm_count();
    kern<<<pl.n_items < sms ? pl.n_items : sms, kChThreads, smem, s>>>(tq, tk, tv, a, pl, partial, ml);
    return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA;
}

template <int NH>
csp_status launch_nh(const ChunkArgs& a, const ChunkPlan& pl, const CUtensorMap& tq, const CUtensorMap& tk,
                     const CUtensorMap& tv, float* partial, float2* ml, cudaStream_t s) {
    const int which = (a.mods.softcap > 0.f ? 4 : 0) | (a.mods.slopes ? 2 : 0) | (a.mods.documents ? 1 : 0);
    switch (which) {
        case 0: return launch_variant<NH, false, false, false>(a, pl, tq, tk, tv, partial, ml, s);
        case 1: return launch_variant<NH, false, false, true>(a, pl, tq, tk, tv, partial, ml, s);
        case 2: return launch_variant<NH, false, true, false>(a, pl, tq, tk, tv, partial, ml, s);
        case 3: return launch_variant<NH, false, true, true>(a, pl, tq, tk, tv, partial, ml, s);
        case 4: return launch_variant<NH, true, false, false>(a, pl, tq, tk, tv, partial, ml, s);
        case 5: return launch_variant<NH, true, false, true>(a, pl, tq, tk, tv, partial, ml, s);
        case 6: return launch_variant<NH, true, true, false>(a, pl, tq, tk, tv, partial, ml, s);
        default: return launch_variant<NH, true, true, true>(a, pl, tq, tk, tv, partial, ml, s);
    }
}

}  // namespace

size_t chunk_workspace_bytes(const csp_params& p, int max_new) {
    const ChunkPlan pl = chunk_plan(p, max_new);
    return partial_layout(p, pl).total;
}

csp_status launch_chunk_attn(const csp_params& p, const ChunkArgs& a, const csp_tensor& q, const csp_tensor& k,
                             const csp_tensor& v, const csp_pages* pages, void* ws, cudaStream_t s) {
    const ChunkPlan pl = chunk_plan(p, a.max_new);
    if (pl.n_items < 0) return CSP_ERR_UNSUPPORTED;
    const PartialLayout lay = partial_layout(p, pl);
    float* const partial = reinterpret_cast<float*>(static_cast<char*>(ws) + lay.o);
    float2* const ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + lay.ml);
    CUtensorMap tq, tk, tv;
    const int map_rows = pages ? pages->page_rows : (p.out_capacity > 0 ? p.out_capacity : 1);
    const int map_outer = pages ? pages->n_pages : p.batch;
    const int box_tokens = pl.tok_tile < a.max_new ? pl.tok_tile : a.max_new;
    if (!make_cache_tensor_map(&tk, k, p.dtype, p.head_dim, map_rows, p.n_kv_heads, map_outer, pl.key_tile) ||
        !make_cache_tensor_map(&tv, v, p.dtype, p.head_dim, map_rows, p.n_kv_heads, map_outer, pl.key_tile))
        return CSP_ERR_UNSUPPORTED;
    csp_status st;
    if (pl.row_slots <= kFewRows) {
        st = launch_chunk_few(p, a, pl, q, tk, tv, partial, ml, s);
    } else {
        if (!make_query_tensor_map(&tq, q, p.head_dim, p.n_q_heads, a.max_new, p.batch, a.group, box_tokens))
            return CSP_ERR_UNSUPPORTED;
        st = p.head_dim == 64 ? launch_nh<1>(a, pl, tq, tk, tv, partial, ml, s) : launch_nh<2>(a, pl, tq, tk, tv, partial, ml, s);
    }
    if (st != CSP_OK || pl.splits == 1) return st;
    const int64_t rows = int64_t(pl.n_items / pl.splits) * pl.row_slots;
    const unsigned blocks = unsigned((rows + 7) / 8);
    if (p.head_dim == 64) chunk_merge_kernel<64><<<blocks, 256, 0, s>>>(a, pl, partial, ml);
    else chunk_merge_kernel<128><<<blocks, 256, 0, s>>>(a, pl, partial, ml);
    return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA;
}

}  // namespace csp
