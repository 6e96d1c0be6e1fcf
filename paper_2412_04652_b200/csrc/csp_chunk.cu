// Attention of a chunk of new tokens over a dense or paged cache with the n-softmax normaliser (Eq. 5-7):
//   out[b, hq, i, :] = sum_t e^{o_t} / (n + sum_j e^{o_j}) v_t,   o_t = modified(scale <q_i, k_t>),   t visible to token i.
//
// One pass over the keys with a running reference m (base-2 exponent) and sum l per query row.  The G query heads that
// share a KV head and the tokens of the chunk together are the rows of a tcgen05 tile of 128: row = token * G + head,
// so a tile of keys is fetched once for all of them.  A work item is a pair of such row tiles (up to 256 rows) of one
// (sequence, KV head) unit against its 128-key tiles; one CTA per SM stays resident and works off an equal share of all
// key tiles (see Share).  An item that was cut between CTAs leaves un-normalised partial results for a second small kernel.
//
// Inside a CTA
//   warp 16     producer: looks up pages, streams K and V tiles (128-byte swizzle, TMA, no multicast) through a ring of
//               shared-memory stages, stages positions and documents of the keys, and tells the other warps through a
//               small ring of entries which tile comes next (so that whatever it skips is skipped by everybody)
//   warp 17     one elected lane issues tcgen05.mma: S_g = Q K^T (128 x 128, fp32 in tensor memory) and O_g += P_g V
//   warps 0-7, 8-15  two softmax groups g = 0, 1; two threads share a query row, half of the columns each.  A group reads
//               its S from tensor memory, applies modifiers and mask, and writes the weights as bf16 back over S, where
//               the second product reads them as its A operand; O stays in tensor memory.  The reference is raised only when a logit
//               exceeds it by more than 2^8, which is rare after the first tile, so the O rows are rescaled (by the
//               softmax thread itself) hardly ever.
// With more than 128 rows in an item, group g takes row tile g and both see every key tile; with fewer, both take the
// same rows and alternate over the key tiles (their results are joined when the item ends): either way one group's
// softmax runs while the tensor cores work for the other.
//
// Bound by the exponentials and the matrix products, which need the same 1024 clocks per 128 x 128 tile and are both busy 55 % of
// the clocks in which an SM works.  Measured at d = 128: 513 - 1024 tokens over 8 K - 32 K positions, 4 sequences, 28 / 4 heads (904
// GFLOP): 835 - 870 us (1.04 - 1.08 PFLOP/s) at first, 945 - 980 (0.92 - 0.96) back to back, when the power limit lowers the
// clocks; 512 tokens over 4 K, 32 heads (32 GFLOP): 48 us, of which 10 are the start and end of items, and 9 us for joining.
//
// Precision.  Sums, maxima and O are fp32.  The weights are rounded to bf16 (by 2^-8 of a weight at most, independently of
// each other): the error of the result against 64 bits is 0.0023 of it instead of the 0.0017 that its own rounding
// to bf16 leaves.  A second product with the weights' remainders brings it back to 0.0017, but takes half as many matrix
// operations again: 66 us instead of 57 for 512 tokens over 4 K, 81 instead of 75 with documents, 1150 - 1200 instead of 870 - 950
// for the largest; for long prompts the faster one was chosen (few rows have both products: HBM is their bound).  The cap
// is c - 2 c / (1 + e^{2 o / c}): one exponential and one reciprocal on the pipe that is the bound, exact to c 2^-20; the tanh
// instruction, the only shorter form, has 11 bits.
#include <limits.h>

#include "csp_chunk.cuh"
#include "csp_tc.cuh"

namespace csp {
namespace {
using namespace dev;

constexpr int kGroupWarps = 8;                           // two per TMEM lane quarter: each takes half of the columns
constexpr int kSoftmaxWarps = 2 * kGroupWarps;
constexpr int kChProducerWarp = kSoftmaxWarps, kChMmaWarp = kSoftmaxWarps + 1;
constexpr int kChThreads = 32 * (kSoftmaxWarps + 4);      // registers are shared out by groups of four warps: two stay idle
// Registers per thread.  The kernel is launched with 96 (what 640 threads may have); the softmax threads, which hold a
// quarter of a row of S at a time, take 104, the other four warps make do with 64: 512 * 104 + 128 * 64 = 640 * 96.
constexpr int kSoftmaxRegs = 104, kOtherRegs = 64;
constexpr int kEntries = 8;                              // ring of tile entries
constexpr int kEntryWords = 12;
constexpr uint32_t kUnset = 0xBF800000u;                 // -1.0f: no sum of weights has these bits

// What an entry says.  The first two words are all that a tile needs (one 8-byte load): flags and the tile's first key;
// the others describe the item and are read where it starts and ends.
enum EntryWord { kFlags, kTile0, kSeq, kHead, kTok0, kRows, kNew, kPart, kPrefix };
enum EntryFlags { kTileOf0 = 1, kTileOf1 = 2, kEnd = 4, kStop = 8, kFirst = 16, kSlot0 = 32, kSlot1 = 64, kHasQ = 128 };

struct ChunkSmem { uint32_t q, meta, entries, pair, join, bars, misc, total; };
template <int NH, bool kMeta>
struct ChunkShape {
    static constexpr int kStages = NH == 2 ? 4 : 8;
    static constexpr uint32_t kStageBytes = NH * kBlockBytes;            // one tile of K or of V
    static constexpr uint32_t kQBytes = NH * kBlockBytes;                // one row tile of Q
    static constexpr int kBars = 2 * kStages + 2 * kEntries + 4 + 6 + 2 + 8;
    __host__ __device__ static constexpr ChunkSmem plan() {
        ChunkSmem s = {};
        uint32_t off = uint32_t(kStages) * kStageBytes;
        s.q = off;       off += 2 * kQBytes;
        s.meta = off;    off += kMeta ? kEntries * 1024 : 0;             // [entry][128] positions, then documents
        s.entries = off; off += kEntries * kEntryWords * 4;
        s.pair = off;    off += 2 * 4 * 128 * 4;                         // [parity][group][half][row]: exchanged by the halves of a row
        s.join = off;    off += 2 * 2 * 128 * 4;                         // [group][row] reference, then sum
        s.bars = off;    off += kBars * 8;
        s.misc = off;    off += 32;
        s.total = off;
        return s;
    }
};

template <int NH, bool kCap, bool kBias, bool kDoc>
__global__ void __launch_bounds__(kChThreads, 1)
chunk_attn_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                  const __grid_constant__ CUtensorMap tmap_v, const ChunkArgs a, const ChunkPlan pl,
                  ChunkParts* const parts, float* const partial, float2* const partial_ml) {
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
    float* const pair_buf = reinterpret_cast<float*>(base_ptr + sp.pair);
    float* const join_buf = reinterpret_cast<float*>(base_ptr + sp.join);
    const uint32_t kv_full = base + sp.bars, kv_empty = kv_full + 8 * NST;
    const uint32_t ent_full = kv_empty + 8 * NST, ent_empty = ent_full + 8 * kEntries;
    const uint32_t q_full = ent_empty + 8 * kEntries, q_empty = q_full + 16;      // [2] each
    const uint32_t s_full = q_empty + 16, pv_done = s_full + 16, p_full = pv_done + 16;   // [2] each
    const uint32_t join_bar = p_full + 16, drain_bar = join_bar + 8;
    const uint32_t pair_bar = drain_bar + 8;                                      // [2][4]: the two warps of a lane quarter
    volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + sp.misc);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(base_ptr + sp.misc + 4);
    volatile uint32_t* const fills = tmem_slot + 2;      // when the producer ends: its loads into the ring and into the slots of Q

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        *abort_flag = 0;
        for (int s = 0; s < NST; ++s) { mbar_init(kv_full + 8 * s, 1); mbar_init(kv_empty + 8 * s, 1); }
        for (int e = 0; e < kEntries; ++e) { mbar_init(ent_full + 8 * e, 1); mbar_init(ent_empty + 8 * e, kSoftmaxWarps + 1); }
        for (int g = 0; g < 2; ++g) {
            mbar_init(q_full + 8 * g, 1); mbar_init(q_empty + 8 * g, 1);
            mbar_init(s_full + 8 * g, 1); mbar_init(pv_done + 8 * g, 1);
            mbar_init(p_full + 8 * g, kGroupWarps);
            for (int q = 0; q < 4; ++q) mbar_init(pair_bar + 32 * g + 8 * q, 2);
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
    Share share = find_share<kChThreads>(a, pl, reinterpret_cast<int*>(base_ptr + sp.pair));      // (synchronises)
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
            warp_wait(ent_empty + 8 * e, ((n_entry / kEntries) & 1u) ^ 1u, abort_flag);
            ok = ok && !warp_aborted(abort_flag);
            if (lane < kEntryWords) entries[e * kEntryWords + lane] = word;
            return e;
        };
        auto announce = [&](uint32_t e) {
            __syncwarp();
            if (ok && lane == 0) mbar_arrive(ent_full + 8 * e);
            ++n_entry;
        };
        if (lane == 0) parts[blockIdx.x] = ChunkParts{-1, 0};
        // Items drawn whole, one after the other, are the last tokens of every unit first: these see the most keys, and an item
        // drawn near the end is a short one.
        const bool drawn = kDoc && share.drawn;
        const int n_units = pl.n_items / pl.n_pairs;
        auto unit_of = [&](int item) { return drawn ? item % n_units : item / pl.n_pairs; };
        ItemDraw draw;
        const uint32_t tiles_per_page = uint32_t(a.page_rows) / uint32_t(kTileKeys);      // (dense: not used)
        auto page_of = [&](int b, int tile) {            // the page of a tile that lies inside the cache
            return a.page_table[int64_t(b) * a.max_pages + uint32_t(tile) / tiles_per_page];
        };
        PairRange next = {};
        int next_page = 0;                               // lane l: page of the next item's tile l (of its first 32)
        auto look_up = [&](int item) {
            if (item > share.item1 || (item == share.item1 && share.tile1 == 0 && !drawn) || item >= pl.n_items) return;
            const int u = unit_of(item);
            next = pair_range(a, pl, u, drawn ? pl.n_pairs - 1 - item / n_units : item - u * pl.n_pairs);
            const int tile = (item == share.item0 ? share.tile0 : 0) + lane;
            if (a.page_table && next.count > 0 && tile < next.tiles) next_page = page_of(u / a.n_kv_heads, tile);
        };
        if (drawn) draw.init(lane, a.status, pl.n_items);
        int item = drawn ? int(blockIdx.x) : share.item0, coming = 0;
        look_up(item);
        for (; ok && item <= share.item1 && item < pl.n_items; item = coming) {
            coming = drawn ? draw.next(lane) : item + 1;
            const int u = unit_of(item), b = u / a.n_kv_heads, h = u % a.n_kv_heads;
            const PairRange x = next;
            int pages = next_page;                       // lane l: the page of tile 32 j + l
            const int tile0 = item == share.item0 ? share.tile0 : 0, tile1 = item == share.item1 ? share.tile1 : x.tiles;
            if (x.count <= 0 || (item == share.item1 && tile1 == 0)) { look_up(coming); continue; }
            // which partial result the item goes to: none (the item is whole), the one that goes on, the one that begins
            const int part = tile0 > 0 ? 2 * int(blockIdx.x) : tile1 < x.tiles ? 2 * int(blockIdx.x) + 1 : -1;
            if (lane == 0 && part >= 0) {
                if (tile0 > 0) parts[blockIdx.x].last = tile1 == x.tiles;
                else parts[blockIdx.x].first = item;
            }
            const bool big = x.count > pl.tok_tile;      // more than one row tile
            const int q_slots = big ? kSlot0 | kSlot1 : n_small++ & 1u ? kSlot1 : kSlot0;   // slot g for group g, or one for both
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
                case kPart: word = part; break;
                case kFlags: word = kFirst | q_slots; break;
                case kPrefix: word = x.prefix; break;
            }
            int n_done = 0;
            bool q_loaded = false;
            auto load_q = [&] {
                q_loaded = true;
#pragma unroll
                for (int slot = 0; slot < 2; ++slot) {
                    if (!(q_slots & kSlot0 << slot)) continue;
                    warp_wait(q_empty + 8 * slot, (q_uses[slot] & 1u) ^ 1u, abort_flag);
                    ok = ok && !warp_aborted(abort_flag);
                    if (!ok) return;
                    ++q_uses[slot];
                    if (lane == 0) {
                        mbar_expect_tx(q_full + 8 * slot, uint32_t(NH * a.group * min(pl.tok_tile, a.max_new)) * 128u);
#pragma unroll
                        for (int hb = 0; hb < NH; ++hb)
                            tma_load_4d(base + sp.q + slot * Shape::kQBytes + hb * kBlockBytes, &tmap_q, q_full + 8 * slot,
                                        hb * 64, h * a.group, x.tok0 + (big ? slot * pl.tok_tile : 0), b);
                    }
                }
            };
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
            bool q_free = tile0 < tile1;
#pragma unroll
            for (int slot = 0; slot < 2; ++slot)
                if (q_slots & kSlot0 << slot) q_free = q_free && mbar_test(q_empty + 8 * slot, (q_uses[slot] & 1u) ^ 1u);
            if (__all_sync(0xffffffffu, q_free)) load_q();
            for (int tile = tile0; tile < tile1 && ok; ++tile) {
                const int t0 = tile * kTileKeys;
                if (a.page_table && tile > tile0 && ((tile - tile0) & 31) == 0) pages = tile + lane < tile1 ? page_of(b, tile + lane) : 0;
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
                const uint32_t e = publish(lane == kTile0 ? t0 : lane == kFlags ? word | act : word);
                if (lane == kFlags) word &= ~kFirst;
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
                    row = int(uint32_t(tile) % tiles_per_page) * kTileKeys;
                }
#pragma unroll
                for (int which = 0; which < 2; ++which, ++n_stage) {
                    const uint32_t s = n_stage % NST;
                    warp_wait(kv_empty + 8 * s, ((n_stage / NST) & 1u) ^ 1u, abort_flag);
                    ok = ok && !warp_aborted(abort_flag);
                    if (!ok) break;
                    if (lane == 0) {
                        mbar_expect_tx(kv_full + 8 * s, kStageBytes);
                        tma_load_5d(base + s * kStageBytes, which ? &tmap_v : &tmap_k, kv_full + 8 * s, 0, row, 0, h, outer);
                    }
                }
                // Q goes behind the first two tiles (which need no more than four stages) if its slot is still in use
                if (++n_done == 1) look_up(coming);
                if (n_done == 2 && !q_loaded) load_q();
            }
            if (n_done == 1 && !q_loaded) load_q();
            if (n_done == 0) look_up(coming);
            announce(publish(lane == kFlags ? word | kEnd | (q_loaded ? kHasQ : 0) : word));
        }
        if (ok) announce(publish(lane == kFlags ? kStop : 0));
        if (lane == 0) {
            if (drawn) draw.done();
            fills[0] = n_stage;
            fills[1] = q_uses[0];
            fills[2] = q_uses[1];
        }
        __syncwarp();
    } else if (warp == kChMmaWarp) {
        // =============================== MMA issuer ===============================
        // The whole warp walks the entries, so that everything is uniform; one elected lane issues.  (With the loop inside
        // `lane == 0` every descriptor went through vector registers: issuing took 140 clocks per instruction, twice
        // what the tensor core needs to execute it.)
        uint32_t n_entry = 0, q_uses[2] = {0, 0}, n_p[2] = {0, 0};
        int n_tile = 0, pend[2] = {-1, -1}, v_here = -1; // tiles so far; tile whose P V product a group still owes; last tile of V seen
        bool started[2] = {false, false};                // the group has a product in this item (O holds something)
        auto product = [&](int g) {                      // O_g += P_g V of the owed tile
            const uint32_t n = 2u * uint32_t(pend[g]) + 1u, s = n % NST;
            if (v_here != pend[g]) { warp_wait(kv_full + 8 * s, (n / NST) & 1u, abort_flag); v_here = pend[g]; }
            const uint64_t vd = sw128_desc_mn(base + s * kStageBytes, kBlockBytes);
            warp_wait(p_full + 8 * g, n_p[g] & 1u, abort_flag);
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < kTileKeys / 16; ++k)
                    tc_mma_bf16_ts(tmem_o[g], tmem_s[g] + 8u * (k & 3) + 64u * (k >> 2), vd + uint64_t(k * (2048 >> 4)), kIdescO, (k > 0 || started[g]) ? 1u : 0u);
                tc_commit(pv_done + 8 * g);
                if (pend[g ^ 1] != pend[g]) tc_commit(kv_empty + 8 * s);         // nobody else waits for this tile of V
            }
            __syncwarp();
            ++n_p[g];
            started[g] = true;
            pend[g] = -1;
        };
        for (;;) {
            const uint32_t e = n_entry % kEntries;
            warp_wait(ent_full + 8 * e, (n_entry / kEntries) & 1u, abort_flag);
            if (warp_aborted(abort_flag)) break;
            const int flags = entries[e * kEntryWords + kFlags];
            __syncwarp();
            if (lane == 0) mbar_arrive(ent_empty + 8 * e);
            ++n_entry;
            if (flags & kStop) break;
            if (flags & kFirst) {
                started[0] = started[1] = false;
                // (an item without any tile, an END at once, has its Q or not; one that was loaded is waited for all the same)
#pragma unroll
                for (int slot = 0; slot < 2; ++slot) {
                    if (!(flags & kSlot0 << slot) || (flags & (kEnd | kHasQ)) == kEnd) continue;
                    warp_wait(q_full + 8 * slot, q_uses[slot] & 1u, abort_flag);
                    ++q_uses[slot];
                }
            }
            if (!(flags & kEnd)) {
                const uint32_t n = 2u * uint32_t(n_tile), s = n % NST;
                warp_wait(kv_full + 8 * s, (n / NST) & 1u, abort_flag);
                const uint64_t kd = sw128_desc(base + s * kStageBytes);
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    if (!(flags & kTileOf0 << g)) continue;
                    if (pend[g] >= 0) product(g);
                    tc_fence_after();
                    const uint64_t qd = sw128_desc(base + sp.q + ((flags & kSlot1) && (g == 1 || !(flags & kSlot0)) ? Shape::kQBytes : 0u));
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            constexpr int kColumnStep = 32 >> 4, kBlockStep = kBlockBytes >> 4;
                            const uint64_t off = uint64_t((k >> 2) * kBlockStep + (k & 3) * kColumnStep);
                            tc_mma_bf16(tmem_s[g], qd + off, kd + off, kIdescS, k > 0 ? 1u : 0u);
                        }
                        tc_commit(s_full + 8 * g);
                        if (g == 1 || !(flags & kTileOf1)) tc_commit(kv_empty + 8 * s);
                    }
                    __syncwarp();
                    pend[g] = n_tile;
                }
                // a group that sits this tile out pays what it owes now: its tile of V must not hold up the ring
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    if (!(flags & kTileOf0 << g) && pend[g] >= 0) product(g);
                ++n_tile;
            } else {
#pragma unroll
                for (int g = 0; g < 2; ++g)
                    if (pend[g] >= 0) product(g);
                if (elect_one()) {
#pragma unroll
                    for (int slot = 0; slot < 2; ++slot)
                        if ((flags & kHasQ) && (flags & kSlot0 << slot)) tc_commit(q_empty + 8 * slot);
                }
                __syncwarp();
            }
        }
        // nothing may be in flight when the tensor memory goes back
        if (elect_one()) {
            tc_commit(drain_bar);
            const unsigned long long t0 = global_ns();
            while (!mbar_try_wait(drain_bar, 0) && global_ns() - t0 < kWaitLimitNs / 8) {}
        }
        __syncwarp();
    }
    } else {
        // =============================== softmax groups ===============================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int g = warp / kGroupWarps, half = (warp >> 2) & 1, m = (warp & 3) * 32 + lane, G = a.group;
        const uint32_t lane_base = uint32_t((warp & 3) * 32) << 16;
        // this thread's 64 columns of its row of S; its 64 weights go over the first half of them
        const uint32_t my_s = tmem_s[g] + lane_base + 64u * half;
        const float scale2 = a.scale * kLog2e;
        // capped: x = c tanh(o / c) = c - 2 c / (1 + e^{2 o / c}), all in the base-2 domain
        const float cap2 = kCap ? a.mods.softcap * kLog2e : 0.f, cap_in = kCap ? 2.f * kLog2e * a.scale / a.mods.softcap : 0.f;
        uint32_t n_entry = 0, n_tile = 0, n_mine = 0, n_join = 0, n_pair = 0;
        float m_run = kNeg, l_run = 0.f;
        int lim = -1, q_doc = 0, rows = 0;
        float q_pos = 0.f, slope2 = 0.f;
        bool valid = false, live = false, started = false;     // started: the group has a tile in this item
        // what the other half of this row says
        auto other_half = [&](float mine) {
            float* const box = pair_buf + ((n_pair & 1u) * 4 + g * 2) * 128 + m;
            const uint32_t bar = pair_bar + 32 * g + 8 * (warp & 3);
            box[half * 128] = mine;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
            warp_wait(bar, n_pair & 1u, abort_flag);
            ++n_pair;
            return box[(half ^ 1) * 128];
        };
        auto join = [&] {                                // all warps of both groups
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(join_bar);
            warp_wait(join_bar, n_join++ & 1u, abort_flag);
            tc_fence_after();
        };
        for (;;) {
            const uint32_t e = n_entry % kEntries;
            warp_wait(ent_full + 8 * e, (n_entry / kEntries) & 1u, abort_flag);
            if (warp_aborted(abort_flag)) break;
            const int32_t* const en = entries + e * kEntryWords;
            const int2 head_words = *reinterpret_cast<const int2*>(en);
            const int flags = head_words.x, t0 = head_words.y;
            if (flags & kStop) break;
            if (flags & kFirst) {
                // this thread's query row: token m / G of its row tile, head m % G
                const int n_new = en[kNew], local = m / G, b = en[kSeq], h = en[kHead];
                const bool big = (flags & kSlot0) && (flags & kSlot1);
                rows = en[kRows];
                const int head = h * G + m - local * G, tok = en[kTok0] + (big ? g * pl.tok_tile : 0) + local;
                valid = local < pl.tok_tile && tok < n_new;
                const int r = rows - n_new + tok;
                const bool sees = valid && r >= 0;
                // rows that nobody asked for see everything: they must not send their warp through the masked path
                lim = !valid ? kSeesAll : r >= 0 ? max(r, en[kPrefix] - 1) : -1;
                live = __any_sync(0xffffffffu, valid);
                m_run = kNeg;
                l_run = 0.f;
                started = false;
                if (kDoc) q_doc = sees ? a.mods.documents[int64_t(b) * a.mods.doc_sb + int64_t(h) * a.mods.doc_sh + r] : 0;
                if (kBias) {
                    const int32_t* const poss = a.mods.positions ? a.mods.positions + int64_t(b) * a.mods.pos_sb + int64_t(h) * a.mods.pos_sh : nullptr;
                    const int row_last = max(rows - n_new + en[kTok0] + min(n_new - en[kTok0], 2 * pl.tok_tile) - 1, 0);
                    const int ref = rows > 0 ? (poss ? poss[row_last] : row_last) : 0;
                    q_pos = sees ? float((poss ? poss[r] : r) - ref) : 0.f;
                    slope2 = sees ? a.mods.slopes[head] * kLog2e : 0.f;
                }
            }
            if (!(flags & kEnd)) {
                const uint32_t v_stage = 2u * n_tile + 1u;
                ++n_tile;
                ++n_entry;
                if (!(flags & kTileOf0 << g)) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(ent_empty + 8 * e);
                    continue;
                }
                warp_wait(s_full + 8 * g, n_mine & 1u, abort_flag);
                if (t0 + kTileKeys > rows) {
                    // Rows past the end hold whatever the cache holds: their weights are zero, but zero times a non-finite
                    // value is not, so clear these rows of V.  (Both groups may do it: they write the same zeros.)  Only now that
                    // S is there: the product with what this stage held before has been issued, so that stage's barrier cannot be two
                    // phases behind, where the parity waited for would look complete.
                    const uint32_t s = v_stage % NST;
                    warp_wait(kv_full + 8 * s, (v_stage / NST) & 1u, abort_flag);
                    for (int j = tid % (32 * kGroupWarps); j < (kTileKeys - (rows - t0)) * NH * 8; j += 32 * kGroupWarps) {
                        const int r = rows - t0 + j / (NH * 8), c = j % (NH * 8);
                        *reinterpret_cast<uint4*>(base_ptr + s * kStageBytes + (c >> 3) * kBlockBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4)) =
                            make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                tc_fence_after();
                if (live) {
                    constexpr bool kScaled = kCap || kBias;           // the logits are scaled before the maximum is known
                    const bool masked = __any_sync(0xffffffffu, t0 + kTileKeys - 1 > lim);
                    float mx = -INFINITY;
                    // First pass over the row, 32 columns at a time: modifiers, mask and maximum.  What was changed goes back to
                    // tensor memory; holding the row instead would take the registers that two warps per quarter need.
#pragma unroll 1
                    for (int j = 0; j < 2; ++j) {
                        uint32_t v[32];
                        tc_ld_row32(v, my_s + 32u * j);
                        tc_wait_ld();
                        tc_loaded(v);
                        if (kScaled) {
                            const float4* const mp = reinterpret_cast<const float4*>(base_ptr + sp.meta + e * 1024 + 256 * half) + 8 * j;
#pragma unroll
                            for (int c = 0; c < 32; c += 4) {
                                float4 pos = make_float4(0.f, 0.f, 0.f, 0.f);
                                if (kBias) pos = mp[c >> 2];
                                const float pp[4] = {pos.x, pos.y, pos.z, pos.w};
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    float x = __uint_as_float(v[c + k]);
                                    x = kCap ? fmaf(-2.f * cap2, rcpf(1.f + ex2f(x * cap_in)), cap2) : x * scale2;
                                    if (kBias) x = fmaf(-slope2, fabsf(q_pos - pp[k]), x);
                                    v[c + k] = __float_as_uint(x);
                                }
                            }
                        }
                        if (kDoc) {
                            const int4* const md = reinterpret_cast<const int4*>(base_ptr + sp.meta + e * 1024 + 512 + 256 * half) + 8 * j;
#pragma unroll
                            for (int c = 0; c < 32; c += 4) {
                                const int4 d4 = md[c >> 2];
                                const int dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    if (dd[k] != q_doc) v[c + k] = __float_as_uint(-INFINITY);
                            }
                        }
                        if (masked) {
                            const int n_see = lim - t0 + 1 - 64 * half - 32 * j;      // columns c < n_see are visible
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (c >= n_see) v[c] = __float_as_uint(-INFINITY);
                        }
                        if (kScaled || kDoc || masked) tc_st_row32(my_s + 32u * j, v);
                        float m4[4] = {mx, -INFINITY, -INFINITY, -INFINITY};          // four chains: the latency of one would show
#pragma unroll
                        for (int c = 0; c < 32; c += 8)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                m4[k] = fmax3_nan(m4[k], __uint_as_float(v[c + 2 * k]), __uint_as_float(v[c + 2 * k + 1]));
                        mx = fmax3_nan(fmax3_nan(m4[0], m4[1], m4[2]), m4[3], m4[3]);
                    }
                    if (kScaled || kDoc || masked) tc_wait_st();
                    if (!kScaled) mx *= scale2;
                    const float mx_other = other_half(mx);
                    mx = fmax3_nan(mx, mx_other, mx_other);
                    // (a NaN among the logits raises the reference to NaN, and the whole row with it)
                    const bool raise = valid && !(mx <= m_run + (started ? kLazy : 0.f));
                    if (__any_sync(0xffffffffu, raise)) {
                        const float m_new = raise ? mx : m_run, alpha = ex2f(m_run - m_new);
                        if (started) {
                            // O holds products with weights relative to the old reference; each half rescales half of the row
                            const uint32_t my_o = tmem_o[g] + lane_base + uint32_t(half * (D / 2));
                            warp_wait(pv_done + 8 * g, (n_mine - 1u) & 1u, abort_flag);
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D / 2; c += 16) {
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
                    const float2 neg = make_float2(-ref, -ref), sc = make_float2(scale2, scale2);
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
                    for (int j = 0; j < 2; ++j) {
                        uint32_t v[32], pk[16];
                        tc_ld_row32(v, my_s + 32u * j);
                        tc_wait_ld();
                        tc_loaded(v);
#pragma unroll
                        for (int c = 0; c < 32; c += 2) {
                            float2 x = make_float2(__uint_as_float(v[c]), __uint_as_float(v[c + 1]));
                            x = kScaled ? __fadd2_rn(x, neg) : __ffma2_rn(x, sc, neg);
                            const float2 p = ex2f2(x);
                            sum[c / 2 % 2] = __fadd2_rn(sum[c / 2 % 2], p);
                            pk[c >> 1] = pack_bf16(p.x, p.y);
                        }
                        tc_st_row16(my_s + 16u * j, pk);
                    }
                    l_run += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                    tc_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) { mbar_arrive(p_full + 8 * g); mbar_arrive(ent_empty + 8 * e); }
                ++n_mine;
                started = true;
                continue;
            }
            // ---------------------------------- end of the item ----------------------------------
            const int part_slot = en[kPart], b = en[kSeq], h = en[kHead], tok0 = en[kTok0];
            const bool big = (flags & kSlot0) && (flags & kSlot1);
            __syncwarp();
            if (lane == 0) mbar_arrive(ent_empty + 8 * e);
            ++n_entry;
            if (kBias && fabsf(q_pos) > kFarToken) atomicOr(a.status, CSP_DEV_BAD_LEN);
            if (started) warp_wait(pv_done + 8 * g, (n_mine - 1u) & 1u, abort_flag);
            tc_fence_after();
            float l_all = l_run + other_half(l_run);
            float m_all = m_run, w0 = 1.f, w1 = 0.f;
            bool has0 = started, has1 = false;
            if (!big) {
                // both groups hold part of the same rows: exchange reference and sum, then each half row writes a quarter
                if (half == 0) {
                    join_buf[g * 128 + m] = m_run;
                    join_buf[256 + g * 128 + m] = started ? l_all : __uint_as_float(kUnset);     // the group had no tile: its O is not set
                }
                join();
                const float m0 = join_buf[m], m1 = join_buf[128 + m], l0 = join_buf[256 + m], l1 = join_buf[384 + m];
                has0 = __float_as_uint(l0) != kUnset;
                has1 = __float_as_uint(l1) != kUnset;
                m_all = fmax3_nan(m0, m1, m1);
                w0 = ex2f(m0 - m_all);
                w1 = ex2f(m1 - m_all);
                l_all = (has0 ? l0 * w0 : 0.f) + (has1 ? l1 * w1 : 0.f);
            }
            if (live) {
                const int local = m / G, head = h * G + m - local * G, tok = tok0 + (big ? g * pl.tok_tile : 0) + local;
                const bool final = part_slot < 0;
                const float denom = n_term(a.n, m_all) + l_all;
                const float inv = final ? 1.f / denom : 1.f;
                const uint32_t o0 = (big ? tmem_o[g] : tmem_o[0]) + lane_base, o1 = tmem_o[1] + lane_base;
                uint16_t* const out = a.out + int64_t(b) * a.o_sb + int64_t(head) * a.o_sh + int64_t(tok) * a.o_st;
                const int row = (tok - tok0) * G + (head - h * G);
                float* const part = partial + (int64_t(part_slot) * (D / 4) * pl.row_slots + row) * 4;
                const bool zero = l_all == 0.f;          // saw nothing; a NaN among what it saw comes out as NaN
                // a row tile's columns are shared by the two halves, those of shared rows by both groups' halves
                const int c_begin = big ? half * (D / 2) : (g * 2 + half) * (D / 4), c_end = c_begin + (big ? D / 2 : D / 4);
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
                        uint32_t y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = pack_bf16(__uint_as_float(x0[2 * j]), __uint_as_float(x0[2 * j + 1]));
                        if (a.out_wide) {
                            st_global_32(out + c, y);
                        } else {
                            *reinterpret_cast<uint4*>(out + c) = make_uint4(y[0], y[1], y[2], y[3]);
                            *reinterpret_cast<uint4*>(out + c + 8) = make_uint4(y[4], y[5], y[6], y[7]);
                        }
                    } else {
                        // four columns of neighbouring rows lie next to each other: a warp's store is one piece of 512 bytes
#pragma unroll
                        for (int j = 0; j < 16; j += 4)
                            *reinterpret_cast<uint4*>(part + int64_t((c + j) / 4) * pl.row_slots * 4) = make_uint4(x0[j], x0[j + 1], x0[j + 2], x0[j + 3]);
                    }
                }
                if (valid && half == 0 && (big || g == 0)) {
                    if (!final) partial_ml[int64_t(part_slot) * pl.row_slots + row] = make_float2(m_all, l_all);
                    else if (a.lse)
                        a.lse[(int64_t(b) * a.n_kv_heads * G + head) * a.max_new + tok] = zero ? -INFINITY : (m_all + log2f(l_all)) * kLn2;
                }
            }
            // the other group has read this group's O, and the exchange area is free again
            if (!big) join();
        }
    }

    tc_fence_before();
    __syncthreads();
    if (*abort_flag && tid == 0) {
        atomicOr(a.status, CSP_DEV_TIMEOUT);
        drain_ring(kv_full, fills[0], NST);
        drain_ring(q_full, fills[1], 1);
        drain_ring(q_full + 8, fills[2], 1);
    }
    if (warp == kChMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 512u);
    }
}

// out = sum_s O_s 2^(m_s - m) / (n 2^-m + sum_s l_s 2^(m_s - m)) over the parts of a cut item.  Block (c, r) joins kRows rows of
// the item that begins in block c of the main kernel and goes on in c + 1, ... until one says it is the last.  A thread has
// C chunks of four columns of a row; the parts are laid out [column / 4][row][4], so that eight rows are one line.  Bound by
// the latency of its few loads and of its instructions (which are cold), so the code is kept short.  For few rows, which are
// cut often, eight rows and eight parts in flight (one token over 8 K - 32 K rows, ten parts: 5.9 us; with 32 rows and
// four parts 14); elsewhere 16 rows and two parts (an item has two or three, of 256 rows; 512 tokens over 4 K: 9.4 us, with eight rows
// and parts 14; 1 K tokens over 8 K - 32 K: 15.5 us, with 32 rows or four parts 19).
// Launched ahead of the main kernel's end (programmatic dependence) it gained nothing.
template <int D, int kRows>
struct JoinShape {
    static constexpr int kCols = D / 4 < 256 / kRows ? D / 4 : 256 / kRows, C = D / 4 / kCols, kThreads = kRows * kCols;
};
template <int D, int kRows, int kAhead>
__global__ void __launch_bounds__(JoinShape<D, kRows>::kThreads)
chunk_join_kernel(const ChunkArgs a, const ChunkPlan pl, const ChunkParts* parts, const float* partial, const float2* partial_ml) {
    constexpr int C = JoinShape<D, kRows>::C;
    const int c0 = blockIdx.x, item = parts[c0].first;
    if (item < 0) return;
    const int lane = threadIdx.x & 31, col = threadIdx.x / kRows * C, G = a.group;
    int n_parts = 1;
    for (int c = c0 + 1; c < pl.grid; c += 32) {
        const bool in = c + lane < pl.grid;
        const uint32_t last = __ballot_sync(0xffffffffu, in && parts[c + lane].last);
        if (last) { n_parts += __ffs(last); break; }
        n_parts += 32;
    }
    n_parts = min(n_parts, pl.grid - c0);
    const int u = item / pl.n_pairs, pair = item - u * pl.n_pairs, b = u / a.n_kv_heads, h = u % a.n_kv_heads;
    const int n_new = a.n_new ? min(max(a.n_new[b], 0), a.max_new) : a.max_new;
    const int row = blockIdx.y * kRows + threadIdx.x % kRows, i = row / G, head = h * G + row - i * G, tok = pair * 2 * pl.tok_tile + i;
    if (row >= pl.row_slots || tok >= n_new) return;
    float m = kNeg, l = 0.f;
    float4 o[C];
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int s0 = 0; s0 < n_parts; s0 += kAhead) {
        float2 ml[kAhead];
        float4 y[kAhead][C];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            // partial results 2 c0 + 1, 2 (c0 + 1), 2 (c0 + 2), ...
            const int s = s0 + j, slot = (2 * (c0 + s) + (s == 0 ? 1 : 0)) * pl.row_slots;
            const bool in = s < n_parts;
            ml[j] = in ? partial_ml[slot + row] : make_float2(kNeg, 0.f);
#pragma unroll
            for (int c = 0; c < C; ++c)
                y[j][c] = in ? reinterpret_cast<const float4*>(partial)[slot * (D / 4) + (col + c) * pl.row_slots + row] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        float m_now = m;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) m_now = fmaxf(m_now, ml[j].x);
        const float keep = ex2f(m - m_now);
        m = m_now;
        l *= keep;
#pragma unroll
        for (int c = 0; c < C; ++c) { o[c].x *= keep; o[c].y *= keep; o[c].z *= keep; o[c].w *= keep; }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const float w = ex2f(ml[j].x - m_now);
            l += ml[j].y * w;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                o[c].x += y[j][c].x * w; o[c].y += y[j][c].y * w; o[c].z += y[j][c].z * w; o[c].w += y[j][c].w * w;
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / (n_term(a.n, m) + l);
    uint2* const out = reinterpret_cast<uint2*>(a.out + int64_t(b) * a.o_sb + int64_t(head) * a.o_sh + int64_t(tok) * a.o_st) + col;
#pragma unroll
    for (int c = 0; c < C; ++c) out[c] = make_uint2(pack_bf16(o[c].x * inv, o[c].y * inv), pack_bf16(o[c].z * inv, o[c].w * inv));
    if (a.lse && col == 0)
        a.lse[(int64_t(b) * a.n_kv_heads * G + head) * a.max_new + tok] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}
template <int D, int kRows, int kAhead>
void join_parts(const ChunkArgs& a, const ChunkPlan& pl, const ChunkParts* parts, const float* partial, const float2* ml, cudaStream_t s) {
    const dim3 blocks(pl.grid, (pl.row_slots + kRows - 1) / kRows);
    chunk_join_kernel<D, kRows, kAhead><<<blocks, JoinShape<D, kRows>::kThreads, 0, s>>>(a, pl, parts, partial, ml);
}

// ---- host side -----------------------------------------------------------------------------------------------------

// Up to sixteen query rows per KV head (single tokens above all) go to the kernel that streams the cache through
// warp-level products: its rows are spread over all threads, where a tcgen05 row tile would leave most of them idle.
// Measured at d = 128, here and in row tiles: 32 sequences x 32 heads, 410 - 1640 rows each, 1 row 103 and 133 us, 8 rows 110 and
// 135, 12 rows 133 and 135, 16 rows 144 and 135; 4 x 28 / 4 heads, 8 K - 32 K, 7 rows 42.5 and 52.6, 14 rows 47.9 and 52.5; 8 x 32 / 4
// heads, 1 K - 6 K, 8 rows 26.7 and 30.8, 16 rows 30.8 and 30.8; one short sequence, 2 rows 10.3 and 17, 16 rows 18 and 16.4.  Up
// to eight rows it is faster everywhere; from there to sixteen the two are about even, and here only the result is rounded.
constexpr int kFewRows = 16;

ChunkPlan chunk_plan(const csp_params& p, int max_new) {
    ChunkPlan pl;
    const int G = p.n_q_heads / p.n_kv_heads;
    pl.tok_tile = 128 / G;
    pl.drawn = false;
    pl.n_pairs = (max_new + 2 * pl.tok_tile - 1) / (2 * pl.tok_tile);
    if (pl.n_pairs < 1) pl.n_pairs = 1;
    pl.row_slots = (max_new < 2 * pl.tok_tile ? max_new : 2 * pl.tok_tile) * G;
    const bool few = pl.row_slots <= kFewRows;
    pl.key_tile = few ? 64 : kTileKeys;
    pl.min_tiles = 2;
    pl.item_cost = 2;
    // A cut costs a row pair about four tiles (256 rows of partial results and their joining), few rows next to nothing,
    // but there an uneven share costs nothing either: HBM is the bound, whoever reads.  1 K tokens over 8 K - 32 K: 923 us without
    // this limit, 850 - 870 with 4, 862 with 2, 840 - 874 with 0; one token, serving batch: 103 us without, 104 with 8, 100 with 1.
    pl.snap = few ? 0x3fffffff : 4;
    const int64_t items = int64_t(p.batch) * p.n_kv_heads * pl.n_pairs;
    const int64_t weight = (int64_t(p.out_capacity) + pl.key_tile - 1) / pl.key_tile + pl.item_cost;      // of an item, at most
    pl.n_items = items > 0x3fffffffLL / weight ? -1 : int(items);
    // no more blocks than there can be shares of the smallest size
    const int64_t most = (items > 65536 ? 65536 : items) * weight / (pl.item_cost + pl.min_tiles) + 1;
    pl.grid = most < sm_count() ? int(most) : sm_count();
    return pl;
}

struct PartialLayout { size_t parts, ml, o, total; };
PartialLayout partial_layout(const csp_params& p, const ChunkPlan& pl) {
    PartialLayout x;
    const size_t rows = size_t(2) * pl.grid * pl.row_slots;
    x.parts = kStatusBytes;
    x.ml = x.parts + round256(size_t(pl.grid) * sizeof(ChunkParts));
    x.o = x.ml + round256(rows * sizeof(float2));
    x.total = x.o + round256(rows * size_t(p.head_dim) * 4);
    return x;
}

template <int NH, bool kCap, bool kBias, bool kDoc>
csp_status launch_variant(const ChunkArgs& a, const ChunkPlan& pl, const CUtensorMap& tq, const CUtensorMap& tk,
                          const CUtensorMap& tv, ChunkParts* parts, float* partial, float2* ml, cudaStream_t s) {
    constexpr int smem = int(ChunkShape<NH, kBias || kDoc>::plan().total) + 1024;
    static_assert(smem <= 227 * 1024, "shared memory of one CTA");
    auto kern = chunk_attn_kernel<NH, kCap, kBias, kDoc>;
    static std::atomic<bool> configured[kMaxDevices];
    if (!raise_smem_limit(kern, smem, configured)) return CSP_ERR_CUDA;
    kern<<<pl.grid, kChThreads, smem, s>>>(tq, tk, tv, a, pl, parts, partial, ml);
    return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA;
}

template <int NH>
csp_status launch_nh(const ChunkArgs& a, const ChunkPlan& pl, const CUtensorMap& tq, const CUtensorMap& tk,
                     const CUtensorMap& tv, ChunkParts* parts, float* partial, float2* ml, cudaStream_t s) {
    const int which = (a.mods.softcap > 0.f ? 4 : 0) | (a.mods.slopes ? 2 : 0) | (a.mods.documents ? 1 : 0);
    switch (which) {
        case 0: return launch_variant<NH, false, false, false>(a, pl, tq, tk, tv, parts, partial, ml, s);
        case 1: return launch_variant<NH, false, false, true>(a, pl, tq, tk, tv, parts, partial, ml, s);
        case 2: return launch_variant<NH, false, true, false>(a, pl, tq, tk, tv, parts, partial, ml, s);
        case 3: return launch_variant<NH, false, true, true>(a, pl, tq, tk, tv, parts, partial, ml, s);
        case 4: return launch_variant<NH, true, false, false>(a, pl, tq, tk, tv, parts, partial, ml, s);
        case 5: return launch_variant<NH, true, false, true>(a, pl, tq, tk, tv, parts, partial, ml, s);
        case 6: return launch_variant<NH, true, true, false>(a, pl, tq, tk, tv, parts, partial, ml, s);
        default: return launch_variant<NH, true, true, true>(a, pl, tq, tk, tv, parts, partial, ml, s);
    }
}

}  // namespace

size_t chunk_workspace_bytes(const csp_params& p, int max_new) {
    if (p.dtype != CSP_BF16 || (p.head_dim != 64 && p.head_dim != 128)) return 0;
    if (p.out_capacity > (1 << 30)) return 0;                                    // a row index plus some tiles fits 32 bits
    if (int64_t(max_new) * (p.n_q_heads / p.n_kv_heads) > (1 << 24)) return 0;   // and so do a chunk's rows
    const ChunkPlan pl = chunk_plan(p, max_new);
    if (pl.n_items < 0) return 0;                                                // key tiles are counted in 32 bits
    // Enough for shorter chunks as well: those of few rows have smaller key tiles, so more blocks have a share of them, and may
    // need more than a somewhat longer chunk.  (Among chunks of either kind the size grows with max_new.)
    const int few = kFewRows / (p.n_q_heads / p.n_kv_heads);
    const size_t mine = partial_layout(p, pl).total;
    const size_t shorter = partial_layout(p, chunk_plan(p, max_new < few ? max_new : few)).total;
    return mine > shorter ? mine : shorter;
}

csp_status launch_chunk_attn(const csp_params& p, const ChunkArgs& a, const csp_tensor& q, const csp_tensor& k,
                             const csp_tensor& v, const csp_pages* pages, void* ws, cudaStream_t s) {
    ChunkPlan pl = chunk_plan(p, a.max_new);
    // Documents make the weight of an item unknown (tiles without any of its documents are skipped): where every block has
    // several items anyway, and none is longer than a share, they are drawn whole.  2 x 32 heads, 2 K tokens of four documents:
    // 98.5 us shared out, 72.5 drawn with the longest first; in ascending order it was a tenth slower.
    pl.drawn = a.mods.documents && pl.row_slots > kFewRows && pl.n_items >= 2 * pl.grid;
    const PartialLayout lay = partial_layout(p, pl);
    ChunkParts* const parts = reinterpret_cast<ChunkParts*>(static_cast<char*>(ws) + lay.parts);
    float* const partial = reinterpret_cast<float*>(static_cast<char*>(ws) + lay.o);
    float2* const ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + lay.ml);
    CUtensorMap tq, tk, tv;
    const int map_rows = pages ? pages->page_rows : (p.out_capacity > 0 ? p.out_capacity : 1);
    const int map_outer = pages ? pages->n_pages : p.batch;
    const int box_tokens = pl.tok_tile < a.max_new ? pl.tok_tile : a.max_new;
    if (!make_cache_block_map(&tk, k, p.head_dim, map_rows, p.n_kv_heads, map_outer, pl.key_tile) ||
        !make_cache_block_map(&tv, v, p.head_dim, map_rows, p.n_kv_heads, map_outer, pl.key_tile))
        return CSP_ERR_UNSUPPORTED;
    csp_status st;
    if (pl.row_slots <= kFewRows) {
        st = launch_chunk_few(p, a, pl, q, tk, tv, parts, partial, ml, s);
    } else {
        if (!make_query_tensor_map(&tq, q, p.head_dim, p.n_q_heads, a.max_new, p.batch, a.group, box_tokens))
            return CSP_ERR_UNSUPPORTED;
        st = p.head_dim == 64 ? launch_nh<1>(a, pl, tq, tk, tv, parts, partial, ml, s) : launch_nh<2>(a, pl, tq, tk, tv, parts, partial, ml, s);
    }
    // nothing is cut by a single block, and where two parts of min_tiles are more than a cache has
    if (st != CSP_OK || pl.grid == 1 || p.out_capacity <= (2 * pl.min_tiles - 1) * pl.key_tile) return st;
    const bool few = pl.row_slots <= kFewRows;
    if (p.head_dim == 64) (few ? join_parts<64, 8, 8> : join_parts<64, 16, 2>)(a, pl, parts, partial, ml, s);
    else (few ? join_parts<128, 8, 8> : join_parts<128, 16, 2>)(a, pl, parts, partial, ml, s);
    return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA;
}

}  // namespace csp
