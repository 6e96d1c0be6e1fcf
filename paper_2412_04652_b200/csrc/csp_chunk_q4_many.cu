// Attention over pages held in 4 bits with more than three items of sixteen query rows per KV head: tcgen05 products over row tiles of 128, as
// for a bf16 cache (two row tiles to an item, one CTA per SM, equal shares of all 128-key tiles), except that a tile of keys is
// unpacked on its way.
//
// A row is base + scale code.  Of K the products see the codes, exactly: a half whose lowest four bits are a code is the number
// code 2^-24, with the code in the next four bits it is code 2^-20, so that unpacking eight codes takes four ANDs and a
// shift and no arithmetic.  S = Q' codes^T with Q' the query in halves, scaled by a power of two per row (largest value in [2^10, 2^11)) and by
// 16 where a code is in the lower place; then  logit = up (scale_t S + base_t sum Q')  with the two numbers of a row applied in fp32
// by the softmax threads: nothing of K is rounded.  (Half of the products scale x code would not fit the eleven bits of a half.)
// Of V they see the values base + scale code, rounded to halves relative to a power of two that follows the largest value of
// the item; the weights are rounded to halves as well.  (Applied to the weights instead, scale and base of V cost the softmax threads
// another two of seven instructions per logit: 1.37 ms for the largest case below.)
//
// Inside a CTA
//   warp 16     producer: looks up pages, brings the scales and bases of a tile's keys (and positions, documents) beside the entry
//               that announces it, loads the queries with TMA
//   warps 18, 19  unpack: copy a tile's codes into places of their own (cp.async, a tile ahead), then write them as halves into the
//               swizzled stages that the tensor core reads.  16-byte pieces of codes are taken in such an order that a quarter
//               warp's 16-byte stores fall into eight different bank groups
//   warp 17     one elected lane issues tcgen05.mma
//   warps 0-7, 8-15  two softmax groups, two threads per query row; at an item's start they turn the queries into halves in place
//
// Measured: 513 - 1024 tokens, 4 x 28 / 4 heads of 128, over 8 K - 32 K rows: 1.16 ms, 780 TFLOP/s of the two products' 1650 (a bf16
// cache 0.84 - 0.95 ms).  Neither HBM (5 %) nor the tensor cores (36 % of the clocks) nor instructions (50 %) are the bound, but the chain
// of a step of 128 keys, some 5400 clocks for two row tiles: products, first pass over the logits, second pass with the weights, products.
// With a cap 1.87 ms, a bias 1.56, both 2.09, four documents 0.98, a prefix of 8 K 1.15.  The compiler spills 100 bytes, with a bias 180, with
// documents 250 - 280, with both 530.
// Slower were: one pass with the weights in registers (they spill), four unpacking warps (1.19 ms), codes held in registers a tile ahead
// (1.22), scales of V applied to the weights (1.37).
#include <limits.h>

#include "csp_chunk.cuh"
#include "csp_tc.cuh"

namespace csp {
namespace {
using namespace dev;

constexpr int kGroupWarps = 8;                           // two per TMEM lane quarter: each takes half of the columns
constexpr int kSoftmaxWarps = 2 * kGroupWarps;
constexpr int kProducerWarp = kSoftmaxWarps, kMmaWarp = kSoftmaxWarps + 1, kUnpackWarp = kSoftmaxWarps + 2;
constexpr int kUnpackWarps = 2;
constexpr int kManyThreads = 32 * (kUnpackWarp + kUnpackWarps);
// registers per thread: launched with 96; 512 * 104 + 128 * 64 = 640 * 96
constexpr int kSoftmaxRegs = 104, kOtherRegs = 64;
constexpr int kEntries = 4;                              // ring of tile entries
constexpr int kEntryWords = 12;
constexpr int kRawTiles = 2;                             // tiles of codes under way
constexpr uint32_t kUnset = 0xBF800000u;                 // -1.0f: no sum of weights has these bits
constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;
constexpr float kTiny = 0x1p-126f, kHuge = 0x1p126f;     // bounds of the reference of the values

// What an entry says.  The first two words are all that a tile needs at once: flags and the tile's first key.
enum EntryWord { kFlags, kTile0, kSeq, kHead, kTok0, kRows, kNew, kPart, kPrefix, kPage, kPageRow, kScaleRef };
enum EntryFlags { kTileOf0 = 1, kTileOf1 = 2, kEnd = 4, kStop = 8, kFirst = 16, kSlot0 = 32, kSlot1 = 64, kHasQ = 128 };

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float lo_bf16(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
// of two pairs of bf16 numbers: the larger magnitudes
__device__ __forceinline__ uint32_t max_abs2(uint32_t x, uint32_t y) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x & 0x7fff7fffu), "r"(y & 0x7fff7fffu));
    return r;
}
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// eight codes -> eight halves, values 0, 4, 1, 5, 2, 6, 3, 7 of the word: for K as they are (times 2^-24, the odd ones 2^-20) ...
__device__ __forceinline__ uint4 unpack_codes(uint32_t x) {
    const uint32_t y = x >> 8;
    return make_uint4(x & kLow, x & kHigh, y & kLow, y & kHigh);
}
// ... for V as values: times scale 2^24 or 2^20, plus base, with one rounding (both halves of the factors and of `base` the same)
__device__ __forceinline__ uint32_t fma_f16(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint4 unpack_values(uint32_t x, uint32_t scale24, uint32_t scale20, uint32_t base) {
    const uint4 y = unpack_codes(x);
    return make_uint4(fma_f16(y.x, scale24, base), fma_f16(y.y, scale20, base), fma_f16(y.z, scale24, base), fma_f16(y.w, scale20, base));
}
// Values of V are held as value / reference x 2^-7, the reference the power of two that is at most the largest value so far: below
// 2^-6, so that scale 2^24 is still a half (15 scale <= 2^-5); a value below 2^-7 of the largest is off by up to 2^-17 of it (base and sum, 2^-18 each).
constexpr float kValueUnit = 0x1p-7f;
// A weight is a half as well: the reference is put this far (powers of two) below a row's largest logit, so that a weight may be up to
// 2^(7 + kLazy) and keeps its eleven bits down to 2^-21 of the largest; one below 2^-32 of it is lost.  A weight times kValueUnit
// is then what it is, and products need only the values' reference.
constexpr float kHeadroom = 7.f;
static_assert(kValueUnit == 0x1p-7f && kHeadroom == 7.f, "these cancel");

struct ManySmem { uint32_t q, raw, meta, entries, pair, join, rows, bars, misc, total; };
template <int NH, bool kMeta>
struct ManyShape {
    static constexpr int kStages = NH == 2 ? 3 : 6;
    static constexpr uint32_t kStageBytes = NH * kBlockBytes;            // one tile of K or of V in halves
    static constexpr uint32_t kQBytes = NH * kBlockBytes;                // one row tile of Q
    static constexpr uint32_t kRawBytes = kStageBytes / 4;               // one tile of K or of V in 4 bits
    // [128] scale of K, base of K, (position, document); then as pairs of halves scale 2^24 of V, scale 2^20, base
    static constexpr uint32_t kPositions = 2 * kTileKeys * 4, kDocuments = 3 * kTileKeys * 4, kValues = (kMeta ? 4 : 2) * kTileKeys * 4;
    static constexpr uint32_t kMetaBytes = kValues + 4 * kTileKeys * 4;
    static constexpr int kBars = 2 * kStages + 2 * kEntries + 6 + 6 + 2 + 8;
    __host__ __device__ static constexpr ManySmem plan() {
        ManySmem s = {};
        uint32_t off = uint32_t(kStages) * kStageBytes;
        s.q = off;       off += 2 * kQBytes;
        s.raw = off;     off += kRawTiles * 2 * kRawBytes;
        s.meta = off;    off += kEntries * kMetaBytes;
        s.entries = off; off += kEntries * kEntryWords * 4;
        s.pair = off;    off += 2 * 4 * 128 * 4;                         // [parity][group][half][row]: exchanged by the halves of a row
        s.join = off;    off += 3 * 2 * 128 * 4;                         // [what][group][row]: reference, sum, the values' reference
        s.rows = off;    off += 2 * 128 * 8;                             // [slot][row]: factor of the logits, sum of the query
        s.bars = off;    off += kBars * 8;
        s.misc = off;    off += 32;
        s.total = off;
        return s;
    }
};

template <int NH, bool kCap, bool kBias, bool kDoc>
__global__ void __launch_bounds__(kManyThreads, 1)
chunk_q4_many_kernel(const __grid_constant__ CUtensorMap tmap_q, const Q4Args cache, const ChunkArgs a, const ChunkPlan pl,
                     ChunkParts* const parts, float* const partial, float2* const partial_ml) {
    constexpr int D = 64 * NH;
    constexpr bool kMeta = kBias || kDoc;
    using Shape = ManyShape<NH, kMeta>;
    constexpr int NST = Shape::kStages;
    constexpr uint32_t kStageBytes = Shape::kStageBytes;
    // Halves.  S: 128 x 128, both operands K-major.  O: 128 x D, B (V) with its rows along K
    constexpr uint32_t kIdescS = (1u << 4) | (uint32_t(128 >> 3) << 17) | (uint32_t(128 >> 4) << 24);
    constexpr uint32_t kIdescO = (1u << 4) | (1u << 16) | (uint32_t(D >> 3) << 17) | (uint32_t(128 >> 4) << 24);

    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    constexpr ManySmem sp = Shape::plan();
    int32_t* const entries = reinterpret_cast<int32_t*>(base_ptr + sp.entries);
    float* const pair_buf = reinterpret_cast<float*>(base_ptr + sp.pair);
    float* const join_buf = reinterpret_cast<float*>(base_ptr + sp.join);
    float2* const row_const = reinterpret_cast<float2*>(base_ptr + sp.rows);
    const uint32_t kv_full = base + sp.bars, kv_empty = kv_full + 8 * NST;
    const uint32_t ent_full = kv_empty + 8 * NST, ent_empty = ent_full + 8 * kEntries;
    const uint32_t q_full = ent_empty + 8 * kEntries, q_empty = q_full + 16, q_ready = q_empty + 16;      // [2] each
    const uint32_t s_full = q_ready + 16, pv_done = s_full + 16, p_full = pv_done + 16;   // [2] each
    const uint32_t join_bar = p_full + 16, drain_bar = join_bar + 8;
    const uint32_t pair_bar = drain_bar + 8;                                      // [2][4]: the two warps of a lane quarter
    volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + sp.misc);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(base_ptr + sp.misc + 4);
    volatile uint32_t* const fills = tmem_slot + 2;      // when the producer ends: its loads into the slots of Q (at 1 and 2)

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        *abort_flag = 0;
        for (int s = 0; s < NST; ++s) { mbar_init(kv_full + 8 * s, kUnpackWarps); mbar_init(kv_empty + 8 * s, 1); }
        for (int e = 0; e < kEntries; ++e) { mbar_init(ent_full + 8 * e, 1); mbar_init(ent_empty + 8 * e, kSoftmaxWarps + 1 + kUnpackWarps); }
        for (int g = 0; g < 2; ++g) {
            mbar_init(q_full + 8 * g, 1); mbar_init(q_empty + 8 * g, 1); mbar_init(q_ready + 8 * g, kGroupWarps);
            mbar_init(s_full + 8 * g, 1); mbar_init(pv_done + 8 * g, 1);
            mbar_init(p_full + 8 * g, kGroupWarps);
            for (int q = 0; q < 4; ++q) mbar_init(pair_bar + 32 * g + 8 * q, 2);
        }
        mbar_init(join_bar, kSoftmaxWarps);
        mbar_init(drain_bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512u);
        tmem_relinquish();
    }
    tc_fence_before();
    Share share = find_share<kManyThreads>(a, pl, reinterpret_cast<int*>(base_ptr + sp.pair));      // (synchronises)
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t tmem_o[2] = {tmem, tmem + 128u}, tmem_s[2] = {tmem + 256u, tmem + 384u};

    if (warp >= kSoftmaxWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == kProducerWarp) {
        // =============================== producer ===============================
        uint32_t n_entry = 0, q_uses[2] = {0, 0}, n_small = 0;
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
        const uint32_t tiles_per_page = uint32_t(a.page_rows) / uint32_t(kTileKeys);
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
            if (next.count > 0 && tile < next.tiles) next_page = page_of(u / a.n_kv_heads, tile);
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
            uint4 ks_next = make_uint4(0, 0, 0, 0), vs_next = ks_next;       // scales and bases of keys 4 lane to 4 lane + 3
            int page_next = -1;                          // -1: outside the pool, zeros
            float v_ref = kTiny;                         // power of two that the values of V are relative to
            auto fetch_scales = [&](int tile, int page) {
                page_next = page >= 0 && page < a.n_pages ? page : -1;
                ks_next = vs_next = make_uint4(0, 0, 0, 0);
                if (page_next < 0) return;
                const int64_t at = (int64_t(uint32_t(tile) % tiles_per_page) * kTileKeys + 4 * lane) * 4;
                ks_next = *reinterpret_cast<const uint4*>(cache.ks + page * cache.ks_sb + h * cache.ks_sh + at);
                vs_next = *reinterpret_cast<const uint4*>(cache.vs + page * cache.vs_sb + h * cache.vs_sh + at);
            };
            auto fetch_meta = [&](int tile) {            // documents and positions of keys 4 lane to 4 lane + 3, a tile ahead of their use
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int t = tile * kTileKeys + 4 * lane + j;
                    if (t >= x.rows) { d_next[j] = 0; p_next[j] = 0; continue; }
                    if (kDoc) d_next[j] = docs[t];
                    if (kBias) p_next[j] = poss ? poss[t] : t;
                }
            };
            if (kMeta && tile0 < tile1) fetch_meta(tile0);
            if (tile0 < tile1) fetch_scales(tile0, __shfl_sync(0xffffffffu, pages, 0));
            bool q_free = tile0 < tile1;
#pragma unroll
            for (int slot = 0; slot < 2; ++slot)
                if (q_slots & kSlot0 << slot) q_free = q_free && mbar_test(q_empty + 8 * slot, (q_uses[slot] & 1u) ^ 1u);
            if (__all_sync(0xffffffffu, q_free)) load_q();
            for (int tile = tile0; tile < tile1 && ok; ++tile) {
                const int t0 = tile * kTileKeys;
                // (one tile ahead)
                if (tile + 1 < tile1 && ((tile + 1 - tile0) & 31) == 0) pages = tile + 1 + lane < tile1 ? page_of(b, tile + 1 + lane) : 0;
                const uint4 ks_now = ks_next, vs_now = vs_next;
                const int page = page_next;
                if (tile + 1 < tile1) fetch_scales(tile + 1, __shfl_sync(0xffffffffu, pages, (tile + 1 - tile0) & 31));
                int d_now[4], p_now[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) { d_now[j] = d_next[j]; p_now[j] = p_next[j]; }
                if (kMeta && tile + 1 < tile1) fetch_meta(tile + 1);
                int act = 0;
                bool seen[4] = {false, false, false, false};     // keys that the tokens may see: not those behind all of them, nor other documents'
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    if (g == 1 && !big) continue;
                    const int end = big && g == 0 ? x.kv_end[0] : x.kv_end[1];
                    bool hit = false;                    // (a tile without any of the tokens' documents is skipped)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const bool here = t0 + 4 * lane + j < end && (!kDoc || (d_now[j] >= doc_lo[g] && d_now[j] <= doc_hi[g]));
                        hit |= here;
                        seen[j] |= here;
                    }
                    act |= (kDoc ? __any_sync(0xffffffffu, hit) : t0 < end) ? 1 << g : 0;
                }
                if (act == 0) continue;
                if (!big) act = 1 << (n_done & 1);       // the groups take turns
                // Scales and bases in fp32, zeros behind the last row (what stands there may be no number).  Of V zeros where nobody sees the
                // row as well: what it holds must not be what the others are relative to.
                const uint32_t kp[4] = {ks_now.x, ks_now.y, ks_now.z, ks_now.w}, vp[4] = {vs_now.x, vs_now.y, vs_now.z, vs_now.w};
                float sk[4], bk[4], sv[4], bv[4], v_top = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool in = t0 + 4 * lane + j < x.rows;
                    sk[j] = in ? lo_bf16(kp[j]) : 0.f; bk[j] = in ? hi_bf16(kp[j]) : 0.f;
                    sv[j] = seen[j] ? lo_bf16(vp[j]) : 0.f; bv[j] = seen[j] ? hi_bf16(vp[j]) : 0.f;
                    v_top = fmaxf(v_top, fmaxf(fabsf(bv[j]), fabsf(fmaf(15.f, sv[j], bv[j]))));
                }
                // (magnitudes: their bits are in order)
                const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(fminf(v_top, kHuge))) & 0x7f800000u;
                v_ref = fmaxf(v_ref, __uint_as_float(top));
                if (page < 0 && lane == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
                const int page_row = int(uint32_t(tile) % tiles_per_page) * kTileKeys;
                int32_t told = word;
                switch (lane) {
                    case kTile0: told = t0; break;
                    case kFlags: told = word | act; break;
                    case kPage: told = page; break;
                    case kPageRow: told = page_row; break;
                    case kScaleRef: told = __float_as_int(v_ref); break;
                }
                const uint32_t e = publish(told);
                if (lane == kFlags) word &= ~kFirst;
                float4* const numbers = reinterpret_cast<float4*>(base_ptr + sp.meta + e * Shape::kMetaBytes);
                numbers[lane] = make_float4(sk[0], sk[1], sk[2], sk[3]);
                numbers[lane + 32] = make_float4(bk[0], bk[1], bk[2], bk[3]);
                const float v_unit = kValueUnit / v_ref;
                uint4* const values = reinterpret_cast<uint4*>(base_ptr + sp.meta + e * Shape::kMetaBytes + Shape::kValues);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float s24 = sv[j] * v_unit * 0x1p24f, zero = bv[j] * v_unit;
                    values[4 * lane + j] = make_uint4(pack_f16(s24, s24), pack_f16(0x1p-4f * s24, 0x1p-4f * s24), pack_f16(zero, zero), 0u);
                }
                if (kMeta) {
                    float* const mp = reinterpret_cast<float*>(base_ptr + sp.meta + e * Shape::kMetaBytes + Shape::kPositions);
                    int32_t* const md = reinterpret_cast<int32_t*>(base_ptr + sp.meta + e * Shape::kMetaBytes + Shape::kDocuments);
                    if (kBias) reinterpret_cast<float4*>(mp)[lane] = make_float4(float(p_now[0] - pos_ref), float(p_now[1] - pos_ref), float(p_now[2] - pos_ref), float(p_now[3] - pos_ref));
                    if (kDoc) reinterpret_cast<int4*>(md)[lane] = make_int4(d_now[0], d_now[1], d_now[2], d_now[3]);
                }
                announce(e);
                // Q goes behind the first two tiles if its slot is still in use
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
            fills[1] = q_uses[0];
            fills[2] = q_uses[1];
        }
        __syncwarp();
    } else if (warp == kMmaWarp) {
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
                    warp_wait(q_ready + 8 * slot, q_uses[slot] & 1u, abort_flag);
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
    } else {
        // =============================== unpackers ===============================
        // Each thread copies and unpacks pieces of its own (16 bytes: 32 codes of one row): no one else waits for its copies.
        constexpr int kThreads = 32 * kUnpackWarps, kRowPieces = 2 * NH, kPieces = int(Shape::kRawBytes) / 16 / kThreads;
        const int ut = tid - 32 * kUnpackWarp, piece = ut % kRowPieces, row_of = ut / kRowPieces;
        constexpr int kRowStep = kThreads / kRowPieces;
        const uint32_t raw = base + sp.raw + ut * 16;
        uint32_t n_entry = 0, n_copied = 0, n_done = 0;
        int entry_of[kRawTiles] = {};                    // of the tiles that have been copied, the oldest first
        auto unpack = [&] {                              // the oldest tile that has been copied
            const uint4* const values = reinterpret_cast<const uint4*>(base_ptr + sp.meta + entry_of[0] * Shape::kMetaBytes + Shape::kValues);
            if (n_copied - n_done == kRawTiles) asm volatile("cp.async.wait_group %0;" ::"n"(kRawTiles - 1) : "memory");
            else asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll 1
            for (int which = 0; which < 2; ++which) {
                const uint32_t n = 2u * n_done + which, s = n % NST;
                warp_wait(kv_empty + 8 * s, ((n / NST) & 1u) ^ 1u, abort_flag);
                uint8_t* const to = base_ptr + s * kStageBytes;
                const uint8_t* const from = base_ptr + (raw - base) + (n_done % kRawTiles) * 2 * Shape::kRawBytes + which * Shape::kRawBytes;
#pragma unroll 4
                for (int i = 0; i < kPieces; ++i) {
                    const int row = row_of + i * kRowStep;
                    uint4 x = *reinterpret_cast<const uint4*>(from + i * kThreads * 16);
                    // words 4 piece to 4 piece + 3 of the row, each one 16-byte piece of halves; the second half of a row (of four
                    // pieces) in another order, or its stores would meet those of the first one in the same banks
                    const int turn = piece & 2;
                    if (turn) x = make_uint4(x.z, x.w, x.x, x.y);
                    uint8_t* const line = to + (piece >> 1) * kBlockBytes + row * 128;
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                    auto place = [&](int j) { return reinterpret_cast<uint4*>(line + ((((piece & 1) * 4 + (j ^ turn)) ^ (row & 7)) << 4)); };
                    if (which == 0) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) *place(j) = unpack_codes(w[j]);
                    } else {
                        const uint4 f = values[row];
#pragma unroll
                        for (int j = 0; j < 4; ++j) *place(j) = unpack_values(w[j], f.x, f.y, f.z);
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(kv_full + 8 * s);
            }
            ++n_done;
            if (lane == 0) mbar_arrive(ent_empty + 8 * entry_of[0]);
#pragma unroll
            for (int i = 1; i < kRawTiles; ++i) entry_of[i - 1] = entry_of[i];
        };
        for (;;) {
            const uint32_t e = n_entry % kEntries, parity = (n_entry / kEntries) & 1u;
            // (what has been copied is not held back by an entry that is not there yet)
            if (n_copied != n_done && !__all_sync(0xffffffffu, mbar_test(ent_full + 8 * e, parity))) unpack();
            warp_wait(ent_full + 8 * e, parity, abort_flag);
            if (warp_aborted(abort_flag)) break;
            const int32_t* const en = entries + e * kEntryWords;
            const int flags = en[kFlags], page = en[kPage], row0 = en[kPageRow], h = en[kHead];
            ++n_entry;
            if (flags & (kStop | kEnd)) {                // (the entry of a tile is held until the tile has been unpacked)
                __syncwarp();
                if (lane == 0) mbar_arrive(ent_empty + 8 * e);
                if (flags & kStop) break;
                continue;
            }
            if (n_copied - n_done == kRawTiles) unpack();
#pragma unroll
            for (int i = 0; i < kRawTiles; ++i)
                if (int(n_copied - n_done) == i) entry_of[i] = int(e);
            if (page >= 0) {
                // (pieces lie one behind the other: all rows of a head in a page are neighbours)
                const int64_t at = int64_t(row0) * (D / 2) + ut * 16;
                const uint8_t* const kf = cache.k + page * cache.k_sb + h * cache.k_sh + at;
                const uint8_t* const vf = cache.v + page * cache.v_sb + h * cache.v_sh + at;
                const uint32_t to = raw + (n_copied % kRawTiles) * 2 * Shape::kRawBytes;
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    cp_async_16(to + i * kThreads * 16, kf + i * kThreads * 16);
                    cp_async_16(to + Shape::kRawBytes + i * kThreads * 16, vf + i * kThreads * 16);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            ++n_copied;
        }
        while (n_done != n_copied && !warp_aborted(abort_flag)) unpack();
        asm volatile("cp.async.wait_all;" ::: "memory");
    }
    } else {
        // =============================== softmax groups ===============================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int g = warp / kGroupWarps, half = (warp >> 2) & 1, m = (warp & 3) * 32 + lane, G = a.group;
        const uint32_t lane_base = uint32_t((warp & 3) * 32) << 16;
        // this thread's 64 columns of its row of S; its 64 weights go over the first half of them
        const uint32_t my_s = tmem_s[g] + lane_base + 64u * half;
        // capped: x = c tanh(o / c) = c - 2 c / (1 + e^{2 o / c}), all in the base-2 domain
        const float cap2 = kCap ? a.mods.softcap * kLog2e : 0.f, cap_in = kCap ? 2.f / a.mods.softcap : 0.f;
        uint32_t n_entry = 0, n_mine = 0, n_join = 0, n_pair = 0, q_uses = 0;        // q_uses: bit s, the parity of slot s
        float m_run = kNeg, l_run = 0.f, v_run = kTiny;
        float factor = 0.f, q_sum = 0.f;                 // logit = factor (scale S + base q_sum)
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
                v_run = kTiny;
                if ((flags & (kEnd | kHasQ)) != kEnd) {  // (an item without any tile may come without its queries)
                    const int slot = big ? g : (flags & kSlot1) ? 1 : 0;
                    if (slot == g) {
                        // ---- the query row in halves, in the order of the codes; each thread has half of it
                        warp_wait(q_full + 8 * slot, (q_uses >> slot) & 1u, abort_flag);
                        uint8_t* const line = base_ptr + sp.q + slot * Shape::kQBytes + (NH == 2 ? half * kBlockBytes : 0) + m * 128;
                        constexpr int kChunks = 4 * NH;
                        auto chunk = [&](int c) { return reinterpret_cast<uint4*>(line + (((NH == 2 ? c : 4 * half + c) ^ (m & 7)) << 4)); };
                        uint32_t top2 = 0;
#pragma unroll
                        for (int c = 0; c < kChunks; ++c) {
                            const uint4 y = *chunk(c);
                            top2 = max_abs2(max_abs2(max_abs2(max_abs2(top2, y.x), y.y), y.z), y.w);
                        }
                        top2 = max_abs2(top2, top2 >> 16 | top2 << 16);
                        top2 = max_abs2(top2, __float_as_uint(other_half(__uint_as_float(top2))));
                        const uint32_t top = (top2 & 0x7fffu) >> 7, ex = max(top, 14u);      // top 255: an infinity, the row is no number
                        const float down = __uint_as_float((264u - ex) << 23), down16 = 16.f * down;         // 2^(10 - e)
                        float sum = 0.f;
#pragma unroll
                        for (int c = 0; c < kChunks; ++c) {
                            const uint4 y = *chunk(c);
                            const float f[8] = {lo_bf16(y.x), hi_bf16(y.x), lo_bf16(y.y), hi_bf16(y.y), lo_bf16(y.z), hi_bf16(y.z), lo_bf16(y.w), hi_bf16(y.w)};
#pragma unroll
                            for (int j = 0; j < 8; ++j) sum = fmaf(f[j], down, sum);
                            *chunk(c) = make_uint4(pack_f16(down16 * f[0], down16 * f[4]), pack_f16(down * f[1], down * f[5]),
                                                   pack_f16(down16 * f[2], down16 * f[6]), pack_f16(down * f[3], down * f[7]));
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        sum += other_half(sum);
                        // S is the product with codes 2^-20
                        // (never zero: it meets the minus infinities of hidden keys)
                        factor = top == 255u ? __uint_as_float(0x7fc00000u) : fmaxf(a.scale * kLog2e * 0x1p10f * __uint_as_float(ex << 23), 0x1p-126f);
                        q_sum = sum * 0x1p-20f;
                        if (half == 0) row_const[slot * 128 + m] = make_float2(factor, q_sum);
                        __syncwarp();
                        if (lane == 0) mbar_arrive(q_ready + 8 * slot);
                    }
                    warp_wait(q_ready + 8 * slot, (q_uses >> slot) & 1u, abort_flag);
                    // (also where the other group uses the other slot: a later wait must not find its barrier a phase behind)
                    if (big) warp_wait(q_ready + 8 * (slot ^ 1), (q_uses >> (slot ^ 1)) & 1u, abort_flag);
                    if (big) q_uses ^= 3u;
                    else q_uses ^= 1u << slot;
                    if (slot != g) {
                        const float2 rc = row_const[slot * 128 + m];
                        factor = rc.x;
                        q_sum = rc.y;
                    }
                }
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
                const float v_ref = __int_as_float(en[kScaleRef]);
                ++n_entry;
                if (!(flags & kTileOf0 << g)) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(ent_empty + 8 * e);
                    continue;
                }
                warp_wait(s_full + 8 * g, n_mine & 1u, abort_flag);
                tc_fence_after();
                if (live) {
                    const float4* const numbers = reinterpret_cast<const float4*>(base_ptr + sp.meta + e * Shape::kMetaBytes) + 16 * half;
                    const bool masked = __any_sync(0xffffffffu, t0 + kTileKeys - 1 > lim);
                    float mx = -INFINITY;
                    // First pass over the row, 32 columns at a time: scale and base of the keys, modifiers, mask and maximum.  The
                    // logits go back to tensor memory; holding the row instead would take the registers that two warps per quarter need.
#pragma unroll 1
                    for (int j = 0; j < 2; ++j) {
                        uint32_t v[32];
                        tc_ld_row32(v, my_s + 32u * j);
                        tc_wait_ld();
                        tc_loaded(v);
                        const float2 f2 = make_float2(factor, factor), q2 = make_float2(q_sum, q_sum);
#pragma unroll
                        for (int c = 0; c < 32; c += 4) {
                            const float4 sk = numbers[8 * j + (c >> 2)], bk = numbers[32 + 8 * j + (c >> 2)];
                            float2 y0 = __ffma2_rn(make_float2(sk.x, sk.y), make_float2(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), __fmul2_rn(make_float2(bk.x, bk.y), q2));
                            float2 y1 = __ffma2_rn(make_float2(sk.z, sk.w), make_float2(__uint_as_float(v[c + 2]), __uint_as_float(v[c + 3])), __fmul2_rn(make_float2(bk.z, bk.w), q2));
                            if (kCap || kBias) { y0 = __fmul2_rn(y0, f2); y1 = __fmul2_rn(y1, f2); }     // (else when the weights are computed)
                            v[c] = __float_as_uint(y0.x); v[c + 1] = __float_as_uint(y0.y);
                            v[c + 2] = __float_as_uint(y1.x); v[c + 3] = __float_as_uint(y1.y);
                        }
                        if (kCap || kBias) {
                            const float4* const mp = reinterpret_cast<const float4*>(base_ptr + sp.meta + e * Shape::kMetaBytes + Shape::kPositions + 256 * half) + 8 * j;
#pragma unroll
                            for (int c = 0; c < 32; c += 4) {
                                float4 pos = make_float4(0.f, 0.f, 0.f, 0.f);
                                if (kBias) pos = mp[c >> 2];
                                const float pp[4] = {pos.x, pos.y, pos.z, pos.w};
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    float x = __uint_as_float(v[c + i]);
                                    if (kCap) x = fmaf(-2.f * cap2, rcpf(1.f + ex2f(x * cap_in)), cap2);
                                    if (kBias) x = fmaf(-slope2, fabsf(q_pos - pp[i]), x);
                                    v[c + i] = __float_as_uint(x);
                                }
                            }
                        }
                        if (kDoc) {
                            const int4* const md = reinterpret_cast<const int4*>(base_ptr + sp.meta + e * Shape::kMetaBytes + Shape::kDocuments + 256 * half) + 8 * j;
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
                        tc_st_row32(my_s + 32u * j, v);
                        float m4[4] = {mx, -INFINITY, -INFINITY, -INFINITY};          // four chains: the latency of one would show
#pragma unroll
                        for (int c = 0; c < 32; c += 8)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                m4[k] = fmax3_nan(m4[k], __uint_as_float(v[c + 2 * k]), __uint_as_float(v[c + 2 * k + 1]));
                        mx = fmax3_nan(fmax3_nan(m4[0], m4[1], m4[2]), m4[3], m4[3]);
                    }
                    tc_wait_st();
                    if (!(kCap || kBias)) mx *= factor;
                    const float mx_other = other_half(mx);
                    mx = fmax3_nan(mx, mx_other, mx_other);
                    // (a NaN among the logits raises the reference to NaN, and the whole row with it)
                    const bool raise = valid && !(mx <= m_run + (started ? kHeadroom + kLazy : kHeadroom));
                    if (__any_sync(0xffffffffu, raise) || v_ref != v_run) {
                        const float m_new = raise ? mx - kHeadroom : m_run, alpha = ex2f(m_run - m_new), shrink = alpha * (v_run / v_ref);
                        v_run = v_ref;
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
                                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * shrink);
                                tc_st_row16(my_o + c, o);
                            }
                        }
                        l_run *= alpha;
                        m_run = m_new;
                    }
                    const float ref = m_run == kNeg ? 0.f : m_run;    // a row that has seen nothing yet: all weights zero
                    const float2 neg = make_float2(-ref, -ref), f2 = make_float2(factor, factor);
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
                            x = kCap || kBias ? __fadd2_rn(x, neg) : __ffma2_rn(x, f2, neg);
                            const float2 p = ex2f2(x);
                            sum[c / 2 % 2] = __fadd2_rn(sum[c / 2 % 2], p);
                            pk[c >> 1] = pack_f16(p.x, p.y);
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
            float l_all = (l_run + other_half(l_run)) * kValueUnit;
            float m_all = m_run + kHeadroom, w0 = 1.f, w1 = 0.f, v0 = v_run, v1 = 0.f;        // what the two groups' products are multiplied by
            bool has0 = started, has1 = false;
            if (!big) {
                // both groups hold part of the same rows: exchange reference and sum, then each half row writes a quarter
                if (half == 0) {
                    join_buf[g * 128 + m] = m_all;
                    join_buf[256 + g * 128 + m] = started ? l_all : __uint_as_float(kUnset);     // the group had no tile: its O is not set
                    join_buf[512 + g * 128 + m] = v_run;
                }
                join();
                const float m0 = join_buf[m], m1 = join_buf[128 + m], l0 = join_buf[256 + m], l1 = join_buf[384 + m];
                has0 = __float_as_uint(l0) != kUnset;
                has1 = __float_as_uint(l1) != kUnset;
                m_all = fmax3_nan(m0, m1, m1);
                w0 = ex2f(m0 - m_all);
                w1 = ex2f(m1 - m_all);
                l_all = (has0 ? l0 * w0 : 0.f) + (has1 ? l1 * w1 : 0.f);
                v0 = join_buf[512 + m];
                v1 = join_buf[640 + m];
            }
            if (live) {
                const int local = m / G, head = h * G + m - local * G, tok = tok0 + (big ? g * pl.tok_tile : 0) + local;
                const bool final = part_slot < 0;
                const float denom = n_term(a.n, m_all) + l_all;
                const float inv = final ? 1.f / denom : 1.f;
                w0 *= inv;                               // (apart from the references, so that large values' sums are numbers)
                w1 *= inv;
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
                    float o[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {       // dimension c + j
                        const int d = j & 7, at = (j & 8) + (d < 4 ? 2 * d : 2 * d - 7);
                        const float y0 = has0 ? __uint_as_float(x0[at]) * w0 * v0 : 0.f, y1 = has1 ? __uint_as_float(x1[at]) * w1 * v1 : 0.f;
                        o[j] = zero ? 0.f : y0 + y1;
                    }
                    if (!valid) continue;
                    if (final) {
                        uint32_t y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = pack_bf16(o[2 * j], o[2 * j + 1]);
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
                            *reinterpret_cast<uint4*>(part + int64_t((c + j) / 4) * pl.row_slots * 4) = make_uint4(__float_as_uint(o[j]), __float_as_uint(o[j + 1]), __float_as_uint(o[j + 2]), __float_as_uint(o[j + 3]));
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
        drain_ring(q_full, fills[1], 1);
        drain_ring(q_full + 8, fills[2], 1);
    }
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, 512u);
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------

template <int NH, bool kCap, bool kBias, bool kDoc>
csp_status launch_variant(const ChunkArgs& a, const ChunkPlan& pl, const CUtensorMap& tq, const Q4Args& c, ChunkParts* parts,
                          float* partial, float2* ml, cudaStream_t s) {
    constexpr int smem = int(ManyShape<NH, kBias || kDoc>::plan().total) + 1024;
    static_assert(smem <= 227 * 1024, "shared memory of one CTA");
    auto kern = chunk_q4_many_kernel<NH, kCap, kBias, kDoc>;
    static std::atomic<bool> configured[kMaxDevices];
    if (!raise_smem_limit(kern, smem, configured)) return CSP_ERR_CUDA;
    kern<<<pl.grid, kManyThreads, smem, s>>>(tq, c, a, pl, parts, partial, ml);
    return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA;
}

template <int NH>
csp_status launch_nh(const ChunkArgs& a, const ChunkPlan& pl, const CUtensorMap& tq, const Q4Args& c, ChunkParts* parts, float* partial,
                     float2* ml, cudaStream_t s) {
    const int which = (a.mods.softcap > 0.f ? 4 : 0) | (a.mods.slopes ? 2 : 0) | (a.mods.documents ? 1 : 0);
    switch (which) {
        case 0: return launch_variant<NH, false, false, false>(a, pl, tq, c, parts, partial, ml, s);
        case 1: return launch_variant<NH, false, false, true>(a, pl, tq, c, parts, partial, ml, s);
        case 2: return launch_variant<NH, false, true, false>(a, pl, tq, c, parts, partial, ml, s);
        case 3: return launch_variant<NH, false, true, true>(a, pl, tq, c, parts, partial, ml, s);
        case 4: return launch_variant<NH, true, false, false>(a, pl, tq, c, parts, partial, ml, s);
        case 5: return launch_variant<NH, true, false, true>(a, pl, tq, c, parts, partial, ml, s);
        case 6: return launch_variant<NH, true, true, false>(a, pl, tq, c, parts, partial, ml, s);
        default: return launch_variant<NH, true, true, true>(a, pl, tq, c, parts, partial, ml, s);
    }
}

}  // namespace

csp_status launch_chunk_q4_many(const csp_params& p, const ChunkArgs& a, const ChunkPlan& pl, const csp_tensor& q, const Q4Args& c,
                                ChunkParts* parts, float* partial, float2* ml, cudaStream_t s) {
    CUtensorMap tq;
    const int box_tokens = pl.tok_tile < a.max_new ? pl.tok_tile : a.max_new;
    if (!make_query_tensor_map(&tq, q, p.head_dim, p.n_q_heads, a.max_new, p.batch, a.group, box_tokens)) return CSP_ERR_UNSUPPORTED;
    return p.head_dim == 64 ? launch_nh<1>(a, pl, tq, c, parts, partial, ml, s) : launch_nh<2>(a, pl, tq, c, parts, partial, ml, s);
}

}  // namespace csp
