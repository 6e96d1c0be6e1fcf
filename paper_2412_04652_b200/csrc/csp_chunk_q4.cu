// Attention of new tokens over pages held in 4 bits, up to sixteen query rows (token x head) per item, up to three of these per KV head.
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
// dimensions come: the query is laid out alike.  For the second one the rows of V are transposed as 16-bit pieces of four codes on
// their way into registers.
//
// Queries are scaled by a power of two, row by row, so that their largest value lies in [2^10, 2^11): a half holds every bf16
// value exactly from there down to 2^-24 of it, and 16 times the largest.  A weight times its row's scale is rounded to a half (11 bits)
// after multiplication by a factor of the query's own, which follows the largest such product that the query has seen as the softmax's
// reference follows the largest logit: it comes to 2^8 - 2^14, so that bits are lost below 2^-22 of it and a product below
// 2^-33 of it is.  (One factor for all queries that followed the scales alone, hidden rows' and faint ones' among them: 39.2 us
// instead of 39.4 below, 40.9 instead of 41.4 for five capped tokens.  Codes less 7.5, against the sum of the rounded products, take another
// 3 % and bring the error without the result's own rounding from 6e-4 to 3e-4.)
// (Codes of K as e4m3 bytes, which four zeros and a code are as well, take half of the ANDs, but the compiler makes halves of
// them before it multiplies: 650 instructions per tile of 32 keys instead of 510.)
//
// Organisation: one CTA per SM works off an equal share of all 32-key tiles, and inside it every warp an equal share of that,
// tile after tile: no warp waits for another one before the end.  A warp has a ring of its own that it refills itself as soon as it
// has read a slot.  An item (up to sixteen query rows of a unit) that lies in one warp's share is finished by
// it; of one that is cut the pieces stay in shared memory until all warps are done and are joined then, in order; of one that
// goes on in another CTA a partial result is left, and the CTA that leaves the last one joins them, in order.
//
// Measured: 32 x 32 heads of 128, 410 - 1640 rows, one token: 39.4 us, 3.6 TB/s over all.  A tile takes a warp 2800 clocks (eight query
// rows, twelve warps: 5.2 TB/s while they run); in front of the first one lie 12 K clocks, six dependent loads and much code that runs
// once, and behind the last one 10 K: the item's sums 3 K, from there to the first piece 3 K, the join across blocks 3 K.
// So long GQA (five tiles per warp) takes 27 us where its bytes take 7.
// A third tile in flight or eleven warps do not help; sixteen warps leave too few registers.
#include <cuda_fp16.h>
#include <limits.h>

#include <initializer_list>

#include "csp_chunk.cuh"

namespace csp {
namespace {
using namespace dev;

constexpr int kQ4Tile = 32;                              // keys per tile
constexpr int kCountWord = 16, kMostBlocks = 192;        // of the status area: a byte per block
constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;
// Of a weight times its row's scale, which enters the second product as a half: the largest factor it is held by (times a weight of
// at most 2^8 still a number), the largest value it may have, and what a query's largest one is brought to when it is above that.
constexpr float kMostGain = 0x1p119f, kMostProduct = 0x1p14f, kMostProductLog = 14.f;
constexpr uint32_t kTopProduct = 8;                      // 2^8 to 2^9

struct FewQuery { const uint16_t* q; int64_t sb, sh, st; Divider by_page; };      // by_page: tiles per page

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
__device__ __forceinline__ void ldsm_x4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
// of two pairs of bf16 numbers: the larger magnitudes
__device__ __forceinline__ uint32_t max_abs2(uint32_t x, uint32_t y) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x & 0x7fff7fffu), "r"(y & 0x7fff7fffu));
    return r;
}
__device__ __forceinline__ float lg2f(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float fmax3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// four bytes of global memory into shared memory, zeros where there is nothing
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ float lo_bf16(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

constexpr int kDeskBytes = 512;
// What a variant's code deals with.  (One variant for all of them: 49 -> 52 us for five capped tokens, 30.5 -> 32 us for a bias.)
enum Mods { kNone, kCap, kBias, kAny };

template <int NH, int RH>   // head_dim = 64 NH, 8 RH query rows
struct Q4Shape {
    static constexpr int D = 64 * NH, R = 8 * RH;
    // As many warps as their registers allow: eight rows 160 each, sixteen 240.  (Eight warps for eight rows: 47 us instead of 45 for the
    // serving batch, 33 instead of 30 for long GQA when this was measured.)
    static constexpr int kWarps = RH == 1 ? 12 : 8;
    // Tiles in flight per warp, 4.6 KB each at d = 128.  (Three instead of two of them: serving batch 40.7 us instead of 39.5.)
    static constexpr int kSlots = NH == 2 ? 2 : 4;
    static constexpr uint32_t kCodeBytes = kQ4Tile * D / 2, kScaleBytes = kQ4Tile * 4; // of K or of V
    static constexpr uint32_t kLoadBytes = 2 * kCodeBytes + 2 * kScaleBytes;
    static constexpr uint32_t kSlotBytes = kLoadBytes + 2 * kQ4Tile * 4;               // then positions and documents
    static constexpr int kPieceRow = D + 4;                                            // floats: sums, reference, sum of weights
    static constexpr uint32_t kPieceBytes = R * kPieceRow * 4;
    static constexpr uint32_t kFront = kWarps * kSlots * kSlotBytes;                   // [warp]: the piece that a warp begins with
    static constexpr uint32_t kNotes = kFront + kWarps * kPieceBytes;                  // [warp]
    static constexpr uint32_t kTable = kNotes + kWarps * 16;                           // [warp][R] RowNote
    static constexpr uint32_t kDesk = kTable + kWarps * R * 16;                        // [warp] Desk
    static constexpr uint32_t kScratch = kDesk + kWarps * kDeskBytes;                  // of find_share
    static constexpr uint32_t kChains = kScratch + 68 * 4;                             // of find_share; then whether this block joins them
    static constexpr uint32_t kTotal = kChains + 6 * 4;
    static constexpr int kThreads = 32 * kWarps;
    static_assert(kSlots * kSlotBytes >= kPieceBytes, "the piece that a warp ends with goes into its ring");
};

// One warp's part of the block's share: from tile begin_tile of item begin on, up to tile end_tile of item end (none of that
// item's where end_tile is the block's first).  The block's tiles, and one more per item, are cut into equal parts; everybody goes
// over the block's items, a lane per item.  *first: the range of item begin.
struct WarpShare { int begin, begin_tile, end, end_tile; };
__device__ __forceinline__ WarpShare warp_share(const ChunkArgs& a, const ChunkPlan& pl, const Share& sh, int warp, int warps, int lane, PairRange* first) {
    const int last = min(sh.item1, pl.n_items - 1);
    WarpShare got = {pl.n_items, 0, pl.n_items, 0};
    int total = 0, part = 0;
    // (Most of this kernel's code runs once, at the speed at which it is fetched: both passes are one, and the second is all there
    // is where one step covers the block's items.)
    const bool once = last - sh.item0 < 32;
#pragma unroll 1
    for (int pass = once ? 1 : 0; pass < 2; ++pass) {
        int before = 0;
#pragma unroll 1
        for (int i = sh.item0; i <= last; i += 32) {
            const int item = i + lane, lo = item == sh.item0 ? sh.tile0 : 0;
            int w = 0;
            PairRange r = {};
            if (item <= last && !(item == sh.item1 && sh.tile1 == 0)) {
                const int u = pl.by_pairs(item);
                r = pair_range(a, pl, u, item - u * pl.n_pairs);
                w = r.count > 0 ? max((item == sh.item1 ? sh.tile1 : r.tiles) - lo, 0) + 1 : 0;
            }
            int x = w;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, d);
                if (lane >= d) x += y;
            }
            const int all = __shfl_sync(0xffffffffu, x, 31);
            if (once) part = max((all + warps - 1) / warps, 2);
            if (pass) {
                const int p = before + x - w;            // weight in front of this lane's item
#pragma unroll 1
                for (int k = 0; k < 2; ++k) {
                    const int cut = (warp + k) * part;
                    const uint32_t hit = __ballot_sync(0xffffffffu, cut >= p && cut < p + w);
                    if (!hit) continue;
                    const int from = __ffs(hit) - 1, tile = __shfl_sync(0xffffffffu, lo + max(cut - p - 1, 0), from);
                    if (k == 0) { got.begin = i + from; got.begin_tile = tile; if (lane == from) *first = r; }
                    else { got.end = i + from; got.end_tile = tile; }
                }
            }
            before += all;
        }
        total = before;
        if (!once) part = max((total + warps - 1) / warps, 2);
    }
    return got;
}

// What a warp says of its pieces: the item that it went on with (-1: none) and whether that ended with it, the item that it began
// and did not end.
struct Notes { int front, front_ends, back, unused; };
// What a warp has of one item: its tiles [lo, hi).
struct Segment { int item, b, h, lo, hi; PairRange x; };
// What is seldom needed stays out of the registers: what is loaded, what is computed, what the front piece belongs to, and the
// range of the warp's first item.
struct Desk { Segment loaded, computed, front; PairRange first; };
static_assert(sizeof(Desk) <= kDeskBytes, "a warp's place in shared memory");
// A query row's last visible key, document, position and slope.
struct RowNote { int lim, doc; float pos, slope2; };

template <int NH, int RH, int kMods>
__global__ void __launch_bounds__(Q4Shape<NH, RH>::kThreads, 1)
chunk_q4_few_kernel(const ChunkArgs a, const ChunkPlan pl, const FewQuery qy, const Q4Args cache,
                    float* const partial, float2* const partial_ml) {
    using Shape = Q4Shape<NH, RH>;
    constexpr int D = Shape::D, NW = Shape::kWarps, NST = Shape::kSlots;
    constexpr int KW = D / 32;                           // words of a key that a lane has in the first product
    constexpr int MT = D / 16;                           // 16-dimension tiles of the output

    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 127u) & ~127u;
    uint8_t* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    Notes* const notes = reinterpret_cast<Notes*>(base_ptr + Shape::kNotes);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = a.group;
    const ModArgs& md = a.mods;
    const Share share = find_share<Shape::kThreads>(a, pl, reinterpret_cast<int*>(base_ptr + Shape::kScratch), reinterpret_cast<int*>(base_ptr + Shape::kChains));      // (synchronises)
    Desk& desk = *reinterpret_cast<Desk*>(base_ptr + Shape::kDesk + kDeskBytes * warp);
    const WarpShare mine = warp_share(a, pl, share, warp, NW, lane, &desk.first);
    __syncwarp();

    const int gr = lane >> 2, qd = lane & 3;             // fragment row (a key, then dimensions) and column pair (query rows)
    const bool capped = kMods == kCap || (kMods == kAny && md.softcap > 0.f), by_doc = kMods == kAny && md.documents;
    const bool biased = kMods == kBias || (kMods == kAny && md.slopes);
    // capped: x = c tanh(o / c) = c - 2 c / (1 + e^{2 o / c}), all in the base-2 domain
    const float cap2 = md.softcap * kLog2e, cap_in = capped ? 2.f / md.softcap : 0.f;
    uint8_t* const my_ring = base_ptr + warp * NST * Shape::kSlotBytes;
    const uint32_t ring = base + warp * NST * Shape::kSlotBytes;
    const int tiles_per_page = a.page_rows / kQ4Tile;

    auto segment = [&](int from, Segment& s) {           // the first one at or behind item `from`
        for (s.item = from; s.item <= min(mine.end, share.item1) && s.item < pl.n_items; ++s.item) {
            const int u = pl.by_pairs(s.item), block_lo = s.item == share.item0 ? share.tile0 : 0;
            s.lo = s.item == mine.begin ? mine.begin_tile : block_lo;
            if (s.item == mine.end && mine.end_tile == block_lo) return false;
            if (s.item == share.item1 && share.tile1 == 0) return false;
            if (s.item == mine.begin) s.x = desk.first;
            else s.x = pair_range(a, pl, u, s.item - u * pl.n_pairs);
            s.hi = s.item == mine.end ? mine.end_tile : s.item == share.item1 ? share.tile1 : s.x.tiles;
            if (s.x.count > 0) { s.b = pl.by_heads(u); s.h = u - s.b * a.n_kv_heads; return true; }
        }
        return false;
    };

    // ---- what comes: tiles on their way into the ring.  A lane copies 16 bytes of every 512 of the codes, the first sixteen lanes the
    // scales.  V's 16-byte chunks change places, so that eight rows' pieces of one column lie in different banks.
    constexpr int kCopies = Shape::kCodeBytes / 512;
    const uint32_t v_to = NH == 2 ? (lane >> 2) * 64 + (((lane & 3) ^ (lane >> 3)) << 4) : (lane >> 1) * 32 + (((lane & 1) ^ ((lane >> 3) & 1)) << 4);
    bool f_open = false, f_more = true;
    int f_item = mine.begin - 1, f_end = 0, f_tile = 0, f_left = 0, f_next = 0, f_index = 0, f_lo = 0, f_hi = 0;     // f_left: tiles of the current page
    bool f_there = false;                                // the current page lies in the pool
    const uint8_t* f_k = nullptr, * f_v = nullptr, * f_s = nullptr;              // what this lane copies of the next tile
    int tile_of[NST], item_of[NST];                      // what is in the slots, the next one first; item -1: no more
    auto page_at = [&](int index) { return index < a.max_pages ? a.page_table[int64_t(desk.loaded.b) * a.max_pages + index] : -1; };
    auto turn_page = [&](int page, int row) {
        const int h = desk.loaded.h;
        f_there = uint32_t(page) < uint32_t(a.n_pages);
        if (!f_there) page = 0;                          // (nothing is read through it)
        f_k = cache.k + page * cache.k_sb + h * cache.k_sh + int64_t(row) * (D / 2) + lane * 16;
        f_v = cache.v + page * cache.v_sb + h * cache.v_sh + int64_t(row) * (D / 2) + lane * 16;
        f_s = (lane < 8 ? cache.ks + page * cache.ks_sb + h * cache.ks_sh : cache.vs + page * cache.vs_sb + h * cache.vs_sh) +
              int64_t(row) * 4 + (lane & 7) * 16;
    };
    auto refill = [&](int j) {                           // the next tile into slot j, which has been read
#pragma unroll
        for (int i = 1; i < NST; ++i) { item_of[i - 1] = item_of[i]; tile_of[i - 1] = tile_of[i]; }
        item_of[NST - 1] = -1;
        for (;;) {
            if (!f_open) {
                if (!f_more) break;
                Segment f;
                f_more = segment(f_item + 1, f);
                if (!f_more) break;
                __syncwarp();
                if (lane == 0) desk.loaded = f;
                __syncwarp();
                f_item = f.item;
                f_end = f.hi;
                f_tile = f.lo;
                f_index = qy.by_page(f_tile);
                f_left = (f_index + 1) * tiles_per_page - f_tile;
                {                                        // the item's queries, positions and slopes will be asked for soon
                    constexpr int kLines = D / 64;       // of 128 bytes
                    const int m = lane / kLines, tok = pl.by_group(m);
                    if (tok < f.x.count && m < Shape::R)
                        asm volatile("prefetch.global.L2 [%0];" ::"l"(qy.q + int64_t(f.b) * qy.sb + int64_t(f.h * G + m - tok * G) * qy.sh + int64_t(f.x.tok0 + tok) * qy.st + lane % kLines * 64));
                }
                if (f_tile < f_end) {
                    const int page = page_at(f_index);
                    f_next = page_at(f_index + 1);
                    turn_page(page, (tiles_per_page - f_left) * kQ4Tile);
                }
                if (by_doc) {                            // of the tokens: sixteen rows at most
                    const int r = f.x.row0 + lane;
                    const bool in = lane < f.x.count && r >= 0;
                    const int d = in ? md.documents[int64_t(f.b) * md.doc_sb + int64_t(f.h) * md.doc_sh + r] : 0;
                    f_lo = __reduce_min_sync(0xffffffffu, in ? d : INT_MAX);
                    f_hi = __reduce_max_sync(0xffffffffu, in ? d : INT_MIN);
                }
                f_open = true;
            }
            if (f_tile >= f_end) { f_open = false; continue; }
            if (f_left == 0) {
                turn_page(f_next, 0);
                f_next = page_at(++f_index + 1);
                f_left = tiles_per_page;
            }
            const int tile = f_tile++;
            const uint8_t* const k_from = f_k, * const v_from = f_v, * const s_from = f_s;
            f_k += Shape::kCodeBytes; f_v += Shape::kCodeBytes; f_s += Shape::kScaleBytes;
            --f_left;
            const uint32_t to = ring + j * Shape::kSlotBytes;
            if (by_doc || biased) {
                const int t = tile * kQ4Tile + lane;
                const Segment& f = desk.loaded;
                const bool in = t < f.x.rows;
                if (by_doc) {                            // a tile without any of the tokens' documents is skipped
                    const int32_t* const at = md.documents + int64_t(f.b) * md.doc_sb + int64_t(f.h) * md.doc_sh + (in ? t : 0);
                    const int doc = *at;
                    if (!__any_sync(0xffffffffu, in && doc >= f_lo && doc <= f_hi)) continue;
                    cp_async_4(to + Shape::kLoadBytes + 4 * (kQ4Tile + lane), at, in);
                }
                if (biased) {
                    if (md.positions) cp_async_4(to + Shape::kLoadBytes + 4 * lane, md.positions + int64_t(f.b) * md.pos_sb + int64_t(f.h) * md.pos_sh + (in ? t : 0), in);
                    else *reinterpret_cast<int32_t*>(my_ring + j * Shape::kSlotBytes + Shape::kLoadBytes + 4 * lane) = t;
                }
            }
            if (f_there) {
#pragma unroll
                for (int i = 0; i < kCopies; ++i) {
                    cp_async_16(to + lane * 16 + i * 512, k_from + i * 512);
                    cp_async_16(to + Shape::kCodeBytes + v_to + i * 512, v_from + i * 512);
                }
                if (lane < 16) cp_async_16(to + 2 * Shape::kCodeBytes + lane * 16, s_from);
            } else {                                     // outside the pool: rows of zeros, whatever their codes
                uint32_t* const sc = reinterpret_cast<uint32_t*>(my_ring + j * Shape::kSlotBytes + 2 * Shape::kCodeBytes);
                sc[lane] = sc[lane + kQ4Tile] = 0u;
                if (lane == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
            }
            item_of[NST - 1] = f_item;
            tile_of[NST - 1] = tile;
            break;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int note_front = -1, note_ends = 0, note_back = -1;
    RowNote* const table = reinterpret_cast<RowNote*>(base_ptr + Shape::kTable) + warp * Shape::R;
    int item = mine.begin - 1, lim_all = 0, rows = 0, pos_ref = 0;
    bool open = false;                                   // an item is being worked on
    uint32_t qb[RH][2 * KW][2];
    float acc[RH][MT][4];
    float2 factor[RH], q_sum[RH], m_run[RH], l_run[RH], b_run[RH];               // of query rows 2 qd and 2 qd + 1
    float2 gain[RH], room[RH];                           // what weight times scale is multiplied by; largest logit times scale (base 2) so far
    // (one loop for everything, so that the code stands here once; the first NST rounds only fill the ring)
    for (int n_used = -NST;; ++n_used) {
        const int j = (n_used + NST) % NST;
        if (n_used >= 0) {
        if (open && item_of[0] != item) {
            // ---- the item's end: sums over the lanes' keys
#pragma unroll
            for (int n = 0; n < RH; ++n)
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    l_run[n].x += __shfl_xor_sync(0xffffffffu, l_run[n].x, d);
                    l_run[n].y += __shfl_xor_sync(0xffffffffu, l_run[n].y, d);
                    b_run[n].x += __shfl_xor_sync(0xffffffffu, b_run[n].x, d);
                    b_run[n].y += __shfl_xor_sync(0xffffffffu, b_run[n].y, d);
                }
            const Segment seg = desk.computed;
            const int count = seg.x.count;
            const bool begins = seg.lo == 0, ends = seg.hi >= seg.x.tiles;
            if (!begins) { note_front = seg.item; note_ends = ends; if (lane == 0) desk.front = seg; }
            else if (!ends) note_back = seg.item;
            // (a back piece is the last thing that its warp has: nothing is on its way into the ring any more)
            float* const piece = reinterpret_cast<float*>(begins ? my_ring : base_ptr + Shape::kFront + warp * Shape::kPieceBytes);
#pragma unroll
            for (int n = 0; n < RH; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int m = 8 * n + 2 * qd + c;
                    if (biased && fabsf(table[m].pos) > kFarToken) atomicOr(a.status, CSP_DEV_BAD_LEN);
                    if (m >= count * G) continue;
                    const float base_sum = c ? b_run[n].y : b_run[n].x, l = c ? l_run[n].y : l_run[n].x, mm = c ? m_run[n].y : m_run[n].x;
                    const float unit = rcpf(c ? gain[n].y : gain[n].x);
                    const int tok = pl.by_group(m), head = seg.h * G + m - tok * G;
                    const float inv = l == 0.f ? 0.f : 1.f / (n_term(a.n, mm) + l);      // l == 0: nothing was seen
                    uint16_t* const out = a.out + int64_t(seg.b) * a.o_sb + int64_t(head) * a.o_sh + int64_t(seg.x.tok0 + tok) * a.o_st + 4 * gr;
#pragma unroll
                    for (int t = 0; t < MT; t += 2) {        // dimensions 16 t + 4 gr to 16 t + 4 gr + 3
                        const float4 o = make_float4(fmaf(acc[n][t][c] * 0x1p24f, unit, base_sum), fmaf(acc[n][t][2 + c] * 0x1p20f, unit, base_sum),
                                                     fmaf(acc[n][t + 1][c] * 0x1p24f, unit, base_sum), fmaf(acc[n][t + 1][2 + c] * 0x1p20f, unit, base_sum));
                        if (begins && ends)
                            *reinterpret_cast<uint2*>(out + 16 * t) = l == 0.f ? make_uint2(0u, 0u) : make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
                        else
                            *reinterpret_cast<float4*>(piece + m * Shape::kPieceRow + 16 * t + 4 * gr) = o;
                    }
                    if (gr == 0) {
                        if (!(begins && ends)) *reinterpret_cast<float2*>(piece + m * Shape::kPieceRow + D) = make_float2(mm, l);
                        else if (a.lse)
                            a.lse[(int64_t(seg.b) * a.n_kv_heads * G + head) * a.max_new + seg.x.tok0 + tok] = l == 0.f ? -INFINITY : (mm + log2f(l)) * kLn2;
                    }
                }
            open = false;
        }
        if (!open) {
        Segment seg;
        if (f_item == item + 1) seg = desk.loaded;
        else if (!segment(item + 1, seg)) break;
        open = true;
        __syncwarp();
        if (lane == 0) desk.computed = seg;
        item = seg.item;
        rows = seg.x.rows;
        const int count = seg.x.count;
        const int32_t* const docs = by_doc ? md.documents + int64_t(seg.b) * md.doc_sb + int64_t(seg.h) * md.doc_sh : nullptr;
        const int32_t* const poss = biased && md.positions ? md.positions + int64_t(seg.b) * md.pos_sb + int64_t(seg.h) * md.pos_sh : nullptr;
        // ---- what comes from memory, all of it asked for before any of it is looked at: query row 8 n + gr, this lane's quarter of
        // it, and what the modifiers need to know of query row `lane`
        uint4 q[RH][KW];
#pragma unroll
        for (int n = 0; n < RH; ++n) {
            const int m = 8 * n + gr, tok = pl.by_group(m);       // rows that are none are zeros
            const uint16_t* const from = qy.q + int64_t(seg.b) * qy.sb + int64_t(seg.h * G + m - tok * G) * qy.sh + int64_t(seg.x.tok0 + tok) * qy.st + qd * KW * 8;
#pragma unroll
            for (int w = 0; w < KW; ++w) q[n][w] = tok < count ? reinterpret_cast<const uint4*>(from)[w] : make_uint4(0, 0, 0, 0);
        }
        {
            // positions are taken relative to the last token's, so that near ones are exact in fp32
            const int tok = pl.by_group(lane), r = seg.x.row0 + tok, row_last = max(seg.x.row0 + count - 1, 0);
            const bool valid = lane < Shape::R && tok < count, sees = valid && r >= 0;
            pos_ref = biased && rows > 0 ? (poss ? poss[row_last] : row_last) : 0;
            const int pos = biased && sees ? (poss ? poss[r] : r) : pos_ref, doc = docs && sees ? docs[r] : 0;
            const float slope = biased && sees ? md.slopes[seg.h * G + lane - tok * G] : 0.f;
            // rows that nobody asked for see everything: they must not send their warp through the masked path
            lim_all = !valid ? kSeesAll : sees ? max(r, seg.x.prefix - 1) : -1;
            if (lane < Shape::R) table[lane] = RowNote{lim_all, doc, float(pos - pos_ref), slope * kLog2e};
        }
        lim_all = min(__reduce_min_sync(0xffffffffu, lim_all), rows - 1);
        // ---- the queries in halves and in the order of the codes
#pragma unroll
        for (int n = 0; n < RH; ++n) {
            uint32_t top2 = 0;                           // the row's largest magnitude, two candidates
#pragma unroll
            for (int w = 0; w < KW; ++w) top2 = max_abs2(max_abs2(max_abs2(max_abs2(top2, q[n][w].x), q[n][w].y), q[n][w].z), q[n][w].w);
            top2 = max_abs2(top2, top2 >> 16 | top2 << 16);
            top2 = max_abs2(top2, __shfl_xor_sync(0xffffffffu, top2, 1));
            top2 = max_abs2(top2, __shfl_xor_sync(0xffffffffu, top2, 2));
            const uint32_t top = (top2 & 0x7fffu) >> 7, ex = max(top, 14u);      // top 255: an infinity, the row is no number
            const float down = __uint_as_float((264u - ex) << 23);        // 2^(10 - e)
            // logit = up (scale S + base sum 2^-20), S the product with codes 2^-20
            const float up = a.scale * kLog2e * 0x1p10f * (top == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(ex << 23));
            factor[n] = make_float2(__shfl_sync(0xffffffffu, up, 8 * qd), __shfl_sync(0xffffffffu, up, 8 * qd + 4));
            float total = 0.f;                           // the query's sum (in fp32: an error of it is one of all logits)
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float f[8] = {lo_bf16(q[n][w].x) * down, hi_bf16(q[n][w].x) * down, lo_bf16(q[n][w].y) * down, hi_bf16(q[n][w].y) * down,
                                    lo_bf16(q[n][w].z) * down, hi_bf16(q[n][w].z) * down, lo_bf16(q[n][w].w) * down, hi_bf16(q[n][w].w) * down};
                total += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
                qb[n][2 * w][0] = pack_f16(16.f * f[0], 16.f * f[4]);
                qb[n][2 * w][1] = pack_f16(f[1], f[5]);
                qb[n][2 * w + 1][0] = pack_f16(16.f * f[2], 16.f * f[6]);
                qb[n][2 * w + 1][1] = pack_f16(f[3], f[7]);
            }
            total += __shfl_xor_sync(0xffffffffu, total, 1);
            total = (total + __shfl_xor_sync(0xffffffffu, total, 2)) * 0x1p-20f;
            q_sum[n] = make_float2(__shfl_sync(0xffffffffu, total, 8 * qd), __shfl_sync(0xffffffffu, total, 8 * qd + 4));
            m_run[n] = make_float2(kNeg, kNeg);
            l_run[n] = b_run[n] = make_float2(0.f, 0.f);
            gain[n] = make_float2(kMostGain, kMostGain);
            room[n] = make_float2(kNeg, kNeg);
#pragma unroll
            for (int t = 0; t < MT; ++t) acc[n][t][0] = acc[n][t][1] = acc[n][t][2] = acc[n][t][3] = 0.f;
        }
        __syncwarp();
        if (item_of[0] != item) { --n_used; continue; }  // (an item without any tile for this warp)
        }
        {
            const int tile = tile_of[0];
            asm volatile("cp.async.wait_group %0;" ::"n"(NST - 1) : "memory");
            __syncwarp();
            const uint8_t* const k_s = my_ring + j * Shape::kSlotBytes;
            const uint32_t v_s = ring + j * Shape::kSlotBytes + Shape::kCodeBytes;
            const uint32_t* const ks_s = reinterpret_cast<const uint32_t*>(k_s + 2 * Shape::kCodeBytes);
            const uint32_t* const vs_s = ks_s + kQ4Tile;
            const int32_t* const pos_s = reinterpret_cast<const int32_t*>(vs_s + kQ4Tile), * const doc_s = pos_s + kQ4Tile;
            const int t0 = tile * kQ4Tile;
            // ---- S^T = K Q^T for 32 keys: two blocks of sixteen
            float2 x[2][RH][2];                      // [block][..][i]: key 8 i + gr, query rows 2 qd and 2 qd + 1
            uint32_t k_pair[2][2], v_pair[2][2];     // scale and base
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t kw[2][KW];
                float sum[RH][4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int key = 16 * k + 8 * i + gr;
                    k_pair[k][i] = ks_s[key];
                    v_pair[k][i] = vs_s[key];
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
                for (int n = 0; n < RH; ++n) sum[n][0] = sum[n][1] = sum[n][2] = sum[n][3] = 0.f;
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    const uint32_t y0 = kw[0][w], y1 = kw[1][w];
                    const uint32_t z0 = y0 >> 8, z1 = y1 >> 8;
#pragma unroll
                    for (int n = 0; n < RH; ++n) {
                        mma_f16(sum[n], y0 & kLow, y1 & kLow, y0 & kHigh, y1 & kHigh, qb[n][2 * w][0], qb[n][2 * w][1]);
                        mma_f16(sum[n], z0 & kLow, z1 & kLow, z0 & kHigh, z1 & kHigh, qb[n][2 * w + 1][0], qb[n][2 * w + 1][1]);
                    }
                }
#pragma unroll
                for (int n = 0; n < RH; ++n) { x[k][n][0] = make_float2(sum[n][0], sum[n][1]); x[k][n][1] = make_float2(sum[n][2], sum[n][3]); }
            }
            // ---- logits (base 2)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float sk = lo_bf16(k_pair[k][i]), bk = hi_bf16(k_pair[k][i]);
#pragma unroll
                    for (int n = 0; n < RH; ++n)
                        x[k][n][i] = make_float2(fmaf(sk, x[k][n][i].x, bk * q_sum[n].x) * factor[n].x, fmaf(sk, x[k][n][i].y, bk * q_sum[n].y) * factor[n].y);
                }
            if (capped) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int n = 0; n < RH; ++n)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float2& y = x[k][n][i];
                            y.x = fmaf(-2.f * cap2, rcpf(1.f + ex2f(y.x * cap_in)), cap2);
                            y.y = fmaf(-2.f * cap2, rcpf(1.f + ex2f(y.y * cap_in)), cap2);
                        }
            }
            if (biased) {
#pragma unroll
                for (int n = 0; n < RH; ++n) {
                    const RowNote r0 = table[8 * n + 2 * qd], r1 = table[8 * n + 2 * qd + 1];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float pos = float(pos_s[16 * k + 8 * i + gr] - pos_ref);
                            float2& y = x[k][n][i];
                            y.x = fmaf(-r0.slope2, fabsf(r0.pos - pos), y.x);
                            y.y = fmaf(-r1.slope2, fabsf(r1.pos - pos), y.y);
                        }
                }
            }
            if (by_doc || t0 + 31 > lim_all) {           // some query row does not see all of the tile's keys
                asm volatile("");                        // (a branch, and not all of it with predicates)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int key = 16 * k + 8 * i + gr, t = t0 + key, doc = by_doc ? doc_s[key] : 0;
                        if (t >= rows) v_pair[k][i] = 0u;            // what stands behind the last row may be no number
#pragma unroll
                        for (int n = 0; n < RH; ++n) {
                            const RowNote r0 = table[8 * n + 2 * qd], r1 = table[8 * n + 2 * qd + 1];
                            if (t > r0.lim || t >= rows || (by_doc && doc != r0.doc)) x[k][n][i].x = -INFINITY;
                            if (t > r1.lim || t >= rows || (by_doc && doc != r1.doc)) x[k][n][i].y = -INFINITY;
                        }
                    }
            }
            // ---- references: of the softmax, raised when exceeded by 2^8, and the products' factors, lowered when a product may exceed
            // kMostProduct (what it may be at most: the largest weight times the largest scale of this lane's keys)
            float2 mx[RH];
            const float v_top = lg2f(fmaxf(fmax3(lo_bf16(v_pair[0][0]), lo_bf16(v_pair[0][1]), lo_bf16(v_pair[1][0])), lo_bf16(v_pair[1][1])));
            float over = -INFINITY;
#pragma unroll
            for (int n = 0; n < RH; ++n) {
                mx[n].x = fmaxf(fmax3(x[0][n][0].x, x[0][n][1].x, x[1][n][0].x), x[1][n][1].x);
                mx[n].y = fmaxf(fmax3(x[0][n][0].y, x[0][n][1].y, x[1][n][0].y), x[1][n][1].y);
                over = fmax3(over, mx[n].x - fminf(m_run[n].x + kLazy, room[n].x - v_top), mx[n].y - fminf(m_run[n].y + kLazy, room[n].y - v_top));
            }
            if (__any_sync(0xffffffffu, over > 0.f)) {
#pragma unroll
                for (int n = 0; n < RH; ++n) {
                    float2 y = mx[n], top = make_float2(0.f, 0.f), alpha, keep;
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        y.x = fmaxf(y.x, __shfl_xor_sync(0xffffffffu, y.x, d));
                        y.y = fmaxf(y.y, __shfl_xor_sync(0xffffffffu, y.y, d));
                    }
                    const float2 m = make_float2(y.x > m_run[n].x + kLazy ? y.x : m_run[n].x, y.y > m_run[n].y + kLazy ? y.y : m_run[n].y);
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {        // (2^-16: a number, whatever the scale)
                            const float sv = lo_bf16(v_pair[k][i]);
                            top.x = fmaxf(top.x, ex2f(x[k][n][i].x - m.x) * 0x1p-16f * sv);
                            top.y = fmaxf(top.y, ex2f(x[k][n][i].y - m.y) * 0x1p-16f * sv);
                        }
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        top.x = fmaxf(top.x, __shfl_xor_sync(0xffffffffu, top.x, d));
                        top.y = fmaxf(top.y, __shfl_xor_sync(0xffffffffu, top.y, d));
                    }
                    // With the softmax's reference raised, the products so far stay as they are and those to come are held by as much
                    // more; where that is too much those so far are made smaller.
                    auto settle = [](float& m_old, float& g, float& r, float m_new, float w, float& alpha, float& keep) {
                        alpha = ex2f(m_old - m_new);
                        const float most = w * kMostGain > kMostProduct * 0x1p-16f
                            ? __uint_as_float(((254u - 16u + kTopProduct) << 23) - (__float_as_uint(fminf(w, 0x1p116f)) & 0x7f800000u)) : kMostGain;
                        const float more = g * ex2f(m_new - m_old);
                        const bool fits = more <= kMostGain && !(w * more > kMostProduct * 0x1p-16f);
                        keep = fits ? 1.f : alpha * most * rcpf(g);
                        g = fits ? more : most;
                        m_old = m_new;
                        r = m_new + (kMostProductLog - lg2f(g));
                    };
                    settle(m_run[n].x, gain[n].x, room[n].x, m.x, top.x, alpha.x, keep.x);
                    settle(m_run[n].y, gain[n].y, room[n].y, m.y, top.y, alpha.y, keep.y);
                    l_run[n] = __fmul2_rn(l_run[n], alpha);
                    b_run[n] = __fmul2_rn(b_run[n], alpha);
#pragma unroll
                    for (int t = 0; t < MT; ++t) { acc[n][t][0] *= keep.x; acc[n][t][1] *= keep.y; acc[n][t][2] *= keep.x; acc[n][t][3] *= keep.y; }
                }
            }
            // ---- weights
            uint32_t pb[2][RH][2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float sv = lo_bf16(v_pair[k][i]), bv = hi_bf16(v_pair[k][i]);
#pragma unroll
                    for (int n = 0; n < RH; ++n) {
                        const float2 y = __fadd2_rn(x[k][n][i], make_float2(-m_run[n].x, -m_run[n].y));
                        const float2 p = make_float2(ex2f(y.x), ex2f(y.y));
                        l_run[n] = __fadd2_rn(l_run[n], p);
                        b_run[n] = __ffma2_rn(p, make_float2(bv, bv), b_run[n]);
                        const float2 w = __fmul2_rn(__fmul2_rn(p, gain[n]), make_float2(sv, sv));
                        pb[k][n][i] = transpose8(pack_f16(w.x, w.y));
                    }
                }
            // ---- O^T += V^T P^T: pieces of four codes (dimensions 4 gr to 4 gr + 3 of 32), two keys each
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int c = 0; c < D / 32; c += 2) {
                    // matrices 1, 3: the second eight keys; 2, 3: the next sixteen bytes
                    const int row = 16 * k + ((lane >> 3) & 1) * 8 + (lane & 7), chunk = c + (lane >> 4);
                    uint32_t y[4];
                    ldsm_x4_t(y, v_s + row * (D / 2) + ((NH == 2 ? chunk ^ ((row >> 1) & 3) : chunk ^ ((row >> 2) & 1)) << 4));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t y0 = y[2 * i], y1 = y[2 * i + 1], z0 = y0 >> 8, z1 = y1 >> 8;
                        const int t = 2 * (c + i);
#pragma unroll
                        for (int n = 0; n < RH; ++n) {
                            mma_f16(acc[n][t], y0 & kLow, y0 & kHigh, y1 & kLow, y1 & kHigh, pb[k][n][0], pb[k][n][1]);
                            mma_f16(acc[n][t + 1], z0 & kLow, z0 & kHigh, z1 & kLow, z1 & kHigh, pb[k][n][0], pb[k][n][1]);
                        }
                    }
                }
            __syncwarp();
        }
        }
        refill(j);
    }
    if (lane == 0) notes[warp] = Notes{note_front, note_ends, note_back, 0};
    __syncthreads();
    // ---- the pieces of cut items: chain 0 goes on with what the block before began, chain c begins with warp c - 1's back piece
    // query row m of an item, joined: four columns per lane
    auto finish = [&](int b, int h, int tok0, int m, float mm, float l, const float4& o) {
        const int at = pl.by_group(m), tok = tok0 + at, head = (h - at) * G + m;
        const float inv = l == 0.f ? 0.f : 1.f / (n_term(a.n, mm) + l);
        if (lane < D / 4)
            *reinterpret_cast<uint2*>(a.out + int64_t(b) * a.o_sb + int64_t(head) * a.o_sh + int64_t(tok) * a.o_st + 4 * lane) =
                l == 0.f ? make_uint2(0u, 0u) : make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
        if (a.lse && lane == 0)
            a.lse[(int64_t(b) * a.n_kv_heads * G + head) * a.max_new + tok] = l == 0.f ? -INFINITY : (mm + log2f(l)) * kLn2;
    };
    int cut[2] = {-1, -1};                               // the item that goes on from the block before, the one that goes on in the next
    const Notes said = lane < NW ? notes[lane] : Notes{-1, 0, -1, 0};
    const uint32_t fronts = __ballot_sync(0xffffffffu, said.front >= 0), ended = __ballot_sync(0xffffffffu, said.front >= 0 && said.front_ends);
    uint32_t starts = __ballot_sync(0xffffffffu, said.back >= 0) << 1 | (fronts & 1u);
    // (the weighted sum of n rows of sums that lie at `row(p)`, with reference and sum of weights behind them: lane p looks at those)
    auto join = [&](auto row, int n, float& mm, float& l, float4& o) {
        mm = kNeg;
        l = 0.f;
        o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p0 = 0; p0 < n; p0 += 32) {
            const float2 ml = p0 + lane < n ? row.ml(p0 + lane) : make_float2(kNeg, 0.f);
            float top = fmaxf(mm, ml.x);
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float keep = ex2f(mm - top), mine = ex2f(ml.x - top);
            mm = top;
            float sum = ml.y * mine;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            l = fmaf(l, keep, sum);
            o.x *= keep; o.y *= keep; o.z *= keep; o.w *= keep;
#pragma unroll 4
            for (int p = 0; p < min(n - p0, 32); ++p) {
                const float w = __shfl_sync(0xffffffffu, mine, p);
                const float4 y = row.sums(p0 + p);
                o.x = fmaf(y.x, w, o.x); o.y = fmaf(y.y, w, o.y); o.z = fmaf(y.z, w, o.z); o.w = fmaf(y.w, w, o.w);
            }
        }
    };
    const int col = lane % (D / 4) * 4;                  // four columns per lane (at d = 64 two lanes have the same)
    while (starts) {
        const int c = __ffs(starts) - 1;
        starts &= starts - 1;
        const int from = c == 0 ? 0 : c - 1;             // pieces: of warps from up to next - 1
        const uint32_t mine_f = fronts >> c, mine_e = ended >> c;
        int next = c + __ffs(~mine_f) - 1;               // the first warp from c on that did not go on with anything
        const int end = mine_e ? c + __ffs(mine_e) : NW + 1;
        const bool done = end <= next;
        if (done) next = end;
        const Desk* const whose = reinterpret_cast<const Desk*>(base_ptr + Shape::kDesk + kDeskBytes * from);
        const Segment* const d = c == 0 ? &whose->front : &whose->computed;
        if (!(c > 0 && done)) cut[c > 0] = d->item;
        struct Pieces {
            const uint8_t* front; const uint8_t* first; int col;
            __device__ __forceinline__ const float* at(int p) const { return reinterpret_cast<const float*>(p == 0 ? first : front + p * Shape::kPieceBytes); }
            __device__ __forceinline__ float2 ml(int p) const { return *reinterpret_cast<const float2*>(at(p) + D); }
            __device__ __forceinline__ float4 sums(int p) const { return *reinterpret_cast<const float4*>(at(p) + col); }
        };
        for (int m = (warp + NW - c % NW) % NW; m < d->x.count * G; m += NW) {           // (another chain begins with another warp)
            const uint8_t* const front = base_ptr + Shape::kFront + from * Shape::kPieceBytes + m * Shape::kPieceRow * 4;
            float mm, l;
            float4 o;
            join(Pieces{front, c == 0 ? front : base_ptr + from * NST * Shape::kSlotBytes + m * Shape::kPieceRow * 4, col}, next - from, mm, l, o);
            if (c > 0 && done) {
                finish(d->b, d->h, d->x.tok0, m, mm, l, o);
            } else {
                const int64_t slot = int64_t(2 * blockIdx.x + (c > 0 ? 1 : 0)) * pl.row_slots + m;
                *reinterpret_cast<float4*>(partial + slot * D + col) = o;
                if (lane == 0) partial_ml[slot] = make_float2(mm, l);
            }
        }
    }
    if (cut[0] < 0 && cut[1] < 0) return;
    // ---- the parts of an item that is cut between blocks are joined by the block that brings the last one.  Of how many have
    // been brought, the status area counts in a byte for each block that such an item begins in; they are zero again at the end.
    int* const chains = reinterpret_cast<int*>(base_ptr + Shape::kChains);
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        for (int k = 0; k < 2; ++k) {
            chains[4 + k] = 0;
            if (cut[k] < 0) continue;
            const int first = chains[2 * k], n = chains[2 * k + 1], shift = 8 * (first & 3);
            uint32_t* const count = reinterpret_cast<uint32_t*>(a.status) + kCountWord + (first >> 2);
            if (int(atomicAdd(count, 1u << shift) >> shift & 255u) != n - 1) continue;
            atomicSub(count, uint32_t(n) << shift);
            chains[4 + k] = 1;
        }
        __threadfence();
    }
    __syncthreads();
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
        if (cut[k] < 0 || !chains[4 + k]) continue;
        const int first = chains[2 * k], n = chains[2 * k + 1], item = cut[k];
        const int u = pl.by_pairs(item), b = pl.by_heads(u), h = u - b * a.n_kv_heads;
        const PairRange x = pair_range(a, pl, u, item - u * pl.n_pairs);
        struct Parts {
            const float* o; const float2* m; int first, rows, col;
            __device__ __forceinline__ int64_t at(int p) const { return int64_t(2 * (first + p) + (p == 0 ? 1 : 0)) * rows; }
            __device__ __forceinline__ float2 ml(int p) const { return __ldcg(m + at(p)); }
            __device__ __forceinline__ float4 sums(int p) const { return __ldcg(reinterpret_cast<const float4*>(o + at(p) * D + col)); }
        };
        for (int m = warp; m < x.count * G; m += NW) {
            float mm, l;
            float4 o;
            join(Parts{partial + m * D, partial_ml + m, first, pl.row_slots, col}, n, mm, l, o);
            finish(b, h, x.tok0, m, mm, l, o);
        }
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------

// Tokens of an item here; 0: more query rows than this kernel is for, row tiles of 128.  The cache is read once per item, of which
// there are n8 of up to eight rows or n16 of up to sixteen.  One of sixteen takes as long as one and a half of eight where caches
// are long; where they are short the smaller code starts and ends 3 us earlier.  Measured, 8 x 32 / 8 heads, items of 8 and of 16:
// 16 query rows over 4 K rows 26.5 and 28 us, over 16 K rows 65.5 and 58; 20 query rows 32.6 and 36, 94 and 99.5; 32 query rows
// 38.6 and 38.2, 123 and 99; 48 query rows 51 and 47.4 (row tiles 59.6), 175 and 142 (157).
constexpr int kMostItems = 3;                            // of sixteen rows
int few_tokens(const csp_params& p, int max_new) {
    const int G = p.n_q_heads / p.n_kv_heads, eight = 8 / G, sixteen = 16 / G;
    const int64_t n8 = (int64_t(max_new) + eight - 1) / eight, n16 = (int64_t(max_new) + sixteen - 1) / sixteen;
    if (n16 > kMostItems) return 0;
    return (2 * n8 - 3 * n16) * p.batch * p.n_kv_heads <= (1 << 19) / (int64_t(p.out_capacity) + 1) ? eight : sixteen;
}

ChunkPlan chunk_q4_plan(const csp_params& p, int max_new, bool* few) {
    ChunkPlan pl = chunk_plan(p, max_new);
    const int G = p.n_q_heads / p.n_kv_heads, tokens = few_tokens(p, max_new);
    *few = tokens > 0;
    if (!*few) return pl;
    pl.tok_tile = pl.pair_tokens = tokens;
    pl.n_pairs = max_new > tokens ? (max_new + tokens - 1) / tokens : 1;
    pl.row_slots = (max_new < tokens ? max_new : tokens) * G;
    pl.snap = 0x3fffffff;
    pl.key_tile = kQ4Tile;
    pl.min_tiles = 4;
    pl.item_cost = 4;
    const int64_t items = int64_t(p.batch) * p.n_kv_heads * pl.n_pairs;
    const int64_t weight = (int64_t(p.out_capacity) + pl.key_tile - 1) / pl.key_tile + pl.item_cost;      // of an item, at most
    pl.n_items = items > 0x3fffffffLL / weight ? -1 : int(items);
    // no more blocks than there can be shares of the smallest size
    const int64_t most = (items > 65536 ? 65536 : items) * weight / (pl.item_cost + pl.min_tiles) + 1;
    const int blocks = sm_count() < kMostBlocks ? sm_count() : kMostBlocks;
    pl.grid = most < blocks ? int(most) : blocks;
    set_dividers(p, pl);
    return pl;
}

template <int NH, int RH, int kMods>
csp_status launch_few_mods(const ChunkArgs& a, const ChunkPlan& pl, const FewQuery& q, const Q4Args& c, float* partial, float2* ml,
                      cudaStream_t s) {
    constexpr int smem = int(Q4Shape<NH, RH>::kTotal) + 128;
    static_assert(smem <= 227 * 1024, "shared memory of one CTA");
    auto kern = chunk_q4_few_kernel<NH, RH, kMods>;
    static std::atomic<bool> configured[kMaxDevices];
    if (!raise_smem_limit(kern, smem, configured)) return CSP_ERR_CUDA;
    kern<<<pl.grid, Q4Shape<NH, RH>::kThreads, smem, s>>>(a, pl, q, c, partial, ml);
    return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA;
}

template <int NH, int RH>
csp_status launch_few(const ChunkArgs& a, const ChunkPlan& pl, const FewQuery& q, const Q4Args& c, float* partial, float2* ml,
                      cudaStream_t s) {
    const bool cap = a.mods.softcap > 0.f, bias = a.mods.slopes;
    if (a.mods.documents || (cap && bias)) return launch_few_mods<NH, RH, kAny>(a, pl, q, c, partial, ml, s);
    return cap ? launch_few_mods<NH, RH, kCap>(a, pl, q, c, partial, ml, s) : bias ? launch_few_mods<NH, RH, kBias>(a, pl, q, c, partial, ml, s)
                                                                                   : launch_few_mods<NH, RH, kNone>(a, pl, q, c, partial, ml, s);
}

}  // namespace

size_t chunk_q4_workspace_bytes(const csp_params& p, int max_new) {
    if (p.dtype != CSP_BF16 || (p.head_dim != 64 && p.head_dim != 128)) return 0;
    if (p.out_capacity > (1 << 30)) return 0;                                    // a row index plus some tiles fits 32 bits
    if (int64_t(max_new) * (p.n_q_heads / p.n_kv_heads) > (1 << 24)) return 0;   // and so do a chunk's rows
    bool few;
    const ChunkPlan pl = chunk_q4_plan(p, max_new, &few);
    if (pl.n_items < 0) return 0;                                                // key tiles are counted in 32 bits
    // Enough for shorter chunks as well: those of a few small items have other tiles and shares.  (Among chunks with items of one
    // size the need grows with max_new.)
    size_t mine = partial_layout(p, pl).total;
    const int G = p.n_q_heads / p.n_kv_heads, longest = kMostItems * (16 / G);
    int eight = -1, sixteen = -1;                        // the longest chunks of either kind
    for (int n = 0; n <= (max_new < longest ? max_new : longest); ++n) (few_tokens(p, n) == 8 / G ? eight : sixteen) = n;
    for (const int n : {eight, sixteen}) {
        if (n < 0 || n == max_new) continue;
        const size_t shorter = partial_layout(p, chunk_q4_plan(p, n, &few)).total;
        if (shorter > mine) mine = shorter;
    }
    return mine;
}

csp_status launch_chunk_q4(const csp_params& p, const ChunkArgs& a, const csp_tensor& q, const Q4Args& c, void* ws, cudaStream_t s) {
    bool few;
    ChunkPlan pl = chunk_q4_plan(p, a.max_new, &few);
    const PartialLayout lay = partial_layout(p, pl);
    float* const partial = reinterpret_cast<float*>(static_cast<char*>(ws) + lay.o);
    float2* const ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + lay.ml);
    if (few) {
        const FewQuery qy = {static_cast<const uint16_t*>(q.ptr), q.stride_b, q.stride_h, q.stride_t, divider(a.page_rows / kQ4Tile)};
        if (pl.row_slots <= 8)
            return p.head_dim == 64 ? launch_few<1, 1>(a, pl, qy, c, partial, ml, s) : launch_few<2, 1>(a, pl, qy, c, partial, ml, s);
        return p.head_dim == 64 ? launch_few<1, 2>(a, pl, qy, c, partial, ml, s) : launch_few<2, 2>(a, pl, qy, c, partial, ml, s);
    }
    pl.drawn = a.mods.documents && pl.n_items >= 2 * pl.grid;
    ChunkParts* const parts = reinterpret_cast<ChunkParts*>(static_cast<char*>(ws) + lay.parts);
    const csp_status st = launch_chunk_q4_many(p, a, pl, q, c, parts, partial, ml, s);
    // nothing is cut by a single block, and where two parts of min_tiles are more than a cache has
    if (st != CSP_OK || pl.grid == 1 || p.out_capacity <= (2 * pl.min_tiles - 1) * pl.key_tile) return st;
    return launch_chunk_join(p, a, pl, false, parts, partial, ml, s);
}

}  // namespace csp
