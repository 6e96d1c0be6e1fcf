// New rows on their way into the pages: keys and queries rotated by their positions, rows quantised to 4 bits, and rows of a
// 4-bit cache read back.
//
// Rotation.  Dimensions (x1, x2) of a pair become (x1 cos - x2 sin, x2 cos + x1 sin), the angles from the caller's table; four
// products and two sums, each rounded to fp32, and one rounding to the row's type.
// Four bits.  base = min x, scale = (max x - base) / 15 rounded to bf16, code = the whole number nearest to (x - base) / scale.  The
// quotient is a product with 1 / scale (1 + 2^-21): the three roundings on the way (2^-24 each) cannot bring a quotient that lies
// halfway between two codes, which values of 8 bits often do, below the middle, so that the upper code is taken always and not
// now and then.
//
// A row of d values is held by d / 16 neighbouring lanes, sixteen values each, so that the row's extremes take three shuffles, and
// a pair is always in one thread: with halves paired a lane takes eight values from each half.  A group of lanes keeps its
// token and goes over the heads, so that its eight cosines and sines are loaded once.
//
// Measured (bound by HBM where there are many rows, by launch and dependent loads where there are few): rotation of one token of
// 32 x 32 heads 2.8 us, of 513 - 1024 tokens of 4 x 32 / 8 heads 17.7 us (4.35 TB/s); 262 K unrotated rows to 4 bits 37 us (4.6 TB/s, two
// thirds of the issue slots); 650 K rows read back as bf16 71 us (6 TB/s).
#include "csp_internal.cuh"

namespace csp {
namespace {

constexpr int kThreads = 256;
constexpr int kCountWord = 12;                           // of the status area: blocks that are done; left at zero
constexpr float kSmallest = 1.17549435e-38f;             // 2^-126

__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint4 ld_stream(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// eight neighbouring values of a row, as they lie in memory
template <bool kF32> struct Eight { uint4 x[kF32 ? 2 : 1]; };
template <bool kF32>
__device__ __forceinline__ Eight<kF32> load_eight(const void* row, int chunk) {
    Eight<kF32> r;
    const uint4* const p = static_cast<const uint4*>(row) + chunk * (kF32 ? 2 : 1);
#pragma unroll
    for (int j = 0; j < (kF32 ? 2 : 1); ++j) r.x[j] = ld_stream(p + j);
    return r;
}
template <bool kF32>
__device__ __forceinline__ void store_eight(void* row, int chunk, const Eight<kF32>& r) {
    uint4* const p = static_cast<uint4*>(row) + chunk * (kF32 ? 2 : 1);
#pragma unroll
    for (int j = 0; j < (kF32 ? 2 : 1); ++j) p[j] = r.x[j];
}
template <bool kF32>
__device__ __forceinline__ void widen(const Eight<kF32>& r, float* f) {
    const uint32_t* const w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = kF32 ? __uint_as_float(w[j]) : (j & 1 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]));
}
template <bool kF32>
__device__ __forceinline__ Eight<kF32> narrow(const float* f) {
    Eight<kF32> r;
    uint32_t* const w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
    for (int j = 0; j < (kF32 ? 8 : 4); ++j) w[j] = kF32 ? __float_as_uint(f[j]) : pack_bf16(f[2 * j], f[2 * j + 1]);
    return r;
}

// What the call does with unit (b, h): its first new row, how many follow, and how many the caller brings (of which none
// are stored where they do not fit).  Flags what it refuses.
struct NewRows { int first, stored, brought; };
__device__ __forceinline__ NewRows new_rows(const AppendRowsArgs& a, int b, int h, bool flag) {
    NewRows x;
    int bad = 0;
    const int u = b * a.n_kv_heads + h;
    x.first = a.n_rows[u];
    x.brought = a.n_new ? a.n_new[a.n_new_per_head ? u : b] : a.max_new;
    if (x.brought < 0 || x.brought > a.max_new) { bad |= CSP_DEV_BAD_LEN; x.brought = x.brought < 0 ? 0 : a.max_new; }
    x.stored = x.brought;
    if (x.first < 0) { bad |= CSP_DEV_BAD_LEN; x.stored = 0; }
    else if (int64_t(x.first) + x.brought > a.capacity) { bad |= CSP_DEV_CAPACITY; x.stored = 0; }
    if (flag && bad) atomicOr(a.status, bad);
    return x;
}

__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// the smallest and the largest of a bf16 row's values, of which every lane has sixteen (two at a time: they are bf16 values)
template <int kLanes>
__device__ __forceinline__ void row_range(const Eight<false>& r0, const Eight<false>& r1, uint32_t lanes, float& lo, float& hi) {
    const uint32_t w[8] = {r0.x[0].x, r0.x[0].y, r0.x[0].z, r0.x[0].w, r1.x[0].x, r1.x[0].y, r1.x[0].z, r1.x[0].w};
    uint32_t l = w[0], h = w[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) { l = min2_nan(l, w[j]); h = max2_nan(h, w[j]); }
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) {
        l = min2_nan(l, __shfl_xor_sync(lanes, l, d));
        h = max2_nan(h, __shfl_xor_sync(lanes, h, d));
    }
    lo = min_nan(bf16_lo(l), bf16_hi(l));
    hi = max_nan(bf16_lo(h), bf16_hi(h));
}
__device__ __forceinline__ uint32_t eight_codes(const float* f, float lo, float inv) {
    // Adding 1.5 x 2^23 rounds to a whole number, which is then what the number's bits are more than 0x4b400000.  The code before
    // goes along as sixteen times itself, so that four of them end up in the lowest sixteen bits: values 0 - 3 in one float, 4 - 7 in
    // another.
    constexpr float kWhole = 12582912.f;
    const float2 neg = make_float2(-lo, -lo), inv2 = make_float2(inv, inv);
    float2 r = make_float2(kWhole, kWhole);
#pragma unroll
    for (int j = 3; j >= 0; --j) {
        if (j < 3) r = __ffma2_rn(r, make_float2(16.f, 16.f), make_float2(-15.f * kWhole, -15.f * kWhole));
        r = __ffma2_rn(__fadd2_rn(make_float2(f[j], f[j + 4]), neg), inv2, r);
    }
    return __byte_perm(__float_as_uint(r.x), __float_as_uint(r.y), 0x5410);
}
// t / n and what is left, with m = 2^32 / n + 1 rounded down (t < 2^31: the product is at most one too many)
__device__ __forceinline__ uint32_t divide(uint32_t t, uint32_t n, uint32_t m, uint32_t& rest) {
    uint32_t q = __umulhi(t, m);
    rest = t - q * n;
    if (int32_t(rest) < 0) { --q; rest += n; }
    return q;
}

// (hi - lo) / 15 as a number that bf16 rounds like the exact quotient.  A product with fl(1/15) is off by less than two units in the last
// place: enough to be on the other side of the middle between two bf16 numbers.  Only next to one is the remainder looked at: 15 times the
// middle has thirteen bits, so that hi - lo less it, and what rounding hi - lo has lost, are exact in their signs.
__device__ __forceinline__ float fifteenth(float lo, float hi) {
    const float spread = __fsub_rn(hi, lo);
    float q = __fmul_rn(spread, 1.f / 15.f);
    const uint32_t bits = __float_as_uint(q);
    if (((bits + 0x8004u) & 0xffffu) < 8u) {             // up to four units from the middle
        const uint32_t middle = (bits & 0xffff0000u) | 0x8000u;
        const float back = __fsub_rn(spread, hi);        // -lo, as far as it is in `spread`
        const float lost = __fsub_rn(__fsub_rn(hi, __fsub_rn(spread, back)), __fadd_rn(lo, back));
        const float rest = __fadd_rn(__fmaf_rn(-15.f, __uint_as_float(middle), spread), lost);
        q = __uint_as_float(rest > 0.f ? middle + 1u : rest < 0.f ? middle - 1u : middle);
    }
    return q;
}
// A row of bf16 values in 4 bits: the lane's two words, and what the row's first lane writes beside them.
template <int kLanes>
__device__ __forceinline__ uint32_t quantise(const Eight<false>* z, uint32_t lanes, uint32_t& w0, uint32_t& w1) {
    float lo, hi, f[16];
    row_range<kLanes>(z[0], z[1], lanes, lo, hi);
    uint32_t pair = pack_bf16(fifteenth(lo, hi), lo);
    float scale = bf16_lo(pair);
    if (scale < kSmallest) { scale = 0.f; pair &= 0xffff0000u; }
    if (!(scale < INFINITY)) pair |= 0x7fffu;            // the whole row is no number
    const float inv = scale > 0.f ? __fmul_rn(__frcp_rn(scale), 1.f + 0x1p-21f) : 0.f;
    widen<false>(z[0], f);
    widen<false>(z[1], f + 8);
    w0 = eight_codes(f, lo, inv);
    w1 = eight_codes(f + 8, lo, inv);
    return pair;
}

// The counts.  Where they are updated in place, only the last block to finish does it: all others have read them.  `mine`: this block
// writes heads [h0, h1) of sequence b where they go elsewhere.
__device__ __forceinline__ void count_rows(const AppendRowsArgs& a, bool mine, int b, int h0, int h1) {
    const int tid = threadIdx.x, H = a.n_kv_heads;
    if (a.n_rows_out != a.n_rows) {
        if (!mine) return;
        for (int h = h0 + tid; h < h1; h += kThreads) {
            const NewRows x = new_rows(a, b, h, true);
            a.n_rows_out[b * H + h] = x.first + x.stored;
        }
        return;
    }
    __shared__ int last;
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        last = atomicAdd(a.status + kCountWord, 1) == int(gridDim.x * gridDim.y) - 1;
    }
    __syncthreads();
    if (!last) return;
    for (int u = tid; u < a.batch * H; u += kThreads) {
        const NewRows x = new_rows(a, u / H, u % H, true);
        a.n_rows_out[u] = x.first + x.stored;
    }
    if (tid == 0) a.status[kCountWord] = 0;
}

// Grid (token tiles of a sequence x sequences, pieces of the heads).  Bound by memory: every byte is read and written once.  A
// step takes two rows of a token, K and V of a head or two heads of Q, so that what belongs to the token is computed once for
// both and 64 bytes are on their way per lane.
template <bool kF32, bool kFour, int kLanes>             // kLanes = d / 16
__global__ void __launch_bounds__(kThreads, kF32 ? 3 : 4) append_rows_kernel(const AppendRowsArgs a) {
    const int tid = threadIdx.x, L = tid % kLanes, group = tid / kLanes;
    const uint32_t lanes = ((1u << kLanes) - 1u) << (tid % 32 - L);                  // of the row
    const int b = blockIdx.x / a.token_tiles, tile = blockIdx.x - b * a.token_tiles;
    const int H = a.n_kv_heads, pairs = H + (a.n_q_heads + 1) / 2;
    const int log_tok = a.log_tokens, strides = (kThreads / kLanes) >> log_tok;      // groups per token
    const int local = group & ((1 << log_tok) - 1);
    const int pair0 = int(blockIdx.y) * a.pairs_per_block, pair1 = min(pair0 + a.pairs_per_block, pairs);
    const int pair_lanes = a.rope.dim / 16;              // lanes whose values are rotated
    const bool turned = L < pair_lanes, halves = turned && !a.rope.interleaved;
    // Eights of a row that the lane has: neighbouring lanes' side by side, so that 32-byte sectors are whole in every access (with
    // 2 L and 2 L + 1 reading back takes 80 us instead of 72) ...
    const int c0 = L, c1 = L + kLanes;
    // ... but of a row that is rotated those with whole pairs, of which the first pair_lanes lanes have all
    const int r0 = halves ? L : 2 * L, r1 = halves ? L + pair_lanes : 2 * L + 1;
    const bool lead = tile == 0 && blockIdx.y == 0;
    // (token tiles beyond the grid's: a tile per step)
    for (int64_t t0 = int64_t(tile) << log_tok; t0 + local < a.max_new; t0 += int64_t(a.token_tiles) << log_tok) {
        const int i = int(t0) + local;
        auto token = [&](const RowTensor& x) { return static_cast<char*>(x.ptr) + b * x.sb + i * x.st; };
        float cs[8], sn[8];
        int at = -1;                                     // row of the table that cs and sn come from
        auto turn = [&](Eight<kF32>& x0, Eight<kF32>& x1, int row) {
            if (!turned) return;
            float f[16];
            widen<kF32>(x0, f);
            widen<kF32>(x1, f + 8);
            int pos = a.rope.positions ? a.rope.positions[b * a.rope.pos_sb + i] : row;
            if (pos < 0 || pos >= a.rope.table_rows) {
                if (L == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
                pos = pos < 0 ? 0 : a.rope.table_rows - 1;
            }
            if (pos != at) {
                at = pos;
                const float* const row_cs = a.rope.cos_sin + pos * a.rope.row_stride + 8 * L;
                const float* const row_sn = row_cs + a.rope.dim / 2;
#pragma unroll
                for (int j = 0; j < 8; j += 4) {
                    const float4 y = *reinterpret_cast<const float4*>(row_cs + j), z = *reinterpret_cast<const float4*>(row_sn + j);
                    cs[j] = y.x; cs[j + 1] = y.y; cs[j + 2] = y.z; cs[j + 3] = y.w;
                    sn[j] = z.x; sn[j + 1] = z.y; sn[j + 2] = z.z; sn[j + 3] = z.w;
                }
            }
            if (halves) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float y1 = f[j], y2 = f[j + 8];
                    f[j] = __fsub_rn(__fmul_rn(y1, cs[j]), __fmul_rn(y2, sn[j]));
                    f[j + 8] = __fadd_rn(__fmul_rn(y2, cs[j]), __fmul_rn(y1, sn[j]));
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float y1 = f[2 * j], y2 = f[2 * j + 1];
                    f[2 * j] = __fsub_rn(__fmul_rn(y1, cs[j]), __fmul_rn(y2, sn[j]));
                    f[2 * j + 1] = __fadd_rn(__fmul_rn(y2, cs[j]), __fmul_rn(y1, sn[j]));
                }
            }
            x0 = narrow<kF32>(f);
            x1 = narrow<kF32>(f + 8);
        };
        for (int s = pair0 + (group >> log_tok); s < pair1; s += strides) {
            Eight<kF32> x[2], y[2];
            if (s < H) {                                 // K and V of a head
                const NewRows n = new_rows(a, b, s, false);
                if (i >= n.stored) continue;
                const char* const k_row = token(a.k_new) + s * a.k_new.sh, * const v_row = token(a.v_new) + s * a.v_new.sh;
                x[0] = load_eight<kF32>(k_row, r0);
                x[1] = load_eight<kF32>(k_row, r1);
                y[0] = load_eight<kF32>(v_row, c0);
                y[1] = load_eight<kF32>(v_row, c1);
                uint32_t slot;
                const int page = a.page_table[int64_t(b) * a.max_pages + divide(uint32_t(n.first + i), uint32_t(a.page_rows), a.page_inverse, slot)];
                if (page < 0 || page >= a.n_pages) {
                    if (L == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
                    continue;
                }
                turn(x[0], x[1], n.first + i);           // (rounded to bf16 as a cache of these would hold it, and then to 4 bits)
                auto store = [&](const RowTensor& to, const RowTensor& sc, const Eight<kF32>* z, int z0, int z1) {
                    char* const row = static_cast<char*>(to.ptr) + page * to.sb + s * to.sh + slot * to.st;
                    if constexpr (!kFour) {
                        store_eight<kF32>(row, z0, z[0]);
                        store_eight<kF32>(row, z1, z[1]);
                    } else {
                        uint32_t w0, w1;
                        const uint32_t pair = quantise<kLanes>(z, lanes, w0, w1);
                        reinterpret_cast<uint32_t*>(row)[z0] = w0;
                        reinterpret_cast<uint32_t*>(row)[z1] = w1;
                        if (L == 0) *reinterpret_cast<uint32_t*>(static_cast<char*>(sc.ptr) + page * sc.sb + s * sc.sh + int64_t(slot) * 4) = pair;
                    }
                };
                store(a.k, a.k_scales, x, r0, r1);
                store(a.v, a.v_scales, y, c0, c1);
            } else {                                     // two heads of Q
                const int h0 = 2 * (s - H), h1 = h0 + 1;
                uint32_t rest;
                auto kv_head = [&](int h) { return a.group > 1 ? int(divide(uint32_t(h), uint32_t(a.group), a.group_inverse, rest)) : h; };
                const NewRows n0 = new_rows(a, b, kv_head(h0), false), n1 = h1 < a.n_q_heads ? new_rows(a, b, kv_head(h1), false) : NewRows{0, 0, 0};
                const char* const from = token(a.q);
                char* const to = token(a.q_out);
                const bool do0 = i < n0.brought, do1 = i < n1.brought;
                if (do0) { x[0] = load_eight<kF32>(from + h0 * a.q.sh, r0); x[1] = load_eight<kF32>(from + h0 * a.q.sh, r1); }
                if (do1) { y[0] = load_eight<kF32>(from + h1 * a.q.sh, r0); y[1] = load_eight<kF32>(from + h1 * a.q.sh, r1); }
                if (do0) {
                    turn(x[0], x[1], n0.first + i);
                    store_eight<kF32>(to + h0 * a.q_out.sh, r0, x[0]);
                    store_eight<kF32>(to + h0 * a.q_out.sh, r1, x[1]);
                }
                if (do1) {
                    turn(y[0], y[1], n1.first + i);
                    store_eight<kF32>(to + h1 * a.q_out.sh, r0, y[0]);
                    store_eight<kF32>(to + h1 * a.q_out.sh, r1, y[1]);
                }
            }
        }
    }
    count_rows(a, lead, b, 0, H);
}

// Rows that are not rotated, to pages in 4 bits.  Block (u, .) takes kGroups x kAppendDepth rows of a unit's K and V at a time, so that
// what belongs to the unit is computed once; behind the unit's last row there is nothing to do.  (In the kernel above, whose blocks
// go over the heads: 42 us for 262 K rows, of which a head has between a quarter and all, against 37.)
constexpr int kAppendDepth = 2;
template <int kLanes>
__global__ void __launch_bounds__(kThreads, 4) append_units_kernel(const AppendRowsArgs a) {
    constexpr int kGroups = kThreads / kLanes;           // rows per step
    const int u = blockIdx.x, b = u / a.n_kv_heads, h = u - b * a.n_kv_heads;
    const int L = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    const uint32_t lanes = ((1u << kLanes) - 1u) << (threadIdx.x % 32 - L);          // of the row
    const NewRows n = new_rows(a, b, h, false);
    const int32_t* const table = a.page_table + int64_t(b) * a.max_pages;
    const char* const from[2] = {static_cast<const char*>(a.k_new.ptr) + b * a.k_new.sb + h * a.k_new.sh,
                                 static_cast<const char*>(a.v_new.ptr) + b * a.v_new.sb + h * a.v_new.sh};
    const uint32_t stored = uint32_t(n.stored);          // (below 2^31: a step past it is still a number of 32 bits)
    for (uint32_t i0 = blockIdx.y * kGroups * kAppendDepth; i0 < stored; i0 += gridDim.y * kGroups * kAppendDepth) {
        Eight<false> x[kAppendDepth][2][2];
        int page[kAppendDepth];
        uint32_t slot[kAppendDepth];
#pragma unroll
        for (int j = 0; j < kAppendDepth; ++j) {
            const uint32_t i = i0 + j * kGroups + group;
            if (i >= stored) continue;
            page[j] = table[divide(uint32_t(n.first) + i, uint32_t(a.page_rows), a.page_inverse, slot[j])];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const char* const row = from[k] + i * (k ? a.v_new.st : a.k_new.st);
                x[j][k][0] = load_eight<false>(row, L);
                x[j][k][1] = load_eight<false>(row, L + kLanes);
            }
        }
#pragma unroll
        for (int j = 0; j < kAppendDepth; ++j) {
            if (i0 + j * kGroups + group >= stored) continue;
            if (page[j] < 0 || page[j] >= a.n_pages) {
                if (L == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
                continue;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const RowTensor& to = k ? a.v : a.k, & sc = k ? a.v_scales : a.k_scales;
                uint32_t w0, w1;
                const uint32_t pair = quantise<kLanes>(x[j][k], lanes, w0, w1);
                uint32_t* const row = reinterpret_cast<uint32_t*>(static_cast<char*>(to.ptr) + page[j] * to.sb + h * to.sh + slot[j] * to.st);
                row[L] = w0;
                row[L + kLanes] = w1;
                if (L == 0) *reinterpret_cast<uint32_t*>(static_cast<char*>(sc.ptr) + page[j] * sc.sb + h * sc.sh + int64_t(slot[j]) * 4) = pair;
            }
        }
    }
    count_rows(a, blockIdx.y == 0, b, h, h + 1);
}

// Rows [first, n_rows) of every unit as numbers again: base + scale code, rounded once to fp32 and, for bf16, once more.  Block
// (u, .) takes kLoadDepth rows per group of lanes at a time; a lane has sixteen values (8 bytes of codes), a row d / 16 lanes.
// Bound by memory, above all by what it writes.
template <bool kF32, int kLanes, int kLoadDepth>
__global__ void __launch_bounds__(kThreads) load_rows_kernel(const LoadRowsArgs a) {
    constexpr int kGroups = kThreads / kLanes;           // rows per step
    const int u = blockIdx.x, b = u / a.n_kv_heads, h = u - b * a.n_kv_heads;
    const int L = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    int rows = a.n_rows[u], first = a.first ? a.first[u] : 0, bad = 0;
    if (rows < 0 || rows > a.capacity) { bad |= CSP_DEV_BAD_LEN; rows = rows < 0 ? 0 : a.capacity; }
    if (first < 0) { bad |= CSP_DEV_BAD_LEN; first = 0; }
    int count = first < rows ? rows - first : 0;
    if (count > a.max_rows) { bad |= CSP_DEV_CAPACITY; count = a.max_rows; }
    if (bad && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(a.status, bad);
    const int32_t* const table = a.page_table + int64_t(b) * a.max_pages;
#pragma unroll 1
    for (int which = 0; which < (a.v.ptr ? 2 : 1); ++which) {
        const RowTensor& from = which ? a.v : a.k;
        const RowTensor& sc = which ? a.v_scales : a.k_scales;
        const RowTensor& to = which ? a.v_out : a.k_out;
        const char* const codes = static_cast<const char*>(from.ptr) + h * from.sh;
        const char* const scales = static_cast<const char*>(sc.ptr) + h * sc.sh;
        char* const out = static_cast<char*>(to.ptr) + b * to.sb + h * to.sh;
        for (int i0 = blockIdx.y * kGroups * kLoadDepth; i0 < count; i0 += int(gridDim.y) * kGroups * kLoadDepth) {
            uint2 w[kLoadDepth];
            uint32_t pair[kLoadDepth];
#pragma unroll
            for (int j = 0; j < kLoadDepth; ++j) {
                const int i = i0 + j * kGroups + group;
                w[j] = make_uint2(0u, 0u);
                pair[j] = 0u;
                if (i >= count) continue;
                uint32_t slot;
                const int page = table[divide(uint32_t(first + i), uint32_t(a.page_rows), a.page_inverse, slot)];
                if (page < 0 || page >= a.n_pages) {     // reads as zeros
                    if (which == 0 && L == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
                    continue;
                }
                const uint32_t* const row = reinterpret_cast<const uint32_t*>(codes + page * from.sb + slot * from.st);
                w[j] = make_uint2(__ldcs(row + L), __ldcs(row + L + kLanes));
                pair[j] = *reinterpret_cast<const uint32_t*>(scales + page * sc.sb + int64_t(slot) * 4);
            }
#pragma unroll
            for (int j = 0; j < kLoadDepth; ++j) {
                const int i = i0 + j * kGroups + group;
                if (i >= count) continue;
                const float scale = bf16_lo(pair[j]), base = bf16_hi(pair[j]);
                // A code in bits 4 k to 4 k + 3 of a float that is 2^23 otherwise is the number code 2^4k more: it stays where it is,
                // and the scale is divided instead (exactly: of its eight bits none is lost, as 2^-126 2^-12 is still 2^11 times the
                // smallest number).
                float f[16];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float part = scale * (k == 0 ? 1.f : k == 1 ? 0x1p-4f : k == 2 ? 0x1p-8f : 0x1p-12f);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t x = e ? w[j].y : w[j].x, m = 15u << (4 * k);
                        const float2 c = __fadd2_rn(make_float2(__uint_as_float((x & m) | 0x4b000000u), __uint_as_float(((x >> 16) & m) | 0x4b000000u)),
                                                    make_float2(-8388608.f, -8388608.f));
                        const float2 y = __ffma2_rn(c, make_float2(part, part), make_float2(base, base));
                        f[8 * e + k] = y.x;
                        f[8 * e + k + 4] = y.y;
                    }
                }
                char* const row = out + i * to.st;
                const Eight<kF32> r0 = narrow<kF32>(f), r1 = narrow<kF32>(f + 8);
                store_eight<kF32>(row, L, r0);
                store_eight<kF32>(row, L + kLanes, r1);
            }
        }
    }
}

inline csp_status launched() { return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA; }

template <bool kF32, bool kFour, int kLanes>
csp_status append_rows(const AppendRowsArgs& a, dim3 grid, cudaStream_t s) {
    append_rows_kernel<kF32, kFour, kLanes><<<grid, kThreads, 0, s>>>(a);
    return launched();
}

}  // namespace

csp_status launch_append_rows(AppendRowsArgs a, int head_dim, bool f32, bool four, cudaStream_t s) {
    if (a.batch == 0) return CSP_OK;
    const int groups = kThreads / (head_dim / 16), pairs = a.n_kv_heads + (a.n_q_heads + 1) / 2;
    a.page_inverse = uint32_t((uint64_t(1) << 32) / uint32_t(a.page_rows)) + 1u;
    a.group_inverse = a.group > 1 ? uint32_t((uint64_t(1) << 32) / uint32_t(a.group)) + 1u : 0u;
    if (!a.rope.dim) {                                   // (only calls for 4 bits come without)
        const int rows = groups * kAppendDepth;
        const int64_t tiles = a.max_new > 0 ? (int64_t(a.max_new) + rows - 1) / rows : 1;
        const dim3 grid{unsigned(a.batch * a.n_kv_heads), unsigned(tiles < 65535 ? tiles : 65535)};
        if (head_dim == 64) append_units_kernel<4><<<grid, kThreads, 0, s>>>(a);
        else append_units_kernel<8><<<grid, kThreads, 0, s>>>(a);
        return launched();
    }
    // Few tokens: the lane groups of a block spread over the heads; from four on, four tokens share a block and every group goes over
    // some of the heads with one set of cosines.  (1 K tokens of 4 x 32 / 8 heads, one token to a block 21.3 us, two 19.1, four 17.6, eight
    // 17.8; fp32 with 15 units of 333 tokens 4.2, 2.9, 3.1, 3.3.)
    a.log_tokens = 0;
    while (a.log_tokens < 2 && (2 << a.log_tokens) <= a.max_new && (2 << a.log_tokens) <= groups) ++a.log_tokens;
    const int tiles = a.max_new > 0 ? (a.max_new + (1 << a.log_tokens) - 1) >> a.log_tokens : 1;
    const int most = (1 << 30) / a.batch;
    a.token_tiles = tiles < most ? tiles : most;
    const int step = groups >> a.log_tokens;             // heads at a time
    const int64_t blocks = int64_t(a.token_tiles) * a.batch;
    // as many pieces of the heads as it takes to give every SM eight blocks (four: 1 K rotated tokens 19 us instead of 17.7)
    int pieces = (pairs + step - 1) / step;
    const int64_t want = (8 * int64_t(sm_count()) + blocks - 1) / blocks;
    if (pieces > want) pieces = int(want);
    a.pairs_per_block = ((pairs + step - 1) / step + pieces - 1) / pieces * step;
    pieces = (pairs + a.pairs_per_block - 1) / a.pairs_per_block;
    const dim3 grid{unsigned(blocks), unsigned(pieces)};
    if (four) return head_dim == 64 ? append_rows<false, true, 4>(a, grid, s) : append_rows<false, true, 8>(a, grid, s);
    if (f32) return head_dim == 32 ? append_rows<true, false, 2>(a, grid, s) : head_dim == 64 ? append_rows<true, false, 4>(a, grid, s) : append_rows<true, false, 8>(a, grid, s);
    return head_dim == 64 ? append_rows<false, false, 4>(a, grid, s) : head_dim == 128 ? append_rows<false, false, 8>(a, grid, s) : append_rows<false, false, 16>(a, grid, s);
}

csp_status launch_load_rows(LoadRowsArgs a, int head_dim, bool f32, cudaStream_t s) {
    if (a.units == 0 || a.max_rows == 0) return CSP_OK;
    a.page_inverse = uint32_t((uint64_t(1) << 32) / uint32_t(a.page_rows)) + 1u;
    // Four rows in flight per lane, but one where that leaves SMs without a block (5 K rows as fp32: 2.5 us instead of 4.4; 650 K
    // rows of K and of V with two 72.5 us instead of 71).
    const int groups = kThreads / (head_dim / 16), rows = a.max_rows < a.capacity ? a.max_rows : a.capacity;
    const int depth = int64_t(a.units) * rows < 4 * int64_t(groups) * sm_count() ? 1 : 4;
    const int64_t tiles = (int64_t(rows) + groups * depth - 1) / (groups * depth);
    if (tiles == 0) return CSP_OK;
    const dim3 grid{unsigned(a.units), unsigned(tiles < 65535 ? tiles : 65535)};
    const auto kernel = head_dim == 64 ? f32 ? depth == 1 ? load_rows_kernel<true, 4, 1> : load_rows_kernel<true, 4, 4>
                                             : depth == 1 ? load_rows_kernel<false, 4, 1> : load_rows_kernel<false, 4, 4>
                                       : f32 ? depth == 1 ? load_rows_kernel<true, 8, 1> : load_rows_kernel<true, 8, 4>
                                             : depth == 1 ? load_rows_kernel<false, 8, 1> : load_rows_kernel<false, 8, 4>;
    kernel<<<grid, kThreads, 0, s>>>(a);
    return launched();
}

}  // namespace csp
