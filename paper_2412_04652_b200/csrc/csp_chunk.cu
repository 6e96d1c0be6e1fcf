// Attention of a chunk of new tokens over a dense or paged cache (Eq. 5-7), with score modifiers.
// One block per (sequence, query head, token): the plainest form that is right for every case.
#include "csp_device.cuh"
#include "csp_internal.cuh"

namespace csp {
namespace {
using namespace dev;

struct SimpleTensors {
    const uint16_t* q; int64_t q_sb, q_sh, q_st;
    const uint16_t* k; int64_t k_sb, k_sh, k_st;
    const uint16_t* v; int64_t v_sb, v_sh, v_st;
};

constexpr int kSimpleThreads = 128;

__device__ __forceinline__ float bf(uint16_t x) { return __uint_as_float(uint32_t(x) << 16); }

template <int D>
__global__ void __launch_bounds__(kSimpleThreads) chunk_simple_kernel(const ChunkArgs a, const SimpleTensors x) {
    __shared__ float qs[D], wgt[kSimpleThreads], red[kSimpleThreads / 32];
    __shared__ int64_t vrow[kSimpleThreads];
    const int tid = threadIdx.x, i = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, h = hq / a.group;
    const int n_q = a.n_kv_heads * a.group;
    int rows = a.n_rows[int64_t(b) * a.n_kv_heads + h], n_new = a.n_new ? a.n_new[b] : a.max_new;
    if (rows < 0 || rows > a.capacity || n_new < 0 || n_new > a.max_new) {
        if (tid == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
        rows = rows < 0 ? 0 : min(rows, a.capacity);
        n_new = n_new < 0 ? 0 : min(n_new, a.max_new);
    }
    if (i >= n_new) return;
    const int r = rows - n_new + i;
    if (r < 0 && tid == 0) atomicOr(a.status, CSP_DEV_BAD_LEN);
    if (tid < D) qs[tid] = bf(x.q[b * x.q_sb + hq * x.q_sh + i * x.q_st + tid]) * a.scale;
    const ModArgs& m = a.mods;
    int prefix = m.prefix ? m.prefix[b * m.prefix_sb + h * m.prefix_sh] : 0;
    const int last = r < 0 ? -1 : min(max(r, prefix - 1), rows - 1);
    const float slope = m.slopes ? m.slopes[hq] : 0.f;
    auto pos = [&](int t) { return m.positions ? m.positions[b * m.pos_sb + h * m.pos_sh + t] : t; };
    const int qpos = m.slopes && r >= 0 ? pos(r) : 0;
    const int32_t* const docs = m.documents ? m.documents + b * m.doc_sb + h * m.doc_sh : nullptr;
    const int qdoc = docs && r >= 0 ? docs[r] : 0;
    __syncthreads();
    float mx = -INFINITY, l = 0.f, acc = 0.f;
    for (int t0 = 0; t0 <= last; t0 += kSimpleThreads) {
        const int t = t0 + tid;
        float o = -INFINITY;
        if (t <= last && (!docs || docs[t] == qdoc)) {
            int64_t outer = b, row = t;
            bool ok = true;
            if (a.page_table) {
                outer = a.page_table[int64_t(b) * a.max_pages + t / a.page_rows];
                ok = outer >= 0 && outer < a.n_pages;
                if (!ok) atomicOr(a.status, CSP_DEV_BAD_LEN);
                row = t % a.page_rows;
            }
            o = 0.f;
            vrow[tid] = ok ? outer * x.v_sb + h * x.v_sh + row * x.v_st : -1;
            if (ok) {
                const uint16_t* kr = x.k + outer * x.k_sb + h * x.k_sh + row * x.k_st;
                for (int c = 0; c < D; c += 8) {
                    const uint4 w = *reinterpret_cast<const uint4*>(kr + c);
                    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
                    for (int j = 0; j < 4; ++j)
                        o += qs[c + 2 * j] * __uint_as_float(ww[j] << 16) + qs[c + 2 * j + 1] * __uint_as_float(ww[j] & 0xffff0000u);
                }
            }
            if (m.softcap > 0.f) o = m.softcap * tanhf(o / m.softcap);
            if (m.slopes) o -= slope * fabsf(float(qpos - pos(t)));
        }
        float tile = o;
        for (int d = 16; d; d >>= 1) tile = fmaxf(tile, __shfl_xor_sync(0xffffffffu, tile, d));
        if (tid % 32 == 0) red[tid / 32] = tile;
        __syncthreads();
        for (int w = 0; w < kSimpleThreads / 32; ++w) tile = fmaxf(tile, red[w]);
        const float mn = fmaxf(mx, tile);
        const float e = o == -INFINITY ? 0.f : expf(o - mn);
        wgt[tid] = e;
        __syncthreads();
        const float keep = mx == -INFINITY ? 0.f : expf(mx - mn);
        l *= keep;
        acc *= keep;
        for (int j = 0; j < kSimpleThreads; ++j) {
            const float w = wgt[j];
            if (w == 0.f) continue;
            l += w;
            if (tid < D && vrow[j] >= 0) acc += w * bf(x.v[vrow[j] + tid]);
        }
        mx = mn;
        __syncthreads();
    }
    if (tid < D) {
        const float denom = a.n * expf(-mx) + l;
        const float o = l > 0.f ? acc / denom : 0.f;
        uint32_t u = __float_as_uint(o);
        u += 0x7fffu + ((u >> 16) & 1u);
        a.out[b * a.o_sb + hq * a.o_sh + i * a.o_st + tid] = uint16_t(u >> 16);
    }
    if (a.lse && tid == 0) a.lse[(int64_t(b) * n_q + hq) * a.max_new + i] = l > 0.f ? mx + logf(l) : -INFINITY;
}

}  // namespace

size_t chunk_workspace_bytes(const csp_params&, int) { return kStatusBytes; }

csp_status launch_chunk_attn(const csp_params& p, const ChunkArgs& a, const csp_tensor& q, const csp_tensor& k,
                             const csp_tensor& v, const csp_pages*, void*, cudaStream_t s) {
    const SimpleTensors x = {static_cast<const uint16_t*>(q.ptr), q.stride_b, q.stride_h, q.stride_t,
                             static_cast<const uint16_t*>(k.ptr), k.stride_b, k.stride_h, k.stride_t,
                             static_cast<const uint16_t*>(v.ptr), v.stride_b, v.stride_h, v.stride_t};
    const dim3 grid(a.max_new, p.n_q_heads, p.batch);
    if (p.head_dim == 64) chunk_simple_kernel<64><<<grid, kSimpleThreads, 0, s>>>(a, x);
    else chunk_simple_kernel<128><<<grid, kSimpleThreads, 0, s>>>(a, x);
    return cudaGetLastError() == cudaSuccess ? CSP_OK : CSP_ERR_CUDA;
}

}  // namespace csp
