// Attention of tree nodes over a paged cache (include/spechub_cache.h).
#pragma once

#include "spechub_pages.cuh"

namespace spechub {

constexpr int kAttRowThreads = 128;

// One warp per (sequence, node, query head), key by key: s = scale q.k, running maximum m and sum l,
// o = o 2^(m - m') + 2^(s - m') v.
template <class T, int D>
__global__ void __launch_bounds__(kAttRowThreads) attention_rows_kernel(const __grid_constant__ AttentionArgs A) {
    constexpr int E = D / 32;   // elements of a row per lane
    pdl_begin();
    const CacheArgs &c = A.c;
    const int lane = threadIdx.x & 31;
    const int64_t at = blockIdx.x * int64_t(kAttRowThreads / 32) + (threadIdx.x >> 5);
    if (at >= int64_t(c.batch) * c.nodes * c.heads) return;
    const int h = at % c.heads, n = at / c.heads % c.nodes, b = at / c.heads / c.nodes, hk = h / (c.heads / c.kv_heads);
    const int64_t len = c.lens[b];
    if (len < 0) return;
    const int32_t *row = c.table + b * c.stride_table;
    auto load = [&](const void *p, int64_t off, float (&x)[E]) {
        const T *src = static_cast<const T *>(p) + off + lane * E;
#pragma unroll
        for (int i = 0; i < E; i += 2) {
            const float2 f = unpack2<T>(*reinterpret_cast<const uint32_t *>(src + i));
            x[i] = f.x; x[i + 1] = f.y;
        }
    };
    float q[E], o[E] = {}, m = neg_inf(), l = 0.f;
    load(A.q.data, b * A.q.seq + n * A.q.node + h * A.q.head, q);
    auto key = [&](int page, int64_t slot) {
        const int64_t in = slot & ((1 << c.page_shift) - 1);
        float k[E] = {}, v[E] = {}, s = 0.f;
        if (page >= 0) {
            load(c.k.data, page * c.k.page + in * c.k.token + hk * c.k.head, k);
            load(c.v.data, page * c.v.page + in * c.v.token + hk * c.v.head, v);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) s = fmaf(q[i], k[i], s);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(kFull, s, x);
        s *= A.scale_log2;
        const float m2 = fmaxf(m, s), ref = m2 == neg_inf() ? 0.f : m2, f = ex2(m - ref), p = ex2(s - ref);
        l = l * f + p;
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] = o[i] * f + p * v[i];
        m = m2;
    };
    for (int64_t j = 0; j < A.shared_len; ++j) {
        const int page = A.shared_table[j >> c.page_shift];
        key(page >= 0 && page < c.pages ? page : -1, j);
    }
    const int64_t slots = static_cast<int64_t>(c.table_width) << c.page_shift;
    for (int64_t j = 0; j < min(len, slots); ++j) key(page_of(c, row, j), j);
    const int32_t *mask = A.mask + b * A.mask_stride_seq + n * static_cast<int64_t>((c.nodes + 31) / 32);
    for (int i = 0; i < c.nodes && len + i < slots; ++i)
        if (mask[i >> 5] >> (i & 31) & 1) key(page_of(c, row, len + i), len + i);
    T *dst = static_cast<T *>(A.out.data) + b * A.out.seq + n * A.out.node + h * A.out.head + lane * E;
    const bool none = m == neg_inf() && l == 0.f;
    const float f = none ? 0.f : 1.f / l;
#pragma unroll
    for (int i = 0; i < E; i += 2) *reinterpret_cast<uint32_t *>(dst + i) = pack2<T>(o[i] * f, o[i + 1] * f);
    if (A.lse && lane == 0) A.lse[at] = none ? neg_inf() : (m + log2f(l)) * 0.6931471805599453f;
}

constexpr int kAttStatusThreads = 256;

// Which sequences' pages are bad.  One CTA per sequence.
__global__ void __launch_bounds__(kAttStatusThreads) attention_status_kernel(const __grid_constant__ AttentionArgs A) {
    pdl_begin();
    const CacheArgs &c = A.c;
    const int b = blockIdx.x, tid = threadIdx.x, ps = 1 << c.page_shift;
    const int64_t len = c.lens[b];
    bool bad = false;
    if (len >= 0) {
        const int64_t need = (len + c.nodes + ps - 1) >> c.page_shift;
        bad = need > c.table_width;
        const int32_t *row = c.table + b * c.stride_table;
        for (int64_t i = tid; i < min(need, static_cast<int64_t>(c.table_width)); i += kAttStatusThreads) bad |= row[i] < 0 || row[i] >= c.pages;
        for (int i = tid; i < (A.shared_len + ps - 1) >> c.page_shift; i += kAttStatusThreads)
            bad |= A.shared_table[i] < 0 || A.shared_table[i] >= c.pages;
    }
    bad = __syncthreads_or(bad);
    if (tid == 0) c.status[b] = bad ? SPECHUB_ST_PAGE : 0u;
}

}  // namespace spechub
