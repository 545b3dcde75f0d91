// Attention of tree nodes over a paged cache (include/spechub_cache.h), on the tensor cores.
//
// Mathematics.  A block of up to 256 rows (row = (sequence, node, query head of one cache head)) goes over its keys in tiles of
// 128.  S = Q K^T; per row p = 2^(c s - r), l += sum p, O += P V, with c = scale log2(e) and r the row's reference, at first the
// maximum of the first tile.  r follows the maximum only when that has outgrown it by kSlack (2^kSlack is far from the end of
// every type here), and then O and l are scaled by 2^(r_old - r): the division by l at the end makes the result the same.  Pieces of
// one row are joined by their references: out = sum_j 2^(r_j - R) O_j / sum_j 2^(r_j - R) l_j.
//
// Work.  Rows that share keys are one block: the query heads of a cache head and all nodes of a sequence for its own context (7
// nodes of 4 heads are 28 rows), and the whole batch for the shared prefix, which is thus read once per 256 rows, from L2 but for the
// first time.  (block, tile) pairs are the units; every CTA (one per SM) takes one run of consecutive units, found on the device from
// the lengths alone.  So a few long sequences are split as finely as many short ones are gathered.  A run that covers a block's tiles
// is finished in place; other pieces go to the workspace and attention_join_kernel adds them in the order of the CTAs.
//
// CTA.  Warp 8 brings K and V tiles through a ring of bulk tensor copies (a box per page and 64 dimensions), warp 9 issues the
// matrix instructions, warps 0-3 and 4-7 are two softmax groups, a row per thread, each with its own S, P and O in tensor memory.
// More than 128 rows: each group has 128 of them and every K / V tile serves both.  Up to 128 rows: the groups take the tiles in turn,
// for the same rows, and are joined at the end of the piece; else the tensor core and the loads would wait while one group computes.
// P takes the place of S (head_dim 64 has room for its own).
//
// What lies behind a sequence's end in a page may be anything.  Its scores are replaced, and its values, and values of tree nodes
// that are no finite numbers, are cleared in shared memory before the product, since 0 * NaN would reach every row; the rows that do see
// such a node get it added at the end.
#pragma once

#include "spechub_pages.cuh"
#include "spechub_tmem.cuh"
#include "spechub_umma.cuh"

namespace spechub {

constexpr int kTile = 128;         // keys of a tile, rows of a softmax group
constexpr int kBlockRows = 256;
constexpr int kAttThreads = 384;
constexpr float kSlack = 8.f;
// Costs of a unit in the split of the work, shared : own.
constexpr int kCostShared = 1, kCostOwn = 1;

// Weights are stored as 2^bias times themselves.  fp16 has numbers down to 2^-24 only: with the reference 7 below, weights of
// 2^-31 of the largest still count, and the largest is 2^(7 + kSlack) < 65504.
template <class T> struct Weight;
template <> struct Weight<__nv_bfloat16> { static constexpr bool kBf16 = true; static constexpr float kBias = 0.f; };
template <> struct Weight<__half> { static constexpr bool kBf16 = false; static constexpr float kBias = 7.f; };

template <int D>
struct AttShape {
    static constexpr int kHalves = D / 64;
    static constexpr int kHalfBytes = kTile * 128;                   // 128 rows of 64 elements
    static constexpr int kTileBytes = kHalves * kHalfBytes;          // a tile of keys, of values, or of queries
    static constexpr int kStages = 160 * 1024 / kTileBytes;
    static constexpr int kSmem = (2 + kStages) * kTileBytes + 1024;  // (1024: alignment)
    // columns of tensor memory
    static constexpr int kS = 0, kO = 256, kP = D == 64 ? 384 : 0, kPStep = D == 64 ? 64 : 128;
};

// What the host knows of the work.
struct AttPlan {
    int shared_tiles, shared_blocks, own_blocks, grid;   // tiles of the prefix; row blocks per cache head: of all rows, of a sequence
    int shared_rows, own_rows;                           // rows of a slot in the workspace
    int64_t shared_items, shared_units, slots;           // slots of the shared pieces
    int64_t *before;                                     // [batch + 1] own units before sequence b
    int *error;                                          // [grid]
    float2 *ml;                                          // (reference, sum) of every row of every slot
    float *o;                                            // [..][head_dim], not divided by the sum
};

struct AttKernelArgs {
    AttentionArgs a;
    AttPlan p;
};

__device__ __forceinline__ int64_t own_end(const CacheArgs &c, int len) {   // keys of a sequence that is there
    const int64_t slots = static_cast<int64_t>(c.table_width) << c.page_shift;
    return min(static_cast<int64_t>(len) + c.nodes, slots);
}
__device__ __forceinline__ int own_tiles(const CacheArgs &c, int len) {
    return len < 0 ? 0 : static_cast<int>((own_end(c, len) + kTile - 1) / kTile);
}
// Units are numbered: all of the shared prefix, then sequence by sequence.  CTA i takes those whose cost before them is in
// [i, i + 1) / grid of the whole.
struct AttSplit {
    int64_t shared_units, units, cost;
    int grid;
    __device__ AttSplit(const AttPlan &p, int64_t own_units)
        : shared_units(p.shared_units), units(p.shared_units + own_units), cost(p.shared_units * kCostShared + own_units * kCostOwn), grid(p.grid) {}
    __device__ int64_t first(int cta) const {
        const int64_t y = (cta * cost + grid - 1) / grid, s = shared_units * kCostShared;
        return y <= s ? (y + kCostShared - 1) / kCostShared : shared_units + (y - s + kCostOwn - 1) / kCostOwn;
    }
    __device__ int cta(int64_t unit) const {
        const int64_t before = unit <= shared_units ? unit * kCostShared : shared_units * kCostShared + (unit - shared_units) * kCostOwn;
        return static_cast<int>(before * grid / cost);
    }
};

// Consecutive tiles of one block of rows.
struct AttPiece {
    bool shared, two;      // two: more than 128 rows
    int b, head, block, rows, t0, t1, tiles;
    int64_t item;          // among the shared or among the own blocks
    int plain, keys;       // keys that every row sees; all keys
    __device__ bool masked(int t) const { return (t + 1) * int64_t(kTile) > plain; }
};

// The pieces of a CTA's run; every role walks through them by itself.
struct AttWalk {
    const CacheArgs &c;
    const AttPlan &p;
    int shared_len;
    int64_t left, item;
    bool shared;
    int b, in_b, tile, len, tiles;

    __device__ AttWalk(const AttKernelArgs &K, int64_t units, bool in_shared, int64_t shared_item, int b0, int in_b0, int tile0)
        : c(K.a.c), p(K.p), shared_len(K.a.shared_len), left(units), item(shared_item), shared(in_shared), b(b0), in_b(in_b0), tile(tile0), len(0), tiles(0) {
        if (!shared && left > 0) look();
    }
    __device__ void look() {
        len = b < c.batch ? c.lens[b] : -1;
        tiles = own_tiles(c, len);
    }
    __device__ bool next(AttPiece &x) {
        if (left <= 0) return false;
        x.shared = shared;
        x.t0 = tile;
        if (shared) {
            x.b = 0;
            x.head = static_cast<int>(item / p.shared_blocks);
            x.block = static_cast<int>(item % p.shared_blocks);
            x.item = item;
            x.tiles = p.shared_tiles;
            x.plain = x.keys = shared_len;
            x.rows = min(kBlockRows, c.batch * c.nodes * (c.heads / c.kv_heads) - x.block * kBlockRows);
        } else {
            const int per_b = c.kv_heads * p.own_blocks;
            while (b < c.batch && (in_b == per_b || tiles == 0)) { ++b; in_b = 0; look(); }
            if (b >= c.batch) return false;
            x.b = b;
            x.head = in_b / p.own_blocks;
            x.block = in_b % p.own_blocks;
            x.item = static_cast<int64_t>(b) * per_b + in_b;
            x.tiles = tiles;
            x.keys = static_cast<int>(own_end(c, len));
            x.plain = min(len, x.keys);
            x.rows = min(kBlockRows, c.nodes * (c.heads / c.kv_heads) - x.block * kBlockRows);
        }
        x.two = x.rows > kTile;
        x.t1 = static_cast<int>(min(static_cast<int64_t>(x.tiles), tile + left));
        left -= x.t1 - x.t0;
        tile = x.t1;
        if (tile == x.tiles) {
            tile = 0;
            if (shared) {
                if (++item == p.shared_items) { shared = false; b = 0; in_b = 0; if (left > 0) look(); }
            } else ++in_b;
        }
        return true;
    }
};

// Where row `i` of a block is.
struct AttRow { int b, n, h; };
__device__ __forceinline__ AttRow row_of(const CacheArgs &c, const AttPiece &x, int i) {
    const unsigned g = c.heads / c.kv_heads, r = x.block * kBlockRows + i, node = r / g;
    AttRow o;
    o.h = x.head * g + (r - node * g);
    if (x.shared) { o.b = node / c.nodes; o.n = node - o.b * c.nodes; }
    else { o.b = x.b; o.n = node; }
    return o;
}

// Bits of the keys of a masked tile that a row sees (bit j of word w: key 128 t + 32 w + j).
__device__ __forceinline__ void row_bits(const AttentionArgs &A, const AttPiece &x, int t, int n, uint32_t (&bits)[4]) {
    const int words = (A.c.nodes + 31) / 32;
    const int32_t *mask = A.mask + x.b * A.mask_stride_seq + n * static_cast<int64_t>(words);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int64_t at = t * int64_t(kTile) + 32 * w;
        uint32_t m;
        if (at + 32 <= x.plain) m = ~0u;
        else if (x.shared) m = 0u;
        else {
            const int64_t i = at - x.plain;   // node of the first key; > -32
            const int lo = static_cast<int>(i >> 5), sh = static_cast<int>(i & 31);
            const uint32_t a = lo < 0 ? ~0u : lo < words ? mask[lo] : 0u, z = lo + 1 < words ? mask[lo + 1] : 0u;
            m = __funnelshift_r(a, z, sh);
        }
        if (x.shared && at < x.plain && at + 32 > x.plain) m = (1u << (x.plain - at)) - 1;
        if (at + 32 > x.keys) m &= at >= x.keys ? 0u : (1u << (x.keys - at)) - 1;   // (the masks' bits behind the last node may be anything)
        bits[w] = m;
    }
}

template <class T> __device__ __forceinline__ bool not_finite(uint16_t e);
template <> __device__ __forceinline__ bool not_finite<__nv_bfloat16>(uint16_t e) { return (e & 0x7f80) == 0x7f80; }
template <> __device__ __forceinline__ bool not_finite<__half>(uint16_t e) { return (e & 0x7c00) == 0x7c00; }

// 32 columns of a row's output at most: the tree nodes that the row sees and whose value there is no finite number.
template <class T>
__device__ __noinline__ void add_not_finite(const AttentionArgs &A, const AttPiece &x, int n, int col0, float *o) {
    const CacheArgs &c = A.c;
    const int32_t *mask = A.mask + x.b * A.mask_stride_seq + n * static_cast<int64_t>((c.nodes + 31) / 32);
    const int32_t *row = c.table + x.b * c.stride_table;
    for (int m = max(0, x.t0 * kTile - x.plain); m < x.keys - x.plain && x.plain + m < x.t1 * int64_t(kTile); ++m) {
        if (!(mask[m >> 5] >> (m & 31) & 1)) continue;
        const int slot = x.plain + m, page = page_of(c, row, slot);
        if (page < 0) continue;
        const uint16_t *v = static_cast<const uint16_t *>(c.v.data) + page * c.v.page + (slot & ((1 << c.page_shift) - 1)) * c.v.token + x.head * c.v.head + col0;
        for (int i = 0; i < 32; ++i)
            if (not_finite<T>(v[i])) o[i] += unpack2<T>(v[i]).x;
    }
}

template <class T, int D>
__global__ void __launch_bounds__(kAttThreads, 1) attention_kernel(const __grid_constant__ AttKernelArgs K, const __grid_constant__ CUtensorMap map_k,
                                                                   const __grid_constant__ CUtensorMap map_v) {
    using L = AttShape<D>;
    constexpr bool kBf16 = Weight<T>::kBf16;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * L::kStages + 7];
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up_, bad_values;
    __shared__ float2 other[kTile];           // (reference, sum) of the second group's rows
    __shared__ int64_t warp_sum[kAttThreads / 32];
    __shared__ struct { int64_t units, item; int shared, b, in_b, tile; } start;
    volatile int *const gave_up = &gave_up_;

    const AttentionArgs &A = K.a;
    const CacheArgs &c = A.c;
    const AttPlan &P = K.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t *const smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t s_q = saddr(smem), s_kv = s_q + 2 * L::kTileBytes, bar0 = saddr(bars);
    const auto kv_full = [&](int s) { return bar0 + 8u * s; };
    const auto kv_empty = [&](int s) { return bar0 + 8u * (L::kStages + s); };
    const uint32_t q_full = bar0 + 16u * L::kStages;
    const auto s_full = [&](int t) { return q_full + 8u + 8u * t; };
    const auto p_full = [&](int t) { return q_full + 24u + 8u * t; };
    const auto o_full = [&](int t) { return q_full + 40u + 8u * t; };

    if (warp == 9) tmem_alloc(saddr(&tmem_base), 512);
    if (tid == 0) {
        for (int s = 0; s < L::kStages; ++s) { bar_init(kv_full(s), 1); bar_init(kv_empty(s), 1); }
        bar_init(q_full, 256);
        for (int t = 0; t < 2; ++t) { bar_init(s_full(t), 1); bar_init(p_full(t), kTile); bar_init(o_full(t), 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        gave_up_ = 0;
        bad_values = 0;
        tma_prefetch_map(&map_k);
        tma_prefetch_map(&map_v);
    }
    pdl_begin();

    // This CTA's run of units: own units of all sequences summed up, in the order of the sequences.
    {
        const int per = (c.batch + kAttThreads - 1) / kAttThreads, b0 = min(c.batch, tid * per), b1 = min(c.batch, b0 + per);
        const int64_t per_b = static_cast<int64_t>(c.kv_heads) * P.own_blocks;
        int64_t mine = 0;
        for (int b = b0; b < b1; ++b) mine += own_tiles(c, c.lens[b]) * per_b;
        int64_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t v = __shfl_up_sync(kFull, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) warp_sum[warp] = upto;
        __syncthreads();
        int64_t all = 0;
        for (int w = 0; w < kAttThreads / 32; ++w) {
            if (w < warp) upto += warp_sum[w];
            all += warp_sum[w];
        }
        const AttSplit split(P, all);
        const int64_t u0 = split.first(blockIdx.x), u1 = min(split.units, split.first(blockIdx.x + 1));
        int64_t before = upto - mine;
        if (tid == 0) {
            start.units = max(int64_t(0), u1 - u0);
            start.shared = u0 < P.shared_units;
            start.item = start.shared ? u0 / P.shared_tiles : 0;
            start.tile = start.shared ? static_cast<int>(u0 % P.shared_tiles) : 0;
            start.b = 0; start.in_b = 0;
        }
        __syncthreads();
        const int64_t uo = u0 - P.shared_units;
        const bool here = uo >= before && uo < upto;
        if (here || (blockIdx.x == 0 && b0 < b1)) {
            for (int b = b0; b < b1; ++b) {
                const int64_t n = own_tiles(c, c.lens[b]) * per_b;
                if (here && uo >= before && uo < before + n) {
                    const int64_t in = uo - before, tiles = n / per_b;
                    start.b = b; start.in_b = static_cast<int>(in / tiles); start.tile = static_cast<int>(in % tiles);
                }
                if (blockIdx.x == 0) P.before[b] = before;
                before += n;
            }
            if (blockIdx.x == 0 && b1 == c.batch) P.before[c.batch] = before;
        }
        tmem_fence_before();
        __syncthreads();
        tmem_fence_after();
    }
    const uint32_t tm = tmem_base;
    AttWalk walk(K, start.units, start.shared, start.item, start.b, start.in_b, start.tile);
    AttPiece x = {};

    if (warp == 8) {
        // ---- K and V tiles -------------------------------------------------------------------------
        int stage = 0;
        uint32_t phase = 0;
        const int ps = 1 << c.page_shift, box = min(ps, kTile), boxes = kTile / box;
        const auto page_at = [&](int t) -> int {   // lane i: the page of the tile's i-th box (c.pages: reads as zeros)
            const int64_t slot = t * int64_t(kTile) + lane * box;
            if (lane >= boxes || t >= x.t1 || slot >= x.keys) return c.pages;
            int page;
            if (x.shared) page = A.shared_table[slot >> c.page_shift];
            else {
                const int64_t at = slot >> c.page_shift;
                if (at >= c.table_width) return c.pages;
                page = c.table[x.b * c.stride_table + at];
            }
            return page >= 0 && page < c.pages ? page : c.pages;
        };
        const auto bring = [&](const CUtensorMap *map, int t, int page) {
            bar_wait(kv_empty(stage), phase ^ 1u, gave_up);
            if (lane == 0) bar_expect(kv_full(stage), L::kTileBytes);
            __syncwarp();
            if (lane < boxes) {
                const uint32_t dst = s_kv + stage * L::kTileBytes + lane * box * 128;
                const int y = ps > kTile ? static_cast<int>((t * int64_t(kTile)) & (ps - 1)) : 0;
#pragma unroll
                for (int h = 0; h < L::kHalves; ++h) tma_load(dst + h * L::kHalfBytes, map, 64 * h, y, x.head, page, kv_full(stage));
            }
            if (++stage == L::kStages) { stage = 0; phase ^= 1u; }
        };
        while (walk.next(x)) {
            const int ahead = x.two ? 1 : 2;   // keys are this many tiles ahead of the values
            int p0 = page_at(x.t0), p1 = page_at(x.t0 + 1), p2 = page_at(x.t0 + 2);
            bring(&map_k, x.t0, p0);
            if (ahead == 2 && x.t0 + 1 < x.t1) bring(&map_k, x.t0 + 1, p1);
            for (int t = x.t0; t < x.t1; ++t) {
                const int p3 = page_at(t + 3);
                bring(&map_v, t, p0);
                if (t + ahead < x.t1) bring(&map_k, t + ahead, ahead == 1 ? p1 : p2);
                p0 = p1; p1 = p2; p2 = p3;
            }
        }
        // the ring's last arrivals come before the CTA ends
        for (int s = 0; s < L::kStages; ++s) {
            bar_wait(kv_empty(stage), phase ^ 1u, gave_up);
            if (++stage == L::kStages) { stage = 0; phase ^= 1u; }
        }
    } else if (warp == 9) {
        // ---- matrix instructions -------------------------------------------------------------------
        int stage = 0;
        uint32_t phase = 0, q_phase = 0, p_phase[2] = {0, 0};
        constexpr uint32_t desc_s = mma_desc(kBf16, kTile, false), desc_o = mma_desc(kBf16, D, true);
        const auto arrived = [&]() {   // the next stage of the ring
            bar_wait(kv_full(stage), phase, gave_up);
            const int s = stage;
            if (++stage == L::kStages) { stage = 0; phase ^= 1u; }
            return s;
        };
        const auto scores = [&](int t, int q, int s) {   // S_t = Q_q K^T
            if (lane != 0) return;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint32_t off = (k / 4) * L::kHalfBytes + (k % 4) * 32;
                mma_ss(tm + L::kS + t * kTile, smem_desc(s_q + q * L::kTileBytes + off, 16, 1024), smem_desc(s_kv + s * L::kTileBytes + off, 16, 1024),
                       desc_s, k > 0);
            }
            mma_commit(s_full(t));
        };
        const auto products = [&](int t, int s, bool add) {   // O_t (+)= P_t V
            bar_wait(p_full(t), p_phase[t], gave_up);
            p_phase[t] ^= 1u;
            tmem_fence_after();
            if (lane != 0) return;
#pragma unroll
            for (int k = 0; k < kTile / 16; ++k)
                mma_ts(tm + L::kO + t * D, tm + L::kP + t * L::kPStep + 8 * k, smem_desc(s_kv + s * L::kTileBytes + k * 2048, L::kHalfBytes, 1024), desc_o,
                       add || k > 0);
        };
        // values behind the end, and those of tree nodes that are no numbers: zero
        const auto clear = [&](int tile, int s) {
            constexpr int kVecs = D / 8;
            const int r0 = max(0, x.plain - tile * kTile), r1 = min(kTile, x.keys - tile * kTile);
            uint8_t *const v = smem + 2 * L::kTileBytes + s * L::kTileBytes;
            bool bad = false;
            for (int i = lane + r0 * kVecs; i < kTile * kVecs; i += 32) {
                const int r = i / kVecs, h = i % kVecs / 8, vec = i % 8;
                uint4 *at = reinterpret_cast<uint4 *>(v + h * L::kHalfBytes + r * 128 + vec * 16);
                if (r >= r1) { *at = make_uint4(0, 0, 0, 0); continue; }
                uint4 u = *at;
                uint32_t *w = &u.x;
                bool any = false;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (not_finite<T>(w[j] & 0xffff)) { w[j] &= 0xffff0000u; any = true; }
                    if (not_finite<T>(w[j] >> 16)) { w[j] &= 0xffffu; any = true; }
                }
                if (any) *at = u;
                bad |= any;
            }
            if (__any_sync(kFull, bad) && lane == 0) *static_cast<volatile int *>(&bad_values) = 1;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __threadfence_block();
            __syncwarp();
        };
        while (walk.next(x)) {
            bar_wait(q_full, q_phase, gave_up);
            q_phase ^= 1u;
            tmem_fence_after();
            if (lane == 0) *static_cast<volatile int *>(&bad_values) = 0;
            __syncwarp();
            const int ahead = x.two ? 1 : 2;
            for (int i = 0; i < ahead && x.t0 + i < x.t1; ++i) {
                const int s = arrived();
                scores(i, 0, s);
                if (x.two) scores(1, 1, s);
                if (lane == 0) mma_commit(kv_empty(s));
            }
            for (int t = x.t0; t < x.t1; ++t) {
                const int v = arrived();
                if (x.masked(t)) clear(t, v);
                const bool more = t + ahead < x.t1;
                if (x.two) {
                    const int s = more ? arrived() : 0;
                    for (int g = 0; g < 2; ++g) {
                        products(g, v, t > x.t0);
                        if (more) scores(g, g, s);
                        else if (lane == 0) mma_commit(o_full(g));
                    }
                    if (lane == 0) {
                        mma_commit(kv_empty(v));
                        if (more) mma_commit(kv_empty(s));
                    }
                } else {
                    const int g = (t - x.t0) & 1;
                    products(g, v, t >= x.t0 + 2);
                    if (lane == 0) mma_commit(kv_empty(v));
                    if (more) {
                        const int s = arrived();
                        scores(g, 0, s);
                        if (lane == 0) mma_commit(kv_empty(s));
                    } else if (lane == 0) mma_commit(o_full(g));
                }
            }
        }
    } else if (warp < 8) {
        // ---- softmax ---------------------------------------------------------------------------------
        const int g = warp >> 2, gt = tid & (kTile - 1);
        const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
        const uint32_t t_s = tm + lanes + L::kS + g * kTile, t_p = tm + lanes + L::kP + g * L::kPStep, t_o = tm + lanes + L::kO;
        uint32_t s_phase = 0, o_phase = 0;
        const float cs = A.scale_log2;
        while (walk.next(x)) {
            {   // queries: of this group's rows, or half of the rows that both have
                constexpr int kVecs = D / 8, kStep = kTile / kVecs;
                const int q = x.two ? g : 0, r0 = x.two ? 0 : g * (kTile / 2), r1 = x.two ? kTile : r0 + kTile / 2;
                const int vec = gt % kVecs;
                uint8_t *dst = smem + q * L::kTileBytes + (vec / 8) * L::kHalfBytes;
#pragma unroll 4
                for (int r = r0 + gt / kVecs; r < r1; r += kStep) {
                    uint4 u = make_uint4(0, 0, 0, 0);
                    if (q * kTile + r < x.rows) {
                        const AttRow o = row_of(c, x, q * kTile + r);
                        u = *reinterpret_cast<const uint4 *>(static_cast<const T *>(A.q.data) + o.b * A.q.seq + o.n * A.q.node + o.h * A.q.head + vec * 8);
                    }
                    *reinterpret_cast<uint4 *>(dst + r * 128 + ((vec & 7) ^ (r & 7)) * 16) = u;
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tmem_fence_before();
                bar_arrive(q_full);
            }
            const int row = (x.two ? g * kTile : 0) + gt;
            const bool warp_on = row - lane < x.rows;   // any row in this warp
            const AttRow at = row_of(c, x, min(row, x.rows - 1));
            float ref = neg_inf(), sum = 0.f;
            const int step = x.two ? 1 : 2, first = x.two ? x.t0 : x.t0 + g;
            for (int t = first; t < x.t1; t += step) {
                bar_wait(s_full(g), s_phase, gave_up);
                s_phase ^= 1u;
                tmem_fence_after();
                if (warp_on) {
                    float s[kTile];
#pragma unroll
                    for (int i = 0; i < 4; ++i) tmem_ld32_async(t_s + 32 * i, s + 32 * i);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < kTile; ++i) asm volatile("" : "+f"(s[i]));
                    if (x.masked(t)) {
                        uint32_t bits[4];
                        row_bits(A, x, t, at.n, bits);
#pragma unroll
                        for (int i = 0; i < kTile; ++i) s[i] = bits[i / 32] >> (i & 31) & 1 ? s[i] : neg_inf();
                    }
                    float m0 = neg_inf(), m1 = neg_inf(), m2 = neg_inf(), m3 = neg_inf();
#pragma unroll
                    for (int i = 0; i < kTile; i += 8) {
                        m0 = fmaxf(m0, fmaxf(s[i], s[i + 1]));
                        m1 = fmaxf(m1, fmaxf(s[i + 2], s[i + 3]));
                        m2 = fmaxf(m2, fmaxf(s[i + 4], s[i + 5]));
                        m3 = fmaxf(m3, fmaxf(s[i + 6], s[i + 7]));
                    }
                    const float top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)) * cs - Weight<T>::kBias;
                    if (t == first) ref = top;
                    else if (__any_sync(kFull, top > ref + kSlack)) {
                        // (the product that added the last tile to O is done: it was issued before these scores)
                        const float now = fmaxf(ref, top), f = now == neg_inf() ? 1.f : ex2(ref - now);
                        sum *= f;
                        ref = now;
#pragma unroll 1
                        for (int i = 0; i < D; i += 32) {
                            float o[32];
                            tmem_ld32(t_o + g * D + i, o);
#pragma unroll
                            for (int j = 0; j < 32; ++j) o[j] *= f;
                            tmem_st32(t_o + g * D + i, o);
                        }
                    }
                    const float sub = ref == neg_inf() ? 0.f : -ref;
                    float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t w[32];
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const float *y = s + 64 * h + 2 * i;
                            const float a = ex2(fmaf(y[0], cs, sub)), b = ex2(fmaf(y[1], cs, sub));
                            const float e = ex2(fmaf(y[2], cs, sub)), f = ex2(fmaf(y[3], cs, sub));
                            l0 += a; l1 += b; l2 += e; l3 += f;
                            w[i] = pack2<T>(a, b);
                            w[i + 1] = pack2<T>(e, f);
                        }
                        tmem_st32_async(t_p + 32 * h, w);
                    }
                    sum += (l0 + l1) + (l2 + l3);
                    tmem_wait_st();
                    tmem_fence_before();
                }
                bar_arrive(p_full(g));
            }
            // ---- the end of the piece ------------------------------------------------------------------
            const bool any = first < x.t1;
            if (any) {
                bar_wait(o_full(g), o_phase, gave_up);
                o_phase ^= 1u;
            }
            tmem_fence_after();
            float f0 = 1.f, f1 = 0.f;   // factors of this group's O, of the other group's
            bool write = warp_on;
            if (!x.two) {
                if (g == 1) other[gt] = make_float2(ref, sum);
                tmem_fence_before();
                asm volatile("bar.sync 1, 256;" ::: "memory");
                tmem_fence_after();
                write = warp_on && g == 0;
                if (g == 0 && x.t1 - x.t0 > 1) {
                    const float2 z = other[gt];
                    const float now = fmaxf(ref, z.x), r = now == neg_inf() ? 0.f : now;
                    f0 = ex2(ref - r); f1 = ex2(z.x - r);
                    sum = sum * f0 + z.y * f1;
                    ref = now;
                }
            }
            if (write) {
                const bool whole = !x.shared && P.shared_tiles == 0 && x.t1 - x.t0 == x.tiles, join = !x.two && x.t1 - x.t0 > 1;
                const bool mine = row < x.rows, none = sum == 0.f;
                const float inv = none ? 0.f : 1.f / sum;
                const int bad = *static_cast<volatile int *>(&bad_values);
                int64_t slot_row = 0;
                if (!whole) {
                    slot_row = x.shared ? (x.item + blockIdx.x) * P.shared_rows + row
                                        : P.slots * P.shared_rows + (x.item + blockIdx.x) * P.own_rows + row;
                    if (mine) P.ml[slot_row] = make_float2(ref, sum);
                } else if (mine && A.lse) {
                    A.lse[(static_cast<int64_t>(at.b) * c.nodes + at.n) * c.heads + at.h] = none ? neg_inf() : (ref + log2f(sum)) * 0.6931471805599453f;
                }
#pragma unroll 1
                for (int i = 0; i < D; i += 32) {
                    float o[32];
                    tmem_ld32(t_o + g * D + i, o);
                    if (join) {
                        float z[32];
                        tmem_ld32(t_o + D + i, z);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = o[j] * f0 + z[j] * f1;
                    }
                    if (bad && !x.shared && mine) {
                        float z[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[j] = o[j];
                        add_not_finite<T>(A, x, at.n, i, z);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = z[j];
                    }
                    if (mine && whole) {
                        T *dst = static_cast<T *>(A.out.data) + at.b * A.out.seq + at.n * A.out.node + at.h * A.out.head + i;
#pragma unroll
                        for (int j = 0; j < 32; j += 8) {
                            uint4 u;
                            u.x = pack2<T>(o[j] * inv, o[j + 1] * inv); u.y = pack2<T>(o[j + 2] * inv, o[j + 3] * inv);
                            u.z = pack2<T>(o[j + 4] * inv, o[j + 5] * inv); u.w = pack2<T>(o[j + 6] * inv, o[j + 7] * inv);
                            *reinterpret_cast<uint4 *>(dst + j) = u;
                        }
                    } else if (mine) {
                        float *dst = P.o + slot_row * D + i;
#pragma unroll
                        for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4 *>(dst + j) = make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
                    }
                    __syncwarp();
                }
            }
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (*gave_up) {   // copies that were not waited for are in shared memory long before this ends
        const unsigned long long t0 = now_ns();
        while (now_ns() - t0 < 2000000ull) __nanosleep(10000);
        __syncthreads();
    }
    if (tid == 0) P.error[blockIdx.x] = gave_up_;
    if (warp == 9) tmem_dealloc(tm, 512);
}

constexpr int kJoinThreads = 256;

// Joins the pieces of every row that has more than one (a warp per row), and finds bad pages (the first `batch` CTAs, if wanted).
template <class T, int D>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const __grid_constant__ AttKernelArgs K) {
    constexpr int E = D / 32;
    pdl_begin();
    const AttentionArgs &A = K.a;
    const CacheArgs &c = A.c;
    const AttPlan &P = K.p;
    const int tid = threadIdx.x, lane = tid & 31;
    unsigned block = blockIdx.x;
    if (c.status) {
        if (block < static_cast<unsigned>(c.batch)) {
            const int b = block, ps = 1 << c.page_shift, len = c.lens[b];
            bool bad = false, error = false;
            if (len >= 0) {
                const int64_t need = (static_cast<int64_t>(len) + c.nodes + ps - 1) >> c.page_shift;
                bad = need > c.table_width;
                const int32_t *row = c.table + b * c.stride_table;
                for (int64_t i = tid; i < min(need, static_cast<int64_t>(c.table_width)); i += kJoinThreads) bad |= row[i] < 0 || row[i] >= c.pages;
                for (int i = tid; i < (A.shared_len + static_cast<int64_t>(ps) - 1) >> c.page_shift; i += kJoinThreads)
                    bad |= A.shared_table[i] < 0 || A.shared_table[i] >= c.pages;
            }
            for (int i = tid; i < P.grid; i += kJoinThreads) error |= P.error[i] != 0;
            bad = __syncthreads_or(bad);
            error = __syncthreads_or(error);
            if (tid == 0) c.status[b] = (bad ? SPECHUB_ST_PAGE : 0u) | (error ? SPECHUB_ST_INTERNAL : 0u);
            return;
        }
        block -= c.batch;
    }
    const int64_t at = block * int64_t(kJoinThreads / 32) + (tid >> 5);
    if (at >= static_cast<int64_t>(c.batch) * c.nodes * c.heads) return;
    const int h = at % c.heads, n = at / c.heads % c.nodes, b = static_cast<int>(at / c.heads / c.nodes);
    const int len = c.lens[b];
    if (len < 0) return;
    const int g = c.heads / c.kv_heads, hk = h / g, own_row = n * g + (h - hk * g), tiles = own_tiles(c, len);
    const AttSplit split(P, P.before[c.batch]);
    const int in_b = hk * P.own_blocks + own_row / kBlockRows;
    const int64_t own_item = static_cast<int64_t>(b) * c.kv_heads * P.own_blocks + in_b;
    const int64_t own0 = P.shared_units + P.before[b] + static_cast<int64_t>(in_b) * tiles, own1 = own0 + tiles;
    if (P.shared_tiles == 0 && split.cta(own0) == split.cta(own1 - 1)) return;   // finished in place
    const int64_t all_row = static_cast<int64_t>(b) * c.nodes * g + own_row, shared_item = P.shared_tiles ? hk * static_cast<int64_t>(P.shared_blocks) + all_row / kBlockRows : 0;
    float ref = neg_inf(), sum = 0.f, o[E] = {};
    const auto add = [&](int64_t slot_row) {
        const float2 ml = P.ml[slot_row];
        float z[E];
        const float *src = P.o + slot_row * D + lane * E;
        if (E == 4) { const float4 v = *reinterpret_cast<const float4 *>(src); z[0] = v.x; z[1] = v.y; z[E - 2] = v.z; z[E - 1] = v.w; }
        else { const float2 v = *reinterpret_cast<const float2 *>(src); z[0] = v.x; z[1] = v.y; }
        const float now = fmaxf(ref, ml.x), r = now == neg_inf() ? 0.f : now, f0 = ex2(ref - r), f1 = ex2(ml.x - r);
        sum = sum * f0 + ml.y * f1;
        ref = now;
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] = o[i] * f0 + z[i] * f1;
    };
    for (int64_t u = shared_item * P.shared_tiles, u1 = u + P.shared_tiles; u < u1;) {
        const int cta = split.cta(u);
        add((shared_item + cta) * P.shared_rows + all_row % kBlockRows);
        u = split.first(cta + 1);
    }
    for (int64_t u = own0; u < own1;) {
        const int cta = split.cta(u);
        add(P.slots * P.shared_rows + (own_item + cta) * P.own_rows + own_row % kBlockRows);
        u = split.first(cta + 1);
    }
    const bool none = sum == 0.f;
    const float inv = none ? 0.f : 1.f / sum;
    T *dst = static_cast<T *>(A.out.data) + b * A.out.seq + n * A.out.node + h * A.out.head + lane * E;
#pragma unroll
    for (int i = 0; i < E; i += 2) *reinterpret_cast<uint32_t *>(dst + i) = pack2<T>(o[i] * inv, o[i + 1] * inv);
    if (A.lse && lane == 0) A.lse[at] = none ? neg_inf() : (ref + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace spechub
