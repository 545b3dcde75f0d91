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
// Registers of a thread: what the block is launched with, and how its warpgroups share them then (a row of scores is 128).
constexpr int kLaunchRegs = 168, kSoftmaxRegs = 200, kOtherRegs = 104;
static_assert(256 * kSoftmaxRegs + 128 * kOtherRegs <= kAttThreads * kLaunchRegs, "the block's own registers");
constexpr float kSlack = 8.f;
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

// x / d for x < 2^31 by a product (Granlund, Montgomery: Division by invariant integers using multiplication).
struct FastDiv {
    uint32_t d, m, s;
    __host__ static FastDiv of(uint32_t d) {
        uint32_t s = 0;
        while ((1ull << s) < d) ++s;
        return FastDiv{d, static_cast<uint32_t>((((1ull << s) - d) << 32) / d + 1), s};
    }
    __device__ uint32_t quot(uint32_t x) const { return (__umulhi(m, x) + x) >> s; }
};

// What the host knows of the work.  A block of `tiles` tiles costs kBlockCost + tiles * (shared_cost or own_cost), and the CTAs share
// the sum of the costs evenly.
constexpr int kBlockCost = 6, kTileCost = 4;
struct AttPlan {
    int shared_tiles, shared_blocks, own_blocks, grid;   // tiles of the prefix; row blocks per cache head: of all rows, of a sequence
    int shared_rows, own_rows;                           // rows of a slot in the workspace
    int shared_items, shared_cost;                       // blocks of the prefix, what they cost
    int64_t slots;                                       // slots of the shared pieces
    FastDiv group, nodes;
    int *before;                                         // [batch + 1] cost of the own blocks before sequence b
    int *error;                                          // [grid]
    float2 *ml;                                          // (reference, sum) of every row of every slot
    float *o;                                            // [..][head_dim], not divided by the sum
};

struct AttKernelArgs {
    AttentionArgs a;
    AttPlan p;
};

__device__ __forceinline__ int own_end(const CacheArgs &c, int len) {   // keys of a sequence that is there
    const int64_t slots = static_cast<int64_t>(c.table_width) << c.page_shift;
    return static_cast<int>(min(static_cast<int64_t>(len) + c.nodes, slots));
}
__device__ __forceinline__ int own_tiles(const CacheArgs &c, int len) {
    return len < 0 ? 0 : static_cast<int>((static_cast<unsigned>(own_end(c, len)) + kTile - 1) / kTile);
}
__device__ __forceinline__ int block_cost(int tiles) { return tiles ? kBlockCost + tiles * kTileCost : 0; }
// tiles of a block that lie before `cost`, counted from the block's start
__device__ __forceinline__ int tiles_before(int cost, int tiles) {
    return min(tiles, max(0, (cost - kBlockCost + kTileCost - 1) / kTileCost));
}
// Blocks are numbered: all of the shared prefix, then sequence by sequence.  Of the whole cost `all`, CTA i takes [first(i), first(i + 1)).
__device__ __forceinline__ int split_first(int cta, int all, int grid) {
    const unsigned q = static_cast<unsigned>(all) / grid, r = static_cast<unsigned>(all) - q * grid;
    return cta * q + (cta * r + grid - 1) / grid;
}
__device__ __forceinline__ int split_cta(int cost, int all, int grid) {
    return static_cast<int>(static_cast<unsigned long long>(static_cast<unsigned>(cost)) * grid / static_cast<unsigned>(all));
}

// Consecutive tiles of one block of rows.
struct AttPiece {
    bool shared, two;      // two: more than 128 rows
    int b, head, block, rows, t0, t1, tiles;
    int item;              // among the shared or among the own blocks
    int plain, keys;       // keys that every row sees; all keys
    __device__ bool masked(int t) const { return t >= plain / kTile; }
};

// The pieces of a CTA's run; every role walks through them by itself.
struct AttStart { int from, to, at; bool shared; int b, head, block; };   // costs; `at`: where the block begins
struct AttWalk {
    const CacheArgs &c;
    const AttPlan &p;
    int shared_len, from, to, at, b, head, block, len, tiles;
    bool shared;

    __device__ AttWalk(const AttKernelArgs &K, const AttStart &s)
        : c(K.a.c), p(K.p), shared_len(K.a.shared_len), from(s.from), to(s.to), at(s.at), b(s.b), head(s.head), block(s.block), shared(s.shared) {
        look();
    }
    __device__ void look() {
        if (shared) { tiles = p.shared_tiles; return; }
        tiles = 0;
        if (at >= to) return;
        for (; b < c.batch; ++b) {
            len = c.lens[b];
            tiles = own_tiles(c, len);
            if (tiles) break;
        }
    }
    __device__ bool next(AttPiece &x) {
        while (at < to && tiles) {
            x.shared = shared;
            x.head = head;
            x.block = block;
            x.tiles = tiles;
            x.t0 = from > at ? tiles_before(from - at, tiles) : 0;
            x.t1 = tiles_before(to - at, tiles);
            int rows;
            if (shared) {
                x.b = 0;
                x.item = head * p.shared_blocks + block;
                x.plain = x.keys = shared_len;
                rows = c.batch * c.nodes * p.group.d;
            } else {
                x.b = b;
                x.item = (b * c.kv_heads + head) * p.own_blocks + block;
                x.keys = own_end(c, len);
                x.plain = min(len, x.keys);
                rows = c.nodes * p.group.d;
            }
            x.rows = min(kBlockRows, rows - block * kBlockRows);
            x.two = x.rows > kTile;
            at += block_cost(tiles);
            if (++block == (shared ? p.shared_blocks : p.own_blocks)) {
                block = 0;
                if (++head == c.kv_heads) {
                    head = 0;
                    if (shared) { shared = false; b = 0; }
                    else ++b;
                    look();
                }
            }
            if (x.t1 > x.t0) return true;
        }
        return false;
    }
};

// Where row `i` of a block is.
struct AttRow { int b, n, h; };
__device__ __forceinline__ AttRow row_of(const AttPlan &p, const AttPiece &x, int i) {
    const unsigned r = x.block * kBlockRows + i, node = p.group.quot(r);
    AttRow o;
    o.h = x.head * p.group.d + (r - node * p.group.d);
    if (x.shared) { o.b = p.nodes.quot(node); o.n = node - o.b * p.nodes.d; }
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
    __shared__ __align__(8) uint64_t bars[2 * L::kStages + 11];
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up_, bad_values;
    __shared__ float2 other[kTile];           // (reference, sum) of the second group's rows
    __shared__ int warp_sum[kAttThreads / 32];
    __shared__ AttStart start;
    volatile int *const gave_up = &gave_up_;

    const AttentionArgs &A = K.a;
    const CacheArgs &c = A.c;
    const AttPlan &P = K.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t *const smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t s_q = saddr(smem), s_kv = s_q + 2 * L::kTileBytes, bar0 = saddr(bars);
    const auto kv_full = [&](int s) { return bar0 + 8u * s; };
    const auto kv_empty = [&](int s) { return bar0 + 8u * (L::kStages + s); };
    const uint32_t bar1 = bar0 + 16u * L::kStages;
    const auto q_full = [&](int q) { return bar1 + 8u * q; };
    const auto q_empty = [&](int q) { return bar1 + 16u + 8u * q; };
    const auto s_full = [&](int t) { return bar1 + 32u + 8u * t; };
    const auto p_full = [&](int t) { return bar1 + 48u + 8u * t; };
    const auto o_full = [&](int t) { return bar1 + 64u + 8u * t; };
    const uint32_t o_free = bar1 + 80u;

    if (warp == 9) tmem_alloc(saddr(&tmem_base), 512);
    if (tid == 0) {
        for (int s = 0; s < L::kStages; ++s) { bar_init(kv_full(s), 1); bar_init(kv_empty(s), 1); }
        for (int t = 0; t < 2; ++t) {
            bar_init(q_full(t), 64); bar_init(q_empty(t), 1);
            bar_init(s_full(t), 1); bar_init(p_full(t), kTile); bar_init(o_full(t), 1);
        }
        bar_init(o_free, 2 * kTile);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        gave_up_ = 0;
        bad_values = 0;
        tma_prefetch_map(&map_k);
        tma_prefetch_map(&map_v);
    }
    pdl_begin();

    // This CTA's run: own costs of all sequences summed up, in the order of the sequences.
    {
        const int per = (c.batch + kAttThreads - 1) / kAttThreads, b0 = min(c.batch, tid * per), b1 = min(c.batch, b0 + per);
        const int per_b = c.kv_heads * P.own_blocks;
        int last = 0, mine = 0;   // of the thread's only or last sequence
        for (int b = b0; b < b1; ++b) {
            last = block_cost(own_tiles(c, c.lens[b]));
            mine += last * per_b;
        }
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(kFull, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) warp_sum[warp] = upto;
        __syncthreads();
        int all = P.shared_cost;
#pragma unroll
        for (int w = 0; w < kAttThreads / 32; ++w) {
            const int v = warp_sum[w];
            if (w < warp) upto += v;
            all += v;
        }
        upto += P.shared_cost;
        const int from = split_first(blockIdx.x, all, P.grid), to = split_first(blockIdx.x + 1, all, P.grid);
        int before = upto - mine;
        const bool here = from >= before && from < upto;
        if (tid == 0 && from == to) start = AttStart{0, 0, 0, false, 0, 0, 0};
        if (tid == 0 && from < to && from < P.shared_cost) {
            const int each = block_cost(P.shared_tiles), item = from / each;
            start = AttStart{from, to, item * each, true, 0, item / P.shared_blocks, item % P.shared_blocks};
        }
        if (here && from < to) {
            int b = b0;
            if (per > 1)
                for (; b < b1; ++b) {
                    last = block_cost(own_tiles(c, c.lens[b]));
                    if (from < before + last * per_b) break;
                    before += last * per_b;
                }
            const int in_b = (from - before) / last;
            start = AttStart{from, to, before + in_b * last, false, b, in_b / P.own_blocks, in_b % P.own_blocks};
        }
        if (blockIdx.x == 0 && b0 < b1) {   // for the kernel that joins
            before = upto - mine;
            for (int b = b0; b < b1; ++b) {
                P.before[b] = before;
                before += block_cost(own_tiles(c, c.lens[b])) * per_b;
            }
            if (b1 == c.batch) P.before[c.batch] = before;
        }
        tmem_fence_before();
        __syncthreads();
        tmem_fence_after();
    }
    const uint32_t tm = tmem_base;
    AttWalk walk(K, start);
    AttPiece x = {};

    if (warp < 8) {
        // ---- softmax ---------------------------------------------------------------------------------
        more_registers<kSoftmaxRegs>();
        const int g = warp >> 2, gt = tid & (kTile - 1);
        const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
        const uint32_t t_s = tm + lanes + L::kS + g * kTile, t_p = tm + lanes + L::kP + g * L::kPStep, t_o = tm + lanes + L::kO;
        uint32_t s_phase = 0, o_phase = 0;
        const float cs = A.scale_log2;
        while (walk.next(x)) {
            const int row = (x.two ? g * kTile : 0) + gt;
            const bool warp_on = row - lane < x.rows;   // any row in this warp
            const AttRow at = row_of(P, x, min(row, x.rows - 1));
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
                    tmem_wait_ld(s);
                    if (x.masked(t)) {
                        uint32_t bits[4];
                        row_bits(A, x, t, at.n, bits);
#pragma unroll
                        for (int i = 0; i < kTile; ++i) s[i] = bits[i / 32] >> (i & 31) & 1 ? s[i] : neg_inf();
                    }
                    float m0 = neg_inf(), m1 = neg_inf(), m2 = neg_inf(), m3 = neg_inf();
#pragma unroll
                    for (int i = 0; i < kTile; i += 8) {
                        m0 = max3(m0, s[i], s[i + 1]);
                        m1 = max3(m1, s[i + 2], s[i + 3]);
                        m2 = max3(m2, s[i + 4], s[i + 5]);
                        m3 = max3(m3, s[i + 6], s[i + 7]);
                    }
                    const float top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)) * cs - Weight<T>::kBias;
                    if (t == first) ref = top;
                    else if (__any_sync(kFull, top > ref + kSlack && row < x.rows)) {
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
                    const float2 cs2 = make_float2(cs, cs), sub2 = make_float2(sub, sub);
                    float2 l0 = make_float2(0.f, 0.f), l1 = l0;
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        uint32_t w[16];
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const float *y = s + 32 * h + 2 * i;
                            const float2 a = fma2(make_float2(y[0], y[1]), cs2, sub2), b = fma2(make_float2(y[2], y[3]), cs2, sub2);
                            const float2 e = make_float2(ex2(a.x), ex2(a.y)), f = make_float2(ex2(b.x), ex2(b.y));
                            l0 = add2(l0, e);
                            l1 = add2(l1, f);
                            w[i] = pack2<T>(e.x, e.y);
                            w[i + 1] = pack2<T>(f.x, f.y);
                        }
                        tmem_st16_async(t_p + 16 * h, w);
                    }
                    sum += (l0.x + l0.y) + (l1.x + l1.y);
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
                    slot_row = x.shared ? (x.item + int64_t(blockIdx.x)) * P.shared_rows + row
                                        : P.slots * P.shared_rows + (x.item + int64_t(blockIdx.x)) * P.own_rows + row;
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
            tmem_fence_before();
            bar_arrive(o_free);
        }
    } else if (fewer_registers<kOtherRegs>(), warp == 8) {
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
        uint32_t phase = 0, q_phase = 0, p_phase = 0, free_phase = 1;
        int q_slot = 0;
        constexpr uint32_t desc_s = mma_desc(kBf16, kTile, false), desc_o = mma_desc(kBf16, D, true);
        const auto arrived = [&]() {   // the next stage of the ring
            bar_wait(kv_full(stage), phase, gave_up);
            const int s = stage;
            if (++stage == L::kStages) { stage = 0; phase ^= 1u; }
            return s;
        };
        const bool lead = lane == 0;
        const uint32_t tmu = uniform(tm), kv_op = operand(uniform(s_kv), L::kHalfBytes), q_op = operand(uniform(s_q), L::kHalfBytes);
        const auto scores = [&](int t, int q, int s) {   // S_t = Q_q K^T
            uint32_t a = uniform(q_op + q * (L::kTileBytes >> 4)), b = uniform(kv_op + s * (L::kTileBytes >> 4));
            const uint32_t d = uniform(tmu + L::kS + t * kTile);
#pragma unroll 1
            for (int h = 0; h < L::kHalves; ++h) {
#pragma unroll
                for (int k = 0; k < 4; ++k) mma_ss(d, a + 2 * k, b + 2 * k, desc_s, h + k > 0, lead);
                a += L::kHalfBytes >> 4;
                b += L::kHalfBytes >> 4;
            }
            mma_commit(s_full(t), lead);
        };
        const auto products = [&](int t, int s, bool add) {   // O_t (+)= P_t V
            uint32_t a = uniform(tmu + L::kP + t * L::kPStep), b = uniform(kv_op + s * (L::kTileBytes >> 4));
            const uint32_t d = uniform(tmu + L::kO + t * D);
            bar_wait(p_full(t), p_phase >> t & 1u, gave_up);
            p_phase ^= 1u << t;
            tmem_fence_after();
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int k = 0; k < 4; ++k) mma_ts(d, a + 8 * k, b + k * (2048 >> 4), desc_o, add || h + k > 0, lead);
                a += 32;
                b += 4 * (2048 >> 4);
            }
        };
        // values behind the end, and those of tree nodes that are no numbers: zero
        const auto clear = [&](int tile, int s) {
            constexpr int kVecs = D / 8;
            constexpr uint32_t kExp = kBf16 ? 0x7f807f80u : 0x7c007c00u;   // all ones: no finite number
            const int r0 = max(0, x.plain - tile * kTile), r1 = min(kTile, x.keys - tile * kTile);
            uint8_t *const v = smem + 2 * L::kTileBytes + s * L::kTileBytes;
            const auto at = [&](int i) { return reinterpret_cast<uint4 *>(v + (i % kVecs / 8) * L::kHalfBytes + (i / kVecs) * 128 + (i % 8) * 16); };
            bool bad = false;
            for (int i = lane + r0 * kVecs; i < r1 * kVecs; i += 128) {
                uint4 u[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) u[j] = i + 32 * j < r1 * kVecs ? *at(i + 32 * j) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t *w = &u[j].x, hit = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t t = (w[k] & kExp) ^ kExp;   // a half that is zero: no finite number
                        hit |= (t - 0x00010001u) & ~t & 0x80008000u;
                    }
                    if (hit) {
                        bad = true;
                        for (int k = 0; k < 4; ++k) {
                            if ((w[k] & kExp & 0xffffu) == (kExp & 0xffffu)) w[k] &= 0xffff0000u;
                            if ((w[k] & kExp & 0xffff0000u) == (kExp & 0xffff0000u)) w[k] &= 0xffffu;
                        }
                        *at(i + 32 * j) = u[j];
                    }
                }
            }
            for (int i = lane + r1 * kVecs; i < kTile * kVecs; i += 32) *at(i) = make_uint4(0, 0, 0, 0);
            if (__any_sync(kFull, bad) && lane == 0) *static_cast<volatile int *>(&bad_values) = 1;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __threadfence_block();
            __syncwarp();
        };
        while (walk.next(x)) {
            // Queries of both groups, or of one block in whichever slot is next.
            int q0 = q_slot, q1;
            bar_wait(q_full(q_slot), q_phase, gave_up);
            if (++q_slot == 2) { q_slot = 0; q_phase ^= 1u; }
            q1 = x.two ? q_slot : q0;
            if (x.two) {
                bar_wait(q_full(q_slot), q_phase, gave_up);
                if (++q_slot == 2) { q_slot = 0; q_phase ^= 1u; }
            }
            // Products of tile t, scores of tile t + ahead: each once in the code, which other warps push out of the instruction cache.
            const int ahead = x.two ? 1 : 2;
            for (int t = x.t0 - ahead; t < x.t1; ++t) {
                const bool now = t >= x.t0, more = t + ahead < x.t1;
                int v = 0, s = 0;
                if (t == x.t0) {   // O of the piece before has been read by now or soon, and what was said of its values
                    bar_wait(o_free, free_phase, gave_up);
                    free_phase ^= 1u;
                    tmem_fence_after();
                    if (lane == 0) *static_cast<volatile int *>(&bad_values) = 0;
                    __syncwarp();
                }
                if (now) {
                    v = arrived();
                    if (x.masked(t)) clear(t, v);
                }
                const int g0 = x.two ? 0 : (t + ahead - x.t0) & 1, g1 = x.two ? 2 : g0 + 1;
                for (int g = g0; g < g1; ++g) {
                    if (now) {
                        products(g, v, t >= x.t0 + ahead);
                        if (g == g1 - 1) mma_commit(kv_empty(v), lead);
                    }
                    if (more) {
                        if (g == g0) s = arrived();
                        scores(g, g ? q1 : q0, s);
                        if (g == g1 - 1) {
                            mma_commit(kv_empty(s), lead);
                            if (t + ahead == x.t1 - 1) {   // the last ones
                                mma_commit(q_empty(q0), lead);
                                if (x.two) mma_commit(q_empty(q1), lead);
                            }
                        }
                    } else if (now) mma_commit(o_full(g), lead);
                }
            }
        }
        // (the last arrivals come before the CTA ends)
        bar_wait(o_free, free_phase, gave_up);
    } else if (warp >= 10) {
        // ---- queries -----------------------------------------------------------------------------------
        constexpr int kVecs = D / 8, kStep = 64 / kVecs, kBatch = 8;   // rows that the two warps bring at once; loads in flight per thread
        int slot = 0;
        uint32_t phase = 1;
        const int qt = tid - 320, vec = qt % kVecs;
        while (walk.next(x)) {
            for (int i = 0; i < (x.two ? 2 : 1); ++i) {
                bar_wait(q_empty(slot), phase, gave_up);
                uint8_t *dst = smem + slot * L::kTileBytes + (vec / 8) * L::kHalfBytes;
                const int rows = min(kTile, x.rows - i * kTile);   // (what the other rows hold matters to nobody)
                for (int r0 = qt / kVecs; r0 < rows; r0 += kBatch * kStep) {
                    uint4 u[kBatch];
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        const AttRow o = row_of(P, x, i * kTile + min(rows - 1, r0 + j * kStep));
                        u[j] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(A.q.data) + o.b * A.q.seq + o.n * A.q.node + o.h * A.q.head + vec * 8);
                    }
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        const int r = r0 + j * kStep;
                        if (r < rows) *reinterpret_cast<uint4 *>(dst + r * 128 + ((vec & 7) ^ (r & 7)) * 16) = u[j];
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                bar_arrive(q_full(slot));
                if (++slot == 2) { slot = 0; phase ^= 1u; }
            }
        }
        for (int i = 0; i < 2; ++i) {
            bar_wait(q_empty(slot), phase, gave_up);
            if (++slot == 2) { slot = 0; phase ^= 1u; }
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (*gave_up) {   // copies that were not waited for are in shared memory long before this ends
        const long long t0 = clock64();
        while (clock64() - t0 < 4000000) __nanosleep(10000);
        __syncthreads();
    }
    if (tid == 0) P.error[blockIdx.x] = gave_up_;
    if (warp == 9) tmem_dealloc(tm, 512);
}

constexpr int kJoinThreads = 256, kJoinRows = 32;

// Joins the pieces of every block that has more than one, kJoinRows of its rows per CTA, a warp per row; and finds bad pages (the first
// `batch` CTAs, if wanted).
template <class T, int D>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const __grid_constant__ AttKernelArgs K) {
    constexpr int E = D / 32;
    pdl_begin();
    const AttentionArgs &A = K.a;
    const CacheArgs &c = A.c;
    const AttPlan &P = K.p;
    const int tid = threadIdx.x, lane = tid & 31;
    int block = blockIdx.x;
    if (c.status) {
        if (block < c.batch) {
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
    const int chunks = (P.own_rows + kJoinRows - 1) / kJoinRows, chunk = block % chunks;
    const int item = block / chunks, per_b = c.kv_heads * P.own_blocks, b = item / per_b, in_b = item - b * per_b;
    const int len = c.lens[b];
    if (len < 0) return;
    const int tiles = own_tiles(c, len), each = block_cost(tiles), all = P.before[c.batch];
    const int own0 = P.before[b] + in_b * each;                       // the block's cost interval, and where its tiles begin
    const int c0 = split_cta(own0 + kBlockCost, all, P.grid), c1 = split_cta(own0 + each - 1, all, P.grid);
    if (P.shared_tiles == 0 && tiles_before(split_first(c0 + 1, all, P.grid) - own0, tiles) == tiles) return;   // finished in place
    const int hk = in_b / P.own_blocks, first = (in_b - hk * P.own_blocks) * kBlockRows, rows = min(P.own_rows, c.nodes * static_cast<int>(P.group.d) - first);
    for (int row = chunk * kJoinRows + (tid >> 5); row < min(rows, (chunk + 1) * kJoinRows); row += kJoinThreads / 32) {
        float ref = neg_inf(), sum = 0.f, o[E] = {};
        // pieces of CTAs i0..i1 of a block at `at` in the costs (one whose run has no tile of it left nothing)
        const auto add = [&](int at, int n, int i0, int i1, int64_t slot_row, int step) {
            for (int i = i0; i <= i1; ++i) {
                const int t0 = tiles_before(split_first(i, all, P.grid) - at, n), t1 = tiles_before(split_first(i + 1, all, P.grid) - at, n);
                if (t1 <= t0) continue;
                const float2 ml = P.ml[slot_row + int64_t(i) * step];
                const float *src = P.o + (slot_row + int64_t(i) * step) * D + lane * E;
                float z[E];
                if (E == 4) { const float4 v = *reinterpret_cast<const float4 *>(src); z[0] = v.x; z[1] = v.y; z[E - 2] = v.z; z[E - 1] = v.w; }
                else { const float2 v = *reinterpret_cast<const float2 *>(src); z[0] = v.x; z[1] = v.y; }
                const float now = fmaxf(ref, ml.x), r = now == neg_inf() ? 0.f : now, f0 = ex2(ref - r), f1 = ex2(ml.x - r);
                sum = sum * f0 + ml.y * f1;
                ref = now;
#pragma unroll
                for (int k = 0; k < E; ++k) o[k] = o[k] * f0 + z[k] * f1;
            }
        };
        if (P.shared_tiles) {
            const int64_t r = static_cast<int64_t>(b) * c.nodes * P.group.d + first + row;
            const int in = hk * P.shared_blocks + static_cast<int>(r / kBlockRows), s_each = block_cost(P.shared_tiles), at = in * s_each;
            add(at, P.shared_tiles, split_cta(at + kBlockCost, all, P.grid), split_cta(at + s_each - 1, all, P.grid),
                int64_t(in) * P.shared_rows + r % kBlockRows, P.shared_rows);
        }
        add(own0, tiles, c0, c1, P.slots * P.shared_rows + int64_t(item) * P.own_rows + row, P.own_rows);
        const bool none = sum == 0.f;
        const float inv = none ? 0.f : 1.f / sum;
        const int n = P.group.quot(first + row), h = hk * P.group.d + (first + row - n * P.group.d);
        T *dst = static_cast<T *>(A.out.data) + b * A.out.seq + n * A.out.node + h * A.out.head + lane * E;
#pragma unroll
        for (int i = 0; i < E; i += 2) *reinterpret_cast<uint32_t *>(dst + i) = pack2<T>(o[i] * inv, o[i + 1] * inv);
        if (A.lse && lane == 0) A.lse[(int64_t(b) * c.nodes + n) * c.heads + h] = none ? neg_inf() : (ref + log2f(sum)) * 0.6931471805599453f;
    }
}

}  // namespace spechub
