// Attention of tree nodes over a paged cache (include/spechub_cache.h), on the tensor cores.
//
// Mathematics.  A block of up to 256 rows (row = (sequence, node, query head of one cache head)) goes over its keys in tiles of
// 128.  S = Q K^T; per row p = 2^(c s - r), l += sum p, O += P V, with c = scale log2(e) and r the row's reference, at first the
// maximum of the first kStep keys.  Later maxima are not looked for: r is raised only where the weights of kStep keys sum up to more than
// kMostSum (so no weight is larger than that, and all are numbers in fp16 too), to their maximum in whole steps, and O and l are scaled by 2^(r_old - r): the division
// by l at the end makes the result the same.  Pieces of one row are joined by their references: out = sum_j 2^(r_j - R) O_j /
// sum_j 2^(r_j - R) l_j.
//   S, r, l, O and all that joins them are 32 bits.  P is rounded once to the cache's type, because the tensor core takes P and V in one 16-bit
// type; P in two terms of 16 bits would keep 32 bits' worth and double the product.  l adds the weights before that rounding.  Against 64
// bits out is then off by 0.0021 to 0.0023 in relation in bf16 and 0.00029 in fp16, where weights in 32 bits leave the 0.0017 and 0.00021 of out's own
// rounding.
//
// Work.  Rows that share keys are one block: the query heads of a cache head and all nodes of a sequence for its own context (7
// nodes of 4 heads are 28 rows), and the whole batch for the shared prefix, which is thus read once per 256 rows, from L2 but for the
// first time.  (block, tile) pairs are the units; every CTA (one per SM) takes one run of consecutive units, found on the device from
// the lengths alone.  So a few long sequences are split as finely as many short ones are gathered.  A run that covers a block's tiles
// is finished in place; other pieces go to the workspace and attention_join_kernel adds them in the order of the CTAs.
//
// CTA.  Warp 8 brings queries and keys, warp 11 values (bulk tensor copies, a box per page and 64 dimensions, each through a ring of its
// own), warps 0-3 and 4-7 are two softmax groups, a row per thread, each with its own S, P and O in tensor memory and a thread of its own
// (of warps 9 and 10) that issues its matrix instructions.  Two tiles of 128 rows: each group has one of them and every K / V tile serves
// both.  One: the groups take the K / V tiles in turn, for the same rows, and are joined at the end of the piece; else the tensor core
// and the loads would wait while one group computes.  P takes the place of S (head_dim 64 has room for its own).
//
// A single warp gets through an instruction in 4 to 5 clocks, and more when the others' code pushes its own out of the instruction
// cache.  So what single warps and the turnover between pieces do is kept short: queries and outputs are copied as tensors too (a box of
// all heads of some nodes), pieces of the workspace as they lie in shared memory; warp 8 alone finds the pieces, ahead of the others.
// One thread for the matrix instructions of both groups was late for each of them (4400 clocks for 256 rows and 128 keys, of which the
// tensor core needs 2050).
//
// What lies behind a sequence's end in a page may be anything.  Its scores are replaced, and its values, and values of tree nodes
// that are no finite numbers, are cleared in shared memory before the product (by the softmax group whose weights they meet), since
// 0 * NaN would reach every row; the rows that do see such a node get it added at the end.
//
// What bounds it, measured on inputs larger than L2: few rows, memory (64 sequences of one node, 1000 to 8192 tokens of 8 heads of 128:
// 205 us, 5.9 TB/s); many rows, the chain scores, weights, product of two groups, with the tensor cores and the special-function units
// busy half of the time each (64 x 31 nodes of 32 heads, 8192 tokens shared and 100 to 1000 own: 345 us, 823 TFLOP/s); short contexts,
// the 3 us between pieces.  In loops of seconds the power limit holds the first two at 221 and 369 us.  (What other comments here compare was
// measured side by side when the choice was made; both sides have become faster since.)
#pragma once

#include "spechub_pages.cuh"
#include "spechub_shapes.h"
#include "spechub_tmem.cuh"
#include "spechub_umma.cuh"

namespace spechub {

constexpr int kTile = 128;         // keys of a tile, rows of a softmax group
constexpr int kAttThreads = 384;
constexpr int kPieces = 4, kPieceReaders = 11;   // pieces that are known ahead; who reads them: 8 softmax warps, warps 9 to 11
// Registers of a thread: what the block is launched with, and how its warpgroups share them then (a row of scores is 128).
constexpr int kLaunchRegs = 168, kSoftmaxRegs = 200, kOtherRegs = 104;
static_assert(256 * kSoftmaxRegs + 128 * kOtherRegs <= kAttThreads * kLaunchRegs, "the block's own registers");
// What kStep weights may sum up to before the reference is raised.  None of them is negative, so none is larger than their sum, and all are
// numbers in fp16, which ends at 65504.
constexpr float kMostSum = 60000.f;
static_assert(kMostSum < 65504.f, "weights of fp16 are numbers");
// Scores that a thread has in registers at a time (32 / 64 / 128: 64 x 31 nodes behind 8192 shared tokens 370 / 339 / 348 us, 64 sequences of
// 31 nodes 139 / 139 / 152).
constexpr int kStep = 64;
// Weights are stored as 2^bias times themselves.  fp16 has numbers down to 2^-24 only: with the reference 7 below, weights of
// 2^-31 of the largest still count.
template <class T> struct Weight;
template <> struct Weight<__nv_bfloat16> { static constexpr bool kBf16 = true; static constexpr float kBias = 0.f; };
template <> struct Weight<__half> { static constexpr bool kBf16 = false; static constexpr float kBias = 7.f; };

template <int D>
struct AttShape {
    static constexpr int kHalves = D / 64;
    static constexpr int kHalfBytes = kTile * 128;                   // 128 rows of 64 elements
    static constexpr int kTileBytes = kHalves * kHalfBytes;          // a tile of keys, of values, or of queries
    static constexpr int kKeyStages = D == 64 ? 4 : 2, kValueStages = D == 64 ? 4 : 2;   // powers of two
    static constexpr int kStaging = 2 * kHalfBytes;                  // outputs leave through 16 KB of each group
    static constexpr int kSmem = (2 + kKeyStages + kValueStages) * kTileBytes + kStaging + 1024;  // (1024: alignment)
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

// What the host knows of the work.  A block of rows costs kBlockCost, kMaskedCost for every tile of keys that not all of its rows see
// whole, and AttRows::tile_cost for every tile; the CTAs share the sum of the costs evenly.
//   Measured, in units of 0.4 us: a tile of one tile of rows is what its bytes take (1.5 us; half of that for heads of 64), with two it is
// their exponentials (2.4 us); the turnover between pieces 3 us; a masked tile 3 us more.  (Without the difference: the prompt's chunk
// 198 us and not 149, 64 sequences of 31 nodes 153 and not 137.)
constexpr int kBlockCost = 8, kMaskedCost = 8;
constexpr int tile_cost(int head_dim, bool two) { return two ? 6 : head_dim == 64 ? 3 : 4; }

// Rows in tiles.  A tile is `nodes` nodes (all query heads of a cache head), at most 128 rows.  `parts` tiles follow each other within
// `period` nodes, then the next period begins: the nodes of one sequence, or (parts = 1, period = nodes) of the batch as it goes on.
struct AttRows {
    int nodes, parts, period, tiles, blocks;   // blocks of two tiles, per cache head
    int tile_cost;                             // of a tile of keys
    int slot_tiles, slot_rows;                 // of a block in the workspace: tiles, and rows of each
    FastDiv by_nodes, by_period, by_parts;
};
struct AttPlan {
    AttRows own, shared;          // a sequence's rows; the batch's
    int shared_tiles, grid;       // tiles of keys of the prefix
    int shared_cost;
    int64_t shared_slots;         // of the shared blocks' pieces, before those of the own: block + CTA is a piece's number
    bool merged;                  // the batch's nodes are one axis of the queries' shared tensor map, else sequences are its last
    FastDiv group, sequence;      // query heads per cache head; nodes per sequence
    int *before;                  // [batch + 1] cost of the own blocks before sequence b
    int *first;                   // [grid + 1] where each CTA's costs begin, and the sum of all
    int *error;                   // [grid]
    int4 *begin;                  // [grid] where each CTA's first piece is: sequence, head, block, first tile (0 also if it has none)
    int join_rows;                // rows of a tile that a warp joins
    float2 *ml;                   // (reference, sum) of every row of every slot
    float *o;                     // of every tile of a slot [head_dim / 32][rows][32], not divided by the sum; vectors of four swapped (row & 7)
};

struct AttKernelArgs {
    AttentionArgs a;
    AttPlan p;
};
struct AttMaps { CUtensorMap k, v, q, q_shared, out; };

__device__ __forceinline__ int own_end(const CacheArgs &c, int len) {   // keys of a sequence that is there
    const int64_t slots = static_cast<int64_t>(c.table_width) << c.page_shift;
    return static_cast<int>(min(static_cast<int64_t>(len) + c.nodes, slots));
}
__device__ __forceinline__ int own_tiles(const CacheArgs &c, int len) {
    return len < 0 ? 0 : static_cast<int>((static_cast<unsigned>(own_end(c, len)) + kTile - 1) / kTile);
}
// What precedes a block's tiles in the costs; the block's cost; and tiles that lie before `cost`, counted from the block's start.
__device__ __forceinline__ int head_cost(int plain, int tiles) { return kBlockCost + (tiles - plain / kTile) * kMaskedCost; }
__device__ __forceinline__ int block_cost(int head, int tiles, int tile_cost) { return tiles ? head + tiles * tile_cost : 0; }
__device__ __forceinline__ int tiles_before(int cost, int head, int tiles, int tile_cost) {
    return min(tiles, max(0, cost - head + tile_cost - 1) / tile_cost);
}
__device__ __forceinline__ int own_cost(const CacheArgs &c, const AttRows &r, int len) {
    const int tiles = own_tiles(c, len);
    return tiles ? block_cost(head_cost(min(len, own_end(c, len)), tiles), tiles, r.tile_cost) : 0;
}
// Blocks are numbered: all of the shared prefix, then sequence by sequence.  Of the whole cost `all`, CTA i takes [first(i), first(i + 1)).
__device__ __forceinline__ int split_first(int cta, int all, int grid) {
    const unsigned q = static_cast<unsigned>(all) / grid, r = static_cast<unsigned>(all) - q * grid;
    return cta * q + (cta * r + grid - 1) / grid;
}
// Consecutive tiles of keys for one block of rows.
struct AttPiece {
    bool shared, two;      // two: the block has two tiles of rows
    int b, head, block, t0, t1, tiles;
    int item;              // among the shared or among the own blocks
    int plain, keys;       // keys that every row sees; all keys
    __device__ bool masked(int t) const { return t >= plain / kTile; }
};

// The pieces of a CTA's run, one after the other (warp 8 does this and tells the others).
struct AttStart { int from, to, at; bool shared; int b, head, block; };   // costs; `at`: where the block begins
struct AttWalk {
    const CacheArgs &c;
    const AttPlan &p;
    int shared_len, from, to, at, b, head, block, len, next_len, tiles;
    bool shared;

    __device__ AttWalk(const AttKernelArgs &K, const AttStart &s)
        : c(K.a.c), p(K.p), shared_len(K.a.shared_len), from(s.from), to(s.to), at(s.at), b(s.b), head(s.head), block(s.block), len(0), shared(s.shared) {
        next_len = at < to ? c.lens[b] : -1;
        if (shared) tiles = p.shared_tiles;
        else look();
    }
    __device__ void look() {   // the next sequence that is there
        tiles = 0;
        if (at >= to) return;
        for (; b < c.batch; ++b) {
            len = next_len;
            next_len = b + 1 < c.batch ? c.lens[b + 1] : -1;
            tiles = own_tiles(c, len);
            if (tiles) break;
        }
    }
    __device__ bool next(AttPiece &x) {
        while (at < to && tiles) {
            const AttRows &r = shared ? p.shared : p.own;
            x.shared = shared;
            x.head = head;
            x.block = block;
            x.tiles = tiles;
            x.two = 2 * block + 1 < r.tiles;
            x.b = shared ? 0 : b;
            x.item = (x.b * c.kv_heads + head) * r.blocks + block;
            x.keys = shared ? shared_len : own_end(c, len);
            x.plain = shared ? shared_len : min(len, x.keys);
            const int ahead = head_cost(x.plain, tiles);
            x.t0 = from > at ? tiles_before(from - at, ahead, tiles, r.tile_cost) : 0;
            x.t1 = tiles_before(to - at, ahead, tiles, r.tile_cost);
            at += block_cost(ahead, tiles, r.tile_cost);
            if (++block == r.blocks) {
                block = 0;
                if (++head == c.kv_heads) {
                    head = 0;
                    if (shared) shared = false;   // (b is the first)
                    else ++b;
                    look();
                }
            }
            if (x.t1 > x.t0) return true;
        }
        return false;
    }
};

// Where a tile of rows begins: node among those of the batch (shared) or of the sequence, and its nodes.
struct AttTile { int node, count; };
__device__ __forceinline__ AttTile tile_of(const AttKernelArgs &K, bool shared, int tile) {
    const CacheArgs &c = K.a.c;
    const AttRows &r = shared ? K.p.shared : K.p.own;
    const int period = r.parts == 1 ? tile : r.by_parts.quot(tile), part = tile - period * r.parts;
    AttTile o;
    o.node = period * r.period + part * r.nodes;
    o.count = min(r.nodes, min((period + 1) * r.period, shared ? c.batch * c.nodes : c.nodes) - o.node);
    return o;
}

// Bits of the keys of a masked tile that a row sees (bit j of word w: key 128 t + 32 w + j).
__device__ __noinline__ uint4 row_bits(const AttentionArgs &A, const AttPiece &x, int t, int n) {
    uint32_t bits[4];
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
    return make_uint4(bits[0], bits[1], bits[2], bits[3]);
}

// A row's scores that it does not see, in tensor memory: -inf.
__device__ __noinline__ void mask_scores(uint32_t t_s, uint4 bits) {
#pragma unroll 1
    for (int h = 0; h < 4; ++h) {
        float s[32];
        tmem_ld32(t_s + 32 * h, s);
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i] = bits.x >> i & 1 ? s[i] : neg_inf();
        tmem_st32(t_s + 32 * h, s);
        bits = make_uint4(bits.y, bits.z, bits.w, 0);
    }
    tmem_wait_st();
}

// A row's new reference, where the weights of kStep scores are too large for the one it has, or it has none yet; and what that multiplies its
// sum, its `there` weights of the tile (t_p) and its O (t_o) by.  The latter two are done here.  A power of two: weights stay as they were
// rounded, but for those that become too small for fp16, 2^-31 of the largest.
constexpr uint32_t kNone = ~0u;
template <class T, int D>
__device__ __noinline__ float2 raise_reference(uint32_t t_s, uint32_t t_p, int there, uint32_t t_o, float cs, float ref, bool needed) {
    float top = neg_inf();
#pragma unroll 1
    for (int i = 0; i < kStep; i += 32) {
        float s[32];
        tmem_ld32(t_s + i, s);
#pragma unroll
        for (int j = 0; j < 32; j += 2) top = max3(top, s[j], s[j + 1]);
    }
    top = top * cs - Weight<T>::kBias;
    const float up = needed ? fmaxf(0.f, ceilf(top - ref)) : 0.f;   // (a row is what it is whichever rows are in its warp)
    const float now = ref == neg_inf() ? top : ref + up, f = ref == neg_inf() ? 1.f : up < 126.f ? __int_as_float((127 - static_cast<int>(up)) << 23) : 0.f;
    if (t_p != kNone) {
        tmem_wait_st();
#pragma unroll 1
        for (int i = 0; i < there; i += 8) {
            float w[8];
            tmem_ld8(t_p + i, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 e = unpack2<T>(__float_as_uint(w[j]));
                w[j] = __uint_as_float(pack2<T>(e.x * f, e.y * f));
            }
            tmem_st8(t_p + i, w);
        }
    }
    if (t_o != kNone)   // (the product that added the last tile to O is done: it was issued before these scores)
#pragma unroll 1
        for (int i = 0; i < D; i += 8) {
            float o[8];
            tmem_ld8(t_o + i, o);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] *= f;
            tmem_st8(t_o + i, o);
        }
    tmem_wait_st();
    return make_float2(now, f);
}

template <class T> __device__ __forceinline__ bool not_finite(uint16_t e);
template <> __device__ __forceinline__ bool not_finite<__nv_bfloat16>(uint16_t e) { return (e & 0x7f80) == 0x7f80; }
template <> __device__ __forceinline__ bool not_finite<__half>(uint16_t e) { return (e & 0x7c00) == 0x7c00; }

__device__ __forceinline__ void st_shared(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

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

// A tile of values in shared memory, looked through by 128 threads: rows from r1 become zero, and in rows r0..r1 what is no finite number.
// *found is set then, before the place is cleared: the other group may look at the place afterwards, and finds nothing there.
template <class T, int D>
__device__ __noinline__ void clear_values(uint8_t *v, int thread, int r0, int r1, volatile int *found) {
    constexpr int kVecs = D / 8;
    constexpr uint32_t kExp = Weight<T>::kBf16 ? 0x7f807f80u : 0x7c007c00u;   // all ones: no finite number
    const auto place = [&](int i) { return reinterpret_cast<uint4 *>(v + (i % kVecs / 8) * (kTile * 128) + (i / kVecs) * 128 + (i % 8) * 16); };
    for (int i = thread + r1 * kVecs; i < kTile * kVecs; i += kTile) *place(i) = make_uint4(0, 0, 0, 0);
#pragma unroll 4
    for (int i = thread + r0 * kVecs; i < r1 * kVecs; i += kTile) {
        uint4 u = *place(i);
        uint32_t most = __vimax3_u16x2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu, u.z & 0x7fff7fffu);   // magnitudes as numbers of 15 bits
        most = __vmaxu2(most, u.w & 0x7fff7fffu);
        if ((most & 0xffffu) < (kExp & 0xffffu) && most >> 16 < kExp >> 16) continue;
        uint32_t *w = &u.x;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if ((w[k] & kExp & 0xffffu) == (kExp & 0xffffu)) w[k] &= 0xffff0000u;
            if ((w[k] & kExp & 0xffff0000u) == (kExp & 0xffff0000u)) w[k] &= 0xffffu;
        }
        *found = 1;
        __threadfence_block();
        *place(i) = u;
    }
}

template <class T, int D>
__global__ void __launch_bounds__(kAttThreads, 1) attention_kernel(const __grid_constant__ AttKernelArgs K, const __grid_constant__ AttMaps maps) {
    using L = AttShape<D>;
    constexpr bool kBf16 = Weight<T>::kBf16;
    constexpr int SK = L::kKeyStages, SV = L::kValueStages;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * (SK + SV) + 16 + 2 * kPieces];
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up_, bad_values;
    __shared__ float2 other[kTile];           // of each row: (reference, sum) of group 1, then both groups' factors
    __shared__ int warp_sum[kAttThreads / 32];
    __shared__ AttStart start;
    __shared__ AttPiece pieces[kPieces];      // the next ones; t1 = 0: there are no more
    volatile int *const gave_up = &gave_up_;

    const AttentionArgs &A = K.a;
    const CacheArgs &c = A.c;
    const AttPlan &P = K.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t *const smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t s_q = saddr(smem), s_k = s_q + 2 * L::kTileBytes, s_v = s_k + SK * L::kTileBytes, s_out = s_v + SV * L::kTileBytes, bar0 = saddr(bars);
    const auto k_full = [&](int s) { return bar0 + 8u * s; };
    const auto k_empty = [&](int s) { return bar0 + 8u * (SK + s); };
    const auto v_full = [&](int s) { return bar0 + 8u * (2 * SK + s); };
    const auto v_empty = [&](int s) { return bar0 + 8u * (2 * SK + SV + s); };
    const uint32_t bar1 = bar0 + 16u * (SK + SV);
    const auto q_full = [&](int q) { return bar1 + 8u * q; };
    const auto q_empty = [&](int q) { return bar1 + 16u + 8u * q; };
    const auto s_full = [&](int t) { return bar1 + 32u + 8u * t; };
    const auto p_full = [&](int t) { return bar1 + 48u + 8u * t; };
    const auto o_full = [&](int t) { return bar1 + 64u + 8u * t; };
    const uint32_t o_free = bar1 + 80u;
    const auto meet = [&](int i) { return bar1 + 88u + 8u * i; };   // of softmax warps: of all, of either group
    const auto turn = [&](int t) { return bar1 + 112u + 8u * t; };   // at the tensor core
    const auto piece_full = [&](int i) { return bar1 + 128u + 8u * i; };
    const auto piece_empty = [&](int i) { return bar1 + 128u + 8u * (kPieces + i); };

    if (warp == 9) tmem_alloc(saddr(&tmem_base), 512);
    if (tid == 0) {
        for (int s = 0; s < SK; ++s) { bar_init(k_full(s), 1); bar_init(k_empty(s), 2); }
        for (int s = 0; s < SV; ++s) { bar_init(v_full(s), 1); bar_init(v_empty(s), 2); }
        for (int t = 0; t < 2; ++t) {
            bar_init(q_full(t), 1); bar_init(q_empty(t), 2);
            bar_init(s_full(t), 1); bar_init(p_full(t), 4); bar_init(o_full(t), 1);
            bar_init(turn(t), 1);
        }
        bar_init(o_free, 8);
        bar_init(meet(0), 8);
        bar_init(meet(1), 4);
        bar_init(meet(2), 4);
        for (int i = 0; i < kPieces; ++i) { bar_init(piece_full(i), 1); bar_init(piece_empty(i), kPieceReaders); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        gave_up_ = 0;
        bad_values = 0;
        tma_prefetch_map(&maps.k);
        tma_prefetch_map(&maps.v);
        tma_prefetch_map(&maps.q);
    }
    // The tensor core multiplies rows that are not there too, and what long runs of calls take goes by the power limit: such rows of the
    // queries and of the weights are zeros (64 sequences of one node 261 -> 233 us, two of 15 nodes 206 -> 199, in loops of seconds).
    for (int i = tid; i < 2 * L::kTileBytes / 16; i += kAttThreads) st_shared(s_q + 16 * i, 0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    pdl_begin();

    // This CTA's run: own costs of all sequences summed up, in the order of the sequences.
    {
        const int per = (c.batch + kAttThreads - 1) / kAttThreads, b0 = min(c.batch, tid * per), b1 = min(c.batch, b0 + per);
        const int per_b = c.kv_heads * P.own.blocks;
        int last = 0, mine = 0;   // of the thread's only or last sequence
        for (int b = b0; b < b1; ++b) {
            last = own_cost(c, P.own, c.lens[b]);
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
            const int each = block_cost(head_cost(A.shared_len, P.shared_tiles), P.shared_tiles, P.shared.tile_cost), item = from / each;
            start = AttStart{from, to, item * each, true, 0, item / P.shared.blocks, item % P.shared.blocks};
        }
        if (here && from < to) {
            int b = b0;
            if (per > 1)
                for (; b < b1; ++b) {
                    last = own_cost(c, P.own, c.lens[b]);
                    if (from < before + last * per_b) break;
                    before += last * per_b;
                }
            const int in_b = (from - before) / last;
            start = AttStart{from, to, before + in_b * last, false, b, in_b / P.own.blocks, in_b % P.own.blocks};
        }
        // for the kernel that joins
        if (tid == 0) {
            P.first[blockIdx.x] = from;
            if (blockIdx.x == gridDim.x - 1) P.first[gridDim.x] = all;
        }
        if (blockIdx.x == 0 && b0 < b1) {
            before = upto - mine;
            for (int b = b0; b < b1; ++b) {
                P.before[b] = before;
                before += own_cost(c, P.own, c.lens[b]) * per_b;
            }
            if (b1 == c.batch) P.before[c.batch] = before;
        }
        tmem_fence_before();
        __syncthreads();
        tmem_fence_after();
    }
    const uint32_t tm = tmem_base;
    AttPiece x = {};
    int piece_slot = 0;
    uint32_t piece_phase = 0;
    const auto next_piece = [&](AttPiece &y) {   // one arrival per reader: a warp, or a thread of warps 9 and 10
        bar_wait_one(piece_full(piece_slot), piece_phase, gave_up);
        y = pieces[piece_slot];
        if (warp < 8 || warp == 11) __syncwarp();
        if (lane == 0) bar_arrive(piece_empty(piece_slot));
        if (++piece_slot == kPieces) { piece_slot = 0; piece_phase ^= 1u; }
        return y.t1 > 0 && *gave_up == 0;
    };

    if (warp < 8) {
        // ---- softmax ---------------------------------------------------------------------------------
        more_registers<kSoftmaxRegs>();
        const int g = warp >> 2, gt = tid & (kTile - 1);
        const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
        const uint32_t t_s = tm + lanes + L::kS + g * kTile, t_p = tm + lanes + L::kP + g * L::kPStep, t_o = tm + lanes + L::kO;
        uint32_t s_phase = 0, o_phase = 0, meet_phase[2] = {0, 0};
        const auto together = [&](bool all) {   // (with an end, unlike the hardware's barriers: a warp may have given up)
            __syncwarp();
            const uint32_t bar = meet(all ? 0 : 1 + g);
            if (lane == 0) bar_arrive(bar);
            bar_wait(bar, meet_phase[all], gave_up);
            meet_phase[all] ^= 1u;
        };
        if (D == 64) {   // (else the weights take the place of scores, which are zeros there)
            const float none[32] = {};
            tmem_st32(t_p, none);
            tmem_st32(t_p + 32, none);
            tmem_wait_st();
            tmem_fence_before();
        }
        const float cs = A.scale_log2;
        float ref = neg_inf(), sum = 0.f;
        const auto raise = [&](int h, bool first, bool needed) {   // (where `needed` or it has none)
            const float2 r = raise_reference<T, D>(t_s + kStep * h, h ? t_p : kNone, kStep / 2 * h, first ? kNone : t_o + g * D, cs, ref, needed);
            ref = r.x;
            sum *= r.y;
        };
        uint32_t n0 = 0;   // tiles of values before this piece
        bool there = next_piece(x);
        while (there) {
            const int tile = 2 * x.block + (x.two ? g : 0);
            const AttTile rows = tile_of(K, x.shared, tile);
            const int valid = rows.count * P.group.d, in = P.group.quot(gt);   // rows of the tile; the row's node
            const bool warp_on = gt - lane < valid, mine = gt < valid;           // any row in this warp
            ref = neg_inf();
            sum = 0.f;
            const int step = x.two ? 1 : 2, first = x.two ? x.t0 : x.t0 + g;
            for (int t = first; t < x.t1; t += step) {
                const bool masked = x.masked(t);
                uint4 bits = {};
                if (masked && warp_on) bits = row_bits(A, x, t, x.shared ? 0 : rows.node + min(in, rows.count - 1));
                bar_wait(s_full(g), s_phase, gave_up);
                s_phase ^= 1u;
                tmem_fence_after();
                if (warp_on) {
                    // A loop, and what is rare in functions: the warps wait less for their code (all 128 scores in one stretch of code and in
                    // registers: 502 us instead of 372 for 64 x 31 nodes behind 8192 shared tokens).  With a pass of its own for each tile's
                    // maximum 350 us, without 339.  Exponentials by a polynomial, for a part of them, bring nothing here.
                    if (masked) mask_scores(t_s, bits);
#pragma unroll 1
                    for (int h = 0; h < kTile / kStep; ++h) {
                        if (__any_sync(kFull, mine && ref == neg_inf())) raise(h, t == first, false);
                        uint32_t w[kStep / 2];
                        float l;
#pragma unroll 1
                        for (int tries = 0; tries < 2; ++tries) {
                            const float sub = !mine ? neg_inf() : ref == neg_inf() ? 0.f : -ref;
                            const float2 sub2 = make_float2(sub, sub), cs2 = make_float2(cs, cs);
                            float2 l0 = make_float2(0.f, 0.f), l1 = l0;
                            float s[kStep];
#pragma unroll
                            for (int i = 0; i < kStep; i += 32) tmem_ld32_async(t_s + kStep * h + i, s + i);
                            tmem_wait_ld(s);
#pragma unroll
                            for (int i = 0; i < kStep / 2; ++i) {
                                const float2 a = fma2(make_float2(s[2 * i], s[2 * i + 1]), cs2, sub2);
                                const float2 e = make_float2(ex2(a.x), ex2(a.y));
                                if (i & 1) l1 = add2(l1, e);
                                else l0 = add2(l0, e);
                                w[i] = pack2<T>(e.x, e.y);
                            }
                            l = (l0.x + l0.y) + (l1.x + l1.y);
                            if (!__any_sync(kFull, l > kMostSum)) break;
                            raise(h, t == first, l > kMostSum);
                        }
                        sum += l;
#pragma unroll
                        for (int i = 0; i < kStep / 2; i += 16) tmem_st16_async(t_p + kStep / 2 * h + i, w + i);   // (over scores that have been read)
                    }
                    tmem_wait_st();
                    tmem_fence_before();
                }
                if (masked) {
                    // Values behind the end, and those of tree nodes that are no numbers: zero.  (Both groups do it where both have the tile;
                    // the ring is neither before nor behind this place: these scores came after the last products, these weights are waited for.)
                    const uint32_t n = n0 + t - x.t0;
                    bar_wait(v_full(n % SV), n / SV & 1u, gave_up);
                    // (From here on the CTA looks for such nodes.  Both groups' rows do: who finds a place cleared sees the flag behind this fence.)
                    clear_values<T, D>(smem + (2 + SK + n % SV) * L::kTileBytes, gt, max(0, x.plain - t * kTile), min(kTile, x.keys - t * kTile), &bad_values);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __threadfence_block();
                }
                __syncwarp();
                if (lane == 0) bar_arrive(p_full(g));
            }
            // ---- the end of the piece ------------------------------------------------------------------
            AttPiece y = {};
            there = next_piece(y);   // (while the last product runs)
            bar_wait(o_full(g), o_phase, gave_up);
            o_phase ^= 1u;
            const bool whole = !x.shared && P.shared_tiles == 0 && x.t1 - x.t0 == x.tiles;
            const bool join = !x.two && x.t1 - x.t0 > 1;   // of both groups
            float f0 = 1.f, f1 = 0.f;                      // factors of O: of group 0 (a group's own where it is alone), of group 1
            if (!x.two) {   // the groups have the same rows, and each writes half of the columns
                if (g == 1) other[gt] = make_float2(ref, sum);
                tmem_fence_before();
                together(true);
                if (g == 0 && join) {
                    const float2 z = other[gt];
                    const float both = fmaxf(ref, z.x), r = both == neg_inf() ? 0.f : both;
                    f0 = ex2(ref - r); f1 = ex2(z.x - r);
                    sum = sum * f0 + z.y * f1;
                    ref = both;
                }
            }
            const bool none = sum == 0.f;
            if (whole) {
                const float inv = none ? 0.f : 1.f / sum;
                f0 *= inv; f1 *= inv;
            }
            if (!x.two) {
                if (g == 0) other[gt] = make_float2(f0, f1);
                together(true);
                if (g == 1) { const float2 z = other[gt]; f0 = z.x; f1 = z.y; }
            }
            tmem_fence_after();
            const uint32_t o0 = t_o + (x.two ? g * D : 0);
            const int col0 = x.two ? 0 : g * (D / 2), col1 = x.two ? D : col0 + D / 2;
            // 64 columns of a finished tile are in shared memory: on their way
            const auto half_done = [&](int half) {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                const bool both = D == 64 && !x.two;   // (each group has 32 of them)
                together(both);
                if (lane == 0 && (warp & 3) == 0 && !(both && g)) {
                    tma_store(&maps.out, s_out + (both ? 0 : g * L::kHalfBytes), 64 * half, x.head * P.group.d, rows.node, x.b);
                    store_commit();
                    store_wait_read();
                }
                if (x.two && half == 0 && D == 128) together(false);   // (the second half goes the same way)
            };
            if (warp_on) {
                const int bad = *static_cast<volatile int *>(&bad_values);
                const AttRows &r = x.shared ? P.shared : P.own;
                int64_t row0 = 0;   // in the workspace
                if (!whole) {
                    const int64_t slot = P.shared_tiles ? x.item + int64_t(blockIdx.x) : 2 * blockIdx.x + (x.t0 == 0);
                    row0 = (slot * r.slot_tiles + (x.two ? g : 0)) * r.slot_rows + (x.shared ? 0 : P.shared_slots * P.shared.slot_tiles * P.shared.slot_rows);
                    if (mine && (x.two || g == 0)) P.ml[row0 + gt] = make_float2(ref, sum);
                } else if (mine && A.lse && (x.two || g == 0)) {
                    A.lse[(static_cast<int64_t>(x.b) * c.nodes + rows.node + in) * c.heads + x.head * P.group.d + (gt - in * P.group.d)] =
                        none ? neg_inf() : (ref + log2f(sum)) * 0.6931471805599453f;
                }
                // 16 KB of staging per group: 64 columns of a tile as its type, or 4 KB of each warp
                const uint32_t half_at = s_out + (D == 64 && !x.two ? 0 : g * L::kHalfBytes), own_at = s_out + 4096 * warp;
                const uint32_t lane_rows = min(32, valid - (gt - lane));
#pragma unroll 1
                for (int i = col0; i < col1; i += 32) {
                    float o[32];
                    tmem_ld32(o0 + i, o);
#pragma unroll
                    for (int j = 0; j < 32; ++j) o[j] *= f0;
                    if (join) {
                        float z[32];
                        tmem_ld32(t_o + D + i, z);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = fmaf(z[j], f1, o[j]);
                    }
                    if (bad && !x.shared && mine) {
                        float z[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) z[j] = o[j];
                        add_not_finite<T>(A, x, rows.node + in, i, z);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = z[j];
                    }
                    __syncwarp();
                    if (whole) {
                        const uint32_t at = half_at + gt * 128;
                        if ((i & 32) == 0 && i > col0) half_done(i / 64 - 1);   // (a group that is alone: its first half goes before)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float *y8 = o + 8 * j;
                            st_shared(at + (((i & 32) / 8 + j) ^ (gt & 7)) * 16, pack2<T>(y8[0], y8[1]), pack2<T>(y8[2], y8[3]),
                                      pack2<T>(y8[4], y8[5]), pack2<T>(y8[6], y8[7]));
                        }
                    } else {
                        if (lane == 0) store_wait_read();
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            st_shared(own_at + lane * 128 + (j ^ (lane & 7)) * 16, __float_as_uint(o[4 * j]), __float_as_uint(o[4 * j + 1]), __float_as_uint(o[4 * j + 2]),
                                      __float_as_uint(o[4 * j + 3]));
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            bulk_store(P.o + row0 * D + (i / 32) * int64_t(r.slot_rows) * 32 + (gt - lane) * 32, own_at, lane_rows * 128);
                            store_commit();
                        }
                    }
                }
            } else if (whole && x.two && D == 128) half_done(0);
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(o_free);
            if (whole) half_done(x.two ? L::kHalves - 1 : D == 64 ? 0 : g);
            // Copies to the workspace have read their staging before the warp goes on: the next piece's outputs, those of other warps too, may
            // take its place (they are written behind barriers of the next piece at which this warp arrives).
            else if (lane == 0) store_wait_read();
            n0 += x.t1 - x.t0;
            x = y;
        }
        if (lane == 0) store_wait();
    } else if (fewer_registers<kOtherRegs>(), warp == 9 || warp == 10) {
        // ---- matrix instructions of a group: one thread ---------------------------------------------------
        if (lane == 0) {
            const int g = warp - 9;
            uint32_t k_n = 0, v_n = 0, q_n = 0;   // tiles and slots gone by
            uint32_t p_phase = 0, free_phase = 1, turn_phase = g == 0;
            constexpr uint32_t desc_s = mma_desc(kBf16, kTile, false), desc_o = mma_desc(kBf16, D, true);
            const uint32_t k_op = operand(s_k, L::kHalfBytes), v_op = operand(s_v, L::kHalfBytes), q_op = operand(s_q, L::kHalfBytes);
            const uint32_t d_s = tm + L::kS + g * kTile, d_o = tm + L::kO + g * D, a_p = tm + L::kP + g * L::kPStep;
            const auto k_arrived = [&]() { bar_wait_one(k_full(k_n % SK), k_n / SK & 1u, gave_up); };
            const auto v_arrived = [&]() { bar_wait_one(v_full(v_n % SV), v_n / SV & 1u, gave_up); };
            // tiles that are the other group's: both say when they have passed one, or a wait could take one time round the ring for another
            const auto pass_k = [&](int upto) {
                for (; static_cast<int>(k_n) < upto; ++k_n) { k_arrived(); bar_arrive(k_empty(k_n % SK)); }
            };
            const auto pass_v = [&](int upto) {
                for (; static_cast<int>(v_n) < upto; ++v_n) { v_arrived(); bar_arrive(v_empty(v_n % SV)); }
            };
            int n0 = 0;   // tiles before this piece
            while (next_piece(x)) {
                const int n = x.t1 - x.t0, step = x.two ? 1 : 2, first = x.two ? 0 : g;
                const uint32_t q = q_n + (x.two ? g : 0);   // the slot of queries
                q_n += x.two ? 2 : 1;
                bar_wait_one(q_full(q & 1u), q / 2 & 1u, gave_up);   // (not the other group's: that may be two rounds on)
                // Two tiles of rows: the groups' products and scores go in turns, whole.  Mixed, both would be done at the same time, and
                // both groups would then compute their weights at the same time, and the tensor core would wait for both (5400 clocks
                // for a tile of keys; in turns 4100).
                const auto my_turn = [&]() {
                    if (!x.two) return;
                    bar_wait_one(turn(g), turn_phase, gave_up);
                    turn_phase ^= 1u;
                };
                for (int i = first - step; i < n; i += step) {
                    const bool now = i >= first, more = i + step < n;
                    if (now) {
                        pass_v(n0 + i);
                        v_arrived();
                        if (i == first) bar_wait_one(o_free, free_phase, gave_up);   // O of the piece before has been read by now or soon
                    }
                    const uint32_t v_slot = v_n % SV;
                    if (more) pass_k(n0 + i + step);
                    if (more && (x.two || !now)) k_arrived();   // (else the products first: these keys may still be on their way)
                    if (now) {   // O (+)= P V
                        const uint32_t b = v_op + v_slot * (L::kTileBytes >> 4);
                        const bool add = i > first;
                        my_turn();
                        bar_wait_one(p_full(g), p_phase, gave_up);
                        p_phase ^= 1u;
                        tmem_fence_after();
#pragma unroll
                        for (int k = 0; k < kTile / 16; ++k) mma_ts(d_o, a_p + 8 * k, b + k * (2048 >> 4), desc_o, add || k > 0);
                        ++v_n;
                        if (!x.two) mma_commit(v_empty(v_slot));
                    } else my_turn();
                    if (more) {   // S = Q K^T
                        if (now && !x.two) k_arrived();
                        const uint32_t k_slot = k_n % SK, a = q_op + (q & 1u) * (L::kTileBytes >> 4), b = k_op + k_slot * (L::kTileBytes >> 4);
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint32_t off = ((k / 4) * L::kHalfBytes + (k % 4) * 32) >> 4;
                            mma_ss(d_s, a + off, b + off, desc_s, k > 0);
                        }
                        mma_commit(s_full(g));
                        if (x.two) bar_arrive(turn(1 - g));
                        mma_commit(k_empty(k_slot));
                        ++k_n;
                        if (i + 2 * step >= n) {   // the last ones
                            mma_commit(q_empty(q & 1u));
                            if (x.two) mma_commit(q_empty(q & 1u));
                        }
                    } else {
                        if (now) mma_commit(o_full(g));
                        if (x.two) bar_arrive(turn(1 - g));
                    }
                    if (now && x.two) mma_commit(v_empty(v_slot));
                }
                if (first >= n) {   // no tile for this group, but its part in the piece: else the others could be two pieces on
                    bar_arrive(q_empty(q & 1u));
                    bar_wait_one(o_free, free_phase, gave_up);
                    bar_arrive(o_full(g));
                }
                n0 += n;
                pass_k(n0);
                pass_v(n0);
                free_phase ^= 1u;
            }
            bar_wait_one(o_free, free_phase, gave_up);
        }
        __syncwarp();
    } else {
        // ---- tiles of keys, queries and pieces (warp 8); tiles of values (warp 11) ------------------------------
        const int ps = 1 << c.page_shift, box = min(ps, kTile), boxes = kTile / box;
        const auto page_at = [&](int t) -> int {   // lane i: the page of the tile's i-th box (c.pages: reads as zeros)
            const int slot = t * kTile + lane * box;
            if (lane >= boxes || t >= x.t1 || slot >= x.keys) return c.pages;
            const int at = slot >> c.page_shift;
            const int page = x.shared ? A.shared_table[at] : c.table[x.b * c.stride_table + at];   // (no key lies behind the table)
            return page >= 0 && page < c.pages ? page : c.pages;
        };
        const auto bring = [&](const CUtensorMap *map, int t, int page, uint32_t dst, uint32_t full) {
            if (lane == 0) bar_expect(full, L::kTileBytes);
            __syncwarp();
            if (lane < boxes) {
                const int y = ps > kTile ? (t * kTile) & (ps - 1) : 0;
#pragma unroll
                for (int h = 0; h < L::kHalves; ++h) tma_load(dst + lane * box * 128 + h * L::kHalfBytes, map, 64 * h, y, x.head, page, full);
            }
            __syncwarp();
        };
        if (warp == 8) {
            AttWalk walk(K, start);
            uint32_t n = 0, q_n = 0;
            const auto publish = [&](AttPiece &y, bool there) {
                if (!there) y.t1 = 0;
                bar_wait(piece_empty(piece_slot), piece_phase ^ 1u, gave_up);
                if (lane == 0) {
                    pieces[piece_slot] = y;
                    bar_arrive(piece_full(piece_slot));
                }
                if (++piece_slot == kPieces) { piece_slot = 0; piece_phase ^= 1u; }
            };
            bool there = walk.next(x);
            if (lane == 0) P.begin[blockIdx.x] = make_int4(x.b, x.head, x.block, there && !x.shared ? x.t0 : 0);
            publish(x, there);
            while (there && *gave_up == 0) {
                AttPiece y = {};
                bool then = false;
                int page = page_at(x.t0);
                for (int t = x.t0; t < x.t1; ++t, ++n) {
                    const int next = page_at(t + 1);
                    bar_wait(k_empty(n % SK), (n / SK & 1u) ^ 1u, gave_up);
                    bring(&maps.k, t, page, s_k + n % SK * L::kTileBytes, k_full(n % SK));
                    page = next;
                    if (t != x.t0) continue;
                    // behind the first keys: the queries (a slot may not be free yet), and the piece after this one
                    for (int i = 0; i < (x.two ? 2 : 1); ++i, ++q_n) {
                        const uint32_t slot = q_n & 1u;
                        bar_wait(q_empty(slot), (q_n / 2 & 1u) ^ 1u, gave_up);
                        if (lane == 0) {
                            const AttRows &r = x.shared ? P.shared : P.own;
                            const AttTile o = tile_of(K, x.shared, 2 * x.block + i);
                            int z = o.node, w = x.b;
                            if (x.shared) {
                                w = P.merged ? 0 : P.sequence.quot(o.node);
                                z = o.node - w * c.nodes;
                            }
                            bar_expect(q_full(slot), r.nodes * P.group.d * 2 * D);   // (what is out of range counts too)
                            for (int h = 0; h < L::kHalves; ++h)
                                tma_load(s_q + slot * L::kTileBytes + h * L::kHalfBytes, x.shared ? &maps.q_shared : &maps.q, 64 * h, x.head * P.group.d, z, w, q_full(slot));
                        }
                        __syncwarp();
                    }
                    then = walk.next(y);
                    publish(y, then);
                }
                x = y;
                there = then;
            }
            // the last arrivals come before the CTA ends
            for (int i = 0; i < SK; ++i, ++n) bar_wait(k_empty(n % SK), (n / SK & 1u) ^ 1u, gave_up);
            for (int i = 0; i < 2; ++i, ++q_n) bar_wait(q_empty(q_n & 1u), (q_n / 2 & 1u) ^ 1u, gave_up);
        } else {
            uint32_t n = 0;
            while (next_piece(x)) {
                int page = page_at(x.t0);
                for (int t = x.t0; t < x.t1; ++t, ++n) {
                    const int next = page_at(t + 1);
                    bar_wait(v_empty(n % SV), (n / SV & 1u) ^ 1u, gave_up);
                    bring(&maps.v, t, page, s_v + n % SV * L::kTileBytes, v_full(n % SV));
                    page = next;
                }
            }
            for (int i = 0; i < SV; ++i, ++n) bar_wait(v_empty(n % SV), (n / SV & 1u) ^ 1u, gave_up);
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

constexpr int kJoinThreads = 256, kJoinAtOnce = 4;

// Joins the pieces of the blocks that have more than one, P.join_rows rows of a tile per warp; and finds bad pages (the first `batch` CTAs,
// if wanted).  Where there is a prefix that is all blocks; where there is none, it is those that some CTA begins in the middle of,
// found from that CTA.  What bounds it is the chain of loads: where the pieces are, then their rows, kJoinAtOnce at a time.
template <class T, int D>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const __grid_constant__ AttKernelArgs K) {
    constexpr int E = D / 32;
    pdl_begin();
    const AttentionArgs &A = K.a;
    const CacheArgs &c = A.c;
    const AttPlan &P = K.p;
    const int tid = threadIdx.x, lane = tid & 31;
    int task = blockIdx.x;
    if (c.status) {
        if (task < c.batch) {
            const int b = task, ps = 1 << c.page_shift, len = c.lens[b];
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
        task -= c.batch;
    }
    task = task * (kJoinThreads / 32) + (tid >> 5);
    const int chunks = (P.own.slot_rows + P.join_rows - 1) / P.join_rows, chunk = task % chunks;   // of a tile of rows
    task /= chunks;
    const int tb = task % P.own.slot_tiles;
    task /= P.own.slot_tiles;
    int b, hk, block;
    if (P.shared_tiles) {
        const int per_b = c.kv_heads * P.own.blocks;
        b = task / per_b;
        hk = (task - b * per_b) / P.own.blocks;
        block = task - b * per_b - hk * P.own.blocks;
        if (b >= c.batch) return;
    } else {
        if (task >= P.grid) return;
        const int4 at = P.begin[task];
        if (at.w == 0) return;
        b = at.x; hk = at.y; block = at.z;
    }
    const int tile = 2 * block + tb, len = c.lens[b];
    if (len < 0 || tile >= P.own.tiles) return;
    const AttTile t = tile_of(K, false, tile);
    const int row0 = chunk * P.join_rows, row1 = min(t.count * static_cast<int>(P.group.d), row0 + P.join_rows);
    if (row0 >= row1) return;
    const int tiles = own_tiles(c, len), own_head = head_cost(min(len, own_end(c, len)), tiles),
              own0 = P.before[b] + (hk * P.own.blocks + block) * block_cost(own_head, tiles, P.own.tile_cost), all = P.first[P.grid];
    if (!P.shared_tiles) {   // of the CTAs that begin within the block, the first one's task is this
        const int from = P.begin[task].w;
        int i = task - 1, before = 0;
        while (i > 0 && (before = tiles_before(P.first[i] - own0, own_head, tiles, P.own.tile_cost)) == from) --i;   // (a run can be too short for a tile)
        if (i > 0 && before > 0) return;
    }
    const int item = (b * c.kv_heads + hk) * P.own.blocks + block;
    const int step = P.own.slot_tiles * P.own.slot_rows, s_step = P.shared.slot_tiles * P.shared.slot_rows;
    const int64_t own_row = P.shared_slots * s_step + (P.shared_tiles ? static_cast<int64_t>(item) * step : 0) + tb * P.own.slot_rows;
    // the first CTA whose run may have tiles of a block whose costs begin at `at`
    const auto first_cta = [&](int at) {
        int i = min(P.grid - 1, at / max(1, all / P.grid));   // (not before the one that has cost `at`, and hardly behind it)
        while (i > 0 && P.first[i] > at) --i;
        return i;
    };
    const int own_cta = first_cta(own0);
    for (int row = row0; row < row1; ++row) {
        const int in = P.group.quot(row), n = t.node + in, h = hk * P.group.d + (row - in * P.group.d), col = lane * E;
        float ref = neg_inf(), sum = 0.f, o[E] = {};
        // The pieces of a block: of the CTAs from `cta`, a lane looks at each.  Their first rows in the workspace are row_0 + i * by, or where
        // there is no prefix, and a CTA has two pieces at most, row_0 + (2 i + (whether it is the block's first)) * by.
        const auto add = [&](int at, int head, int n_tiles, int tile_cost, int cta, int64_t row_0, int by, int rows_of, int r) {
            const float *src = P.o + row_0 * D + ((col / 32) * rows_of + r) * 32 + ((col % 32 / 4) ^ (r & 7)) * 4 + col % 4;
            const int end = at + block_cost(head, n_tiles, tile_cost);
            int begins = P.shared_tiles ? 0 : 1;
            for (; cta < P.grid; cta += 32) {
                const int i = cta + lane, from = i <= P.grid ? P.first[i] : 0x7fffffff, to = i < P.grid ? P.first[i + 1] : 0x7fffffff;
                const bool piece = i < P.grid && from < end && tiles_before(to - at, head, n_tiles, tile_cost) > tiles_before(from - at, head, n_tiles, tile_cost);
                unsigned left = __ballot_sync(kFull, piece);
                while (left) {
                    float z[kJoinAtOnce][E];
                    float2 ml[kJoinAtOnce];
#pragma unroll
                    for (int j = 0; j < kJoinAtOnce; ++j) {
                        ml[j] = make_float2(neg_inf(), 0.f);
#pragma unroll
                        for (int k = 0; k < E; ++k) z[j][k] = 0.f;
                        if (left) {
                            const int who = cta + __ffs(left) - 1;
                            const int64_t off = static_cast<int64_t>(P.shared_tiles ? who : 2 * who + begins) * by;
                            begins = 0;
                            ml[j] = P.ml[row_0 + off + r];
                            if (E == 4) { const float4 v = *reinterpret_cast<const float4 *>(src + off * D); z[j][0] = v.x; z[j][1] = v.y; z[j][E - 2] = v.z; z[j][E - 1] = v.w; }
                            else { const float2 v = *reinterpret_cast<const float2 *>(src + off * D); z[j][0] = v.x; z[j][1] = v.y; }
                            left &= left - 1;
                        }
                    }
                    float now = ref;
#pragma unroll
                    for (int j = 0; j < kJoinAtOnce; ++j) now = fmaxf(now, ml[j].x);
                    const float m = now == neg_inf() ? 0.f : now, f0 = ex2(ref - m);
                    sum *= f0;
#pragma unroll
                    for (int k = 0; k < E; ++k) o[k] *= f0;
#pragma unroll
                    for (int j = 0; j < kJoinAtOnce; ++j) {
                        const float f = ex2(ml[j].x - m);
                        sum = fmaf(ml[j].y, f, sum);
#pragma unroll
                        for (int k = 0; k < E; ++k) o[k] = fmaf(z[j][k], f, o[k]);
                    }
                    ref = now;
                }
                if (__any_sync(kFull, from >= end)) break;
            }
        };
        if (P.shared_tiles) {   // the row's place among those of the whole batch
            const AttRows &r = P.shared;
            const int node = b * c.nodes + n, period = r.by_period.quot(node), in_p = node - period * r.period, part = r.by_nodes.quot(in_p);
            const int s_tile = period * r.parts + part, s_row = (in_p - part * r.nodes) * P.group.d + (row - in * P.group.d);
            const int s_item = hk * r.blocks + s_tile / 2, s_head = head_cost(A.shared_len, P.shared_tiles);
            const int at = s_item * block_cost(s_head, P.shared_tiles, r.tile_cost);
            add(at, s_head, P.shared_tiles, r.tile_cost, first_cta(at), static_cast<int64_t>(s_item) * s_step + s_tile % 2 * r.slot_rows, s_step, r.slot_rows, s_row);
        }
        add(own0, own_head, tiles, P.own.tile_cost, own_cta, own_row, step, P.own.slot_rows, row);
        const bool none = sum == 0.f;
        const float inv = none ? 0.f : 1.f / sum;
        T *dst = static_cast<T *>(A.out.data) + b * A.out.seq + n * A.out.node + h * A.out.head + col;
        uint32_t w[E / 2];
#pragma unroll
        for (int k = 0; k < E; k += 2) w[k / 2] = pack2<T>(o[k] * inv, o[k + 1] * inv);
        if (E == 4) *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[E / 2 - 1]);
        else *reinterpret_cast<uint32_t *>(dst) = w[0];
        if (A.lse && lane == 0) A.lse[(int64_t(b) * c.nodes + n) * c.heads + h] = none ? neg_inf() : (ref + log2f(sum)) * 0.6931471805599453f;
    }
}

}  // namespace spechub
