// Attention of tree nodes over a paged cache: tensor maps, workspace, launches.
#include <algorithm>
#include <mutex>

#include "spechub_attention.cuh"
#include "spechub_cache_launch.h"

namespace spechub {

namespace {

using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                            const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode encoder() {
    static std::mutex mutex;
    static Encode found = nullptr;
    std::lock_guard<std::mutex> lock(mutex);
    if (!found) {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        found = reinterpret_cast<Encode>(f);
    }
    return found;
}

int encode_map(int dtype, void *data, const cuuint64_t (&dims)[4], const int64_t (&strides)[3], const cuuint32_t (&box)[4], CUtensorMap *map) {
    const Encode encode = encoder();
    if (!encode) return SPECHUB_ERR_LAUNCH;
    const cuuint64_t bytes[3] = {static_cast<cuuint64_t>(strides[0]) * 2, static_cast<cuuint64_t>(strides[1]) * 2, static_cast<cuuint64_t>(strides[2]) * 2};
    const cuuint32_t each[4] = {1, 1, 1, 1};
    const CUresult r = encode(map, dtype == SPECHUB_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, data, dims, bytes, box,
                              each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SPECHUB_OK : SPECHUB_ERR_ALIGN;
}

// (head_dim, token of a page, head, page), boxes of 64 dimensions of a page's tokens (128 of them at most)
int page_map(int dtype, const PagesPtr &x, const CacheArgs &c, CUtensorMap *map) {
    const cuuint32_t ps = 1u << c.page_shift;
    return encode_map(dtype, x.data, {static_cast<cuuint64_t>(c.head_dim), ps, static_cast<cuuint64_t>(c.kv_heads), static_cast<cuuint64_t>(c.pages)},
                      {x.token, x.head, x.page}, {64, ps < kTile ? ps : kTile, 1, 1}, map);
}

// (head_dim, head, node, sequence), boxes of 64 dimensions of a cache head's query heads of `nodes` nodes of `sequences` sequences
int heads_map(int dtype, const HeadsPtr &x, const CacheArgs &c, int64_t nodes_all, int64_t sequences_all, int nodes, int sequences, CUtensorMap *map) {
    return encode_map(dtype, x.data, {static_cast<cuuint64_t>(c.head_dim), static_cast<cuuint64_t>(c.heads), static_cast<cuuint64_t>(nodes_all),
                                      static_cast<cuuint64_t>(sequences_all)},
                      {x.head, x.node, x.seq}, {64, static_cast<cuuint32_t>(c.heads / c.kv_heads), static_cast<cuuint32_t>(nodes), static_cast<cuuint32_t>(sequences)}, map);
}

AttRows rows_of(int head_dim, int64_t group, int64_t nodes, int64_t period, int64_t all) {
    AttRows r = {};
    r.nodes = static_cast<int>(nodes);
    r.parts = static_cast<int>((period + nodes - 1) / nodes);
    r.period = static_cast<int>(period);
    r.tiles = static_cast<int>((all + period - 1) / period * r.parts);
    r.blocks = (r.tiles + 1) / 2;
    r.slot_tiles = r.tiles > 1 ? 2 : 1;
    r.tile_cost = tile_cost(head_dim, r.tiles > 1);
    r.slot_rows = static_cast<int>(nodes * group);
    r.by_nodes = FastDiv::of(static_cast<uint32_t>(nodes));
    r.by_period = FastDiv::of(static_cast<uint32_t>(period));
    r.by_parts = FastDiv::of(static_cast<uint32_t>(r.parts));
    return r;
}

constexpr double kMostCost = 2.0e9;   // of a call

size_t up(size_t n) { return (n + 255) & ~size_t(255); }

// The plan, and the workspace's size; its parts are at `base`.  false: costs are counted in 31 bits, and there may be more than that (by the
// shape alone, as the size: with either layout of the prefix's rows, every context as long as its table, every tile of keys masked).
bool plan_of(const CacheArgs &c, const HeadsPtr &q, int64_t shared_len, uint8_t *base, AttPlan *p, size_t *bytes) {
    const int64_t group = c.heads / c.kv_heads, most_nodes = kTile / group, all = static_cast<int64_t>(c.batch) * c.nodes;
    const int64_t own_nodes = c.nodes < most_nodes ? c.nodes : most_nodes;
    p->own = rows_of(c.head_dim, group, own_nodes, c.nodes, c.nodes);
    // Rows of the whole batch: tiles go on from one sequence to the next where one stride leads through all nodes; otherwise they hold as
    // many whole sequences as fit, or parts of one.  (The workspace has room for either.)
    p->merged = c.batch == 1 || c.nodes == 1 || q.seq == q.node * c.nodes;
    const int64_t merged_nodes = all < most_nodes ? all : most_nodes;
    const int64_t whole = most_nodes / c.nodes < c.batch ? most_nodes / c.nodes : c.batch;   // sequences in a tile
    const AttRows merged = rows_of(c.head_dim, group, merged_nodes, merged_nodes, all);
    const AttRows apart = whole >= 1 ? rows_of(c.head_dim, group, whole * c.nodes, whole * c.nodes, all) : rows_of(c.head_dim, group, own_nodes, c.nodes, all);
    p->shared = p->merged ? merged : apart;
    p->shared_tiles = static_cast<int>((shared_len + kTile - 1) / kTile);
    const int64_t own_items = static_cast<int64_t>(c.batch) * c.kv_heads * p->own.blocks;
    const int64_t shared_items = shared_len ? static_cast<int64_t>(c.kv_heads) * p->shared.blocks : 0;
    const int64_t own_tiles = ((static_cast<int64_t>(c.table_width) << c.page_shift) + kTile - 1) / kTile;   // of a sequence, at most
    const auto cost = [](const AttRows &r, double tiles) { return kBlockCost + tiles * (r.tile_cost + kMaskedCost); };
    const auto shared_most = [&](const AttRows &r) { return shared_len ? double(c.kv_heads) * r.blocks * cost(r, p->shared_tiles) : 0.; };
    const double own_most = double(own_items) * cost(p->own, double(own_tiles));
    if (std::max(shared_most(merged), shared_most(apart)) + own_most > kMostCost) return false;
    const int64_t masked = p->shared_tiles - shared_len / kTile;
    p->shared_cost = static_cast<int>(shared_items * (kBlockCost + masked * kMaskedCost + static_cast<int64_t>(p->shared.tile_cost) * p->shared_tiles));
    p->group = FastDiv::of(static_cast<uint32_t>(group));
    p->sequence = FastDiv::of(static_cast<uint32_t>(c.nodes));
    // as many CTAs as there can be tiles, at most one per SM
    const int64_t tiles = shared_items * p->shared_tiles + own_items * own_tiles;
    p->grid = static_cast<int>(tiles < kSms ? tiles : kSms);
    p->shared_slots = shared_len ? shared_items + p->grid : 0;
    const auto slot = [](const AttRows &r) { return static_cast<int64_t>(r.slot_tiles) * r.slot_rows; };
    const int64_t own_rows = (shared_len ? own_items + kSms : 2 * kSms) * slot(p->own);   // (without a prefix: a CTA's first and last pieces)
    const int64_t rows = p->shared_slots * slot(p->shared) + own_rows;
    // (the size goes by the shape alone, whichever strides the queries have)
    const auto shared_rows = [&](const AttRows &r) { return shared_len ? (static_cast<int64_t>(c.kv_heads) * r.blocks + kSms) * slot(r) : 0; };
    const int64_t room = own_rows + (shared_rows(merged) > shared_rows(apart) ? shared_rows(merged) : shared_rows(apart));
    // four rows for each warp that joins, or one where that leaves SMs idle
    p->join_rows = shared_len && own_items * c.nodes * group >= 4 * 32 * kSms ? 4 : 1;
    size_t at = 0;
    p->before = reinterpret_cast<int *>(base);
    at += up(sizeof(int) * (static_cast<size_t>(c.batch) + 1));
    p->first = reinterpret_cast<int *>(base + at);
    at += up(sizeof(int) * (kSms + 1));
    p->error = reinterpret_cast<int *>(base + at);
    at += up(sizeof(int) * kSms);
    p->begin = reinterpret_cast<int4 *>(base + at);
    at += up(sizeof(int4) * kSms);
    p->ml = reinterpret_cast<float2 *>(base + at);
    at += up(sizeof(float2) * static_cast<size_t>(rows));
    p->o = reinterpret_cast<float *>(base + at);
    *bytes = up(sizeof(int) * (static_cast<size_t>(c.batch) + 1)) + up(sizeof(int) * (kSms + 1)) + up(sizeof(int) * kSms) + up(sizeof(int4) * kSms) + up(sizeof(float2) * static_cast<size_t>(room)) +
             up(sizeof(float) * static_cast<size_t>(room) * c.head_dim);
    return true;
}

template <class T, int D>
int launch_type(const AttKernelArgs &k, const AttMaps &maps, cudaStream_t s) {
    static bool configured[kMaxDevices] = {};
    const int rc = allow_smem(reinterpret_cast<const void *>(attention_kernel<T, D>), AttShape<D>::kSmem, configured);
    if (rc != SPECHUB_OK) return rc;
    // the kernel's warps share out kLaunchRegs registers a thread: a build that gives it others must not run
    static int regs[kMaxDevices] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return SPECHUB_ERR_LAUNCH;
    if (regs[dev] == 0) {
        cudaFuncAttributes fa;
        if (cudaFuncGetAttributes(&fa, attention_kernel<T, D>) != cudaSuccess) { cudaGetLastError(); return SPECHUB_ERR_LAUNCH; }
        regs[dev] = fa.numRegs;
    }
    if (regs[dev] != kLaunchRegs) return SPECHUB_ERR_LAUNCH;
    const int lrc = launch_grid(attention_kernel<T, D>, k.p.grid, kAttThreads, AttShape<D>::kSmem, 1, s, k, maps);
    if (lrc != SPECHUB_OK) return lrc;
    const AttRows &r = k.p.own;
    const int64_t blocks = k.p.shared_tiles ? static_cast<int64_t>(k.a.c.batch) * k.a.c.kv_heads * r.blocks : k.p.grid;
    // (no more than there are rows, of which the host takes 31 bits)
    const int64_t tasks = blocks * r.slot_tiles * ((r.slot_rows + k.p.join_rows - 1) / k.p.join_rows), per = kJoinThreads / 32;
    const int64_t grid = (tasks + per - 1) / per + (k.a.c.status ? k.a.c.batch : 0);
    return launch_grid(attention_join_kernel<T, D>, static_cast<unsigned>(grid), kJoinThreads, 0, 1, s, k);
}

}  // namespace

bool attention_workspace(const CacheArgs &c, int64_t shared_len, size_t *bytes) {
    AttPlan p;
    return plan_of(c, HeadsPtr{}, shared_len, nullptr, &p, bytes);
}

int launch_attention(int dtype, const AttentionArgs &a, void *workspace, cudaStream_t s) {
    AttKernelArgs k;
    k.a = a;
    size_t bytes;
    if (!plan_of(a.c, a.q, a.shared_len, static_cast<uint8_t *>(workspace), &k.p, &bytes)) return SPECHUB_ERR_WORK;
    const CacheArgs &c = a.c;
    const AttRows &sh = k.p.shared;
    AttMaps maps;
    int rc = page_map(dtype, c.k, c, &maps.k);
    if (rc == SPECHUB_OK) rc = page_map(dtype, c.v, c, &maps.v);
    if (rc == SPECHUB_OK) rc = heads_map(dtype, a.q, c, c.nodes, c.batch, k.p.own.nodes, 1, &maps.q);
    if (rc == SPECHUB_OK) rc = heads_map(dtype, a.out, c, c.nodes, c.batch, k.p.own.nodes, 1, &maps.out);
    maps.q_shared = maps.q;
    if (rc == SPECHUB_OK && a.shared_len) {
        if (k.p.merged) {   // (one sequence, or one node each: the other's stride leads on)
            HeadsPtr q = a.q;
            if (c.nodes == 1) q.node = q.seq;
            rc = heads_map(dtype, q, c, static_cast<int64_t>(c.batch) * c.nodes, 1, sh.nodes, 1, &maps.q_shared);
        } else if (sh.nodes >= c.nodes) {
            rc = heads_map(dtype, a.q, c, c.nodes, c.batch, c.nodes, sh.nodes / c.nodes, &maps.q_shared);
        }
    }
    if (rc != SPECHUB_OK) return rc;
    if (dtype == SPECHUB_BF16) return c.head_dim == 64 ? launch_type<__nv_bfloat16, 64>(k, maps, s) : launch_type<__nv_bfloat16, 128>(k, maps, s);
    return c.head_dim == 64 ? launch_type<__half, 64>(k, maps, s) : launch_type<__half, 128>(k, maps, s);
}

}  // namespace spechub
