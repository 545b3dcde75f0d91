// Attention of tree nodes over a paged cache: tensor maps, workspace, launches.
#include <mutex>

#include "spechub_attention.cuh"
#include "spechub_cache_launch.h"
#include "spechub_shapes.h"

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

// (head_dim, token of a page, head, page), boxes of 64 dimensions of a page's tokens (128 of them at most)
int page_map(int dtype, const PagesPtr &x, const CacheArgs &c, CUtensorMap *map) {
    const Encode encode = encoder();
    if (!encode) return SPECHUB_ERR_LAUNCH;
    const cuuint32_t ps = 1u << c.page_shift;
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(c.head_dim), ps, static_cast<cuuint64_t>(c.kv_heads), static_cast<cuuint64_t>(c.pages)};
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(x.token) * 2, static_cast<cuuint64_t>(x.head) * 2, static_cast<cuuint64_t>(x.page) * 2};
    const cuuint32_t box[4] = {64, ps < kTile ? ps : kTile, 1, 1}, each[4] = {1, 1, 1, 1};
    const CUresult r = encode(map, dtype == SPECHUB_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, x.data, dims, strides, box,
                              each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SPECHUB_OK : SPECHUB_ERR_ALIGN;
}

size_t up(size_t n) { return (n + 255) & ~size_t(255); }

// The plan, and the workspace's size; its parts are at `base`.  false: costs are counted in 31 bits, and there may be more than that.
bool plan_of(const CacheArgs &c, int64_t shared_len, uint8_t *base, AttPlan *p, size_t *bytes) {
    const int64_t group = c.heads / c.kv_heads, own = c.nodes * group, all = own * c.batch;
    p->shared_tiles = static_cast<int>((shared_len + kTile - 1) / kTile);
    p->shared_blocks = shared_len ? static_cast<int>((all + kBlockRows - 1) / kBlockRows) : 0;
    p->own_blocks = static_cast<int>((own + kBlockRows - 1) / kBlockRows);
    p->shared_rows = static_cast<int>(all < kBlockRows ? all : kBlockRows);
    p->own_rows = static_cast<int>(own < kBlockRows ? own : kBlockRows);
    const int64_t shared_items = static_cast<int64_t>(c.kv_heads) * p->shared_blocks, own_items = static_cast<int64_t>(c.batch) * c.kv_heads * p->own_blocks;
    const int64_t own_tiles = ((static_cast<int64_t>(c.table_width) << c.page_shift) + kTile - 1) / kTile;   // of a sequence, at most
    const int64_t shared_cost = shared_len ? shared_items * (kBlockCost + static_cast<int64_t>(kTileCost) * p->shared_tiles) : 0;
    const double most = double(shared_cost) + double(own_items) * (kBlockCost + double(kTileCost) * own_tiles);
    if (most > 2.0e9) return false;
    p->shared_items = static_cast<int>(shared_items);
    p->shared_cost = static_cast<int>(shared_cost);
    p->group = FastDiv::of(static_cast<uint32_t>(group));
    p->nodes = FastDiv::of(static_cast<uint32_t>(c.nodes));
    // as many CTAs as there can be tiles, at most one per SM
    const int64_t tiles = shared_items * p->shared_tiles + own_items * own_tiles;
    p->grid = static_cast<int>(tiles < kSms ? tiles : kSms);
    p->slots = shared_len ? shared_items + p->grid : 0;
    const int64_t rows = p->slots * p->shared_rows + (own_items + p->grid) * p->own_rows;
    size_t at = 0;
    p->before = reinterpret_cast<int *>(base);
    at += up(sizeof(int) * (static_cast<size_t>(c.batch) + 1));
    p->error = reinterpret_cast<int *>(base + at);
    at += up(sizeof(int) * static_cast<size_t>(p->grid));
    p->ml = reinterpret_cast<float2 *>(base + at);
    at += up(sizeof(float2) * static_cast<size_t>(rows));
    p->o = reinterpret_cast<float *>(base + at);
    *bytes = at + up(sizeof(float) * static_cast<size_t>(rows) * c.head_dim);
    return true;
}

template <class T, int D>
int launch_type(const AttKernelArgs &k, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t s) {
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
    const int lrc = launch_grid(attention_kernel<T, D>, k.p.grid, kAttThreads, AttShape<D>::kSmem, 1, s, k, mk, mv);
    if (lrc != SPECHUB_OK) return lrc;
    const int64_t grid = static_cast<int64_t>(k.a.c.batch) * k.a.c.kv_heads * k.p.own_blocks * ((k.p.own_rows + kJoinRows - 1) / kJoinRows) +
                         (k.a.c.status ? k.a.c.batch : 0);
    if (grid > 0x7fffffffLL) return SPECHUB_ERR_SHAPE;
    return launch_grid(attention_join_kernel<T, D>, static_cast<unsigned>(grid), kJoinThreads, 0, 1, s, k);
}

}  // namespace

bool attention_workspace(const CacheArgs &c, int64_t shared_len, size_t *bytes) {
    AttPlan p;
    return plan_of(c, shared_len, nullptr, &p, bytes);
}

int launch_attention(int dtype, const AttentionArgs &a, void *workspace, cudaStream_t s) {
    AttKernelArgs k;
    k.a = a;
    size_t bytes;
    if (!plan_of(a.c, a.shared_len, static_cast<uint8_t *>(workspace), &k.p, &bytes)) return SPECHUB_ERR_SHAPE;
    CUtensorMap mk, mv;
    int rc = page_map(dtype, a.c.k, a.c, &mk);
    if (rc == SPECHUB_OK) rc = page_map(dtype, a.c.v, a.c, &mv);
    if (rc != SPECHUB_OK) return rc;
    if (dtype == SPECHUB_BF16) return a.c.head_dim == 64 ? launch_type<__nv_bfloat16, 64>(k, mk, mv, s) : launch_type<__nv_bfloat16, 128>(k, mk, mv, s);
    return a.c.head_dim == 64 ? launch_type<__half, 64>(k, mk, mv, s) : launch_type<__half, 128>(k, mk, mv, s);
}

}  // namespace spechub
