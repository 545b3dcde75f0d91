// Attention of tree nodes over a paged cache.
#include "spechub_attention.cuh"
#include "spechub_cache_launch.h"

namespace spechub {

template <class T>
static int launch_rows(const AttentionArgs &a, cudaStream_t s) {
    const int64_t rows = int64_t(a.c.batch) * a.c.nodes * a.c.heads, per = kAttRowThreads / 32;
    const unsigned grid = static_cast<unsigned>((rows + per - 1) / per);
    return a.c.head_dim == 64 ? launch_grid(attention_rows_kernel<T, 64>, grid, kAttRowThreads, 0, 1, s, a)
                              : launch_grid(attention_rows_kernel<T, 128>, grid, kAttRowThreads, 0, 1, s, a);
}

size_t attention_workspace(const CacheArgs &, int64_t) { return 0; }

int launch_attention(int dtype, const AttentionArgs &a, void *, cudaStream_t s) {
    const int rc = dtype == SPECHUB_BF16 ? launch_rows<__nv_bfloat16>(a, s) : launch_rows<__half>(a, s);
    if (rc != SPECHUB_OK || !a.c.status) return rc;
    return launch_grid(attention_status_kernel, a.c.batch, kAttStatusThreads, 0, 1, s, a);
}

}  // namespace spechub
