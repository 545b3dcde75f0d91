// Kernel arguments of the cache operators (include/spechub_cache.h).
#pragma once

#include <stdint.h>

namespace spechub {

struct HeadsPtr {   // [batch][nodes][heads][head_dim], element strides
    void *data;
    int64_t seq, node, head;
};
struct PagesPtr {   // keys or values of all pages, element strides
    void *data;
    int64_t layer, page, token, head;
};

struct CacheArgs {
    const int32_t *table, *lens;
    int64_t stride_table;
    PagesPtr k, v;
    int batch, nodes, heads, kv_heads, head_dim;
    int page_shift, pages, table_width, layers;
    uint32_t *status;
};

struct AppendArgs {
    CacheArgs c;
    HeadsPtr q, k, v, q_out;   // q.data null: keys and values only
    const int32_t *depth;      // null: node n is n tokens behind the context's end
    int64_t depth_stride_seq;
    const float *inv_freq;
    int64_t pos_offset;
    int rotated;
};

struct AcceptArgs {
    CacheArgs c;
    const int32_t *path;
    int32_t *lens_out;
    int levels;
};

struct AttentionArgs {
    CacheArgs c;
    HeadsPtr q, out;
    const int32_t *mask;
    int64_t mask_stride_seq;
    const int32_t *shared_table;
    int shared_len;
    float scale_log2;          // scale * log2(e)
    float *lse;                // may be null
};

}  // namespace spechub
