// C ABI of the cache operators (include/spechub_cache.h): host-side argument checks.
#include <math.h>

#include "spechub_cache.h"
#include "spechub_cache_launch.h"

namespace {

using namespace spechub;

int check_cache_desc(const spechub_cache_desc *d) {
    if (!d) return SPECHUB_ERR_NULL;
    if (d->struct_size != sizeof(spechub_cache_desc) || d->version != SPECHUB_ABI_VERSION) return SPECHUB_ERR_VERSION;
    if (d->dtype != SPECHUB_BF16 && d->dtype != SPECHUB_F16) return SPECHUB_ERR_DTYPE;
    if (d->batch < 0 || d->nodes < 1) return SPECHUB_ERR_SHAPE;
    if (d->kv_heads < 1 || d->heads < d->kv_heads || d->heads % d->kv_heads != 0 || (d->head_dim != 64 && d->head_dim != 128) ||
        d->page_size < 8 || d->page_size > 1024 || (d->page_size & (d->page_size - 1)) != 0 || d->pages < 1 || d->layers < 1 ||
        d->table_width < 1)
        return SPECHUB_ERR_CACHE;
    if (static_cast<int64_t>(d->batch) * d->nodes > 0x7fffffffLL / d->heads) return SPECHUB_ERR_SHAPE;
    // a sequence's slots, and those of the tile behind them, are counted in 31 bits
    if (static_cast<int64_t>(d->table_width) * d->page_size > 0x7ffff000LL) return SPECHUB_ERR_CACHE;
    if (d->batch > 1 && d->stride_table < d->table_width) return SPECHUB_ERR_STRIDE;
    return SPECHUB_OK;
}

constexpr int64_t kMaxShared = 0x3fffffff;
constexpr int64_t kMostOffset = 1ll << 53;   // positions are whole numbers in 64-bit floating point up to here

bool at16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// A stride as the kernels take it: that of a dimension of size 1 is any.  `apart`: places of the dimension may not be the same.
bool stride(int64_t s, int64_t count, int64_t least, bool apart, int64_t *out) {
    *out = count > 1 ? s : least;
    return count <= 1 || (s >= (apart ? least : 0) && s % 8 == 0);
}

// Places of a tensor, or differences of places: sums of index x stride, the index from lo to hi.
struct Axis {
    int64_t stride, lo, hi;
    int64_t low, high;   // the least and the largest sum of the axes behind this one
};

// Is there a choice of indices, other than all 0 if `other`, whose sum and `at` are less than `width` together, either way?  Axes by falling
// strides; where they nest, as those of a tensor's views do, each has one index to look at.  Strides that do not nest may take more:
// after kMostSteps the answer is no.
constexpr int kMostSteps = 4096;
bool near(const Axis *x, const Axis *end, int64_t at, int64_t width, bool other, int *steps) {
    if (x == end) return !other && at < width && at > -width;
    const auto down = [](int64_t a, int64_t b) { return a / b - (a % b < 0); };   // the quotient's whole part, b > 0
    const int64_t first = down(-width - (at + x->high), x->stride) + 1, last = -down(at + x->low - width, x->stride) - 1;
    for (int64_t i = first > x->lo ? first : x->lo; i <= last && i <= x->hi; ++i) {
        if (--*steps < 0) return false;
        if (near(x + 1, end, at + x->stride * i, width, other && i == 0, steps)) return true;
    }
    return false;
}
bool near(Axis *x, int axes, int64_t at, int64_t width, bool other) {
    int n = 0;
    for (int i = 0; i < axes; ++i) {   // sorted; axes that lead nowhere are left out
        const Axis a = x[i];
        if (a.stride == 0 || (a.lo == 0 && a.hi == 0)) continue;
        int j = n++;
        for (; j > 0 && x[j - 1].stride < a.stride; --j) x[j] = x[j - 1];
        x[j] = a;
    }
    constexpr int64_t kMost = 1ll << 58;   // no memory is that large
    int64_t low = 0, high = 0, by;
    bool nested = other && at == 0;
    for (int i = n - 1; i >= 0; --i) {
        x[i].low = low;
        x[i].high = high;
        nested = nested && x[i].stride >= width + high;
        if (__builtin_mul_overflow(x[i].stride, x[i].lo, &by) || by < -kMost) return false;
        low += by;
        if (__builtin_mul_overflow(x[i].stride, x[i].hi, &by) || by > kMost) return false;
        high += by;
    }
    int steps = kMostSteps;
    return !nested && near(x, x + n, at, width, other, &steps);
}

// Do two rows of the tensor share an element?
template <int N>
bool over_itself(const int64_t (&strides)[N], const int64_t (&counts)[N], int head_dim) {
    Axis x[N];
    for (int i = 0; i < N; ++i) x[i] = {strides[i], 1 - counts[i], counts[i] - 1};
    return near(x, N, 0, head_dim, true);
}
bool over_itself(const HeadsPtr &h, const spechub_cache_desc *d, int heads) {
    return over_itself({h.seq, h.node, h.head}, {d->batch, d->nodes, heads}, d->head_dim);
}
bool over_itself(const PagesPtr &p, const spechub_cache_desc *d) {
    return over_itself({p.layer, p.page, p.token, p.head}, {d->layers, d->pages, d->page_size, d->kv_heads}, d->head_dim);
}

// Does a row of one tensor share an element with a row of another?
template <int N>
bool meet(const void *a, const int64_t (&a_strides)[N], const int64_t (&a_counts)[N], const void *b, const int64_t (&b_strides)[N],
          const int64_t (&b_counts)[N], int head_dim) {
    Axis x[2 * N];
    int n = 0;
    for (int i = 0; i < N; ++i) {
        if (a_strides[i] == b_strides[i]) x[n++] = {a_strides[i], 1 - b_counts[i], a_counts[i] - 1};
        else {
            x[n++] = {a_strides[i], 0, a_counts[i] - 1};
            x[n++] = {b_strides[i], 1 - b_counts[i], 0};
        }
    }
    return near(x, n, (static_cast<const char *>(a) - static_cast<const char *>(b)) / 2, head_dim, false);
}
bool meet(const HeadsPtr &a, int a_heads, const HeadsPtr &b, int b_heads, const spechub_cache_desc *d) {
    return meet(a.data, {a.seq, a.node, a.head}, {d->batch, d->nodes, a_heads}, b.data, {b.seq, b.node, b.head}, {d->batch, d->nodes, b_heads}, d->head_dim);
}
bool meet(const PagesPtr &a, const PagesPtr &b, const spechub_cache_desc *d) {
    return meet(a.data, {a.layer, a.page, a.token, a.head}, {d->layers, d->pages, d->page_size, d->kv_heads}, b.data, {b.layer, b.page, b.token, b.head},
                {d->layers, d->pages, d->page_size, d->kv_heads}, d->head_dim);
}

int heads_of(const spechub_heads *x, const spechub_cache_desc *d, int heads, bool written, HeadsPtr *out) {
    if (!x || !x->data) return SPECHUB_ERR_NULL;
    out->data = x->data;
    return at16(x->data) && stride(x->stride_seq, d->batch, d->head_dim, written, &out->seq) &&
                   stride(x->stride_node, d->nodes, d->head_dim, written, &out->node) &&
                   stride(x->stride_head, heads, d->head_dim, written, &out->head)
               ? SPECHUB_OK
               : SPECHUB_ERR_ALIGN;
}

int pages_of(const spechub_pages *x, const spechub_cache_desc *d, PagesPtr *out) {
    if (!x || !x->data) return SPECHUB_ERR_NULL;
    out->data = x->data;
    return at16(x->data) && stride(x->stride_layer, d->layers, d->head_dim, true, &out->layer) &&
                   stride(x->stride_page, d->pages, d->head_dim, true, &out->page) &&
                   stride(x->stride_token, d->page_size, d->head_dim, true, &out->token) &&
                   stride(x->stride_head, d->kv_heads, d->head_dim, true, &out->head)
               ? SPECHUB_OK
               : SPECHUB_ERR_ALIGN;
}

int cache_args(const spechub_cache_desc *d, const spechub_pages *k, const spechub_pages *v, uint32_t *status, CacheArgs *c) {
    if (!d->table || !d->lens) return SPECHUB_ERR_NULL;
    int rc = pages_of(k, d, &c->k);
    if (rc == SPECHUB_OK) rc = pages_of(v, d, &c->v);
    if (rc != SPECHUB_OK) return rc;
    c->table = d->table;
    c->lens = d->lens;
    c->stride_table = d->batch > 1 ? d->stride_table : d->table_width;
    c->batch = d->batch; c->nodes = d->nodes; c->heads = d->heads; c->kv_heads = d->kv_heads; c->head_dim = d->head_dim;
    c->page_shift = __builtin_ctz(static_cast<unsigned>(d->page_size));
    c->pages = d->pages; c->table_width = d->table_width; c->layers = d->layers;
    c->status = status;
    return SPECHUB_OK;
}

}  // namespace

extern "C" {

int spechub_cache_append(const spechub_cache_desc *desc, const spechub_heads *q, const spechub_heads *k,
                         const spechub_heads *v, const spechub_pages *k_cache, const spechub_pages *v_cache,
                         const int32_t *depth, int64_t depth_stride_seq, const float *inv_freq, int32_t rotated,
                         int32_t interleaved, int64_t pos_offset, const spechub_heads *q_out, uint32_t *status,
                         void *stream) {
    int rc = check_cache_desc(desc);
    if (rc != SPECHUB_OK) return rc;
    if (desc->layers != 1) return SPECHUB_ERR_CACHE;
    if (rotated < 0 || rotated > desc->head_dim || rotated % 16 != 0 || (interleaved != 0 && interleaved != 1)) return SPECHUB_ERR_ROTARY;
    if (rotated > 0 && (pos_offset > kMostOffset || pos_offset < -kMostOffset)) return SPECHUB_ERR_ROTARY;
    if (depth_stride_seq < 0 || (depth_stride_seq != 0 && depth_stride_seq < desc->nodes)) return SPECHUB_ERR_STRIDE;
    if (desc->batch == 0) return SPECHUB_OK;
    AppendArgs a = {};
    rc = cache_args(desc, k_cache, v_cache, status, &a.c);
    if (rc == SPECHUB_OK) rc = heads_of(k, desc, desc->kv_heads, false, &a.k);
    if (rc == SPECHUB_OK) rc = heads_of(v, desc, desc->kv_heads, false, &a.v);
    if (rc == SPECHUB_OK && q) {
        rc = heads_of(q, desc, desc->heads, false, &a.q);
        if (rc == SPECHUB_OK) rc = heads_of(q_out, desc, desc->heads, true, &a.q_out);
    }
    if (rc != SPECHUB_OK) return rc;
    if (rotated > 0 && !inv_freq) return SPECHUB_ERR_NULL;
    if (over_itself(a.c.k, desc) || over_itself(a.c.v, desc) || (q && over_itself(a.q_out, desc, desc->heads))) return SPECHUB_ERR_ALIGN;
    if (q) {
        const bool in_place = a.q_out.data == a.q.data && a.q_out.seq == a.q.seq && a.q_out.node == a.q.node && a.q_out.head == a.q.head;
        if ((!in_place && meet(a.q_out, desc->heads, a.q, desc->heads, desc)) || meet(a.q_out, desc->heads, a.k, desc->kv_heads, desc) ||
            meet(a.q_out, desc->heads, a.v, desc->kv_heads, desc))
            return SPECHUB_ERR_ALIGN;
    }
    a.depth = depth;
    a.depth_stride_seq = depth_stride_seq;
    a.inv_freq = inv_freq;
    a.rotated = rotated;
    a.pos_offset = pos_offset;
    return launch_append(desc->dtype, a, interleaved == 1, static_cast<cudaStream_t>(stream));
}

size_t spechub_tree_attention_workspace_bytes(const spechub_cache_desc *desc, int64_t shared_len) {
    if (check_cache_desc(desc) != SPECHUB_OK || desc->heads / desc->kv_heads > SPECHUB_MAX_GROUP || shared_len < 0 || shared_len > kMaxShared ||
        desc->batch == 0)
        return 0;
    CacheArgs c = {};
    c.batch = desc->batch; c.nodes = desc->nodes; c.heads = desc->heads; c.kv_heads = desc->kv_heads; c.head_dim = desc->head_dim;
    c.page_shift = __builtin_ctz(static_cast<unsigned>(desc->page_size)); c.table_width = desc->table_width;
    size_t bytes = 0;
    return attention_workspace(c, shared_len, &bytes) ? bytes : 0;
}

int spechub_tree_attention(const spechub_cache_desc *desc, const spechub_heads *q, const spechub_pages *k_cache,
                           const spechub_pages *v_cache, const int32_t *mask, int64_t mask_stride_seq,
                           const int32_t *shared_table, int32_t shared_width, int64_t shared_len, float scale,
                           const spechub_heads *out, float *lse, uint32_t *status, void *workspace,
                           size_t workspace_bytes, void *stream) {
    int rc = check_cache_desc(desc);
    if (rc != SPECHUB_OK) return rc;
    if (desc->layers != 1 || desc->heads / desc->kv_heads > SPECHUB_MAX_GROUP) return SPECHUB_ERR_CACHE;
    const float scale_log2 = scale * 1.4426950408889634f;
    if (!(scale > 0.f && isfinite(scale_log2))) return SPECHUB_ERR_SCALE;
    if (shared_len < 0 || shared_len > kMaxShared || shared_width < 0 || shared_len > static_cast<int64_t>(shared_width) * desc->page_size)
        return SPECHUB_ERR_SHARED;
    const int64_t words = (desc->nodes + 31) / 32;
    if (mask_stride_seq < 0 || (mask_stride_seq != 0 && mask_stride_seq < words * desc->nodes)) return SPECHUB_ERR_STRIDE;
    if (desc->batch == 0) return SPECHUB_OK;
    AttentionArgs a = {};
    rc = cache_args(desc, k_cache, v_cache, status, &a.c);
    if (rc == SPECHUB_OK) rc = heads_of(q, desc, desc->heads, true, &a.q);   // (rows of a tensor copy lie apart)
    if (rc == SPECHUB_OK) rc = heads_of(out, desc, desc->heads, true, &a.out);
    if (rc != SPECHUB_OK) return rc;
    if (!mask || (shared_len > 0 && !shared_table)) return SPECHUB_ERR_NULL;
    size_t need = 0;
    if (!attention_workspace(a.c, shared_len, &need)) return SPECHUB_ERR_WORK;
    if (workspace_bytes < need) return SPECHUB_ERR_WORKSPACE;
    if (need && !workspace) return SPECHUB_ERR_NULL;
    if (need && !at16(workspace)) return SPECHUB_ERR_ALIGN;
    // (queries are read again after the first outputs are there)
    if (over_itself(a.out, desc, desc->heads) || meet(a.out, desc->heads, a.q, desc->heads, desc)) return SPECHUB_ERR_ALIGN;
    a.mask = mask;
    a.mask_stride_seq = mask_stride_seq;
    a.shared_table = shared_table;
    a.shared_len = static_cast<int>(shared_len);
    a.scale_log2 = scale_log2;
    a.lse = lse;
    return launch_attention(desc->dtype, a, workspace, static_cast<cudaStream_t>(stream));
}

int spechub_cache_accept(const spechub_cache_desc *desc, const spechub_pages *k_cache, const spechub_pages *v_cache,
                         const int32_t *path_nodes, int32_t levels, int32_t *lens_out, uint32_t *status, void *stream) {
    int rc = check_cache_desc(desc);
    if (rc != SPECHUB_OK) return rc;
    if (levels < 1) return SPECHUB_ERR_SHAPE;
    if (desc->batch == 0) return SPECHUB_OK;
    AcceptArgs a = {};
    rc = cache_args(desc, k_cache, v_cache, status, &a.c);
    if (rc != SPECHUB_OK) return rc;
    // (one CTA writes the new length while others still read the old ones)
    if (!path_nodes || !lens_out || (lens_out < desc->lens + desc->batch && desc->lens < lens_out + desc->batch)) return SPECHUB_ERR_NULL;
    // (entries of keys that are values too would be moved twice, the second time perhaps after what they were is gone)
    if (over_itself(a.c.k, desc) || over_itself(a.c.v, desc) || meet(a.c.k, a.c.v, desc)) return SPECHUB_ERR_ALIGN;
    a.path = path_nodes;
    a.levels = levels;
    a.lens_out = lens_out;
    return launch_accept(a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
