/*
 * spechub_cache.h -- C ABI of the target model's side of a decoding iteration:
 * scoring a token tree with a paged cache of keys and values.
 *
 * Between the draft step and verification (spechub.h) the target model scores
 * all nodes of every sequence's tree in one pass (Figure 2 of arXiv
 * 2411.05289: the tree's tokens share the context before them, and each node
 * sees its ancestors).  In every layer the nodes' keys and values are appended
 * to the cache (spechub_cache_append) and attended to
 * (spechub_tree_attention); after the tree walk the entries of the accepted
 * path move up to the end of the context (spechub_cache_accept).
 *
 * The general rules of spechub.h hold: device pointers owned by the caller,
 * work enqueued on `stream` without synchronising, negative codes for what the
 * host refuses (nothing is launched then), no allocation, no state between
 * calls, batch = 0 is a valid empty call.  The calls may be captured into CUDA
 * graphs; lengths, page tables and masks are read when the graph runs.
 *
 * The cache
 *   Pages of `page_size` tokens (a power of two from 8 to 1024), `pages` of
 *   them, each token with kv_heads heads of head_dim (64 or 128) elements of
 *   16 bits.  Keys and values have element strides of their own for layer,
 *   page, token and head, so that both common orders of a page (token by
 *   token, head by head) and interleaved keys and values are taken as they
 *   are.  Row b of `table` ([batch][table_width] page ids, rows stride_table
 *   apart) says where sequence b's slots are: slot i lies in page
 *   table[b][i / page_size] at i % page_size.  Entries behind the last slot in
 *   use are not looked at.
 *   lens[b] is the length of sequence b's own context, without the nodes of
 *   this iteration.  Node n of the tree is kept in slot lens[b] + n.
 *   lens[b] < 0: the sequence is absent (a padded batch).  Nothing is written
 *   for it, neither to the cache nor to its rows of the outputs.
 *   What lies in slots and pages that no sequence uses is never part of a
 *   result, NaN and infinities included.
 *   Two sequences may share pages that both only read; where two calls or two
 *   sequences write one slot, the result is undefined.
 * Status
 *   status[b] (may be NULL everywhere) is 0 or a sum of
 *   SPECHUB_ST_PAGE: a page id that the call had to follow is outside [0,
 *     pages), or a slot lies behind the table's last page: append and accept
 *     leave those entries out, attention reads a page whose id is bad as zeros
 *     and takes slots behind the table as not there;
 *   SPECHUB_ST_PATH (accept): the path has an entry that no walk leaves; it
 *     ends before that entry;
 *   SPECHUB_ST_INTERNAL (attention): a bounded wait inside the kernel ran out
 *     and the outputs are not valid.
 * Alignment
 *   Every data pointer to 16-bit elements is a multiple of 16 bytes and every
 *   stride a multiple of 8 elements; the last dimension is contiguous.  A
 *   stride of a dimension of size 1 is not looked at.  Strides of the cache, of
 *   outputs and of q of spechub_tree_attention are at least head_dim.
 * Overlaps
 *   Rows (a head of a node, of a token) that a call writes share no element
 *   with each other; strides for which they do are refused.  So are a q_out that
 *   shares elements with k or v, or with q where it is not q itself, and an out
 *   that does with q; and, by spechub_cache_accept, keys that share elements with
 *   values.  (Slices of one tensor may lie between each other.  Strides
 *   that do not nest, as those of views do, are looked at in up to 4096 steps.)
 *   That outputs, the cache, the workspace and the inputs share nothing else is the
 *   caller's to see to.
 */
#ifndef SPECHUB_CACHE_H_
#define SPECHUB_CACHE_H_

#include "spechub.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element type of the cache (SPECHUB_BF16 is the other one) */
#define SPECHUB_F16 2
#define SPECHUB_MAX_GROUP 128 /* most query heads per cache head that spechub_tree_attention takes */

#define SPECHUB_ERR_ALIGN (-11)  /* a pointer or stride is not a multiple of 16 bytes, or rows overlap: see Overlaps */
#define SPECHUB_ERR_CACHE (-12)  /* bad cache or head shape: see spechub_cache_desc */
#define SPECHUB_ERR_ROTARY (-13) /* rotated is not a multiple of 16 from 0 to head_dim, interleaved is not 0 / 1, or |pos_offset| > 2^53 where rotated > 0 */
#define SPECHUB_ERR_SHARED (-14) /* shared_len < 0, or more tokens than shared_width pages hold */
#define SPECHUB_ERR_SCALE (-15)  /* scale is not > 0, or scale * log2(e) is no finite number */
#define SPECHUB_ERR_WORK (-16)   /* more work than one call of spechub_tree_attention counts: see there */

#define SPECHUB_ST_PAGE 128u
#define SPECHUB_ST_PATH 256u

typedef struct spechub_cache_desc {
    uint32_t struct_size;  /* sizeof(spechub_cache_desc)                              */
    uint32_t version;      /* SPECHUB_ABI_VERSION                                     */
    int32_t dtype;         /* SPECHUB_BF16 or SPECHUB_F16: cache, q, k, v and outputs */
    int32_t batch;         /* sequences B                                             */
    int32_t nodes;         /* N >= 1 nodes per sequence (accept: of the tree walked)  */
    int32_t heads;         /* query heads, a multiple of kv_heads                     */
    int32_t kv_heads;      /* >= 1; query head h reads head h / (heads / kv_heads)    */
    int32_t head_dim;      /* 64 or 128                                               */
    int32_t page_size;     /* tokens per page: a power of two, 8..1024                */
    int32_t pages;         /* pages of the cache, >= 1                                */
    int32_t layers;        /* layers that accept moves, >= 1; 1 for the other calls   */
    int32_t table_width;   /* page ids per row of `table`, >= 1                       */
    int64_t stride_table;  /* page ids between rows, >= table_width                   */
    const int32_t *table;  /* device [batch][table_width]                             */
    const int32_t *lens;   /* device [batch]                                          */
} spechub_cache_desc;

/* keys or values of all pages */
typedef struct spechub_pages {
    void *data;
    int64_t stride_layer, stride_page, stride_token, stride_head; /* elements */
} spechub_pages;

/* [batch][nodes][heads or kv_heads][head_dim] */
typedef struct spechub_heads {
    void *data;
    int64_t stride_seq, stride_node, stride_head; /* elements */
} spechub_heads;

/*
 * Append the nodes' keys and values, rotated by position on the way.
 *   Node n of sequence b is at position p = pos_offset + lens[b] + depth[n]
 *   (depth [nodes] for all sequences, depth_stride_seq = 0, or [batch][nodes];
 *   NULL: depth[n] = n, a chunk of a prompt).  Of every head of q and k the
 *   first `rotated` dimensions are rotated: pair i = (x0, x1) becomes
 *   (x0 cos a - x1 sin a, x0 sin a + x1 cos a) with a = p * inv_freq[i],
 *   i < rotated / 2; a pair is (i, i + rotated / 2), or (2i, 2i + 1) if
 *   `interleaved`.  The angle is formed in 64 bits (far positions lose their
 *   turns' fraction in 32) and the result rounded once.  The angle is off by
 *   2^-51 of itself at most, less than 2^-20 at 2^31 with an inv_freq of 1.
 *   k goes to slot lens[b] + n of k_cache, v unchanged to v_cache, rotated q
 *   to q_out; q_out may be q itself.  q may be NULL (then q_out is not looked
 *   at), and inv_freq where rotated = 0.
 */
int spechub_cache_append(const spechub_cache_desc *desc, const spechub_heads *q, const spechub_heads *k,
                         const spechub_heads *v, const spechub_pages *k_cache, const spechub_pages *v_cache,
                         const int32_t *depth, int64_t depth_stride_seq, const float *inv_freq, int32_t rotated,
                         int32_t interleaved, int64_t pos_offset, const spechub_heads *q_out, uint32_t *status,
                         void *stream);

/*
 * Attention of the nodes to the prefix that the whole batch shares, to their
 * sequence's own context and to the nodes that they see.
 *   out[b][n][h] = sum_j softmax_j(scale * q[b][n][h] . k_j) v_j
 * over the shared_len tokens of the pages shared_table [shared_width] (read
 * once for the whole batch), the lens[b] slots of the context, and the slots
 * lens[b] + m for which bit m of node n's mask is set.  mask is int32
 * [nodes][ceil(nodes / 32)], bit m % 32 of word m / 32 (mask_stride_seq = 0:
 * one tree for all sequences; otherwise [batch] of them, so many words apart).
 *   out and q share no element.  heads / kv_heads is at most SPECHUB_MAX_GROUP.
 *   lse[b][n][h] (may be NULL) is the natural logarithm of sum_j exp(scale * q
 * . k_j).  A row that sees nothing is 0 with lse = -inf.
 *   A key or value that is NaN or infinite concerns the rows that see it only.
 *   Scores, sums and the output before its one rounding are held in 32 bits;
 * the weights are rounded to the cache's type for their product with the
 * values.  Scores (scale * q . k) are up to 2^25 in magnitude; where they are
 * larger, 32 bits hold them to whole numbers only, and a row may lose its weights.  The result does not depend on when which block runs: the same call
 * on the same GPU model gives the same bits.
 *   workspace: device scratch, 16-byte aligned, of at least
 * spechub_tree_attention_workspace_bytes(desc, shared_len) bytes.  It need not
 * be cleared; calls that may overlap need one each.
 *   The work is counted on the host, before the lengths are known: 8 and at most 14
 * for every 128 keys, for each cache head and each block of up to 256 rows (nodes
 * times heads / kv_heads; of a sequence with the keys that its whole row of the
 * table holds, of the batch with the prefix).  Above 2e9, some seconds if the
 * tables are full, the call is refused (SPECHUB_ERR_WORK).
 * spechub_tree_attention_workspace_bytes is 0 then, as for an empty batch and for
 * what else it knows to be refused; otherwise it is not.
 */
size_t spechub_tree_attention_workspace_bytes(const spechub_cache_desc *desc, int64_t shared_len);
int spechub_tree_attention(const spechub_cache_desc *desc, const spechub_heads *q, const spechub_pages *k_cache,
                           const spechub_pages *v_cache, const int32_t *mask, int64_t mask_stride_seq,
                           const int32_t *shared_table, int32_t shared_width, int64_t shared_len, float scale,
                           const spechub_heads *out, float *lse, uint32_t *status, void *workspace,
                           size_t workspace_bytes, void *stream);

/*
 * Take over the accepted path.  path_nodes [batch][levels] is what the tree
 * walk leaves (spechub_seq_out): the visited nodes, then -1.  In every layer
 * the entry of slot lens[b] + path_nodes[b][d] moves to slot lens[b] + d;
 * lens_out[b] = lens[b] + the number of visited nodes (lens[b] itself for an
 * absent sequence).  lens_out may not overlap lens (SPECHUB_ERR_NULL, as if it
 * were not given).  The entries need no other
 * rotation: a node's position goes by its depth, which is its place in the
 * path.  (The slots behind the path keep what they hold.)
 */
int spechub_cache_accept(const spechub_cache_desc *desc, const spechub_pages *k_cache, const spechub_pages *v_cache,
                         const int32_t *path_nodes, int32_t levels, int32_t *lens_out, uint32_t *status, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SPECHUB_CACHE_H_ */
