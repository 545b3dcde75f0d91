// The paged cache's kernels that move entries: append (with the rotation by position) and accept.
//
// Both are copies: what bounds them is bytes (append: every element of q, k, v once in, once out; accept: the moved entries
// once in, once out), and for small batches the chain length -> page id -> address -> data.
#pragma once

#include "spechub_pages.cuh"

namespace spechub {

constexpr int kAppendThreads = 512;   // at most

// One CTA per node.  An item is 32 bytes of a head: eight pairs (two vectors of eight elements: of both halves of the
// rotated part, or neighbours), or sixteen elements that are copied.  The node's cosines and sines are found once, for all heads.
template <class T, bool NEXT>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const __grid_constant__ AppendArgs A) {
    __shared__ float2 turn[64];   // (cos, sin) of each pair
    pdl_begin();
    const CacheArgs &c = A.c;
    const int b = blockIdx.x / c.nodes, n = blockIdx.x - b * c.nodes, tid = threadIdx.x;
    const int64_t len = c.lens[b];
    const int32_t *row = c.table + b * c.stride_table;
    if (n == 0 && c.status) {
        bool bad = false;
        for (int i = tid; i < c.nodes && len >= 0; i += blockDim.x) bad |= page_of(c, row, len + i) < 0;
        bad = __syncthreads_or(bad);
        if (tid == 0) c.status[b] = bad ? SPECHUB_ST_PAGE : 0u;
    }
    if (len < 0) return;
    const int half = A.rotated / 2;
    for (int i = tid; i < half; i += blockDim.x) {
        const int64_t d = A.depth ? A.depth[b * A.depth_stride_seq + n] : n;
        // the angle in turns, its whole turns dropped before 32 bits are enough
        const double turns = static_cast<double>(A.pos_offset + len + d) * (static_cast<double>(A.inv_freq[i]) * 0.15915494309189535);
        const float f = static_cast<float>(2.0 * (turns - rint(turns)));
        float s, cs;
        sincospif(f, &s, &cs);
        turn[i] = make_float2(cs, s);
    }
    const int page = page_of(c, row, len + n);
    const int64_t place = (len + n) & ((1 << c.page_shift) - 1);
    const int64_t k_at = page * c.k.page + place * c.k.token, v_at = page * c.v.page + place * c.v.token;
    __syncthreads();
    const int per_head = c.head_dim / 16, qn = A.q.data ? c.heads * per_head : 0, kn = c.kv_heads * per_head;
    const int rot_items = A.rotated / 16;
    for (int it = tid; it < qn + 2 * kn; it += blockDim.x) {
        const int what = it < qn ? 0 : it < qn + kn ? 1 : 2;
        const int j = it - (what == 0 ? 0 : what == 1 ? qn : qn + kn);
        const int h = j / per_head, i = j - h * per_head;
        const HeadsPtr &x = what == 0 ? A.q : what == 1 ? A.k : A.v;
        const T *src = static_cast<const T *>(x.data) + b * x.seq + n * x.node + h * x.head;
        T *dst;
        if (what == 0) dst = static_cast<T *>(A.q_out.data) + b * A.q_out.seq + n * A.q_out.node + h * A.q_out.head;
        else if (page < 0) continue;
        else if (what == 1) dst = static_cast<T *>(c.k.data) + k_at + h * c.k.head;
        else dst = static_cast<T *>(c.v.data) + v_at + h * c.v.head;
        const bool rot = what < 2 && i < rot_items;
        const int e0 = rot && !NEXT ? 8 * i : 16 * i, e1 = rot && !NEXT ? half + 8 * i : 16 * i + 8;
        uint4 u0 = *reinterpret_cast<const uint4 *>(src + e0), u1 = *reinterpret_cast<const uint4 *>(src + e1);
        if (rot) {
            uint32_t *w0 = &u0.x, *w1 = &u1.x;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                if (NEXT) {
                    const float2 a = unpack2<T>(w0[p]), z = unpack2<T>(w1[p]), t = turn[8 * i + p], r = turn[8 * i + 4 + p];
                    w0[p] = pack2<T>(a.x * t.x - a.y * t.y, a.x * t.y + a.y * t.x);
                    w1[p] = pack2<T>(z.x * r.x - z.y * r.y, z.x * r.y + z.y * r.x);
                } else {
                    const float2 a = unpack2<T>(w0[p]), z = unpack2<T>(w1[p]), t = turn[8 * i + 2 * p], r = turn[8 * i + 2 * p + 1];
                    w0[p] = pack2<T>(a.x * t.x - z.x * t.y, a.y * r.x - z.y * r.y);
                    w1[p] = pack2<T>(a.x * t.y + z.x * t.x, a.y * r.y + z.y * r.x);
                }
            }
        }
        *reinterpret_cast<uint4 *>(dst + e0) = u0;
        *reinterpret_cast<uint4 *>(dst + e1) = u1;
    }
}

constexpr int kAcceptThreads = 256;
constexpr int kAcceptMoves = 256;   // entries of the path that are looked at together

// The moves of one sequence, by columns: a thread takes one 16-byte vector of a head of a layer, of keys or of values, through the
// path from its front.  In that order nothing is overwritten before it is read, whatever the threads of other columns do: a path's
// d-th node is at least d, so slot lens + d can only be the source of entries up to d.  blockIdx.x: sequence, blockIdx.y: columns.
__global__ void __launch_bounds__(kAcceptThreads) accept_kernel(const __grid_constant__ AcceptArgs A) {
    __shared__ int2 page[kAcceptMoves], place[kAcceptMoves];   // of source and destination
    __shared__ int s_moves, s_end;
    pdl_begin();
    const CacheArgs &c = A.c;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
    const int64_t len = c.lens[b];
    if (len < 0) {
        if (blockIdx.y == 0 && tid == 0) {
            A.lens_out[b] = static_cast<int32_t>(len);
            if (c.status) c.status[b] = 0;
        }
        return;
    }
    const int32_t *row = c.table + b * c.stride_table, *path = A.path + static_cast<int64_t>(b) * A.levels;
    const int vecs = c.head_dim / 8;
    const int64_t columns = 2LL * c.layers * c.kv_heads * vecs;
    uint32_t st = 0;
    int kept = 0, last = -1;
    for (int base = 0; base < A.levels; base += kAcceptMoves) {
        __syncthreads();
        if (tid < 32) {   // one warp reads the path; what is not a move is dropped
            int moves = 0, end = 0;
            for (int d0 = base; d0 < min(base + kAcceptMoves, A.levels) && !end; d0 += 32) {
                const int d = d0 + lane;
                const int node = d < A.levels ? path[d] : -1;
                int before = __shfl_up_sync(kFull, node, 1);
                if (lane == 0) before = last;
                const bool over = node < 0, wrong = !over && (node < d || node >= c.nodes || node <= before);
                const unsigned stop = __ballot_sync(kFull, over || wrong);
                const int first = stop ? __ffs(stop) - 1 : 32;
                if (__ballot_sync(kFull, wrong) & (first < 32 ? 1u << first : 0u)) st |= SPECHUB_ST_PATH;
                kept += first;
                end = stop != 0;
                bool move = lane < first && node != d;
                int2 pg = make_int2(-1, -1);
                if (lane < first) {
                    pg = make_int2(page_of(c, row, len + node), page_of(c, row, len + d));
                    if (pg.x < 0 || pg.y < 0) move = false;
                }
                if (__ballot_sync(kFull, lane < first && (pg.x < 0 || pg.y < 0))) st |= SPECHUB_ST_PAGE;
                const unsigned all = __ballot_sync(kFull, move);
                if (move) {
                    const int at = moves + __popc(all & ((1u << lane) - 1)), in = (1 << c.page_shift) - 1;
                    page[at] = pg;
                    place[at] = make_int2((len + node) & in, (len + d) & in);
                }
                moves += __popc(all);
                last = __shfl_sync(kFull, node, 31);
            }
            if (lane == 0) { s_moves = moves; s_end = end; }
        }
        __syncthreads();
        const int moves = s_moves;
        for (int64_t col = blockIdx.y * int64_t(kAcceptThreads) + tid; col < columns && moves > 0; col += int64_t(gridDim.y) * kAcceptThreads) {
            const int vec = col % vecs;
            int64_t r = col / vecs;
            const int head = r % c.kv_heads;
            r /= c.kv_heads;
            const PagesPtr &x = r & 1 ? c.v : c.k;
            uint16_t *at = static_cast<uint16_t *>(x.data) + (r >> 1) * x.layer + head * x.head + vec * 8;
            for (int m = 0; m < moves; m += 4) {   // (four sources before their destinations: sources lie behind)
                uint4 u[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (m + i < moves) u[i] = *reinterpret_cast<const uint4 *>(at + page[m + i].x * x.page + place[m + i].x * x.token);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (m + i < moves) *reinterpret_cast<uint4 *>(at + page[m + i].y * x.page + place[m + i].y * x.token) = u[i];
            }
        }
        if (s_end) break;
    }
    if (blockIdx.y == 0 && tid == 0) {
        A.lens_out[b] = static_cast<int32_t>(min(len + kept, int64_t(0x7fffffff)));   // (not the length of an absent sequence)
        if (c.status) c.status[b] = st;
    }
}

}  // namespace spechub
