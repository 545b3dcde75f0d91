// Append and accept: the kernels that move entries of the paged cache.
#include "spechub_cache.cuh"
#include "spechub_cache_launch.h"
#include "spechub_shapes.h"

namespace spechub {

template <class T>
static int launch_append_type(const AppendArgs &a, bool interleaved, cudaStream_t s) {
    const unsigned grid = static_cast<unsigned>(a.c.batch) * a.c.nodes;
    const int items = ((a.q.data ? a.c.heads : 0) + 2 * a.c.kv_heads) * (a.c.head_dim / 16);
    // Threads of a node's CTA: three items each where there are more nodes than a wave of CTAs (1 / 2 / 3 / 4 items: 7936 nodes of 384 items
    // 40.1 / 36.4 / 35.8 / 35.8 us, 8000 of 144 items 17.8 / 17.0 / 16.2 / 16.2), one where there are few (one node 5.36 / 5.44 / 5.56 / 5.58).
    const int each = grid > 8 * kSms ? 3 : 1, wanted = (items + 32 * each - 1) / (32 * each) * 32;
    const int threads = wanted < kAppendThreads ? wanted : kAppendThreads;
    return interleaved ? launch_grid(append_kernel<T, true>, grid, threads, 0, 1, s, a)
                       : launch_grid(append_kernel<T, false>, grid, threads, 0, 1, s, a);
}

int launch_append(int dtype, const AppendArgs &a, bool interleaved, cudaStream_t s) {
    return dtype == SPECHUB_BF16 ? launch_append_type<__nv_bfloat16>(a, interleaved, s) : launch_append_type<__half>(a, interleaved, s);
}

int launch_accept(const AcceptArgs &a, cudaStream_t s) {
    const int64_t columns = 2LL * a.c.layers * a.c.kv_heads * (a.c.head_dim / 8);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    // as many CTAs as one wave holds: each finds its path's pages once (128 sequences, 32 CTAs of 256 columns each / that: 14.1 / 11.7 us)
    const int64_t all = (columns + kAcceptThreads - 1) / kAcceptThreads, wave = (8 * kSms + a.c.batch - 1) / a.c.batch;
    const int64_t blocks = all < wave ? all : wave;
    cfg.gridDim = dim3(a.c.batch, static_cast<unsigned>(blocks < 65535 ? blocks : 65535));
    cfg.blockDim = dim3(kAcceptThreads); cfg.stream = s;
    return launch_status(cudaLaunchKernelEx(&cfg, accept_kernel, a));
}

}  // namespace spechub
