// Append and accept: the kernels that move entries of the paged cache.
#include "spechub_cache.cuh"
#include "spechub_cache_launch.h"

namespace spechub {

template <class T>
static int launch_append_type(const AppendArgs &a, bool interleaved, cudaStream_t s) {
    const unsigned grid = static_cast<unsigned>(a.c.batch) * a.c.nodes;
    return interleaved ? launch_grid(append_kernel<T, true>, grid, kAppendThreads, 0, 1, s, a)
                       : launch_grid(append_kernel<T, false>, grid, kAppendThreads, 0, 1, s, a);
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
    const int64_t blocks = (columns + kAcceptThreads - 1) / kAcceptThreads;
    cfg.gridDim = dim3(a.c.batch, static_cast<unsigned>(blocks < 65535 ? blocks : 65535));
    cfg.blockDim = dim3(kAcceptThreads); cfg.stream = s;
    return launch_status(cudaLaunchKernelEx(&cfg, accept_kernel, a));
}

}  // namespace spechub
