// Launch functions of the cache operators.  Every function enqueues on `s` and returns a SPECHUB_* code.
#pragma once

#include "spechub_cache_args.cuh"
#include "spechub_launch.h"

namespace spechub {

int launch_append(int dtype, const AppendArgs &a, bool interleaved, cudaStream_t s);
int launch_accept(const AcceptArgs &a, cudaStream_t s);
bool attention_workspace(const CacheArgs &c, int64_t shared_len, size_t *bytes);   // false: more work than a call may have
int launch_attention(int dtype, const AttentionArgs &a, void *workspace, cudaStream_t s);

}  // namespace spechub
