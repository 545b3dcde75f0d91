// Device-side helpers of the cache operators: page look-up, pairs of 16-bit elements.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "spechub.h"
#include "spechub_cache.h"
#include "spechub_cache_args.cuh"
#include "spechub_common.cuh"

namespace spechub {

// Page of `slot` in row `row` of the page table, or -1 if there is none.
__device__ __forceinline__ int page_of(const CacheArgs &c, const int32_t *row, int64_t slot) {
    const int64_t at = slot >> c.page_shift;
    if (at >= c.table_width) return -1;
    const int page = row[at];
    return page >= 0 && page < c.pages ? page : -1;
}

template <class T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
template <class T> __device__ __forceinline__ uint32_t pack2(float a, float b);   // rounded to nearest even
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 r = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&r);
}

}  // namespace spechub
