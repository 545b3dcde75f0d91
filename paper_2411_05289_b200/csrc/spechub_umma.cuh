// Tensor-core building blocks (sm_100a): bounded waits on mbarriers, tiled TMA loads, descriptors and issue of tcgen05.mma.
#pragma once

#include <cuda.h>
#include <stdint.h>

#include "spechub_common.cuh"

namespace spechub {

__device__ __forceinline__ uint32_t saddr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
constexpr long long kWaitClocks = 4000000000ll;   // two seconds and more; no wait of a working kernel comes near it

// Wait for a phase, for kWaitClocks at most.  When a wait runs out, `gave_up` (shared memory) is set; every wait of the CTA then
// returns at once, so that the kernel runs to its end (over data that is not valid, within its bounds) and can say so.
__device__ __forceinline__ void bar_wait_one(uint32_t bar, uint32_t parity, volatile int *gave_up) {
    if (bar_try(bar, parity)) return;
    const long long t0 = clock64();
    for (unsigned polls = 1; !bar_try(bar, parity); ++polls) {
        if (polls % 64 != 0) continue;
        if (*gave_up) return;
        if (clock64() - t0 > kWaitClocks) {
            *gave_up = 1;
            return;
        }
    }
}
// ... for whole warps, which are together again afterwards.
__device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up) {
    bar_wait_one(bar, parity, gave_up);
    __syncwarp();
}

// One box of a tiled tensor map into shared memory; out-of-range coordinates of the outer dimensions fill with zeros.
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
// ... out of shared memory (what is out of range is left out); and plain bytes.  Stores are counted in groups of the issuing thread.
__device__ __forceinline__ void tma_store(const CUtensorMap *map, uint32_t src, int x, int y, int z, int w) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void bulk_store(void *dst, uint32_t src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }   // shared memory may change
__device__ __forceinline__ void store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// Operand in shared memory, rows of 128 bytes, swizzled by 128 bytes (eight rows of 1024 bytes repeat, and groups of eight rows follow
// each other): the low word of its descriptor.  `lbo`: bytes between blocks of 64 elements along the axis that lies in a row (operands
// whose rows run along M or N; not used by those whose rows run along K).  16 further bytes are one more.
__device__ __forceinline__ uint32_t operand(uint32_t addr, uint32_t lbo) { return (lbo >> 4 << 16) | addr >> 4; }
constexpr uint32_t kOperandHigh = 2u << 29 | 1u << 14 | 1024u >> 4;
// M = 128, fp32 accumulator, both operands bf16 or both fp16
__host__ __device__ constexpr uint32_t mma_desc(bool bf16, int n, bool b_rows_along_n) {
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (b_rows_along_n ? 1u << 16 : 0u) | (static_cast<uint32_t>(n / 8) << 17) | (8u << 24);
}
// d (tensor memory, 128 x n) = a b (+ d), 16 elements of K; one thread issues
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t desc, bool add) {
    asm volatile("{ .reg .pred p; .reg .b64 x, y; mov.b64 x, {%1, %5}; mov.b64 y, {%2, %5}; setp.ne.u32 p, %4, 0; "
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p; }"
                 ::"r"(d), "r"(a), "r"(b), "r"(desc), "r"(static_cast<uint32_t>(add)), "r"(kOperandHigh) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t desc, bool add) {   // a in tensor memory
    asm volatile("{ .reg .pred p; .reg .b64 y; mov.b64 y, {%2, %5}; setp.ne.u32 p, %4, 0; "
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p; }"
                 ::"r"(d), "r"(a), "r"(b), "r"(desc), "r"(static_cast<uint32_t>(add)), "r"(kOperandHigh) : "memory");
}
// the barrier gets an arrival when everything that this thread has issued to the tensor core is done
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// 32 columns of the warp's 32 lanes, not waited for
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, float *v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
          "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]),
          "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]),
          "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16_async(uint32_t taddr, const uint32_t *v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
          "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
// 8 columns, waited for
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(taddr) : "memory");
}
// waits for all of this thread's loads; v: what they bring (not looked at before)
template <int N> __device__ __forceinline__ void tmem_wait_ld(float (&v)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+f"(v[i]));
}

// How the warpgroups of a block share its registers; at the beginning of what a role alone does.
template <int N> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// two at once
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{ .reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; fma.rn.f32x2 x, x, y, z; mov.b64 {%0, %1}, x; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{ .reg .b64 x, y; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 x, x, y; mov.b64 {%0, %1}, x; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {   // (a NaN is not taken)
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

}  // namespace spechub
