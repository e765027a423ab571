// Shared pieces of the language-model operators (sm_100a): element types, row access at any
// alignment, barriers and bulk copies.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/sbc_lm.h"

namespace sbclm {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Two floats in a register pair: one instruction does both.
__device__ __forceinline__ unsigned long long pair(float a, float b) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(float& a, float& b, unsigned long long p) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Eight consecutive elements in registers.
template <typename T> union Pack8 {
    T e[8];
    uint32_t w[2 * sizeof(T)];
    uint2 d[sizeof(T)];
    uint4 q[sizeof(T) / 2];
};

// Loads `have` (1..8) elements, zeros behind them; `align` is what every such address is a
// multiple of (uniform over the launch), so one branch picks the widest load it allows.
template <typename T> __device__ __forceinline__ void load8(Pack8<T>& v, const T* p, int have, int align) {
    if (have >= 8 && align >= 16) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v.q[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    } else if (have >= 8 && align >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) v.d[i] = __ldg(reinterpret_cast<const uint2*>(p) + i);
    } else if (have >= 8 && align >= 4) {
#pragma unroll
        for (int i = 0; i < 2 * (int)sizeof(T); ++i) v.w[i] = __ldg(reinterpret_cast<const uint32_t*>(p) + i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v.e[i] = i < have ? p[i] : from_float<T>(0.f);
    }
}

// Every kernel here is launched so that its blocks may start while the kernel in front of it on the
// stream ends (its own preparation, barriers and tensor memory, then costs nothing).  This waits until
// everything in front is done and visible; nothing in global memory is touched before it.  The next
// kernel may start from here on.
__device__ __forceinline__ void after_earlier_kernels() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// ---- shared-memory barriers and bulk copies ------------------------------------

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Waits for the phase of the given parity; gives up after a bounded number of tries (each of
// which the hardware may suspend for a while), far beyond what any copy or product takes.
constexpr uint32_t kWaitTries = 1u << 21;
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {
    for (uint32_t i = 0; i < kWaitTries; ++i)
        if (mbar_try(bar, parity)) return true;
    return false;
}

// Waits for copies into shared memory; true if they are late.  Late ones still write, so they are waited for as long
// again before anything takes their place or the block ends.
__device__ __forceinline__ bool copies_late(uint32_t bar, uint32_t parity) {
    uint32_t i = 0;
    while (i < 2 * kWaitTries && !mbar_try(bar, parity)) ++i;
    return i >= kWaitTries;
}

// Arrives at a barrier of a block of the cluster (`bar` from map_rank).  It orders this thread's tensor
// memory accesses only (behind tcgen05.wait and tcgen05.fence); a release to the whole cluster would
// wait for every earlier write, which cost more than the rest of a stage.
__device__ __forceinline__ void mbar_arrive_remote(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Box of a 2-D byte matrix into shared memory; x is the byte within the row (a multiple of 16).
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// The same in a block of a pair; the barrier may be the other block's (`bar` from map_rank).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// A run of bytes (both addresses and the size multiples of 16).
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}

// This thread's own accesses to shared memory come before copies that write over it (started after a
// barrier).
__device__ __forceinline__ void before_copies() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// Address of `local` (a shared-memory address of this block) in block `rank` of the cluster.
__device__ __forceinline__ uint32_t map_rank(uint32_t local, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
    return r;
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

}  // namespace sbclm
