// A thread's own ring in shared memory.
//
// Loads run ahead of their use by stages of such a ring: a thread copies 16 bytes at a time to places that it alone reads,
// so nothing but its own wait stands between the two, registers hold only what is used next, and an SM has
// tens of kilobytes under way.
#pragma once

#include "lm_common.cuh"

namespace sbclm {

// 16 bytes, or zeros (p is then not read).  SHARED: other warps load the same, so it may stay in the first-level cache.
template <bool SHARED> __device__ __forceinline__ void ring_copy16(uint32_t to, const void* p, bool zeros) {
    if (SHARED)
        asm volatile("{\n\t.reg .pred z;\n\tsetp.ne.u32 z, %2, 0;\n\tcp.async.ca.shared.global [%0], [%1], 16, z;\n\t}" ::"r"(to), "l"(p), "r"((uint32_t)zeros) : "memory");
    else
        asm volatile("{\n\t.reg .pred z;\n\tsetp.ne.u32 z, %2, 0;\n\tcp.async.cg.shared.global [%0], [%1], 16, z;\n\t}" ::"r"(to), "l"(p), "r"((uint32_t)zeros) : "memory");
}
template <bool SHARED> __device__ __forceinline__ void ring_copy16(uint32_t to, const void* p) {
    if (SHARED)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(to), "l"(p) : "memory");
    else
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(p) : "memory");
}
__device__ __forceinline__ void ring_store16(uint32_t to, const uint4& v) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 ring_read16(uint32_t from) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from) : "memory");
    return v;
}
__device__ __forceinline__ void ring_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Waits until at most `left` (0 .. 7) of this thread's groups of copies are under way.
__device__ __forceinline__ void ring_wait(int left) {
    switch (left) {
        case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        case 3: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
        case 4: asm volatile("cp.async.wait_group 4;" ::: "memory"); break;
        case 5: asm volatile("cp.async.wait_group 5;" ::: "memory"); break;
        case 6: asm volatile("cp.async.wait_group 6;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 7;" ::: "memory"); break;
    }
}

}  // namespace sbclm
