// Host side that the language-model operators share: checks of matrix arguments, launches, tensor maps.
#pragma once

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "lm_common.cuh"

namespace {

constexpr int64_t kMaxDim = 0x7fffffff;

int width_of(int dtype) { return dtype == SBC_F32 ? 4 : (dtype == SBC_BF16 || dtype == SBC_F16) ? 2 : 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// SMs of the current device (asked for once per device: the question costs as much as half a launch).
int sm_count() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 148;
    if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 148;
    if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

// What every row of a matrix starts at a multiple of, at most 16 bytes.
int row_align(const void* p, int64_t stride, int width) {
    const uintptr_t bits = (uintptr_t)p | (uintptr_t)(stride * width) | 16u;
    return (int)(bits & (~bits + 1));
}

// A matrix argument: base, type and stride fit together.
bool matrix_ok(const void* p, int dtype, int64_t rows, int64_t cols, int64_t stride) {
    const int width = width_of(dtype);
    return p && width && aligned(p, (uintptr_t)width) && rows >= 0 && rows <= kMaxDim && cols >= 1 && cols <= kMaxDim && stride >= cols &&
           stride <= (int64_t)1 << 40;
}

// dtype -> element type
template <typename F> int by_dtype(int dtype, F f) {
    switch (dtype) {
        case SBC_F32: return f((float*)nullptr);
        case SBC_BF16: return f((__nv_bfloat16*)nullptr);
        case SBC_F16: return f((__half*)nullptr);
    }
    return SBC_EINVAL;
}

// Raises a kernel's limit of dynamic shared memory, once per device.
template <auto Kernel> bool allow_smem(int bytes) {
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return true;
    if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

// One launch: `cluster` blocks along `axis` (0: x, 2: z) together, allowed to start while the kernel in
// front ends (the kernels wait for it themselves).
template <typename... P, typename... A>
int launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, int axis, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = axis == 0 ? (unsigned)cluster : 1;
    attr[1].val.clusterDim.y = axis == 1 ? (unsigned)cluster : 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...) == cudaSuccess ? SBC_OK : SBC_ECUDA;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (EncodeTiled)p;
    }();
    return fn;
}

constexpr int kSmemMost = 227 * 1024;

}  // namespace
