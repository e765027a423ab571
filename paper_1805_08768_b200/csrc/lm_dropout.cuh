// Dropout into a residual, with random bits that are made where they are used.
//
//   out = residual + (bits(n) >= d ? x * 65536 / (65536 - d) : 0)
//
// Bound by memory (x, the residual and out once each) as long as the generator keeps up: 16 bits decide an
// element, so the ten rounds of one Philox-4x32 (two 32 x 32 bit products each) serve eight.  A probability
// is a multiple of 2^-16, and the scale is that of the multiple taken, so the expectation is exact.
#pragma once

#include "lm_common.cuh"

namespace sbclm {

constexpr int kDropThreads = 256;

struct DropoutArgs {
    const void *x, *residual;
    void* out;
    const long long* rng;
    long long rows, cols, x_stride, residual_stride, out_stride, groups;   // groups of eight elements
    unsigned long long at;
    unsigned dropped;
    float scale;
};

// Philox-4x32-10 of Salmon, Moraes, Dror and Shaw (2011).
__device__ __forceinline__ uint4 philox(uint4 c, uint2 k) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long p = 0xD2511F53ull * c.x, q = 0xCD9E8D57ull * c.z;
        c = make_uint4((uint32_t)(q >> 32) ^ c.y ^ k.x, (uint32_t)q, (uint32_t)(p >> 32) ^ c.w ^ k.y, (uint32_t)p);
        k.x += 0x9E3779B9u, k.y += 0xBB67AE85u;
    }
    return c;
}

// (plain loads: out may be x or the residual)
template <typename T> __device__ __forceinline__ void read8(Pack8<T>& v, const T* p, int have) {
    if (have == 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v.q[i] = reinterpret_cast<const uint4*>(p)[i];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v.e[e] = e < have ? p[e] : from_float<T>(0.f);
    }
}

template <typename T> __device__ __forceinline__ void drop8(Pack8<T>& x, const Pack8<T>& residual, bool add, const uint4& bits, unsigned dropped, float scale) {
    const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t half = e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu;
        const float r = add ? to_float(residual.e[e]) : 0.f;
        x.e[e] = from_float<T>(half >= dropped ? fmaf(to_float(x.e[e]), scale, r) : r);
    }
}

// FLAT: all matrices are without gaps and at multiples of 16 bytes.
template <typename T, bool FLAT> __global__ void __launch_bounds__(kDropThreads) k_dropout(DropoutArgs a) {
    after_earlier_kernels();
    const unsigned long long key = (unsigned long long)a.rng[0], step = (unsigned long long)a.rng[1];
    const uint2 k = make_uint2((uint32_t)key, (uint32_t)(key >> 32));
    const T *x = static_cast<const T*>(a.x), *residual = static_cast<const T*>(a.residual);
    T* out = static_cast<T*>(a.out);
    const long long all = a.rows * a.cols;
    for (long long g = (long long)blockIdx.x * kDropThreads + threadIdx.x; g < a.groups; g += (long long)gridDim.x * kDropThreads) {
        const unsigned long long n = (unsigned long long)g + a.at;
        const int have = (int)min(8ll, all - 8 * g);
        Pack8<T> v, r;
        if (FLAT) {
            read8(v, x + 8 * g, have);
            if (residual) read8(r, residual + 8 * g, have);
        } else {
            long long row = 8 * g / a.cols, col = 8 * g - row * a.cols;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e >= have) break;
                v.e[e] = x[row * a.x_stride + col];
                if (residual) r.e[e] = residual[row * a.residual_stride + col];
                if (++col == a.cols) col = 0, ++row;
            }
        }
        const uint4 bits = philox(make_uint4((uint32_t)n, (uint32_t)(n >> 32), (uint32_t)step, (uint32_t)(step >> 32)), k);
        drop8(v, r, residual != nullptr, bits, a.dropped, a.scale);
        if (FLAT && have == 8) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(out + 8 * g)[i] = v.q[i];
        } else {
            long long row = 8 * g / a.cols, col = 8 * g - row * a.cols;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e >= have) break;
                out[row * a.out_stride + col] = v.e[e];
                if (++col == a.cols) col = 0, ++row;
            }
        }
    }
}

}  // namespace sbclm
