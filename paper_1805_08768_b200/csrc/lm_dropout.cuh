// Dropout into a residual, with random bits that are made where they are used.
//
//   out = residual + (bits(n) >= d ? x * 65536 / (65536 - d) : 0)
//
// Bound by memory (x, the residual and out once each) as long as the generator keeps up: 16 bits decide an
// element, so the ten rounds of one Philox-4x32 (two 32 x 32 bit products each) serve eight.  A probability
// is a multiple of 2^-16, and the scale is that of the multiple taken, so the expectation is exact.
//
// 16384 x 4096 bfloat16, into a residual and the gradient: 128 us for 671 MB, 80 % of the copy rate; 193 and 169 instructions for a
// group of eight, about half of them the generator's, whose integer products keep their pipe busy.  Rows with gaps or off 16 bytes are
// taken element by element: the residual's call 213 us instead of 72.
#pragma once

#include "lm_common.cuh"
#include "lm_product.cuh"

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

// Philox-4x32-10 of Salmon, Moraes, Dror and Shaw (2011).  The rounds' keys do not change, so they are made once.
struct PhiloxKeys {
    uint32_t x[10], y[10];
    __device__ __forceinline__ explicit PhiloxKeys(unsigned long long key) {
#pragma unroll
        for (uint32_t i = 0; i < 10; ++i) {
            x[i] = (uint32_t)key + i * 0x9E3779B9u;
            y[i] = (uint32_t)(key >> 32) + i * 0xBB67AE85u;
        }
    }
};
__device__ __forceinline__ uint4 philox(uint4 c, const PhiloxKeys& k) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long p = 0xD2511F53ull * c.x, q = 0xCD9E8D57ull * c.z;
        c = make_uint4((uint32_t)(q >> 32) ^ c.y ^ k.x[i], (uint32_t)q, (uint32_t)(p >> 32) ^ c.w ^ k.y[i], (uint32_t)p);
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

// A half is below d where its word, the half in its upper bits, is below d << 16: the lower half is moved up, the upper one is
// compared with what is below it.  d = 65536 does not fit: then the words are zeros and the border one.
template <typename T> __device__ __forceinline__ void drop8(Pack8<T>& x, const Pack8<T>& residual, bool add, const uint4& bits, uint32_t border, float scale) {
    const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float a = w[e / 2] << 16 >= border ? to_float(x.e[e]) : 0.f, b = w[e / 2] >= border ? to_float(x.e[e + 1]) : 0.f;
        const float p = fmaf(a, scale, add ? to_float(residual.e[e]) : 0.f), q = fmaf(b, scale, add ? to_float(residual.e[e + 1]) : 0.f);
        if constexpr (sizeof(T) == 4)
            x.e[e] = p, x.e[e + 1] = q;
        else
            x.w[e / 2] = pack2(p, q, (const T*)nullptr);
    }
}

// FLAT: all matrices are without gaps and at multiples of 16 bytes.
template <typename T, bool FLAT> __global__ void __launch_bounds__(kDropThreads) k_dropout(DropoutArgs a) {
    after_earlier_kernels();
    const unsigned long long key = (unsigned long long)a.rng[0], step = (unsigned long long)a.rng[1];
    const PhiloxKeys k(key);
    const bool none = a.dropped == 65536;
    const uint32_t border = none ? 1u : a.dropped << 16;
    const auto draw = [&](unsigned long long n) {
        return none ? make_uint4(0, 0, 0, 0) : philox(make_uint4((uint32_t)n, (uint32_t)(n >> 32), (uint32_t)step, (uint32_t)(step >> 32)), k);
    };
    const T *x = static_cast<const T*>(a.x), *residual = static_cast<const T*>(a.residual);
    T* out = static_cast<T*>(a.out);
    const long long all = a.rows * a.cols;
    const long long across = (long long)gridDim.x * kDropThreads;
    if (FLAT) {
        // two groups at a time: both loads are under way while the first one's bits are made
        for (long long g = (long long)blockIdx.x * kDropThreads + threadIdx.x; g < a.groups; g += 2 * across) {
            Pack8<T> v[2], r[2];
            int have[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const long long at = g + i * across;
                have[i] = (int)max(0ll, min(8ll, all - 8 * at));
                if (have[i] > 0) {
                    read8(v[i], x + 8 * at, have[i]);
                    if (residual) read8(r[i], residual + 8 * at, have[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const long long at = g + i * across;
                const unsigned long long n = (unsigned long long)at + a.at;
                const uint4 bits = draw(n);
                drop8(v[i], r[i], residual != nullptr, bits, border, a.scale);
                if (have[i] == 8) {
#pragma unroll
                    for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4*>(out + 8 * at)[j] = v[i].q[j];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < have[i]) out[8 * at + e] = v[i].e[e];
                }
            }
        }
    } else {
        for (long long g = (long long)blockIdx.x * kDropThreads + threadIdx.x; g < a.groups; g += across) {
            const unsigned long long n = (unsigned long long)g + a.at;
            const int have = (int)min(8ll, all - 8 * g);
            Pack8<T> v, r;
            const long long first_row = 8 * g / a.cols, first_col = 8 * g - first_row * a.cols;
            long long row = first_row, col = first_col;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e >= have) break;
                v.e[e] = x[row * a.x_stride + col];
                if (residual) r.e[e] = residual[row * a.residual_stride + col];
                if (++col == a.cols) col = 0, ++row;
            }
            const uint4 bits = draw(n);
            drop8(v, r, residual != nullptr, bits, border, a.scale);
            row = first_row, col = first_col;
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
