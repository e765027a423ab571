// Layer norm of rows, forward and backward.
//
//   y = h w + b with h = (x - m) s, m the row's mean, s = 1 / sqrt(mean((x - m)^2) + eps)
//   dx = s (t - mean(t) - h mean(t h)) with t = dy w;  dw = sum over rows of dy h,  db = sum of dy
//
// What memory needs is x and y once, and backward x, dy and dx once.  A group of
// threads holds a row in registers, so each is touched once; the variance is the second pass over those
// registers (no difference of large sums).  Groups stay and take row after row, so the weights, and in the
// backward pass the sums over rows, stay too.  A row is cut into granules of eight elements
// whose boundaries in memory are multiples of 16 bytes, wherever the row begins: rows of odd lengths are loaded
// and stored in whole granules but for their ends.  All rows of a group
// begin at the same place within 16 bytes (their distance is a multiple of eight rows), so an element's
// column, weight and sum never change place.
//
// 16384 x 4096 bfloat16 (cold, the buffers before in the caches): forward 79 us for 268 MB, backward 89 us for 403 MB and 7 us for the
// blocks' sums; 8191 x 2601 float16 forward 40 us for 85 MB.  The latency of a row's steps bounds the forward pass: no load of the next
// row runs under this one's sums and stores, and 15 warps an SM issue 22 to 32 instructions an element at half of the rate that
// they could (DRAM at 14 to 34 % of its peak).  Backward, with the next row's loads ahead, 30 an element at 0.64 a cycle (DRAM 52 %).  Rows
// above 8192 elements go through the long kernels, which keep no row: 4096 x 16384 bfloat16 252 us forward, 222 for the input's gradient, 704 with the
// sums over rows, which are read and written in memory for every row.
#pragma once

#include <type_traits>

#include "lm_common.cuh"
#include "lm_product.cuh"

namespace sbclm {

constexpr int kNormThreads = 512;   // most threads of a group of the kernels that hold a row
constexpr int kNormLong = 1024;     // threads of the kernels for longer rows

struct NormArgs {
    const void *x, *dy;
    void* out;               // y or dx (NULL: not asked for)
    const void *weight, *bias;
    float2* stats;
    float* partial;          // backward: sums of blocks, [block][2][cols]; NULL: not asked for
    long long rows, x_stride, dy_stride, out_stride;
    int cols, group, groups;  // threads that share a row, such groups in a block
    int weight_f32;
    float eps;
};

// Sum over the threads of a group, the same bits in all of them.  `buf` alternates between two places, so one barrier
// separates a sum's reads from the next but one's writes.  All threads of the block take part.
__device__ __forceinline__ float2 group_sum(float2 v, float2* red, int group_warps) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, d);
    }
    if (group_warps == 1) return v;
    const int warp = threadIdx.x >> 5, first = warp / group_warps * group_warps;
    if ((threadIdx.x & 31) == 0) red[warp] = v;
    __syncthreads();
    float2 s = red[first];
    for (int i = 1; i < group_warps; ++i) s.x += red[first + i].x, s.y += red[first + i].y;
    return s;
}

__device__ __forceinline__ float weight_at(const void* p, long long i, int f32, const float*) { return static_cast<const float*>(p)[i]; }
template <typename T> __device__ __forceinline__ float weight_at(const void* p, long long i, int f32, const T*) {
    return f32 ? static_cast<const float*>(p)[i] : to_float(static_cast<const T*>(p)[i]);
}

// Where a granule of a row lies: elements lo .. hi of its eight are in the row, the first of which (lo = 0)
// would be column `col`.
struct Granule {
    long long col;
    int lo, hi;
    __device__ __forceinline__ Granule(int i, int phase, int cols) {
        col = 8ll * i - phase;
        lo = (int)max(0ll, -col);
        hi = (int)min(8ll, cols - col);
    }
    __device__ __forceinline__ bool whole() const { return lo == 0 && hi == 8; }
};

// `vec`: whole granules of these rows begin at multiples of 16 bytes.
template <typename T> __device__ __forceinline__ void load_granule(Pack8<T>& v, const T* row, const Granule& g, bool vec) {
    if (vec && g.whole()) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v.q[i] = reinterpret_cast<const uint4*>(row + g.col)[i];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v.e[e] = e >= g.lo && e < g.hi ? row[g.col + e] : from_float<T>(0.f);
    }
}
template <typename T> __device__ __forceinline__ void store_granule(T* row, const Pack8<T>& v, const Granule& g, bool vec) {
    if (vec && g.whole()) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(row + g.col)[i] = v.q[i];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= g.lo && e < g.hi) row[g.col + e] = v.e[e];
    }
}

template <typename T> __device__ __forceinline__ int phase_of(const T* row) { return (int)((uintptr_t)row / sizeof(T) % (16 / sizeof(T))); }

// Whole granules of one row are whole granules of the other's memory too (for all rows of a group, if for its first).
__device__ __forceinline__ bool same_phase(const void* p, const void* q) { return ((uintptr_t)p - (uintptr_t)q) % 16 == 0; }

// Arithmetic is on two neighbours at a time: one instruction does both.
typedef unsigned long long Two;
__device__ __forceinline__ Two both(float v) { return pair(v, v); }
template <typename T> __device__ __forceinline__ void as_pairs(Two* to, const Pack8<T>& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (std::is_same<T, __nv_bfloat16>::value)
            to[i] = pair(__uint_as_float(v.w[i] << 16), __uint_as_float(v.w[i] & 0xffff0000u));
        else
            to[i] = pair(to_float(v.e[2 * i]), to_float(v.e[2 * i + 1]));
    }
}
__device__ __forceinline__ float sum_of(Two v) {
    float a, b;
    unpair(a, b, v);
    return a + b;
}
// What of a thread's eight elements is not in the row becomes zero.
__device__ __forceinline__ void clear_outside(Two* v, const Granule& g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        unpair(a, b, v[i]);
        v[i] = pair(2 * i < g.lo || 2 * i >= g.hi ? 0.f : a, 2 * i + 1 < g.lo || 2 * i + 1 >= g.hi ? 0.f : b);
    }
}


// Eight results of a row; the first of them would be column `col`.
template <typename T> __device__ __forceinline__ void store_row(T* row, const float* f, int col, bool whole, const Granule& g) {
    if (whole) {
        Pack8<T> v;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            if constexpr (sizeof(T) == 4)
                v.e[e] = f[e], v.e[e + 1] = f[e + 1];
            else
                v.w[e / 2] = pack2(f[e], f[e + 1], (const T*)nullptr);
        }
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(row + col)[i] = v.q[i];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= g.lo && e < g.hi) row[col + e] = from_float<T>(f[e]);
    }
}

// Whether all of a row's granules may be loaded whole: rows that are whole granules themselves (no `ends`), or whose neighbours,
// eight elements or more each, cover what a granule reaches beyond the row (at most seven elements on either side).
__host__ __device__ constexpr bool whole_granules_within(long long r, long long rows, int cols, bool ends) {
    return !ends || (cols >= 8 && r > 0 && r < rows - 1);
}

// Few threads hold a row, each up to 64 elements of it: a sum over threads is a wait for all of them.  The weights
// wait in shared memory as fours, so placed that a row's granules begin at them: all rows of a block begin at the same
// place within 16 bytes.

template <typename T, int NV> __global__ void __maxnreg__(NV * sizeof(T) <= 8 ? 80 : 128) k_norm(NormArgs a) {
    __shared__ float2 red[2][kNormThreads / 32];
    extern __shared__ __align__(16) uint8_t raw[];   // weights [w of the first four, of the last four, b likewise][granules] of four floats
    const int t = threadIdx.x % a.group, warps = a.group / 32;
    after_earlier_kernels();
    const long long all = (long long)gridDim.x * a.groups;
    const long long begin = blockIdx.x % 8 + 8ll * a.groups * (blockIdx.x / 8), first = begin + 8 * (threadIdx.x / a.group);
    const T* x = static_cast<const T*>(a.x) + first * a.x_stride;
    T* y = static_cast<T*>(a.out) + first * a.out_stride;
    const int phase = phase_of(x), n = (a.cols + phase + 7) / 8, last = (n - 1) / a.group;   // (last: granule of a thread that may be the row's last)
    const bool vec = same_phase(x, y);
    float4* weights = reinterpret_cast<float4*>(raw);
    for (int i = threadIdx.x; i < n * 2; i += blockDim.x) {
        float w[4], b[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = 4 * i + e - phase;
            const bool is = c >= 0 && c < a.cols;
            w[e] = !is ? 0.f : a.weight ? weight_at(a.weight, c, a.weight_f32, (const T*)nullptr) : 1.f;
            b[e] = is && a.bias ? weight_at(a.bias, c, a.weight_f32, (const T*)nullptr) : 0.f;
        }
        weights[(i & 1) * n + i / 2] = make_float4(w[0], w[1], w[2], w[3]);
        weights[(2 + (i & 1)) * n + i / 2] = make_float4(b[0], b[1], b[2], b[3]);
    }
    __syncthreads();
    const float share = 1.f / (float)a.cols;
    const bool ends = (phase | (a.cols & 7)) != 0;   // a row has granules that are not whole
    for (long long base = begin, r = first; base < a.rows; base += all, r += all, x += all * a.x_stride, y += all * a.out_stride) {
        Pack8<T> p[NV];
        if (r < a.rows && whole_granules_within(r, a.rows, a.cols, ends)) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (t + v * a.group < n)
#pragma unroll
                    for (int i = 0; i < (int)sizeof(T) / 2; ++i) p[v].q[i] = reinterpret_cast<const uint4*>(x + (8 * (t + v * a.group) - phase))[i];
        } else if (r < a.rows) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (t + v * a.group < n) load_granule(p[v], x, Granule(t + v * a.group, phase, a.cols), true);
        }
        // pairs of granule v, what is not in the row as zeros
        const auto pairs_of = [&](Two* f, int v, float mean) {
            as_pairs(f, p[v]);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = add2(f[i], both(-mean));
            if ((v == 0 && ends) || v == last) clear_outside(f, Granule(t + v * a.group, phase, a.cols));
        };
        Two total = 0ull, f[4];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (v > last) break;
            pairs_of(f, v, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) total = add2(total, f[i]);
        }
        const float mean = group_sum(make_float2(sum_of(total), 0.f), red[0], warps).x * share;
        total = 0ull;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (v > last) break;
            pairs_of(f, v, mean);
#pragma unroll
            for (int i = 0; i < 4; ++i) total = fma2(f[i], f[i], total);
        }
        // (the fast root is off by 2^-22 of itself, in 16 bits less than a result's rounding, in 32 about as much as the sum under it)
        const float rstd = rsqrtf(group_sum(make_float2(sum_of(total), 0.f), red[1], warps).x * share + a.eps);
        if (r >= a.rows) continue;
        if (t == 0 && a.stats) a.stats[r] = make_float2(mean, rstd);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = t + v * a.group;
            if (v > last) break;
            if (at >= n) continue;
            const float4 w0 = weights[at], w1 = weights[n + at], b0 = weights[2 * n + at], b1 = weights[3 * n + at];
            pairs_of(f, v, mean);
            float o[8];
            unpair(o[0], o[1], fma2(mul2(f[0], both(rstd)), pair(w0.x, w0.y), pair(b0.x, b0.y)));
            unpair(o[2], o[3], fma2(mul2(f[1], both(rstd)), pair(w0.z, w0.w), pair(b0.z, b0.w)));
            unpair(o[4], o[5], fma2(mul2(f[2], both(rstd)), pair(w1.x, w1.y), pair(b1.x, b1.y)));
            unpair(o[6], o[7], fma2(mul2(f[3], both(rstd)), pair(w1.z, w1.w), pair(b1.z, b1.w)));
            const Granule g(at, phase, a.cols);
            store_row(y, o, 8 * at - phase, vec && ((v > 0 || !ends) && v < last ? true : g.whole()), g);
        }
    }
}

// A thread has one or two granules of a row (their weights and sums over rows take 24 registers each), and loads the next row's while
// it works on this one.  The sums over rows stay in the registers of the threads that hold the columns until the block's last row.
template <typename T, int NV> __global__ void __launch_bounds__(kNormThreads) k_norm_grad(NormArgs a) {
    __shared__ float2 red[2][kNormThreads / 32];
    after_earlier_kernels();
    const int t = threadIdx.x % a.group, warps = a.group / 32;
    const long long all = (long long)gridDim.x * a.groups, first = (long long)blockIdx.x * a.groups + threadIdx.x / a.group;
    const T* x = static_cast<const T*>(a.x) + first * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + first * a.dy_stride;
    T* dx = a.out ? static_cast<T*>(a.out) + first * a.out_stride : nullptr;
    const int phase = phase_of(x);
    const bool vec = same_phase(x, dx), vec_dy = same_phase(x, dy);
    const float share = 1.f / (float)a.cols;
    float w[NV * 8], dw[NV * 8], db[NV * 8];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const Granule g(t + v * a.group, phase, a.cols);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[v * 8 + e] = !(e >= g.lo && e < g.hi) ? 0.f : a.weight ? weight_at(a.weight, g.col + e, a.weight_f32, (const T*)nullptr) : 1.f;
            dw[v * 8 + e] = db[v * 8 + e] = 0.f;
        }
    }
    Pack8<T> next_x[NV], next_dy[NV];
    float2 next_st = make_float2(0.f, 0.f);
    const auto fetch = [&](const T* row, const T* dy_row, long long r) {
        if (r < a.rows) next_st = a.stats[r];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const Granule g(t + v * a.group, phase, a.cols);
            if (r < a.rows && g.hi > g.lo) {
                load_granule(next_x[v], row, g, true);
                load_granule(next_dy[v], dy_row, g, vec_dy);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) next_x[v].e[e] = next_dy[v].e[e] = from_float<T>(0.f);
            }
        }
    };
    fetch(x, dy, first);
    int turn = 0;
    for (long long base = (long long)blockIdx.x * a.groups, r = first; base < a.rows; base += all, r += all, dx += all * a.out_stride, turn ^= 1) {
        const float2 st = next_st;
        float h[NV * 8], d[NV * 8];
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < NV * 8; ++i) {
            // (a place outside of the row has dy = w = 0, and no h of it is used)
            d[i] = to_float(next_dy[i / 8].e[i % 8]);
            h[i] = (to_float(next_x[i / 8].e[i % 8]) - st.x) * st.y;
            dw[i] = fmaf(d[i], h[i], dw[i]);
            db[i] += d[i];
            d[i] *= w[i];
            sum.x += d[i];
            sum.y = fmaf(d[i], h[i], sum.y);
        }
        x += all * a.x_stride;
        dy += all * a.dy_stride;
        fetch(x, dy, r + all);
        if (!a.out) continue;
        const float2 s = group_sum(sum, red[turn], warps);
        if (r >= a.rows) continue;
        const float mean = s.x * share, dot = s.y * share;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const Granule g(t + v * a.group, phase, a.cols);
            if (g.hi <= g.lo) continue;
            Pack8<T> o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o.e[e] = from_float<T>(st.y * (d[v * 8 + e] - mean - h[v * 8 + e] * dot));
            store_granule(dx, o, g, vec);
        }
    }
    if (!a.partial) return;
    // groups may have their granules at other places of a row, so they meet in shared memory, one after the other
    extern __shared__ float sums[];
    float* to = a.partial + (long long)blockIdx.x * 2 * a.cols;
    for (int i = 0; i < a.groups; ++i) {
        if (threadIdx.x / a.group == i) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const Granule g(t + v * a.group, phase, a.cols);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (e < g.lo || e >= g.hi) continue;
                    const long long c = g.col + e;
                    float p = dw[v * 8 + e], q = db[v * 8 + e];
                    if (i > 0) p += sums[c], q += sums[a.cols + c];
                    if (i + 1 < a.groups)
                        sums[c] = p, sums[a.cols + c] = q;
                    else
                        to[c] = p, to[a.cols + c] = q;
                }
            }
        }
        if (i + 1 < a.groups) __syncthreads();
    }
}

// Rows that no group holds: a block reads its row three times (the second and third time from the caches).
template <typename T> __global__ void __launch_bounds__(kNormLong) k_norm_long(NormArgs a) {
    __shared__ float2 red[2][kNormLong / 32];
    after_earlier_kernels();
    const float share = 1.f / (float)a.cols;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
        T* y = static_cast<T*>(a.out) + r * a.out_stride;
        const int phase = phase_of(x), n = (int)(((long long)a.cols + phase + 7) / 8);
        const bool vec = same_phase(x, y);
        float2 sum = make_float2(0.f, 0.f);
        for (int i = threadIdx.x; i < n; i += kNormLong) {
            const Granule g(i, phase, a.cols);
            Pack8<T> v;
            load_granule(v, x, g, true);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum.x += to_float(v.e[e]);
        }
        const float mean = group_sum(sum, red[0], kNormLong / 32).x * share;
        sum.x = 0.f;
        for (int i = threadIdx.x; i < n; i += kNormLong) {
            const Granule g(i, phase, a.cols);
            Pack8<T> v;
            load_granule(v, x, g, true);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = e >= g.lo && e < g.hi ? to_float(v.e[e]) - mean : 0.f;
                sum.x = fmaf(d, d, sum.x);
            }
        }
        const float rstd = 1.f / sqrtf(group_sum(sum, red[1], kNormLong / 32).x * share + a.eps);
        if (threadIdx.x == 0 && a.stats) a.stats[r] = make_float2(mean, rstd);
        for (int i = threadIdx.x; i < n; i += kNormLong) {
            const Granule g(i, phase, a.cols);
            Pack8<T> v;
            load_granule(v, x, g, true);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= g.lo && e < g.hi) {
                    const float w = a.weight ? weight_at(a.weight, g.col + e, a.weight_f32, (const T*)nullptr) : 1.f;
                    const float b = a.bias ? weight_at(a.bias, g.col + e, a.weight_f32, (const T*)nullptr) : 0.f;
                    v.e[e] = from_float<T>(fmaf((to_float(v.e[e]) - mean) * rstd, w, b));
                }
            store_granule(y, v, g, vec);
        }
    }
}

// The block's sums over rows are in its part of `partial`, read and written by the thread that has the column: granules
// here begin at column 0, so rows that begin elsewhere than at 16 bytes are taken element by element.
template <typename T> __global__ void __launch_bounds__(kNormLong) k_norm_grad_long(NormArgs a) {
    __shared__ float2 red[2][kNormLong / 32];
    after_earlier_kernels();
    const float share = 1.f / (float)a.cols;
    const int n = (int)(((long long)a.cols + 7) / 8);
    float* sums = a.partial ? a.partial + (long long)blockIdx.x * 2 * a.cols : nullptr;
    int turn = 0;
    for (long long r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
        const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + r * a.dy_stride;
        T* dx = a.out ? static_cast<T*>(a.out) + r * a.out_stride : nullptr;
        const bool vec_x = (uintptr_t)x % 16 == 0, vec_dy = (uintptr_t)dy % 16 == 0, vec = (uintptr_t)dx % 16 == 0;
        const float2 st = a.stats[r];
        float2 sum = make_float2(0.f, 0.f);
        for (int i = threadIdx.x; i < n; i += kNormLong) {
            const Granule g(i, 0, a.cols);
            Pack8<T> v, d;
            load_granule(v, x, g, vec_x);
            load_granule(d, dy, g, vec_dy);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e >= g.hi) break;
                const float h = (to_float(v.e[e]) - st.x) * st.y, u = to_float(d.e[e]);
                const float w = a.weight ? weight_at(a.weight, g.col + e, a.weight_f32, (const T*)nullptr) : 1.f;
                sum.x = fmaf(u, w, sum.x);
                sum.y = fmaf(u * w, h, sum.y);
                if (sums) {
                    float &dw = sums[g.col + e], &db = sums[a.cols + g.col + e];
                    const bool begun = r != blockIdx.x;
                    dw = fmaf(u, h, begun ? dw : 0.f);
                    db = u + (begun ? db : 0.f);
                }
            }
        }
        if (!a.out) continue;
        const float2 s = group_sum(sum, red[turn], kNormLong / 32);
        const float mean = s.x * share, dot = s.y * share;
        for (int i = threadIdx.x; i < n; i += kNormLong) {
            const Granule g(i, 0, a.cols);
            Pack8<T> v, d;
            load_granule(v, x, g, vec_x);
            load_granule(d, dy, g, vec_dy);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e >= g.hi) break;
                const float h = (to_float(v.e[e]) - st.x) * st.y;
                const float w = a.weight ? weight_at(a.weight, g.col + e, a.weight_f32, (const T*)nullptr) : 1.f;
                v.e[e] = from_float<T>(st.y * (to_float(d.e[e]) * w - mean - h * dot));
            }
            store_granule(dx, v, g, vec);
        }
    }
}

// The blocks' sums of a column: each row of threads takes every sixteenth block's, then one adds up the rows.
constexpr int kNormSumCols = 32, kNormSumRows = 16;
struct NormSumArgs {
    const float* partial;
    void *dweight, *dbias;
    int cols, parts, dtype;
};
__device__ __forceinline__ void store_as(void* p, long long i, float v, int dtype) {
    if (dtype == SBC_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == SBC_BF16) static_cast<__nv_bfloat16*>(p)[i] = from_float<__nv_bfloat16>(v);
    else static_cast<__half*>(p)[i] = from_float<__half>(v);
}
__global__ void __launch_bounds__(kNormSumCols * kNormSumRows) k_norm_sum(NormSumArgs a) {
    __shared__ float part[kNormSumRows][kNormSumCols + 1];
    after_earlier_kernels();
    const int lane = threadIdx.x % kNormSumCols, row = threadIdx.x / kNormSumCols;
    const long long c = (long long)blockIdx.x * kNormSumCols + lane;   // both rows of sums, one behind the other
    float s = 0.f;
    if (c < 2ll * a.cols) {
        const float* p = a.partial + c;
#pragma unroll 8
        for (int i = row; i < a.parts; i += kNormSumRows) s += p[(long long)i * 2 * a.cols];
    }
    part[row][lane] = s;
    __syncthreads();
    if (row != 0 || c >= 2ll * a.cols) return;
#pragma unroll
    for (int i = 1; i < kNormSumRows; ++i) s += part[i][lane];
    if (c < a.cols) {
        if (a.dweight) store_as(a.dweight, c, s, a.dtype);
    } else if (a.dbias) {
        store_as(a.dbias, c - a.cols, s, a.dtype);
    }
}

}  // namespace sbclm
