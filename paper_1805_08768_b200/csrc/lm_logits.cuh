// A teacher's largest logits, and the loss and gradient of a student against them.
//
// A row of logits belongs to one block, or to a cluster of blocks where there are few rows (each
// then takes a segment of the row).  Exponentials are powers of two: c = log2(e) / temperature.
#pragma once

#include "lm_common.cuh"

namespace sbclm {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kDistillStats = 8;   // floats per row that the forward call leaves for the backward one

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float infinity() { return __uint_as_float(0x7f800000u); }

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

__device__ __forceinline__ void unpack8(float* x, const Pack8<float>& v) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = v.e[j];
}
__device__ __forceinline__ void unpack8(float* x, const Pack8<__nv_bfloat16>& v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(v.w[j] << 16);
        x[2 * j + 1] = __uint_as_float(v.w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack8(float* x, const Pack8<__half>& v) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __half2float(v.e[j]);
}
__device__ __forceinline__ float max8(const float* x) {
    return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}
__device__ __forceinline__ bool any_nan8(const float* x) {
    float s = 0.f;   // a NaN survives a product with zero, infinities become NaN too (and are looked at)
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(x[j], 0.f, s);
    return s != s;
}

// Sum of 2^((x - m) c) with the largest x so far, m, as its reference.
struct Mass {
    float m, s;
    __device__ __forceinline__ void clear() { m = -infinity(), s = 0.f; }
    __device__ __forceinline__ float base() const { return m == -infinity() ? 0.f : m; }
    __device__ __forceinline__ void add8(const float* x, float c) {
        const float top = max8(x);
        if (top > m) {
            s *= exp2_fast((m - top) * c);
            m = top;
        }
        const float b = base();
        const unsigned long long off = pair(-b, -b), cc = pair(c, c);
        unsigned long long sum = 0;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            float u, v;
            unpair(u, v, mul2(add2(pair(x[j], x[j + 1]), off), cc));
            sum = add2(sum, pair(exp2_fast(u), exp2_fast(v)));
        }
        float u, v;
        unpair(u, v, sum);
        s += u + v;
    }
    __device__ __forceinline__ void join(float om, float os, float c) {
        const float top = fmaxf(m, om), b = top == -infinity() ? 0.f : top;
        s = s * exp2_fast((m - b) * c) + os * exp2_fast((om - b) * c);
        m = top;
    }
    __device__ __forceinline__ void warp(float c) {   // every lane gets the warp's
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            const float om = __shfl_xor_sync(0xffffffffu, m, d), os = __shfl_xor_sync(0xffffffffu, s, d);
            join(om, os, c);
        }
    }
};

// A segment of a row: up to 7 single elements, whole vectors of 8 from a 16-byte boundary on, up to
// 7 single elements.
template <typename T> struct Segment {
    const T* p;
    int first, n;        // element of the row that p points at, elements
    int head, vecs;      // single elements in front, vectors
    __device__ Segment(const T* row, int lo, int hi) : p(row + lo), first(lo), n(hi - lo) {
        head = min(n, (int)((16u - ((uint32_t)(uintptr_t)p & 15u)) & 15u) / (int)sizeof(T));
        vecs = (n - head) / 8;
    }
    __device__ int tail() const { return n - head - 8 * vecs; }
    __device__ void load(Pack8<T>& v, int i) const {
        const uint4* q = reinterpret_cast<const uint4*>(p + head + 8LL * i);
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) v.q[j] = q[j];   // not the read-only path: a gradient may be written in place
    }
    // offset of the single element that thread t takes (threads 0..7 the head, 8..15 the tail), -1: none
    __device__ int single(int t) const {
        if (t < 8) return t < head ? t : -1;
        return t < 16 && t - 8 < tail() ? n - tail() + t - 8 : -1;
    }
};

// The part of [0, cols) that block `rank` of `size` takes, in whole multiples of 64 elements.
__device__ __forceinline__ int segment_start(int cols, int rank, int size) {
    if (rank == size) return cols;
    const int units = (cols + 63) / 64;
    return min(cols, (int)((long long)units * rank / size) * 64);
}

// ---- distillation ------------------------------------------------------------------

struct DistillArgs {
    const void* logits;
    void* grad;
    long long rows, stride, grad_stride;
    int cols, k;
    float temperature, alpha;
    const float* values;       // teacher: rows x k logits
    const int32_t* indices;    // rows x k, negative: slot not used
    const float* rest;         // rows, or null: nothing outside
    const long long* labels;   // rows, negative: none; or null
    const float* grad_loss;    // rows, or null: ones
    float* loss;
    float* stats;
    uint32_t* status;
};

// What a row's elements need for their gradient; logarithms are to base 2, +inf switches a term off.
// Differences of logits are taken before they are scaled, so logits of any size (a type's lowest
// value as a mask) keep their distances.
//   not sent  coef 2^((z - others) c - log_others): its share of the mass outside
//   sent      alpha temperature (2^((z - top) c - log_whole) - 2^((t / temperature - high) log2e - log_total))
//   label's   (1 - alpha) (2^((z - top) log2e - log_whole1) - [is the label])
struct RowStats {
    float others, log_others, top, log_whole, high, log_total, log_whole1, coef;
};

struct DistillShared {
    float m[32], s[32], s1[32];
    RowStats row;
};

// dL/dz of a segment.  sent_*: the row's sent words (shared memory), whose elements are written after all others.
template <typename T, bool CE2>
__device__ __forceinline__ void write_gradient(const DistillArgs& a, long long row, const Segment<T>& seg, const RowStats& r, const int* sent_at,
                                               const float* sent_t, const float* sent_z, int label, float label_z) {
    const int t = threadIdx.x, threads = blockDim.x;
    const float g = a.grad_loss ? a.grad_loss[row] : 1.f;
    const float c = kLog2e / a.temperature, inv = 1.f / a.temperature;
    const float coef = g * r.coef, kl = g * a.alpha * a.temperature;
    const float ce = label >= 0 && r.log_whole1 < infinity() ? g * (1.f - a.alpha) : 0.f;
    T* out = static_cast<T*>(a.grad) + row * a.grad_stride + seg.first;
    const auto off = [&](float z) {
        float v = coef * exp2_fast(fmaf(z - r.others, c, -r.log_others));
        if (CE2) v += ce * exp2_fast(fmaf(z - r.top, kLog2e, -r.log_whole1));
        return v;
    };
    const bool wide = (((uintptr_t)(out + seg.head)) & 15) == 0;
    for (int i = t; i < seg.vecs; i += threads) {
        Pack8<T> v;
        seg.load(v, i);
#pragma unroll
        for (int j = 0; j < 8; ++j) v.e[j] = from_float<T>(off(to_float(v.e[j])));
        store8(out + seg.head + 8LL * i, v, 8, wide ? 16 : (int)sizeof(T));
    }
    const int one = seg.single(t);
    if (one >= 0) out[one] = from_float<T>(off(to_float(seg.p[one])));
    __syncthreads();
    bool has_label = false;
    for (int k = t; k < a.k; k += threads) {
        const int at = sent_at[k];
        if (at < 0) continue;
        if (at == label) has_label = true;
        const int i = at - seg.first;
        if (i < 0 || i >= seg.n) continue;
        const float z = sent_z[k];
        const float q = exp2_fast(fmaf(z - r.top, c, -r.log_whole));
        const float p = exp2_fast(fmaf(sent_t[k] * inv - r.high, kLog2e, -r.log_total));
        float v = kl * (q - p);
        if (ce != 0.f) v += ce * (exp2_fast(fmaf(z - r.top, kLog2e, -r.log_whole1)) - (at == label ? 1.f : 0.f));
        out[i] = from_float<T>(v);
    }
    has_label = __syncthreads_or(has_label);
    if (t == 0 && label >= seg.first && label < seg.first + seg.n && !has_label && ce != 0.f)
        out[label - seg.first] = from_float<T>(off(label_z) - ce);
}

// One row per cluster.  Shared memory: a bit per element of the segment that the teacher sent, then the
// sent words.
template <typename T, bool CE2, bool GRAD> __global__ void __launch_bounds__(1024) k_distill(DistillArgs a) {
    extern __shared__ uint32_t dyn[];
    __shared__ DistillShared sh;
    const int t = threadIdx.x, threads = blockDim.x, warp = t >> 5, lane = t & 31, warps = threads >> 5;
    const int size = (int)cluster_size(), rank = (int)cluster_rank();
    const long long row = blockIdx.x / size;
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    const Segment<T> seg(z, segment_start(a.cols, rank, size), segment_start(a.cols, rank + 1, size));
    const int words = (((a.cols + 63) / 64 + size - 1) / size * 64 + 64) / 32;  // the longest segment's, and the shift of the head
    uint8_t* bits = reinterpret_cast<uint8_t*>(dyn);
    int* sent_at = reinterpret_cast<int*>(dyn + words);
    float* sent_t = reinterpret_cast<float*>(sent_at + a.k);
    float* sent_z = sent_t + a.k;
    const float c = kLog2e / a.temperature;

    for (int i = t; i < words; i += threads) dyn[i] = 0;
    __syncthreads();
    for (int k = t; k < a.k; k += threads) {
        int at = a.indices[row * a.k + k];
        const float tv = a.values[row * a.k + k];
        if (at >= a.cols) {
            if (a.status && rank == 0) atomicOr(a.status, SBC_STATUS_RANGE);
            at = -1;
        }
        float zv = -infinity();
        if (at >= 0) {
            zv = to_float(z[at]);
            const int i = at - seg.first;
            // bit 8 + (offset from the first vector): a vector's bits are one byte, the head's are byte 0
            if (i >= 0 && i < seg.n) atomicOr(&dyn[(i - seg.head + 8) >> 5], 1u << ((i - seg.head + 8) & 31));
        }
        sent_at[k] = at;
        sent_t[k] = at >= 0 ? tv : -infinity();
        sent_z[k] = zv;
    }
    long long label_in = a.labels ? a.labels[row] : -1;
    if (label_in >= a.cols) {
        if (a.status && rank == 0 && t == 0) atomicOr(a.status, SBC_STATUS_RANGE);
        label_in = -1;
    }
    const int label = label_in < 0 ? -1 : (int)label_in;
    const float label_z = label >= 0 ? to_float(z[label]) : 0.f;
    __syncthreads();

    // the student's mass outside the sent words
    float m = -infinity(), base = 0.f, s = 0.f, s1 = 0.f;
    const auto take = [&](float* x) {
        float top = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, x[j]);
        if (top > m) {
            s *= exp2_fast((m - top) * c);
            if (CE2) s1 *= exp2_fast((m - top) * kLog2e);
            m = base = top;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s += exp2_fast((x[j] - base) * c);
            if (CE2) s1 += exp2_fast((x[j] - base) * kLog2e);
        }
    };
    for (int i = t; i < seg.vecs; i += threads) {
        Pack8<T> v;
        seg.load(v, i);
        const uint32_t sent = bits[i + 1];
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = to_float(v.e[j]);
        if (sent) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (sent >> j & 1) x[j] = -infinity();
        }
        take(x);
    }
    const int one = seg.single(t);
    if (one >= 0) {
        const int b = one - seg.head + 8;
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = -infinity();
        if (!(dyn[b >> 5] >> (b & 31) & 1)) x[0] = to_float(seg.p[one]);
        take(x);
    }
    // a warp's, a block's and a cluster's mass
    const auto join = [&](float om, float os, float os1) {
        const float top = fmaxf(m, om), base = top == -infinity() ? 0.f : top;
        s = s * exp2_fast((m - base) * c) + os * exp2_fast((om - base) * c);
        if (CE2) s1 = s1 * exp2_fast((m - base) * kLog2e) + os1 * exp2_fast((om - base) * kLog2e);
        m = top;
    };
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, m, d), os = __shfl_xor_sync(0xffffffffu, s, d);
        join(om, os, CE2 ? __shfl_xor_sync(0xffffffffu, s1, d) : 0.f);
    }
    if (lane == 0) {
        sh.m[warp] = m;
        sh.s[warp] = s;
        sh.s1[warp] = s1;
    }
    if (size > 1)
        cluster_sync();
    else
        __syncthreads();
    if (warp == 0) {
        m = -infinity(), s = 0.f, s1 = 0.f;
        for (int i = lane; i < warps * size; i += 32) {
            const uint32_t r = (uint32_t)(i / warps), w = (uint32_t)(i % warps);
            if (size > 1)
                join(ld_cluster(map_rank(smem_u32(&sh.m[w]), r)), ld_cluster(map_rank(smem_u32(&sh.s[w]), r)),
                     ld_cluster(map_rank(smem_u32(&sh.s1[w]), r)));
            else
                join(sh.m[w], sh.s[w], sh.s1[w]);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            const float om = __shfl_xor_sync(0xffffffffu, m, d), os = __shfl_xor_sync(0xffffffffu, s, d);
            join(om, os, CE2 ? __shfl_xor_sync(0xffffffffu, s1, d) : 0.f);
        }
        // the sent words: maxima, then sums, then the divergence
        const float inv = 1.f / a.temperature;
        const float rest = a.rest ? a.rest[row] : -infinity();
        float top = m, high = rest;
        for (int k = lane; k < a.k; k += 32) {
            top = fmaxf(top, sent_z[k]);
            high = fmaxf(high, sent_t[k] * inv);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, d));
        }
        const bool seen = top > -infinity(), taught = high > -infinity();
        const float top0 = seen ? top : 0.f, high0 = taught ? high : 0.f;
        float mass = 0.f, mass1 = 0.f, total = 0.f;
        for (int k = lane; k < a.k; k += 32) {
            mass += exp2_fast((sent_z[k] - top0) * c);
            mass1 += exp2_fast((sent_z[k] - top0) * kLog2e);
            total += exp2_fast((sent_t[k] * inv - high0) * kLog2e);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            mass += __shfl_xor_sync(0xffffffffu, mass, d);
            mass1 += __shfl_xor_sync(0xffffffffu, mass1, d);
            total += __shfl_xor_sync(0xffffffffu, total, d);
        }
        total += exp2_fast((rest - high0) * kLog2e);
        const float away = s * exp2_fast((m - top0) * c);   // mass outside, below top (none: 0 * 0)
        const float whole = away + mass;
        const float whole1 = (CE2 ? s1 * exp2_fast((m - top0) * kLog2e) : s * exp2_fast((m - top0) * kLog2e)) + mass1;
        const float q_r = away / whole, p_r = exp2_fast((rest - high0) * kLog2e) / total;
        const float shift = (high0 - top0 * inv) + (logf(total) - logf(whole));
        // p d - p + q, every term positive; p (exp(-d) - 1 + d) keeps a small d's digits
        const auto term = [](float p, float q, float d) {
            if (!(p > 0.f)) return q;
            return fabsf(d) < 0.5f ? p * (expm1f(-d) + d) : p * d - p + q;
        };
        float kl = 0.f;
        for (int k = lane; k < a.k; k += 32) {
            if (sent_at[k] < 0) continue;
            const float p = exp2_fast((sent_t[k] * inv - high0) * kLog2e) / total, q = exp2_fast((sent_z[k] - top0) * c) / whole;
            kl += term(p, q, (sent_t[k] - sent_z[k]) * inv - shift);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) kl += __shfl_xor_sync(0xffffffffu, kl, d);
        kl += term(p_r, q_r, ((rest - m * inv) - logf(s)) - shift);
        const float ce_weight = label >= 0 && seen ? 1.f - a.alpha : 0.f;
        const bool live = seen && taught;
        if (lane == 0) {
            float loss = live ? a.alpha * a.temperature * a.temperature * kl : (whole != whole || total != total) ? whole + total : 0.f;
            if (ce_weight != 0.f) loss += ce_weight * (logf(whole1) - (label_z - top0));
            RowStats r;
            r.others = m == -infinity() ? 0.f : m;
            r.log_others = s == 0.f ? infinity() : log2f(s);
            r.top = top0;
            r.log_whole = live ? log2f(whole) : infinity();
            r.high = high0;
            r.log_total = live ? log2f(total) : infinity();
            r.log_whole1 = seen ? log2f(whole1) : infinity();
            r.coef = (live ? a.alpha * a.temperature * (q_r - p_r) : 0.f) + (!CE2 && ce_weight != 0.f ? ce_weight * q_r : 0.f);
            sh.row = r;
            if (rank == 0) {
                if (a.loss) a.loss[row] = loss;
                if (a.stats) {
                    float4* st = reinterpret_cast<float4*>(a.stats + row * kDistillStats);
                    st[0] = make_float4(r.others, r.log_others, r.top, r.log_whole);
                    st[1] = make_float4(r.high, r.log_total, r.log_whole1, r.coef);
                }
            }
        }
    }
    if (GRAD) {
        __syncthreads();
        const RowStats r = sh.row;
        // an in-place gradient may not overtake another block's reading of the sent words
        if (size > 1) cluster_sync();
        write_gradient<T, CE2>(a, row, seg, r, sent_at, sent_t, sent_z, label, label_z);
    } else if (size > 1) {
        cluster_sync();   // the blocks' partial sums are read from each other's shared memory
    }
}

// The backward call: statistics come from the forward one.  `size` blocks share a row, none needs another.
template <typename T, bool CE2> __global__ void __launch_bounds__(1024) k_distill_grad(DistillArgs a, int size) {
    extern __shared__ uint32_t dyn[];
    const int t = threadIdx.x, threads = blockDim.x;
    const long long row = blockIdx.x / size;
    const int rank = (int)(blockIdx.x % size);
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    const Segment<T> seg(z, segment_start(a.cols, rank, size), segment_start(a.cols, rank + 1, size));
    int* sent_at = reinterpret_cast<int*>(dyn);
    float* sent_t = reinterpret_cast<float*>(sent_at + a.k);
    float* sent_z = sent_t + a.k;
    const float4 lo = *reinterpret_cast<const float4*>(a.stats + row * kDistillStats);
    const float4 hi = *reinterpret_cast<const float4*>(a.stats + row * kDistillStats + 4);
    const RowStats r = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    // the words of this segment (the label's place among the sent ones is asked for in every segment)
    for (int k = t; k < a.k; k += threads) {
        const int at = a.indices[row * a.k + k];
        const bool here = at >= seg.first && at < seg.first + seg.n;
        sent_at[k] = at >= 0 && at < a.cols ? at : -1;
        sent_t[k] = here ? a.values[row * a.k + k] : 0.f;
        sent_z[k] = here ? to_float(z[at]) : 0.f;
    }
    const long long label_in = a.labels ? a.labels[row] : -1;
    const int label = label_in >= 0 && label_in < a.cols ? (int)label_in : -1;
    const float label_z = label >= seg.first && label < seg.first + seg.n ? to_float(z[label]) : 0.f;
    __syncthreads();
    write_gradient<T, CE2>(a, row, seg, r, sent_at, sent_t, sent_z, label, label_z);
}

// ---- the largest logits --------------------------------------------------------------

constexpr int kTopMost = SBC_TOP_MOST;
constexpr int kTopRoom = 2048;     // candidates that are ranked: at least kTopMost from each of 8 blocks
constexpr int kTopThreads = 256, kTopWarps = kTopThreads / 32;

struct TopArgs {
    const void* logits;
    long long rows, stride;
    int cols, k;
    float temperature;
    float* values;
    int32_t* indices;
    float* rest;
};

// Order of values as whole numbers: NaN above everything, -0 as +0.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
// Larger value first, then lower index.
__device__ __forceinline__ unsigned long long composite(float x, int index) {
    return (unsigned long long)order_key(x) << 32 | (uint32_t)~index;
}

struct TopShared {
    unsigned long long cand[kTopRoom];
    uint16_t rank[kTopRoom];
    unsigned long long best[kTopMost];   // this block's largest, in order
    float warp_m[2][kTopWarps], warp_s[2][kTopWarps];
    uint32_t warp_bound[kTopWarps];
    float m, s;                          // mass of what this block does not send, s * 2^((x - m) c)
    unsigned long long threshold;
    int count, have;
};

// f(values, index of the first, how many) for a thread's share of a segment.
template <typename T, typename F> __device__ __forceinline__ void for_each8(const Segment<T>& seg, F f) {
    for (int i = threadIdx.x; i < seg.vecs; i += kTopThreads) {
        Pack8<T> v;
        seg.load(v, i);
        float x[8];
        unpack8(x, v);
        f(x, seg.first + seg.head + 8 * i, 8);
    }
    const int one = seg.single(threadIdx.x);
    if (one >= 0) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = -infinity();
        x[0] = to_float(seg.p[one]);
        f(x, seg.first + one, 1);
    }
}

// The block's mass from every thread's; `turn` keeps two uses in a row apart.
__device__ __forceinline__ void block_mass(Mass& a, TopShared& sh, int turn, float c) {
    a.warp(c);
    if ((threadIdx.x & 31) == 0) {
        sh.warp_m[turn][threadIdx.x >> 5] = a.m;
        sh.warp_s[turn][threadIdx.x >> 5] = a.s;
    }
    __syncthreads();
    a.clear();
    for (int i = 0; i < kTopWarps; ++i) a.join(sh.warp_m[turn][i], sh.warp_s[turn][i], c);
}

// Ranks sh.cand[0, n) (all different): sh.rank, and the first min(k, n) in order to sh.best.
__device__ __forceinline__ void rank_candidates(TopShared& sh, int n, int k) {
    for (int i = threadIdx.x; i < n; i += kTopThreads) {
        const unsigned long long mine = sh.cand[i];
        int r = 0;
        for (int j = 0; j < n; ++j) r += sh.cand[j] > mine;
        sh.rank[i] = (uint16_t)r;
        if (r < k) sh.best[r] = mine;
    }
    __syncthreads();
}

// Mass of the ranked candidates that are not sent.
__device__ __forceinline__ void unsent_mass(Mass& a, const TopShared& sh, int n, int k, float c) {
    for (int i = threadIdx.x; i < n; i += kTopThreads)
        if (sh.rank[i] >= k) a.join(key_value((uint32_t)(sh.cand[i] >> 32)), 1.f, c);
}

// The composite at or above which between k and kTopRoom elements lie: the k-th largest one's leading
// digits, found digit by digit until few enough elements share them.  For rows whose values crowd at
// the threshold (ties, masks).
template <typename T> __device__ __noinline__ unsigned long long exact_threshold(const Segment<T>& seg, TopShared& sh, int k) {
    const int t = threadIdx.x, lane = t & 31;
    uint32_t* hist = reinterpret_cast<uint32_t*>(sh.cand);
    unsigned long long prefix = 0;
    int need = k, shift = 64;
    while (shift > 0) {
        const int digit = min(11, shift), upper = shift;
        shift -= digit;
        for (int i = t; i < 2048; i += kTopThreads) hist[i] = 0;
        __syncthreads();
        for_each8(seg, [&](const float* x, int index, int cnt) {
            for (int j = 0; j < cnt; ++j) {
                const unsigned long long mine = composite(x[j], index + j);
                if (upper == 64 || (mine >> upper) == prefix) atomicAdd(&hist[(mine >> shift) & ((1u << digit) - 1)], 1u);
            }
        });
        __syncthreads();
        if (t < 32) {
            // 64 bins a lane, from the top
            uint32_t sum = 0;
            for (int b = 0; b < 64; ++b) sum += hist[(31 - lane) * 64 + b];
            uint32_t upto = sum;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += o;
            }
            uint32_t before = upto - sum;
            if (before < (uint32_t)need && upto >= (uint32_t)need) {
                for (int b = 63; b >= 0; --b) {
                    const uint32_t h = hist[(31 - lane) * 64 + b];
                    if (before + h >= (uint32_t)need) {
                        sh.threshold = prefix << digit | (unsigned long long)((31 - lane) * 64 + b);
                        sh.count = (int)before;
                        sh.have = (int)h;
                        break;
                    }
                    before += h;
                }
            }
        }
        __syncthreads();
        prefix = sh.threshold;
        need -= sh.count;
        const int all = k - need + sh.have;
        __syncthreads();
        if (all <= kTopRoom) break;
    }
    return prefix << shift;
}

// Gathers what is at or above the threshold; the mass of everything else.
template <typename T> __device__ __forceinline__ Mass gather_top(const Segment<T>& seg, TopShared& sh, unsigned long long threshold, float c) {
    const float low = threshold == 0 ? -infinity() : key_value((uint32_t)(threshold >> 32));
    Mass mass;
    mass.clear();
    for_each8(seg, [&](float* x, int index, int n) {
        if (!(max8(x) < low) || any_nan8(x)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= n || x[j] < low) continue;
                const unsigned long long mine = composite(x[j], index + j);
                if (mine >= threshold) {
                    const int at = atomicAdd(&sh.count, 1);
                    if (at < kTopRoom) sh.cand[at] = mine;
                    x[j] = -infinity();
                }
            }
        }
        mass.add8(x, c);
    });
    return mass;
}

// One row per cluster.  A lower bound of the k-th largest: every warp takes the (k / 8)-th largest of
// its lanes' maxima (two groups of elements a lane), the least of these has k elements at or above
// it.  What is (little more than k, where values are spread at random) is ranked by comparing all
// pairs, everything else only adds to the mass.
template <typename T> __global__ void __launch_bounds__(kTopThreads, 5) k_top_logits(TopArgs a) {
    __shared__ TopShared sh;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int size = (int)cluster_size(), rank = (int)cluster_rank();
    const long long row = blockIdx.x / size;
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    const Segment<T> seg(z, segment_start(a.cols, rank, size), segment_start(a.cols, rank + 1, size));
    const float c = kLog2e / a.temperature;
    const int k = min(a.k, seg.n);

    if (t == 0) sh.count = 0;
    unsigned long long threshold = 0;
    if (seg.n > kTopThreads) {
        float m0 = -infinity(), m1 = -infinity();
        for_each8(seg, [&](const float* x, int, int) {
            m0 = fmaxf(fmaxf(m0, fmaxf(x[0], x[1])), fmaxf(x[2], x[3]));
            m1 = fmaxf(fmaxf(m1, fmaxf(x[4], x[5])), fmaxf(x[6], x[7]));
        });
        const uint32_t k0 = order_key(m0) >> 16, k1 = order_key(m1) >> 16;
        const int share = (k + kTopWarps - 1) / kTopWarps;
        uint32_t bound = 0;    // upper half of the threshold's key
        for (uint32_t bit = 0x8000u; bit; bit >>= 1) {
            const uint32_t next = bound | bit;
            if (__popc(__ballot_sync(0xffffffffu, k0 >= next)) + __popc(__ballot_sync(0xffffffffu, k1 >= next)) >= share) bound = next;
        }
        if (lane == 0) sh.warp_bound[warp] = bound;
        __syncthreads();
        for (int i = 0; i < kTopWarps; ++i) bound = min(bound, sh.warp_bound[i]);
        threshold = (unsigned long long)bound << 48;
    }
    __syncthreads();
    Mass mass = gather_top(seg, sh, threshold, c);
    __syncthreads();
    int n = sh.count;
    if (n > kTopRoom) {
        __syncthreads();
        threshold = exact_threshold(seg, sh, k);
        if (t == 0) sh.count = 0;
        __syncthreads();
        mass = gather_top(seg, sh, threshold, c);
        __syncthreads();
        n = sh.count;
    }
    rank_candidates(sh, n, k);
    unsent_mass(mass, sh, n, k, c);
    block_mass(mass, sh, 0, c);
    if (size > 1) {
        if (t == 0) {
            sh.m = mass.m;
            sh.s = mass.s;
            sh.have = k;
        }
        cluster_sync();
        if (rank == 0) {
            // the blocks' lists, ranked together
            n = 0;
            for (int b = 0; b < size; ++b) {
                const int have = (int)__float_as_uint(ld_cluster(map_rank(smem_u32(&sh.have), (uint32_t)b)));
                for (int i = t; i < have; i += kTopThreads) {
                    const uint32_t at = map_rank(smem_u32(&sh.best[i]), (uint32_t)b);
                    sh.cand[n + i] = (unsigned long long)__float_as_uint(ld_cluster(at + 4)) << 32 | __float_as_uint(ld_cluster(at));
                }
                n += have;
            }
            mass.clear();
            if (t < size) mass.join(ld_cluster(map_rank(smem_u32(&sh.m), (uint32_t)t)), ld_cluster(map_rank(smem_u32(&sh.s), (uint32_t)t)), c);
            __syncthreads();
        }
        cluster_sync();   // nobody reads another block's list any more
        if (rank != 0) return;
        rank_candidates(sh, n, a.k);
        unsent_mass(mass, sh, n, a.k, c);
        block_mass(mass, sh, 1, c);
    }
    for (int i = t; i < a.k; i += kTopThreads) {
        const unsigned long long mine = sh.best[i];
        a.values[row * a.k + i] = key_value((uint32_t)(mine >> 32));
        a.indices[row * a.k + i] = (int32_t)~(uint32_t)mine;
    }
    if (t == 0) a.rest[row] = mass.s == 0.f ? -infinity() : mass.m / a.temperature + logf(mass.s);
}

}  // namespace sbclm
