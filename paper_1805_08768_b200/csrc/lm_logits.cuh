// A teacher's largest logits, and the loss and gradient of a student against them.
//
// A row of logits belongs to one block, or to a cluster of blocks where there are few rows or the row
// is long; each then takes a segment of the row, which it keeps in shared memory between its passes
// over it.  Exponentials are powers of two: c = log2(e) / temperature.
#pragma once

#include "lm_common.cuh"

namespace sbclm {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float infinity() { return __uint_as_float(0x7f800000u); }

// A granule: 16 bytes of a row, the unit of loads and stores.
template <typename T> struct Gran {
    static constexpr int E = 16 / (int)sizeof(T);
};
__device__ __forceinline__ void unpack(float* x, const uint4& q, const float*) {
    x[0] = __uint_as_float(q.x), x[1] = __uint_as_float(q.y), x[2] = __uint_as_float(q.z), x[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack(float* x, const uint4& q, const __nv_bfloat16*) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(float* x, const uint4& q, const __half*) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        x[2 * j] = f.x, x[2 * j + 1] = f.y;
    }
}
__device__ __forceinline__ uint4 pack(const float* x, const float*) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <typename P, typename F> __device__ __forceinline__ uint4 pack_pairs(const float* x, F two) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const P h = two(x[2 * j], x[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack(const float* x, const __nv_bfloat16*) {
    return pack_pairs<__nv_bfloat162>(x, [](float a, float b) { return __floats2bfloat162_rn(a, b); });
}
__device__ __forceinline__ uint4 pack(const float* x, const __half*) {
    return pack_pairs<__half2>(x, [](float a, float b) { return __floats2half2_rn(a, b); });
}
// Running maxima of granules, two groups of elements apart.  NAN: a NaN is the largest (otherwise it
// does not count).
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
template <typename T, bool NAN_> struct GranMax;
template <bool NAN_> struct GranMax<float, NAN_> {
    float m0 = -__builtin_huge_valf(), m1 = -__builtin_huge_valf();
    static __device__ __forceinline__ float max2(float a, float b) { return NAN_ ? max_nan(a, b) : fmaxf(a, b); }
    __device__ __forceinline__ void add(const uint4& q) {
        m0 = max2(m0, max2(__uint_as_float(q.x), __uint_as_float(q.y)));
        m1 = max2(m1, max2(__uint_as_float(q.z), __uint_as_float(q.w)));
    }
    __device__ __forceinline__ void add(const GranMax& o) { m0 = max2(m0, o.m0), m1 = max2(m1, o.m1); }
    __device__ __forceinline__ float first() const { return m0; }
    __device__ __forceinline__ float second() const { return m1; }
    __device__ __forceinline__ float get() const { return max2(m0, m1); }
};
template <typename T2, typename F> __device__ __forceinline__ uint32_t on_words(uint32_t a, uint32_t b, F f) {
    const T2 r = f(*reinterpret_cast<const T2*>(&a), *reinterpret_cast<const T2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <typename T, typename T2, bool NAN_> struct WordMax {
    uint32_t w;
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        return on_words<T2>(a, b, [](T2 x, T2 y) { return NAN_ ? __hmax2_nan(x, y) : __hmax2(x, y); });
    }
    __device__ __forceinline__ void add(const uint4& q) { w = max2(max2(w, max2(q.x, q.y)), max2(q.z, q.w)); }
    __device__ __forceinline__ void add(const WordMax& o) { w = max2(w, o.w); }
    __device__ __forceinline__ float get() const { return NAN_ ? max_nan(first(), second()) : fmaxf(first(), second()); }
    __device__ __forceinline__ float first() const { return to_float(reinterpret_cast<const T*>(&w)[0]); }
    __device__ __forceinline__ float second() const { return to_float(reinterpret_cast<const T*>(&w)[1]); }
};
template <bool NAN_> struct GranMax<__nv_bfloat16, NAN_> : WordMax<__nv_bfloat16, __nv_bfloat162, NAN_> {
    __device__ __forceinline__ GranMax() { this->w = 0xff80ff80u; }
};
template <bool NAN_> struct GranMax<__half, NAN_> : WordMax<__half, __half2, NAN_> {
    __device__ __forceinline__ GranMax() { this->w = 0xfc00fc00u; }
};

// x c - m c for x near or below m, ready for 2^: in one rounding of the product's difference where |m c|
// is moderate (NEAR; what the rounded m c lacks is returned by `lack` and made up for once per sum),
// else from the difference of the logits, which stays exact for logits of any size (a type's lowest
// value as a mask).
constexpr float kNear = 1048576.f;
template <bool NEAR> struct Scale {
    unsigned long long mul, off;
    __device__ __forceinline__ Scale(float m, float c) : mul(pair(c, c)) {
        const float o = NEAR ? -__fmul_rn(m, c) : -m;
        off = pair(o, o);
    }
    __device__ __forceinline__ unsigned long long two(unsigned long long x) const {
        return NEAR ? fma2(x, mul, off) : mul2(add2(x, off), mul);
    }
    static __device__ __forceinline__ float lack(float m, float c) { return NEAR ? fmaf(m, c, -__fmul_rn(m, c)) : 0.f; }
};

// The same for an infinite reference.
struct InfiniteScale {
    static __device__ __forceinline__ float one(float x) { return x == __builtin_huge_valf() ? 0.f : x != x ? x : -__builtin_huge_valf(); }
    __device__ __forceinline__ unsigned long long two(unsigned long long x) const {
        float u, v;
        unpair(u, v, x);
        return pair(one(u), one(v));
    }
    static __device__ __forceinline__ float lack(float, float) { return 0.f; }
};

// sum += 2^(...) over a granule
template <int E, typename S> __device__ __forceinline__ void add_powers(unsigned long long& sum, const float* x, const S& scale) {
#pragma unroll
    for (int j = 0; j < E; j += 2) {
        float u, v;
        unpair(u, v, scale.two(pair(x[j], x[j + 1])));
        sum = add2(sum, pair(exp2_fast(u), exp2_fast(v)));
    }
}
__device__ __forceinline__ float sum_of(unsigned long long p) {
    float u, v;
    unpair(u, v, p);
    return __fadd_rn(u, v);
}
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}

// Sums of 2^((x - m) c), and with CE2 of 2^((x - m) log2e), with the largest x as their reference.
// Every operation is rounded by itself wherever this is compiled, so that two calls and one for both
// give the same bits.  INF: infinities count, each as the reference itself (2^0); otherwise they make a NaN.
template <bool CE2, bool INF = false> struct Mass {
    float m = -__builtin_huge_valf(), s = 0.f, s1 = 0.f;
    __device__ __forceinline__ float base() const { return m == -infinity() ? 0.f : m; }
    static __device__ __forceinline__ float gap(float x, float base) { return INF && x == base ? 0.f : x - base; }
    __device__ __forceinline__ void join(float om, float os, float os1, float c) {
        const float top = fmaxf(m, om), b = top == -infinity() ? 0.f : top;
        s = fmaf(s, exp2_fast(__fmul_rn(gap(m, b), c)), __fmul_rn(os, exp2_fast(__fmul_rn(gap(om, b), c))));
        if (CE2) s1 = fmaf(s1, exp2_fast(__fmul_rn(gap(m, b), kLog2e)), __fmul_rn(os1, exp2_fast(__fmul_rn(gap(om, b), kLog2e))));
        m = top;
    }
    // every lane gets the warp's
    __device__ __forceinline__ void lanes(float c) {
        const float top = warp_max(m), b = top == -infinity() ? 0.f : top;
        s = warp_sum(__fmul_rn(s, exp2_fast(__fmul_rn(gap(m, b), c))));
        if (CE2) s1 = warp_sum(__fmul_rn(s1, exp2_fast(__fmul_rn(gap(m, b), kLog2e))));
        m = top;
    }
};
using RestMass = Mass<false, true>;   // of what is not sent

// The part of [0, cols) that block `rank` of 2^shift takes, in whole multiples of 64 elements.
__device__ __forceinline__ int segment_start(int cols, int rank, int shift) {
    if (rank >> shift) return cols;
    const uint32_t units = ((uint32_t)cols + 63u) / 64u;
    return min(cols, (int)(units * (uint32_t)rank >> shift) * 64);
}

// n elements of a row from p on, cut into granules where 16-byte boundaries fall: element i sits in
// slot `phase` + i, slots that are no elements read as -inf.
template <typename T> struct Cut {
    static constexpr int E = Gran<T>::E;
    const T* p;
    int n, phase, grans;
    __device__ __forceinline__ Cut(const T* at, int count) : p(at), n(count) {
        phase = (int)((uint32_t)(uintptr_t)p & 15u) / (int)sizeof(T);
        grans = n > 0 ? (phase + n + E - 1) / E : 0;
    }
    __device__ __forceinline__ bool whole(int g) const { return g * E >= phase && g * E + E <= phase + n; }
    // From global memory (not the read-only path: a gradient may be written in place).
    __device__ __forceinline__ uint4 load(int g) const {
        if (whole(g)) return *reinterpret_cast<const uint4*>(p - phase + (long long)g * E);
        uint4 q;
        T* e = reinterpret_cast<T*>(&q);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int i = g * E + j - phase;
            e[j] = i >= 0 && i < n ? p[i] : from_float<T>(-infinity());
        }
        return q;
    }
    // Into shared memory: the whole granules by bulk copies that one thread starts (`bar` counts their
    // bytes), the edges by the threads that hold them.
    __device__ __forceinline__ void stage(T* room, uint32_t bar) const {
        const int g0 = phase > 0 ? 1 : 0, g1 = (phase + n) / E;
        if (threadIdx.x == 0) {
            const int whole_bytes = max(g1 - g0, 0) * 16;
            mbar_expect(bar, (uint32_t)whole_bytes);
            const uint8_t* src = reinterpret_cast<const uint8_t*>(p - phase) + 16LL * g0;
            for (int at = 0; at < whole_bytes; at += kBulk)
                bulk_load(smem_u32(room + g0 * E) + (uint32_t)at, src + at, (uint32_t)min(kBulk, whole_bytes - at), bar);
        } else if (threadIdx.x <= 2) {
            const int g = threadIdx.x == 1 ? 0 : grans - 1;
            if (grans > 0 && !whole(g)) *reinterpret_cast<uint4*>(room + g * E) = load(g);
        }
    }
    static constexpr int kBulk = 16384;
};

// ---- distillation ------------------------------------------------------------------

struct DistillArgs {
    const void* logits;
    void* grad;
    long long rows, stride, grad_stride;
    int cols, k;
    int part;                  // elements of a segment that a block holds at a time (a multiple of 8)
    int shift;                 // 2^shift blocks share a row
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

// Gradients of a row's elements.
template <typename T, bool CE2> struct Slope {
    RowStats r;
    float c, inv, kl, ce, coef;
    __device__ __forceinline__ Slope(const DistillArgs& a, const RowStats& stats, float g, bool label) : r(stats) {
        c = kLog2e / a.temperature, inv = 1.f / a.temperature;
        kl = __fmul_rn(g, __fmul_rn(a.alpha, a.temperature));
        ce = label && r.log_whole1 < infinity() ? __fmul_rn(g, 1.f - a.alpha) : 0.f;
        coef = __fmul_rn(g, r.coef);
    }
    __device__ __forceinline__ bool near() const {
        return fmaxf(fabsf(r.others), fabsf(r.top)) * fmaxf(c, kLog2e) < kNear;
    }
    // Elements of granules, two at a time: y = coef 2^(..) / others' sum, + ce 2^(..) / the whole's
    template <bool NEAR> struct Granules {
        Scale<NEAR> scale, scale1;
        unsigned long long by, by1;
        __device__ __forceinline__ Granules(const Slope& s) : scale(s.r.others, s.c), scale1(s.r.top, kLog2e) {
            const float k = __fmul_rn(s.coef, exp2_fast(-Scale<NEAR>::lack(s.r.others, s.c) - s.r.log_others));
            const float k1 = __fmul_rn(s.ce, exp2_fast(-Scale<NEAR>::lack(s.r.top, kLog2e) - s.r.log_whole1));
            by = pair(k, k), by1 = pair(k1, k1);
        }
        __device__ __forceinline__ unsigned long long two(unsigned long long z) const {
            float u, v;
            unpair(u, v, scale.two(z));
            unsigned long long y = mul2(by, pair(exp2_fast(u), exp2_fast(v)));
            if (CE2) {
                unpair(u, v, scale1.two(z));
                y = fma2(by1, pair(exp2_fast(u), exp2_fast(v)), y);
            }
            return y;
        }
        __device__ __forceinline__ uint4 granule(const uint4& q) const {
            constexpr int E = Gran<T>::E;
            float x[E];
            unpack(x, q, (const T*)nullptr);
#pragma unroll
            for (int j = 0; j < E; j += 2) unpair(x[j], x[j + 1], two(pair(x[j], x[j + 1])));
            return pack(x, (const T*)nullptr);
        }
    };
    template <typename F> __device__ __forceinline__ void granules(F f) const {
        if (near())
            f(Granules<true>(*this));
        else
            f(Granules<false>(*this));
    }
    // The label's, where the teacher did not send it.
    __device__ __forceinline__ float unsent_label(float z) const {
        float y = 0.f;
        granules([&](const auto& g) {
            float v;
            unpair(y, v, g.two(pair(z, z)));
        });
        return y - ce;
    }
    __device__ __forceinline__ float sent(float z, float t, bool is_label) const {
        const float q = exp2_fast(fmaf(z - r.top, c, -r.log_whole)), p = exp2_fast(fmaf(__fmul_rn(t, inv) - r.high, kLog2e, -r.log_total));
        float v = __fmul_rn(kl, q - p);
        if (ce != 0.f) v = fmaf(ce, exp2_fast(fmaf(z - r.top, kLog2e, -r.log_whole1)) - (is_label ? 1.f : 0.f), v);
        return v;
    }
};

// Writes granule g of a cut to `out` (where the cut's first element goes).
template <typename T> __device__ __forceinline__ void store_granule(T* out, const Cut<T>& cut, int g, const uint4& q, bool wide) {
    constexpr int E = Gran<T>::E;
    const int i0 = g * E - cut.phase;
    if (wide && cut.whole(g)) {
        *reinterpret_cast<uint4*>(out + i0) = q;
        return;
    }
    const T* e = reinterpret_cast<const T*>(&q);
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (i0 + j >= 0 && i0 + j < cut.n) out[i0 + j] = e[j];
}
// make(load(i)) for every granule i of a cut: whole ones side by side, four loads ahead of their stores
// (a gradient written in place only replaces what its own thread has read), then the edges.
template <typename T, typename L, typename M> __device__ __forceinline__ void store_all(T* out, const Cut<T>& cut, L load, M make) {
    constexpr int E = Gran<T>::E, kAhead = 4;
    const int t = threadIdx.x, threads = blockDim.x;
    if (((uint32_t)(uintptr_t)out & 15u) != (uint32_t)cut.phase * sizeof(T)) {
        for (int i = t; i < cut.grans; i += threads) store_granule(out, cut, i, make(load(i)), false);
        return;
    }
    const int g0 = cut.phase > 0 ? 1 : 0, g1 = (cut.phase + cut.n) / E;
    uint4* wide = reinterpret_cast<uint4*>(out - cut.phase);
    int i = g0 + t;
    for (; i + (kAhead - 1) * threads < g1; i += kAhead * threads) {
        uint4 q[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) q[j] = load(i + j * threads);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) wide[i + j * threads] = make(q[j]);
    }
    for (; i < g1; i += threads) wide[i] = make(load(i));
    if (t < 2) {
        const int e = t == 0 ? 0 : cut.grans - 1;
        if (cut.grans > 0 && !cut.whole(e) && (t == 0 || e > 0)) store_granule(out, cut, e, make(load(e)), false);
    }
}

// After all other elements of a segment are written: the sent words', and a label's that was not sent.
// words: elements of this segment at sent_at (negative: none of this block's).
template <typename T, typename S>
__device__ __forceinline__ void write_sent(T* out, const S& slope, int first, int n, int k, const int* sent_at, const float* sent_t,
                                           const float* sent_z, int label, float label_z) {
    bool has_label = false;
    for (int i = threadIdx.x; i < k; i += blockDim.x) {
        const int at = sent_at[i];
        if (at < 0) continue;
        has_label |= at == label;
        out[at - first] = from_float<T>(slope.sent(sent_z[i], sent_t[i], at == label));
    }
    has_label = __syncthreads_or(has_label);
    if (threadIdx.x == 0 && label >= first && label < first + n && !has_label && slope.ce != 0.f)
        out[label - first] = from_float<T>(slope.unsent_label(label_z));
}

constexpr int kDistillThreads = 128, kDistillWarps = kDistillThreads / 32;

struct DistillShared {
    uint64_t bar;                                                    // the logits' arrival
    float om[kDistillWarps], os[kDistillWarps], os1[kDistillWarps];  // a warp's mass of words that were not sent
    float sm[kDistillWarps], ss[kDistillWarps], ss1[kDistillWarps];  // ... that were
    float tm[kDistillWarps], ts[kDistillWarps];                      // ... of the teacher's sent words (natural units)
    float kl[kDistillWarps], kl_block;
    RowStats row;
    float shift, inv_total, inv_whole;                               // for the divergence's terms
    float rest_term, cross, missing;                                 // the loss's other parts
};

// One row per cluster; a block keeps its segment in shared memory, with the sent words taken out (-inf),
// so the sum over the others is a plain one.  Longer segments are taken in parts, for a gradient twice
// (the forward call sums in the same order, so two calls and one give the same bits).
//
// log q = z c ln 2 - logZ with logZ from a running maximum and sum; the loss is the sum of p d - p + q over
// sent words and the rest, d = log p - log q, times alpha tau^2; its gradient is alpha tau (q - p) at a sent
// word, alpha tau q (1 - p_rest / q_rest) at another.  4480 x 10000 bfloat16 with its gradient 48 us,
// 3.8 TB/s; its bytes alone take 28 us.  Bound by the latency between a block's steps (load, maximum and
// sum, join, statistics, store), so small blocks of which many share an SM.
// 4095 x 50001 bfloat16 forward 92 us, 4.4 TB/s: parts of 40 KB leave five blocks on an SM.
template <typename T, bool CE2, bool GRAD> __global__ void __launch_bounds__(kDistillThreads, 10) k_distill(DistillArgs a) {
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ DistillShared sh;
    constexpr int E = Gran<T>::E;
    const int t = threadIdx.x, threads = blockDim.x, warp = t >> 5, lane = t & 31, warps = threads >> 5;
    const int size = 1 << a.shift, rank = (int)(blockIdx.x & (uint32_t)(size - 1));
    const long long row = blockIdx.x >> a.shift;
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    const int first = segment_start(a.cols, rank, a.shift), n = segment_start(a.cols, rank + 1, a.shift) - first;
    T* held = reinterpret_cast<T*>(dyn);
    float* sent_t = reinterpret_cast<float*>(dyn + (size_t)a.part * sizeof(T));
    float* sent_z = sent_t + a.k;
    int* sent_at = reinterpret_cast<int*>(sent_z + a.k);
    const float c = kLog2e / a.temperature, inv = 1.f / a.temperature;

    const uint32_t bar = smem_u32(&sh.bar);
    if (t == 0) {
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    after_earlier_kernels();
    const Cut<T> segment(z + first, n);
    const int part_grans = a.part / E, parts = max(1, (segment.grans + part_grans - 1) / part_grans);   // whole granules
    const auto part_of = [&](int part) {
        const int slot = part * part_grans * E, from = max(0, slot - segment.phase), to = min(n, slot + part_grans * E - segment.phase);
        return Cut<T>(segment.p + from, max(0, to - from));
    };
    Cut<T> cut = part_of(0);
    cut.stage(held, bar);
    uint32_t phase = 0;
    bool late = false;
    // the barrier in front of it is for the edges, and for its own initialisation; a thread that was late once waits no
    // more, and the one that starts the copies starts no more
    const auto landed = [&] {
        __syncthreads();
        if (!late) late = copies_late(bar, phase);
        phase ^= 1;
    };
    // the teacher, while the logits are on their way
    long long label_in = a.labels ? a.labels[row] : -1;
    if (label_in >= a.cols) {
        if (a.status && rank == 0 && t == 0) atomicOr(a.status, SBC_STATUS_RANGE);
        label_in = -1;
    }
    const int label = label_in < 0 ? -1 : (int)label_in;
    const float label_z = label >= 0 ? to_float(z[label]) : 0.f;
    const float rest = a.rest ? a.rest[row] : -infinity();
    const float g = GRAD && a.grad_loss ? a.grad_loss[row] : 1.f;
    Mass<false> teacher;
    for (int i = t; i < a.k; i += threads) {
        int at = a.indices[row * a.k + i];
        const float tv = a.values[row * a.k + i];
        if (at >= a.cols) {
            if (a.status && rank == 0) atomicOr(a.status, SBC_STATUS_RANGE);
            at = -1;
        }
        const bool here = at >= first && at < first + n;
        sent_at[i] = here ? at : -1;
        sent_t[i] = at >= 0 ? tv : -infinity();
        if (at >= 0) teacher.join(__fmul_rn(tv, inv), 1.f, 0.f, kLog2e);
    }
    teacher.lanes(kLog2e);
    if (lane == 0) sh.tm[warp] = teacher.m, sh.ts[warp] = teacher.s;

    Mass<CE2> others, sent;
    for (int part = 0; part < parts; ++part) {
        if (part > 0) {
            before_copies();
            __syncthreads();
            cut = part_of(part);
            if (!late) cut.stage(held, bar);
        }
        landed();
        const int lo = first + (int)(cut.p - segment.p);
        for (int i = t; i < a.k; i += threads) {
            const int at = sent_at[i] - lo;
            if (sent_at[i] < 0 || at < 0 || at >= cut.n) continue;
            const float zv = to_float(held[cut.phase + at]);
            held[cut.phase + at] = from_float<T>(-infinity());
            sent_z[i] = zv;
            sent.join(zv, 1.f, 1.f, c);
        }
        __syncthreads();
        GranMax<T, false> top;
#pragma unroll 4
        for (int i = t; i < cut.grans; i += threads) top.add(*reinterpret_cast<const uint4*>(held + i * E));
        Mass<CE2> mine;
        mine.m = top.get();
        const float base = mine.base();
        const auto add_all = [&](const auto& scale, const auto& scale1) {
            unsigned long long sum = 0, sum1 = 0;
#pragma unroll 2
            for (int i = t; i < cut.grans; i += threads) {
                float x[E];
                unpack(x, *reinterpret_cast<const uint4*>(held + i * E), (const T*)nullptr);
                add_powers<E>(sum, x, scale);
                if (CE2) add_powers<E>(sum1, x, scale1);
            }
            mine.s = __fmul_rn(sum_of(sum), exp2_fast(-scale.lack(base, c)));
            if (CE2) mine.s1 = __fmul_rn(sum_of(sum1), exp2_fast(-scale1.lack(base, kLog2e)));
        };
        if (fabsf(base) * fmaxf(c, kLog2e) < kNear)
            add_all(Scale<true>(base, c), Scale<true>(base, kLog2e));
        else
            add_all(Scale<false>(base, c), Scale<false>(base, kLog2e));
        if (parts == 1)
            others = mine;
        else
            others.join(mine.m, mine.s, mine.s1, c);
    }
    if (late) others.s = __uint_as_float(0x7fffffffu);   // the logits never came: everything is NaN
    others.lanes(c);
    sent.lanes(c);
    if (lane == 0) {
        sh.om[warp] = others.m, sh.os[warp] = others.s, sh.os1[warp] = others.s1;
        sh.sm[warp] = sent.m, sh.ss[warp] = sent.s, sh.ss1[warp] = sent.s1;
    }
    if (size > 1)
        cluster_sync();
    else
        __syncthreads();
    // p d - p + q of an outcome, d = log p - log q: their sum is the divergence, every one is positive, and
    // p (exp(-d) - 1 + d) keeps a small d's digits
    const auto term = [](float p, float q, float d) {
        if (!(p > 0.f)) return q;
        return fabsf(d) < 0.5f ? p * (expm1f(-d) + d) : p * d - p + q;
    };
    if (warp == 0) {
        others = Mass<CE2>(), sent = Mass<CE2>(), teacher = Mass<false>();
        for (int i = lane; i < warps * size; i += 32) {
            const uint32_t r = (uint32_t)(i / warps), w = (uint32_t)(i % warps);
            const auto at = [&](float* p) { return size > 1 ? ld_cluster(map_rank(smem_u32(p), r)) : *p; };
            others.join(at(&sh.om[w]), at(&sh.os[w]), CE2 ? at(&sh.os1[w]) : 0.f, c);
            sent.join(at(&sh.sm[w]), at(&sh.ss[w]), CE2 ? at(&sh.ss1[w]) : 0.f, c);
        }
        if (lane < warps) teacher.m = sh.tm[lane], teacher.s = sh.ts[lane];
        others.lanes(c), sent.lanes(c), teacher.lanes(kLog2e);
        const float m = others.m, s = others.s;
        teacher.join(rest, 1.f, 0.f, kLog2e);
        Mass<CE2> all = others;
        all.join(sent.m, sent.s, sent.s1, c);
        const bool seen = all.m > -infinity(), taught = teacher.m > -infinity();
        const float top = all.base(), high = teacher.base(), whole = all.s, total = teacher.s;
        const float whole1 = CE2 ? all.s1 : whole;
        // one logarithm and one division for all of them, a lane each
        const float arg = lane == 0 ? s : lane == 1 ? whole : lane == 2 ? total : whole1;
        const float log_arg = log2f(arg), inv_arg = 1.f / arg;
        const float log_s = __shfl_sync(0xffffffffu, log_arg, 0), log_whole = __shfl_sync(0xffffffffu, log_arg, 1),
                    log_total = __shfl_sync(0xffffffffu, log_arg, 2), log_whole1 = __shfl_sync(0xffffffffu, log_arg, 3);
        const float inv_whole = __shfl_sync(0xffffffffu, inv_arg, 1), inv_total = __shfl_sync(0xffffffffu, inv_arg, 2);
        const float q_r = __fmul_rn(__fmul_rn(s, exp2_fast(__fmul_rn(m - top, c))), inv_whole);
        const float p_r = __fmul_rn(exp2_fast(__fmul_rn(rest - high, kLog2e)), inv_total);
        const float ce_weight = label >= 0 && seen ? 1.f - a.alpha : 0.f;
        const bool live = seen && taught;
        RowStats r;
        r.others = others.base();
        r.log_others = s == 0.f ? infinity() : log_s;
        r.top = top;
        r.log_whole = live ? log_whole : infinity();
        r.high = high;
        r.log_total = live ? log_total : infinity();
        r.log_whole1 = seen ? log_whole1 : infinity();
        r.coef = __fadd_rn(live ? __fmul_rn(a.alpha * a.temperature, q_r - p_r) : 0.f, !CE2 && ce_weight != 0.f ? __fmul_rn(ce_weight, q_r) : 0.f);
        if (s != s) r.coef = s;   // a NaN among the others is everybody's
        // log p - log q: differences from the largest first, so that logits of any size (a type's lowest value as a mask) leave
        // the logarithms their digits
        const float shift = (log_total - log_whole) * kLn2;
        if (lane == 0) {
            sh.row = r;
            sh.shift = shift;
            sh.inv_total = inv_total;
            sh.inv_whole = inv_whole;
            sh.rest_term = live ? term(p_r, q_r, fmaf(-log_s, kLn2, fmaf(top - m, inv, rest - high)) - shift) : 0.f;
            sh.cross = ce_weight != 0.f ? ce_weight * (log_whole1 * kLn2 - (label_z - top)) : 0.f;
            // (without weight it is left out, not multiplied by 0: it may be infinite)
            sh.missing = live && a.alpha > 0.f ? 1.f : (whole != whole || total != total) ? whole + total : 0.f;   // the divergence's factor
            if (a.stats && rank == 0) {
                float4* st = reinterpret_cast<float4*>(a.stats + row * SBC_DISTILL_STATS);
                st[0] = make_float4(r.others, r.log_others, r.top, r.log_whole);
                st[1] = make_float4(r.high, r.log_total, r.log_whole1, r.coef);
            }
        }
    }
    __syncthreads();
    const RowStats r = sh.row;
    T* out = nullptr;
    Slope<T, CE2> slope(a, r, g, label >= 0);
    if (GRAD) {
        out = static_cast<T*>(a.grad) + row * a.grad_stride + first;
        for (int part = 0; part < parts; ++part) {
            if (parts > 1) {
                before_copies();
                __syncthreads();
                cut = part_of(part);
                if (!late) cut.stage(held, bar);
                landed();
                if (late) slope.coef = __uint_as_float(0x7fffffffu);   // this thread's granules become NaN
            }
            const int lo = (int)(cut.p - segment.p);
            slope.granules([&](const auto& gr) {
                store_all(out + lo, cut, [&](int i) { return *reinterpret_cast<const uint4*>(held + i * E); }, [&](const uint4& q) { return gr.granule(q); });
            });
        }
    }
    if (GRAD) __syncthreads();   // the sent words' gradients come after all others'
    const bool live = sh.missing == 1.f;
    float kl = 0.f;
    bool has_label = false;
    for (int i = t; i < a.k; i += threads) {
        const int at = sent_at[i];
        if (at < 0) continue;
        const float zv = sent_z[i], tv = sent_t[i];
        if (live) {
            const float over = __fmul_rn(tv, inv) - r.high, under = zv - r.top;
            const float p = exp2_fast(over * kLog2e) * sh.inv_total, q = exp2_fast(under * c) * sh.inv_whole;
            kl += term(p, q, fmaf(-under, inv, over) - sh.shift);
        }
        if (GRAD) {
            has_label |= at == label;
            out[at - first] = from_float<T>(slope.sent(zv, tv, at == label));
        }
    }
    kl = warp_sum(kl);
    if (lane == 0) sh.kl[warp] = kl;
    has_label = __syncthreads_or(has_label);
    if (size > 1) {
        if (t == 0) {
            kl = 0.f;
            for (int i = 0; i < warps; ++i) kl += sh.kl[i];
            sh.kl_block = kl;
        }
        cluster_sync();
    }
    if (rank == 0 && warp == 0) {
        const int parts_of = size > 1 ? size : warps;
        kl = lane >= parts_of ? 0.f : size > 1 ? ld_cluster(map_rank(smem_u32(&sh.kl_block), (uint32_t)lane)) : sh.kl[lane];
        kl = warp_sum(kl);
        if (lane == 0) a.loss[row] = (live ? a.alpha * a.temperature * a.temperature * (kl + sh.rest_term) : sh.missing) + sh.cross;
    }
    if (late && a.status) atomicOr(a.status, SBC_STATUS_TIMEOUT);
    if (GRAD && t == 0 && label >= first && label < first + n && !has_label && slope.ce != 0.f)
        out[label - first] = from_float<T>(slope.unsent_label(label_z));
    if (size > 1) cluster_sync();   // blocks read each other's sums up to here
}

// The backward call: statistics come from the forward one.  Blocks that share a row do not need one another.
// Every logit is read once, every gradient written once: bound by memory, 4095 x 50001 bfloat16 145 us,
// 5.6 TB/s.
template <typename T, bool CE2> __global__ void __launch_bounds__(256, 4) k_distill_grad(DistillArgs a) {
    extern __shared__ uint32_t words[];
    const int t = threadIdx.x, threads = blockDim.x;
    const int rank = (int)(blockIdx.x & ((1u << a.shift) - 1u));
    const long long row = blockIdx.x >> a.shift;
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    const int first = segment_start(a.cols, rank, a.shift), n = segment_start(a.cols, rank + 1, a.shift) - first;
    const Cut<T> cut(z + first, n);
    float* sent_t = reinterpret_cast<float*>(words);
    float* sent_z = sent_t + a.k;
    int* sent_at = reinterpret_cast<int*>(sent_z + a.k);
    after_earlier_kernels();
    const float4 lo = *reinterpret_cast<const float4*>(a.stats + row * SBC_DISTILL_STATS);
    const float4 hi = *reinterpret_cast<const float4*>(a.stats + row * SBC_DISTILL_STATS + 4);
    const RowStats r = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    const long long label_in = a.labels ? a.labels[row] : -1;
    const int label = label_in >= 0 && label_in < a.cols ? (int)label_in : -1;
    const float label_z = label >= first && label < first + n ? to_float(z[label]) : 0.f;
    for (int i = t; i < a.k; i += threads) {
        const int at = a.indices[row * a.k + i];
        const bool here = at >= first && at < first + n;
        sent_at[i] = here ? at : -1;
        if (here) sent_t[i] = a.values[row * a.k + i], sent_z[i] = to_float(z[at]);
    }
    const Slope<T, CE2> slope(a, r, a.grad_loss ? a.grad_loss[row] : 1.f, label >= 0);
    __syncthreads();   // an in-place gradient comes after the words are read
    T* out = static_cast<T*>(a.grad) + row * a.grad_stride + first;
    slope.granules([&](const auto& gr) {
        store_all(
            out, cut,
            [&](int i) { return cut.whole(i) ? *reinterpret_cast<const uint4*>(cut.p - cut.phase + (long long)i * Gran<T>::E) : cut.load(i); },
            [&](const uint4& q) { return gr.granule(q); });
    });
    __syncthreads();
    write_sent(out, slope, first, n, a.k, sent_at, sent_t, sent_z, label, label_z);
}

// ---- the largest logits --------------------------------------------------------------

struct TopArgs {
    const void* logits;
    long long rows, stride;
    int cols, k;
    int shift;                 // 2^shift blocks share a row
    int room;                  // candidates a block can hold: at least 2 k, and k for every block of a row; whole eights
    float temperature;
    float* values;
    int32_t* indices;
    float* rest;
};

// So many candidates are ranked by comparing all pairs, more by bins (us by pairs / bins: 2240 x 10000 for
// 64 29.3 / 30.1, for 16 23.2 / 27.2; 1000 x 20000 for 256 62.6 / 31.5).
constexpr int kTopPairs = 192;
constexpr int kTopBins = 256;
constexpr int kTopThreads = 256, kTopWarps = kTopThreads / 32;

// Order of values as whole numbers: NaN above everything, -0 as +0.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
constexpr uint32_t kLowestKey = 0x00800000u;   // of the lowest finite number: -inf lies below
// Larger value first, then lower index.
__device__ __forceinline__ unsigned long long composite(float x, int index) {
    return (unsigned long long)order_key(x) << 32 | (uint32_t)~index;
}

struct TopShared {
    uint64_t bar;                            // the logits' arrival
    unsigned long long best[SBC_TOP_MOST];   // this block's largest, in order
    uint32_t bins[kTopBins + 1];             // how many a bin holds, then where it starts
    uint32_t next[kTopBins];                 // where a bin's next candidate goes
    uint32_t warp_hi[kTopWarps], warp_lo[kTopWarps];
    float warp_m[2][kTopWarps], warp_s[2][kTopWarps];
    uint32_t warp_bound[kTopWarps];
    float m, s;                              // mass of what this block does not send
    unsigned long long threshold;
    int count, have;
};
// What a block gathers, behind the logits it holds: larger value first, then lower index.  A candidate is
// stored as its value's bits and its index, and becomes a composite when it is ranked.
constexpr int kCandidateBytes = 8 + 2;   // in the list and in its order
struct Candidates {
    unsigned long long* at;
    uint16_t* order;           // by bin
    int room;
};

// (the compiler would gather a warp's additions first, which costs more than these few)
__device__ __forceinline__ uint32_t add_shared(void* p, uint32_t n = 1) {
    uint32_t r;
    asm volatile("atom.shared.add.u32 %0, [%1], %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(n) : "memory");
    return r;
}

// A segment's granules, held in shared memory or read from global memory.
template <typename T, bool HELD> struct Source {
    const Cut<T>& cut;
    T* held;
    __device__ __forceinline__ uint4 get(int g) const {
        if (HELD) return *reinterpret_cast<const uint4*>(held + g * Gran<T>::E);
        return cut.load(g);
    }
};

// The block's mass from every thread's, for warp 0; `turn` keeps two uses in a row apart.
__device__ __forceinline__ void block_mass(RestMass& a, TopShared& sh, int turn, float c) {
    a.lanes(c);
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) {
        sh.warp_m[turn][threadIdx.x >> 5] = a.m;
        sh.warp_s[turn][threadIdx.x >> 5] = a.s;
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        a = RestMass();
        if (lane < warps) a.m = sh.warp_m[turn][lane], a.s = sh.warp_s[turn][lane];
        a.lanes(c);
    }
}

// Bins for keys between lo and hi, the largest in bin 0: equal parts of the values' range where that is
// finite (logits crowd around zero only in their keys), else of the keys'.  A larger key is never in a
// later bin.
struct KeyBins {
    uint32_t hi;
    int shift;
    float top, scale;
    __device__ __forceinline__ KeyBins(uint32_t hi_key, uint32_t lo_key) : hi(hi_key), top(key_value(hi_key)) {
        shift = max(0, 32 - __clz((int)(hi_key - lo_key)) - 8);   // 2^8 bins
        const float range = top - key_value(lo_key);
        scale = range > 1e-30f && range < 1e30f ? ((float)kTopBins - 0.5f) / range : 0.f;
    }
    __device__ __forceinline__ uint32_t of(uint32_t key) const {
        if (scale > 0.f) return min((uint32_t)kTopBins - 1u, (uint32_t)((top - key_value(key)) * scale));
        return (hi - key) >> shift;
    }
};

// Ranks the candidates [0, n) (all different): the first min(k, n) in order to sh.best, the others join
// the mass of what is not sent.  Few are compared with each other; otherwise the keys' range is cut into
// equal bins, largest first, and a candidate's rank is its bin's start and how many of the same bin are
// larger.
__device__ __forceinline__ void rank_candidates(TopShared& sh, const Candidates& cand, int n, int k, RestMass& mass, float c) {
    const int t = threadIdx.x, threads = blockDim.x, lane = t & 31, warps = threads >> 5;
    if (n <= kTopPairs) {
        for (int i = t; i < n; i += threads) {
            const unsigned long long mine = cand.at[i];
            int r = 0;
            int j = 0;
            for (; j + 2 <= n; j += 2) {
                const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(cand.at + j);
                r += (two.x > mine) + (two.y > mine);
            }
            if (j < n) r += cand.at[j] > mine;
            if (r < k)
                sh.best[r] = mine;
            else
                mass.join(key_value((uint32_t)(mine >> 32)), 1.f, 0.f, c);
        }
        __syncthreads();
        return;
    }
    uint32_t hi = 0, lo = 0xffffffffu;
    for (int i = t; i < n; i += threads) {
        const uint32_t key = (uint32_t)(cand.at[i] >> 32);
        hi = max(hi, key), lo = min(lo, key);
    }
    hi = __reduce_max_sync(0xffffffffu, hi), lo = __reduce_min_sync(0xffffffffu, lo);
    if (lane == 0) sh.warp_hi[t >> 5] = hi, sh.warp_lo[t >> 5] = lo;
    for (int i = t; i < kTopBins; i += threads) sh.bins[i] = 0;
    __syncthreads();
    hi = __reduce_max_sync(0xffffffffu, sh.warp_hi[min(lane, warps - 1)]);
    lo = __reduce_min_sync(0xffffffffu, sh.warp_lo[min(lane, warps - 1)]);
    const KeyBins bins(hi, lo);
    const auto bin_of = [&](unsigned long long x) { return bins.of((uint32_t)(x >> 32)); };
    for (int i = t; i < n; i += threads) add_shared(&sh.bins[bin_of(cand.at[i])]);
    __syncthreads();
    if (t < 32) {
        uint32_t count[kTopBins / 32], sum = 0;
#pragma unroll
        for (int b = 0; b < kTopBins / 32; ++b) {
            count[b] = sum;
            sum += sh.bins[lane * (kTopBins / 32) + b];
        }
        uint32_t upto = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
#pragma unroll
        for (int b = 0; b < kTopBins / 32; ++b) sh.bins[lane * (kTopBins / 32) + b] = sh.next[lane * (kTopBins / 32) + b] = upto - sum + count[b];
        if (lane == 31) sh.bins[kTopBins] = upto;
    }
    __syncthreads();
    for (int i = t; i < n; i += threads) cand.order[add_shared(&sh.next[bin_of(cand.at[i])])] = (uint16_t)i;
    __syncthreads();
    for (int i = t; i < n; i += threads) {
        const unsigned long long mine = cand.at[i];
        const uint32_t bin = bin_of(mine);
        int r = (int)sh.bins[bin];
        if (r < k) {
            const int end = (int)sh.bins[bin + 1];
            for (int j = (int)sh.bins[bin]; j < end; ++j) r += cand.at[cand.order[j]] > mine;
        }
        if (r < k)
            sh.best[r] = mine;
        else
            mass.join(key_value((uint32_t)(mine >> 32)), 1.f, 0.f, c);
    }
    __syncthreads();
}

// The composite at or above which between k and `cand.room` elements lie: the k-th largest one's leading
// digits, found digit by digit until few enough elements share them.  For rows whose values crowd at
// the threshold (ties).
template <typename T> __device__ __noinline__ unsigned long long exact_threshold(const Cut<T>& cut, int first, TopShared& sh, const Candidates& cand, int k) {
    constexpr int E = Gran<T>::E;
    const int t = threadIdx.x, lane = t & 31;
    uint32_t* hist = sh.bins;
    unsigned long long prefix = 0;
    int need = k, shift = 64;
    while (shift > 0) {
        const int digit = 8, upper = shift;
        shift -= digit;
        for (int i = t; i < 256; i += blockDim.x) hist[i] = 0;
        __syncthreads();
        for (int g = t; g < cut.grans; g += blockDim.x) {
            float x[E];
            unpack(x, cut.load(g), (const T*)nullptr);
            int bin = -1, times = 0;   // equal neighbours are counted together
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int i = g * E + j - cut.phase;
                if (i < 0 || i >= cut.n) continue;
                const unsigned long long mine = composite(x[j], first + i);
                if (upper < 64 && (mine >> upper) != prefix) continue;
                const int b = (int)((mine >> shift) & ((1u << digit) - 1));
                if (b != bin) {
                    if (times) atomicAdd(&hist[bin], (uint32_t)times);
                    bin = b, times = 0;
                }
                ++times;
            }
            if (times) atomicAdd(&hist[bin], (uint32_t)times);
        }
        __syncthreads();
        if (t < 32) {
            // 8 bins a lane, from the top
            uint32_t sum = 0;
            for (int b = 0; b < 8; ++b) sum += hist[(31 - lane) * 8 + b];
            uint32_t upto = sum;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += o;
            }
            uint32_t before = upto - sum;
            if (before < (uint32_t)need && upto >= (uint32_t)need) {
                for (int b = 7; b >= 0; --b) {
                    const uint32_t h = hist[(31 - lane) * 8 + b];
                    if (before + h >= (uint32_t)need) {
                        sh.threshold = prefix << digit | (unsigned long long)((31 - lane) * 8 + b);
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
        if (all <= cand.room) break;
    }
    return prefix << shift;
}

// Gathers what is at or above the threshold; returns the thread's mass of everything else.  PLAIN: the
// threshold is a value's (whole composites need not be compared) above -inf.
template <typename T, bool HELD, bool PLAIN>
__device__ __forceinline__ RestMass gather_top(const Source<T, HELD>& src, int first, TopShared& sh, const Candidates& cand,
                                                  unsigned long long threshold, float c) {
    constexpr int E = Gran<T>::E;
    const Cut<T>& cut = src.cut;
    const float low = !PLAIN && threshold == 0 ? -infinity() : key_value((uint32_t)(threshold >> 32));
    GranMax<T, true> top;
    float top_left = -infinity();   // of granules that hold a candidate, where they are not held: what is left
    const int threads = blockDim.x;
    // (all lanes of a warp go around together: apart, each would take its own turns)
    for (int gw = threadIdx.x & ~31; gw < cut.grans; gw += 32 * threads) {
        const int g0 = gw + (threadIdx.x & 31);
        // mark the granules first: a warp then goes through its fullest lane's, not through all that any lane has
        uint32_t marked = 0;
#pragma unroll 4
        for (int j = 0; j < 32; ++j) {
            const int g = g0 + j * threads;
            if (gw + j * threads >= cut.grans) break;
            if (g >= cut.grans) continue;
            GranMax<T, true> here;
            here.add(src.get(g));
            if (here.get() < low)
                top.add(here);
            else
                marked |= 1u << j;
        }
        while (__any_sync(0xffffffffu, marked != 0)) {
            const bool any = marked != 0;
            const int g = any ? g0 + (__ffs((int)marked) - 1) * threads : 0;
            marked &= marked - 1;
            float x[E];
            unpack(x, src.get(g), (const T*)nullptr);
            const int i0 = g * E - cut.phase;
            uint32_t hits = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                bool hit = !(x[j] < low);
                if (!PLAIN) hit = hit && i0 + j >= 0 && i0 + j < cut.n && composite(x[j], first + i0 + j) >= threshold;
                hits |= hit ? 1u << j : 0u;
            }
            if (!any) hits = 0;
            if (!HELD) {
#pragma unroll
                for (int j = 0; j < E; ++j) top_left = any && !(hits >> j & 1) ? fmaxf(top_left, x[j]) : top_left;
            }
            uint32_t at = 0;
            if (hits) at = add_shared(&sh.count, (uint32_t)__popc(hits));
            __syncwarp();
            while (__any_sync(0xffffffffu, hits != 0)) {
                const int j = __ffs((int)hits) - 1;
                if (hits) {
                    const float v = to_float(HELD ? src.held[g * E + j] : cut.p[i0 + j]);
                    if (at < (uint32_t)cand.room) cand.at[at] = (unsigned long long)__float_as_uint(v) << 32 | (uint32_t)(first + i0 + j);
                    if (HELD) src.held[g * E + j] = from_float<T>(-infinity());
                }
                ++at;
                hits &= hits - 1;
                __syncwarp();
            }
            if (HELD && any) top.add(src.get(g));
        }
    }
    RestMass mass;
    mass.m = fmaxf(top.get(), top_left);
    const float base = mass.base();
    const auto add_all = [&](const auto& scale) {
        unsigned long long sum = 0;
#pragma unroll 2
        for (int g = threadIdx.x; g < cut.grans; g += blockDim.x) {
            const uint4 q = src.get(g);
            float x[E];
            unpack(x, q, (const T*)nullptr);
            if (!HELD) {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (!(x[j] < low) && composite(x[j], first + g * E + j - cut.phase) >= threshold) x[j] = -infinity();
            }
            add_powers<E>(sum, x, scale);
        }
        mass.s = __fmul_rn(sum_of(sum), exp2_fast(-scale.lack(base, c)));
    };
    if (fabsf(base) * c < kNear)
        add_all(Scale<true>(base, c));
    else if (PLAIN || base != infinity())   // (no infinity is below a value's threshold)
        add_all(Scale<false>(base, c));
    else
        add_all(InfiniteScale());
    return mass;
}

// One row per cluster.  A lower bound of the k-th largest: every warp takes the (k / warps)-th largest
// of its lanes' maxima (two groups of elements a lane), the least of these has k elements at or above
// it.  What is (little more than k, where values are spread at random) is ranked by the cluster's
// first block, everything else only adds to the mass.
//
// A warp that owns fewer groups than its share bounds nothing, and rows of more columns than there is room for
// candidates then always take exact_threshold: 16-bit rows of 513 to 768 columns (k up to 8), to 824 (64), to
// 1912 (256); float32 rows of 513 to 944 (k of 100 to 200).  2240 bfloat16 rows for 64: 512 columns 23 us, 768 33 us,
// 1000 18 us; for 128: 512 36 us, 1848 67 us, 2000 36 us.
//
// rest = log of the sum of exp(z / tau) over what is not sent, from a running maximum and sum.  2240 x 10000
// bfloat16 for 64: 29 us, 1.6 TB/s; its bytes alone take 7 us.  Bound by instructions and the latency between a row's
// steps (0.62 a cycle and scheduler): a quarter exponentials, a fifth ranking, a sixth the bound.
template <typename T, bool HELD> __global__ void __launch_bounds__(kTopThreads, 4) k_top_logits(TopArgs a) {
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ TopShared sh;
    const int t = threadIdx.x, threads = blockDim.x, lane = t & 31, warp = t >> 5, warps = threads >> 5;
    const int size = 1 << a.shift, rank = (int)(blockIdx.x & (uint32_t)(size - 1));
    const long long row = blockIdx.x >> a.shift;
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    const int first = segment_start(a.cols, rank, a.shift), len = segment_start(a.cols, rank + 1, a.shift) - first;
    const Cut<T> cut(z + first, len);
    Candidates cand;
    cand.at = reinterpret_cast<unsigned long long*>(dyn);
    cand.order = reinterpret_cast<uint16_t*>(cand.at + a.room);
    cand.room = a.room;
    const Source<T, HELD> src = {cut, reinterpret_cast<T*>(cand.order + a.room)};
    const float c = kLog2e / a.temperature;
    const int k = a.k;
    const auto sync = [&] {
        if (size > 1)
            cluster_sync();
        else
            __syncthreads();
    };

    bool late = false;
    if (t == 0) sh.count = 0;
    const uint32_t bar = smem_u32(&sh.bar);
    if (HELD && t == 0) {
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    after_earlier_kernels();
    if (HELD) {
        cut.stage(src.held, bar);
        __syncthreads();
        late = copies_late(bar, 0);
    }
    unsigned long long threshold = 0;
    const bool bounded = a.cols > threads;
    RestMass mass;
    if (bounded) {
        GranMax<T, true> top;
#pragma unroll 4
        for (int g = t; g < cut.grans; g += threads) top.add(src.get(g));
        const uint32_t k0 = order_key(top.first()) >> 16, k1 = order_key(top.second()) >> 16;
        const int share = (k + warps * size - 1) / (warps * size);
        // upper half of the threshold's key: what all have in common, then bit by bit
        const uint32_t all = __reduce_and_sync(0xffffffffu, k0 & k1), any = __reduce_or_sync(0xffffffffu, k0 | k1);
        const int bits = 32 - __clz((int)(all ^ any));
        uint32_t bound = all >> bits << bits;
        for (int b = bits - 1; b >= 0; --b) {
            const uint32_t next = bound | 1u << b;
            if (__popc(__ballot_sync(0xffffffffu, k0 >= next)) + __popc(__ballot_sync(0xffffffffu, k1 >= next)) >= share) bound = next;
        }
        if (lane == 0) sh.warp_bound[warp] = bound;
        sync();
        for (int i = lane; i < warps * size; i += 32) {
            const uint32_t r = (uint32_t)(i / warps), w = (uint32_t)(i % warps);
            bound = min(bound, size > 1 ? __float_as_uint(ld_cluster(map_rank(smem_u32(&sh.warp_bound[w]), r))) : sh.warp_bound[w]);
        }
        bound = __reduce_min_sync(0xffffffffu, bound);
        // -inf is asked for only where nothing else is left
        threshold = (unsigned long long)max(bound << 16, kLowestKey) << 32;
        mass = gather_top<T, HELD, true>(src, first, sh, cand, threshold, c);
    } else {
        __syncthreads();
        mass = gather_top<T, HELD, false>(src, first, sh, cand, threshold, c);
    }
    if (late) mass.s = __uint_as_float(0x7fffffffu);   // the logits never came
    sync();
    // how many candidates the cluster has
    const auto have = [&](int b) { return size > 1 ? (int)__float_as_uint(ld_cluster(map_rank(smem_u32(&sh.count), (uint32_t)b))) : sh.count; };
    int n = 0;
    for (int b = 0; b < size; ++b) n += min(have(b), a.room + 1);
    const auto compose = [&](int count) {
        for (int i = t; i < count; i += threads) {
            const unsigned long long raw = cand.at[i];
            cand.at[i] = composite(__uint_as_float((uint32_t)(raw >> 32)), (int)(uint32_t)raw);
        }
        __syncthreads();
    };
    if (n > a.room) {
        // more than can be ranked: every block keeps no more than k
        sync();
        const int most = min(k, len);
        if (most > 0) {
            threshold = exact_threshold(cut, first, sh, cand, most);
            if (t == 0) sh.count = 0;
            __syncthreads();
            mass = gather_top<T, false, false>(Source<T, false>{cut, nullptr}, first, sh, cand, threshold, c);
            __syncthreads();
            compose(sh.count);
            if (size > 1) {
                rank_candidates(sh, cand, sh.count, most, mass, c);
                for (int i = t; i < most; i += threads) cand.at[i] = sh.best[i];
                if (t == 0) sh.count = most;
            }
        }
        sync();
        n = 0;
        for (int b = 0; b < size; ++b) n += have(b);
    } else {
        compose(sh.count);
    }
    if (size > 1) {
        block_mass(mass, sh, 0, c);
        if (t == 0) sh.m = mass.m, sh.s = mass.s;
        cluster_sync();
        if (rank == 0) {
            n = sh.count;
            for (int b = 1; b < size; ++b) {
                const int count = have(b);
                for (int i = t; i < count; i += threads) {
                    const uint32_t at = map_rank(smem_u32(&cand.at[i]), (uint32_t)b);
                    cand.at[n + i] = (unsigned long long)__float_as_uint(ld_cluster(at + 4)) << 32 | __float_as_uint(ld_cluster(at));
                }
                n += count;
            }
            mass = RestMass();
            if (t < size) mass.m = ld_cluster(map_rank(smem_u32(&sh.m), (uint32_t)t)), mass.s = ld_cluster(map_rank(smem_u32(&sh.s), (uint32_t)t));
        }
        cluster_sync();   // nobody reads another block's candidates any more
        if (rank != 0) return;
    }
    if (n < k) {
        // fewer than k are above -inf, so enough of the first k elements are -inf
        if (t == 0) sh.count = n;
        __syncthreads();
        for (int i = t; i < k; i += threads)
            if (to_float(z[i]) == -infinity()) cand.at[add_shared(&sh.count)] = composite(-infinity(), i);
        __syncthreads();
        n = sh.count;
        __syncthreads();
    }
    rank_candidates(sh, cand, n, k, mass, c);
    block_mass(mass, sh, 1, c);
    for (int i = t; i < k; i += threads) {
        const unsigned long long mine = sh.best[i];
        a.values[row * k + i] = key_value((uint32_t)(mine >> 32));
        a.indices[row * k + i] = (int32_t)~(uint32_t)mine;
    }
    if (t == 0) a.rest[row] = mass.s == 0.f ? -infinity() : mass.m / a.temperature + logf(mass.s);
}

// ---- long rows, one block each --------------------------------------------------------
//
// A block streams its row through two buffers in shared memory and reads it once.  The first part's
// group maxima bound the k-th largest from below; whenever many candidates have come together the bound
// is raised to (about) their own k-th largest, so a part of a long row adds few.  2048 x 131072 bfloat16 for
// 128: 223 us, 2.4 TB/s.  Bound by instructions, 0.71 a cycle and scheduler, 5700 a part: unpacking,
// comparing with the bound and an exponential for every element.

constexpr int kStreamBytes = 16384;
constexpr int kStreamThreads = 256, kStreamRoom = 1024;   // threads of a block, candidates it can hold
constexpr int kLate = 1 << 20;                            // added to their number when a part's copies came late

template <typename T> struct StreamShared {
    uint64_t bar[2];
    TopShared top;
};

// Keeps about the k largest of the candidates: those in the bins (of equal parts of the keys' range) down
// to the k-th largest's.  Returns the smallest key kept; the others join the mass.
__device__ __forceinline__ uint32_t keep_largest(TopShared& sh, const Candidates& cand, int n, int k, RestMass& mass, float c) {
    const int t = threadIdx.x, threads = blockDim.x, lane = t & 31, warps = threads >> 5;
    constexpr int kMost = kStreamRoom / kStreamThreads;   // candidates a thread holds
    unsigned long long mine[kMost];
    uint32_t hi = 0, lo = 0xffffffffu;
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
        const int i = t + j * threads;
        mine[j] = i < n ? cand.at[i] : 0;
        if (i < n) {
            const uint32_t key = order_key(__uint_as_float((uint32_t)(mine[j] >> 32)));
            hi = max(hi, key), lo = min(lo, key);
        }
    }
    hi = __reduce_max_sync(0xffffffffu, hi), lo = __reduce_min_sync(0xffffffffu, lo);
    if (lane == 0) sh.warp_hi[t >> 5] = hi, sh.warp_lo[t >> 5] = lo;
    for (int i = t; i < kTopBins; i += threads) sh.bins[i] = 0;
    __syncthreads();
    hi = __reduce_max_sync(0xffffffffu, sh.warp_hi[min(lane, warps - 1)]);
    lo = __reduce_min_sync(0xffffffffu, sh.warp_lo[min(lane, warps - 1)]);
    const KeyBins bins(hi, lo);
#pragma unroll
    for (int j = 0; j < kMost; ++j)
        if (t + j * threads < n) add_shared(&sh.bins[bins.of(order_key(__uint_as_float((uint32_t)(mine[j] >> 32))))]);
    if (t == 0) sh.count = 0;
    __syncthreads();
    if (t < 32) {
        uint32_t sum = 0;
#pragma unroll
        for (int b = 0; b < kTopBins / 32; ++b) sum += sh.bins[lane * (kTopBins / 32) + b];
        uint32_t upto = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        uint32_t before = upto - sum;
        if (before < (uint32_t)k && upto >= (uint32_t)k) {
            int b = 0;
            for (; before + sh.bins[lane * (kTopBins / 32) + b] < (uint32_t)k; ++b) before += sh.bins[lane * (kTopBins / 32) + b];
            sh.have = lane * (kTopBins / 32) + b;
        }
    }
    __syncthreads();
    const uint32_t bin = (uint32_t)sh.have;
    uint32_t least = 0xffffffffu;
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
        if (t + j * threads >= n) continue;
        const float x = __uint_as_float((uint32_t)(mine[j] >> 32));
        const uint32_t key = order_key(x);
        if (bins.of(key) <= bin) {
            cand.at[add_shared(&sh.count)] = mine[j];
            least = min(least, key);
        } else {
            mass.join(x, 1.f, 0.f, c);
        }
    }
    least = __reduce_min_sync(0xffffffffu, least);
    __syncthreads();
    if (lane == 0) sh.warp_lo[t >> 5] = least;
    __syncthreads();
    return __reduce_min_sync(0xffffffffu, sh.warp_lo[min(lane, warps - 1)]);
}

template <typename T> __global__ void __launch_bounds__(kStreamThreads, 4) k_top_stream(TopArgs a) {
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ StreamShared<T> shared;
    TopShared& sh = shared.top;
    constexpr int E = Gran<T>::E, kGrans = kStreamBytes / 16;
    const int t = threadIdx.x, threads = blockDim.x, lane = t & 31, warp = t >> 5, warps = threads >> 5;
    const long long row = blockIdx.x;
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    const Cut<T> cut(z, a.cols);
    T* const buffer = reinterpret_cast<T*>(dyn);
    Candidates cand;
    cand.at = reinterpret_cast<unsigned long long*>(dyn + 2 * kStreamBytes);
    cand.order = reinterpret_cast<uint16_t*>(cand.at + a.room);
    cand.room = a.room;
    const float c = kLog2e / a.temperature;
    const int k = a.k, parts = (cut.grans + kGrans - 1) / kGrans;

    if (t == 0) {
        sh.count = 0;
        mbar_init(smem_u32(&shared.bar[0]), 1);
        mbar_init(smem_u32(&shared.bar[1]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    after_earlier_kernels();
    // part p of the row into its buffer: whole granules by a bulk copy, the row's edges by hand
    const auto part_of = [&](int p) {
        const int g0 = p * kGrans;
        const int from = max(0, g0 * E - cut.phase), to = min(cut.n, g0 * E + kGrans * E - cut.phase);
        return Cut<T>(z + from, to - from);
    };
    const auto fetch = [&](int p) { part_of(p).stage(buffer + (p & 1) * (kGrans * E), smem_u32(&shared.bar[p & 1])); };
    fetch(0);
    if (parts > 1) fetch(1);

    RestMass mass;
    uint32_t least = 0;   // key of the bound
    bool crowded = false;
    int on_way = 1;   // parts on their way when the loop ends early
    int p = 0;
    for (; p < parts; ++p) {
        __syncthreads();
        if (copies_late(smem_u32(&shared.bar[p & 1]), (uint32_t)(p >> 1) & 1)) add_shared(&sh.count, kLate);   // ends the loop
        const Cut<T> part = part_of(p);
        const Source<T, true> src = {part, buffer + (p & 1) * (kGrans * E)};
        if (p == 0) {
            GranMax<T, true> top;
#pragma unroll 4
            for (int g = t; g < part.grans; g += threads) top.add(src.get(g));
            const uint32_t k0 = order_key(top.first()) >> 16, k1 = order_key(top.second()) >> 16;
            const int share = (k + warps - 1) / warps;
            const uint32_t all = __reduce_and_sync(0xffffffffu, k0 & k1), any = __reduce_or_sync(0xffffffffu, k0 | k1);
            const int bits = 32 - __clz((int)(all ^ any));
            uint32_t bound = all >> bits << bits;
            for (int b = bits - 1; b >= 0; --b) {
                const uint32_t next = bound | 1u << b;
                if (__popc(__ballot_sync(0xffffffffu, k0 >= next)) + __popc(__ballot_sync(0xffffffffu, k1 >= next)) >= share) bound = next;
            }
            if (lane == 0) sh.warp_bound[warp] = bound;
            __syncthreads();
            least = max(__reduce_min_sync(0xffffffffu, sh.warp_bound[min(lane, warps - 1)]) << 16, kLowestKey);
        }
        const RestMass more = gather_top<T, true, true>(src, part.p - z, sh, cand, (unsigned long long)least << 32, c);
        mass.join(more.m, more.s, 0.f, c);
        before_copies();
        __syncthreads();
        const int n = sh.count;
        if (n > a.room) {
            crowded = true;
            break;
        }
        if (p + 2 < parts) fetch(p + 2);
        if (n > a.room / 2 && p + 1 < parts) {
            least = keep_largest(sh, cand, n, k, mass, c);
            if (sh.count > a.room / 2) {
                crowded = true;
                ++on_way;
                break;
            }
        }
    }
    int n = sh.count;
    bool late = n >= kLate;
    __syncthreads();
    if (crowded) {
        // values crowd at the bound: an exact one, from the whole row once more (what is on its way is not used)
        for (int q = p + 1; q <= min(p + on_way, parts - 1); ++q) late |= copies_late(smem_u32(&shared.bar[q & 1]), (uint32_t)(q >> 1) & 1);
        const unsigned long long threshold = exact_threshold(cut, 0, sh, cand, k);
        if (t == 0) sh.count = 0;
        __syncthreads();
        mass = gather_top<T, false, false>(Source<T, false>{cut, nullptr}, 0, sh, cand, threshold, c);
        __syncthreads();
        n = sh.count;
        __syncthreads();
    }
    if (late) mass.s = __uint_as_float(0x7fffffffu);   // the logits never came
    for (int i = t; i < n; i += threads) {
        const unsigned long long raw = cand.at[i];
        cand.at[i] = composite(__uint_as_float((uint32_t)(raw >> 32)), (int)(uint32_t)raw);
    }
    __syncthreads();
    if (n < k) {
        // fewer than k are above -inf, so enough of the first k elements are -inf
        if (t == 0) sh.count = n;
        __syncthreads();
        for (int i = t; i < k; i += threads)
            if (to_float(z[i]) == -infinity()) cand.at[add_shared(&sh.count)] = composite(-infinity(), i);
        __syncthreads();
        n = sh.count;
        __syncthreads();
    }
    rank_candidates(sh, cand, n, k, mass, c);
    block_mass(mass, sh, 1, c);
    for (int i = t; i < k; i += threads) {
        const unsigned long long mine = sh.best[i];
        a.values[row * k + i] = key_value((uint32_t)(mine >> 32));
        a.indices[row * k + i] = (int32_t)~(uint32_t)mine;
    }
    if (t == 0) a.rest[row] = mass.s == 0.f ? -infinity() : mass.m / a.temperature + logf(mass.s);
}

}  // namespace sbclm
