// Low-rank adapters of many clients or requests beside a shared projection.
//
//   forward   mid = x D_i^T,  y = base + s mid P_i           (D_i: rank x inner, P_i: rank x outer)
//   backward  dmid = s dy P_i^T,  dx = base + dmid D_i,  dD_i = dmid_i^T x_i,  dP_i = s mid_i^T dy_i
//
// i is the adapter of a token.  Both factors have `rank` rows of a wide matrix, so two kernels make all six
// products: into the rank (contracting the wide axis), out of it, and a third sums over an adapter's tokens.
// What memory needs is x, base and y once: a rank of 16 is 16 to 32 operations for each byte of them, which warp-wide
// products (16 x 8 x 16, 516 TFLOP/s) make several times over, without staging operands in the tensor cores' layouts.
//
// 8191 tokens of 12 requests and 8 adapters of rank 64, 4096 -> 8192 bfloat16, there and back 424 to 480 us (by the requests'
// lengths): into the rank 41 and 67 us (67 and 134 MB of x), out of it 96 and 55 (268 and 134 MB), both sums over tokens 178.  The instructions between the products bound
// the first two (LSU pipe 39 to 56 %, tensor pipe 19 to 33 %); the third's 192 blocks, one an SM, are a round and a third, and keep the tensor
// pipe 55 % busy while they run.
//
// Operands go into the products as the bfloat16 terms that they are the sum of (one for bfloat16, two for float16, three for float32,
// cut off rather than rounded, so that none overflows): n terms leave less than 2^(1 - 8 n) of a value.  mid and dmid are kept as three
// terms, and where a result has 32 bits all operands have theirs.  Of three by three products the six largest count; the others are below
// 2^-21 of a product (2^-25 on average), which measures as 32-bit arithmetic does (1e-7 of the result after 4096 elements).  There a
// step's sum starts from zero and is added by an ordinary addition: the tensor cores cut off what they align to a running sum, which
// came to 1.6e-6.  Where a result has 16 bits, two terms of mid, dmid and float32 factors are taken, and all of their products: what is
// left out is below 2^-14 of a product (half a step of the result is 2^-9 or 2^-12 of it), and each error against 64 bits measures
// the same as that of 32-bit arithmetic, rounded once (1.00 times over all cases).
//
// Tokens come in any order.  A plan groups them: the tokens of an adapter one behind the other in the order in which
// they came (so sums have one order), cut into tiles of 64.
#pragma once

#include "../../include/sbc_block.h"
#include "lm_common.cuh"
#include "lm_product.cuh"
#include "lm_ring.cuh"

namespace sbclm {

constexpr int kATile = 64;        // tokens of a tile
constexpr int kAThreads = 256;
constexpr int kAFewThreads = 256;
constexpr int kAPlanThreads = 1024;

// ---- plan -----------------------------------------------------------------------------------

// tiles[0].x: how many follow; a tile: adapter (count: none), first place in `order`, tokens.
struct AdapterPlan {
    int4* tiles;
    int* offsets;   // first place of an adapter's tokens, count + 2 of them (the last: tokens without one, and the end)
    int* order;
};

struct PlanArgs {
    const int* ids;
    AdapterPlan plan;
    uint32_t* status;
    int tokens, count, warps;
};

__device__ __forceinline__ int adapter_of(int id, int count) { return id >= 0 && id < count ? id : count; }

// A stable counting sort by one block.  A warp has a run of tokens and counters of its own; the counters are summed over adapters
// and, for one adapter, over warps, and then say where each warp's next token of it goes.
__global__ void __launch_bounds__(kAPlanThreads) k_adapter_plan(PlanArgs a) {
    extern __shared__ int counters[];   // [warps][count + 1]
    __shared__ int2 scan[32];
    after_earlier_kernels();
    const int bins = a.count + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < bins * a.warps; i += kAPlanThreads) counters[i] = 0;
    __syncthreads();
    const int run = (a.tokens + a.warps - 1) / a.warps;
    const int first = (int)min((long long)a.tokens, (long long)warp * run), last = warp < a.warps ? (int)min((long long)a.tokens, (long long)first + run) : first;
    int* mine = counters + (long long)min(warp, a.warps - 1) * bins;
    bool beyond = false;
    constexpr int kSteps = 8;   // ids of so many steps are loaded together
    for (int t0 = first; t0 < last; t0 += 32 * kSteps) {
        int ids[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) ids[i] = t0 + 32 * i + lane < last ? a.ids[t0 + 32 * i + lane] : -1;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (t0 + 32 * i >= last) break;
            const bool in = t0 + 32 * i + lane < last;
            beyond |= ids[i] >= a.count;
            const int bin = in ? adapter_of(ids[i], a.count) : -1;
            const unsigned same = __match_any_sync(0xffffffffu, bin);
            if (in && (same & ((1u << lane) - 1)) == 0) mine[bin] += __popc(same);
            __syncwarp();
        }
    }
    if (beyond && a.status) atomicOr(a.status, SBC_STATUS_RANGE);
    __syncthreads();
    int2 before = make_int2(0, 0);   // tokens and tiles of the adapters in front
    for (int b0 = 0; b0 < bins; b0 += kAPlanThreads) {
        const int b = b0 + threadIdx.x;
        int n = 0;
        if (b < bins)
            for (int w = 0; w < a.warps; ++w) n += counters[(long long)w * bins + b];
        const int tiles = (n + kATile - 1) / kATile;
        int2 v = make_int2(n, tiles);
        for (int d = 1; d < 32; d <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, v.x, d), y = __shfl_up_sync(0xffffffffu, v.y, d);
            if (lane >= d) v.x += x, v.y += y;
        }
        if (lane == 31) scan[warp] = v;
        __syncthreads();
        int2 front = before, total = make_int2(0, 0);
        for (int w = 0; w < kAPlanThreads / 32; ++w) {
            if (w < warp) front.x += scan[w].x, front.y += scan[w].y;
            total.x += scan[w].x, total.y += scan[w].y;
        }
        const int at = front.x + v.x - n;
        if (b < bins) {
            a.plan.offsets[b] = at;
            for (int w = 0, p = at; w < a.warps; ++w) {
                int& c = counters[(long long)w * bins + b];
                const int k = c;
                c = p;
                p += k;
            }
            for (int i = 0; i < tiles; ++i) a.plan.tiles[1 + front.y + v.y - tiles + i] = make_int4(b, at + i * kATile, min(kATile, n - i * kATile), 0);
        }
        before.x += total.x, before.y += total.y;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        a.plan.offsets[bins] = a.tokens;
        a.plan.tiles[0] = make_int4(before.y, 0, 0, 0);
    }
    for (int t0 = first; t0 < last; t0 += 32 * kSteps) {
        int ids[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) ids[i] = t0 + 32 * i + lane < last ? a.ids[t0 + 32 * i + lane] : -1;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (t0 + 32 * i >= last) break;
            const bool in = t0 + 32 * i + lane < last;
            const int bin = in ? adapter_of(ids[i], a.count) : -1;
            const unsigned same = __match_any_sync(0xffffffffu, bin), ahead = same & ((1u << lane) - 1);
            int at = 0;
            if (in && ahead == 0) {
                at = mine[bin];
                mine[bin] = at + __popc(same);
            }
            at = __shfl_sync(0xffffffffu, at, __ffs(same) - 1) + __popc(ahead);
            if (in) a.plan.order[at] = t0 + 32 * i + lane;
            __syncwarp();
        }
    }
}

// ---- terms ------------------------------------------------------------------------------------

template <typename T> struct Terms { static constexpr int n = 1; };
template <> struct Terms<__half> { static constexpr int n = 2; };
template <> struct Terms<float> { static constexpr int n = 3; };

// The first N bfloat16 terms of v, in the upper halves of words.  An infinity or a NaN is its first term alone.
template <int N> __device__ __forceinline__ void cut(uint32_t* out, float v) {
    out[0] = __float_as_uint(v) & 0xffff0000u;
    if (N == 1) return;
    const bool finite = (out[0] & 0x7f800000u) != 0x7f800000u;
    float rest = finite ? v - __uint_as_float(out[0]) : 0.f;
    // (what is left of a NaN whose payload lies in the lower half would be an infinity)
    if (!finite && v != v) out[0] |= 0x00400000u;
#pragma unroll
    for (int i = 1; i < N; ++i) {
        out[i] = __float_as_uint(rest) & 0xffff0000u;
        rest -= __uint_as_float(out[i]);
    }
}
// Two terms as the products take them: the first in the lower half.
__device__ __forceinline__ uint32_t halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }

// Words of N terms for four pairs of neighbours.
template <int N, typename T> __device__ __forceinline__ void cut_row(uint32_t (*out)[4], const Pack8<T>& v) {
    if constexpr (sizeof(T) == 2 && Terms<T>::n == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[0][i] = v.w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a[N], b[N];
            cut<N>(a, to_float(v.e[2 * i]));
            cut<N>(b, to_float(v.e[2 * i + 1]));
#pragma unroll
            for (int k = 0; k < N; ++k) out[k][i] = halves(a[k], b[k]);
        }
    }
}
// Words of N terms of the pairs (v[e], w[e]), e = 0 .. 7: two rows of a matrix that is contracted along its columns' other axis.
template <int N, typename T> __device__ __forceinline__ void cut_rows(uint32_t (*out)[8], const Pack8<T>& v, const Pack8<T>& w) {
    if constexpr (sizeof(T) == 2 && Terms<T>::n == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) out[0][e] = __byte_perm(v.w[e / 2], w.w[e / 2], e & 1 ? 0x7632 : 0x5410);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t a[N], b[N];
            cut<N>(a, to_float(v.e[e]));
            cut<N>(b, to_float(w.e[e]));
#pragma unroll
            for (int k = 0; k < N; ++k) out[k][e] = halves(a[k], b[k]);
        }
    }
}

__device__ __forceinline__ void mma_terms(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Sixteen rows x sixteen k of terms in shared memory as the products take them: from rows, or (TRANS) from columns.  `from`: this
// lane's row and half of sixteen elements.
template <bool TRANS> __device__ __forceinline__ void load_terms(uint32_t* w, uint32_t from) {
    if (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from) : "memory");
}
// Products of sixteen rows of X terms with eight columns of Y terms (at a time: b0[o * next], b1[o * next]).
template <int X, int Y, bool APART>
__device__ __forceinline__ void add_products(float* acc, const uint32_t (*w)[4], const uint32_t* b0, const uint32_t* b1, int next) {
    float part[4] = {};
    float* d = APART ? part : acc;
#pragma unroll
    for (int order = 2; order >= 0; --order)   // the small products first
#pragma unroll
        for (int n = 0; n < X; ++n) {
            const int o = order - n;
            if (o >= 0 && o < Y) mma_terms(d, w[n], b0[o * next], b1[o * next]);
        }
    if (APART)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] += part[k];
}

// An infinity's first term meets all terms of the other operand, and where one of those is zero the products' sum is a NaN that the
// operands' product is not.  So what is a NaN is summed up again, by ordinary multiplications of whole operands, which says
// whether it is one.  (Out of line: nothing of it costs what is finite more than the question.)
//
// out[e] = first(e) + scale * sum over k < n of factor(k) row(k)[e], e < have; done once all of them are NaNs.
template <typename O, typename F, typename R, typename B>
__device__ __forceinline__ void sum_again(int n, F factor, R row, float scale, O* out, int have, B first) {
    float s[8] = {};
    bool open = true;
    for (int k = 0; k < n && open; k += 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (k + i >= n) break;
            const float f = factor(k + i);
            const auto* r = row(k + i);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < have) s[e] = fmaf(f, to_float(r[e]), s[e]);
        }
        open = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) open |= e < have && s[e] == s[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < have) out[e] = from_float<O>(fmaf(scale, s[e], first(e)));
}
// The value whose terms lie `plane` apart.
__device__ __forceinline__ float joined(const uint16_t* terms, long long plane) {
    float v = 0.f;
#pragma unroll
    for (int n = 2; n >= 0; --n) v += __uint_as_float((uint32_t)terms[n * plane] << 16);
    return v;
}
template <typename T, typename W> __device__ __noinline__ float into_again(const T* x, const W* factor, int wide) {
    float s;
    sum_again(wide, [&](int k) { return to_float(x[k]); }, [&](int k) { return factor + k; }, 1.f, &s, 1, [](int) { return 0.f; });
    return s;
}
// (eight neighbours of a row, whose base is in `out`)
template <typename T, typename W>
__device__ __noinline__ void out_again(const uint16_t* mid, long long plane, const W* factor, int rank, int wide, float scale, T* out, int have) {
    sum_again(rank, [&](int j) { return joined(mid + j, plane); }, [&](int j) { return factor + (long long)j * wide; }, scale, out, have, [&](int e) { return to_float(out[e]); });
}
template <typename T, typename W>
__device__ __noinline__ void over_again(const uint16_t* mid, long long plane, int ranks, const T* x, long long x_stride, const int* order, int n, float scale, W* out, int have) {
    sum_again(n, [&](int k) { return joined(mid + (long long)order[k] * ranks, plane); }, [&](int k) { return x + order[k] * x_stride; }, scale, out, have,
              [](int) { return 0.f; });
}

// ---- packs in a thread's ring -----------------------------------------------------------
//
// A pack's granules of 16 bytes are 512 bytes apart: a warp's are side by side.

// Copies eight elements at a multiple of 16 bytes, or zeros (p is then not read).  SHARED: other warps load the same, so it may
// stay in the first-level cache.  (Zeros by a predicate: a number of bytes in a register costs tens of instructions.)
template <bool SHARED, typename T> __device__ __forceinline__ void ring_load8(uint32_t to, const T* p, bool zeros = false) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) ring_copy16<SHARED>(to + 512 * i, reinterpret_cast<const uint4*>(p) + i, zeros);
}
// Copies `have` elements (at most 8, zeros behind them) whose address is a multiple of `align`.
template <typename T> __device__ __forceinline__ void ring_load(uint32_t to, const T* p, int have, int align) {
    constexpr int kEach = 16 / (int)sizeof(T), kWord = 4 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i, to += 512, p += kEach, have -= kEach) {
        if (align >= 4) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (kWord == 2 && have == 2 * k + 1)   // half a word
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + 4 * k), "r"((uint32_t)reinterpret_cast<const uint16_t*>(p)[2 * k]) : "memory");
                else
                    asm volatile("{\n\t.reg .pred z;\n\tsetp.le.s32 z, %2, %3;\n\tcp.async.ca.shared.global [%0], [%1], 4, z;\n\t}" ::"r"(to + 4 * k),
                                 "l"(reinterpret_cast<const char*>(p) + 4 * k), "r"(have), "r"(kWord * k)
                                 : "memory");
            }
        } else {
            union {
                T e[kEach];
                uint4 q;
            } v;
            v.q = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < kEach; ++k)
                if (k < have) v.e[k] = p[k];
            ring_store16(to, v.q);
        }
    }
}
template <typename T> __device__ __forceinline__ void ring_read(Pack8<T>& v, uint32_t from) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v.q[i] = ring_read16(from + 512 * i);
}
template <typename T> constexpr uint32_t kPackBytes = 32 * 8 * sizeof(T);   // of a warp
template <typename T> __device__ __forceinline__ void pack8(Pack8<T>& v, const float* f) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        if constexpr (sizeof(T) == 4)
            v.e[e] = f[e], v.e[e + 1] = f[e + 1];
        else
            v.w[e / 2] = pack2(f[e], f[e + 1], (const T*)nullptr);
    }
}
template <typename T> __device__ __forceinline__ void write8(T* p, const Pack8<T>& v, int have, bool vec) {
    if (have >= 8 && vec) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = v.q[i];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < have) p[e] = v.e[e];
    }
}

struct AdapterArgs {
    const void* x;          // the wide input (x or dy)
    const void* factor;     // [count][rank][wide]
    const void* base;
    void* out;              // y or dx
    uint16_t* mid;          // terms, [3][tokens][rank in whole sixteens, zeros behind the rank]
    AdapterPlan plan;
    long long x_stride, base_stride, out_stride;
    int tokens, count, rank, wide, parts;
    int align_x, align_base, align_out, align_factor;
    float scale;
};
__host__ __device__ constexpr int sixteens(int rank) { return (rank + 15) / 16 * 16; }

// ---- into the rank ------------------------------------------------------------------------------

// mid[t][j] = scale sum_k x[t][k] factor[i][j][k] for a tile of tokens and up to 8 JT rows.  A thread takes eight neighbours
// of a row, its four k's of two products (which element is which k is free as long as both operands agree).  A warp has half
// of the tokens, so that two blocks fit an SM's registers; warps, and blocks of a cluster, take the wide axis in turns.  Their
// sums meet in shared memory in a fixed order.  VEC: all rows are whole eights that begin at multiples of 16 bytes.
template <typename T, typename W, int JT> struct InShape {
    static constexpr int MT = 2, kHalves = 4 / MT, kRuns = 8 / kHalves, kPer = MT * JT * 4;
    static constexpr int kStage = MT * 2 * (int)kPackBytes<T> + JT * (int)kPackBytes<W>;   // of a warp
    // two blocks of an SM share it while each has two stages
    static constexpr int kFit = 108 * 1024 / (8 * kStage), kStages = kFit >= 4 ? 4 : kFit >= 2 ? kFit : 200 * 1024 / (8 * kStage) >= 3 ? 3 : 2;
    static constexpr int kSmem = 8 * (kStages * kStage > kPer * 128 ? kStages * kStage : kPer * 128);
};
template <typename T, typename W, int JT, bool VEC>
__global__ void __launch_bounds__(kAThreads, Terms<T>::n + Terms<W>::n <= 3 ? 2 : 1) k_adapter_in(AdapterArgs a) {
    using S = InShape<T, W, JT>;
    constexpr int X = Terms<T>::n, Y = Terms<W>::n, MT = S::MT, kPer = S::kPer;
    extern __shared__ __align__(16) uint8_t raw[];   // rings of the warps; in the end sums [8 warps][kPer][32]
    __shared__ int tokens[kATile];
    after_earlier_kernels();
    const int part = (int)blockIdx.x % a.parts, tile = (int)blockIdx.x / a.parts;
    if (tile >= a.plan.tiles[0].x) return;
    const int4 at = a.plan.tiles[1 + tile];
    if (at.x >= a.count) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3, half = warp % S::kHalves, run = warp / S::kHalves;
    const int j0 = (int)blockIdx.y * 8 * JT;
    if (threadIdx.x < kATile) tokens[threadIdx.x] = threadIdx.x < at.z ? a.plan.order[at.y + threadIdx.x] : -1;
    __syncthreads();
    // (a row that is none has no sums that are used: nothing is loaded for it where others' places cannot be mistaken for it)
    const T* x[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = tokens[half * 32 + m * 16 + h * 8 + g];
            x[m][h] = t < 0 ? nullptr : static_cast<const T*>(a.x) + (long long)t * a.x_stride + q * 8;
        }
    const W* factor = static_cast<const W*>(a.factor) + ((long long)at.x * a.rank + j0 + g) * a.wide + q * 8;
    const int rows = a.rank - j0 - g;   // of the factor, this thread's first among them
    const uint32_t ring = smem_u32(raw) + (uint32_t)(warp * S::kStages * S::kStage) + 16u * lane;
    float acc[MT][JT][4] = {};
    const int left = at.z - half * 32;   // tokens of this warp
    const int units = (a.wide + 31) / 32;   // of 32 elements; this block's run of them
    const int u0 = (int)((long long)units * part / a.parts), u1 = left > 0 ? (int)((long long)units * (part + 1) / a.parts) : u0;
    const auto fill = [&](int u, int stage) {
        if (u < u1) {
            const int k = u * 32, have = a.wide - k - q * 8;
            const uint32_t to = ring + (uint32_t)(stage * S::kStage), to_f = to + MT * 2 * kPackBytes<T>;
            if (VEC) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (x[m][h]) ring_load8<false>(to + (m * 2 + h) * kPackBytes<T>, x[m][h] + k, have <= 0);
                const W* f = factor + k;
#pragma unroll
                for (int j = 0; j < JT; ++j, f += 8ll * a.wide)
                    if (8 * j < rows) ring_load8<true>(to_f + j * kPackBytes<W>, f, have <= 0);
            } else {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (x[m][h]) ring_load(to + (m * 2 + h) * kPackBytes<T>, x[m][h] + k, have, a.align_x);
                const W* f = factor + k;
#pragma unroll
                for (int j = 0; j < JT; ++j, f += 8ll * a.wide)
                    if (8 * j < rows) ring_load(to_f + j * kPackBytes<W>, f, have, a.align_factor);
            }
        }
        ring_commit();
    };
#pragma unroll
    for (int s = 0; s < S::kStages - 1; ++s) fill(u0 + run + s * S::kRuns, s);
    int stage = 0;
    for (int u = u0 + run; u < u1; u += S::kRuns) {
        fill(u + (S::kStages - 1) * S::kRuns, stage == 0 ? S::kStages - 1 : stage - 1);
        ring_wait(S::kStages - 1);
        const uint32_t from = ring + (uint32_t)(stage * S::kStage);
        if (++stage == S::kStages) stage = 0;
        // all of the factor's terms where they are few, otherwise all of x's
        constexpr bool kHold = JT * Y <= MT * 2 * X;
        uint32_t held[kHold ? JT : MT * 2][kHold ? Y : X][4];
        if constexpr (kHold) {
#pragma unroll
            for (int j = 0; j < JT; ++j) {
                Pack8<W> v;
                ring_read(v, from + MT * 2 * kPackBytes<T> + j * kPackBytes<W>);
                cut_row<Y>(held[j], v);
            }
        } else {
#pragma unroll
            for (int m = 0; m < MT * 2; ++m) {
                Pack8<T> v;
                ring_read(v, from + m * kPackBytes<T>);
                cut_row<X>(held[m], v);
            }
        }
#pragma unroll
        for (int outer = 0; outer < (kHold ? MT : JT); ++outer) {
            uint32_t now[kHold ? 2 : 1][kHold ? X : Y][4];
            if constexpr (kHold) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    Pack8<T> v;
                    ring_read(v, from + (outer * 2 + h) * kPackBytes<T>);
                    cut_row<X>(now[h], v);
                }
            } else {
                Pack8<W> v;
                ring_read(v, from + MT * 2 * kPackBytes<T> + outer * kPackBytes<W>);
                cut_row<Y>(now[0], v);
            }
#pragma unroll
            for (int inner = 0; inner < (kHold ? JT : MT); ++inner) {
                const int m = kHold ? outer : inner, j = kHold ? inner : outer;
                float part_sum[4] = {};
                float* d = sizeof(W) == 4 ? part_sum : acc[m][j];
#pragma unroll
                for (int order = 2; order >= 0; --order)   // the small products first
#pragma unroll
                    for (int n = 0; n < X; ++n) {
                        const int o = order - n;
                        if (o < 0 || o >= Y) continue;
#pragma unroll
                        for (int s = 0; s < 4; s += 2) {
                            const uint32_t(&r0)[4] = kHold ? now[0][n] : held[m * 2 % (kHold ? JT : MT * 2)][n];
                            const uint32_t(&r1)[4] = kHold ? now[kHold ? 1 : 0][n] : held[(m * 2 + 1) % (kHold ? JT : MT * 2)][n];
                            const uint32_t(&f)[4] = kHold ? held[j % (kHold ? JT : MT * 2)][o] : now[0][o];
                            const uint32_t w[4] = {r0[s], r1[s], r0[s + 1], r1[s + 1]};
                            mma_terms(d, w, f[s], f[s + 1]);
                        }
                    }
                if (sizeof(W) == 4)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[m][j][e] += part_sum[e];
            }
        }
    }
    ring_wait(0);
    __syncthreads();   // all rings are read: sums take their place
    float* sums = reinterpret_cast<float*>(raw);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[(warp * kPer + (m * JT + j) * 4 + e) * 32 + lane] = acc[m][j][e];
    __syncthreads();
    // [halves][kPer][32] sums of kRuns warps, left in the first ones' places for the cluster
    constexpr int kSums = S::kHalves * kPer * 32;
    const int wide_rank = sixteens(a.rank);
    const auto store = [&](int i, float v) {
        const int n = i % 32, e = i / 32 % 4, j = i / 128 % JT, m = i / (128 * JT);   // m: halves and their tiles
        const int t = m * 16 + (e >> 1) * 8 + (n >> 2), r = j0 + 8 * j + (n & 3) * 2 + (e & 1);
        if (t >= at.z || r >= wide_rank) return;
        if (v != v && r < a.rank)
            v = into_again(static_cast<const T*>(a.x) + tokens[t] * a.x_stride, static_cast<const W*>(a.factor) + ((long long)at.x * a.rank + r) * a.wide, a.wide);
        uint32_t w[3];
        cut<3>(w, r < a.rank ? v * a.scale : 0.f);
        uint16_t* to = a.mid + (long long)tokens[t] * wide_rank + r;
#pragma unroll
        for (int k = 0; k < 3; ++k, to += (long long)a.tokens * wide_rank) {
            *to = (uint16_t)(w[k] >> 16);
            if (JT == 1) to[8] = 0;
        }
    };
    for (int i = threadIdx.x; i < kSums; i += kAThreads) {
        float v = sums[i];
#pragma unroll
        for (int w = 1; w < S::kRuns; ++w) v += sums[i + w * kSums];
        if (a.parts == 1)
            store(i, v);
        else
            sums[i] = v;
    }
    if (a.parts == 1) return;
    cluster_sync();
    for (int i = part * kAThreads + threadIdx.x; i < kSums; i += a.parts * kAThreads) {
        const uint32_t from = smem_u32(&sums[i]);
        float v = 0.f;
        for (int p = 0; p < a.parts; ++p) v += ld_cluster(map_rank(from, (uint32_t)p));
        store(i, v);
    }
    cluster_sync();
}

// ---- out of the rank ------------------------------------------------------------------------------

// out[t][c] = base[t][c] + scale sum_j mid[t][j] factor[i][j][c].  A block has CB columns, whose factor waits in shared memory as
// terms (again only where the adapter changes), and takes a run of the tiles of tokens: base and mid's terms of the next
// tile are on their way while this one's products are made.  A warp has 64 columns and as many tokens as leaves eight
// warps busy.  The factor's columns are so placed that a thread ends with eight neighbours of a row, twice.
template <typename T, typename W, int CB> struct OutShape {
    // 16-bit results: two terms, what is left out is below 2^-15 of a factor
    static constexpr int X = sizeof(T) == 4 ? 3 : 2, Y = sizeof(T) == 4 ? Terms<W>::n : (Terms<W>::n < 2 ? Terms<W>::n : 2);
    static constexpr int kGroups = CB / 64, MT = kGroups / 2, kBase = MT * 4 * (int)kPackBytes<T>, kFactorPitch = CB + 8;
    static __host__ __device__ constexpr int pitch(int rank) { return sixteens(rank) + 8; }
    static __host__ __device__ constexpr int factor_bytes(int rank) { return Y * sixteens(rank) * kFactorPitch * 2; }
    static __host__ __device__ constexpr int terms_bytes(int rank) { return X * kATile * pitch(rank) * 2; }
    static constexpr int kMost = 225 * 1024;
    // mid's terms of two tiles, where they fit
    static __host__ __device__ constexpr int buffers(int rank) { return 8 * kBase + factor_bytes(rank) + 2 * terms_bytes(rank) <= kMost ? 2 : 1; }
    static __host__ __device__ constexpr int smem(int rank) { return 8 * kBase + factor_bytes(rank) + buffers(rank) * terms_bytes(rank); }
};
template <typename T, typename W, int CB, bool VEC>
__global__ void __launch_bounds__(kAThreads, sizeof(T) == 2 && Terms<W>::n == 1 ? 2 : 1) k_adapter_out(AdapterArgs a) {
    using S = OutShape<T, W, CB>;
    constexpr int X = S::X, Y = S::Y, MT = S::MT;
    extern __shared__ __align__(16) uint8_t raw[];   // rings of base, the factor's terms [Y][ranks][pitch], mid's [2][X][kATile][pitch]
    __shared__ int tokens[3][kATile];
    after_earlier_kernels();
    const int all = a.plan.tiles[0].x, ranks = sixteens(a.rank), steps = ranks / 16, pitch = S::pitch(a.rank);
    const bool two = S::buffers(a.rank) == 2;
    const int first = (int)((long long)all * blockIdx.y / gridDim.y), last = (int)((long long)all * (blockIdx.y + 1) / gridDim.y);
    if (first == last) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int group = warp % S::kGroups, row0 = warp / S::kGroups * 16 * MT;
    const int cb = (int)blockIdx.x * CB, col = cb + group * 64;
    const uint32_t ring = smem_u32(raw) + (uint32_t)(warp * S::kBase) + 16u * lane;
    uint16_t* factor = reinterpret_cast<uint16_t*>(raw + 8 * S::kBase);
    const uint32_t terms = smem_u32(raw) + (uint32_t)(8 * S::kBase + S::factor_bytes(a.rank));
    // The plan is asked for ahead of its use: a tile's place for five tiles later, its tokens for four, and in shared memory three.
    const auto place = [&](int tile) { return tile < last ? a.plan.tiles[1 + tile] : make_int4(0, 0, 0, 0); };
    const auto token = [&](const int4& at) { return (int)threadIdx.x < at.z ? a.plan.order[at.y + threadIdx.x] : -1; };   // (a tile has at most kATile)
    const auto fill_terms = [&](int tile) {
        const int* t = tokens[tile % 3];
        const uint32_t to = terms + (uint32_t)((two ? tile & 1 : 0) * S::terms_bytes(a.rank));
#pragma unroll
        for (int row = (int)threadIdx.x / 8; row < kATile; row += kAThreads / 8) {
            const int tok = t[row];
            for (int c = (int)threadIdx.x % 8 * 8; c < ranks; c += 64) {
                const uint16_t* from = a.mid + (long long)max(tok, 0) * ranks + c;
#pragma unroll
                for (int n = 0; n < X; ++n)
                    ring_load8<false>(to + (uint32_t)(((n * kATile + row) * pitch + c) * 2), reinterpret_cast<const __nv_bfloat16*>(from + (long long)n * a.tokens * ranks), tok < 0);
            }
        }
    };
    const auto fill_base = [&](int tile) {
        if (!a.base) return;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = tokens[tile % 3][row0 + m * 16 + h * 8 + g];
                const T* from = static_cast<const T*>(a.base) + (long long)t * a.base_stride + col + 8 * q;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int have = a.wide - col - 32 * p - 8 * q;
                    if (t < 0 || have <= 0) continue;
                    if (VEC)
                        ring_load8<false>(ring + ((m * 2 + h) * 2 + p) * kPackBytes<T>, from + 32 * p);
                    else
                        ring_load(ring + ((m * 2 + h) * 2 + p) * kPackBytes<T>, from + 32 * p, have, a.align_base);
                }
            }
    };
    const int4 at0 = place(first), at1 = place(first + 1), at2 = place(first + 2);
    int4 at4 = place(first + 4);
    int token3 = token(place(first + 3));
    if (threadIdx.x < kATile) {
        tokens[first % 3][threadIdx.x] = token(at0);
        tokens[(first + 1) % 3][threadIdx.x] = token(at1);
        tokens[(first + 2) % 3][threadIdx.x] = token(at2);
    }
    __syncthreads();
    fill_base(first);
    if (at0.x < a.count) fill_terms(first);
    ring_commit();
    int adapter = -1, now = at0.x, after = at1.x;   // this tile's adapter, and the next one's
    for (int tile = first; tile < last; ++tile) {
        const int later = place(tile + 2).x;
        const bool none = now >= a.count;
        if (now != adapter && !none) {
            // (the tile before has been read behind the barrier at its end)
            adapter = now;
            const W* f = static_cast<const W*>(a.factor) + (long long)now * a.rank * a.wide;
            for (int i = threadIdx.x; i < ranks * (CB / 8); i += kAThreads) {
                const int j = i / (CB / 8), pack = i % (CB / 8), c = cb + 8 * pack;
                Pack8<W> v;
                load8(v, f + (long long)min(j, a.rank - 1) * a.wide + c, j < a.rank ? a.wide - c : 0, VEC ? 16 : a.align_factor);
                // neighbour e of these eight is column 2 (place of the eight in its 32) + (which 32) of tile e
                uint16_t* to = factor + j * S::kFactorPitch + pack / 8 * 64 + (pack & 3) * 2 + (pack >> 2 & 1);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    uint32_t w[Y];
                    cut<Y>(w, to_float(v.e[e]));
#pragma unroll
                    for (int o = 0; o < Y; ++o) to[o * ranks * S::kFactorPitch + 8 * e] = (uint16_t)(w[o] >> 16);
                }
            }
        }
        ring_wait(0);
        Pack8<T> b[MT][2][2];
#pragma unroll
        for (int i = 0; i < MT * 4; ++i) ring_read(b[i / 4][i / 2 % 2][i % 2], ring + i * kPackBytes<T>);
        __syncthreads();   // this tile's terms, the factor and the tokens of the next are there
        if (tile + 1 < last) {
            fill_base(tile + 1);
            if (two && after < a.count) fill_terms(tile + 1);
        }
        ring_commit();
        float acc[MT][8][4] = {};
        if (!none) {
            const uint32_t terms_at = terms + (uint32_t)((two ? tile & 1 : 0) * S::terms_bytes(a.rank) + ((row0 + (lane & 15)) * pitch + (lane >> 4) * 8) * 2);
            const uint32_t factor_at = smem_u32(factor) + (uint32_t)(((lane & 15) * S::kFactorPitch + group * 64 + (lane >> 4) * 8) * 2);
            for (int s = 0; s < steps; ++s) {
                uint32_t w[MT][X][4];
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < X; ++n) load_terms<false>(w[m][n], terms_at + (uint32_t)(((n * kATile + m * 16) * pitch + s * 16) * 2));
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    uint32_t f[Y][4];
#pragma unroll
                    for (int o = 0; o < Y; ++o) load_terms<true>(f[o], factor_at + (uint32_t)(((o * ranks + s * 16) * S::kFactorPitch + e * 8) * 2));
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        add_products<X, Y, sizeof(T) == 4>(acc[m][e], w[m], &f[0][0], &f[0][1], 4);
                        add_products<X, Y, sizeof(T) == 4>(acc[m][e + 1], w[m], &f[0][2], &f[0][3], 4);
                    }
                }
            }
        }
        unsigned redo = 0;   // packs with a NaN
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = tokens[tile % 3][row0 + m * 16 + h * 8 + g];
                if (t < 0 || (none && a.base == a.out)) continue;
                T* out = static_cast<T*>(a.out) + (long long)t * a.out_stride + col + 8 * q;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    Pack8<T> v = b[m][h][p];
                    if (!a.base) v = {};
                    if (!none) {
                        float f[8];
                        bool again = false;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float sum = acc[m][e][2 * h + p];
                            f[e] = fmaf(a.scale, sum, to_float(v.e[e]));
                            again |= sum != sum;
                        }
                        if (again)
                            redo |= 1u << ((m * 2 + h) * 2 + p);   // (the base is left in its place)
                        else
                            pack8(v, f);
                    }
                    write8(out + 32 * p, v, a.wide - col - 32 * p - 8 * q, VEC || a.align_out >= 16);
                }
            }
        for (; redo; redo &= redo - 1) {
            const int i = __ffs(redo) - 1, t = tokens[tile % 3][row0 + i / 2 * 8 + g], c = col + i % 2 * 32 + 8 * q;
            out_again<T, W>(a.mid + (long long)t * ranks, (long long)a.tokens * ranks, static_cast<const W*>(a.factor) + (long long)now * a.rank * a.wide + c, a.rank, a.wide,
                            a.scale, static_cast<T*>(a.out) + (long long)t * a.out_stride + c, min(8, a.wide - c));
        }
        __syncthreads();   // this tile's terms and tokens, and the factor, are read
        if (!two && tile + 1 < last && after < a.count) {
            fill_terms(tile + 1);
            ring_commit();
        }
        if (threadIdx.x < kATile) tokens[tile % 3][threadIdx.x] = token3;   // of tile + 3
        token3 = token(at4);
        at4 = place(tile + 5);
        now = after;
        after = later;
    }
    ring_wait(0);
}

// ---- over tokens ------------------------------------------------------------------------------------

// out[i][j][c] = scale sum over the tokens t of adapter i of mid[t][j] x[t][c], for one or two such sums in a launch.  A warp
// has 64 columns and 16 RT rows, the warps of a block 512 columns and, for ranks above 32, twice as many rows.  64 tokens' terms of mid wait in
// shared memory; of x, a thread loads eight neighbours of four rows, whose pairs are the products' words.  Blocks of a cluster share an adapter's tokens, and add their sums in their order.
struct AdapterSum {
    const void* x;
    const uint16_t* mid;   // terms
    void* out;             // [count][rank][wide]
    long long x_stride;
    int wide, columns;     // blocks of columns
    int align_x, align_out;
    float scale;
};
struct AdapterGradArgs {
    AdapterSum sums[2];
    AdapterPlan plan;
    int tokens, count, rank, parts;
    int first;             // blocks of the first sum
};
template <typename T, typename W, int RT, int RH, bool VEC> struct GradShape {
    static constexpr int X = sizeof(W) == 4 ? 3 : 2, Y = sizeof(W) == 4 ? Terms<T>::n : (Terms<T>::n < 2 ? Terms<T>::n : 2), kThreads = kAThreads * RH, kRows = 16 * RT * RH, kPitch = kRows + 8;
    static constexpr int kStage = 4 * (int)kPackBytes<T>, kStages = sizeof(T) == 4 ? (RH == 2 ? 2 : 3) : 5;   // of a warp: at most a tile ahead
    // x comes as a tile's rows by bulk copies (two tiles have room), or through the warps' rings
    static constexpr bool kBulk = VEC && sizeof(T) == 2;
    static constexpr int kRowPitch = 512 * (int)sizeof(T) + 16;
    static constexpr int kRings = kBulk ? 2 * kATile * kRowPitch : 8 * RH * kStages * kStage, kTerms = 2 * X * kATile * kPitch * 2, kSums = RT * 32 * kThreads * 4;
    static constexpr int kSmem = kRings + kTerms > kSums ? kRings + kTerms : kSums;
};
template <typename T, typename W, int RT, int RH, bool VEC>
__global__ void __launch_bounds__(kAThreads * RH, RH == 1 && Terms<T>::n + Terms<W>::n <= 3 ? 2 : 1) k_adapter_grad(const __grid_constant__ AdapterGradArgs b) {
    using S = GradShape<T, W, RT, RH, VEC>;
    constexpr int X = S::X, Y = S::Y, pitch = S::kPitch, kRows = S::kRows, kThreads = S::kThreads;
    extern __shared__ __align__(16) uint8_t raw[];   // rings of the warps, terms [2][X][kATile][pitch]; in the end sums [32 RT][threads]
    after_earlier_kernels();
    const bool second = (int)blockIdx.x >= b.first;
    const AdapterSum& a = b.sums[second ? 1 : 0];
    const int block = (int)blockIdx.x - (second ? b.first : 0);
    const int part = block % b.parts, blocks = (b.rank + kRows - 1) / kRows, at_row = block / b.parts / a.columns;
    const int i = at_row / blocks, j0 = at_row % blocks * kRows, ranks = min(kRows, b.rank - j0);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3, group = warp % 8, row0 = warp / 8 * 16 * RT;
    const long long cb = (long long)(block / b.parts % a.columns) * (kAThreads * 2);
    const long long c0 = cb + group * 64 + 8 * g;
    const int have = (int)max(0ll, min(8ll, a.wide - c0));
    const bool idle = cb + group * 64 >= a.wide || row0 >= ranks;
    const int begin = b.plan.offsets[i], end = b.plan.offsets[i + 1], groups = (end - begin + 15) / 16;
    const int t_first = begin + (int)((long long)groups * part / b.parts) * 16, t_last = min(end, begin + (int)((long long)groups * (part + 1) / b.parts) * 16);
    uint16_t* terms = reinterpret_cast<uint16_t*>(raw + S::kRings);
    __shared__ int order[3 * kATile];
    __shared__ long long offset[3 * kATile];   // of the tokens' rows
    __shared__ uint64_t bars[2];
    const uint32_t ring = smem_u32(raw) + (uint32_t)(warp * S::kStages * S::kStage) + 16u * (q * 8 + g);   // (requests are rows of 128 bytes)
    float acc[RT][8][4] = {};
    bool late = false;
    if (t_first < t_last) {   // (the same in all threads)
        const T* x = static_cast<const T*>(a.x) + c0;
        const uint32_t terms_at = smem_u32(terms) + (uint32_t)((((lane & 7) + (lane >> 4) * 8) * pitch + row0 + (lane >> 3 & 1) * 8) * 2);
        const bool loads = !idle && have > 0;   // (a column that is none has no sum that is used)
        // which tokens: those of three tiles, asked for another tile ahead
        const auto token = [&](int tile) {
            const int at = t_first + tile * kATile + (int)threadIdx.x;
            return threadIdx.x < kATile && at < t_last ? b.plan.order[at] : -1;
        };
        const auto keep = [&](int tile, int row) {
            if (threadIdx.x >= kATile) return;
            order[tile % 3 * kATile + threadIdx.x] = row;
            offset[tile % 3 * kATile + threadIdx.x] = row * a.x_stride;
        };
        const int ranks_all = sixteens(b.rank);
        const auto fill_terms = [&](int tile) {
            const uint32_t to = smem_u32(terms) + (uint32_t)((tile & 1) * X * kATile * pitch * 2);
#pragma unroll
            for (int row = (int)threadIdx.x / (kRows / 8); row < kATile; row += kThreads / (kRows / 8)) {
                const int tok = order[tile % 3 * kATile + row], c = (int)threadIdx.x % (kRows / 8) * 8;
                const bool zeros = tok < 0 || j0 + c >= ranks_all;
                const uint16_t* from = a.mid + (zeros ? 0 : (long long)tok * ranks_all + j0 + c);
#pragma unroll
                for (int n = 0; n < X; ++n)
                    ring_load8<false>(to + (uint32_t)(((n * kATile + row) * pitch + c) * 2), reinterpret_cast<const __nv_bfloat16*>(from + (long long)n * b.tokens * ranks_all), zeros);
            }
        };
        int t_next = t_first, next = 0, fstage = 0;   // next: t_next's place in `order`
        const auto fill = [&]() {
            if (t_next < t_last && loads) {
                const uint32_t to = ring + (uint32_t)(fstage * S::kStage);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    // tokens behind the last are zeros: their terms are, and zero times a NaN is none
                    const long long row = offset[next + 2 * q + (k & 1) + (k >> 1) * 8];
                    if (VEC)
                        ring_load8<(RH > 1)>(to + k * kPackBytes<T>, x + row, row < 0);
                    else
                        ring_load(to + k * kPackBytes<T>, x + row, row >= 0 ? have : 0, a.align_x);
                }
            }
            t_next += 16;
            next += 16;
            if (next == 3 * kATile) next = 0;
            ring_commit();
            if (++fstage == S::kStages) fstage = 0;
        };
        const uint32_t bar = smem_u32(bars), rows0 = smem_u32(raw);
        const uint32_t row_bytes = (uint32_t)min((long long)kAThreads * 2, a.wide - cb) * (uint32_t)sizeof(T);
        const auto fill_rows = [&](int tile) {   // a thread a row; rows that fill up the last sixteen are zeros
            const int n = min(kATile, t_last - (t_first + tile * kATile));
            const uint32_t to = rows0 + (uint32_t)((tile & 1) * kATile * S::kRowPitch);
            for (int i = threadIdx.x; i < ((n + 15) / 16 * 16 - n) * (S::kRowPitch / 16); i += kThreads)
                ring_store16(to + (uint32_t)((n + i / (S::kRowPitch / 16)) * S::kRowPitch + i % (S::kRowPitch / 16) * 16), make_uint4(0, 0, 0, 0));
            before_copies();
            if (threadIdx.x == 0) mbar_expect(bar + 8 * (tile & 1), (uint32_t)n * row_bytes);
            if ((int)threadIdx.x < n)
                bulk_load(to + threadIdx.x * S::kRowPitch, static_cast<const T*>(a.x) + offset[tile % 3 * kATile + threadIdx.x] + cb, row_bytes, bar + 8 * (tile & 1));
        };
        if (S::kBulk && threadIdx.x == 0) {
            mbar_init(bar, 1);
            mbar_init(bar + 8, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        keep(0, token(0));
        keep(1, token(1));
        int row2 = token(2);
        __syncthreads();
        fill_terms(0);
        if constexpr (S::kBulk) {
            ring_commit();
            fill_rows(0);
        } else {
            for (int s = 0; s < S::kStages - 1; ++s) fill();
        }
        int stage = 0, tile = 0;
        for (int t0 = t_first; t0 < t_last; t0 += kATile, ++tile) {
            const int n_tokens = min(kATile, t_last - t0);
            if constexpr (S::kBulk) {
                ring_wait(0);
                late = !__syncthreads_and(!copies_late(bar + 8 * (tile & 1), (uint32_t)(tile >> 1) & 1));   // ... and the tile before is read
                if (late) break;
            } else {
                // this tile's terms came with the first group of the tile before, or the first of all
                ring_wait(tile == 0 ? S::kStages - 2 : min(S::kStages - 1, 3));
                __syncthreads();   // ... for all, and the tile before's are read, its tokens, too
            }
            const uint32_t terms_now = terms_at + (uint32_t)((tile & 1) * X * kATile * pitch * 2);
            keep(tile + 2, row2);
            row2 = token(tile + 3);
            if (t0 + kATile < t_last) {
                fill_terms(tile + 1);
                if constexpr (S::kBulk) fill_rows(tile + 1);
            }
            if constexpr (S::kBulk) ring_commit();
#pragma unroll 1
            for (int s = 0; s * 16 < n_tokens; ++s) {
                if constexpr (!S::kBulk) {
                    fill();
                    ring_wait(S::kStages - 1);
                }
                if (!idle) {
                    uint32_t lo[Y][8], hi[Y][8];
                    Pack8<T> f, f2;
                    if constexpr (S::kBulk) {
                        const uint32_t from = rows0 + (uint32_t)(((tile & 1) * kATile + s * 16 + 2 * q) * S::kRowPitch + (group * 64 + 8 * g) * (int)sizeof(T));
                        f.q[0] = ring_read16(from);
                        f2.q[0] = ring_read16(from + S::kRowPitch);
                        cut_rows<Y>(lo, f, f2);
                        f.q[0] = ring_read16(from + 8 * S::kRowPitch);
                        f2.q[0] = ring_read16(from + 9 * S::kRowPitch);
                        cut_rows<Y>(hi, f, f2);
                    } else {
                        const uint32_t from = ring + (uint32_t)(stage * S::kStage);
                        ring_read(f, from);
                        ring_read(f2, from + kPackBytes<T>);
                        cut_rows<Y>(lo, f, f2);
                        ring_read(f, from + 2 * kPackBytes<T>);
                        ring_read(f2, from + 3 * kPackBytes<T>);
                        cut_rows<Y>(hi, f, f2);
                    }
#pragma unroll
                    for (int m = 0; m < RT; ++m) {
                        uint32_t w[X][4];
#pragma unroll
                        for (int n = 0; n < X; ++n) load_terms<true>(w[n], terms_now + (uint32_t)(((n * kATile + s * 16) * pitch + m * 16) * 2));
#pragma unroll
                        for (int e = 0; e < 8; ++e) add_products<X, Y, sizeof(W) == 4>(acc[m][e], w, &lo[0][e], &hi[0][e], 8);
                    }
                }
                if (++stage == S::kStages) stage = 0;
            }
        }
        ring_wait(0);
        __syncthreads();
    }
    float* sums = reinterpret_cast<float*>(raw);
#pragma unroll
    for (int m = 0; m < RT; ++m)
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int n = 0; n < 4; ++n) sums[((m * 8 + e) * 4 + n) * kThreads + threadIdx.x] = late ? __uint_as_float(0x7fffffffu) : acc[m][e][n];   // (summed up again below)
    if (b.parts > 1)
        cluster_sync();
    else
        __syncthreads();
    // a thread: eight neighbours of a row, summed over the cluster's blocks
    W* out = static_cast<W*>(a.out) + ((long long)i * b.rank + j0) * a.wide;
    for (int n = part * kThreads + threadIdx.x; n < kRows * 64; n += b.parts * kThreads) {
        const int j = n / 64, w = n % 64 / 8, qq = n % 8 / 2, r8 = j % 16;
        const int at = (j / 16 % RT * 32 + (n & 1) + (r8 >> 3) * 2) * kThreads + (j / (16 * RT) * 8 + w) * 32 + (r8 & 7) * 4 + qq;
        const long long c = cb + w * 64 + 8 * (n % 8);
        if (j >= ranks || c >= a.wide) continue;
        Pack8<W> v;
        bool again = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t from = smem_u32(&sums[at + e * 4 * kThreads]);
            float s = 0.f;
            for (int p = 0; p < b.parts; ++p) s += b.parts > 1 ? ld_cluster(map_rank(from, (uint32_t)p)) : sums[at + e * 4 * kThreads];
            again |= s != s;
            v.e[e] = from_float<W>(s * a.scale);
        }
        write8(out + (long long)j * a.wide + c, v, (int)min(8ll, a.wide - c), a.align_out >= 16);
        if (again)
            over_again(a.mid + j0 + j, (long long)b.tokens * sixteens(b.rank), sixteens(b.rank), static_cast<const T*>(a.x) + c, a.x_stride, b.plan.order + begin, end - begin, a.scale,
                       out + (long long)j * a.wide + c, (int)min(8ll, a.wide - c));
    }
    if (b.parts > 1) cluster_sync();
}

// ---- single tokens -------------------------------------------------------------------------------------

// Few tokens, each with an adapter of its own choice: a cluster of blocks has a token.  Each block takes a run of the input for
// all rows of the adapter, the runs' sums meet through distributed shared memory, and each block writes a run of the output.  Bound
// by the adapters' bytes and, for a few tokens, by the latency of those two steps (32 tokens, rank 16, 4096 -> 4096 8.1 us).
struct AdapterFewArgs {
    const void *x, *down, *up, *base;
    void* out;
    const int* ids;
    uint32_t* status;
    long long x_stride, base_stride, out_stride;
    int count, rank, inner, outer, parts;
    int align_x, align_down;
    int pairs;   // columns of up, base and out can be taken by twos
    float scale;
};

template <typename T, int N> struct Few { T e[N]; };

template <typename T, typename W, int N> __device__ __forceinline__ void few_columns(const AdapterFewArgs& a, int id, long long t, int begin, int end, const float* mid) {
    using BV = Few<T, N>;
    using WV = Few<W, N>;
    const T* base = static_cast<const T*>(a.base) + (a.base ? t * a.base_stride : 0);
    T* out = static_cast<T*>(a.out) + t * a.out_stride;
    const W* up = static_cast<const W*>(a.up) + (long long)max(id, 0) * a.rank * a.outer;
    const int rank = id < 0 ? 0 : a.rank;
    for (int c = begin + (int)threadIdx.x * N; c < end; c += kAFewThreads * N) {
        float acc[N] = {};
        // (an alignment that the host has seen to: 2 N or 4 N bytes)
        alignas(N * sizeof(T)) BV b = {};
        if (a.base) {
#pragma unroll
            for (int e = 0; e < N; ++e) b.e[e] = base[c + e];
        }
        int j = 0;
        for (; j + 8 <= rank; j += 8) {
            WV w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const W* p = up + (long long)(j + k) * a.outer + c;
                if constexpr (N == 2 && sizeof(W) == 4) {
                    const float2 v = __ldg(reinterpret_cast<const float2*>(p));
                    w[k].e[0] = v.x, w[k].e[1] = v.y;
                } else if constexpr (N == 2) {
                    const uint32_t v = __ldg(reinterpret_cast<const uint32_t*>(p));
                    w[k] = *reinterpret_cast<const WV*>(&v);
                } else {
                    w[k].e[0] = *p;
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] = fmaf(mid[j + k], to_float(w[k].e[e]), acc[e]);
        }
        for (; j < rank; ++j)
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] = fmaf(mid[j], to_float(up[(long long)j * a.outer + c + e]), acc[e]);
#pragma unroll
        for (int e = 0; e < N; ++e) out[c + e] = rank ? from_float<T>(fmaf(a.scale, acc[e], to_float(b.e[e]))) : b.e[e];
    }
}

template <typename T, typename W> __global__ void __launch_bounds__(kAFewThreads) k_adapter_few(AdapterFewArgs a) {
    __shared__ float own[SBC_ADAPTER_RANK], mid[SBC_ADAPTER_RANK];
    after_earlier_kernels();
    const int part = (int)blockIdx.x % a.parts;
    const long long t = blockIdx.x / a.parts;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int id = a.ids[t];
    if (id >= a.count && threadIdx.x == 0 && part == 0 && a.status) atomicOr(a.status, SBC_STATUS_RANGE);
    if (id < 0 || id >= a.count) id = -1;
    if (id >= 0) {
        const int packs = (a.inner + 7) / 8, p0 = (int)((long long)packs * part / a.parts), p1 = (int)((long long)packs * (part + 1) / a.parts);
        const T* x = static_cast<const T*>(a.x) + t * a.x_stride;
        const W* down = static_cast<const W*>(a.down) + (long long)id * a.rank * a.inner;
        // four rows at a time share a piece of x
        for (int j = warp * 4; j < a.rank; j += kAFewThreads / 32 * 4) {
            float s[4] = {};
            for (int p = p0 + lane; p < p1; p += 32) {
                const int have = a.inner - 8 * p;
                Pack8<T> v;
                Pack8<W> w[4];
                load8(v, x + 8 * p, have, a.align_x);
#pragma unroll
                for (int k = 0; k < 4; ++k) load8(w[k], down + (long long)min(j + k, a.rank - 1) * a.inner + 8 * p, have, a.align_down);
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[k] = fmaf(to_float(v.e[e]), to_float(w[k].e[e]), s[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) s[k] += __shfl_xor_sync(0xffffffffu, s[k], d);
                if (lane == 0 && j + k < a.rank) own[j + k] = s[k];
            }
        }
        if (a.parts > 1)
            cluster_sync();
        else
            __syncthreads();
        for (int j = threadIdx.x; j < a.rank; j += kAFewThreads) {
            float v = 0.f;
            for (int p = 0; p < a.parts; ++p) v += a.parts > 1 ? ld_cluster(map_rank(smem_u32(&own[j]), (uint32_t)p)) : own[j];
            mid[j] = v;
        }
        if (a.parts > 1)
            cluster_sync();   // (nobody's sums are read any more: a block may end)
        else
            __syncthreads();
    } else if (a.base == a.out) {
        return;
    }
    const int pieces = (a.outer + 1) / 2, begin = (int)((long long)pieces * part / a.parts) * 2, end = min(a.outer, (int)((long long)pieces * (part + 1) / a.parts) * 2);
    if (a.pairs)
        few_columns<T, W, 2>(a, id, t, begin, end, mid);
    else
        few_columns<T, W, 1>(a, id, t, begin, end, mid);
}

}  // namespace sbclm
