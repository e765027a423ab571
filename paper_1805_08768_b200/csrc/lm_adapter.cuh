// Low-rank adapters of many clients or requests beside a shared projection.
//
//   forward   mid = x D_i^T,  y = base + s mid P_i           (D_i: rank x inner, P_i: rank x outer)
//   backward  dmid = s dy P_i^T,  dx = base + dmid D_i,  dD_i = dmid_i^T x_i,  dP_i = s mid_i^T dy_i
//
// i is the adapter of a token.  Both factors have `rank` rows of a wide matrix, so two kernels make all six
// products: into the rank (contracting the wide axis), out of it, and a third sums over an adapter's tokens.
// All are bound by memory: a rank of 16 is 16 to 32 operations for each byte of x, base and y, which warp-wide
// products (16 x 8 x 16) make many times over; nothing is staged for the tensor cores that a thread
// can load from where it lies.
//
// As good as 32-bit arithmetic whatever the types: an operand goes into the products as the bfloat16 terms that it is the sum of (one
// for bfloat16, two for float16, three for float32, cut off rather than rounded, so that none overflows),
// and of the terms' products those count that are not below 2^-24 of the first.  mid and dmid are floats.  Where a result
// has 32 bits, a product's sum starts from zero and is added by an ordinary addition: the tensor cores cut off what they
// align to a running sum, which over 4096 elements came to 1.6e-6 of the result instead of 1e-7.
//
// Tokens come in any order.  A plan groups them: the tokens of an adapter one behind the other in the order in which
// they came (so sums have one order), cut into tiles of 64.
#pragma once

#include "../../include/sbc_block.h"
#include "lm_common.cuh"

namespace sbclm {

constexpr int kATile = 64;        // tokens of a tile
constexpr int kAThreads = 256;
constexpr int kAFewThreads = 256;
constexpr int kAGradThreads = 128;
constexpr int kAPlanThreads = 1024;
constexpr int kARank = 64;        // rank rows that a block takes at a time

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
    for (int t0 = first; t0 < last; t0 += 32) {
        const bool in = t0 + lane < last;
        const int id = in ? a.ids[t0 + lane] : -1;
        beyond |= id >= a.count;
        const int bin = in ? adapter_of(id, a.count) : -1;
        const unsigned same = __match_any_sync(0xffffffffu, bin);
        if (in && (same & ((1u << lane) - 1)) == 0) mine[bin] += __popc(same);
        __syncwarp();
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
    for (int t0 = first; t0 < last; t0 += 32) {
        const bool in = t0 + lane < last;
        const int bin = in ? adapter_of(a.ids[t0 + lane], a.count) : -1;
        const unsigned same = __match_any_sync(0xffffffffu, bin), ahead = same & ((1u << lane) - 1);
        int at = 0;
        if (in && ahead == 0) {
            at = mine[bin];
            mine[bin] = at + __popc(same);
        }
        at = __shfl_sync(0xffffffffu, at, __ffs(same) - 1) + __popc(ahead);
        if (in) a.plan.order[at] = t0 + lane;
        __syncwarp();
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

// Products of sixteen rows of X terms in shared memory (`p`: this thread's place in the first, `next` from term to term) with
// eight tiles of eight columns of Y terms in registers.
template <int X, int Y, bool APART>
__device__ __forceinline__ void add_products(float (*acc)[4], const uint16_t* p, int next, int pitch, const uint32_t (*lo)[8], const uint32_t (*hi)[8]) {
    uint32_t w[X][4];
#pragma unroll
    for (int n = 0; n < X; ++n) {
        const uint16_t* from = p + n * next;
        w[n][0] = *reinterpret_cast<const uint32_t*>(from);
        w[n][1] = *reinterpret_cast<const uint32_t*>(from + 8 * pitch);
        w[n][2] = *reinterpret_cast<const uint32_t*>(from + 8);
        w[n][3] = *reinterpret_cast<const uint32_t*>(from + 8 * pitch + 8);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float part[4] = {};
        float* d = APART ? part : acc[e];
#pragma unroll
        for (int order = X - 1; order >= 0; --order)   // the small products first
#pragma unroll
            for (int n = 0; n < X; ++n) {
                const int o = order - n;
                if (o >= 0 && o < Y) mma_terms(d, w[n], lo[o][e], hi[o][e]);
            }
        if (APART)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[e][k] += part[k];
    }
}

// (plain loads: what they read may be written in place)
template <typename T> __device__ __forceinline__ void read8(Pack8<T>& v, const T* p, int have, bool vec) {
    if (have >= 8 && vec) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v.q[i] = reinterpret_cast<const uint4*>(p)[i];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v.e[e] = e < have ? p[e] : from_float<T>(0.f);
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
    const void* x;          // the wide input (x or dy) of mid, or what is added up over tokens
    const void* factor;     // [count][rank][wide]
    const void* base;
    void* out;              // y or dx; [count][rank][wide] gradients
    float* mid;             // [tokens][rank]
    AdapterPlan plan;
    long long x_stride, base_stride, out_stride;
    int count, rank, wide, parts;
    int align_x, align_factor;
    float scale;
};

// ---- into the rank ------------------------------------------------------------------------------

// mid[t][j] = scale sum_k x[t][k] factor[i][j][k] for a tile of tokens and up to 8 JT rows.  A thread takes eight neighbours
// of a row, its four k's of two products (which element is which k is free as long as both operands agree).  Warps are
// two halves of the tokens and four runs of the wide axis, blocks of a cluster share it further; sums meet
// in shared memory in a fixed order.
template <typename T, typename W, int JT> __global__ void __launch_bounds__(kAThreads) k_adapter_in(AdapterArgs a) {
    constexpr int X = Terms<T>::n, Y = Terms<W>::n, MT = 2, kPer = MT * JT * 4;
    extern __shared__ float sums[];   // [8 warps][kPer][32]
    __shared__ int tokens[kATile];
    after_earlier_kernels();
    const int part = (int)blockIdx.x % a.parts, tile = (int)blockIdx.x / a.parts;
    if (tile >= a.plan.tiles[0].x) return;
    const int4 at = a.plan.tiles[1 + tile];
    if (at.x >= a.count) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3, half = warp & 1, run = warp >> 1;
    const int j0 = (int)blockIdx.y * 8 * JT;
    if (threadIdx.x < kATile) tokens[threadIdx.x] = threadIdx.x < at.z ? a.plan.order[at.y + threadIdx.x] : -1;
    __syncthreads();
    const T* x[MT][2];
    bool live[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int t = tokens[half * 32 + m * 16 + h * 8 + g];
            live[m][h] = t >= 0;
            x[m][h] = static_cast<const T*>(a.x) + (long long)max(t, 0) * a.x_stride;
        }
    const W* f[JT];
#pragma unroll
    for (int j = 0; j < JT; ++j) f[j] = static_cast<const W*>(a.factor) + ((long long)at.x * a.rank + min(j0 + 8 * j + g, a.rank - 1)) * a.wide;
    float acc[MT][JT][4] = {};
    if (half * 32 < at.z) {
        const int units = (a.wide + 31) / 32;   // of 32 elements; this block's run of them
        const int u0 = (int)((long long)units * part / a.parts), u1 = (int)((long long)units * (part + 1) / a.parts);
        for (int u = u0 + run; u < u1; u += 4) {
            const int k = u * 32 + q * 8, have = a.wide - k;
            Pack8<T> xs[MT][2];
            Pack8<W> fs[JT];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) load8(xs[m][h], x[m][h] + k, live[m][h] ? have : 0, a.align_x);
#pragma unroll
            for (int j = 0; j < JT; ++j) load8(fs[j], f[j] + k, j0 + 8 * j + g < a.rank ? have : 0, a.align_factor);
            uint32_t xt[MT][2][X][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) cut_row<X>(xt[m][h], xs[m][h]);
#pragma unroll
            for (int j = 0; j < JT; ++j) {
                uint32_t ft[Y][4];
                cut_row<Y>(ft, fs[j]);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    float part[4] = {};
                    float* d = sizeof(W) == 4 ? part : acc[m][j];
#pragma unroll
                    for (int order = 2; order >= 0; --order)   // the small products first
#pragma unroll
                        for (int n = 0; n < X; ++n) {
                            const int o = order - n;
                            if (o < 0 || o >= Y) continue;
#pragma unroll
                            for (int s = 0; s < 4; s += 2) {
                                const uint32_t w[4] = {xt[m][0][n][s], xt[m][1][n][s], xt[m][0][n][s + 1], xt[m][1][n][s + 1]};
                                mma_terms(d, w, ft[o][s], ft[o][s + 1]);
                            }
                        }
                    if (sizeof(W) == 4)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[m][j][e] += part[e];
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[(warp * kPer + (m * JT + j) * 4 + e) * 32 + lane] = acc[m][j][e];
    __syncthreads();
    // [2 halves][kPer][32] sums of four warps, left in the first ones' places for the cluster
    const auto place = [&](int i, int w) { return (((i / (kPer * 32)) + 2 * w) * kPer * 32) + i % (kPer * 32); };
    const auto store = [&](int i, float v) {
        const int n = i % 32, e = i / 32 % 4, j = i / 128 % JT, m = i / (128 * JT);   // m: halves and their tiles
        const int t = m * 16 + (e >> 1) * 8 + (n >> 2), r = j0 + 8 * j + (n & 3) * 2 + (e & 1);
        if (t < at.z && r < a.rank) a.mid[(long long)tokens[t] * a.rank + r] = v * a.scale;
    };
    for (int i = threadIdx.x; i < 2 * kPer * 32; i += kAThreads) {
        float v = sums[place(i, 0)];
#pragma unroll
        for (int w = 1; w < 4; ++w) v += sums[place(i, w)];
        if (a.parts == 1)
            store(i, v);
        else
            sums[place(i, 0)] = v;
    }
    if (a.parts == 1) return;
    cluster_sync();
    for (int i = part * kAThreads + threadIdx.x; i < 2 * kPer * 32; i += a.parts * kAThreads) {
        const uint32_t from = smem_u32(&sums[place(i, 0)]);
        float v = 0.f;
        for (int p = 0; p < a.parts; ++p) v += ld_cluster(map_rank(from, (uint32_t)p));
        store(i, v);
    }
    cluster_sync();
}

// ---- out of the rank ------------------------------------------------------------------------------

// out[t][c] = base[t][c] + scale sum_j mid[t][j] factor[i][j][c].  A warp has 32 tokens x 64 columns at a time.  mid's terms
// wait in shared memory; a thread loads eight neighbours of four rows of the factor, whose pairs are the products' words (which
// column is which of a product's eight is free, too), and ends with sixteen neighbours of four rows of out.
template <typename T, typename W> __global__ void __launch_bounds__(kAThreads) k_adapter_out(AdapterArgs a) {
    // 16-bit results: what lies 2^-16 below a factor does not reach them
    constexpr int X = sizeof(T) == 4 ? 3 : 2, Y = sizeof(T) == 4 ? Terms<W>::n : (Terms<W>::n < 2 ? Terms<W>::n : 2), MT = 2;
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ int tokens[kATile];
    after_earlier_kernels();
    if ((int)blockIdx.x >= a.plan.tiles[0].x) return;
    const int4 at = a.plan.tiles[1 + blockIdx.x];
    const bool none = at.x >= a.count;
    if (none && a.base == a.out) return;
    const int steps = none ? 0 : (a.rank + 15) / 16, pitch = (a.rank + 15) / 16 * 16 + 8;
    uint16_t* terms = reinterpret_cast<uint16_t*>(raw);   // [X][kATile][pitch]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3, half = warp & 1;
    if (threadIdx.x < kATile) tokens[threadIdx.x] = threadIdx.x < at.z ? a.plan.order[at.y + threadIdx.x] : -1;
    __syncthreads();
    for (int i = threadIdx.x; i < kATile * steps * 16; i += kAThreads) {
        const int t = i / (steps * 16), j = i - t * steps * 16;
        uint32_t w[X];
        cut<X>(w, tokens[t] >= 0 && j < a.rank ? a.mid[(long long)tokens[t] * a.rank + j] : 0.f);
#pragma unroll
        for (int n = 0; n < X; ++n) terms[(n * kATile + t) * pitch + j] = (uint16_t)(w[n] >> 16);
    }
    __syncthreads();
    if (half * 32 >= at.z) return;
    const W* factor = static_cast<const W*>(a.factor) + (long long)at.x * a.rank * a.wide;
    const bool vec_base = a.align_x >= 16;   // (align_x: of base and out)
    int row[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) row[m][h] = tokens[half * 32 + m * 16 + h * 8 + g];
    for (int c0 = ((int)blockIdx.y * 4 + (warp >> 1)) * 64; c0 < a.wide; c0 += (int)gridDim.y * 256) {
        const int col = c0 + 16 * q;     // of base and out
        Pack8<T> b[MT][2][2];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    read8(b[m][h][p], static_cast<const T*>(a.base) + (a.base ? (long long)row[m][h] * a.base_stride + col + 8 * p : 0),
                          a.base && row[m][h] >= 0 ? a.wide - col - 8 * p : 0, vec_base);
        float acc[MT][8][4] = {};
        const int fc = c0 + 8 * g, have = a.wide - fc;   // of the factor
        for (int s = 0; s < steps; ++s) {
            Pack8<W> f[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int j = s * 16 + 2 * q + (k & 1) + (k >> 1) * 8;
                load8(f[k], factor + (long long)min(j, a.rank - 1) * a.wide + fc, j < a.rank ? have : 0, a.align_factor);
            }
            uint32_t lo[Y][8], hi[Y][8];
            cut_rows<Y>(lo, f[0], f[1]);
            cut_rows<Y>(hi, f[2], f[3]);
#pragma unroll
            for (int m = 0; m < MT; ++m)
                add_products<X, Y, sizeof(T) == 4>(acc[m], terms + (half * 32 + m * 16 + g) * pitch + s * 16 + 2 * q, kATile * pitch, pitch, lo, hi);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (row[m][h] < 0) continue;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    Pack8<T> v;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v.e[e] = none ? b[m][h][p].e[e] : from_float<T>(fmaf(a.scale, acc[m][e][2 * h + p], to_float(b[m][h][p].e[e])));
                    write8(static_cast<T*>(a.out) + (long long)row[m][h] * a.out_stride + col + 8 * p, v, a.wide - col - 8 * p, vec_base);
                }
            }
    }
}

// ---- over tokens ------------------------------------------------------------------------------------

// out[i][j][c] = scale sum over the tokens t of adapter i of mid[t][j] x[t][c].  A warp has 64 columns and up to 16 RT rows; 64
// tokens' terms of mid are laid out in shared memory with the tokens as the contiguous axis, x is loaded as the factor above.
// Blocks of a cluster share an adapter's tokens, and add their sums in their order.
template <typename T, typename W, int RT> __global__ void __launch_bounds__(kAGradThreads) k_adapter_grad(AdapterArgs a) {
    constexpr int X = sizeof(W) == 4 ? 3 : 2, Y = sizeof(W) == 4 ? Terms<T>::n : (Terms<T>::n < 2 ? Terms<T>::n : 2), pitch = kATile + 8;
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ int tokens[kATile];
    uint16_t* terms = reinterpret_cast<uint16_t*>(raw);   // [X][16 RT][pitch], and in the end sums [32 RT][threads]
    float* sums = reinterpret_cast<float*>(raw);
    after_earlier_kernels();
    const int part = (int)(blockIdx.x % a.parts), blocks = (a.rank + 16 * RT - 1) / (16 * RT);
    const int columns = (int)(((long long)a.wide + kAGradThreads * 2 - 1) / (kAGradThreads * 2)), at_row = (int)(blockIdx.x / a.parts / columns);
    const int i = at_row / blocks, j0 = at_row % blocks * 16 * RT, ranks = min(16 * RT, a.rank - j0);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const long long cb = (long long)(blockIdx.x / a.parts % columns) * (kAGradThreads * 2);
    const long long c0 = cb + warp * 64 + 8 * g;
    const int have = (int)max(0ll, min(8ll, a.wide - c0));
    const int begin = a.plan.offsets[i], groups = (a.plan.offsets[i + 1] - begin + 15) / 16, end = a.plan.offsets[i + 1];
    const int g0 = (int)((long long)groups * part / a.parts), g1 = (int)((long long)groups * (part + 1) / a.parts);
    float acc[RT][8][4] = {};
    for (int t0 = begin + g0 * 16; t0 < min(end, begin + g1 * 16); t0 += kATile) {
        const int n_tokens = min(kATile, min(end, begin + g1 * 16) - t0);
        __syncthreads();
        if (threadIdx.x < kATile) tokens[threadIdx.x] = threadIdx.x < n_tokens ? a.plan.order[t0 + threadIdx.x] : -1;
        __syncthreads();
        for (int n = threadIdx.x; n < kATile * 16 * RT; n += kAGradThreads) {
            const int t = n / (16 * RT), j = n % (16 * RT);
            uint32_t w[X];
            cut<X>(w, tokens[t] >= 0 && j < ranks ? a.mid[(long long)tokens[t] * a.rank + j0 + j] : 0.f);
#pragma unroll
            for (int k = 0; k < X; ++k) terms[(k * 16 * RT + j) * pitch + t] = (uint16_t)(w[k] >> 16);
        }
        Pack8<T> next[4];
        const auto fetch = [&](int s) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = tokens[s * 16 + 2 * q + (k & 1) + (k >> 1) * 8];
                load8(next[k], static_cast<const T*>(a.x) + (long long)max(t, 0) * a.x_stride + c0, t >= 0 ? have : 0, a.align_x);
            }
        };
        fetch(0);
        __syncthreads();
#pragma unroll 1
        for (int s = 0; s * 16 < n_tokens; ++s) {
            uint32_t lo[Y][8], hi[Y][8];
            cut_rows<Y>(lo, next[0], next[1]);
            cut_rows<Y>(hi, next[2], next[3]);
            if ((s + 1) * 16 < n_tokens) fetch(s + 1);
#pragma unroll
            for (int m = 0; m < RT; ++m)
                add_products<X, Y, sizeof(W) == 4>(acc[m], terms + (m * 16 + g) * pitch + s * 16 + 2 * q, 16 * RT * pitch, pitch, lo, hi);
        }
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < RT; ++m)
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int n = 0; n < 4; ++n) sums[((m * 8 + e) * 4 + n) * kAGradThreads + threadIdx.x] = acc[m][e][n];
    if (a.parts > 1)
        cluster_sync();
    else
        __syncthreads();
    // a thread: eight neighbours of a row, summed over the cluster's blocks
    W* out = static_cast<W*>(a.out) + ((long long)i * a.rank + j0) * a.wide;
    const bool vec = a.align_factor >= 16;
    for (int n = part * kAGradThreads + threadIdx.x; n < 16 * RT * 32; n += a.parts * kAGradThreads) {
        const int j = n / 32, w = n % 32 / 8, qq = n % 8 / 2, r8 = j % 16;
        const int at = (j / 16 * 32 + (n & 1) + (r8 >> 3) * 2) * kAGradThreads + w * 32 + (r8 & 7) * 4 + qq;
        const long long c = cb + w * 64 + 8 * (n % 8);
        if (j >= ranks || c >= a.wide) continue;
        Pack8<W> v;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t from = smem_u32(&sums[at + e * 4 * kAGradThreads]);
            float s = 0.f;
            for (int p = 0; p < a.parts; ++p) s += a.parts > 1 ? ld_cluster(map_rank(from, (uint32_t)p)) : sums[at + e * 4 * kAGradThreads];
            v.e[e] = from_float<W>(s * a.scale);
        }
        write8(out + (long long)j * a.wide + c, v, (int)min(8ll, a.wide - c), vec);
    }
    if (a.parts > 1) cluster_sync();
}

// ---- single tokens -------------------------------------------------------------------------------------

// Few tokens, each with an adapter of its own choice: a cluster of blocks has a token.  Each block takes a run of the input for
// all rows of the adapter, the runs' sums meet through distributed shared memory, and each block writes a run of the output.  Bound
// by the adapters' bytes and, for a few tokens, by the latency of those two steps.
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
