// The gated feed-forward block h = act(x G^T) * (x U^T), forward and backward, bfloat16 or float16 with
// sums in 32 bits on the tensor cores.
//
//   forward   g = x G^T, u = x U^T, h = act(g) u; for the backward pass P = u act'(g) and Q = act(g) are kept
//   backward  dg = dh P, du = dh Q (rounded to the inputs' type, in which the tensor cores take them)
//             dx = dg G + du U,  dG = dg^T x,  dU = du^T x
//
// One kernel makes all four products.  out[n][m] = sum_k R[m][k] C[n][k]: R's rows are the accumulator's
// lanes (the contiguous axis of the output, so that a warp's stores are), C's its columns.  The
// operands are read as they lie: with k contiguous (forward) or with m or n contiguous (the transposed ones
// of the backward pass), which is a bit of the instruction and another box, no copy.
#pragma once

#include "../../include/sbc_block.h"
#include "lm_common.cuh"
#include "lm_product.cuh"

namespace sbclm {

// ---- activations ------------------------------------------------------------------------

// act(g) and its derivative.  Sigmoids by exp(-|g|), so that small ones keep their digits down to the smallest numbers.  The fast
// exponential and quotient (off by (2 + 1.2 |z|) 2^-23 and 2^-22 of themselves) are far below the results' 2^-9 or 2^-12, and the
// epilogue is what the tensor cores wait for.
template <int ACT, bool SLOPE> __device__ __forceinline__ void activate(float g, float& value, float& slope) {
    if (ACT == SBC_ACT_RELU) {
        value = g < 0.f ? 0.f : g;   // (a NaN stays one)
        if (SLOPE) slope = g > 0.f ? 1.f : 0.f;
        return;
    }
    if (ACT == SBC_ACT_GELU) {
        const float p = normcdff(g);
        value = g * p;
        if (SLOPE) {
            const float density = __expf(-0.5f * g * g);
            slope = density == 0.f ? p : fmaf(g * 0.3989422804f, density, p);   // (an infinite g times nothing)
        }
        return;
    }
    // share = 1 / (1 + exp(-z)), other = 1 - share
    float z = g, dz = 1.f;
    if (ACT == SBC_ACT_GELU_TANH) {
        z = 1.5957691216f * g * fmaf(0.044715f, g * g, 1.f);
        if (SLOPE) dz = 1.5957691216f * fmaf(3.f * 0.044715f, g * g, 1.f);
    }
    const float e = __expf(-fabsf(z)), large = __fdividef(1.f, 1.f + e), small = e * large;   // (the divisor is 1 .. 2)
    const float share = z > 0.f ? large : small, other = z > 0.f ? small : large;
    if (ACT == SBC_ACT_SIGMOID) {
        value = share;
        if (SLOPE) slope = share * other;
    } else {
        value = g * share;
        // (far out g dz leaves 32 bits where what it is multiplied by has become zero)
        if (SLOPE) slope = share == 0.f ? 0.f : other == 0.f ? share : share * fmaf(g * dz, other, 1.f);
    }
}

// f(constant) with the activation of that number: asked once for many elements.
template <int N> struct Act { static constexpr int n = N; };
template <typename F> __device__ __forceinline__ void by_act(int act, F f) {
    switch (act) {
        case SBC_ACT_SILU: return f(Act<SBC_ACT_SILU>());
        case SBC_ACT_GELU: return f(Act<SBC_ACT_GELU>());
        case SBC_ACT_GELU_TANH: return f(Act<SBC_ACT_GELU_TANH>());
        case SBC_ACT_RELU: return f(Act<SBC_ACT_RELU>());
        default: return f(Act<SBC_ACT_SIGMOID>());
    }
}

// ---- products on the tensor cores ---------------------------------------------------------
//
// Pairs of blocks on neighbouring SMs share a tile of 256 lanes x NT (256 or 128) columns, as in the 4-bit
// product: each loads its 128 rows of R and half of C's, the tensor cores of both read both halves.  Blocks
// stay; loads run ahead across tiles, and two accumulators let a tile's epilogue run under the next one's
// products.  Tiles go in groups of eight along C, so that what is under way at a time is about as wide as
// it is high and its operands stay in L2 (one row of tiles at a time would read all of a large R from memory
// for every 256 tokens).
//
// Forward: R is made of both weights, a block's lanes 0..63 are rows of G and 64..127 the same rows of U.  Of the two
// warps that hold the two factors of the same units, each gives the other half of its tokens through shared memory and ends
// with both factors of the rest.  (Sixteen rows of each in turn would leave both in one warp, but eight small boxes
// a stage are slower to load than two: 8192 x 4096 -> 8192 without kept factors 964 us.)
//
// 8192 x 4096 -> 8192 bfloat16, alone: forward 730 us (1.51 PFLOP/s; a library product of that size takes 670 to 690), with kept
// factors 782, input's gradient 692 (1.59 PFLOP/s), weights' gradients 738: the tensor cores under the power limit.  Few tiles leave pairs
// idle, and the contracted axis is not split: 2240 x 650 -> 2600 float16 42, 32 and 20 us.
//
// Warps: 0..7 accumulator to memory (half of the columns each four), 8 loads, 9 multiplies (in the pair's first block).

constexpr int kMThreads = 320;
constexpr int kMStages = 8;
constexpr int kMBytes = 128;    // bytes of a row of a box: 64 elements
constexpr int kMSwap = 8 * 2 * 16 * 32 * 4;   // bytes that eight warps swap factors through, twice sixteen tokens each
enum { kForward, kForwardKeep, kInputGrad, kWeightGrad };

struct MmArgs {
    void *out, *out2;           // out2: kWeightGrad, what the second half of C's tiles goes to
    float2* kept;
    uint32_t* status;
    long long out_stride, kept_stride;
    long long rows_m, rows_n;   // rows_m: hidden units (forward) or columns of the output
    int chunks, sources;        // boxes of 64 along the contracted axis, operands one behind the other
    int stages, tiles_m, tiles_n, tiles;   // tiles_n of one output, all tiles
    int act;
};

template <typename T> __device__ __forceinline__ uint32_t half_kind(const T*);
template <> __device__ __forceinline__ uint32_t half_kind<__half>(const __half*) { return 0u; }
template <> __device__ __forceinline__ uint32_t half_kind<__nv_bfloat16>(const __nv_bfloat16*) { return (1u << 7) | (1u << 10); }

// An operand whose rows (m or n) are contiguous: boxes of 64 of them x 64 k, eight k to a kilobyte.
__device__ __forceinline__ uint64_t operand_desc_mn(uint32_t smem) {
    return (uint64_t)((smem & 0x3ffff) >> 4) | ((uint64_t)(8192 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

__device__ __forceinline__ void multiply_half2(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
}

struct MmTile {
    int m, n;
};
__device__ __forceinline__ MmTile mm_tile(int tile, int tiles_m, int tiles_n) {
    const int group = tile / (8 * tiles_m), wide = min(8, tiles_n - 8 * group), at = tile - group * 8 * tiles_m;
    return {at / wide, group * 8 + at % wide};
}

// Columns of an accumulator, this warp's 32 lanes, to rows of `out` (this lane's element of the first).
template <typename O, int COLS, typename F>
__device__ __forceinline__ void store_columns(uint32_t acc, O* out, long long stride, int most, bool mine, bool pairs, bool bad, F free) {
    const float nan = __uint_as_float(0x7fffffffu);
    if constexpr (sizeof(O) == 2) {
        uint32_t w[COLS / 2];
#pragma unroll
        for (int n0 = 0; n0 < COLS; n0 += 32) {
            float v[32];
            tmem_load32(v, acc + n0);
#pragma unroll
            for (int i = 0; i < 32; i += 2) w[(n0 + i) / 2] = bad ? 0x7fff7fffu : pack2(v[i], v[i + 1], (const O*)nullptr);
        }
        free();
        if (pairs) {   // neighbouring lanes swap halves: two elements of one row each
            const bool odd = threadIdx.x & 1;
            O* to = odd ? out - 1 + stride : out;
            const int have = mine ? most - (odd ? 1 : 0) : 0;
#pragma unroll
            for (int n = 0; n < COLS; n += 2) {
                const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? w[n / 2] : w[n / 2] >> 16, 1);
                if (n < have) store_word(to, odd ? __byte_perm(other, w[n / 2], 0x7610) : __byte_perm(w[n / 2], other, 0x5410));
                to += 2 * stride;
            }
        } else {
            const int have = mine ? most : 0;
#pragma unroll
            for (int n = 0; n < COLS; ++n) {
                if (n < have) store_half(out, n & 1 ? w[n / 2] >> 16 : w[n / 2]);
                out += stride;
            }
        }
    } else {
        const int have = mine ? most : 0;
#pragma unroll
        for (int n0 = 0; n0 < COLS; n0 += 32) {
            float v[32];
            tmem_load32(v, acc + n0);
            if (n0 + 32 == COLS) free();
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                if (n0 + i < have) store_word(out, __float_as_uint(bad ? nan : v[i]));
                out += stride;
            }
        }
    }
}

template <typename T, typename O, int MODE, int NT>
__global__ void __launch_bounds__(kMThreads, 1)
    k_mm(const __grid_constant__ CUtensorMap map_r, const __grid_constant__ CUtensorMap map_r2, const __grid_constant__ CUtensorMap map_c,
         const __grid_constant__ CUtensorMap map_c2, MmArgs a) {
    constexpr bool gated = MODE == kForward || MODE == kForwardKeep, r_rows = !gated, c_rows = MODE == kWeightGrad;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * kMStages + 5];
    __shared__ uint32_t tmem_slot, gave_up;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
    constexpr uint32_t bytes_r = 128 * kMBytes, bytes_c = NT / 2 * kMBytes, stage_bytes = bytes_r + bytes_c;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int s) { return bar0 + 16u * s; };        // (first block) both blocks' loads of a stage have landed
    const auto empty = [&](int s) { return bar0 + 16u * s + 8; };   // the products that read a stage are done
    const uint32_t bar1 = bar0 + 16u * kMStages;
    const auto acc_full = [&](int b) { return bar1 + 8u * b; };
    const auto acc_empty = [&](int b) { return bar1 + 16 + 8u * b; };   // (first block)
    const uint32_t drained = bar1 + 32;
    const int pairs = (int)(gridDim.x / 2), pair = (int)(blockIdx.x / 2);
    const int all = a.chunks * a.sources;

    if (t == 0) {
        gave_up = 0;
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), 16);
        }
        mbar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(2u * NT) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_slot;
    after_earlier_kernels();

    if (warp == 8) {
        if (lane == 0) {
            bool ok = true;
            Ring ring;
            int issued = 0;
            for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
                const MmTile at = mm_tile(tile, a.tiles_m, MODE == kWeightGrad ? 2 * a.tiles_n : a.tiles_n);
                const bool second = MODE == kWeightGrad && at.n >= a.tiles_n;
                const int m0 = at.m * (gated ? 128 : 256) + (int)rank * (gated ? 64 : 128);
                const int n0 = (second ? at.n - a.tiles_n : at.n) * NT + (int)rank * (NT / 2);
                const CUtensorMap* c = second ? &map_c2 : &map_c;
                for (int i = 0; i < all; ++i) {
                    ok = mbar_wait(empty(ring.s), ring.turn ^ 1);
                    if (!ok) break;
                    const uint32_t to = smem + (uint32_t)ring.s * stage_bytes, to_c = to + bytes_r, bar = map_rank(full(ring.s), 0);
                    // the second block's bytes may arrive before they are announced: the turn ends with the announcement
                    if (rank == 0) mbar_expect(full(ring.s), 2 * stage_bytes);
                    const bool next = i >= a.chunks;
                    const int k0 = (next ? i - a.chunks : i) * 64;
                    if (gated) {
                        tma_load_2d_pair(to, &map_r, k0, m0, bar);
                        tma_load_2d_pair(to + 8192u, &map_r2, k0, m0, bar);
                    } else {
                        const CUtensorMap* r = next ? &map_r2 : &map_r;
                        tma_load_2d_pair(to, r, m0, k0, bar);
                        tma_load_2d_pair(to + 8192u, r, m0 + 64, k0, bar);
                    }
                    if (c_rows) {
#pragma unroll
                        for (int j = 0; j < NT / 128; ++j) tma_load_2d_pair(to_c + 8192u * j, c, n0 + 64 * j, k0, bar);
                    } else {
                        tma_load_2d_pair(to_c, next ? &map_c2 : &map_c, k0, n0, bar);
                    }
                    ring.next(a.stages);
                    issued = min(issued + 1, a.stages);
                }
            }
            if (!ok) gave_up = 1;
            // no copy and no arrival at a barrier may be on its way when the block ends: every stage's last turn
            for (int j = 0; j < issued; ++j) {
                const int s = ring.s - 1 - j < 0 ? ring.s - 1 - j + a.stages : ring.s - 1 - j;
                const uint32_t turn = ring.s - 1 - j < 0 ? ring.turn ^ 1 : ring.turn;
                if (rank == 0) mbar_wait(full(s), turn);
                mbar_wait(empty(s), turn);
            }
        }
    } else if (warp == 9) {
        if (lane == 0 && rank != 0) mbar_wait(drained, 0);
        if (lane == 0 && rank == 0) {
            bool ok = true;
            // sums in 32 bits, which operands have their rows contiguous, 256 lanes
            const uint32_t idesc = (1u << 4) | half_kind((const T*)nullptr) | (r_rows ? 1u << 15 : 0u) | (c_rows ? 1u << 16 : 0u) |
                                   ((uint32_t)(NT >> 3) << 17) | (16u << 24);
            Ring ring, accs;
            for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
                const int b = accs.s;
                ok = mbar_wait(acc_empty(b), accs.turn ^ 1);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t acc = tmem + (uint32_t)b * NT;
                for (int i = 0; i < all; ++i) {
                    ok = mbar_wait(full(ring.s), ring.turn);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = smem + (uint32_t)ring.s * stage_bytes, at_c = at + bytes_r;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        multiply_half2(acc, r_rows ? operand_desc_mn(at + 2048 * k) : operand_desc(at + 32 * k),
                                       c_rows ? operand_desc_mn(at_c + 2048 * k) : operand_desc(at_c + 32 * k), idesc, (uint32_t)(i > 0 || k > 0));
                    commit2(empty(ring.s));
                    ring.next(a.stages);
                }
                if (ok) commit2(acc_full(b));
                accs.next(2);
            }
            if (!ok) gave_up = 1;
            // no product may be running when tensor memory is given back
            commit2(drained);
            mbar_wait(drained, 0);
        }
    } else {
        bool ok = true;
        constexpr int kCols = NT / 2;
        const int col0 = warp < 4 ? 0 : kCols, sub = warp & 3;
        Ring accs;
        for (int tile = pair; tile < a.tiles; tile += pairs, accs.next(2)) {
            const int b = accs.s;
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(acc_full(b), accs.turn));
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const MmTile at = mm_tile(tile, a.tiles_m, MODE == kWeightGrad ? 2 * a.tiles_n : a.tiles_n);
            const bool second = MODE == kWeightGrad && at.n >= a.tiles_n;
            const long long n0 = (long long)(second ? at.n - a.tiles_n : at.n) * NT + col0;
            const int most = (int)max(0ll, min((long long)kCols, a.rows_n - n0));
            const uint32_t acc = tmem + (uint32_t)b * NT + (uint32_t)col0 + ((uint32_t)sub << 21);
            const auto free = [&] {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(map_rank(acc_empty(b), 0));
            };
            if constexpr (gated) {
                const long long unit = (long long)at.m * 128 + rank * 64 + (sub & 1) * 32 + lane;
                const bool up = sub >= 2;
                // this warp's half of every 32 tokens; the other's go to the partner's place
                const int have = unit < a.rows_m ? most - (up ? 16 : 0) : 0;
                T* out = static_cast<T*>(a.out) + (n0 + (up ? 16 : 0)) * a.out_stride + unit;
                float2* kept = MODE == kForwardKeep ? a.kept + (n0 + (up ? 16 : 0)) * a.kept_stride + unit : nullptr;
                const uint32_t swap = smem + (uint32_t)a.stages * stage_bytes + (uint32_t)lane * 4u;
                const uint32_t give = swap + (uint32_t)(warp ^ 2) * 2048u, take = swap + (uint32_t)warp * 2048u;
                const int meet = 1 + (warp >> 2) * 2 + (sub & 1);
#pragma unroll 1
                for (int c0 = 0; c0 < kCols; c0 += 32) {
                    const uint32_t half = (uint32_t)(c0 & 32) * (kMSwap / 64);
                    float v[32];
                    tmem_load32(v, acc + c0);
                    if (c0 + 32 == kCols) free();
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(give + half + 128u * i), "f"(up ? v[i] : v[16 + i]) : "memory");
                    asm volatile("bar.sync %0, 64;" ::"r"(meet) : "memory");
                    float g[16], u[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float got;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(got) : "r"(take + half + 128u * i) : "memory");
                        g[i] = up ? got : v[i];
                        u[i] = up ? v[16 + i] : got;
                        if (!ok) g[i] = u[i] = __uint_as_float(0x7fffffffu);
                    }
                    by_act(a.act, [&](auto which) {
                        T* to = out + c0 * a.out_stride;
                        float2* keep = kept + c0 * a.kept_stride;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float value, slope = 0.f;
                            activate<decltype(which)::n, MODE == kForwardKeep>(g[i], value, slope);
                            if (c0 + i < have) {
                                *to = from_float<T>(value * u[i]);
                                if (MODE == kForwardKeep) *keep = make_float2(u[i] * slope, value);
                            }
                            to += a.out_stride;
                            if (MODE == kForwardKeep) keep += a.kept_stride;
                        }
                    });
                }
            } else {
                const long long m = (long long)at.m * 256 + rank * 128 + sub * 32 + lane;
                O* out = static_cast<O*>(second ? a.out2 : a.out);
                const bool words = sizeof(O) == 2 && ((a.out_stride | a.rows_m) & 1) == 0 && ((uintptr_t)out & 3) == 0;
                store_columns<O, kCols>(acc, out + n0 * a.out_stride + m, a.out_stride, most, m < a.rows_m, words, !ok, free);
            }
            __syncwarp();
        }
        if (!ok) gave_up = 1;
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (t == 0 && gave_up && a.status) atomicOr(a.status, SBC_STATUS_TIMEOUT);
    cluster_sync();   // the other block's barriers and tensor memory are used up to here
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2u * NT));
}

// ---- few tokens ---------------------------------------------------------------------------
//
// The weights' bytes are all there is to it, so they go from memory to registers and from there into the
// warp-wide products (16 x 8 x 16), whose rate is far above what memory gives up to 32 tokens; no tensor
// map, no staging, any alignment.  A tile is eight hidden units: rows 0..7 of the product are those
// of G, 8..15 of U, so both factors of a unit and a token end in one thread.  Which element of a row is which k
// of a product is free as long as both operands agree: a thread takes eight neighbours of a row, its four
// k's of two products.  The warps of a block share the units and cut the rows in turn; their sums
// meet in shared memory in the warps' order.
//
// 16 tokens x 4096 -> 16384 bfloat16 55 us for 269 MB, 74 % of the copy rate; 1 x 650 -> 2600 6.0 us, latency.

constexpr int kFThreads = 256;
constexpr int kFMost = 32;      // tokens

struct FewArgs {
    const void *x, *gate, *up;
    void* h;
    long long x_stride, gate_stride, up_stride, h_stride, hidden;
    int inner, tokens, act;
    int align_x, align_w;
};

__device__ __forceinline__ void mma16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, const __nv_bfloat16*) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, const __half*) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// TT: tiles of eight tokens; UT: tiles of eight units that a warp takes with the same tokens in registers.
template <typename T, int TT, int UT> __global__ void __launch_bounds__(kFThreads) k_gated_few(FewArgs a) {
    constexpr int kWarps = kFThreads / 32, kAhead = TT * UT >= 4 ? 2 : 4;
    __shared__ float sums[kWarps][UT * TT * 4][32];
    after_earlier_kernels();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const long long unit0 = (long long)blockIdx.x * 8 * UT;
    const T *gate[UT], *up[UT], *x[TT];
    bool has[UT], token[TT];
#pragma unroll
    for (int i = 0; i < UT; ++i) {
        const long long unit = unit0 + 8 * i + g;
        has[i] = unit < a.hidden;
        gate[i] = static_cast<const T*>(a.gate) + (has[i] ? unit : 0) * a.gate_stride;
        up[i] = static_cast<const T*>(a.up) + (has[i] ? unit : 0) * a.up_stride;
    }
#pragma unroll
    for (int i = 0; i < TT; ++i) {
        token[i] = 8 * i + g < a.tokens;
        x[i] = static_cast<const T*>(a.x) + (token[i] ? 8 * i + g : 0) * a.x_stride;
    }
    float acc[UT][TT][4] = {};
    // (places are unsigned: the widest rows end less than a step of this loop below 2^31)
    const uint32_t inner = (uint32_t)a.inner;
    for (uint32_t k0 = warp * 32 + q * 8; k0 - q * 8 < inner; k0 += kWarps * 32 * kAhead) {
        Pack8<T> wg[kAhead][UT], wu[kAhead][UT], xs[kAhead][TT];
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
            const uint32_t k = k0 + s * kWarps * 32;
            const int have = (int)(inner - k);
#pragma unroll
            for (int i = 0; i < UT; ++i) {
                load8(wg[s][i], gate[i] + k, has[i] ? have : 0, a.align_w);
                load8(wu[s][i], up[i] + k, has[i] ? have : 0, a.align_w);
            }
#pragma unroll
            for (int i = 0; i < TT; ++i) load8(xs[s][i], x[i] + k, token[i] ? have : 0, a.align_x);
        }
#pragma unroll
        for (int s = 0; s < kAhead; ++s)
#pragma unroll
            for (int i = 0; i < UT; ++i)
#pragma unroll
                for (int j = 0; j < TT; ++j) {
                    mma16816(acc[i][j], wg[s][i].w[0], wu[s][i].w[0], wg[s][i].w[1], wu[s][i].w[1], xs[s][j].w[0], xs[s][j].w[1], (const T*)nullptr);
                    mma16816(acc[i][j], wg[s][i].w[2], wu[s][i].w[2], wg[s][i].w[3], wu[s][i].w[3], xs[s][j].w[2], xs[s][j].w[3], (const T*)nullptr);
                }
    }
#pragma unroll
    for (int i = 0; i < UT; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[warp][(i * TT + j) * 4 + e][lane] = acc[i][j][e];
    __syncthreads();
    // element e of a tile: e < 2: g, otherwise u, of unit `lane / 4` and token `lane % 4 * 2 + e % 2`
    for (int n = threadIdx.x; n < UT * TT * 2 * 32; n += kFThreads) {
        const int at = n & 31, e = n >> 5 & 1, tile = n >> 6, j = tile % TT, i = tile / TT;
        float gs = 0.f, us = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            gs += sums[w][tile * 4 + e][at];
            us += sums[w][tile * 4 + 2 + e][at];
        }
        const long long unit = unit0 + 8 * i + (at >> 2);
        const int tok = 8 * j + (at & 3) * 2 + e;
        float value, slope;
        by_act(a.act, [&](auto which) { activate<decltype(which)::n, false>(gs, value, slope); });
        if (unit < a.hidden && tok < a.tokens) static_cast<T*>(a.h)[tok * a.h_stride + unit] = from_float<T>(value * us);
    }
}

// ---- between the products -------------------------------------------------------------------

constexpr int kGThreads = 256;

struct GateGradArgs {
    const void* dh;
    const float2* kept;
    void *dg, *du;
    long long rows, dh_stride, kept_stride, d_stride;
    int cols, align_dh;
};

// dg = dh P, du = dh Q.  Bound by memory: 14 bytes a unit (2 + 8 read, 4 written); 8192 x 8192 157 us, 6.0 TB/s.
//
// Both are rounded to the inputs' type, which is what the tensor cores take: the one rounding on the way, beside the results' own, so that the
// gradients are off by 1.41 (the root of two) times what 32-bit factors would leave.  As two 16-bit terms each they would double the
// backward products (1430 of 2790 us for 8192 x 4096 -> 8192).  float16 has its range, too: above 65504 they are infinities, as dh itself would be.
template <typename T> __global__ void __launch_bounds__(kGThreads) k_gate_grad(GateGradArgs a) {
    after_earlier_kernels();
    const int groups = (a.cols + 7) / 8;
    const long long all = a.rows * groups;
    for (long long n = (long long)blockIdx.x * kGThreads + threadIdx.x; n < all; n += (long long)gridDim.x * kGThreads) {
        const long long r = n / groups;
        const int c = (int)(n - r * groups) * 8, have = min(8, a.cols - c);
        Pack8<T> dh, dg, du;
        load8(dh, static_cast<const T*>(a.dh) + r * a.dh_stride + c, have, a.align_dh);
        const float2* kept = a.kept + r * a.kept_stride + c;
        float2 k[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {   // (rows of an odd length have room for one more)
            const float4 v = e < have ? __ldg(reinterpret_cast<const float4*>(kept + e)) : make_float4(0.f, 0.f, 0.f, 0.f);
            k[e] = make_float2(v.x, v.y);
            k[e + 1] = make_float2(v.z, v.w);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = to_float(dh.e[e]);
            dg.e[e] = from_float<T>(d * k[e].x);
            du.e[e] = from_float<T>(d * k[e].y);
        }
        // rows here are whole eights apart, and nothing reads what lies behind the columns
        *reinterpret_cast<uint4*>(static_cast<T*>(a.dg) + r * a.d_stride + c) = dg.q[0];
        *reinterpret_cast<uint4*>(static_cast<T*>(a.du) + r * a.d_stride + c) = du.q[0];
    }
}

// Matrices whose rows do not begin at multiples of 16 bytes, which copies into shared memory must, to rows that do.
struct LayArgs {
    const void* from[3];
    void* to[3];
    long long rows[3], stride[3], to_stride[3];
    int cols[3], align[3];
};
template <typename T> __global__ void __launch_bounds__(kGThreads) k_lay_rows(LayArgs a) {
    after_earlier_kernels();
    const int which = blockIdx.y;
    const int cols = a.cols[which], groups = (cols + 7) / 8;
    const long long all = a.rows[which] * groups;
    for (long long n = (long long)blockIdx.x * kGThreads + threadIdx.x; n < all; n += (long long)gridDim.x * kGThreads) {
        const long long r = n / groups;
        const int c = (int)(n - r * groups) * 8;
        Pack8<T> v;
        load8(v, static_cast<const T*>(a.from[which]) + r * a.stride[which] + c, min(8, cols - c), a.align[which]);
        *reinterpret_cast<uint4*>(static_cast<T*>(a.to[which]) + r * a.to_stride[which] + c) = v.q[0];
    }
}

}  // namespace sbclm
