// out = A B^T for two matrices in 4-bit floating point, on the tensor cores' block-scaled form.
//
// out[i][j] = t_A t_B sum_b s_A[i][b] s_B[j][b] sum_{k in b} A[i][k] B[j][k]: codes A and B of 4 bits, a
// scale s for each block b of 32 or 16 columns, a scale t for a whole matrix; sums in 32 bits.
//
// The weights' rows are the accumulator's 128 lanes and the tokens its columns.  A stage holds 256
// elements (128 bytes, one swizzle line) of every row of both sides and their block scales, which are
// copied to tensor memory as the tiles they are stored in.  Up to 128 tokens there is one kernel, bound
// by the weights' way from memory; above, another, bound by the tensor cores.
#pragma once

#include "lm_common.cuh"

namespace sbclm {

constexpr int kPThreads = 192;      // four warps for the accumulator, one that loads, one that multiplies
constexpr int kPRows = 128;         // weights per tile
constexpr int kPBytes = 128;        // bytes of a row per stage: 256 elements
constexpr int kPMaxStages = 8;

struct ProductArgs {
    const uint8_t *scales_w, *scales_x;
    const float *tensor_w, *tensor_x;
    void* out;
    uint32_t* status;
    long long rows_w, rows_x, stride;
    long long ktiles;    // scale tiles per 128 rows
    int chunks;          // stages' worth of columns
    int steps;           // 64-element products over all columns
    int nt;              // tokens of the tile: all of them, in whole 16s
    int stages;
    uint32_t tmem_cols;  // allocated columns (a power of two)
};

template <int FMT> struct ProductShape {
    static constexpr int kTiles = FMT == SBC_FP4_E8M0 ? 2 : 4;  // scale tiles per stage and 128 rows
    static constexpr uint32_t kIdesc =                            // 4-bit operands, both K-major, 128 lanes
        (1u << 7) | (1u << 10) | (FMT == SBC_FP4_E8M0 ? 1u << 23 : 0u) | (1u << 27);
};

// The two tensor scales, applied to a sum: by their product, or, where that leaves 32 bits (2^-252 .. 2^234; the result
// may not), one after the other, the larger first.  Two small ones then round once, since a sum is 0 or at least
// 2^-20 (grid values 0.5, block scales 2^-9); two large ones leave 32 bits only if the result does.
template <int FMT> struct ResultScale {
    const float *w, *x;
    float by = 1.f;   // 0: the product leaves 32 bits
    __device__ __forceinline__ ResultScale(const float* tensor_w, const float* tensor_x) : w(tensor_w), x(tensor_x) {
        if (FMT == SBC_FP4_E4M3) {
            by = *w * *x;
            if (fabsf(by) < 0x1p-126f || fabsf(by) == __builtin_huge_valf()) by = 0.f;
        }
    }
    // Takes N sums of an accumulator, in place, to where one factor is left, which it returns.  The factors are asked for
    // anew in the branch that needs both (all warps take the same), so one register holds what is common (8192^3 with its
    // quantisation 361 us; with both factors in registers 365).
    template <int N> __device__ __forceinline__ float last(float* sums) const {
        if (FMT != SBC_FP4_E4M3 || by != 0.f) return by;
        const float a = *w, b = *x;
        const bool larger = fabsf(a) > fabsf(b);
        const float before = larger ? a : b;
#pragma unroll
        for (int i = 0; i < N; ++i) sums[i] = __fmul_rn(sums[i], before);
        return larger ? b : a;
    }
};

// A place in the ring of stages and the parity its barriers have there (no divisions: every role goes
// around it with one thread, whose own latency would otherwise be what a stage costs).
struct Ring {
    int s = 0;
    uint32_t turn = 0;
    __device__ __forceinline__ void next(int stages) {
        if (++s == stages) s = 0, turn ^= 1;
    }
};

__device__ __forceinline__ uint64_t operand_desc(uint32_t smem) {  // 128-byte swizzle, 8 rows of 128 bytes per group
    return (uint64_t)((smem & 0x3ffff) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem) {    // no swizzle, 8 rows of 16 bytes per group
    return (uint64_t)((smem & 0x3ffff) >> 4) | (1ull << 16) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
}

__device__ __forceinline__ void scales_to_tmem(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <int FMT>
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t add) {
    if (FMT == SBC_FP4_E8M0)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(add)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(add)
            : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load16(float* v, uint32_t addr) {
    uint32_t* u = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
          "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
        : "r"(addr)
        : "memory");
}

// Up to 128 tokens, a tile is 128 weights and all of them: grid (weight tiles, blocks per tile), a cluster
// along y.  There are few tiles, so a cluster shares one: each block takes a run of stages, and the
// partial accumulators are added in a fixed order through distributed shared memory.
//
// 16 x 8192 -> 8192 (E8M0, bfloat16 out): 9.9 us, 3.6 TB/s of values and scales, of which 5.5 us is
// what memory would need: the rest is the launch, the first loads' way and the sum over the cluster.
// 1 token 9.3 us, 128 tokens 13.6 us, 1024 x 1024 for 16 tokens 4.1 us.
template <typename T, int FMT>
__global__ void __launch_bounds__(kPThreads) k_fp4_product(const __grid_constant__ CUtensorMap map_w,
                                                           const __grid_constant__ CUtensorMap map_x, ProductArgs a) {
    using S = ProductShape<FMT>;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * kPMaxStages + 1];
    __shared__ uint32_t tmem_slot, gave_up;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t bytes_w = kPRows * kPBytes, bytes_x = (uint32_t)a.nt * kPBytes;
    const uint32_t bytes_x_room = (bytes_x + 1023u) & ~1023u;
    const uint32_t bytes_sc = S::kTiles * 512u;                    // one side's scales
    const uint32_t stage_bytes = bytes_w + bytes_x_room + bytes_sc * 2;
    const uint32_t stage_room = (stage_bytes + 1023u) & ~1023u;
    const uint32_t bar0 = smem_u32(bars), done = bar0 + 16 * kPMaxStages;
    const int rank = (int)blockIdx.y, parts = (int)gridDim.y;
    const int first = (int)((long long)a.chunks * rank / parts), last = (int)((long long)a.chunks * (rank + 1) / parts);
    const long long w0 = (long long)blockIdx.x * kPRows;

    if (t == 0) {
        gave_up = 0;
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(bar0 + 16 * s, 1);
            mbar_init(bar0 + 16 * s + 8, 1);
        }
        mbar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(a.tmem_cols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_slot;
    after_earlier_kernels();
    const uint32_t acc_cols = (uint32_t)(a.nt + 31) & ~31u;
    const uint32_t sc_cols = 8u * S::kTiles;                       // scale columns per stage

    if (warp == 4 && lane == 0) {
        bool ok = true;
        Ring at;
        const uint8_t* sw = a.scales_w + (w0 / 128 * a.ktiles + (long long)first * S::kTiles) * 512;
        const uint8_t* sx = a.scales_x + (long long)first * S::kTiles * 512;
        int left = (int)(a.ktiles - (long long)first * S::kTiles);
        int c = first;
        for (; c < last; ++c) {
            const uint32_t full = bar0 + 16 * at.s;
            ok = mbar_wait(full + 8, at.turn ^ 1);
            if (!ok) break;
            const uint32_t sc = (uint32_t)min(S::kTiles, left) * 512u;
            const uint32_t to = smem + (uint32_t)at.s * stage_room, to_x = to + bytes_w, to_sc = to_x + bytes_x_room;
            mbar_expect(full, bytes_w + bytes_x + sc * 2);
            tma_load_2d(to, &map_w, c * kPBytes, (int)w0, full);
            tma_load_2d(to_x, &map_x, c * kPBytes, 0, full);
            bulk_load(to_sc, sw, sc, full);
            bulk_load(to_sc + bytes_sc, sx, sc, full);
            sw += S::kTiles * 512, sx += S::kTiles * 512, left -= S::kTiles;
            at.next(a.stages);
        }
        if (!ok) gave_up = 1;
        // no copy may be in flight when the block ends
        for (int j = max(0, c - first - a.stages); j < c - first; ++j) mbar_wait(bar0 + 16 * (j % a.stages), (j / a.stages) & 1);
    } else if (warp == 5 && lane == 0) {
        bool ok = true;
        const uint32_t idesc = S::kIdesc | ((uint32_t)(a.nt >> 3) << 17);
        Ring ring;
        for (int c = first; c < last; ++c) {
            const uint32_t full = bar0 + 16 * ring.s, empty = full + 8;
            ok = mbar_wait(full, ring.turn);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t at = smem + (uint32_t)ring.s * stage_room, at_x = at + bytes_w, at_sc = at_x + bytes_x_room;
            const uint32_t sf_w = tmem + acc_cols + (uint32_t)ring.s * sc_cols, sf_x = sf_w + 4 * S::kTiles;
            const int steps = min(4, a.steps - c * 4);
#pragma unroll
            for (int k = 0; k < S::kTiles; ++k) {
                if (k * (4 / S::kTiles) >= steps) break;
                scales_to_tmem(sf_w + 4 * k, scale_desc(at_sc + 512 * k));
                scales_to_tmem(sf_x + 4 * k, scale_desc(at_sc + bytes_sc + 512 * k));
            }
            for (int k = 0; k < steps; ++k) {
                // E8M0: two steps share a scale tile, each takes its half of every word
                const int tile = FMT == SBC_FP4_E8M0 ? k / 2 : k;
                const uint32_t half = FMT == SBC_FP4_E8M0 ? (uint32_t)(k & 1) * 2u : 0u;
                multiply<FMT>(tmem, operand_desc(at + 32 * k), operand_desc(at_x + 32 * k), idesc | (half << 4) | (half << 29),
                              sf_w + 4 * tile, sf_x + 4 * tile, (uint32_t)(c > first || k > 0));
            }
            commit(empty);
            ring.next(a.stages);
        }
        commit(done);
        if (!ok) gave_up = 1;
        mbar_wait(done, 0);   // no product may be running when tensor memory is given back
    }
    __syncwarp();
    // every block of a cluster has at least one chunk, so `done` always means a whole partial sum
    const bool finished = mbar_wait(done, 0);
    if (!finished) gave_up = 1;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    __syncthreads();
    const bool bad = gave_up != 0;
    if (bad && t == 0 && a.status) atomicOr(a.status, SBC_STATUS_TIMEOUT);
    const float nan = __uint_as_float(0x7fffffffu);
    T* out = static_cast<T*>(a.out);
    const ResultScale<FMT> scale(a.tensor_w, a.tensor_x);
    const int tokens = (int)a.rows_x;
    const long long j = w0 + warp * 32 + lane;
    if (parts == 1) {
        if (warp < 4) {
            T* to = out + j;
            const int most = j < a.rows_w ? tokens : 0;
            for (int n0 = 0; n0 < tokens; n0 += 16) {
                float v[16];
                __syncwarp();
                tmem_load16(v, tmem + ((uint32_t)warp << 21) + n0);
                const float by = scale.template last<16>(v);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (n0 + i < most) *to = from_float<T>(bad ? nan : v[i] * by);
                    to += a.stride;
                }
            }
        }
    } else {
        // partial sums, one row of 128 lanes per token, over the stages that nothing uses any more
        if (warp < 4) {
            uint32_t to = smem + (uint32_t)(warp * 32 + lane) * 4u;
            for (int n0 = 0; n0 < tokens; n0 += 16) {
                float v[16];
                __syncwarp();
                tmem_load16(v, tmem + ((uint32_t)warp << 21) + n0);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (n0 + i < tokens) asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + (uint32_t)(n0 + i) * 512u), "f"(bad ? nan : v[i]) : "memory");
            }
        }
        cluster_sync();
        // four weights of a token a thread; the blocks' sums are loaded together and added in their order
        const bool wide = (((uintptr_t)a.out | (uintptr_t)(a.stride * (long long)sizeof(T))) & (4 * sizeof(T) - 1)) == 0;
        for (int i = rank * kPThreads + t; i < tokens * 32; i += parts * kPThreads) {
            float4 v[8];
#pragma unroll
            for (int p = 0; p < 8; ++p)
                if (p < parts) v[p] = ld_cluster4(map_rank(smem + (uint32_t)i * 16u, (uint32_t)p));
            float4 sum = v[0];
#pragma unroll
            for (int p = 1; p < 8; ++p)
                if (p < parts) sum.x += v[p].x, sum.y += v[p].y, sum.z += v[p].z, sum.w += v[p].w;
            const long long w = w0 + i % 32 * 4;
            T* to = out + i / 32 * a.stride + w;
            float sums[4] = {sum.x, sum.y, sum.z, sum.w};
            const float by = scale.template last<4>(sums);
            alignas(16) const T four[4] = {from_float<T>(sums[0] * by), from_float<T>(sums[1] * by), from_float<T>(sums[2] * by),
                                           from_float<T>(sums[3] * by)};
            if (wide && w + 4 <= a.rows_w) {
                if constexpr (sizeof(T) == 2)
                    *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(four);
                else
                    *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(four);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (w + k < a.rows_w) to[k] = four[k];
            }
        }
        cluster_sync();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 5) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(a.tmem_cols));
}

// ---- many tokens ----------------------------------------------------------------------
//
// Pairs of blocks on neighbouring SMs share a tile of 256 weights x NT (256 or 128) tokens: each
// loads its 128 weights and half of the tokens, the tensor cores of both read both halves, so an SM
// loads 0.58 bytes per thousand products where a block alone would load 0.82.  Blocks stay and take
// tile after tile; loads run ahead across tiles.
//
// What a stage costs is its way around the ring (products done, load, products) over the number of
// stages, so nothing else is on that way: both blocks' loads count at the first block's barrier, and
// the scales come through a deeper ring of their own.  They reach tensor memory through registers (four
// warps that do nothing else): copies by the tensor unit (tcgen05.cp) take turns with the products
// there, about 100 cycles each against 128 of a product.
//
// 8192^3: E8M0 223 us, 4.9 PFLOP/s; E4M3 235 us, 4.7 PFLOP/s: stages wait for their loads.  The tensor pipe is busy half
// of the time and L2 at 36 % of its peak, so neither bounds it; whether the way into the SMs or the ring of stages does
// was not measured.  Tiles below half of the pairs leave the rest idle, the columns are not split here (16384 -> 4096:
// 129 to 512 tokens 32 to 33 us).  4096^3 40 us, 3.4 PFLOP/s (256 tiles for 74 pairs: four rounds, the last half full);
// 2240 x 1300 -> 2600 14 us, ramp and drain.
//
// Warps: 0..3 and 12..15 accumulator to memory (half of the columns each), 4..7 scales, 8 loads, 9
// multiplies (in the first block of the pair), 10 loads scales.

constexpr int kWThreads = 512;
constexpr int kWMaxStages = 8;
constexpr int kWScales = 8;   // stages of the scales' ring

struct WideArgs {
    const uint8_t *scales_w, *scales_x;
    const float *tensor_w, *tensor_x;
    void* out;
    uint32_t* status;
    long long rows_w, rows_x, stride, ktiles;
    int chunks, steps, stages;
    int tiles_w, tiles;   // tiles along the weights, all tiles
};

template <int FMT>
__device__ __forceinline__ void multiply2(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t add) {
    if (FMT == SBC_FP4_E8M0)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(add)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(add)
            : "memory");
}
// Arrives at the barrier of this address in both blocks when all products so far are done.
__device__ __forceinline__ void commit2(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)3)
                 : "memory");
}
__device__ __forceinline__ void tmem_load32(float* v, uint32_t addr) {
    uint32_t* u = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
          "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]),
          "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]),
          "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_store4(uint32_t addr, const uint4& q) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
    uint4 q;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(addr) : "memory");
    return q;
}

__device__ __forceinline__ uint32_t pack2(float a, float b, const __nv_bfloat16*) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, const __half*) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ void store_half(void* p, uint32_t v) {
    asm volatile("{\n\t.reg .b16 h, r;\n\tmov.b32 {h, r}, %1;\n\tst.global.b16 [%0], h;\n\t}" ::"l"(p), "r"(v) : "memory");
}

__device__ __forceinline__ void store_word(void* p, uint32_t v) { asm volatile("st.global.b32 [%0], %1;" ::"l"(p), "r"(v) : "memory"); }

// COLS columns of an accumulator, this warp's 32 lanes, to `out` (this lane's weight of the first
// token); `free` is called when they have left tensor memory: results wait in registers (16-bit ones
// two to a word), so that the next tile's products can begin before the stores have.  Stores follow
// one another (volatile: their addresses would otherwise all be formed in front).
// PAIRS: 16-bit results whose even places are 4-byte aligned.  Neighbouring lanes swap halves, so that
// one has two weights of a token and the other the same two of the next.
template <typename T, int FMT, int COLS, bool PAIRS, typename F>
__device__ __forceinline__ void store_tile(uint32_t acc, T* out, long long stride, int tokens, bool mine, const ResultScale<FMT>& scale, F free) {
    if constexpr (sizeof(T) == 2) {
        uint32_t w[COLS / 2];
#pragma unroll
        for (int n0 = 0; n0 < COLS; n0 += 32) {
            float v[32];
            tmem_load32(v, acc + n0);
            const float by = scale.template last<32>(v);
#pragma unroll
            for (int i = 0; i < 32; i += 2) w[(n0 + i) / 2] = pack2(v[i] * by, v[i + 1] * by, (const T*)nullptr);
        }
        free();
        if (PAIRS) {
            const bool odd = threadIdx.x & 1;
            T* to = odd ? out - 1 + stride : out;
            const int most = mine ? tokens - (odd ? 1 : 0) : 0;
#pragma unroll
            for (int n = 0; n < COLS; n += 2) {
                const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? w[n / 2] : w[n / 2] >> 16, 1);
                if (n < most) store_word(to, odd ? __byte_perm(other, w[n / 2], 0x7610) : __byte_perm(w[n / 2], other, 0x5410));
                to += 2 * stride;
            }
        } else {
            const int most = mine ? tokens : 0;
#pragma unroll
            for (int n = 0; n < COLS; ++n) {
                if (n < most) store_half(out, n & 1 ? w[n / 2] >> 16 : w[n / 2]);
                out += stride;
            }
        }
    } else {
        float v[COLS];
#pragma unroll
        for (int n0 = 0; n0 < COLS; n0 += 32) tmem_load32(v + n0, acc + n0);
        free();
        const float by = scale.template last<COLS>(v);
        const int most = mine ? tokens : 0;
#pragma unroll
        for (int n = 0; n < COLS; ++n) {
            if (n < most) store_word(out, __float_as_uint(v[n] * by));
            out += stride;
        }
    }
}

template <typename T, int FMT, int NT>
__global__ void __launch_bounds__(kWThreads, 1)
    k_fp4_product_wide(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, WideArgs a) {
    using S = ProductShape<FMT>;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[3 * kWMaxStages + 2 * kWScales + 5];
    __shared__ uint32_t tmem_slot, gave_up;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t smem = (smem_u32(raw) + 1023u) & ~1023u;
    constexpr int row_tiles = NT / 128, buffers = NT == 128 ? 2 : 1;
    constexpr uint32_t bytes_w = kPRows * kPBytes, bytes_x = NT / 2 * kPBytes, bytes_sc = S::kTiles * 512u;
    constexpr uint32_t stage_bytes = bytes_w + bytes_x, scale_bytes = bytes_sc * (1 + row_tiles);
    const uint32_t scales0 = smem + (uint32_t)a.stages * stage_bytes;
    const uint32_t bar0 = smem_u32(bars);
    const auto full = [&](int s) { return bar0 + 24u * s; };           // (first block) both blocks' loads of a stage have landed
    const auto ready = [&](int s) { return bar0 + 24u * s + 8; };      // (first block) both blocks' scales of it are in tensor memory
    const auto empty = [&](int s) { return bar0 + 24u * s + 16; };     // the products that read a stage are done
    const auto sc_full = [&](int s) { return bar0 + 24u * kWMaxStages + 16u * s; };       // this block's scales have landed
    const auto sc_empty = [&](int s) { return bar0 + 24u * kWMaxStages + 16u * s + 8; };  // ... are in registers
    const uint32_t bar1 = bar0 + 24u * kWMaxStages + 16u * kWScales;
    const auto acc_full = [&](int b) { return bar1 + 8u * b; };
    const auto acc_empty = [&](int b) { return bar1 + 16 + 8u * b; };  // (first block)
    const uint32_t drained = bar1 + 32;
    constexpr uint32_t acc_cols = 256, sc_cols = 4u * S::kTiles * (1 + row_tiles);
    const int pairs = (int)(gridDim.x / 2), pair = (int)(blockIdx.x / 2);

    if (t == 0) {
        gave_up = 0;
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(ready(s), 8);
            mbar_init(empty(s), 1);
        }
        for (int s = 0; s < kWScales; ++s) {
            mbar_init(sc_full(s), 1);
            mbar_init(sc_empty(s), 4);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), 16);
        }
        mbar_init(drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
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
                const int w0 = tile % a.tiles_w * 256 + (int)rank * 128;
                const int x1 = tile / a.tiles_w * NT + (int)rank * (NT / 2);
                for (int c = 0; c < a.chunks; ++c) {
                    ok = mbar_wait(empty(ring.s), ring.turn ^ 1);
                    if (!ok) break;
                    const uint32_t at = smem + (uint32_t)ring.s * stage_bytes, bar = map_rank(full(ring.s), 0);
                    // the second block's bytes may arrive before they are announced: the turn ends with the announcement
                    if (rank == 0) mbar_expect(full(ring.s), 2 * stage_bytes);
                    tma_load_2d_pair(at, &map_w, c * kPBytes, w0, bar);
                    tma_load_2d_pair(at + bytes_w, &map_x, c * kPBytes, x1, bar);
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
    } else if (warp == 10) {
        if (lane == 0) {
            bool ok = true;
            Ring ring;
            int issued = 0;
            for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
                const int w0 = tile % a.tiles_w * 256 + (int)rank * 128, x0 = tile / a.tiles_w * NT;
                const bool has_w = w0 < a.rows_w;
                const int x_tiles = (int)min((long long)row_tiles, (a.rows_x + 127) / 128 - x0 / 128);
                const uint8_t* sw = a.scales_w + w0 / 128 * a.ktiles * 512;
                const uint8_t* sx = a.scales_x + x0 / 128 * a.ktiles * 512;
                const uint8_t* sx2 = sx + a.ktiles * 512;
                int left = (int)a.ktiles;
                for (int c = 0; c < a.chunks; ++c) {
                    const uint32_t bar = sc_full(ring.s);
                    ok = mbar_wait(bar + 8, ring.turn ^ 1);
                    if (!ok) break;
                    const uint32_t sc = (uint32_t)min(S::kTiles, left) * 512u, at = scales0 + (uint32_t)ring.s * scale_bytes;
                    mbar_expect(bar, sc * ((has_w ? 1 : 0) + x_tiles));
                    if (has_w) bulk_load(at, sw, sc, bar);
                    bulk_load(at + bytes_sc, sx, sc, bar);
                    if (x_tiles > 1) bulk_load(at + 2 * bytes_sc, sx2, sc, bar);
                    sw += S::kTiles * 512, sx += S::kTiles * 512, sx2 += S::kTiles * 512, left -= S::kTiles;
                    ring.next(kWScales);
                    issued = min(issued + 1, kWScales);
                }
            }
            if (!ok) gave_up = 1;
            for (int j = 0; j < issued; ++j) {
                const int s = ring.s - 1 - j < 0 ? ring.s - 1 - j + kWScales : ring.s - 1 - j;
                mbar_wait(sc_full(s), ring.s - 1 - j < 0 ? ring.turn ^ 1 : ring.turn);
            }
        }
    } else if (warp == 9) {
        if (lane == 0 && rank != 0) mbar_wait(drained, 0);
        if (lane == 0 && rank == 0) {
            bool ok = true;
            const uint32_t idesc = (1u << 7) | (1u << 10) | (FMT == SBC_FP4_E8M0 ? 1u << 23 : 0u) | (2u << 27) | ((uint32_t)(NT >> 3) << 17);
            Ring ring, accs;
            for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
                const int b = accs.s;
                ok = mbar_wait(acc_empty(b), accs.turn ^ 1);
                if (!ok) break;
                const uint32_t acc = tmem + (uint32_t)b * 128u;
                for (int c = 0; c < a.chunks; ++c) {
                    ok = mbar_wait(ready(ring.s), ring.turn) && mbar_wait(full(ring.s), ring.turn);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = smem + (uint32_t)ring.s * stage_bytes, at_x = at + bytes_w;
                    const uint32_t sf_w = tmem + acc_cols + (uint32_t)ring.s * sc_cols, sf_x = sf_w + 4 * S::kTiles;
                    const int steps = min(4, a.steps - c * 4);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k >= steps) break;
                        // E8M0: two steps share a scale tile, each takes its half of every word
                        const int tile_k = FMT == SBC_FP4_E8M0 ? k / 2 : k;
                        const uint32_t half = FMT == SBC_FP4_E8M0 ? (uint32_t)(k & 1) * 2u : 0u;
                        multiply2<FMT>(acc, operand_desc(at + 32 * k), operand_desc(at_x + 32 * k), idesc | (half << 4) | (half << 29),
                                       sf_w + 4 * tile_k, sf_x + 4 * tile_k * row_tiles, (uint32_t)(c > 0 || k > 0));
                    }
                    commit2(empty(ring.s));
                    ring.next(a.stages);
                }
                if (ok) commit2(acc_full(b));
                accs.next(buffers);
            }
            if (!ok) gave_up = 1;
            // no product may be running when tensor memory is given back
            commit2(drained);
            mbar_wait(drained, 0);
        }
    } else if (warp >= 4 && warp < 8) {
        bool ok = true;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        Ring ring, from;
        for (int tile = pair; tile < a.tiles && ok; tile += pairs) {
            for (int c = 0; c < a.chunks; ++c) {
                ok = __all_sync(0xffffffffu, mbar_wait(sc_full(from.s), from.turn));
                if (!ok) break;
                const uint32_t at = scales0 + (uint32_t)from.s * scale_bytes + 16u * lane;
                const uint32_t sf = tmem + acc_cols + (uint32_t)ring.s * sc_cols + lanes;
                uint4 q[S::kTiles * (1 + row_tiles)];
#pragma unroll
                for (int k = 0; k < S::kTiles; ++k) {
                    q[k] = ld_shared16(at + 512u * k);
#pragma unroll
                    for (int j = 0; j < row_tiles; ++j) q[S::kTiles + k * row_tiles + j] = ld_shared16(at + bytes_sc * (1 + j) + 512u * k);
                }
                // the stage's columns of tensor memory are free when its last products are done
                ok = __all_sync(0xffffffffu, mbar_wait(empty(ring.s), ring.turn ^ 1));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int k = 0; k < S::kTiles * (1 + row_tiles); ++k) tmem_store4(sf + 4u * k, q[k]);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_remote(map_rank(ready(ring.s), 0));
                    mbar_arrive_remote(map_rank(sc_empty(from.s), rank));
                }
                ring.next(a.stages);
                from.next(kWScales);
            }
        }
        if (!ok) gave_up = 1;
    } else if (warp < 4 || warp >= 12) {
        bool ok = true;
        ResultScale<FMT> scale(a.tensor_w, a.tensor_x);
        constexpr int kCols = NT / 2;
        const int col0 = warp < 4 ? 0 : kCols, sub = warp & 3;
        const bool pairs_ok = sizeof(T) == 2 && ((a.stride | a.rows_w) & 1) == 0 && ((uintptr_t)a.out & 3) == 0;
        Ring accs;
        for (int tile = pair; tile < a.tiles; tile += pairs, accs.next(buffers)) {
            const int b = accs.s;
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(acc_full(b), accs.turn));
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const long long j = (long long)(tile % a.tiles_w) * 256 + rank * 128 + sub * 32 + lane, x0 = (long long)(tile / a.tiles_w) * NT + col0;
            const uint32_t acc = tmem + (uint32_t)b * 128u + (uint32_t)col0 + ((uint32_t)sub << 21);
            T* out = static_cast<T*>(a.out) + x0 * a.stride + j;
            const int tokens = (int)min((long long)kCols, a.rows_x - x0);
            if (!ok) scale.by = __uint_as_float(0x7fffffffu);
            const auto free = [&] {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(map_rank(acc_empty(b), 0));
            };
            if (pairs_ok)
                store_tile<T, FMT, kCols, true>(acc, out, a.stride, tokens, j < a.rows_w, scale, free);
            else
                store_tile<T, FMT, kCols, false>(acc, out, a.stride, tokens, j < a.rows_w, scale, free);
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
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

}  // namespace sbclm
