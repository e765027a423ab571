// 4-bit floating point: quantisation along rows and columns, and expansion.
//
// Arithmetic.  With s the block's scale (block scale * tensor scale, an exact product of a float of
// at most 4 significant bits and a power of two) an element becomes the grid point nearest to
// x / s.  For E8M0 the quotient is exact.  For E4M3 the quotient is the correctly rounded one, and
// that decides like the exact one: a grid midpoint m has at most 3 significant bits, m * s is a
// float, so an x that is not m * s differs from it by at least one unit in the last place, and the
// rounded quotient then is not m either.  The same holds for the block scale, amax / (6 * 2^g).
// The quotient comes from an approximate reciprocal r: q = x r, then one correction by the residual
// x - q s, which a fused operation gives exactly (Markstein 1990).  What that can be off by is far below
// the 7 % of half a unit by which x / s stays clear of rounding to a midpoint it is not.  The power of
// two is taken off first, so s is in [2^-9, 448] and nothing over- or underflows that could matter.
#pragma once

#include "lm_common.cuh"

namespace sbclm {

constexpr int kQTile = 128;        // rows and columns of a block's tile: what a 512-byte scale tile spans
constexpr int kQThreads = 256;

template <int FMT> struct Fp4 {
    static constexpr int kBlock = FMT == SBC_FP4_E8M0 ? 32 : 16;
    static constexpr uint32_t kNanScale = FMT == SBC_FP4_E8M0 ? 0xffu : 0x7fu;
};

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // e in [-126, 127]

// 2^g from the bits of the largest finite magnitude.
__device__ __forceinline__ float tensor_scale_of(uint32_t amax_bits) {
    if (amax_bits == 0) return 1.f;
    const int e = (int)(amax_bits >> 23);  // biased; 0 (subnormal) clamps like everything small
    return pow2(max(e - 127 - 10, -126));
}

// x / d, corrected (see above), for r near 1 / d.
__device__ __forceinline__ float quotient(float x, float d, float r) {
    const float q = __fmul_rn(x, r);
    return fmaf(fmaf(-q, d, x), r, q);
}

// A block's scale, ready for its elements.
template <int FMT> struct BlockScale {
    uint32_t code;
    float by, inv;   // E8M0: by = 1 / scale.  E4M3: by = the code's value, inv near its reciprocal.  0: the block is zeros
    __device__ __forceinline__ BlockScale(uint32_t amax_bits, float inv_tensor) : inv(0.f) {
        if (FMT == SBC_FP4_E8M0) {
            code = (uint32_t)max((int)(amax_bits >> 23) - 2, 0);
            by = __uint_as_float((254u - code) << 23);
        } else {
            const float want = quotient(__uint_as_float(amax_bits) * inv_tensor, 6.f, 1.f / 6.f);
            code = __nv_cvt_float_to_fp8(want, __NV_SATFINITE, __NV_E4M3);
            by = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(by));
        }
        if (amax_bits >= 0x7f800000u) {
            code = Fp4<FMT>::kNanScale;
            by = 0.f;
        }
    }
    __device__ __forceinline__ bool zero() const { return by == 0.f; }
    // N quotients, in place (E4M3: of values divided by the tensor's scale on the way)
    template <int N> __device__ __forceinline__ void over(float* y, float inv_tensor) const {
        const unsigned long long b = pair(by, by), minus = pair(-by, -by), r = pair(inv, inv), t = pair(inv_tensor, inv_tensor);
#pragma unroll
        for (int j = 0; j < N; j += 2) {
            unsigned long long x = pair(y[j], y[j + 1]);
            if (FMT == SBC_FP4_E8M0) {
                x = mul2(x, b);
            } else {
                x = mul2(x, t);
                const unsigned long long q = mul2(x, r);
                x = fma2(fma2(q, minus, x), r, q);
            }
            unpair(y[j], y[j + 1], x);
        }
    }
};

// Eight values to eight nibbles, the first one lowest.
__device__ __forceinline__ uint32_t pack_nibbles(const float* y) {
    uint32_t w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w)
        : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
    return w;
}

// Eight values, and the bits of the largest magnitude among them (as a float's; whole numbers, so a NaN
// is above an infinity is above all else).
__device__ __forceinline__ uint32_t unpack_max(float* y, const Pack8<float>& v) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        y[j] = v.e[j];
        top = max(top, __float_as_uint(y[j]) & 0x7fffffffu);
    }
    return top;
}
__device__ __forceinline__ uint32_t max_halves(const uint32_t* w, int n) {
    uint32_t top = w[0] & 0x7fff7fffu;
#pragma unroll
    for (int j = 1; j < n; ++j) top = __vmaxu2(top, w[j] & 0x7fff7fffu);
    return top;
}
__device__ __forceinline__ uint32_t float_bits_of(uint32_t half_bits, const __nv_bfloat16*) { return half_bits << 16; }
__device__ __forceinline__ uint32_t float_bits_of(uint32_t half_bits, const __half*) {
    return __float_as_uint(__half2float(__ushort_as_half((unsigned short)half_bits)));
}
template <typename T> __device__ __forceinline__ uint32_t unpack_max(float* y, const Pack8<T>& v) {
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = to_float(v.e[j]);
    const uint32_t top = max_halves(v.w, 4);
    return float_bits_of(max(top & 0xffffu, top >> 16), (const T*)nullptr);
}

struct QuantiseArgs {
    const void* x;
    long long rows, cols, stride;
    int align, base_align;        // every row, and the first one, starts at a multiple of this many bytes
    uint32_t col_tiles;           // blocks are numbered row tile by row tile
    const uint32_t* amax;         // E4M3: bits of the largest finite magnitudes that the blocks of k_fp4_amax found
    int amax_blocks;              // ... how many; 0: the tensor is small, every block looks for itself
    float* tensor_r;              // where the tensor scale goes (either may be null)
    float* tensor_c;
    uint8_t *values_r, *scales_r; // along the rows: rows x cols
    uint8_t *values_c, *scales_c; // along the columns: cols x rows
    long long pitch_r, pitch_c;   // bytes between rows of values
    long long ktiles_r, ktiles_c; // scale tiles per 128 rows
};

constexpr int kAmaxBlocks = 1024;
// Turns of a block's warps (a piece of a row each; rows without gaps are one long row) up to which every block finds
// the maximum itself, instead of a launch in front.  us without / with the launch, float32: rows without gaps 1 x 650
// 4.4 / 5.7, 16 x 2048 (two turns) 5.4 / 5.2, 64 x 4096 18.8 / 5.2; with gaps 16 x 64 (two turns) 5.2, 17 x 64 6.2 / 5.3,
// 64 x 64 12.3 / 5.5, 40 x 650 9.1 / 5.3, 32768 x 1 6118 / 25.
constexpr long long kAmaxAlone = 2;

// A warp's share of a matrix: rows in pieces of 2048 elements, eight steps of 256.  f(row, column, left):
// where a lane's first eight elements of a piece are, and how many elements the row has from there on.
constexpr int kPiece = 2048, kSteps = kPiece / 256;
template <typename F> __device__ __forceinline__ void warp_pieces(long long rows, long long cols, uint32_t warp, uint32_t warps, F f) {
    const uint32_t per_row = (uint32_t)((cols + kPiece - 1) / kPiece);
    const long long all = rows * per_row;
    for (long long i = warp; i < all; i += warps) {
        const long long r = all < (1ll << 32) ? (long long)((uint32_t)i / per_row) : i / per_row;
        const long long c = (i - r * per_row) * kPiece + (threadIdx.x & 31) * 8;
        f(r, c, (int)min(cols - c, (long long)kPiece));
    }
}

// Largest finite magnitude of the warps' shares, over the block, as float bits (whole numbers: the
// maximum does not depend on the order).
template <typename T> __device__ __forceinline__ uint32_t amax_over(const QuantiseArgs& a, uint32_t warp, uint32_t warps, uint32_t* room) {
    const T* x = static_cast<const T*>(a.x);
    // rows without gaps are one long row
    const bool flat = a.stride == a.cols;
    const long long rows = flat ? 1 : a.rows, cols = flat ? a.rows * a.cols : a.cols;
    uint32_t top = 0;
    const auto look = [&](const Pack8<T>& v) {
        float y[8];
        const uint32_t m = unpack_max(y, v);
        if (m < 0x7f800000u) {
            top = max(top, m);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t b = __float_as_uint(y[j]) & 0x7fffffffu;
                top = max(top, b < 0x7f800000u ? b : 0u);
            }
        }
    };
    const int align = flat ? a.base_align : a.align;
    warp_pieces(rows, cols, warp, warps, [&](long long r, long long c, int left) {
        const T* p = x + r * a.stride + c;
        constexpr int kAhead = 16 / (int)sizeof(T);   // 32 registers of loads under way
#pragma unroll
        for (int k = 0; k < kSteps; k += kAhead) {
            Pack8<T> v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) load8(v[i], p + 256 * (k + i), min(8, left - 256 * (k + i)), align);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) look(v[i]);
        }
    });
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = top;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, room[threadIdx.x & (kQThreads / 32 - 1)]);
}

// A block's share of the largest finite magnitude; the quantising kernel's blocks join the shares.  Bound by
// memory: 8192 x 8192 bfloat16 in 25 us, 5.3 TB/s (1024 blocks; 592, four per SM, 1 to 2 us slower).
template <typename T> __global__ void __launch_bounds__(kQThreads) k_fp4_amax(QuantiseArgs a, uint32_t* amax) {
    __shared__ uint32_t room[kQThreads / 32];
    after_earlier_kernels();
    const uint32_t top = amax_over<T>(a, blockIdx.x * (kQThreads / 32) + threadIdx.x / 32, gridDim.x * (kQThreads / 32), room);
    if (threadIdx.x == 0) amax[blockIdx.x] = top;
}

// The tensor's, in every block of the quantising kernel.
template <typename T> __device__ __forceinline__ uint32_t tensor_amax(const QuantiseArgs& a) {
    __shared__ uint32_t room[kQThreads / 32];
    if (a.amax_blocks == 0) return amax_over<T>(a, threadIdx.x / 32, kQThreads / 32, room);
    uint32_t top = 0;
    for (int i = threadIdx.x; i < a.amax_blocks; i += kQThreads) top = max(top, a.amax[i]);
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = top;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, room[threadIdx.x & (kQThreads / 32 - 1)]);
}

// N (16 or 32, a block's elements) values down a column to nibbles and the block's scale code.
template <int FMT, int N> __device__ __forceinline__ uint32_t quantise_run(uint32_t* nibbles, float* y, uint32_t top, float inv_tensor) {
    const BlockScale<FMT> scale(top, inv_tensor);
    scale.template over<N>(y, inv_tensor);
#pragma unroll
    for (int j = 0; j < N / 8; ++j) nibbles[j] = scale.zero() ? 0u : pack_nibbles(y + 8 * j);
    return scale.code;
}

// 32 rows of a column (16 bytes of nibbles, one or two scales) to the transpose.
template <int FMT>
__device__ __forceinline__ void store_column(const QuantiseArgs& a, long long out_row, long long row, const uint32_t* n, uint32_t codes) {
    if (out_row < a.cols && row / 2 < a.pitch_c) *reinterpret_cast<uint4*>(a.values_c + out_row * a.pitch_c + row / 2) = make_uint4(n[0], n[1], n[2], n[3]);
    const long long block = row / Fp4<FMT>::kBlock, k = block / 4;   // block % 4 is even for two scales
    if (k < a.ktiles_c) {
        uint8_t* p = a.scales_c + (out_row / 128 * a.ktiles_c + k) * 512 + (out_row % 32) * 16 + (out_row % 128 / 32) * 4 + block % 4;
        if (FMT == SBC_FP4_E8M0)
            *p = (uint8_t)codes;
        else
            *reinterpret_cast<uint16_t*>(p) = (uint16_t)codes;
    }
}

// The columns of a pass (128 rows of 16-bit elements, two columns and 32 rows a thread; 64 rows of floats,
// one column and 32 rows a thread) to the transpose.
template <typename T, int FMT>
__device__ __forceinline__ void quantise_columns(const QuantiseArgs& a, const T* tile, int stride, uint32_t row_tile, uint32_t col_tile, int pass,
                                                 float inv_tensor) {
    constexpr int kB = Fp4<FMT>::kBlock;
    const int t = threadIdx.x;
    if constexpr (sizeof(T) == 2) {
        const int c = t % 64 * 2, r0 = t / 64 * 32;
        uint32_t w[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) w[j] = *reinterpret_cast<const uint32_t*>(tile + (r0 + j) * stride + c);
        const long long row = (long long)row_tile * kQTile + pass + r0, out_row = (long long)col_tile * kQTile + c;
        uint32_t top[32 / kB];
#pragma unroll
        for (int b = 0; b < 32 / kB; ++b) top[b] = max_halves(w + b * kB, kB);
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            uint32_t n[4], codes = 0;
#pragma unroll
            for (int b = 0; b < 32 / kB; ++b) {
                float y[kB];
#pragma unroll
                for (int j = 0; j < kB; ++j) y[j] = to_float(reinterpret_cast<const T*>(&w[b * kB + j])[side]);
                codes |= quantise_run<FMT, kB>(n + b * (kB / 8), y, float_bits_of(side ? top[b] >> 16 : top[b] & 0xffffu, (const T*)nullptr), inv_tensor)
                         << (8 * b);
            }
            store_column<FMT>(a, out_row + side, row, n, codes);
        }
    } else {
        const int c = t % kQTile, r0 = t / kQTile * 32;
        const long long row = (long long)row_tile * kQTile + pass + r0;
        uint32_t n[4], codes = 0;
#pragma unroll
        for (int b = 0; b < 32 / kB; ++b) {
            float y[kB];
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < kB; ++j) {
                y[j] = tile[(r0 + b * kB + j) * stride + c];
                top = max(top, __float_as_uint(y[j]) & 0x7fffffffu);
            }
            codes |= quantise_run<FMT, kB>(n + b * (kB / 8), y, top, inv_tensor) << (8 * b);
        }
        store_column<FMT>(a, (long long)col_tile * kQTile + c, row, n, codes);
    }
}

// One block takes a 128 x 128 tile, which is whole scale tiles of either orientation; a value is read once
// for both, through shared memory for the columns' blocks.  16384 x 4096 bfloat16, E8M0: rows 32 us
// (5.3 TB/s), both ways 51 us (4.0 TB/s).  What bounds both ways is instructions, 0.66 a cycle and
// scheduler: two quotients, two roundings and half a transpose per element.
template <typename T, int FMT, bool ROWS, bool COLS> __global__ void __launch_bounds__(kQThreads, 4) k_fp4_quantise(QuantiseArgs a) {
    constexpr int kB = Fp4<FMT>::kBlock, kBlocks = kQTile / kB;  // blocks along a tile's side
    constexpr int kPad = 16 / (int)sizeof(T);
    constexpr int kPass = COLS ? 256 / (int)sizeof(T) : kQTile;  // rows held in shared memory at a time (up to 34 KB)
    __shared__ uint32_t codes[kQTile][kBlocks / 4];              // a row's scale bytes, four to a word
    __shared__ alignas(16) T tile[COLS ? kPass : 1][COLS ? kQTile + kPad : 8];
    const T* x = static_cast<const T*>(a.x);
    const int t = threadIdx.x, lane = t & 31;
    after_earlier_kernels();
    // the matrix was read from its start for the maximum: what L2 still holds of it is its end (8192^2
    // bfloat16 63.4 us from the start, 62.0 from the end, the maximum included)
    const uint32_t at = FMT == SBC_FP4_E4M3 ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
    const uint32_t row_tile = at / a.col_tiles, col_tile = at % a.col_tiles;
    const long long row0 = (long long)row_tile * kQTile, col0 = (long long)col_tile * kQTile;
    float tensor = 1.f, inv_tensor = 1.f;
    if (FMT == SBC_FP4_E4M3) {
        tensor = tensor_scale_of(tensor_amax<T>(a));
        inv_tensor = 1.f / tensor;
    }
    if (blockIdx.x == 0 && t == 0) {
        if (ROWS) *a.tensor_r = tensor;
        if (COLS) *a.tensor_c = tensor;
    }
    // sixteen threads to a row, eight elements each, sixteen rows at a time
    const int cc = (t & 15) * 8;
    const int have = (int)max(0LL, min(8LL, a.cols - (col0 + cc)));
    constexpr int kStep = kQThreads / 16, kBatch = 16 / (int)sizeof(T);   // rows a step, steps whose loads are under way together (32 registers)
    for (int pass = 0; pass < kQTile; pass += kPass) {
#pragma unroll 1
        for (int r1 = 0; r1 < kPass; r1 += kStep * kBatch) {
            Pack8<T> v[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const long long r = row0 + pass + r1 + i * kStep + (t >> 4);
                load8(v[i], x + r * a.stride + col0 + cc, r < a.rows ? have : 0, a.align);
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int rr = r1 + i * kStep + (t >> 4);
                const long long r = row0 + pass + rr;
                if (COLS) {
#pragma unroll
                    for (int q = 0; q < (int)sizeof(T) / 2; ++q) reinterpret_cast<uint4*>(&tile[COLS ? rr : 0][COLS ? cc : 0])[q] = v[i].q[q];
                }
                if (ROWS) {
                    float y[8];
                    uint32_t top = unpack_max(y, v[i]);
#pragma unroll
                    for (int d = 1; d < kB / 8; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
                    const BlockScale<FMT> scale(top, inv_tensor);
                    scale.template over<8>(y, inv_tensor);
                    if (r < a.rows && (col0 + cc) / 2 < a.pitch_r)
                        *reinterpret_cast<uint32_t*>(a.values_r + r * a.pitch_r + (col0 + cc) / 2) = scale.zero() ? 0u : pack_nibbles(y);
                    if (lane % (kB / 8) == 0) reinterpret_cast<uint8_t*>(codes[pass + rr])[cc / kB] = (uint8_t)scale.code;
                }
            }
        }
        if (!COLS) continue;
        __syncthreads();
        quantise_columns<T, FMT>(a, &tile[0][0], kQTile + kPad, row_tile, col_tile, pass, inv_tensor);
        __syncthreads();
    }
    if (ROWS) {
        __syncthreads();
        for (int i = t; i < kQTile * (kBlocks / 4); i += kQThreads) {
            const int kt = i / kQTile, rr = i % kQTile;
            const long long k = (long long)col_tile * (kBlocks / 4) + kt;
            if (k < a.ktiles_r)
                *reinterpret_cast<uint32_t*>(a.scales_r + ((long long)row_tile * a.ktiles_r + k) * 512 + (rr % 32) * 16 + (rr / 32) * 4) =
                    codes[rr][kt];
        }
    }
}

struct DequantiseArgs {
    const uint8_t *values, *scales;
    const float* tensor;
    void* out;
    long long rows, cols, stride, pitch, ktiles;
};

// The grid values of N (4 or 8) nibbles, exact.  A bfloat16 holds them, its two bytes come from tables
// that a byte permutation looks up, four at a time.
template <int N> __device__ __forceinline__ void grid_values(float* x, uint32_t w) {
    const uint32_t m = w & 0x77777777u;
#pragma unroll
    for (int h = 0; h < N / 4; ++h) {
        const uint32_t hi = __byte_perm(0x3f3f3f00u, 0x40404040u, m >> (16 * h)), lo = __byte_perm(0xc0800000u, 0xc0804000u, m >> (16 * h));
        const uint32_t a = __byte_perm(lo, hi, 0x5140), b = __byte_perm(lo, hi, 0x7362);   // values 0, 1 and 2, 3
        const uint32_t s = w >> (16 * h);
        x[4 * h + 0] = __uint_as_float((a << 16) | (s << 28 & 0x80000000u));
        x[4 * h + 1] = __uint_as_float((a & 0xffff0000u) | (s << 24 & 0x80000000u));
        x[4 * h + 2] = __uint_as_float((b << 16) | (s << 20 & 0x80000000u));
        x[4 * h + 3] = __uint_as_float((b & 0xffff0000u) | (s << 16 & 0x80000000u));
    }
}

template <int FMT> __device__ __forceinline__ float scale_value(uint32_t code) {
    if (FMT == SBC_FP4_E8M0)
        return code == 255u ? __uint_as_float(0x7fffffffu) : code == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(code << 23);
    return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
}

// Element = grid point x block scale x tensor scale, rounded once, in the type asked for.  Bound by its
// stores: 16384 x 4096 to bfloat16 33 us, 5.2 TB/s.
//
// A warp's rows in pieces of 2048 elements, cut where the output's 16-byte granules fall: stores are whole
// granules at any alignment.  SHIFT: rows start inside a granule, so what moves is the nibbles (a funnel
// shift of two words) and the place in a granule where a block ends.  (With stores as wide as an odd
// row's alignment 16384 x 4095 bfloat16 took 196 us.)
template <typename T, int FMT, bool SHIFT> __global__ void __launch_bounds__(kQThreads, 4) k_fp4_dequantise(DequantiseArgs a) {
    constexpr int kB = Fp4<FMT>::kBlock, E = 16 / (int)sizeof(T), kAhead = SHIFT ? 4 : 8;
    after_earlier_kernels();
    const float tensor = FMT == SBC_FP4_E4M3 ? *a.tensor : 1.f;
    const int lane = threadIdx.x & 31;
    const uint32_t warp = blockIdx.x * (kQThreads / 32) + threadIdx.x / 32, warps = gridDim.x * (kQThreads / 32);
    const uint32_t per_row = (uint32_t)((a.cols + (SHIFT ? E - 1 : 0) + kPiece - 1) / kPiece);
    const long long all = a.rows * per_row;
    for (long long i = warp; i < all; i += warps) {
        const long long r = all < (1ll << 32) ? (long long)((uint32_t)i / per_row) : i / per_row;
        T* const row = static_cast<T*>(a.out) + r * a.stride;
        const int phase = SHIFT ? (int)((uint32_t)(uintptr_t)row & 15u) / (int)sizeof(T) : 0;
        // this lane's first granule (the next ones are 32 lanes apart), and how many elements there are from it on
        const long long first = (i - r * per_row) * kPiece - phase + lane * E;
        const int left = (int)min(a.cols - first, (long long)kPiece + E);
        const int most = SHIFT ? __shfl_sync(0xffffffffu, left, 0) : left;   // lane 0 has most
        if (most <= 0) continue;
        // positions are counted from the granule that the row starts in (32 bits without a sign: a row may have 2^31 - 1
        // elements, and a piece goes on behind them); element e of the row is at e + phase
        const uint32_t p0 = (uint32_t)(first + phase), end = (uint32_t)a.cols - 1;
        const auto element = [&](uint32_t p) { return max(p, (uint32_t)phase) - (uint32_t)phase; };   // the first one at or behind p
        const uint8_t* const values = a.values + r * a.pitch;
        const uint8_t* const scales = a.scales + r / 128 * a.ktiles * 512 + (r % 32) * 16 + (r % 128 / 32) * 4;
        const auto code_of = [&](uint32_t e) { return (uint32_t)scales[(size_t)(e / (4 * kB)) * 512 + e / kB % 4]; };
        T* const to = row + first;
        constexpr int kGrans = kPiece / (32 * E);
#pragma unroll
        for (int g0 = 0; g0 < kGrans; g0 += kAhead) {
            uint32_t lo[kAhead], hi[kAhead], c0[kAhead], c1[kAhead];
#pragma unroll
            for (int g = 0; g < kAhead; ++g) {
                const int at = (g0 + g) * 32 * E;
                if ((SHIFT ? most : left) <= at) break;
                if (SHIFT) {
                    // what follows a lane's word and block is the next lane's
                    const uint32_t f = min(element(p0 + at), end);
                    lo[g] = reinterpret_cast<const uint32_t*>(values)[f / 8];
                    c0[g] = code_of(f);
                    hi[g] = c1[g] = 0;
                    if (lane == 31) {
                        const uint32_t next = min(f + E, end);
                        hi[g] = reinterpret_cast<const uint32_t*>(values)[next / 8];
                        c1[g] = code_of(next);
                    }
                } else {
                    // (a step of 32 granules is whole scale tiles, or half of one for 32 x 4 elements of 32-element blocks)
                    if (E == 8) lo[g] = *reinterpret_cast<const uint32_t*>(values + (p0 + at) / 2);
                    if (E == 4) lo[g] = *reinterpret_cast<const uint16_t*>(values + (p0 + at) / 2);
                    c0[g] = code_of(p0 + at);
                }
            }
#pragma unroll
            for (int g = 0; g < kAhead; ++g) {
                const int at = (g0 + g) * 32 * E;
                if ((SHIFT ? most : left) <= at) break;
                if (SHIFT) {
                    const uint32_t word = __shfl_down_sync(0xffffffffu, lo[g], 1), code = __shfl_down_sync(0xffffffffu, c0[g], 1);
                    if (lane < 31) hi[g] = word, c1[g] = code;
                }
                if (SHIFT && left <= at) continue;
                float x[E];
                const float s0 = scale_value<FMT>(c0[g]) * tensor;
                uint4 q;
                T* v = reinterpret_cast<T*>(&q);
                int skip = 0;
                if (SHIFT) {
                    const uint32_t f = element(p0 + at);
                    skip = (int)(f + (uint32_t)phase - (p0 + at));
                    grid_values<E>(x, __funnelshift_r(lo[g], hi[g], 4 * (f & 7u)));
                    const float s1 = scale_value<FMT>(c1[g]) * tensor;
                    const int split = kB - (int)(f % kB);   // elements of the granule that belong to the first block
#pragma unroll
                    for (int j = 0; j < E; ++j) v[j] = from_float<T>(x[j] * (j < split ? s0 : s1));
                } else {
                    grid_values<E>(x, lo[g]);
#pragma unroll
                    for (int j = 0; j < E; ++j) v[j] = from_float<T>(x[j] * s0);
                }
                if (skip == 0 && left >= at + E) {
                    *reinterpret_cast<uint4*>(to + at) = q;
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j)
                        if (j + skip < E && at + skip + j < left) to[at + skip + j] = v[j];
                }
            }
        }
    }
}

}  // namespace sbclm
