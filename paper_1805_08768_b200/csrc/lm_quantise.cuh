// 4-bit floating point: quantisation along rows and columns, and expansion.
//
// Arithmetic.  With s the block's scale (block scale * tensor scale, an exact product of a float of
// at most 4 significant bits and a power of two) an element becomes the grid point nearest to
// x / s.  For E8M0 the quotient is exact.  For E4M3 the quotient is the correctly rounded one, and
// that decides like the exact one: a grid midpoint m has at most 3 significant bits, m * s is a
// float, so an x that is not m * s differs from it by at least one unit in the last place, and the
// rounded quotient then is not m either.  The same holds for the block scale, amax / (6 * 2^g).
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

// A block's scale code, and the factor or divisor its elements take.
template <int FMT> __device__ __forceinline__ uint32_t scale_code(uint32_t amax_bits, float tensor, float* by) {
    if (amax_bits >= 0x7f800000u) {
        *by = 0.f;
        return Fp4<FMT>::kNanScale;
    }
    if (FMT == SBC_FP4_E8M0) {
        const uint32_t code = (uint32_t)max((int)(amax_bits >> 23) - 2, 0);
        *by = __uint_as_float((254u - code) << 23);  // 1 / scale, exact
        return code;
    }
    const float want = __uint_as_float(amax_bits) / (6.f * tensor);
    const uint32_t code = __nv_cvt_float_to_fp8(want, __NV_SATFINITE, __NV_E4M3);
    *by = __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3))) * tensor;
    return code;
}

template <int FMT> __device__ __forceinline__ float scaled(float x, float by) {
    if (FMT == SBC_FP4_E8M0) return x * by;
    return by > 0.f ? x / by : 0.f;
}

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

struct QuantiseArgs {
    const void* x;
    long long rows, cols, stride;
    int align;                    // every row starts at a multiple of this many bytes
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
constexpr long long kAmaxAlone = 32768;   // elements up to which every block finds the maximum itself, instead of a launch in front

// Largest finite magnitude of the elements that threads [at, at + step, ...) of the tensor take, over the
// block, as float bits (whole numbers: the maximum does not depend on the order).
template <typename T> __device__ __forceinline__ uint32_t amax_over(const QuantiseArgs& a, long long at, long long step, uint32_t* room) {
    const T* x = static_cast<const T*>(a.x);
    const long long per_row = (a.cols + 7) / 8, all = per_row * a.rows;
    uint32_t top = 0;
    for (long long i = at; i < all; i += step) {
        const long long r = all < (1ll << 31) ? (long long)((uint32_t)i / (uint32_t)per_row) : i / per_row, c = (i - r * per_row) * 8;
        Pack8<T> v;
        load8(v, x + r * a.stride + c, (int)min(8LL, a.cols - c), a.align);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = __float_as_uint(to_float(v.e[j])) & 0x7fffffffu;
            top = max(top, b < 0x7f800000u ? b : 0u);
        }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = top;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, room[threadIdx.x & (kQThreads / 32 - 1)]);
}

template <typename T> __global__ void __launch_bounds__(kQThreads) k_fp4_amax(QuantiseArgs a, uint32_t* amax) {
    __shared__ uint32_t room[kQThreads / 32];
    const uint32_t top = amax_over<T>(a, (long long)blockIdx.x * kQThreads + threadIdx.x, (long long)gridDim.x * kQThreads, room);
    if (threadIdx.x == 0) amax[blockIdx.x] = top;
}

// The tensor's, in every block of the quantising kernel.
template <typename T> __device__ __forceinline__ uint32_t tensor_amax(const QuantiseArgs& a) {
    __shared__ uint32_t room[kQThreads / 32];
    if (a.amax_blocks == 0) return amax_over<T>(a, threadIdx.x, kQThreads, room);
    uint32_t top = 0;
    for (int i = threadIdx.x; i < a.amax_blocks; i += kQThreads) top = max(top, a.amax[i]);
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = top;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, room[threadIdx.x & (kQThreads / 32 - 1)]);
}

// One block takes a 128 x 128 tile, which is whole scale tiles of either orientation.
template <typename T, int FMT, bool ROWS, bool COLS> __global__ void __launch_bounds__(kQThreads) k_fp4_quantise(QuantiseArgs a) {
    constexpr int kB = Fp4<FMT>::kBlock, kBlocks = kQTile / kB;  // blocks along a tile's side
    constexpr int kPad = 16 / (int)sizeof(T);
    constexpr int kPass = COLS ? 256 / (int)sizeof(T) : kQTile;  // rows held in shared memory at a time (up to 34 KB)
    constexpr int kHalf = kPass / 2;                             // rows of a column that one thread takes
    __shared__ uint32_t codes[kQTile][kBlocks / 4];              // a row's scale bytes, four to a word
    __shared__ alignas(16) T tile[COLS ? kPass : 1][COLS ? kQTile + kPad : 8];
    const T* x = static_cast<const T*>(a.x);
    const int t = threadIdx.x, lane = t & 31;
    const uint32_t row_tile = blockIdx.x / a.col_tiles, col_tile = blockIdx.x % a.col_tiles;
    const long long row0 = (long long)row_tile * kQTile, col0 = (long long)col_tile * kQTile;
    float tensor = 1.f;
    if (FMT == SBC_FP4_E4M3) tensor = tensor_scale_of(tensor_amax<T>(a));
    if (blockIdx.x == 0 && t == 0) {
        if (ROWS) *a.tensor_r = tensor;
        if (COLS) *a.tensor_c = tensor;
    }
    // sixteen threads to a row, eight elements each, sixteen rows at a time
    const int cc = (t & 15) * 8;
    const int have = (int)max(0LL, min(8LL, a.cols - (col0 + cc)));
    for (int pass = 0; pass < kQTile; pass += kPass) {
#pragma unroll 2
        for (int rr = t >> 4; rr < kPass; rr += kQThreads / 16) {
            const long long r = row0 + pass + rr;
            Pack8<T> v;
            load8(v, x + r * a.stride + col0 + cc, r < a.rows ? have : 0, a.align);
            if (COLS) {
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(&tile[rr][cc])[i] = v.q[i];
            }
            if (ROWS) {
                float y[8];
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    y[j] = to_float(v.e[j]);
                    top = max(top, __float_as_uint(y[j]) & 0x7fffffffu);
                }
#pragma unroll
                for (int d = 1; d < kB / 8; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
                float by;
                const uint32_t code = scale_code<FMT>(top, tensor, &by);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = scaled<FMT>(y[j], by);
                if (r < a.rows && (col0 + cc) / 2 < a.pitch_r)
                    *reinterpret_cast<uint32_t*>(a.values_r + r * a.pitch_r + (col0 + cc) / 2) = by > 0.f ? pack_nibbles(y) : 0u;
                if (lane % (kB / 8) == 0) reinterpret_cast<uint8_t*>(codes[pass + rr])[cc / kB] = (uint8_t)code;
            }
        }
        if (!COLS) continue;
        __syncthreads();
        {
            const int c = t % kQTile, r0 = (t / kQTile) * kHalf;
            const long long out_row = col0 + c;
            uint32_t word = 0;
#pragma unroll
            for (int b = 0; b < kHalf / kB; ++b) {
                float y[kB];
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < kB; ++j) {
                    y[j] = to_float(tile[COLS ? r0 + b * kB + j : 0][COLS ? c : 0]);
                    top = max(top, __float_as_uint(y[j]) & 0x7fffffffu);
                }
                float by;
                word |= scale_code<FMT>(top, tensor, &by) << (8 * b);
                uint32_t n[kB / 8];
#pragma unroll
                for (int j = 0; j < kB; ++j) y[j] = scaled<FMT>(y[j], by);
#pragma unroll
                for (int j = 0; j < kB / 8; ++j) n[j] = by > 0.f ? pack_nibbles(y + 8 * j) : 0u;
                const long long at = (row0 + pass + r0 + b * kB) / 2;
                if (out_row < a.cols && at < a.pitch_c) {
                    uint8_t* p = a.values_c + out_row * a.pitch_c + at;
                    if (FMT == SBC_FP4_E8M0)
                        *reinterpret_cast<uint4*>(p) = make_uint4(n[0], n[1], n[kB / 8 - 2], n[kB / 8 - 1]);
                    else
                        *reinterpret_cast<uint2*>(p) = make_uint2(n[0], n[1]);
                }
            }
            const int first = (pass + r0) / kB;  // the thread's first block within the tile's rows
            const long long k = (long long)row_tile * (kBlocks / 4) + first / 4;
            if (k < a.ktiles_c) {
                uint8_t* p = a.scales_c + ((long long)col_tile * a.ktiles_c + k) * 512 + (c % 32) * 16 + (c / 32) * 4 + first % 4;
                if (kHalf / kB == 4)
                    *reinterpret_cast<uint32_t*>(p) = word;
                else if (kHalf / kB == 2)
                    *reinterpret_cast<uint16_t*>(p) = (uint16_t)word;
                else
                    *p = (uint8_t)word;
            }
        }
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
    int align;
};

// The grid value of nibble i of `w`, exact.
__device__ __forceinline__ float grid_value(uint32_t w, int i) {
    const uint32_t n = w >> (4 * i), m = n & 7u;
    // 0, 0.5: m / 2; above: exponent m >> 1, fraction m & 1
    const float v = m < 2 ? 0.5f * (float)m : __uint_as_float(((m >> 1) + 126u) << 23 | (m & 1u) << 22);
    return (n & 8u) ? -v : v;
}

template <int FMT> __device__ __forceinline__ float scale_value(uint32_t code) {
    if (FMT == SBC_FP4_E8M0)
        return code == 255u ? __uint_as_float(0x7fffffffu) : code == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(code << 23);
    return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)code, __NV_E4M3)));
}

// Eight elements a thread.
template <typename T, int FMT> __global__ void __launch_bounds__(kQThreads) k_fp4_dequantise(DequantiseArgs a) {
    constexpr int kB = Fp4<FMT>::kBlock;
    T* out = static_cast<T*>(a.out);
    const long long per_row = (a.cols + 7) / 8, all = per_row * a.rows;
    const float tensor = FMT == SBC_FP4_E4M3 ? *a.tensor : 1.f;
    for (long long i = (long long)blockIdx.x * kQThreads + threadIdx.x; i < all; i += (long long)gridDim.x * kQThreads) {
        const long long r = i / per_row, c = (i - r * per_row) * 8, b = c / kB;
        const uint32_t w = *reinterpret_cast<const uint32_t*>(a.values + r * a.pitch + c / 2);
        const uint32_t code = a.scales[((r / 128) * a.ktiles + b / 4) * 512 + (r % 32) * 16 + (r % 128 / 32) * 4 + b % 4];
        const float s = scale_value<FMT>(code) * tensor;
        Pack8<T> v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v.e[j] = from_float<T>(grid_value(w, j) * s);
        store8(out + r * a.stride + c, v, (int)min(8LL, a.cols - c), a.align);
    }
}

}  // namespace sbclm
