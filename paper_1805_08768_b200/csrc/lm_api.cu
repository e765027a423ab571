// C entry points of the language-model operators (include/sbc_lm.h).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "lm_common.cuh"
#include "lm_logits.cuh"
#include "lm_product.cuh"
#include "lm_quantise.cuh"

using namespace sbclm;

namespace {

constexpr int64_t kMaxDim = 0x7fffffff;

int width_of(int dtype) { return dtype == SBC_F32 ? 4 : (dtype == SBC_BF16 || dtype == SBC_F16) ? 2 : 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// SMs of the current device (asked for once per device: the question costs as much as half a launch).
int sm_count() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 148;
    if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 148;
    if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

// What every row of a matrix starts at a multiple of, at most 16 bytes.
int row_align(const void* p, int64_t stride, int width) {
    const uintptr_t bits = (uintptr_t)p | (uintptr_t)(stride * width) | 16u;
    return (int)(bits & (~bits + 1));
}

// A matrix argument: base, type and stride fit together.
bool matrix_ok(const void* p, int dtype, int64_t rows, int64_t cols, int64_t stride) {
    const int width = width_of(dtype);
    return p && width && aligned(p, (uintptr_t)width) && rows >= 0 && rows <= kMaxDim && cols >= 1 && cols <= kMaxDim && stride >= cols &&
           stride <= (int64_t)1 << 40;
}

int64_t ktiles_of(int64_t cols, int format) { return ceil_div(cols, format == SBC_FP4_E8M0 ? 128 : 64); }

bool fp4_ok(const sbc_fp4* q) {
    return q && q->values && q->scales && q->tensor_scale && aligned(q->values, 16) && aligned(q->scales, 16) &&
           aligned(q->tensor_scale, 4) && q->rows >= 1 && q->rows <= kMaxDim && q->cols >= 1 && q->cols <= kMaxDim && q->reserved == 0 &&
           (q->format == SBC_FP4_E8M0 || q->format == SBC_FP4_E4M3);
}

// dtype -> element type
template <typename F> int by_dtype(int dtype, F f) {
    switch (dtype) {
        case SBC_F32: return f((float*)nullptr);
        case SBC_BF16: return f((__nv_bfloat16*)nullptr);
        case SBC_F16: return f((__half*)nullptr);
    }
    return SBC_EINVAL;
}

// Raises a kernel's limit of dynamic shared memory, once per device.
template <auto Kernel> bool allow_smem(int bytes) {
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return true;
    if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

// Blocks that have a piece of a matrix for every warp.
int64_t pieces(int64_t rows, int64_t cols, bool flat) {
    const int64_t n = flat ? ceil_div(rows * cols, kPiece) : rows * ceil_div(cols, kPiece);
    return ceil_div(n, kQThreads / 32);
}

// One launch: `cluster` blocks along `axis` (0: x, 2: z) together, allowed to start while the kernel in
// front ends (the kernels wait for it themselves).
template <typename... P, typename... A>
int launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, int axis, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = axis == 0 ? (unsigned)cluster : 1;
    attr[1].val.clusterDim.y = axis == 1 ? (unsigned)cluster : 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...) == cudaSuccess ? SBC_OK : SBC_ECUDA;
}

template <typename T, int FMT> int launch_quantise(const QuantiseArgs& a, bool rows, bool cols, unsigned grid, cudaStream_t st) {
    const auto kernel = rows && cols ? k_fp4_quantise<T, FMT, true, true> : rows ? k_fp4_quantise<T, FMT, true, false> : k_fp4_quantise<T, FMT, false, true>;
    return launch(kernel, grid, kQThreads, 0, st, 0, 0, a);
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return (EncodeTiled)p;
    }();
    return fn;
}

// Boxes of 128 bytes x `rows` of the elements' bytes, in the swizzle that the tensor cores read.
bool values_map(CUtensorMap* map, const sbc_fp4* q, int rows) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)sbc_fp4_row_bytes(q->cols), (cuuint64_t)q->rows};
    const cuuint64_t strides[1] = {dims[0]};
    const cuuint32_t box[2] = {kPBytes, (cuuint32_t)rows}, ones[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, q->values, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kSmemMost = 227 * 1024;

template <typename T, int FMT>
int launch_product(const CUtensorMap& mw, const CUtensorMap& mx, const ProductArgs& a, dim3 grid, int smem, cudaStream_t st) {
    if (!allow_smem<k_fp4_product<T, FMT>>(kSmemMost - 1024)) return SBC_ECUDA;
    return launch(k_fp4_product<T, FMT>, grid, kPThreads, (size_t)smem, st, (int)grid.y, 1, mw, mx, a);
}

// How a row of logits is cut: blocks that share it, elements a block holds in shared memory at a
// time, threads of a block.
struct RowPlan {
    int size, shift, room, threads;
};

// A segment is at most kRoomBytes where eight blocks are enough for that; few rows are spread over as
// many blocks as keep the GPU busy, each with at least 8192 elements (us alone / spread, 8 float32 rows:
// top 32 of 10000 words 7.1 / 9.5, of 131072 13.4 / 13.4; loss and gradient of 10000 6.7 / 6.4, of 32768
// 15.9 / 7.3, of 131072 48 / 11).
constexpr int kRoomBytes = 100 * 1024;
int spread(int64_t rows, int64_t cols, int shift) {
    const int64_t blocks = 2 * sm_count();
    while (shift < 3 && rows * (2 << shift) <= blocks && cols >= 8192 * (2 << shift)) ++shift;
    return shift;
}
RowPlan plan_rows(int64_t rows, int64_t cols, int width) {
    int shift = 0;
    while (shift < 3 && cols * width > ((int64_t)kRoomBytes << shift)) ++shift;
    RowPlan p;
    p.shift = spread(rows, cols, shift);
    p.size = 1 << p.shift;
    const int64_t segment = ceil_div(ceil_div(cols, 64), p.size) * 64;
    p.room = (int)std::min<int64_t>(segment, kRoomBytes / width);
    p.threads = segment * width <= 32 * 1024 ? 128 : 256;
    return p;
}

// Candidates that a block of k_top_logits has room for, where `size` blocks share a row.  In whole eights:
// the row that the block holds lies behind the two lists and starts at a multiple of 16 bytes.
constexpr int candidate_room(int k, int size) { return (std::max(std::max(512, 4 * k), k * size) + 7) / 8 * 8; }
static_assert(8 * kCandidateBytes % 16 == 0 && kStreamRoom % 8 == 0, "what lies behind the lists is read 16 bytes at a time");

// Beyond these the scaled logits would leave 32 bits.
bool temperature_ok(float t) { return t >= 1e-6f && t <= 1e6f; }

bool distill_ok(const sbc_distill* d, int64_t rows, int64_t cols) {
    return d && (rows == 0 || (d->values && d->indices)) && aligned(d->values, 4) && aligned(d->indices, 4) && aligned(d->rest, 4) &&
           aligned(d->labels, 8) && d->k >= 1 && d->k <= SBC_DISTILL_MOST && temperature_ok(d->temperature) &&
           d->alpha >= 0.f && d->alpha <= 1.f && d->reserved == 0 && cols <= SBC_DISTILL_COLS && rows <= kMaxDim / 8;
}

DistillArgs distill_args(const void* logits, int64_t rows, int64_t cols, int64_t stride, const sbc_distill* d) {
    DistillArgs a = {};
    a.logits = logits;
    a.rows = rows;
    a.stride = stride;
    a.cols = (int)cols;
    a.k = d->k;
    a.temperature = d->temperature;
    a.alpha = d->alpha;
    a.values = d->values;
    a.indices = d->indices;
    a.rest = d->rest;
    a.labels = d->alpha < 1.f ? reinterpret_cast<const long long*>(d->labels) : nullptr;
    return a;
}

// A second exponential per element where labels are mixed in at another temperature than the teacher's.
bool second_exponential(const DistillArgs& a) { return a.labels && a.temperature != 1.f; }

// Bytes of a segment that a block of k_distill holds at a time.  Nine to ten blocks fit an SM for the word
// model's rows, five for longer ones; us for loss / loss and gradient with parts of 24, 32, 40 and 48 KB:
// 4095 x 50001 bfloat16 91, 92, 94, 105 / 201, 194, 189, 200; 4480 x 10000 float32 - / 76, 81, 70, 70;
// 4096 x 32000 bfloat16 - / 121, 114, 117, 126.
constexpr int kPartBytes = 40 * 1024;

template <typename T, bool CE2, bool GRAD> int launch_distill(DistillArgs a, cudaStream_t st) {
    a.shift = spread(a.rows, a.cols, 0);
    const int64_t segment = ceil_div(ceil_div(a.cols, 64), 1 << a.shift) * 64 + 8;   // with the row's offset from a granule
    a.part = (int)std::min<int64_t>(segment, kPartBytes / (int)sizeof(T));
    const size_t smem = (size_t)a.part * sizeof(T) + (size_t)a.k * 12;
    if (!allow_smem<k_distill<T, CE2, GRAD>>(kPartBytes + SBC_DISTILL_MOST * 12)) return SBC_ECUDA;
    return launch(k_distill<T, CE2, GRAD>, dim3((unsigned)(a.rows << a.shift)), kDistillThreads, smem, st, 1 << a.shift, 0, a);
}

template <bool GRAD> int distill_by_type(const DistillArgs& a, int dtype, cudaStream_t st) {
    return by_dtype(dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        return second_exponential(a) ? launch_distill<T, true, GRAD>(a, st) : launch_distill<T, false, GRAD>(a, st);
    });
}

template <typename T, int FMT, int NT>
int launch_wide(const sbc_fp4* a, const sbc_fp4* b, WideArgs p, int64_t tiles, cudaStream_t st) {
    using Shape = ProductShape<FMT>;
    if (tiles > kMaxDim / 2) return SBC_EINVAL;
    p.tiles = (int)tiles;
    const int stage = kPRows * kPBytes + NT / 2 * kPBytes, scales = kWScales * Shape::kTiles * 512 * (1 + NT / 128);
    p.stages = std::min(std::min(kWMaxStages, (224 * 1024 - scales) / stage), 256 / (4 * Shape::kTiles * (1 + NT / 128)));
    CUtensorMap mw, mx;
    if (!values_map(&mw, b, kPRows) || !values_map(&mx, a, NT / 2)) return SBC_ECUDA;
    if (!allow_smem<k_fp4_product_wide<T, FMT, NT>>(kSmemMost - 1024)) return SBC_ECUDA;
    const unsigned blocks = (unsigned)(2 * std::min<int64_t>(std::max(1, sm_count() / 2), tiles));
    // (always more than half of an SM's shared memory: a block takes all of its tensor memory)
    return launch(k_fp4_product_wide<T, FMT, NT>, dim3(blocks), kWThreads, (size_t)(p.stages * stage + scales + 1024), st, 2, 0, mw, mx, p);
}

// Pairs of blocks that stay.  Tiles of 256 tokens, or of 128 with two accumulators: by the rounds that the
// pairs take, a round of 256 counted as 1.6 of 128 (us with tiles of 256 / 128: 8192^3 242 / 404,
// 4096^3 43 / 58, 3000 x 2048 -> 3000 17.3 / 21.5, 2240 x 1300 -> 2600 15.1 / 14.0).  32-bit results
// always take 128: more do not fit in registers until they are stored.
int product_wide(const sbc_fp4* a, const sbc_fp4* b, void* out, int dtype, int64_t row_stride, uint32_t* status, cudaStream_t st) {
    WideArgs p = {};
    p.scales_w = static_cast<const uint8_t*>(b->scales);
    p.scales_x = static_cast<const uint8_t*>(a->scales);
    p.tensor_w = b->tensor_scale;
    p.tensor_x = a->tensor_scale;
    p.out = out;
    p.status = status;
    p.rows_w = b->rows;
    p.rows_x = a->rows;
    p.stride = row_stride;
    p.ktiles = ktiles_of(a->cols, a->format);
    p.chunks = (int)ceil_div(a->cols, 256);
    p.steps = (int)ceil_div(a->cols, 64);
    const int64_t tiles_w = ceil_div(b->rows, 256), tiles256 = tiles_w * ceil_div(a->rows, 256), tiles128 = tiles_w * ceil_div(a->rows, 128);
    p.tiles_w = (int)tiles_w;
    const int64_t pairs = std::max(1, sm_count() / 2);
    const bool big = 16 * ceil_div(tiles256, pairs) <= 10 * ceil_div(tiles128, pairs);
    return by_dtype(dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        if constexpr (sizeof(T) == 2) {
            if (big)
                return a->format == SBC_FP4_E4M3 ? launch_wide<T, SBC_FP4_E4M3, 256>(a, b, p, tiles256, st)
                                                 : launch_wide<T, SBC_FP4_E8M0, 256>(a, b, p, tiles256, st);
        }
        return a->format == SBC_FP4_E4M3 ? launch_wide<T, SBC_FP4_E4M3, 128>(a, b, p, tiles128, st)
                                         : launch_wide<T, SBC_FP4_E8M0, 128>(a, b, p, tiles128, st);
    });
}

}  // namespace

extern "C" {

size_t sbc_fp4_row_bytes(int64_t cols) { return cols >= 1 && cols <= kMaxDim ? (size_t)(ceil_div(cols, 32) * 16) : 0; }

size_t sbc_fp4_scale_bytes(int64_t rows, int64_t cols, int format) {
    if (rows < 1 || rows > kMaxDim || cols < 1 || cols > kMaxDim || (format != SBC_FP4_E8M0 && format != SBC_FP4_E4M3)) return 0;
    return (size_t)(ceil_div(rows, 128) * ktiles_of(cols, format) * 512);
}

size_t sbc_fp4_workspace_bytes(int64_t rows, int64_t cols, int format) {
    return sbc_fp4_scale_bytes(rows, cols, format) ? kAmaxBlocks * 4 : 0;
}

int sbc_fp4_quantise(const void* x, int dtype, int64_t rows, int64_t cols, int64_t row_stride, const sbc_fp4* along_rows,
                     const sbc_fp4* along_cols, void* workspace, size_t workspace_bytes, sbc_cuda_stream_t stream) {
    if (!matrix_ok(x, dtype, rows, cols, row_stride) || rows < 1 || (!along_rows && !along_cols)) return SBC_EINVAL;
    if (along_rows && (!fp4_ok(along_rows) || along_rows->rows != rows || along_rows->cols != cols)) return SBC_EINVAL;
    if (along_cols && (!fp4_ok(along_cols) || along_cols->rows != cols || along_cols->cols != rows)) return SBC_EINVAL;
    const int format = along_rows ? along_rows->format : along_cols->format;
    if (along_rows && along_cols && along_cols->format != format) return SBC_EINVAL;
    if (!workspace || !aligned(workspace, 16)) return SBC_EINVAL;
    if (workspace_bytes < sbc_fp4_workspace_bytes(rows, cols, format)) return SBC_ECAPACITY;
    const int64_t row_tiles = ceil_div(rows, kQTile), col_tiles = ceil_div(cols, kQTile);
    if (row_tiles > kMaxDim / col_tiles) return SBC_EINVAL;

    QuantiseArgs a = {};
    a.x = x;
    a.rows = rows;
    a.cols = cols;
    a.stride = row_stride;
    a.align = row_align(x, row_stride, width_of(dtype));
    a.base_align = row_align(x, 0, 1);
    a.col_tiles = (uint32_t)col_tiles;
    a.amax = static_cast<const uint32_t*>(workspace);
    if (along_rows) {
        a.tensor_r = along_rows->tensor_scale;
        a.values_r = static_cast<uint8_t*>(along_rows->values);
        a.scales_r = static_cast<uint8_t*>(along_rows->scales);
        a.pitch_r = (long long)sbc_fp4_row_bytes(cols);
        a.ktiles_r = ktiles_of(cols, format);
    }
    if (along_cols) {
        a.tensor_c = along_cols->tensor_scale;
        a.values_c = static_cast<uint8_t*>(along_cols->values);
        a.scales_c = static_cast<uint8_t*>(along_cols->scales);
        a.pitch_c = (long long)sbc_fp4_row_bytes(rows);
        a.ktiles_c = ktiles_of(rows, format);
    }
    return by_dtype(dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        cudaStream_t st = stream;
        if (format == SBC_FP4_E4M3) {
            const int64_t blocks = pieces(rows, cols, row_stride == cols);
            if (blocks > kAmaxAlone) {
                a.amax_blocks = (int)std::min<int64_t>(blocks, kAmaxBlocks);
                const int rc = launch(k_fp4_amax<T>, dim3((unsigned)a.amax_blocks), kQThreads, 0, st, 0, 0, a, static_cast<uint32_t*>(workspace));
                if (rc != SBC_OK) return rc;
            }
            return launch_quantise<T, SBC_FP4_E4M3>(a, along_rows, along_cols, (unsigned)(row_tiles * col_tiles), st);
        }
        return launch_quantise<T, SBC_FP4_E8M0>(a, along_rows, along_cols, (unsigned)(row_tiles * col_tiles), st);
    });
}

int sbc_fp4_dequantise(const sbc_fp4* q, void* out, int dtype, int64_t row_stride, sbc_cuda_stream_t stream) {
    if (!fp4_ok(q) || !matrix_ok(out, dtype, q->rows, q->cols, row_stride)) return SBC_EINVAL;
    DequantiseArgs a = {};
    a.values = static_cast<const uint8_t*>(q->values);
    a.scales = static_cast<const uint8_t*>(q->scales);
    a.tensor = q->tensor_scale;
    a.out = out;
    a.rows = q->rows;
    a.cols = q->cols;
    a.stride = row_stride;
    a.pitch = (long long)sbc_fp4_row_bytes(q->cols);
    a.ktiles = ktiles_of(q->cols, q->format);
    const int64_t blocks = std::min<int64_t>(pieces(q->rows, q->cols, false), sm_count() * 8);
    return by_dtype(dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        const bool shift = row_align(out, row_stride, width_of(dtype)) < 16, e4m3 = q->format == SBC_FP4_E4M3;
        const auto kernel = shift ? (e4m3 ? k_fp4_dequantise<T, SBC_FP4_E4M3, true> : k_fp4_dequantise<T, SBC_FP4_E8M0, true>)
                                  : (e4m3 ? k_fp4_dequantise<T, SBC_FP4_E4M3, false> : k_fp4_dequantise<T, SBC_FP4_E8M0, false>);
        return launch(kernel, dim3((unsigned)blocks), kQThreads, 0, stream, 0, 0, a);
    });
}

int sbc_fp4_product(const sbc_fp4* a, const sbc_fp4* b, void* out, int dtype, int64_t row_stride, uint32_t* status,
                    sbc_cuda_stream_t stream) {
    if (!fp4_ok(a) || !fp4_ok(b) || a->format != b->format || a->cols != b->cols) return SBC_EINVAL;
    if (a->rows > kMaxDim - 512 || b->rows > kMaxDim - 512) return SBC_EINVAL;
    if (!matrix_ok(out, dtype, a->rows, b->rows, row_stride) || !aligned(status, 4)) return SBC_EINVAL;
    // This kernel holds 128 tokens.  us of 128 here / there: 8192^2 13.6 / 18.8, 1300 -> 2600 7.3 / 6.9, 2048^2 8.5 / 8.1,
    // 4096 -> 16384 13.7 / 12.4, 16384 -> 4096 15.2 / 31.9, 650 -> 10000 6.0 / 6.1: three shapes would gain up to 1.3 us
    // there, one would take twice as long; of 64 never slower here.  128 here, 129 there: 8192^2 13.3, 19.5;
    // 16384 -> 4096 15.0, 32.0 (few tiles, long columns, which are not split there); 4096 -> 16384 13.3, 15.4
    if (a->rows > 128) return product_wide(a, b, out, dtype, row_stride, status, stream);
    ProductArgs p = {};
    p.scales_w = static_cast<const uint8_t*>(b->scales);
    p.scales_x = static_cast<const uint8_t*>(a->scales);
    p.tensor_w = b->tensor_scale;
    p.tensor_x = a->tensor_scale;
    p.out = out;
    p.status = status;
    p.rows_w = b->rows;
    p.rows_x = a->rows;
    p.stride = row_stride;
    p.ktiles = ktiles_of(a->cols, a->format);
    p.chunks = (int)ceil_div(a->cols, 256);
    p.steps = (int)ceil_div(a->cols, 64);
    p.nt = (int)ceil_div(a->rows, 16) * 16;
    const int tiles_k = a->format == SBC_FP4_E8M0 ? 2 : 4;
    const int stage = (kPRows * kPBytes + p.nt * kPBytes + tiles_k * 512 * 2 + 1023) / 1024 * 1024;
    p.stages = std::min(4, 110 * 1024 / stage);
    const int cols = (p.nt + 31) / 32 * 32 + p.stages * 4 * tiles_k * 2;
    p.tmem_cols = 32;
    while ((int)p.tmem_cols < cols) p.tmem_cols *= 2;
    // as many blocks on an SM as its tensor memory serves, so that none waits for another's columns
    const int smem = std::max(p.stages * stage + 1024, kSmemMost / (512 / (int)p.tmem_cols + 1) + 1024);
    const int64_t tiles_w = ceil_div(b->rows, kPRows);
    // the columns in parts: up to a block per SM while a part has one stage, up to two while it has two (us of
    // 16 tokens in one part / so many: 8192^2 23.8 / 9.9, 1024^2 4.8 / 4.1; 650 -> 10000, two blocks per SM
    // of one stage or two 5.5, one 4.4; four blocks per SM: 8192^2 14.2)
    int parts = 1;
    while (parts < 8) {
        const int64_t blocks = tiles_w * parts * 2;
        if (blocks > 2 * sm_count() || p.chunks < parts * (blocks <= sm_count() ? 2 : 4)) break;
        parts *= 2;
    }
    CUtensorMap mw, mx;
    if (!values_map(&mw, b, kPRows) || !values_map(&mx, a, p.nt)) return SBC_ECUDA;
    const dim3 grid((unsigned)tiles_w, (unsigned)parts);
    return by_dtype(dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        return a->format == SBC_FP4_E4M3 ? launch_product<T, SBC_FP4_E4M3>(mw, mx, p, grid, smem, stream)
                                         : launch_product<T, SBC_FP4_E8M0>(mw, mx, p, grid, smem, stream);
    });
}

int sbc_top_logits(const void* logits, int dtype, int64_t rows, int64_t cols, int64_t row_stride, int k, float temperature,
                   float* values, int32_t* indices, float* rest, sbc_cuda_stream_t stream) {
    if (!width_of(dtype) || rows < 0 || rows > kMaxDim / 8 || cols < 1 || cols > kMaxDim) return SBC_EINVAL;
    if (k < 1 || k > std::min<int64_t>(cols, SBC_TOP_MOST) || !temperature_ok(temperature)) return SBC_EINVAL;
    if (rows == 0) return SBC_OK;
    if (!matrix_ok(logits, dtype, rows, cols, row_stride)) return SBC_EINVAL;
    if (!values || !indices || !rest || !aligned(values, 4) || !aligned(indices, 4) || !aligned(rest, 4)) return SBC_EINVAL;
    TopArgs a = {logits, rows, row_stride, (int)cols, k, 0, 0, temperature, values, indices, rest};
    return by_dtype(dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        const RowPlan p = plan_rows(rows, cols, (int)sizeof(T));
        a.shift = p.shift;
        // many rows that would take four blocks each: 2048 x 131072 bfloat16 232 us streamed, 299 us in clusters
        // (65536: 133 and 132, 32000: 84 and 59)
        if (rows >= sm_count() && cols * (int64_t)sizeof(T) > 2 * kRoomBytes) {
            a.room = kStreamRoom;
            return launch(k_top_stream<T>, dim3((unsigned)rows), kStreamThreads, 2 * kStreamBytes + (size_t)a.room * kCandidateBytes, stream, 0, 0, a);
        }
        // enough groups of elements that the k-th largest of their maxima bounds tightly: two a thread, four times k
        const int threads = std::max(p.threads, std::min(kTopThreads, (int)ceil_div(2 * k, 32 * p.size) * 32));
        a.room = candidate_room(k, p.size);
        const size_t lists = (size_t)a.room * kCandidateBytes;
        const dim3 grid((unsigned)(rows * p.size));
        if (ceil_div(ceil_div(cols, 64), p.size) * 64 > p.room) {   // too long to be held
            return launch(k_top_logits<T, false>, grid, kTopThreads, lists, stream, p.size, 0, a);
        }
        if (!allow_smem<k_top_logits<T, true>>(kRoomBytes + 32 + candidate_room(SBC_TOP_MOST, 8) * kCandidateBytes)) return (int)SBC_ECUDA;
        return launch(k_top_logits<T, true>, grid, threads, lists + (size_t)p.room * sizeof(T) + 32, stream, p.size, 0, a);
    });
}

int sbc_distill_loss(const void* logits, int dtype, int64_t rows, int64_t cols, int64_t row_stride, const sbc_distill* d, float* loss,
                     float* stats, uint32_t* status, sbc_cuda_stream_t stream) {
    if (!distill_ok(d, rows, cols) || !width_of(dtype)) return SBC_EINVAL;
    if (rows == 0) return SBC_OK;
    if (!matrix_ok(logits, dtype, rows, cols, row_stride) || !loss || !aligned(loss, 4) || !aligned(stats, 16) || !aligned(status, 4))
        return SBC_EINVAL;
    DistillArgs a = distill_args(logits, rows, cols, row_stride, d);
    a.loss = loss;
    a.stats = stats;
    a.status = status;
    return distill_by_type<false>(a, dtype, stream);
}

int sbc_distill_grad(const void* logits, int dtype, int64_t rows, int64_t cols, int64_t row_stride, const sbc_distill* d,
                     const float* stats, const float* grad_loss, void* grad, int64_t grad_stride, sbc_cuda_stream_t stream) {
    if (!distill_ok(d, rows, cols) || !width_of(dtype)) return SBC_EINVAL;
    if (rows == 0) return SBC_OK;
    if (!matrix_ok(logits, dtype, rows, cols, row_stride) || !matrix_ok(grad, dtype, rows, cols, grad_stride) || !stats ||
        !aligned(stats, 16) || !aligned(grad_loss, 4))
        return SBC_EINVAL;
    DistillArgs a = distill_args(logits, rows, cols, row_stride, d);
    a.stats = const_cast<float*>(stats);
    a.grad_loss = grad_loss;
    a.grad = grad;
    a.grad_stride = grad_stride;
    return by_dtype(dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        const RowPlan p = plan_rows(rows, cols, (int)sizeof(T));
        const int size = p.size, threads = p.threads;
        const size_t smem = (size_t)a.k * 12;
        a.shift = p.shift;
        const auto kernel = second_exponential(a) ? k_distill_grad<T, true> : k_distill_grad<T, false>;
        return launch(kernel, dim3((unsigned)(rows * size)), threads, smem, stream, 0, 0, a);
    });
}

int sbc_distill_loss_grad(const void* logits, int dtype, int64_t rows, int64_t cols, int64_t row_stride, const sbc_distill* d,
                          const float* grad_loss, float* loss, void* grad, int64_t grad_stride, uint32_t* status,
                          sbc_cuda_stream_t stream) {
    if (!distill_ok(d, rows, cols) || !width_of(dtype)) return SBC_EINVAL;
    if (rows == 0) return SBC_OK;
    if (!matrix_ok(logits, dtype, rows, cols, row_stride) || !matrix_ok(grad, dtype, rows, cols, grad_stride) || !loss ||
        !aligned(loss, 4) || !aligned(grad_loss, 4) || !aligned(status, 4))
        return SBC_EINVAL;
    DistillArgs a = distill_args(logits, rows, cols, row_stride, d);
    a.loss = loss;
    a.grad_loss = grad_loss;
    a.grad = grad;
    a.grad_stride = grad_stride;
    a.status = status;
    return distill_by_type<true>(a, dtype, stream);
}

}  // extern "C"
