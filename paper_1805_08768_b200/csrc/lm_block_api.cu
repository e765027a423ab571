// C entry points of the operators of a client's own layers (include/sbc_block.h).
#include "../../include/sbc_block.h"

#include "lm_adapter.cuh"
#include "lm_dropout.cuh"
#include "lm_gated.cuh"
#include "lm_host.cuh"
#include "lm_norm.cuh"

using namespace sbclm;

namespace {

bool weights_ok(const void* p, int weight_dtype, int dtype) {
    return (weight_dtype == SBC_F32 || weight_dtype == dtype) && aligned(p, (uintptr_t)width_of(weight_dtype));
}

// How rows are shared out: threads that hold a row (0: longer rows than they hold), granules a thread, groups a block.
struct NormPlan {
    int group, granules, groups;
    int64_t blocks;
};

// Backward.  `moved`: rows may begin off a multiple of 16 bytes and then touch one granule more.  Two blocks an SM stay, the
// same number whatever the alignment (the sums of blocks have room by it).
NormPlan plan_norm_grad(int64_t rows, int64_t cols, bool moved) {
    NormPlan p = {};
    const int64_t n = ceil_div(cols + (moved ? 7 : 0), 8), most = std::max<int64_t>(8, sm_count() * 2);
    p.granules = n > 256 ? 2 : 1;
    if (n > (int64_t)kNormThreads * p.granules) {
        p.blocks = std::min(rows, std::min<int64_t>(most, std::max<int64_t>(1, ((int64_t)1 << 25) / cols)));
        return p;
    }
    p.group = (int)ceil_div(n, 32 * p.granules) * 32;
    p.groups = std::max(1, 256 / p.group);
    // rows of a group are a multiple of eight rows apart
    p.blocks = std::min(ceil_div(ceil_div(rows, p.groups), 8) * 8, most / 8 * 8);
    return p;
}

// Forward: as few threads a row as hold it, but enough rows or threads of one for the GPU.
NormPlan plan_norm(int64_t rows, int64_t cols, bool moved, int width) {
    NormPlan p = {};
    const int64_t n = ceil_div(cols + (moved ? 7 : 0), 8), most_granules = 16 / width;
    int64_t group = 32;
    while (group < kNormThreads && (n > group * most_granules || (rows * group < (int64_t)sm_count() * 512 && n > group))) group *= 2;
    if (n > group * most_granules || n * 64 > 96 * 1024) {   // (the weights leave room for two blocks on an SM)
        p.blocks = std::min<int64_t>(rows, std::max(8, sm_count() * 2));
        return p;
    }
    p.granules = 1;
    while (p.granules < ceil_div(n, group)) p.granules *= 2;
    p.group = (int)group;
    p.groups = std::max(1, 256 / p.group);
    // a block's rows are eight apart
    p.blocks = std::min(ceil_div(ceil_div(rows, p.groups), 8) * 8, (int64_t)std::max(8, sm_count() * 2) / 8 * 8);
    return p;
}

template <auto Kernel> int launch_norm(const NormArgs& a, const NormPlan& p, int smem, cudaStream_t st) {
    if (!allow_smem<Kernel>(200 * 1024)) return SBC_ECUDA;
    return launch(Kernel, dim3((unsigned)p.blocks), p.group * p.groups, (size_t)smem, st, 0, 0, a);
}

bool moved(const void* p, int64_t stride, int width) { return row_align(p, stride, width) < 16; }

// ---- gated block ----

constexpr int64_t kGatedMost = kMaxDim - 512;

bool gated_ok(const sbc_gated_weights* w) {
    return w && (w->dtype == SBC_BF16 || w->dtype == SBC_F16) && w->act >= SBC_ACT_SILU && w->act <= SBC_ACT_SIGMOID && w->hidden >= 1 &&
           w->hidden <= kGatedMost && w->inner >= 1 && w->inner <= kGatedMost && matrix_ok(w->gate, w->dtype, w->hidden, w->inner, w->gate_stride) &&
           matrix_ok(w->up, w->dtype, w->hidden, w->inner, w->up_stride);
}

// A matrix as the tensor maps take it.
struct Laid {
    const void* p;
    int64_t stride;
};

// Parts of a workspace, one behind the other.
struct Room {
    uint8_t* base;
    size_t used = 0;
    void* take(int64_t bytes) {
        void* p = base ? base + used : nullptr;
        used += (size_t)((bytes + 255) / 256 * 256);
        return p;
    }
};

// What of x and the weights has to be copied, where to, and the copy's arguments.
struct GatedLayout {
    Laid x, gate, up;
    void *dg = nullptr, *du = nullptr;
    int64_t d_stride = 0;
    LayArgs lay = {};
    int copies = 0;
    int64_t most_groups = 0;
    size_t bytes = 0;
};

bool few_tokens(int64_t tokens, bool keep) { return tokens <= kFMost && !keep; }

GatedLayout gated_layout(const sbc_gated_weights* w, int64_t tokens, const void* x, int64_t x_stride, bool grad, void* workspace) {
    GatedLayout l;
    Room room = {static_cast<uint8_t*>(workspace)};
    const auto lay = [&](const void* p, int64_t rows, int64_t stride) -> Laid {
        if (!moved(p, rows > 1 ? stride : 8, 2)) return {p, rows > 1 ? stride : ceil_div(w->inner, 8) * 8};
        const int64_t to_stride = ceil_div(w->inner, 8) * 8;
        void* to = room.take(rows * to_stride * 2);
        l.lay.from[l.copies] = p;
        l.lay.to[l.copies] = to;
        l.lay.rows[l.copies] = rows;
        l.lay.stride[l.copies] = stride;
        l.lay.to_stride[l.copies] = to_stride;
        l.lay.cols[l.copies] = (int)w->inner;
        l.lay.align[l.copies] = row_align(p, stride, 2);
        l.most_groups = std::max(l.most_groups, rows * to_stride / 8);
        ++l.copies;
        return {to, to_stride};
    };
    l.x = lay(x, tokens, x_stride);
    l.gate = lay(w->gate, w->hidden, w->gate_stride);
    l.up = lay(w->up, w->hidden, w->up_stride);
    if (grad) {
        l.d_stride = ceil_div(w->hidden, 8) * 8;
        l.dg = room.take(tokens * l.d_stride * 2);
        l.du = room.take(tokens * l.d_stride * 2);
    }
    l.bytes = room.used;
    return l;
}

// Boxes of `across` elements (64: a swizzle line) x `rows` of a matrix of 16-bit elements.
bool half_map(CUtensorMap* map, const Laid& m, int64_t rows, int64_t cols, int box_rows) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)m.stride * 2};
    const cuuint32_t box[2] = {kMBytes / 2, (cuuint32_t)box_rows}, ones[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(m.p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles of 256 columns, or of 128 where those take no more rounds of the pairs (a round of 256 counted as 1.6 of 128).
bool wide_columns(int64_t tiles_m, int64_t columns, int outputs) {
    const int64_t pairs = std::max(1, sm_count() / 2);
    return 16 * ceil_div(tiles_m * outputs * ceil_div(columns, 256), pairs) <= 10 * ceil_div(tiles_m * outputs * ceil_div(columns, 128), pairs);
}

template <typename T, typename O, int MODE, int NT>
int launch_mm(const CUtensorMap& r, const CUtensorMap& r2, const CUtensorMap& c, const CUtensorMap& c2, MmArgs a, int64_t tiles, cudaStream_t st) {
    if (tiles > kMaxDim / 2) return SBC_EINVAL;
    a.tiles = (int)tiles;
    const int stage = (128 + NT / 2) * kMBytes;
    constexpr int swap = MODE == kForward || MODE == kForwardKeep ? kMSwap : 0;
    a.stages = std::min(kMStages, (kSmemMost - 2 * 1024 - swap) / stage);
    if (!allow_smem<k_mm<T, O, MODE, NT>>(kSmemMost - 1024)) return SBC_ECUDA;
    const unsigned blocks = (unsigned)(2 * std::min<int64_t>(std::max(1, sm_count() / 2), tiles));
    // (always more than half of an SM's shared memory: a block takes up to all of its tensor memory)
    return launch(k_mm<T, O, MODE, NT>, dim3(blocks), kMThreads, (size_t)(a.stages * stage + swap + 1024), st, 2, 0, r, r2, c, c2, a);
}

template <typename T> int lay_rows(const GatedLayout& l, cudaStream_t st) {
    if (!l.copies) return SBC_OK;
    const int64_t blocks = std::min<int64_t>(ceil_div(l.most_groups, kGThreads), (int64_t)sm_count() * 8);
    return launch(k_lay_rows<T>, dim3((unsigned)blocks, (unsigned)l.copies), kGThreads, 0, st, 0, 0, l.lay);
}

template <typename T, int MODE> int gated_forward(const sbc_gated_weights* w, const GatedLayout& l, int64_t tokens, MmArgs a, cudaStream_t st) {
    a.rows_m = w->hidden;
    a.rows_n = tokens;
    a.chunks = (int)ceil_div(w->inner, 64);
    a.sources = 1;
    a.tiles_m = (int)ceil_div(w->hidden, 128);
    const bool wide = wide_columns(a.tiles_m, tokens, 1);
    a.tiles_n = (int)ceil_div(tokens, wide ? 256 : 128);
    CUtensorMap r, r2, c;
    if (!half_map(&r, l.gate, w->hidden, w->inner, 64) || !half_map(&r2, l.up, w->hidden, w->inner, 64) ||
        !half_map(&c, l.x, tokens, w->inner, wide ? 128 : 64))
        return SBC_ECUDA;
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
    return wide ? launch_mm<T, T, MODE, 256>(r, r2, c, c, a, tiles, st) : launch_mm<T, T, MODE, 128>(r, r2, c, c, a, tiles, st);
}

template <typename T> int gated_input_grad(const sbc_gated_weights* w, const GatedLayout& l, int64_t tokens, void* dx, int64_t stride, uint32_t* status, cudaStream_t st) {
    MmArgs a = {};
    a.out = dx;
    a.out_stride = stride;
    a.status = status;
    a.rows_m = w->inner;
    a.rows_n = tokens;
    a.chunks = (int)ceil_div(w->hidden, 64);
    a.sources = 2;
    a.tiles_m = (int)ceil_div(w->inner, 256);
    const bool wide = wide_columns(a.tiles_m, tokens, 1);
    a.tiles_n = (int)ceil_div(tokens, wide ? 256 : 128);
    CUtensorMap r, r2, c, c2;
    const int box = wide ? 128 : 64;
    if (!half_map(&r, l.gate, w->hidden, w->inner, 64) || !half_map(&r2, l.up, w->hidden, w->inner, 64) ||
        !half_map(&c, {l.dg, l.d_stride}, tokens, w->hidden, box) || !half_map(&c2, {l.du, l.d_stride}, tokens, w->hidden, box))
        return SBC_ECUDA;
    const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
    return wide ? launch_mm<T, T, kInputGrad, 256>(r, r2, c, c2, a, tiles, st) : launch_mm<T, T, kInputGrad, 128>(r, r2, c, c2, a, tiles, st);
}

template <typename T, typename O>
int gated_weight_grad(const sbc_gated_weights* w, const GatedLayout& l, int64_t tokens, void* dgate, void* dup, int64_t stride, uint32_t* status, cudaStream_t st) {
    MmArgs a = {};
    a.out = dgate;
    a.out2 = dup;
    a.out_stride = stride;
    a.status = status;
    a.rows_m = w->inner;
    a.rows_n = w->hidden;
    a.chunks = (int)ceil_div(tokens, 64);
    a.sources = 1;
    a.tiles_m = (int)ceil_div(w->inner, 256);
    const bool wide = wide_columns(a.tiles_m, w->hidden, 2);
    a.tiles_n = (int)ceil_div(w->hidden, wide ? 256 : 128);
    CUtensorMap r, c, c2;
    if (!half_map(&r, l.x, tokens, w->inner, 64) || !half_map(&c, {l.dg, l.d_stride}, tokens, w->hidden, 64) ||
        !half_map(&c2, {l.du, l.d_stride}, tokens, w->hidden, 64))
        return SBC_ECUDA;
    const int64_t tiles = 2ll * a.tiles_m * a.tiles_n;
    return wide ? launch_mm<T, O, kWeightGrad, 256>(r, r, c, c2, a, tiles, st) : launch_mm<T, O, kWeightGrad, 128>(r, r, c, c2, a, tiles, st);
}

template <typename T, int TT> int launch_few(const FewArgs& a, cudaStream_t st) {
    // two tiles of units share the tokens' registers where the tokens' bytes would otherwise pass the weights'
    constexpr int UT = TT > 1 ? 2 : 1;
    return launch(k_gated_few<T, TT, UT>, dim3((unsigned)ceil_div(a.hidden, 8 * UT)), kFThreads, 0, st, 0, 0, a);
}

template <typename F> int by_half(int dtype, F f) { return dtype == SBC_BF16 ? f((__nv_bfloat16*)nullptr) : f((__half*)nullptr); }

// ---- adapters ----

constexpr int64_t kAdapterWide = (int64_t)1 << 30, kAdapterTokens = (int64_t)1 << 24;

bool adapters_ok(const sbc_adapters* w, int dtype) {
    return w && w->down && w->up && width_of(dtype) && (w->dtype == SBC_F32 || w->dtype == dtype) && w->count >= 1 && w->count <= SBC_ADAPTER_COUNT &&
           w->rank >= 1 && w->rank <= SBC_ADAPTER_RANK && w->inner >= 1 && w->inner <= kAdapterWide && w->outer >= 1 && w->outer <= kAdapterWide &&
           w->reserved == 0 && aligned(w->down, (uintptr_t)width_of(w->dtype)) && aligned(w->up, (uintptr_t)width_of(w->dtype));
}

int64_t most_tiles(int64_t tokens, int64_t count) { return tokens / kATile + std::min(count + 1, tokens); }

AdapterPlan plan_at(const void* plan, int64_t tokens, int64_t count) {
    AdapterPlan p;
    p.tiles = static_cast<int4*>(const_cast<void*>(plan));
    p.offsets = reinterpret_cast<int*>(p.tiles + 1 + most_tiles(tokens, count));
    p.order = p.offsets + count + 2;
    return p;
}

// (type of the tokens, type of the adapters) -> element types
template <typename F> int by_types(int dtype, int weights, F f) {
    return by_dtype(dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        if (weights == SBC_F32) return f(as, (float*)nullptr);
        return f(as, (T*)nullptr);
    });
}

template <typename F> int by_vec(bool vec, F f) { return vec ? f(std::true_type()) : f(std::false_type()); }

// Blocks of a cluster that share a sum, while there are fewer pieces of work than `most` blocks; each has at least `least` of `length`.
int shares(int64_t pieces, int64_t most, int64_t length, int64_t least) {
    int parts = 1;
    while (parts < 8 && pieces * parts * 2 <= most && length >= least * parts * 2) parts *= 2;
    return parts;
}

template <typename T, typename W, int JT> int launch_in(AdapterArgs a, int64_t tiles, cudaStream_t st) {
    using S = InShape<T, W, JT>;
    const int64_t blocks = ceil_div(a.rank, 8 * JT);
    a.parts = shares(tiles * blocks, 2 * sm_count(), a.wide, 256);
    return by_vec(a.wide % 8 == 0 && a.align_x >= 16 && a.align_factor >= 16, [&](auto vec) {
        constexpr auto kernel = k_adapter_in<T, W, JT, decltype(vec)::value>;
        if (!allow_smem<kernel>(S::kSmem)) return (int)SBC_ECUDA;
        return launch(kernel, dim3((unsigned)(tiles * a.parts), (unsigned)blocks), kAThreads, S::kSmem, st, a.parts, 0, a);
    });
}

// mid = scale x factor^T
int adapter_in(AdapterArgs a, int dtype, int weights, int64_t tokens, cudaStream_t st) {
    a.align_x = row_align(a.x, a.x_stride, width_of(dtype));
    a.align_factor = row_align(a.factor, a.wide, width_of(weights));
    const int64_t tiles = most_tiles(tokens, a.count);
    return by_types(dtype, weights, [&](auto* t, auto* w) {
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(w)>;
        return a.rank <= 8 ? launch_in<T, W, 1>(a, tiles, st) : a.rank <= 16 ? launch_in<T, W, 2>(a, tiles, st)
             : a.rank <= 32 ? launch_in<T, W, 4>(a, tiles, st) : launch_in<T, W, 8>(a, tiles, st);
    });
}

template <typename T, typename W, int CB> int launch_out(const AdapterArgs& a, int64_t tiles, bool vec, cudaStream_t st) {
    using S = OutShape<T, W, CB>;
    constexpr int largest = std::min(SBC_ADAPTER_RANK, CB == 256 ? 128 / S::Y / 16 * 16 : SBC_ADAPTER_RANK);
    static_assert(S::smem(largest) <= S::kMost, "a block's shared memory");
    // about two blocks an SM, each with a run of the tiles
    const int64_t columns = ceil_div(a.wide, CB), runs = std::min<int64_t>(tiles, std::max<int64_t>(1, (int64_t)sm_count() * 2 / columns));
    return by_vec(vec, [&](auto v) {
        constexpr auto kernel = k_adapter_out<T, W, CB, decltype(v)::value>;
        if (!allow_smem<kernel>(S::kMost)) return (int)SBC_ECUDA;
        return launch(kernel, dim3((unsigned)columns, (unsigned)runs), kAThreads, (size_t)S::smem(a.rank), st, 0, 0, a);
    });
}

// out = base + scale mid factor
int adapter_out(AdapterArgs a, int dtype, int weights, int64_t tokens, cudaStream_t st) {
    const int width = width_of(dtype);
    a.align_base = a.base ? row_align(a.base, a.base_stride, width) : 16;
    a.align_out = row_align(a.out, a.out_stride, width);
    a.align_factor = row_align(a.factor, a.wide, width_of(weights));
    const int64_t tiles = most_tiles(tokens, a.count);
    return by_types(dtype, weights, [&](auto* t, auto* w) {
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(w)>;
        // the factor's terms leave two blocks of 16-bit ones on an SM, and fit one block otherwise
        constexpr int terms = OutShape<T, W, 256>::Y;
        const bool vec = a.wide % 8 == 0 && a.align_base >= 16 && a.align_out >= 16 && a.align_factor >= 16;
        return terms * sixteens(a.rank) <= 128 ? launch_out<T, W, 256>(a, tiles, vec, st) : launch_out<T, W, 128>(a, tiles, vec, st);
    });
}

template <typename T, typename W, int RT, int RH, bool VEC> int launch_adapter_grad(AdapterGradArgs a, int64_t tokens, cudaStream_t st) {
    using S = GradShape<T, W, RT, RH, VEC>;
    static_assert(S::kSmem <= kSmemMost - 4096, "a block's shared memory");
    const int64_t rows = ceil_div(a.rank, S::kRows) * a.count;
    int64_t blocks[2];
    for (int i = 0; i < 2; ++i) blocks[i] = a.sums[i].out ? rows * (a.sums[i].columns = (int)ceil_div(a.sums[i].wide, kAThreads * 2)) : 0;
    if (blocks[0] + blocks[1] > kMaxDim / 8) return SBC_EINVAL;
    constexpr auto kernel = k_adapter_grad<T, W, RT, RH, VEC>;
    if (!allow_smem<kernel>(S::kSmem)) return SBC_ECUDA;
    // adapters differ in their tokens: about two blocks for each that an SM holds
    a.parts = shares(blocks[0] + blocks[1], 2 * sm_count(), tokens, 64);
    a.first = (int)(blocks[0] * a.parts);
    return launch(kernel, dim3((unsigned)((blocks[0] + blocks[1]) * a.parts)), S::kThreads, S::kSmem, st, a.parts, 0, a);
}

// out = scale mid^T x of one sum or both
int adapter_grad(AdapterGradArgs a, int dtype, int weights, int64_t tokens, cudaStream_t st) {
    for (AdapterSum& s : a.sums) {
        s.align_x = row_align(s.x, s.x_stride, width_of(dtype));
        s.align_out = row_align(s.out, s.wide, width_of(weights));
    }
    return by_types(dtype, weights, [&](auto* t, auto* w) {
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(w)>;
        const auto vec_one = [&](const AdapterSum& s) { return !s.out || (s.align_x >= 16 && s.wide % 8 == 0); };
        return by_vec(vec_one(a.sums[0]) && vec_one(a.sums[1]), [&](auto vec) {
            constexpr bool v = decltype(vec)::value;
            return a.rank <= 16 ? launch_adapter_grad<T, W, 1, 1, v>(a, tokens, st) : a.rank <= 32 ? launch_adapter_grad<T, W, 2, 1, v>(a, tokens, st)
                                                                                                    : launch_adapter_grad<T, W, 2, 2, v>(a, tokens, st);
        });
    });
}

}  // namespace

extern "C" {

int sbc_layer_norm(const void* x, int dtype, int64_t rows, int64_t cols, int64_t x_stride, const void* weight, const void* bias,
                   int weight_dtype, float eps, void* y, int64_t y_stride, float* stats, sbc_cuda_stream_t stream) {
    if (!width_of(dtype) || rows < 0 || rows > kMaxDim || cols < 1 || cols > kMaxDim || !(eps >= 0.f) || eps > 3.4e38f) return SBC_EINVAL;
    if (!weights_ok(weight, weight_dtype, dtype) || !weights_ok(bias, weight_dtype, dtype) || !aligned(stats, 8)) return SBC_EINVAL;
    if (rows == 0) return SBC_OK;
    if (!matrix_ok(x, dtype, rows, cols, x_stride) || !matrix_ok(y, dtype, rows, cols, y_stride)) return SBC_EINVAL;
    NormArgs a = {};
    a.x = x;
    a.out = y;
    a.weight = weight;
    a.bias = bias;
    a.weight_f32 = weight_dtype == SBC_F32;
    a.stats = reinterpret_cast<float2*>(stats);
    a.rows = rows;
    a.cols = (int)cols;
    a.x_stride = x_stride;
    a.out_stride = y_stride;
    a.eps = eps;
    const NormPlan p = plan_norm(rows, cols, moved(x, x_stride, width_of(dtype)), width_of(dtype));
    a.group = p.group;
    a.groups = p.groups;
    return by_dtype(dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        if (!p.group) return launch(k_norm_long<T>, dim3((unsigned)p.blocks), kNormLong, 0, stream, 0, 0, a);
        const int smem = (int)ceil_div(cols + 7, 8) * 64;
        if constexpr (sizeof(T) == 2)
            if (p.granules == 8) return launch_norm<k_norm<T, 8>>(a, p, smem, stream);
        return p.granules == 1 ? launch_norm<k_norm<T, 1>>(a, p, smem, stream) : p.granules == 2 ? launch_norm<k_norm<T, 2>>(a, p, smem, stream)
                                                                                                  : launch_norm<k_norm<T, 4>>(a, p, smem, stream);
    });
}

size_t sbc_layer_norm_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || rows > kMaxDim || cols < 1 || cols > kMaxDim) return 0;
    const int64_t blocks = std::max(plan_norm_grad(rows, cols, false).blocks, plan_norm_grad(rows, cols, true).blocks);
    return (size_t)(ceil_div(blocks * 2 * cols * 4, 16) * 16 + 16);
}

int sbc_layer_norm_grad(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, int dtype, int64_t rows, int64_t cols,
                        const float* stats, const void* weight, int weight_dtype, void* dx, int64_t dx_stride, void* dweight,
                        void* dbias, void* workspace, size_t workspace_bytes, sbc_cuda_stream_t stream) {
    if (!width_of(dtype) || rows < 0 || rows > kMaxDim || cols < 1 || cols > kMaxDim) return SBC_EINVAL;
    if (!weights_ok(weight, weight_dtype, dtype) || !weights_ok(dweight, weight_dtype, dtype) || !weights_ok(dbias, weight_dtype, dtype))
        return SBC_EINVAL;
    const bool sums = dweight || dbias;
    if (!dx && !sums) return SBC_EINVAL;
    if (rows > 0 && (!matrix_ok(x, dtype, rows, cols, x_stride) || !matrix_ok(dy, dtype, rows, cols, dy_stride) ||
                     (dx && !matrix_ok(dx, dtype, rows, cols, dx_stride)) || !stats || !aligned(stats, 8)))
        return SBC_EINVAL;
    if (sums && (!workspace || !aligned(workspace, 16))) return SBC_EINVAL;
    if (sums && workspace_bytes < sbc_layer_norm_workspace_bytes(rows, cols)) return SBC_ECAPACITY;
    NormArgs a = {};
    a.x = x;
    a.dy = dy;
    a.out = dx;
    a.weight = weight;
    a.weight_f32 = weight_dtype == SBC_F32;
    a.stats = reinterpret_cast<float2*>(const_cast<float*>(stats));
    a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    a.rows = rows;
    a.cols = (int)cols;
    a.x_stride = x_stride;
    a.dy_stride = dy_stride;
    a.out_stride = dx_stride;
    const NormPlan p = plan_norm_grad(rows, cols, moved(x, x_stride, width_of(dtype)));
    a.group = p.group;
    a.groups = p.groups;
    if (rows > 0) {
        const int rc = by_dtype(dtype, [&](auto* as) {
            using T = std::remove_pointer_t<decltype(as)>;
            if (!p.group) return launch(k_norm_grad_long<T>, dim3((unsigned)p.blocks), kNormLong, 0, stream, 0, 0, a);
            const int smem = sums && p.groups > 1 ? (int)cols * 8 : 0;
            return p.granules == 1 ? launch_norm<k_norm_grad<T, 1>>(a, p, smem, stream) : launch_norm<k_norm_grad<T, 2>>(a, p, smem, stream);
        });
        if (rc != SBC_OK) return rc;
    }
    if (!sums) return SBC_OK;
    NormSumArgs s = {a.partial, dweight, dbias, (int)cols, rows > 0 ? (int)p.blocks : 0, weight_dtype};
    return launch(k_norm_sum, dim3((unsigned)ceil_div(2 * cols, kNormSumCols)), kNormSumCols * kNormSumRows, 0, stream, 0, 0, s);
}

int sbc_dropout(const void* x, int dtype, int64_t rows, int64_t cols, int64_t x_stride, const void* residual, int64_t residual_stride,
                double p, const int64_t* rng, int64_t at, void* out, int64_t out_stride, sbc_cuda_stream_t stream) {
    if (!width_of(dtype) || rows < 0 || rows > kMaxDim || cols < 1 || cols > kMaxDim) return SBC_EINVAL;
    if (!(p >= 0.0 && p <= 1.0) || at < 0 || at > (int64_t)1 << 62 || !rng || !aligned(rng, 8)) return SBC_EINVAL;
    if (rows == 0) return SBC_OK;
    if (!matrix_ok(x, dtype, rows, cols, x_stride) || !matrix_ok(out, dtype, rows, cols, out_stride) ||
        (residual && !matrix_ok(residual, dtype, rows, cols, residual_stride)))
        return SBC_EINVAL;
    DropoutArgs a = {};
    a.x = x;
    a.residual = residual;
    a.out = out;
    a.rng = reinterpret_cast<const long long*>(rng);
    a.rows = rows;
    a.cols = cols;
    a.x_stride = x_stride;
    a.residual_stride = residual_stride;
    a.out_stride = out_stride;
    a.groups = ceil_div(rows * cols, 8);
    a.at = (unsigned long long)at;
    a.dropped = (unsigned)std::llrint(65536.0 * p);
    a.scale = a.dropped < 65536 ? (float)(65536.0 / (65536 - a.dropped)) : 0.f;
    const auto flat_one = [&](const void* m, int64_t stride) { return !m || (aligned(m, 16) && (rows == 1 || stride == cols)); };
    const bool flat = flat_one(x, x_stride) && flat_one(residual, residual_stride) && flat_one(out, out_stride);
    const int64_t blocks = std::min<int64_t>(ceil_div(a.groups, kDropThreads), (int64_t)sm_count() * 8 * 4);
    return by_dtype(dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        return launch(flat ? k_dropout<T, true> : k_dropout<T, false>, dim3((unsigned)blocks), kDropThreads, 0, stream, 0, 0, a);
    });
}

size_t sbc_gated_kept_bytes(int64_t tokens, int64_t hidden) {
    if (tokens < 0 || tokens > kGatedMost || hidden < 1 || hidden > kGatedMost) return 0;
    return (size_t)tokens * (size_t)(ceil_div(hidden, 2) * 16);
}

size_t sbc_gated_workspace_bytes(const sbc_gated_weights* w, int64_t tokens, const void* x, int64_t x_stride, int keep, int grad) {
    if (!gated_ok(w) || tokens < 1 || tokens > kGatedMost || (!grad && few_tokens(tokens, keep != 0))) return 0;
    return gated_layout(w, tokens, x, x_stride, grad != 0, nullptr).bytes;
}

int sbc_gated(const sbc_gated_weights* w, const void* x, int64_t tokens, int64_t x_stride, void* h, int64_t h_stride, float* kept,
              void* workspace, size_t workspace_bytes, uint32_t* status, sbc_cuda_stream_t stream) {
    if (!gated_ok(w) || tokens < 0 || tokens > kGatedMost || !aligned(kept, 16) || !aligned(status, 4)) return SBC_EINVAL;
    if (tokens == 0) return SBC_OK;
    if (!matrix_ok(x, w->dtype, tokens, w->inner, x_stride) || !matrix_ok(h, w->dtype, tokens, w->hidden, h_stride)) return SBC_EINVAL;
    if (few_tokens(tokens, kept != nullptr)) {
        FewArgs a = {};
        a.x = x;
        a.gate = w->gate;
        a.up = w->up;
        a.h = h;
        a.x_stride = x_stride;
        a.gate_stride = w->gate_stride;
        a.up_stride = w->up_stride;
        a.h_stride = h_stride;
        a.hidden = w->hidden;
        a.inner = (int)w->inner;
        a.tokens = (int)tokens;
        a.act = w->act;
        a.align_x = row_align(x, tokens > 1 ? x_stride : 8, 2);
        a.align_w = std::min(row_align(w->gate, w->gate_stride, 2), row_align(w->up, w->up_stride, 2));
        return by_half(w->dtype, [&](auto* as) {
            using T = std::remove_pointer_t<decltype(as)>;
            return tokens <= 8 ? launch_few<T, 1>(a, stream) : tokens <= 16 ? launch_few<T, 2>(a, stream) : launch_few<T, 4>(a, stream);
        });
    }
    const GatedLayout l = gated_layout(w, tokens, x, x_stride, false, workspace);
    if (l.bytes && (!workspace || !aligned(workspace, 16))) return SBC_EINVAL;
    if (workspace_bytes < l.bytes) return SBC_ECAPACITY;
    MmArgs a = {};
    a.out = h;
    a.out_stride = h_stride;
    a.kept = reinterpret_cast<float2*>(kept);
    a.kept_stride = ceil_div(w->hidden, 2) * 2;
    a.status = status;
    a.act = w->act;
    return by_half(w->dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        const int rc = lay_rows<T>(l, stream);
        if (rc != SBC_OK) return rc;
        return kept ? gated_forward<T, kForwardKeep>(w, l, tokens, a, stream) : gated_forward<T, kForward>(w, l, tokens, a, stream);
    });
}

int sbc_gated_grad(const sbc_gated_weights* w, const void* x, int64_t tokens, int64_t x_stride, const void* dh, int64_t dh_stride,
                   const float* kept, void* dx, int64_t dx_stride, void* dgate, void* dup, int grad_dtype, int64_t grad_stride,
                   void* workspace, size_t workspace_bytes, uint32_t* status, sbc_cuda_stream_t stream) {
    if (!gated_ok(w) || tokens < 0 || tokens > kGatedMost || !aligned(status, 4)) return SBC_EINVAL;
    if ((!dx && !dgate) || !dgate != !dup) return SBC_EINVAL;
    if (dgate && ((grad_dtype != SBC_F32 && grad_dtype != w->dtype) || !matrix_ok(dgate, grad_dtype, w->hidden, w->inner, grad_stride) ||
                  !matrix_ok(dup, grad_dtype, w->hidden, w->inner, grad_stride)))
        return SBC_EINVAL;
    if (tokens == 0) {
        if (!dgate) return SBC_OK;
        const size_t width = (size_t)width_of(grad_dtype);
        for (void* p : {dgate, dup})
            if (cudaMemset2DAsync(p, (size_t)grad_stride * width, 0, (size_t)w->inner * width, (size_t)w->hidden, stream) != cudaSuccess) return SBC_ECUDA;
        return SBC_OK;
    }
    if (!matrix_ok(x, w->dtype, tokens, w->inner, x_stride) || !matrix_ok(dh, w->dtype, tokens, w->hidden, dh_stride) ||
        (dx && !matrix_ok(dx, w->dtype, tokens, w->inner, dx_stride)) || !kept || !aligned(kept, 16))
        return SBC_EINVAL;
    const GatedLayout l = gated_layout(w, tokens, x, x_stride, true, workspace);
    if (!workspace || !aligned(workspace, 16)) return SBC_EINVAL;
    if (workspace_bytes < l.bytes) return SBC_ECAPACITY;
    return by_half(w->dtype, [&](auto* as) {
        using T = std::remove_pointer_t<decltype(as)>;
        int rc = lay_rows<T>(l, stream);
        if (rc != SBC_OK) return rc;
        GateGradArgs g = {};
        g.dh = dh;
        g.kept = reinterpret_cast<const float2*>(kept);
        g.dg = l.dg;
        g.du = l.du;
        g.rows = tokens;
        g.dh_stride = dh_stride;
        g.kept_stride = ceil_div(w->hidden, 2) * 2;
        g.d_stride = l.d_stride;
        g.cols = (int)w->hidden;
        g.align_dh = row_align(dh, tokens > 1 ? dh_stride : 8, 2);
        const int64_t blocks = std::min<int64_t>(ceil_div(tokens * ceil_div(w->hidden, 8), kGThreads), (int64_t)sm_count() * 8);
        rc = launch(k_gate_grad<T>, dim3((unsigned)blocks), kGThreads, 0, stream, 0, 0, g);
        if (rc == SBC_OK && dx) rc = gated_input_grad<T>(w, l, tokens, dx, dx_stride, status, stream);
        if (rc == SBC_OK && dgate)
            rc = grad_dtype == SBC_F32 ? gated_weight_grad<T, float>(w, l, tokens, dgate, dup, grad_stride, status, stream)
                                       : gated_weight_grad<T, T>(w, l, tokens, dgate, dup, grad_stride, status, stream);
        return rc;
    });
}

size_t sbc_adapter_mid_bytes(int64_t tokens, int64_t rank) {
    if (tokens < 0 || tokens > kAdapterTokens || rank < 1 || rank > SBC_ADAPTER_RANK) return 0;
    return (size_t)tokens * (size_t)sixteens((int)rank) * 6;
}

size_t sbc_adapter_plan_bytes(int64_t tokens, int64_t count) {
    if (tokens < 0 || tokens > kAdapterTokens || count < 1 || count > SBC_ADAPTER_COUNT) return 0;
    return (size_t)(ceil_div(16 * (1 + most_tiles(tokens, count)) + 4 * (count + 2 + tokens), 16) * 16);
}

int sbc_adapter_plan(const int32_t* ids, int64_t tokens, int64_t count, void* plan, size_t plan_bytes, uint32_t* status, sbc_cuda_stream_t stream) {
    if (tokens < 0 || tokens > kAdapterTokens || count < 1 || count > SBC_ADAPTER_COUNT || !aligned(status, 4)) return SBC_EINVAL;
    if (!plan || !aligned(plan, 16) || (tokens > 0 && (!ids || !aligned(ids, 4)))) return SBC_EINVAL;
    if (plan_bytes < sbc_adapter_plan_bytes(tokens, count)) return SBC_ECAPACITY;
    constexpr int kRoom = 200 * 1024;
    PlanArgs a = {ids, plan_at(plan, tokens, count), status, (int)tokens, (int)count, 0};
    // a warp has at least 64 tokens, and counters for all adapters
    a.warps = (int)std::max<int64_t>(1, std::min<int64_t>({kAPlanThreads / 32, kRoom / (4 * (count + 1)), ceil_div(tokens, 64)}));
    if (!allow_smem<k_adapter_plan>(kRoom)) return SBC_ECUDA;
    return launch(k_adapter_plan, dim3(1), kAPlanThreads, (size_t)a.warps * (size_t)(count + 1) * 4, stream, 0, 0, a);
}

int sbc_adapter(const sbc_adapters* w, const void* x, int dtype, int64_t tokens, int64_t x_stride, const int32_t* ids, const void* plan,
                float scale, const void* base, int64_t base_stride, void* out, int64_t out_stride, void* mid, uint32_t* status,
                sbc_cuda_stream_t stream) {
    if (!adapters_ok(w, dtype) || tokens < 0 || tokens > kAdapterTokens || !aligned(status, 4)) return SBC_EINVAL;
    if (tokens == 0) return SBC_OK;
    if (!matrix_ok(x, dtype, tokens, w->inner, x_stride) || !matrix_ok(out, dtype, tokens, w->outer, out_stride) ||
        (base && !matrix_ok(base, dtype, tokens, w->outer, base_stride)))
        return SBC_EINVAL;
    if (plan ? (!aligned(plan, 16) || !mid || !aligned(mid, 16)) : (!ids || !aligned(ids, 4) || tokens > SBC_ADAPTER_FEW || mid)) return SBC_EINVAL;
    if (!plan) {
        AdapterFewArgs a = {};
        a.x = x;
        a.down = w->down;
        a.up = w->up;
        a.base = base;
        a.out = out;
        a.ids = ids;
        a.status = status;
        a.x_stride = x_stride;
        a.base_stride = base_stride;
        a.out_stride = out_stride;
        a.count = (int)w->count;
        a.rank = (int)w->rank;
        a.inner = (int)w->inner;
        a.outer = (int)w->outer;
        a.scale = scale;
        a.align_x = row_align(x, tokens > 1 ? x_stride : 8, width_of(dtype));
        a.align_down = row_align(w->down, w->inner, width_of(w->dtype));
        a.pairs = w->outer % 2 == 0 && aligned(w->up, (uintptr_t)(2 * width_of(w->dtype)));
        a.parts = shares(tokens, 4 * sm_count(), std::min(w->inner, w->outer), 128);
        return by_types(dtype, w->dtype, [&](auto* t, auto* ws) {
            using T = std::remove_pointer_t<decltype(t)>;
            using W = std::remove_pointer_t<decltype(ws)>;
            return launch(k_adapter_few<T, W>, dim3((unsigned)(tokens * a.parts)), kAFewThreads, 0, stream, a.parts, 0, a);
        });
    }
    AdapterArgs a = {};
    a.plan = plan_at(plan, tokens, w->count);
    a.count = (int)w->count;
    a.rank = (int)w->rank;
    a.mid = static_cast<uint16_t*>(mid);
    a.tokens = (int)tokens;
    a.x = x;
    a.x_stride = x_stride;
    a.factor = w->down;
    a.wide = (int)w->inner;
    a.scale = 1.f;
    const int rc = adapter_in(a, dtype, w->dtype, tokens, stream);
    if (rc != SBC_OK) return rc;
    a.factor = w->up;
    a.wide = (int)w->outer;
    a.base = base;
    a.base_stride = base_stride;
    a.out = out;
    a.out_stride = out_stride;
    a.scale = scale;
    return adapter_out(a, dtype, w->dtype, tokens, stream);
}

int sbc_adapter_grad(const sbc_adapters* w, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, int dtype, int64_t tokens,
                     const void* plan, const void* mid, float scale, const void* base, int64_t base_stride, void* dx, int64_t dx_stride,
                     void* ddown, void* dup, void* dmid, sbc_cuda_stream_t stream) {
    if (!adapters_ok(w, dtype) || tokens < 0 || tokens > kAdapterTokens || (!dx && !ddown && !dup)) return SBC_EINVAL;
    const int width = width_of(w->dtype);
    if (!aligned(ddown, (uintptr_t)width) || !aligned(dup, (uintptr_t)width)) return SBC_EINVAL;
    if (tokens == 0) {
        if (ddown && cudaMemsetAsync(ddown, 0, (size_t)(w->count * w->rank * w->inner) * width, stream) != cudaSuccess) return SBC_ECUDA;
        if (dup && cudaMemsetAsync(dup, 0, (size_t)(w->count * w->rank * w->outer) * width, stream) != cudaSuccess) return SBC_ECUDA;
        return SBC_OK;
    }
    if (!matrix_ok(dy, dtype, tokens, w->outer, dy_stride) || (ddown && !matrix_ok(x, dtype, tokens, w->inner, x_stride)) ||
        (dx && !matrix_ok(dx, dtype, tokens, w->inner, dx_stride)) || (dx && base && !matrix_ok(base, dtype, tokens, w->inner, base_stride)) ||
        !plan || !aligned(plan, 16) || (dup && (!mid || !aligned(mid, 16))) || ((dx || ddown) && (!dmid || !aligned(dmid, 16))))
        return SBC_EINVAL;
    AdapterArgs a = {};
    a.plan = plan_at(plan, tokens, w->count);
    a.count = (int)w->count;
    a.rank = (int)w->rank;
    int rc = SBC_OK;
    if (dx || ddown) {
        a.mid = static_cast<uint16_t*>(dmid);
        a.tokens = (int)tokens;
        a.x = dy;
        a.x_stride = dy_stride;
        a.factor = w->up;
        a.wide = (int)w->outer;
        a.scale = scale;
        rc = adapter_in(a, dtype, w->dtype, tokens, stream);
    }
    if (rc == SBC_OK && dx) {
        a.factor = w->down;
        a.wide = (int)w->inner;
        a.base = base;
        a.base_stride = base_stride;
        a.out = dx;
        a.out_stride = dx_stride;
        a.scale = 1.f;
        rc = adapter_out(a, dtype, w->dtype, tokens, stream);
    }
    if (rc == SBC_OK && (ddown || dup)) {
        AdapterGradArgs g = {};
        g.plan = a.plan;
        g.tokens = (int)tokens;
        g.count = a.count;
        g.rank = a.rank;
        g.sums[0] = {x, static_cast<const uint16_t*>(dmid), ddown, x_stride, (int)w->inner, 0, 0, 0, 1.f};
        g.sums[1] = {dy, static_cast<const uint16_t*>(mid), dup, dy_stride, (int)w->outer, 0, 0, 0, scale};
        rc = adapter_grad(g, dtype, w->dtype, tokens, stream);
    }
    return rc;
}

}  // extern "C"
