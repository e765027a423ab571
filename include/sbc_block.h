/*
 * sbc_block.h -- operators of the layers that a client trains between two
 * rounds of Sparse Binary Compression, next to those of sbc_lm.h and exported
 * by the same shared library, with the same conventions: the caller owns every
 * buffer, work is enqueued on `stream` and not waited for, what the host can
 * see to be wrong is refused before anything is enqueued, and no kernel traps.
 *
 *   sbc_layer_norm, sbc_layer_norm_grad   normalisation of rows, there and back
 *   sbc_dropout                           dropout into a residual; no mask is kept
 *   sbc_gated, sbc_gated_grad             gated feed-forward block, there and back
 *   sbc_adapter, sbc_adapter_grad         low-rank adapters of many clients or
 *                                         requests beside a shared projection
 *
 * Matrices are row-major with their last dimension contiguous; a stride is the
 * distance of two rows in elements (>= the number of columns).  dtype is
 * SBC_F32, SBC_BF16 or SBC_F16.  Outputs may not overlap inputs except where a
 * call says so.
 */
#ifndef SBC_BLOCK_H
#define SBC_BLOCK_H

#include "sbc_lm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- layer norm ------------------------------------------------------------ */

/*
 * y[r, :] = (x[r, :] - mean) / sqrt(variance + eps) * weight + bias, mean and
 * variance (divided by cols) of the row in 32 bits, rounded once at the end.
 *
 * weight, bias  device, cols values of weight_dtype (SBC_F32 or dtype), each may
 *               be NULL (ones, zeros)
 * eps           finite, >= 0
 * y             device, dtype; may be x with x's stride
 * stats         device, 8-byte aligned, rows pairs (mean, 1 / sqrt(variance + eps)),
 *               which sbc_layer_norm_grad takes; may be NULL
 * rows          may be 0
 */
int sbc_layer_norm(const void *x, int dtype, int64_t rows, int64_t cols, int64_t x_stride, const void *weight,
                   const void *bias, int weight_dtype, float eps, void *y, int64_t y_stride, float *stats,
                   sbc_cuda_stream_t stream);

/* Scratch that sbc_layer_norm_grad needs for gradients of the weight or bias.  Host only; 0 on bad arguments. */
size_t sbc_layer_norm_workspace_bytes(int64_t rows, int64_t cols);

/*
 * With h = (x - mean) * rstd and t = dy * weight:
 *   dx      = rstd * (t - mean(t) - h * mean(t * h))   (dtype)
 *   dweight = sum over rows of dy * h,  dbias = sum over rows of dy   (weight_dtype)
 * each rounded once; sums are taken in 32 bits and in an order that depends on
 * the sizes alone.  dx may be dy or x with that one's stride.
 *
 * stats       what sbc_layer_norm left for the same x
 * dx, dweight, dbias  each may be NULL (not all); with no rows, dweight and dbias are zeros
 * workspace   device, 16-byte aligned, sbc_layer_norm_workspace_bytes(rows, cols)
 *             bytes; may be NULL where dweight and dbias are
 */
int sbc_layer_norm_grad(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, int dtype, int64_t rows,
                        int64_t cols, const float *stats, const void *weight, int weight_dtype, void *dx,
                        int64_t dx_stride, void *dweight, void *dbias, void *workspace, size_t workspace_bytes,
                        sbc_cuda_stream_t stream);

/* ---- dropout ------------------------------------------------------------------ */

/*
 * out = residual + (kept ? x * 65536 / (65536 - d) : 0),  d = 65536 p rounded to
 * a whole number, in 32 bits and rounded once.  The same call on the output's
 * gradient, without a residual, is the backward pass.
 *
 * Element n of the matrix (n = row * cols + column, whatever the strides) is
 * kept if its 16 random bits, as a number, are at least d.  The bits are those
 * of Philox-4x32-10 with key rng[0] and counter (n / 8 + at, rng[1]), 64 bits
 * each, low words first: half n % 2 (low one first) of word n % 8 / 2.
 *
 * p         0 .. 1; at 1 nothing is kept.  What is dropped does not count, even
 *           if it is not finite.
 * rng       device, 8-byte aligned, two int64: the key and a step.  They are read
 *           when the kernel runs, so a captured call draws anew once the step
 *           has been raised.
 * at        0 .. 2^62: where in a step's numbers this matrix begins, in groups
 *           of eight; layers that share rng are ceil(rows * cols / 8) apart
 * residual  device, dtype, or NULL
 * out       device, dtype; may be x or the residual with that one's stride
 */
int sbc_dropout(const void *x, int dtype, int64_t rows, int64_t cols, int64_t x_stride, const void *residual,
                int64_t residual_stride, double p, const int64_t *rng, int64_t at, void *out, int64_t out_stride,
                sbc_cuda_stream_t stream);

/* ---- gated feed-forward block ------------------------------------------------- */

#define SBC_ACT_SILU 0      /* g / (1 + exp(-g)) */
#define SBC_ACT_GELU 1      /* g * (the normal distribution's share below g) */
#define SBC_ACT_GELU_TANH 2 /* its approximation by a hyperbolic tangent */
#define SBC_ACT_RELU 3      /* max(g, 0) */
#define SBC_ACT_SIGMOID 4   /* 1 / (1 + exp(-g)) */

/* Both projections' weights, hidden x inner each, SBC_BF16 or SBC_F16 like everything they meet. */
typedef struct sbc_gated_weights {
    const void *gate, *up;            /* device */
    int64_t gate_stride, up_stride;
    int64_t hidden, inner;            /* each 1 .. 2^31-513 */
    int32_t dtype;
    int32_t act;                      /* SBC_ACT_* */
} sbc_gated_weights;

/* Bytes of what a forward call keeps for the backward one: a pair of floats per token and hidden unit, rows in whole
 * pairs.  Host only; 0 on bad arguments. */
size_t sbc_gated_kept_bytes(int64_t tokens, int64_t hidden);

/* Scratch of a call with these operands (0: none): copies of matrices whose rows do not begin at multiples of 16 bytes
 * where the kernels need that; for `grad` the two factors' gradients, too.  Host only. */
size_t sbc_gated_workspace_bytes(const sbc_gated_weights *w, int64_t tokens, const void *x, int64_t x_stride, int keep,
                                 int grad);

/*
 * h[t, :] = act(x[t, :] gate^T) * (x[t, :] up^T), products and sums in 32 bits,
 * rounded once.
 *
 * x     device, tokens x inner; tokens may be 0
 * h     device, tokens x hidden
 * kept  device, 16-byte aligned, sbc_gated_kept_bytes(...) bytes, or NULL: what
 *       sbc_gated_grad takes
 * workspace  device, 16-byte aligned, sbc_gated_workspace_bytes(..., kept != NULL, 0) bytes; may be NULL where that is 0
 * status     device, one uint32 (may be NULL): SBC_STATUS_TIMEOUT is or-ed in if a
 *            bounded device-side wait gave up; the affected outputs are then NaN
 */
int sbc_gated(const sbc_gated_weights *w, const void *x, int64_t tokens, int64_t x_stride, void *h, int64_t h_stride,
              float *kept, void *workspace, size_t workspace_bytes, uint32_t *status, sbc_cuda_stream_t stream);

/*
 * Backward: with g, u the two projections, dg = dh u act'(g) and du = dh act(g),
 * each rounded to the weights' type,
 *   dx    = dg gate + du up                       (tokens x inner, the weights' type)
 *   dgate = dg^T x,  dup = du^T x                 (hidden x inner, grad_dtype: SBC_F32 or the weights' type)
 * sums in 32 bits.  (Float16 dg and du have that type's range: a loss is scaled for
 * them as for dh.)  With no tokens, dgate and dup are zeros.
 *
 * kept   what sbc_gated left for the same x and w
 * dx, dgate and dup  each may be NULL (not all; dgate and dup both or neither, rows grad_stride apart)
 * workspace  as above, sbc_gated_workspace_bytes(..., 0, 1)
 */
int sbc_gated_grad(const sbc_gated_weights *w, const void *x, int64_t tokens, int64_t x_stride, const void *dh,
                   int64_t dh_stride, const float *kept, void *dx, int64_t dx_stride, void *dgate, void *dup,
                   int grad_dtype, int64_t grad_stride, void *workspace, size_t workspace_bytes, uint32_t *status,
                   sbc_cuda_stream_t stream);

/* ---- low-rank adapters ---------------------------------------------------------- */

#define SBC_ADAPTER_RANK 128   /* largest rank */
#define SBC_ADAPTER_FEW 64     /* most tokens of a call without a plan */
#define SBC_ADAPTER_COUNT 32768 /* most adapters */

/* `count` adapters, one behind the other without gaps: down [count][rank][inner], up [count][rank][outer] (the usual
 * out x rank factor transposed, so both factors' rows are a rank's). */
typedef struct sbc_adapters {
    const void *down, *up;   /* device, dtype */
    int64_t count;           /* 1 .. SBC_ADAPTER_COUNT */
    int64_t rank;            /* 1 .. SBC_ADAPTER_RANK */
    int64_t inner, outer;    /* each 1 .. 2^30 */
    int32_t dtype;           /* SBC_F32, or the type of the tokens */
    int32_t reserved;        /* 0 */
} sbc_adapters;

/*
 * The tokens of a batch grouped by their adapters, for all layers that the
 * batch goes through.
 *
 * ids     device, tokens int32: each token's adapter, negative: none.  In any
 *         order.  One >= count counts as none, and SBC_STATUS_RANGE is or-ed
 *         into status (device, one uint32, or NULL).
 * tokens  0 .. 2^24
 * plan    device, 16-byte aligned, sbc_adapter_plan_bytes(tokens, count) bytes
 */
size_t sbc_adapter_plan_bytes(int64_t tokens, int64_t count);
int sbc_adapter_plan(const int32_t *ids, int64_t tokens, int64_t count, void *plan, size_t plan_bytes,
                     uint32_t *status, sbc_cuda_stream_t stream);

/* Bytes of x down_i^T for a batch.  Host only; 0 on bad arguments. */
size_t sbc_adapter_mid_bytes(int64_t tokens, int64_t rank);

/*
 * out[t, :] = base[t, :] + scale * (x[t, :] down_i^T) up_i,  i = ids[t]; sums in
 * 32 bits, rounded once.  x and down are taken with all of their bits, and
 * x down_i^T to 24 bits.  A call with a plan leaves out what is below 2^-21 of a
 * product's magnitude or, in products that end as 16-bit results, 2^-14; so does
 * sbc_adapter_grad.
 * Infinities and NaNs are those of the formula.  Tokens without an adapter get
 * base[t, :] as it is.
 *
 * x     device, dtype, tokens x inner
 * plan  of the batch, made for `count` adapters, or NULL: then ids are read
 *       (at most SBC_ADAPTER_FEW tokens, and mid is NULL).  With a plan ids may be NULL.
 * base  device, dtype, tokens x outer: what the shared projection gave; NULL: zeros
 * out   device, dtype; may be base with base's stride
 * mid   with a plan: device, 16-byte aligned, sbc_adapter_mid_bytes(tokens, rank) bytes for
 *       x down_i^T, which sbc_adapter_grad takes (each value as three bfloat16 whose sum it is:
 *       [3][tokens][rank in whole sixteens]; rows of tokens without an adapter are
 *       undefined).  Otherwise NULL.
 * status  device, one uint32, or NULL: as above, where ids are read
 */
int sbc_adapter(const sbc_adapters *w, const void *x, int dtype, int64_t tokens, int64_t x_stride, const int32_t *ids,
                const void *plan, float scale, const void *base, int64_t base_stride, void *out, int64_t out_stride,
                void *mid, uint32_t *status, sbc_cuda_stream_t stream);

/*
 * Backward:
 *   dmid = scale * dy up_i^T,  dx = base + dmid down_i        (dtype)
 *   ddown_i = sum over i's tokens of dmid^T x,  dup_i = scale * sum of mid^T dy   (the adapters' type)
 * An adapter without tokens gets zeros.  Sums over tokens are taken in an order
 * that the ids alone give.
 *
 * mid    what sbc_adapter left for the same x, w and plan
 * base   device, dtype, tokens x inner: the input's gradient through the shared
 *        projection; NULL: zeros
 * dx, ddown, dup  each may be NULL (not all); dx may be base with base's stride
 * dmid   device, 16-byte aligned, sbc_adapter_mid_bytes(tokens, rank) bytes of scratch
 */
int sbc_adapter_grad(const sbc_adapters *w, const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, int dtype,
                     int64_t tokens, const void *plan, const void *mid, float scale, const void *base,
                     int64_t base_stride, void *dx, int64_t dx_stride, void *ddown, void *dup, void *dmid,
                     sbc_cuda_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* SBC_BLOCK_H */
