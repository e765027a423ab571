/*
 * sbc_lm.h -- operators for clients that train a language model between two
 * rounds of Sparse Binary Compression.  Exported by the same shared library as
 * sbc.h, whose conventions for pointers, streams and return values hold here:
 * the caller owns every buffer, work is enqueued on `stream` and not waited
 * for, what the host can see to be wrong is refused before anything is
 * enqueued, and no kernel traps.
 *
 * What a client of a round receives and learns from, next to what it sends:
 *   - weights in 4-bit floating point with a scale per block (the server's
 *     message in 4.25 or 4.5 bits per weight), multiplied as they are:
 *     sbc_fp4_quantise, sbc_fp4_dequantise, sbc_fp4_product;
 *   - a teacher's k largest logits per position and the mass of all the
 *     others: sbc_top_logits;
 *   - the loss against such a message and its gradient: sbc_distill_loss,
 *     sbc_distill_grad, sbc_distill_loss_grad.
 *
 * Matrices are row-major with their last dimension contiguous; `row_stride` is
 * the distance of two rows in elements (>= the number of columns).
 */
#ifndef SBC_LM_H
#define SBC_LM_H

#include "sbc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of matrices (sums and softmax statistics are 32 bits whatever the type). */
#define SBC_F32 0
#define SBC_BF16 1
#define SBC_F16 2

/* ---- 4-bit floating point ------------------------------------------------ */

/*
 * An element is a sign and an index into {0, 0.5, 1, 1.5, 2, 3, 4, 6}; it
 * stands for grid value * block scale * tensor scale.  Blocks are runs of a
 * row (the axis a product contracts).
 *
 *   SBC_FP4_E8M0  blocks of 32, block scale 2^e, tensor scale 1:
 *                 e = floor(log2(largest magnitude of the block)) - 2
 *   SBC_FP4_E4M3  blocks of 16, block scale an 8-bit float (4 exponent and 3
 *                 fraction bits), tensor scale 2^g:
 *                 g = floor(log2(largest finite magnitude of the tensor)) - 10,
 *                 scale = nearest(largest magnitude of the block / 6 / 2^g)
 *
 * Elements and block scales round to nearest, ties to the even code, elements
 * beyond 6 to 6.  The tensor scale is a power of two, so every decision falls
 * as it would in exact arithmetic.  A block that holds an infinity or a NaN
 * gets the scale's NaN code and stands for NaNs; it does not enter g.  Where an
 * E4M3 scale rounds to zero the block stands for zeros.
 *
 * Layout: nibble i % 2 (low one first) of byte i / 2 of a row holds element i;
 * rows are sbc_fp4_row_bytes(cols) apart, a multiple of 16; the nibbles from
 * cols on are zero.  The scale of row r, block b is byte
 *   (r % 32) * 16 + (r % 128 / 32) * 4 + b % 4
 * of the 512-byte tile (r / 128) * ceil(blocks / 4) + b / 4; the scales of rows
 * and blocks that do not exist are zero bytes.  This is the order in which the
 * tensor cores take scales, so a product copies tiles as they are.
 */
#define SBC_FP4_E8M0 0
#define SBC_FP4_E4M3 1

typedef struct sbc_fp4 {
    void *values;        /* device, rows * sbc_fp4_row_bytes(cols) bytes, 16-byte aligned */
    void *scales;        /* device, sbc_fp4_scale_bytes(rows, cols, format) bytes, 16-byte aligned */
    float *tensor_scale; /* device, one float */
    int64_t rows, cols;  /* each 1 .. 2^31-1 */
    int32_t format;      /* SBC_FP4_* */
    int32_t reserved;    /* 0 */
} sbc_fp4;

/* Bytes of a row's elements, of all scales, and of the scratch that
 * sbc_fp4_quantise needs.  Host only; 0 on bad arguments. */
size_t sbc_fp4_row_bytes(int64_t cols);
size_t sbc_fp4_scale_bytes(int64_t rows, int64_t cols, int format);
size_t sbc_fp4_workspace_bytes(int64_t rows, int64_t cols, int format);

/*
 * Quantise x (rows x cols) along its rows, along its columns, or both in one
 * reading.
 *
 * x           device, dtype, rows `row_stride` elements apart
 * along_rows  receives x (rows x cols); may be NULL
 * along_cols  receives the transpose (cols x rows: its blocks run down the
 *             columns of x), what a backward product contracts; may be NULL
 *             (but not both).  Both get the same tensor scale.
 * workspace   device, 16-byte aligned, sbc_fp4_workspace_bytes(...) bytes
 */
int sbc_fp4_quantise(const void *x, int dtype, int64_t rows, int64_t cols, int64_t row_stride,
                     const sbc_fp4 *along_rows, const sbc_fp4 *along_cols, void *workspace,
                     size_t workspace_bytes, sbc_cuda_stream_t stream);

/* out (rows x cols, dtype) = the values that q stands for. */
int sbc_fp4_dequantise(const sbc_fp4 *q, void *out, int dtype, int64_t row_stride, sbc_cuda_stream_t stream);

/*
 * out[i, j] = sum_k a[i, k] * b[j, k]   (a.rows x b.rows, dtype), products and
 * sums in 32 bits on the tensor cores, rounded once at the end.
 *
 * a  activations: rows are tokens; b  weights: rows are output channels (each
 *    at most 2^31-513 rows).  Both of the same format and the same cols.  The
 *    kernel reads whole weights and as many token rows as there are, so few
 *    tokens cost the weights' bytes.
 * status  device, one uint32 (may be NULL): SBC_STATUS_TIMEOUT is or-ed in if a
 *    bounded device-side wait gave up; the affected outputs are then NaN.
 */
int sbc_fp4_product(const sbc_fp4 *a, const sbc_fp4 *b, void *out, int dtype, int64_t row_stride,
                    uint32_t *status, sbc_cuda_stream_t stream);

/* ---- a teacher's message ------------------------------------------------- */

#define SBC_TOP_MOST 256          /* most logits of a row that sbc_top_logits selects */
#define SBC_DISTILL_MOST 1024     /* most logits of a row that a loss takes */
#define SBC_DISTILL_COLS (1 << 20) /* most columns that a loss takes */
#define SBC_DISTILL_STATS 8       /* floats per row that sbc_distill_loss leaves for sbc_distill_grad */

/*
 * The k largest logits of every row and the mass of the others:
 *   values[r, 0..k), indices[r, 0..k)  in descending order, the lower index
 *                                      first among equals (-0 equals +0)
 *   rest[r] = log sum_{j not sent} exp(logits[r, j] / temperature), -inf if
 *             nothing (or nothing but -inf) is left, +inf if a +inf is
 * Logits of -inf (words ruled out) are sent only where fewer than k others
 * exist.  NaN orders above everything and makes the row's rest NaN if it is
 * not sent.  If a bounded device-side wait gave up, rest is NaN and the row's
 * values and indices say nothing.
 *
 * logits  device, dtype, rows x cols; rows may be 0
 * k       1 .. min(cols, SBC_TOP_MOST); temperature 1e-6 .. 1e6
 * values float, indices int32: device, rows x k;  rest: device, rows floats
 */
int sbc_top_logits(const void *logits, int dtype, int64_t rows, int64_t cols, int64_t row_stride, int k,
                   float temperature, float *values, int32_t *indices, float *rest, sbc_cuda_stream_t stream);

/*
 * What a student is taught, per row:
 *   teacher  p = softmax over (values[r, :] / temperature, rest[r])
 *   student  q = softmax(logits[r, :] / temperature); q_rest its mass outside
 *            the sent words
 *   loss[r] = alpha * temperature^2 * KL(p || q over the same outcomes)
 *           + (1 - alpha) * cross entropy of softmax(logits[r, :]) and labels[r]
 * A row whose teacher has no mass, or whose logits are all -inf, has neither
 * term of that kind; a row without a label has no cross entropy.  A slot of
 * negative index is not used.  Indices of a row differ from each other.  An
 * index or label >= cols is ignored and SBC_STATUS_RANGE or-ed into status.
 *
 * values   device, rows x k floats
 * indices  device, rows x k int32
 * rest     device, rows floats, or NULL: no mass outside (renormalised over k)
 * labels   device, rows int64, negative: none; or NULL
 */
typedef struct sbc_distill {
    const float *values;
    const int32_t *indices;
    const float *rest;
    const int64_t *labels;
    int32_t k;         /* 1 .. SBC_DISTILL_MOST */
    float temperature; /* 1e-6 .. 1e6 */
    float alpha;       /* 0 .. 1 */
    int32_t reserved;  /* 0 */
} sbc_distill;

/* Forward: loss (rows floats) and, unless NULL, stats (rows x SBC_DISTILL_STATS
 * floats, 16-byte aligned) for the backward call.  status: device, one uint32,
 * or NULL; SBC_STATUS_TIMEOUT is or-ed in if a bounded device-side wait gave
 * up, what it was for is then NaN. */
int sbc_distill_loss(const void *logits, int dtype, int64_t rows, int64_t cols, int64_t row_stride,
                     const sbc_distill *d, float *loss, float *stats, uint32_t *status, sbc_cuda_stream_t stream);

/* Backward: grad[r, j] = grad_loss[r] * d loss[r] / d logits[r, j] (dtype of the
 * logits, rows grad_stride apart; may be the logits themselves).  grad_loss:
 * device, rows floats, or NULL: ones.  stats: what sbc_distill_loss left for
 * the same logits and the same d. */
int sbc_distill_grad(const void *logits, int dtype, int64_t rows, int64_t cols, int64_t row_stride,
                     const sbc_distill *d, const float *stats, const float *grad_loss, void *grad,
                     int64_t grad_stride, sbc_cuda_stream_t stream);

/* Both in one reading of the logits, where grad_loss is known beforehand. */
int sbc_distill_loss_grad(const void *logits, int dtype, int64_t rows, int64_t cols, int64_t row_stride,
                          const sbc_distill *d, const float *grad_loss, float *loss, void *grad,
                          int64_t grad_stride, uint32_t *status, sbc_cuda_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* SBC_LM_H */
