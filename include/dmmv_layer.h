/*
 * A quantised linear layer after its codes have been found: the operators with which it is trained
 * and served.
 *
 *   dmmv_layernorm            the norm in front of the layer; writes its result in the input's type,
 *   dmmv_layernorm_backward   in 8 bits (the operand of the product), or both, and an 8-bit
 *                             checkpoint of its input for the backward pass
 *   dmmv_block_quantize       a matrix in 8 bits: the checkpoint of an activation, trained weights
 *   dmmv_block_dequantize     and back
 *   dmmv_block_product        y = x w^T + bias of two such matrices
 *   dmmv_block_backward       its gradients, from the checkpoint of x
 *
 * An 8-bit matrix ("block matrix") holds codes in the e4m3 format of the OCP 8-bit floating-point
 * specification (no infinities, largest value 448, 0x7F and 0xFF are NaN) and a scale for each
 * block of 128 columns:
 *
 *     value(i, j) = e4m3(codes[i * ld + j])
 *                   * scales[(i / scale_rows) * scale_row_stride + (j / 128) * scale_block_stride]
 *
 * scale_rows is 1 (a row's block has its own scale: activations) or 128 (128 x 128 blocks: weights).
 * Scales are powers of two in one byte (DMMV_E8M0: 2^(byte - 127), 255 is NaN) or any floats
 * (DMMV_F32).  A stride of 0 repeats a scale: a layer solved by dmmv_solve with integer levels of
 * magnitude at most 16 is a block matrix whose codes are those integers and whose scale is the
 * row's (scale_rows 1, row stride 1, block stride 0).
 *
 * Conventions are those of dmmv.h: plain C, DEVICE pointers owned by the caller, nothing allocated,
 * all work enqueued on the given hipStream_t (NULL = the default stream) without waiting, statuses
 * and dmmv_last_error().  Matrices are row-major with a row stride >= the columns, any alignment
 * their element type allows; 16-byte aligned rows are the fast ones.  Inputs and outputs do not
 * overlap.  Empty matrices are allowed.  Sums are held in 32 bits (what bf16 products of 8-bit matrices lose on the
 * way there stands at dmmv_block_product), in an order that sizes, types and alignments fix: equal calls give equal
 * bits.  NaN and infinities of the inputs stay visible in what depends on them.
 */
#ifndef DMMV_LAYER_H
#define DMMV_LAYER_H

#include "dmmv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types beside DMMV_F32 (no operator of this header takes DMMV_F64). */
enum { DMMV_BF16 = 2, DMMV_E8M0 = 3 };

typedef struct {
    int64_t rows, cols;
    void* codes;                 /* [rows][ld] e4m3                                               */
    int64_t ld;                  /* >= cols                                                       */
    void* scales;                /* of scale_type, or NULL (all 1; not as an output)              */
    int64_t scale_row_stride;    /* in elements; 0 repeats a scale (not as an output)             */
    int64_t scale_block_stride;
    int32_t scale_type;          /* DMMV_E8M0 or DMMV_F32                                         */
    int32_t scale_rows;          /* 1 or 128                                                      */
} dmmv_block_matrix;

/* q <- x [rows][ldx] of dtype DMMV_F32 or DMMV_BF16, rows and columns as q says.  With a the largest
 * |x| of a block's finite values, its scale is the smallest power of two >= a / 448, at least 2^-126,
 * and 1 if a = 0; a code is x / scale (exact) rounded to the nearest e4m3 value, ties to even; NaN and
 * infinities become the NaN code.  Powers of two cost no significant bit of a floating-point code,
 * and code * scale is then exact in bf16 where it is a multiple of 2^-133 (blocks whose largest |x| is over 2^-116 have
 * no other).  Beyond 248 * 2^120 the nearest value is 2^128, infinite when restored. */
dmmv_status dmmv_block_quantize(int32_t dtype, const void* x, int64_t ldx, const dmmv_block_matrix* q, void* hip_stream);

/* x <- the values of q, rounded once to dtype (exact for scales that are powers of two, between the
 * type's smallest number and its largest). */
dmmv_status dmmv_block_dequantize(const dmmv_block_matrix* q, int32_t dtype, void* x, int64_t ldx, void* hip_stream);

/* y[t][o] = sum_k x(t, k) w(o, k) + bias[o], x [T][K], w [O][K], y [T][ldy] of dtype DMMV_F32 or
 * DMMV_BF16, bias float [O] or NULL.  A 32-bit result is summed in 32 bits; a bf16 result by the 8-bit
 * matrix instructions, which drop what lies some 13 bits below the largest product of a step: an error
 * of about 5e-5 of the result's norm, up to 2^-11 of sum |x w| for a single one, before the rounding to
 * bf16 (1.7e-3).  Who needs the sum takes it in 32 bits.  Scales may be far apart: what counts is that
 * the products x w, their sum and the result are in the range.  The workspace (size from the HOST
 * function for every call of these sizes, 0 is possible, 256-byte aligned) holds, for bf16 results with
 * exponents or scales along rows, the operands of a large product once more where their rows are no
 * multiples of 16 codes, and partial sums where few tiles share a long contraction.  Other calls need
 * none. */
size_t dmmv_block_product_workspace_bytes(int64_t T, int64_t O, int64_t K);
dmmv_status dmmv_block_product(const dmmv_block_matrix* x, const dmmv_block_matrix* w, const float* bias, int32_t dtype,
                               void* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Gradients of the product from those of its result, dy [T][lddy] of dtype DMMV_F32 or DMMV_BF16:
 *   dx[t][k] = sum_o dy[t][o] w(o, k)       [T][lddx] of dtype     (w may be NULL if dx is)
 *   dw[o][k] = sum_t dy[t][o] x(t, k)       [O][lddw] float        (x may be NULL if dw is)
 *   dbias[o] = sum_t dy[t][o]               [O] float
 * Each of the three may be NULL.  They are the gradients with respect to the values that the 8-bit
 * matrices stand for.  T, O, K are the sizes.  Every product is exact or rounded to 24 bits; with bf16
 * dx and 32-bit scales that are the same along a row of w it may come from 16 (dx has 8).  They are
 * made of bf16 numbers: values of exponents are exact for bytes 3 to 246 and multiples of 2^-133 below
 * (infinite beyond the type's largest); of dy, of values with 32-bit scales and of dy times the scale
 * of a row 24 bits count from 2^-110 up, multiples of 2^-133 below.  The workspace (256-byte aligned)
 * holds partial sums, and dy as up to three bf16 parts and codes with aligned rows where a large
 * gradient is made from those.  ..._for is what the call with these arguments needs (dx and dw are
 * asked for if not NULL; nothing is read but the two descriptors), some 2 MB for a large one in bf16
 * with aligned rows and scales that are powers of two; 0 where the call would be refused.  ..._bytes
 * serves every call of these sizes. */
size_t dmmv_block_backward_workspace_bytes(int64_t T, int64_t O, int64_t K);
size_t dmmv_block_backward_workspace_for(int32_t dtype, int64_t T, int64_t O, int64_t K, const void* dy, int64_t lddy,
                                         const dmmv_block_matrix* x, const dmmv_block_matrix* w, const void* dx, const float* dw);
dmmv_status dmmv_block_backward(int32_t dtype, int64_t T, int64_t O, int64_t K, const void* dy, int64_t lddy,
                                const dmmv_block_matrix* x, const dmmv_block_matrix* w, void* dx, int64_t lddx, float* dw,
                                int64_t lddw, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Layer norm of the rows of x [rows][ldx], dtype DMMV_F32 or DMMV_BF16:
 *   mean = sum x / cols, rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps),
 *   v = (x - mean) * rstd * gamma + beta            (gamma, beta float [cols], NULL = 1, 0)
 * Outputs, each may be NULL: y [rows][ldy] = v in dtype; q = v in 8 bits, quantised like
 * dmmv_block_quantize from the 32-bit v; xq = x in 8 bits (scale_rows 1 for both); mean, rstd float
 * [rows] (NaN where cols = 0).  eps >= 0 and finite. */
dmmv_status dmmv_layernorm(int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx, const float* gamma,
                           const float* beta, float eps, void* y, int64_t ldy, const dmmv_block_matrix* q,
                           const dmmv_block_matrix* xq, float* mean, float* rstd, void* hip_stream);

/* Gradients of the layer norm from those of its result, dy [rows][lddy] of dtype.  The input comes
 * as x [rows][ldx] of dtype, or from its 8-bit checkpoint xq (exactly one of the two is not NULL);
 * mean and rstd are the forward pass's.  With h = (x - mean) rstd and a = dy gamma:
 *   dx = rstd (a - sum a / cols - h sum(a h) / cols)       [rows][lddx] of dtype
 *   dgamma = sum over rows of dy h, dbeta = sum over rows of dy      float [cols]
 * Each of the three may be NULL. */
size_t dmmv_layernorm_workspace_bytes(int64_t rows, int64_t cols);
dmmv_status dmmv_layernorm_backward(int32_t dtype, int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* x,
                                    int64_t ldx, const dmmv_block_matrix* xq, const float* gamma, const float* mean,
                                    const float* rstd, void* dx, int64_t lddx, float* dgamma, float* dbeta,
                                    void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DMMV_LAYER_H */
