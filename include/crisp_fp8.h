/*
 * libcrisp, layers in 8 bits: matrices held as 8-bit floating point (e4m3: 4 exponent and 3 mantissa bits, largest
 * value 448) with one fp32 scale for each block of 128, the quantiser that makes them, and the product that reads them.
 *
 * The product is the one of a dense layer, y = x W^T, of its input's gradient, dx = dy W, and of its weight's gradient,
 * dW = dy^T x (Sec. 3.4: the gradient that the saliency |W * G| needs, and that fine-tuning between two pruning steps
 * applies): each is a product of two matrices whose contraction runs along their contiguous columns, so the gradients
 * read operands that were quantised along the other direction.
 *
 * The conventions of crisp.h hold: status codes, arguments checked on the host before any device call, no allocation and
 * no synchronisation, work enqueued on `stream`.  What a call writes must not overlap what it reads, but for a residual that is
 * Y itself, nor its other results (EINVAL where two of them begin at the same address).
 */
#ifndef CRISP_FP8_H
#define CRISP_FP8_H

#include "crisp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What a scale covers */
enum {
    CRISP_FP8_ROWS = 0,  /* 128 columns of one row:  scale[b * lds + r] is that of columns 128b .. 128b+127 of row r */
    CRISP_FP8_TILES = 1  /* 128 rows x 128 columns:  scale[(r / 128) * lds + b]                                      */
};

enum { CRISP_IN_F32 = 0, CRISP_IN_BF16 = 1 };   /* element type of what is quantised (same codes as CRISP_Y_*) */

/*
 * A matrix in 8 bits: element (r, c) stands for q[r * ld + c] * scale(r, c / 128).
 * q is read (and written by crisp_fp8_quant) up to column round_up(cols, 128): the columns behind `cols` must hold zeros.
 */
typedef struct {
    uint8_t *q;          /* rows x ld e4m3 (device), 16-byte aligned                                    */
    float *scale;        /* ROWS: ceil(cols/128) x lds, TILES: ceil(rows/128) x lds fp32 (device)       */
    int64_t ld;          /* >= round_up(cols, 128), multiple of 16                                      */
    int64_t lds;         /* ROWS: >= rows, TILES: >= ceil(cols/128)                                     */
    int64_t rows, cols;  /* 1 .. 2^27                                                                   */
    int32_t kind;        /* CRISP_FP8_ROWS | CRISP_FP8_TILES                                            */
    int32_t reserved;    /* 0                                                                           */
} crisp_fp8_mat;

/*
 * Quantises a matrix, or its transpose, or both in one pass over it.
 *   amax = largest |x| of a block;  s = max(amax / 448, 2^-126);  q = e4m3(x * (1 / s))
 * each step in fp32 and rounded to nearest even.  A block that holds an infinity or a NaN gets that as its scale, and every
 * product that uses the block is NaN.
 *   X: rows x ldx, fp32 or bf16 per in_type (device), aligned to its element; ldx >= cols.
 *   mask: optional, rows x ceil(cols/32) uint32 like crisp_select_mask's nm_mask (device): elements whose bit is not set
 *      count as zero, whatever they hold.
 *   Q: the matrix in 8 bits (rows, cols, kind), or NULL.
 *   Qt: its transpose (Qt->rows = cols, Qt->cols = rows, the same kind), or NULL; at least one of the two.  In ROWS each has
 *      scales of its own, along its own columns; in TILES both have the same values and the same scales.
 * At most 2^28 - 16 blocks of 128 columns (ESHAPE beyond).
 * Columns between cols and round_up(cols, 128) of Q are written with zeros, those behind are left alone; so for Qt.
 * Errors: EINVAL, ESHAPE, EALIGN, EDEVICE.
 */
CRISP_API crisp_status crisp_fp8_quant(const void *X, int32_t in_type, int64_t rows, int64_t cols, int64_t ldx,
                                       const uint32_t *mask, const crisp_fp8_mat *Q, const crisp_fp8_mat *Qt, void *stream);

/*
 * Y[t][s] = sum over blocks b of 128 columns of  scale_x(t, b) * scale_w(s, b) * sum_c X[t][c] * W[s][c],
 * T = X->rows, S = W->rows, X->cols == W->cols; X in ROWS, W in ROWS or TILES.  Sums in fp32, one rounding to y_type.
 * With y_type BF16 the 8-bit matrix instruction adds the products of a block: among eight consecutive ones, what lies more
 * than 13 bits below the largest is cut off before the fp32 sum (at most 2^-10 of the sum of magnitudes, 1.5e-5 of the result
 * on normal operands).  With F32 every product enters the fp32 sum whole, at half the rate.
 * The two scales of a block are multiplied with each other first, in fp32: a product of theirs below 2^-126 is rounded to a multiple
 * of 2^-149, and one above fp32's range is infinite (NaN for results whose sum over that block is zero).
 *   layer:             X = activations (T x K),  W = weights (S x K)        -> y  (T x S)
 *   input's gradient:  X = dy (T x S),           W = W^T (K x S)            -> dx (T x K)
 *   weight's gradient: X = dy^T (S x T),         W = x^T (K x T)            -> dW (S x K)
 *   Y: T x ldy, fp32 or bf16 per y_type (CRISP_Y_*), ldy >= S, aligned to its element; every element of the T x S part is
 *      written, none behind it.
 *   ep: the epilogue of crisp_spmm_ep or NULL; scale and bias are per column of Y (S values), residual is T x ldr of Y's
 *      type, ldr >= S, aligned to its element, and may be Y itself (with ldr == ldy): gradients accumulate.  relu lets NaN
 *      through.
 * At most 2^26 tiles of 16 x 16 outputs, 2^22 - 1 where T or S is up to 32 or a row stride 2^24 or more (ESHAPE beyond).
 * The sum's order depends on sizes, types and row strides only: the same call gives the same bits.
 * Errors: EINVAL, ESHAPE, EALIGN, EDEVICE.
 */
CRISP_API crisp_status crisp_fp8_product(const crisp_fp8_mat *X, const crisp_fp8_mat *W, void *Y, int64_t ldy,
                                         int32_t y_type, const crisp_epilogue *ep, void *stream);

/* Bytes of workspace that crisp_fp8_linear wants for T rows of K columns (host only; 0 for a few rows, and for sizes out of
 * range). */
CRISP_API size_t crisp_fp8_linear_ws(int64_t T, int64_t K);

/*
 * The layer from activations that are not in 8 bits yet: crisp_fp8_quant (ROWS) of X into ws, then crisp_fp8_product; for a
 * few rows one kernel does both and ws is not looked at.  Results are those of the two calls, bit for bit.
 *   X: T x ldx, fp32 or bf16 per in_type (device), aligned to its element; ldx >= W->cols.
 *   ws: crisp_fp8_linear_ws(T, W->cols) bytes (device), 16-byte aligned; its contents are unspecified before and after.
 *      Calls that may run at the same time need one each.
 * Errors: EINVAL, ESHAPE, EALIGN, EBUFSIZE, EDEVICE.
 */
CRISP_API crisp_status crisp_fp8_linear(const void *X, int32_t in_type, int64_t T, int64_t ldx, const crisp_fp8_mat *W,
                                        void *Y, int64_t ldy, int32_t y_type, const crisp_epilogue *ep, void *ws,
                                        size_t ws_bytes, void *stream);

/* Bytes of workspace of crisp_fp8_linear_backward (host only; 0 for sizes out of range). */
CRISP_API size_t crisp_fp8_linear_backward_ws(int64_t T, int64_t S);

/*
 * The layer's gradients: dY is quantised once, along its rows and along its columns, then
 *   dX = crisp_fp8_product(dY, Wt)     (T x K, lddx >= K, fp32 or bf16 per dx_type),
 *   dW = crisp_fp8_product(dY^T, Xt)   (S x K, lddw >= K, fp32 or bf16 per dw_type), with accumulate = 1 added to what is there.
 *   dY: T x ldg of S used columns, fp32 or bf16 per in_type (device), aligned to its element.
 *   Xt: the activations' transpose (K x T, ROWS or TILES);  Wt: the weights' transpose (K x S).
 *   dX or dW may be NULL: that gradient is not computed, and Wt or Xt is not looked at.
 *   ws: crisp_fp8_linear_backward_ws(T, S) bytes (device), 16-byte aligned; as in crisp_fp8_linear.
 * Errors: EINVAL, ESHAPE, EALIGN, EBUFSIZE, EDEVICE.
 */
CRISP_API crisp_status crisp_fp8_linear_backward(const void *dY, int32_t in_type, int64_t T, int64_t S, int64_t ldg,
                                                 const crisp_fp8_mat *Xt, const crisp_fp8_mat *Wt, void *dX, int64_t lddx,
                                                 int32_t dx_type, void *dW, int64_t lddw, int32_t dw_type, int32_t accumulate,
                                                 void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
