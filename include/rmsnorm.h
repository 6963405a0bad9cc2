/*
 * rmsnorm.h -- C ABI of root-mean-square norm in libdgemm (NVIDIA B200, sm_100a).
 *
 * The normalisation in front of a transformer's products in its root-mean-square form, with the
 * addition of the residual stream in the same pass, forward and backward, on row-major device matrices
 * of binary32, binary16 or bfloat16 (HGEMM_TYPE_*); and its output (or any matrix) in 8 bits, e4m3,
 * with one scale per row, as the products of qgemm.h take it. Sums and statistics are binary32, each
 * output is rounded once. (No counterpart in the paper.)
 *
 * Conventions, status codes, streams and scratch memory as in hgemm.h. Any element-aligned address
 * and any leading dimension >= cols may be used. Only the logical part of a matrix is read or written.
 */
#ifndef RMSNORM_H
#define RMSNORM_H

#include <stdint.h>

#include "hgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * For every row x of X (rows x cols), r of R:
 *   s = x + r,  rstd = 1 / sqrt(sum(s^2) / cols + eps),  y = s rstd gamma.
 *
 *   R      the residual, or NULL (s = x)
 *   gamma  cols values of `type`; NULL means ones
 *   S      output for the sum, rounded to `type` (the residual stream's next value and what the
 *          backward pass needs), or NULL. It may be X or R itself (same address and leading dimension)
 *   rstd   one binary32 value per row (what the backward pass needs), or NULL
 *   eps    finite, >= 0
 *
 * y and rstd are computed from the sum before it is rounded. Rows whose squares or whose products with gamma could leave
 * binary32's range (a root of the sum of squares from 2^27 up, or an rstd above 2^20) are scaled by a power of two and multiplied
 * by rstd before gamma. |gamma| up to 2^100 (beyond that s gamma may overflow in other rows); a y that is not 0 may be off by
 * 2^-130 beside its rounding. rows == 0 or cols == 0: DGEMM_OK, nothing is written. Y must not overlap an input or another output.
 */
DGEMM_API int rmsnorm_fwd(int type, int64_t rows, int64_t cols, const void *X, int64_t ldx, const void *R, int64_t ldr,
                          const void *gamma, float eps, void *S, int64_t lds, void *Y, int64_t ldy, float *rstd,
                          void *stream);

/*
 * The same with the output in 8 bits: with y as above and before any rounding,
 *   scale = max(max |y|, 2^-100) / 448,  q = y / scale rounded to e4m3 (to nearest, ties to even),
 * so that q scale stands for y and the row's largest value for itself. A row that holds a NaN (or, under
 * the norm, an infinity) has a scale that is not finite.
 *
 *   Q      rows x cols bytes, leading dimension ldq >= cols (in bytes)
 *   scale  one binary32 value per row
 */
DGEMM_API int rmsnorm_fwd_e4m3(int type, int64_t rows, int64_t cols, const void *X, int64_t ldx, const void *R, int64_t ldr,
                               const void *gamma, float eps, void *S, int64_t lds, void *Q, int64_t ldq, float *scale,
                               float *rstd, void *stream);

/* Rows brought to 8 bits as they are: y = x in the formulas of rmsnorm_fwd_e4m3. q is the value nearest to 448 x / max |x|, exactly
 * for 16-bit types; in binary32 (and under the norm, whose y is known to binary32's precision) values next to the middle between two
 * e4m3 values may fall to either. */
DGEMM_API int quantize_rows_e4m3(int type, int64_t rows, int64_t cols, const void *X, int64_t ldx, void *Q, int64_t ldq,
                                 float *scale, void *stream);

/*
 * Gradients of rmsnorm_fwd for an incoming dY and, where the sum goes on as the residual stream, dS
 * (rows x cols each), with xh = s rstd and w = dy gamma:
 *   dx = rstd (w - xh sum(w xh) / cols) + ds  (the gradient of x and of r),  dgamma = sum over rows of dy xh.
 *
 *   S, rstd    the forward pass's sum (X where there was no residual) and statistics
 *   dS         NULL: none. dX may be dS itself (same address and leading dimension)
 *   dX, dgamma outputs, each NULL if not wanted; dX is of `type`, dgamma cols binary32 values
 *
 * The sum over rows is taken in a fixed order: the same arguments give the same bits. rows == 0
 * gives dgamma = 0.
 */
DGEMM_API int rmsnorm_bwd(int type, int64_t rows, int64_t cols, const void *S, int64_t lds, const void *gamma, const float *rstd,
                          const void *dY, int64_t lddy, const void *dS, int64_t ldds, void *dX, int64_t lddx, float *dgamma,
                          void *stream);

#ifdef __cplusplus
}
#endif
#endif
