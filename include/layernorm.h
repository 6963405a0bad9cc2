/*
 * layernorm.h -- C ABI of layer norm in libdgemm (NVIDIA B200, sm_100a).
 *
 * The normalisation in front of a transformer's products, forward and backward, on row-major device
 * matrices of binary32, binary16 or bfloat16 (HGEMM_TYPE_*). Statistics, sums and parameter
 * gradients are binary32. (No counterpart in the paper.)
 *
 * Conventions, status codes, streams and scratch memory as in hgemm.h. Any element-aligned address
 * and any leading dimension >= cols may be used.
 */
#ifndef LAYERNORM_H
#define LAYERNORM_H

#include <stdint.h>

#include "hgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * For every row x of X (rows x cols):
 *   mean = sum(x) / cols,  rstd = 1 / sqrt(sum((x - mean)^2) / cols + eps),  y = (x - mean) rstd gamma + beta.
 *
 *   gamma, beta  cols values of `type`; NULL means ones / zeros
 *   mean, rstd   one binary32 value per row (what the backward pass needs), each NULL if not wanted
 *   eps          finite, >= 0
 *
 * The variance is taken from the centred values (two sums over the row held on the chip), not from
 * the difference of two large sums. rows == 0 or cols == 0: DGEMM_OK, nothing is written.
 */
DGEMM_API int layernorm_fwd(int type, int64_t rows, int64_t cols, const void *X, int64_t ldx,
                            const void *gamma, const void *beta, float eps,
                            void *Y, int64_t ldy, float *mean, float *rstd, void *stream);

/*
 * Gradients for an incoming dY (rows x cols), with xh = (x - mean) rstd and w = dy gamma:
 *   dx = rstd (w - sum(w)/cols - xh sum(w xh)/cols),  dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy.
 * mean and rstd are the forward pass's. dX (of `type`), dgamma and dbeta (cols binary32 values):
 * outputs, each NULL if not wanted. The sums over rows are taken in a fixed order: the same
 * arguments give the same bits. rows == 0 gives dgamma = dbeta = 0.
 */
DGEMM_API int layernorm_bwd(int type, int64_t rows, int64_t cols, const void *X, int64_t ldx, const void *gamma,
                            const float *mean, const float *rstd, const void *dY, int64_t lddy,
                            void *dX, int64_t lddx, float *dgamma, float *dbeta, void *stream);

#ifdef __cplusplus
}
#endif
#endif
