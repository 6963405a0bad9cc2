/*
 * dropout.h -- C ABI of dropout in libdgemm (NVIDIA B200, sm_100a).
 *
 * Dropout of a sublayer's output with the addition of the residual stream in the same pass, and its
 * backward pass, on row-major device matrices of binary32, binary16 or bfloat16 (HGEMM_TYPE_*). The mask
 * comes from a counter-based generator and is never stored: the backward pass makes it again.
 * (No counterpart in the paper.)
 *
 * Conventions, status codes and streams as in hgemm.h. Any element-aligned address and any leading
 * dimension >= cols may be used.
 */
#ifndef DROPOUT_H
#define DROPOUT_H

#include <stdint.h>

#include "hgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * y = r + (keep ? x / (1 - p) : 0)  for every value of X (rows x cols), r of R.
 *
 *   p       probability of dropping, 0 <= p <= 1 (1: everything is dropped)
 *   seed    64 bits; offset: 64 bits, another one for each use of a seed
 *   step    device address of one 64-bit integer that is added to `offset` when the kernel runs, or
 *           NULL: a captured call gives a new mask in each replay if the program counts it up
 *   R       the residual, or NULL. Y may be X or R itself (same address and leading dimension)
 *
 * keep: word (column % 4) of Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as
 * easy as 1, 2, 3", SC 2011) with the key `seed` (low word first) and the counter words column / 4, row and
 * the low and high word of offset + *step, is not below p 2^32 (rounded to the nearest integer). The
 * mask depends on these alone: not on addresses, leading dimensions, type or device. What is dropped
 * counts as 0 whatever it holds (NaN and infinities too). x / (1 - p) is x times the binary32 value of 1 / (1 - p).
 */
DGEMM_API int dropout_fwd(int type, int64_t rows, int64_t cols, const void *X, int64_t ldx, const void *R, int64_t ldr, double p,
                          uint64_t seed, uint64_t offset, const int64_t *step, void *Y, int64_t ldy, void *stream);

/* The gradient for an incoming dY: dx = keep ? dy / (1 - p) : 0 with the same mask. dX may be dY itself.
 * (The residual's gradient is dY itself.) */
DGEMM_API int dropout_bwd(int type, int64_t rows, int64_t cols, const void *dY, int64_t lddy, double p, uint64_t seed,
                          uint64_t offset, const int64_t *step, void *dX, int64_t lddx, void *stream);

#ifdef __cplusplus
}
#endif
#endif
