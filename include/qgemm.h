/*
 * qgemm.h -- C ABI of the 8-bit matrix products of libdgemm (NVIDIA B200, sm_100a).
 *
 * The products of hgemm.h with operands in 8 bits, e4m3, and a scale for each of their rows: what a model
 * answers with whose weights have been brought to 8 bits and whose activations come from
 * rmsnorm_fwd_e4m3 or quantize_rows_e4m3 (rmsnorm.h). Products are accumulated in binary32 on the tensor cores, the
 * epilogue works on the scaled binary32 sums, and each output is rounded once.
 * (No counterpart in the paper.)
 *
 * Conventions, status codes, activations, streams and scratch memory as in hgemm.h. The contraction index
 * is contiguous in both operands: activations M x K, weights N x K. Any address and any leading dimension
 * >= K may be used; operands whose rows are not 16-byte aligned are first rewritten into scratch memory.
 * hgemm_last_device_status reads the status word of these kernels, too.
 */
#ifndef QGEMM_H
#define QGEMM_H

#include <stdint.h>

#include "hgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Z[m][n] = a_scale[m] b_scale[n] sum_k A[m][k] B[n][k] + bias[n],  D = act(Z) + R.
 *
 *   type     HGEMM_TYPE_F16 or HGEMM_TYPE_BF16: of bias, R, D and Z
 *   A        M x K bytes (e4m3), leading dimension in bytes;  B: N x K
 *   a_scale  M binary32 values, or NULL (ones);  b_scale: N
 *   bias     N values, or NULL
 *   R        M x N residual, or NULL. It may be D itself (same address and leading dimension)
 *   Z        M x N output for the pre-activation, or NULL
 *
 * The sum is multiplied by a_scale[m] first and then by b_scale[n]: with an a_scale from 2^-109 (the least of a row in 8 bits) to 2^80 the
 * product in between stays in binary32's range whatever b_scale is; beyond, it may leave it where Z does not. The same for qgemm_gated.
 *
 * K == 0 is an empty sum: D = act(bias) + R. M == 0 or N == 0: DGEMM_OK, nothing is inspected.
 */
DGEMM_API int qgemm_epilogue(int type, int64_t M, int64_t N, int64_t K, const void *A, int64_t lda, const float *a_scale,
                             const void *B, int64_t ldb, const float *b_scale, const void *bias, int act,
                             const void *R, int64_t ldr, void *D, int64_t ldd, void *Z, int64_t ldz, void *stream);

/*
 * Gated projections: G = x_scale g_scale (X Wg^T),  U = x_scale u_scale (X Wu^T),  H = act(G) * U.
 *
 *   X   M x K bytes (e4m3);  Wg, Wu: F x K
 *   x_scale  M binary32 values, g_scale and u_scale F each; NULL: ones
 *   G, U     M x F outputs of `type`, both or neither; NULL if not wanted
 */
DGEMM_API int qgemm_gated(int type, int64_t M, int64_t F, int64_t K, const void *X, int64_t ldx, const float *x_scale,
                          const void *Wg, int64_t ldwg, const float *g_scale, const void *Wu, int64_t ldwu, const float *u_scale,
                          int act, void *H, int64_t ldh, void *G, int64_t ldg, void *U, int64_t ldu, void *stream);

#ifdef __cplusplus
}
#endif
#endif
