/*
 * hgemm.h -- C ABI of the 16-bit matrix products of libdgemm (NVIDIA B200, sm_100a).
 *
 * What a transformer's feed-forward path computes next to a plain product: the product with bias,
 * activation and residual in its epilogue, and the gated projections act(X Wg) * (X Wu), each with
 * its backward pass. Operands are binary16 or bfloat16; products are accumulated in binary32 on the
 * tensor cores, the epilogue works on the binary32 sums, and each output is rounded once.
 * (No counterpart in the paper, which studies the binary64 product.)
 *
 * Plain C types only; status codes are those of dgemm.h. Matrices are row-major device buffers of the
 * current device with a leading dimension >= the row length (in elements), owned by the caller; any
 * element-aligned address and any leading dimension may be used. Operands that the copy engine can
 * address (16-byte aligned, leading dimension a multiple of 8) are used where they lie; others are
 * first rewritten into scratch memory of the library (leased per call as for dgemm_f64: calls may be
 * in flight on several streams; it is grown with a synchronising cudaMalloc, so make a stream's
 * first call of a size outside stream capture; what a captured call uses stays allocated, whatever later calls need, until
 * dgemm_release_scratch, after which the graph must not be replayed). Only the logical part of a matrix is read or written.
 * All calls are asynchronous on `stream` (a cudaStream_t passed as void*; NULL is the legacy default
 * stream) and give the same bits every time for the same arguments.
 */
#ifndef HGEMM_H
#define HGEMM_H

#include <stdint.h>

#include "dgemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
enum {
  HGEMM_TYPE_F32 = 0, /* binary32: layernorm.h only */
  HGEMM_TYPE_F16 = 1, /* binary16                   */
  HGEMM_TYPE_BF16 = 2 /* bfloat16                   */
};

/* Activations. */
enum {
  HGEMM_ACT_NONE = 0,
  HGEMM_ACT_RELU = 1,      /* max(z, 0); its derivative at 0 is 0                                */
  HGEMM_ACT_GELU = 2,      /* z/2 (1 + erf(z / sqrt 2))                                          */
  HGEMM_ACT_GELU_TANH = 3, /* z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3)))                      */
  HGEMM_ACT_SILU = 4,      /* z / (1 + exp(-z))                                                  */
  HGEMM_ACT_COUNT = 5
};

/*
 * Z = op(A) op(B) + bias,  D = act(Z) + R.
 *
 *   type    HGEMM_TYPE_F16 or HGEMM_TYPE_BF16: of A, B, bias, R, D and Z
 *   transa  DGEMM_OP_N: A is M x K.  DGEMM_OP_T: A is stored K x M
 *   transb  DGEMM_OP_N: B is K x N.  DGEMM_OP_T: B is stored N x K
 *   bias    N values, added to every row, or NULL
 *   R       M x N residual, or NULL. It may be D itself (same address and leading dimension)
 *   Z       M x N output for the pre-activation (what the backward pass needs), or NULL
 *
 * K == 0 is an empty sum: D = act(bias) + R. M == 0 or N == 0: DGEMM_OK, nothing is inspected.
 * D and Z must not overlap an input (except R == D) or one another (DGEMM_ERR_ALIAS).
 */
DGEMM_API int hgemm_epilogue(int type, int transa, int transb, int64_t M, int64_t N, int64_t K,
                             const void *A, int64_t lda, const void *B, int64_t ldb,
                             const void *bias, int act, const void *R, int64_t ldr,
                             void *D, int64_t ldd, void *Z, int64_t ldz, void *stream);

/*
 * Gradients of hgemm_epilogue for an incoming dD (M x N):
 *   dZ = dD * act'(Z),  dA = dZ op(B)^T,  dB = op(A)^T dZ  (stored as A and B are),  dbias = sum over rows of dZ.
 * (The residual's gradient is dD itself.)
 *
 *   Z      the pre-activation kept by the forward pass; not read (may be NULL) for HGEMM_ACT_NONE
 *   dA, dB, dbias  outputs, each NULL if not wanted; dbias is N binary32 values, summed in binary32
 *
 * dZ enters the products rounded to `type`: the tensor cores take 16-bit operands. That rounding is
 * of the size of the outputs' own; dbias sums the unrounded values. In binary16 a dZ whose largest finite
 * magnitude lies outside [2^-4, 65520) is scaled by a power of two before it is rounded, and the products
 * back, so that its range is no limit of theirs (values below 2^-28 of the largest lose bits).
 * M == 0 gives dB = 0 and dbias = 0, N == 0 gives dA = 0.
 */
DGEMM_API int hgemm_epilogue_bwd(int type, int transa, int transb, int64_t M, int64_t N, int64_t K,
                                 const void *A, int64_t lda, const void *B, int64_t ldb,
                                 int act, const void *Z, int64_t ldz, const void *dD, int64_t lddd,
                                 void *dA, int64_t ldda, void *dB, int64_t lddb, float *dbias, void *stream);

/*
 * Gated projections of a feed-forward block, in one kernel:
 *   G = X op(Wg),  U = X op(Wu),  H = act(G) * U.
 *
 *   X       M x K
 *   transw  DGEMM_OP_N: Wg and Wu are K x F.  DGEMM_OP_T: both are stored F x K
 *   G, U    M x F outputs (what the backward pass needs), both or neither; NULL if not wanted
 */
DGEMM_API int hgemm_gated(int type, int transw, int64_t M, int64_t F, int64_t K,
                          const void *X, int64_t ldx, const void *Wg, int64_t ldwg, const void *Wu, int64_t ldwu,
                          int act, void *H, int64_t ldh, void *G, int64_t ldg, void *U, int64_t ldu, void *stream);

/*
 * Gradients of hgemm_gated for an incoming dH (M x F):
 *   dG = dH * U * act'(G),  dU = dH * act(G),
 *   dX = dG op(Wg)^T + dU op(Wu)^T (one sum, rounded once),  dWg = X^T dG,  dWu = X^T dU (stored as Wg and Wu are).
 * dX, dWg, dWu: outputs, each NULL if not wanted. dG and dU enter the products rounded to `type`, in
 * binary16 scaled together as dZ above.
 */
DGEMM_API int hgemm_gated_bwd(int type, int transw, int64_t M, int64_t F, int64_t K,
                              const void *X, int64_t ldx, const void *Wg, int64_t ldwg, const void *Wu, int64_t ldwu,
                              int act, const void *G, int64_t ldg, const void *U, int64_t ldu,
                              const void *dH, int64_t lddh, void *dX, int64_t lddx,
                              void *dWg, int64_t lddwg, void *dWu, int64_t lddwu, void *stream);

/* Synchronises `stream`, then reads and clears the device status word of the kernels of this header
 * (DGEMM_OK, DGEMM_ERR_TIMEOUT if a bounded wait inside a kernel gave up, DGEMM_ERR_CUDA). */
DGEMM_API int hgemm_last_device_status(void *stream);

/*
 * What the library would do with one product (or, `gated` != 0, gated projection) of op(A) M x K and
 * op(B) K x N, without touching a device. `sm_count`: 0 = 148. Writes 8 ints to `out`: CTAs per tile
 * (1, or 2 for a pair), tile rows, tile columns, clusters launched, k-blocks (64 values each), whole
 * rounds of tiles over the clusters, tiles left over, and the k-blocks of those that each cluster
 * takes as one span (0: they run whole, too).
 */
DGEMM_API int hgemm_plan(int64_t M, int64_t N, int64_t K, int gated, int sm_count, int *out);

/*
 * Testing aid: with `limit_us` > 0 the kernels' producers skip their copies (like a message that is
 * dropped) and the bounded waits are limited to that many microseconds (at most 4 000 000), so that
 * calls end in DGEMM_ERR_TIMEOUT through the status word and leave their outputs unspecified. 0
 * restores the default. Nothing faults, traps or spins without a limit.
 */
DGEMM_API int hgemm_set_test_drop_loads(int limit_us);

#ifdef __cplusplus
}
#endif
#endif
