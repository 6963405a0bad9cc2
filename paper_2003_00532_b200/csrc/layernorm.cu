// C ABI of layer norm (include/layernorm.h): validation, choice of kernel, launches.
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>

#include <cuda_runtime.h>

#include "../../include/layernorm.h"
#include "layernorm.cuh"
#include "lm_state.h"
#include "row_launch.h"

namespace {

using namespace lnorm;
using namespace rowop;

// How a row is spread over threads: vectors per thread, and threads (32: one warp per row).
struct Shape {
  int items, threads;
  bool longer;  // does not fit in registers
};
// Forward: a warp for rows of up to 32 values per lane; a block with 16 values per thread beyond (or up to 32, for rows
// that need them). Few rows are spread over as many threads as there are vectors, because then the latency of
// one row counts.
Shape fwd_shape(int64_t rows, int64_t cols, int vec, int sms) {
  const int64_t nv = (cols + vec - 1) / vec;
  const int most = 32 / vec;
  const bool spread = rows * ((nv + 32 * most - 1) / (32 * most)) < (int64_t)sms * 16;  // warps in all
  if (nv <= 32 || (!spread && nv <= 32 * most)) return Shape{pow2((nv + 31) / 32), 32, false};
  int items = spread ? 1 : 16 / vec;
  while (items < most && threads_for(nv, items) > fwd_threads(items * vec)) items *= 2;
  const int threads = threads_for(nv, items);
  if (threads > fwd_threads(items * vec)) return Shape{0, 1024, true};
  return Shape{items, threads, false};
}
// Backward: a warp for rows of up to 16 values per lane; a block with 16 values per thread beyond; 32 (`WIDE`, sums in
// shared memory) for rows that need them: 8193 to 16384 columns. Those do not fit 128 registers (ptxas: 480 bytes of spill stores
// in binary32 with vectors, 230 to 300 with single values, at most 12 in 16-bit types with vectors): 1500 x 9000 binary32 64 us,
// floor 25. Longer rows are read again by scalar accesses in each pass (2048 x 20000 bf16: forward 142 us, backward 244, floors 25 and 38).
Shape bwd_shape(int64_t cols, int vec) {
  const int64_t nv = (cols + vec - 1) / vec;
  const int most = 16 / vec;
  if (nv <= 32 * most) return Shape{pow2((nv + 31) / 32), 32, false};
  for (int items = most; items <= 2 * most; items *= 2)
    if (threads_for(nv, items) <= BWD_THREADS) return Shape{items, threads_for(nv, items), false};
  return Shape{0, 1024, true};
}

template <typename T, int VEC, int ITEMS, bool WARP_ROW>
bool launch_fwd(int sms, int threads, const Params& p, cudaStream_t stream) {
  constexpr auto kernel = &fwd_kernel<T, VEC, ITEMS, WARP_ROW>;
  const size_t smem = (size_t)(WARP_ROW ? 32 : threads) * ITEMS * VEC * 8;  // gamma and beta
  if (!WARP_ROW && !allow_smem<decltype(kernel), kernel>(fwd_threads(VEC * ITEMS) * ITEMS * VEC * 8)) return false;
  const int64_t need = WARP_ROW ? (p.rows + 3) / 4 : p.rows;
  const unsigned blocks = resident_blocks<decltype(kernel), kernel>(sms, threads, smem, need);
  return blocks > 0 && lm::launch(kernel, dim3(blocks), dim3(threads), smem, 1, stream, p);
}
template <typename T, int VEC, int ITEMS>
bool launch_fwd_items(int sms, const Shape& s, const Params& p, cudaStream_t stream) {
  if (s.threads == 32) return launch_fwd<T, VEC, ITEMS, true>(sms, 128, p, stream);
  return launch_fwd<T, VEC, ITEMS, false>(sms, s.threads, p, stream);
}
template <typename T, int VEC>
bool run_fwd_vec(int sms, const Params& p, cudaStream_t stream) {
  const Shape s = fwd_shape(p.rows, p.cols, VEC, sms);
  if (s.longer) return lm::launch(fwd_long_kernel<T>, dim3((unsigned)p.rows), dim3(1024), 0, 1, stream, p);
  switch (s.items) {
    case 1: return launch_fwd_items<T, VEC, 1>(sms, s, p, stream);
    case 2: return launch_fwd_items<T, VEC, 2>(sms, s, p, stream);
    case 4: return launch_fwd_items<T, VEC, 4>(sms, s, p, stream);
    case 8: return VEC <= 4 && launch_fwd_items<T, VEC <= 4 ? VEC : 1, 8>(sms, s, p, stream);
    case 16: return VEC == 1 && launch_fwd_items<T, 1, 16>(sms, s, p, stream);
    default: return VEC == 1 && launch_fwd_items<T, 1, 32>(sms, s, p, stream);
  }
}
template <typename T, int VEC>
bool run_fwd(int sms, bool aligned, const Params& p, cudaStream_t stream) {
  return aligned ? run_fwd_vec<T, VEC>(sms, p, stream) : run_fwd_vec<T, 1>(sms, p, stream);
}

// Blocks of the backward pass: as many as fit at once, but for few rows at least eight rows each (every block leaves
// its own sums to be added), down to one per SM.
template <typename K, K kernel>
int bwd_blocks(int sms, int threads, size_t smem, int64_t rows, int rows_per_block) {
  const int64_t need = (rows + rows_per_block - 1) / rows_per_block;
  const int64_t some = (int)resident_blocks<K, kernel>(sms, threads, smem, need);
  const int64_t eighth = (rows + 8 * rows_per_block - 1) / (8 * rows_per_block);
  const int64_t want = eighth > sms ? eighth : sms;
  return (int)(some < want ? some : want);
}

// Runs the row kernel; `partial` is asked for the matrix of the blocks' sums. Returns the number of blocks, 0 on failure.
template <typename T, int VEC, int ITEMS, bool WARP_ROW, bool WIDE, typename F>
int launch_bwd(int sms, int threads, Params& p, cudaStream_t stream, F partial) {
  constexpr auto kernel = &bwd_kernel<T, VEC, ITEMS, WARP_ROW, WIDE>;
  const size_t smem = WIDE ? (size_t)threads * ITEMS * VEC * 12 : WARP_ROW && p.want_params ? (size_t)p.cols * 8 : 0;
  if (WIDE && !allow_smem<decltype(kernel), kernel>(BWD_THREADS * ITEMS * VEC * 12)) return 0;
  const size_t most = WIDE ? smem : WARP_ROW ? (size_t)32 * ITEMS * VEC * 8 : 0;
  const int blocks = bwd_blocks<decltype(kernel), kernel>(sms, threads, most, p.rows, WARP_ROW ? 8 : 1);
  if (blocks == 0 || !partial(blocks)) return 0;
  return lm::launch(kernel, dim3(blocks), dim3(threads), smem, 1, stream, p) ? blocks : 0;
}
template <typename T, int VEC, typename F>
int run_bwd_vec(int sms, Params& p, cudaStream_t stream, F partial) {
  const Shape s = bwd_shape(p.cols, VEC);
  if (s.longer) {
    const int chunks = (int)((p.rows + 15) / 16 < sms * 2 ? (p.rows + 15) / 16 : sms * 2);
    if (!partial(chunks)) return 0;
    if (p.out && !lm::launch(bwd_long_kernel<T>, dim3((unsigned)p.rows), dim3(1024), 0, 1, stream, p)) return 0;
    if (p.want_params && !lm::launch(bwd_long_params_kernel<T>, dim3((unsigned)((p.cols + 255) / 256), chunks), dim3(256), 0, 1, stream, p))
      return 0;
    return chunks;
  }
  constexpr int MOST = 16 / VEC;
  if (s.threads == 32) {
    if (s.items == 1) return launch_bwd<T, VEC, 1, true, false>(sms, 256, p, stream, partial);
    if (s.items == 2) return launch_bwd<T, VEC, 2, true, false>(sms, 256, p, stream, partial);
    if constexpr (MOST >= 4)
      if (s.items == 4) return launch_bwd<T, VEC, 4, true, false>(sms, 256, p, stream, partial);
    if constexpr (MOST >= 16) {
      if (s.items == 8) return launch_bwd<T, VEC, 8, true, false>(sms, 256, p, stream, partial);
      if (s.items == 16) return launch_bwd<T, VEC, 16, true, false>(sms, 256, p, stream, partial);
    }
    return 0;
  }
  if (s.items == MOST) return launch_bwd<T, VEC, MOST, false, false>(sms, s.threads, p, stream, partial);
  return launch_bwd<T, VEC, 2 * MOST, false, true>(sms, s.threads, p, stream, partial);
}
template <typename T, int VEC, typename F>
int run_bwd(int sms, bool aligned, Params& p, cudaStream_t stream, F partial) {
  return aligned ? run_bwd_vec<T, VEC>(sms, p, stream, partial) : run_bwd_vec<T, 1>(sms, p, stream, partial);
}

}  // namespace

extern "C" {

int layernorm_fwd(int type, int64_t rows, int64_t cols, const void* X, int64_t ldx, const void* gamma, const void* beta, float eps,
                  void* Y, int64_t ldy, float* mean, float* rstd, void* stream) {
  if (bad_type(type) || !std::isfinite(eps) || eps < 0.f) return DGEMM_ERR_VARIANT;
  if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return DGEMM_ERR_BAD_DIM;
  if (rows == 0 || cols == 0) return DGEMM_OK;
  int rc = check(type, X, rows, cols, ldx);
  if (rc == DGEMM_OK) rc = check(type, Y, rows, cols, ldy);
  if (rc != DGEMM_OK) return rc;
  if ((((uintptr_t)gamma | (uintptr_t)beta) & (elem_bytes(type) - 1)) || (((uintptr_t)mean | (uintptr_t)rstd) & 3)) return DGEMM_ERR_ALIGN;
  const struct { const void* p; int64_t n; } r[] = {{Y, span(type, rows, cols, ldy)}, {mean, rows * 4}, {rstd, rows * 4},
                                                    {X, span(type, rows, cols, ldx)}, {gamma, cols * elem_bytes(type)},
                                                    {beta, cols * elem_bytes(type)}};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 6; ++j)
      if (r[i].p && r[j].p && lm::ranges_overlap(r[i].p, r[i].n, r[j].p, r[j].n)) return DGEMM_ERR_ALIAS;
  lm::DeviceState* st = nullptr;
  if ((rc = lm::device_state(&st)) != DGEMM_OK) return rc;
  Params p;
  memset(&p, 0, sizeof(p));
  p.rows = rows;
  p.cols = (int)cols;
  p.X = X;
  p.ldx = ldx;
  p.gamma = gamma;
  p.beta = beta;
  p.out = Y;
  p.ldo = ldy;
  p.mean = mean;
  p.rstd = rstd;
  p.eps = eps;
  const bool aligned = rows_aligned(type, X, ldx) && rows_aligned(type, Y, ldy) && (((uintptr_t)gamma | (uintptr_t)beta) & 15) == 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool ok = type == HGEMM_TYPE_F32   ? run_fwd<float, 4>(st->sm_count, aligned, p, s)
                  : type == HGEMM_TYPE_F16 ? run_fwd<__half, 8>(st->sm_count, aligned, p, s)
                                           : run_fwd<__nv_bfloat16, 8>(st->sm_count, aligned, p, s);
  return ok ? DGEMM_OK : lm::cuda_failed();
}

int layernorm_bwd(int type, int64_t rows, int64_t cols, const void* X, int64_t ldx, const void* gamma, const float* mean,
                  const float* rstd, const void* dY, int64_t lddy, void* dX, int64_t lddx, float* dgamma, float* dbeta, void* stream) {
  if (bad_type(type)) return DGEMM_ERR_VARIANT;
  if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return DGEMM_ERR_BAD_DIM;
  if (cols == 0) return DGEMM_OK;
  int rc = check(type, X, rows, cols, ldx);
  if (rc == DGEMM_OK) rc = check(type, dY, rows, cols, lddy);
  if (rc == DGEMM_OK && dX) rc = check(type, dX, rows, cols, lddx);
  if (rc != DGEMM_OK) return rc;
  if (rows > 0 && (!mean || !rstd)) return DGEMM_ERR_NULL;
  if (((uintptr_t)gamma & (elem_bytes(type) - 1)) || (((uintptr_t)mean | (uintptr_t)rstd | (uintptr_t)dgamma | (uintptr_t)dbeta) & 3))
    return DGEMM_ERR_ALIGN;
  const struct { const void* p; int64_t n; } r[] = {{dX, span(type, rows, cols, lddx)}, {dgamma, cols * 4}, {dbeta, cols * 4},
                                                    {X, span(type, rows, cols, ldx)}, {gamma, cols * elem_bytes(type)},
                                                    {mean, rows * 4}, {rstd, rows * 4}, {dY, span(type, rows, cols, lddy)}};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 8; ++j)
      if (r[i].p && r[j].p && r[i].n > 0 && r[j].n > 0 && lm::ranges_overlap(r[i].p, r[i].n, r[j].p, r[j].n)) return DGEMM_ERR_ALIAS;
  lm::DeviceState* st = nullptr;
  if ((rc = lm::device_state(&st)) != DGEMM_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    for (float* out : {dgamma, dbeta})
      if (out && cudaMemsetAsync(out, 0, (size_t)cols * 4, s) != cudaSuccess) return lm::cuda_failed();
    return DGEMM_OK;
  }
  if (!dX && !dgamma && !dbeta) return DGEMM_OK;
  Params p;
  memset(&p, 0, sizeof(p));
  p.rows = rows;
  p.cols = (int)cols;
  p.X = X;
  p.ldx = ldx;
  p.gamma = gamma;
  p.dY = dY;
  p.ldy = lddy;
  p.out = dX;
  p.ldo = lddx;
  p.mean = const_cast<float*>(mean);
  p.rstd = const_cast<float*>(rstd);
  p.want_params = dgamma || dbeta;
  p.ldp = (cols + 3) / 4 * 4;
  const bool aligned = rows_aligned(type, X, ldx) && rows_aligned(type, dY, lddy) && (!dX || rows_aligned(type, dX, lddx)) &&
                       ((uintptr_t)gamma & 15) == 0;
  scratch::Hold hold(st->scratch, s);
  const auto partial = [&](int blocks) {
    if (p.want_params) p.partial = static_cast<float*>(hold.workspace((size_t)2 * blocks * p.ldp * 4));
    return !p.want_params || p.partial != nullptr;
  };
  const int blocks = type == HGEMM_TYPE_F32   ? run_bwd<float, 4>(st->sm_count, aligned, p, s, partial)
                     : type == HGEMM_TYPE_F16 ? run_bwd<__half, 8>(st->sm_count, aligned, p, s, partial)
                                              : run_bwd<__nv_bfloat16, 8>(st->sm_count, aligned, p, s, partial);
  if (blocks == 0) return lm::cuda_failed();
  const bool many = blocks > MANY_BLOCKS;
  if (p.want_params && !lm::launch(many ? bwd_reduce_kernel<32> : bwd_reduce_kernel<16>, dim3((unsigned)((cols + 31) / 32), 2),
                                   dim3(many ? 1024 : 512), 0, 1, s, (const float*)p.partial, blocks, (int)cols, (int)p.ldp, dgamma, dbeta))
    return lm::cuda_failed();
  return DGEMM_OK;
}

}  // extern "C"
