// C ABI of layer norm (include/layernorm.h): validation, choice of kernel, launches.
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>

#include <cuda_runtime.h>

#include "../../include/layernorm.h"
#include "layernorm.cuh"
#include "lm_state.h"

namespace {

using namespace lnorm;

constexpr int64_t kMaxDim = (int64_t)INT32_MAX - 65536;

int elem_bytes(int type) { return type == HGEMM_TYPE_F32 ? 4 : 2; }

int check(int type, const void* ptr, int64_t rows, int64_t cols, int64_t ld) {
  if (ld < (cols > 0 ? cols : 1) || ld > (int64_t)1 << 38) return DGEMM_ERR_BAD_LD;
  if (rows == 0 || cols == 0) return DGEMM_OK;
  if (!ptr) return DGEMM_ERR_NULL;
  if ((uintptr_t)ptr & (elem_bytes(type) - 1)) return DGEMM_ERR_ALIGN;
  return DGEMM_OK;
}

int64_t span(int type, int64_t rows, int64_t cols, int64_t ld) { return rows > 0 && cols > 0 ? ((rows - 1) * ld + cols) * elem_bytes(type) : 0; }

bool rows_aligned(int type, const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld * elem_bytes(type) % 16 == 0; }

// How a row is spread over threads: vectors per thread, and threads (32: one warp per row).
struct Shape {
  int items, threads;
  bool longer;  // does not fit in registers
};
// A warp takes a row of up to 4 vectors per lane (no block barrier); longer rows take a block, each thread
// holding as few vectors as 256 threads allow, at most `most`, and then as many threads as needed (`limit` of
// the values a thread holds). `spread`: as many threads as possible instead (few rows: the latency of one
// row counts).
Shape shape_for(int64_t cols, int vec, int most, int (*limit)(int), bool spread) {
  const int64_t nv = (cols + vec - 1) / vec;
  const int warp_items = most < 4 ? most : 4;
  if (nv <= 32 * warp_items && !(spread && nv > 64)) return Shape{nv <= 32 ? 1 : nv <= 64 ? 2 : 4, 32, false};
  int items = 1;
  while (items < most && nv > (int64_t)(spread ? limit(items * vec) : 256) * items) items *= 2;
  const int64_t threads = (nv + items - 1) / items;
  if (threads > limit(items * vec)) return Shape{0, 1024, true};
  return Shape{items, (int)((threads + 31) / 32 * 32), false};
}
int fwd_limit(int values) { return fwd_threads(values); }
int bwd_limit(int) { return BWD_THREADS; }

// Blocks of one kernel (one instance of this function per kernel) that fit on the device at once, or fewer
// for few rows.
template <typename K, K kernel>
unsigned resident_blocks(int sms, int threads, int64_t need) {
  static std::atomic<int> known[33];  // by warps per block; the same on every device of this kind
  int per_sm = known[threads / 32].load();
  if (per_sm == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, 0) != cudaSuccess || per_sm < 1) per_sm = 1;
    known[threads / 32].store(per_sm);
  }
  return (unsigned)(need < (int64_t)sms * per_sm ? need : (int64_t)sms * per_sm);
}

template <typename T, int VEC, int ITEMS>
bool launch_fwd(int sms, const Shape& s, const Params& p, cudaStream_t stream) {
  if constexpr (ITEMS <= 4)
    if (s.threads == 32) {
      const unsigned blocks = resident_blocks<decltype(&fwd_kernel<T, VEC, ITEMS, true>), &fwd_kernel<T, VEC, ITEMS, true>>(sms, 256, (p.rows + 7) / 8);
      return lm::launch(fwd_kernel<T, VEC, ITEMS, true>, dim3(blocks), dim3(256), 0, 1, stream, p);
    }
  const unsigned blocks = resident_blocks<decltype(&fwd_kernel<T, VEC, ITEMS, false>), &fwd_kernel<T, VEC, ITEMS, false>>(sms, s.threads, p.rows);
  return lm::launch(fwd_kernel<T, VEC, ITEMS, false>, dim3(blocks), dim3(s.threads), 0, 1, stream, p);
}
template <typename T, int VEC>
bool launch_fwd_items(int sms, const Shape& s, const Params& p, cudaStream_t stream) {
  switch (s.items) {
    case 1: return launch_fwd<T, VEC, 1>(sms, s, p, stream);
    case 2: return launch_fwd<T, VEC, 2>(sms, s, p, stream);
    case 4: return launch_fwd<T, VEC, 4>(sms, s, p, stream);
    case 8: return VEC <= 4 && launch_fwd<T, VEC <= 4 ? VEC : 1, 8>(sms, s, p, stream);
    case 16: return VEC == 1 && launch_fwd<T, 1, 16>(sms, s, p, stream);
    default: return VEC == 1 && launch_fwd<T, 1, 32>(sms, s, p, stream);
  }
}
template <typename T, int VEC>
bool run_fwd(int sms, bool aligned, const Params& p, cudaStream_t stream) {
  const bool spread = p.rows <= sms;
  const Shape s = aligned ? shape_for(p.cols, VEC, 32 / VEC, fwd_limit, spread) : shape_for(p.cols, 1, 32, fwd_limit, spread);
  if (s.longer) return lm::launch(fwd_long_kernel<T>, dim3((unsigned)p.rows), dim3(1024), 0, 1, stream, p);
  return aligned ? launch_fwd_items<T, VEC>(sms, s, p, stream) : launch_fwd_items<T, 1>(sms, s, p, stream);
}

// Blocks of the backward pass: persistent, two per SM, or fewer for few rows.
int bwd_blocks(int sms, const Shape& s, int64_t rows) {
  const int64_t need = s.longer ? (rows + 15) / 16 : s.threads == 32 ? (rows + 7) / 8 : rows;
  return (int)(need < sms * 2 ? need : sms * 2);
}

template <typename T, int VEC, int ITEMS>
bool launch_bwd(const Shape& s, int blocks, const Params& p, cudaStream_t stream) {
  if constexpr (ITEMS <= 4)
    if (s.threads == 32)
      return lm::launch(bwd_kernel<T, VEC, ITEMS, true>, dim3(blocks), dim3(256), p.want_params ? (size_t)p.cols * 8 : 0, 1, stream, p);
  return lm::launch(bwd_kernel<T, VEC, ITEMS, false>, dim3(blocks), dim3(s.threads), 0, 1, stream, p);
}
template <typename T, int VEC>
bool launch_bwd_items(const Shape& s, int blocks, const Params& p, cudaStream_t stream) {
  switch (s.items) {
    case 1: return launch_bwd<T, VEC, 1>(s, blocks, p, stream);
    case 2: return launch_bwd<T, VEC, 2>(s, blocks, p, stream);
    case 4: return VEC <= 4 && launch_bwd<T, VEC <= 4 ? VEC : 1, 4>(s, blocks, p, stream);
    case 8: return VEC == 1 && launch_bwd<T, 1, 8>(s, blocks, p, stream);
    default: return VEC == 1 && launch_bwd<T, 1, 16>(s, blocks, p, stream);
  }
}
template <typename T, int VEC>
bool run_bwd(const Shape& s, int blocks, bool aligned, const Params& p, cudaStream_t stream) {
  if (s.longer) {
    if (p.out && !lm::launch(bwd_long_kernel<T>, dim3((unsigned)p.rows), dim3(1024), 0, 1, stream, p)) return false;
    return !p.want_params || lm::launch(bwd_long_params_kernel<T>, dim3((unsigned)((p.cols + 255) / 256), blocks), dim3(256), 0, 1, stream, p);
  }
  return aligned ? launch_bwd_items<T, VEC>(s, blocks, p, stream) : launch_bwd_items<T, 1>(s, blocks, p, stream);
}

bool bad_type(int type) { return type != HGEMM_TYPE_F32 && type != HGEMM_TYPE_F16 && type != HGEMM_TYPE_BF16; }

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
  return ok ? DGEMM_OK : DGEMM_ERR_CUDA;
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
      if (out && cudaMemsetAsync(out, 0, (size_t)cols * 4, s) != cudaSuccess) return DGEMM_ERR_CUDA;
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
  const bool aligned = rows_aligned(type, X, ldx) && rows_aligned(type, dY, lddy) && (!dX || rows_aligned(type, dX, lddx)) &&
                       ((uintptr_t)gamma & 15) == 0;
  const int vec = type == HGEMM_TYPE_F32 ? 4 : 8;
  const Shape shape = aligned ? shape_for(cols, vec, 16 / vec, bwd_limit, false) : shape_for(cols, 1, 16, bwd_limit, false);
  const int blocks = bwd_blocks(st->sm_count, shape, rows);
  scratch::Hold hold(st->scratch, s);
  if (p.want_params) {
    p.partial = static_cast<float*>(hold.workspace((size_t)2 * blocks * cols * 4));
    if (!p.partial) return DGEMM_ERR_CUDA;
  }
  const bool ok = type == HGEMM_TYPE_F32   ? run_bwd<float, 4>(shape, blocks, aligned, p, s)
                  : type == HGEMM_TYPE_F16 ? run_bwd<__half, 8>(shape, blocks, aligned, p, s)
                                           : run_bwd<__nv_bfloat16, 8>(shape, blocks, aligned, p, s);
  if (!ok) return DGEMM_ERR_CUDA;
  if (p.want_params && !lm::launch(bwd_reduce_kernel, dim3((unsigned)((cols + 31) / 32), 2), dim3(256), 0, 1, s,
                                   (const float*)p.partial, blocks, (int)cols, dgamma, dbeta))
    return DGEMM_ERR_CUDA;
  return DGEMM_OK;
}

}  // extern "C"
