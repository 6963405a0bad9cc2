// C ABI of dropout (include/dropout.h): validation, launches.
#include <cstdint>
#include <cstring>

#include <cuda_runtime.h>

#include "../../include/dropout.h"
#include "dropout.cuh"
#include "lm_state.h"
#include "row_launch.h"

namespace {

using namespace drop;
using namespace rowop;

template <typename T, int VEC, bool ALIGNED>
bool run(int sms, Params& p, cudaStream_t stream) {
  constexpr int UNROLL = 2;
  p.nv = (p.cols + VEC - 1) / VEC;
  const auto kernel = &dropout_kernel<T, VEC, ALIGNED, UNROLL>;
  const int64_t need = (p.rows * p.nv + (int64_t)THREADS * UNROLL - 1) / ((int64_t)THREADS * UNROLL), most = (int64_t)sms * 8;
  return lm::launch(kernel, dim3((unsigned)(need < most ? need : most)), dim3(THREADS), 0, 1, stream, p);
}

int dropout(int type, int64_t rows, int64_t cols, const void* X, int64_t ldx, const void* R, int64_t ldr, double prob, uint64_t seed,
            uint64_t offset, const int64_t* step, void* Y, int64_t ldy, cudaStream_t stream) {
  if (bad_type(type) || !(prob >= 0.0 && prob <= 1.0)) return DGEMM_ERR_VARIANT;
  if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return DGEMM_ERR_BAD_DIM;
  if (rows == 0 || cols == 0) return DGEMM_OK;
  int rc = check(type, X, rows, cols, ldx);
  if (rc == DGEMM_OK && R) rc = check(type, R, rows, cols, ldr);
  if (rc == DGEMM_OK) rc = check(type, Y, rows, cols, ldy);
  if (rc != DGEMM_OK) return rc;
  if ((uintptr_t)step & 7) return DGEMM_ERR_ALIGN;
  const int64_t nx = span(type, rows, cols, ldx), nr = R ? span(type, rows, cols, ldr) : 0, ny = span(type, rows, cols, ldy);
  if (!(Y == X && ldy == ldx) && lm::ranges_overlap(Y, ny, X, nx)) return DGEMM_ERR_ALIAS;
  if (R && !(Y == R && ldy == ldr) && lm::ranges_overlap(Y, ny, R, nr)) return DGEMM_ERR_ALIAS;
  if (step && lm::ranges_overlap(Y, ny, step, 8)) return DGEMM_ERR_ALIAS;
  lm::DeviceState* st = nullptr;
  if ((rc = lm::device_state(&st)) != DGEMM_OK) return rc;
  Params p;
  memset(&p, 0, sizeof(p));
  p.rows = rows;
  p.cols = (int)cols;
  const uint64_t threshold = (uint64_t)(prob * 4294967296.0 + 0.5);
  p.none = threshold >> 32 != 0;
  p.threshold = (uint32_t)threshold;
  p.scale = (float)(1.0 / (1.0 - prob));
  p.key0 = (uint32_t)seed;
  p.key1 = (uint32_t)(seed >> 32);
  p.offset = offset;
  p.step = reinterpret_cast<const long long*>(step);
  p.X = X;
  p.ldx = ldx;
  p.R = R;
  p.ldr = R ? ldr : 0;
  p.Y = Y;
  p.ldy = ldy;
  const bool aligned = rows_aligned(type, X, ldx) && (!R || rows_aligned(type, R, ldr)) && rows_aligned(type, Y, ldy);
  const int sms = st->sm_count;
  const bool ok = type == HGEMM_TYPE_F32   ? (aligned ? run<float, 4, true>(sms, p, stream) : run<float, 4, false>(sms, p, stream))
                  : type == HGEMM_TYPE_F16 ? (aligned ? run<__half, 8, true>(sms, p, stream) : run<__half, 4, false>(sms, p, stream))
                                           : (aligned ? run<__nv_bfloat16, 8, true>(sms, p, stream) : run<__nv_bfloat16, 4, false>(sms, p, stream));
  return ok ? DGEMM_OK : lm::cuda_failed();
}

}  // namespace

extern "C" {

int dropout_fwd(int type, int64_t rows, int64_t cols, const void* X, int64_t ldx, const void* R, int64_t ldr, double p, uint64_t seed,
                uint64_t offset, const int64_t* step, void* Y, int64_t ldy, void* stream) {
  return dropout(type, rows, cols, X, ldx, R, ldr, p, seed, offset, step, Y, ldy, static_cast<cudaStream_t>(stream));
}

int dropout_bwd(int type, int64_t rows, int64_t cols, const void* dY, int64_t lddy, double p, uint64_t seed, uint64_t offset,
                const int64_t* step, void* dX, int64_t lddx, void* stream) {
  return dropout(type, rows, cols, dY, lddy, nullptr, 0, p, seed, offset, step, dX, lddx, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
