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

// Vectors and rows of a block: whole rows, or strips of equal width where they have over 256 vectors; as many rows as
// leave the fewest threads of the last warp idle.
Shape shape_of(int nv) {
  const int strips = (nv + MAX_THREADS - 1) / MAX_THREADS, tx = (nv + strips - 1) / strips;
  Shape best{tx, 1};
  double most = 0.0;
  for (int ty = 1; ty * tx <= MAX_THREADS; ++ty) {
    const double used = (double)(ty * tx) / ((ty * tx + 31) / 32 * 32);
    if (used >= most - 0.02) {
      best.ty = ty;
      if (used > most) most = used;
    }
  }
  return best;
}

template <typename T, int VEC, bool RES>
bool launch(int sms, const Params& p, cudaStream_t stream) {
  constexpr auto kernel = &dropout_kernel<T, VEC, RES>;
  const Shape s = shape_of(p.nv);
  const int threads = (s.tx * s.ty + 31) / 32 * 32;
  const int64_t strips = (p.nv + s.tx - 1) / s.tx, steps = (p.rows + s.ty - 1) / s.ty;
  const int64_t resident = resident_blocks<std::remove_const_t<decltype(kernel)>, kernel>(sms, threads, 0, INT32_MAX);
  if (resident == 0) return false;
  // blocks down the rows: as many as fit at once, each with the same number of steps
  int64_t most = resident / strips;
  if (most < 1) most = 1;
  if (most > 65535) most = 65535;
  const int64_t each = (steps + most - 1) / most;
  return lm::launch(kernel, dim3((unsigned)strips, (unsigned)((steps + each - 1) / each)), dim3(threads), 0, 1, stream, p, s);
}
template <typename T, bool RES>
bool launch_any(int sms, const Params& p, cudaStream_t stream) {
  constexpr auto kernel = &dropout_any_kernel<T, RES>;
  const int64_t resident = resident_blocks<std::remove_const_t<decltype(kernel)>, kernel>(sms, 256, 0, INT32_MAX);
  if (resident == 0) return false;
  int64_t sweep = resident * 8 / p.nv;  // rows at a time
  if (sweep < 1) sweep = 1;
  const int64_t each = (p.rows + sweep - 1) / sweep;
  sweep = (p.rows + each - 1) / each;
  return lm::launch(kernel, dim3((unsigned)((sweep * p.nv + 7) / 8)), dim3(256), 0, 1, stream, p, (int)sweep);
}
template <typename T, int VEC>
bool run(int sms, bool aligned, Params& p, cudaStream_t stream) {
  const int per = aligned ? VEC : 128;
  p.nv = (p.cols + per - 1) / per;
  if (!aligned) return p.R ? launch_any<T, true>(sms, p, stream) : launch_any<T, false>(sms, p, stream);
  return p.R ? launch<T, VEC, true>(sms, p, stream) : launch<T, VEC, false>(sms, p, stream);
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
  p.scale = prob < 1.0 ? (float)(1.0 / (1.0 - prob)) : 0.f;
  for (int i = 0; i < 10; ++i) {
    p.key[0][i] = (uint32_t)seed + i * W0;
    p.key[1][i] = (uint32_t)(seed >> 32) + i * W1;
  }
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
  const bool ok = type == HGEMM_TYPE_F32   ? run<float, 4>(sms, aligned, p, stream)
                  : type == HGEMM_TYPE_F16 ? run<__half, 8>(sms, aligned, p, stream)
                                           : run<__nv_bfloat16, 8>(sms, aligned, p, stream);
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
