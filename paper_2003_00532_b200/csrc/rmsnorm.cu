// C ABI of root-mean-square norm (include/rmsnorm.h): validation, choice of kernel, launches.
#include <cmath>
#include <cstdint>
#include <cstring>

#include <cuda_runtime.h>

#include "../../include/rmsnorm.h"
#include "lm_state.h"
#include "rmsnorm.cuh"
#include "row_launch.h"

namespace {

using namespace rmsn;
using namespace rowop;

// How a row is spread over threads: vectors per thread, and threads (32: one warp per row).
struct Shape {
  int items, threads;
  bool longer;  // does not fit in registers
};

// Forward: a warp for rows of up to 16 values per lane; a block with 16 values per thread beyond (or up to 32, for rows
// that need them, and for vectors that are only brought to 8 bits: 2088 x 8192 10.1 -> 9.5 us when chosen, now 9.6). Few rows are spread over as many threads
// as there are vectors, because then the latency of one row counts.
Shape fwd_shape(int64_t rows, int64_t cols, int vec, int sms, bool rows_only) {
  const int64_t nv = (cols + vec - 1) / vec;
  const int most = 32 / vec, warp_most = 16 / vec;
  const bool spread = rows * ((nv + 32 * most - 1) / (32 * most)) < (int64_t)sms * 16;  // warps in all
  if (nv <= 32 || (!spread && nv <= 32 * warp_most)) return Shape{pow2((nv + 31) / 32), 32, false};
  int items = spread ? 1 : (rows_only && vec > 1 && nv > 32 * most ? 32 : 16) / vec;  // (a block has two warps at least)
  while (items < most && threads_for(nv, items) > fwd_threads(items * vec)) items *= 2;
  const int threads = threads_for(nv, items);
  if (threads > fwd_threads(items * vec)) return Shape{0, 1024, true};
  return Shape{items, threads, false};
}
// Backward, by single values or rows too long for the ring: a warp for rows of up to 16 values per lane; a block with 8 values
// per thread beyond (4097 x 1537, binary32: 21 us, with 16 values 24), 16 up to 8192 columns, 32 (`WIDE`) up to 16384.
Shape bwd_shape(int64_t cols, int vec) {
  const int64_t nv = (cols + vec - 1) / vec;
  if (vec == 1 && cols <= 512) return Shape{pow2((nv + 31) / 32), 32, false};
  for (int values = vec == 1 ? 8 : 32; values <= 32; values *= 2)
    if (threads_for(nv, values / vec) <= BWD_THREADS) return Shape{values / vec, threads_for(nv, values / vec), false};
  return Shape{0, 1024, true};
}

// The kernels with rows on their way through shared memory: 16 values per thread (8 for rows of up to 256), so many warps to a row, as
// many groups of them as make 16 warps.
constexpr int64_t RING_COLS = (int64_t)RING_THREADS * 16;
Groups ring_groups(int64_t cols, int values, int threads = RING_THREADS) {  // cols: as wide() gives them
  const int warps = (int)((cols + 32 * values - 1) / (32 * values));
  return Groups{warps, threads / 32 / warps};
}

// Columns that the vectors of a row cover at the most.
int64_t wide(int64_t cols, int vec, bool any) { return any ? cols + vec - 1 : cols; }

// Blocks whose rows are `each` at a time, not more than `blocks` unless that is not even one round: a block's rows have to have the
// same shift, so they lie a multiple of `vec` rows apart (or a part of it, if the leading dimension allows).
int64_t even_blocks(int64_t blocks, int each, const Params& p, int vec, bool any) {
  if (!any || blocks * each >= p.rows) return blocks;
  int period = 1;  // blocks after which shifts repeat
  while ((int64_t)period * each * p.shift_ld % vec != 0) ++period;
  return blocks < period ? period : blocks / period * period;
}

// Blocks of one of them, `bytes` of shared memory per thread at the most; 0 on failure.
template <typename K, K kernel>
int ring_blocks(int sms, const Groups& gr, int bytes, int64_t rows) {
  const int threads = gr.warps * gr.groups * 32;
  if (!allow_smem<K, kernel>(RING_THREADS * bytes)) return 0;
  return (int)resident_blocks<K, kernel>(sms, threads, (size_t)threads * bytes, (rows + gr.groups - 1) / gr.groups);
}
template <typename T, int OUT, int THREADS, bool ANY>
bool launch_fwd_ring(int sms, const Params& p, cudaStream_t stream) {
  constexpr int VEC = 16 / (int)sizeof(T), DEPTH = OUT == OUT_E4M3 && THREADS == RING_THREADS ? 3 : 2;
  constexpr int BYTES = 16 * (int)sizeof(T) * DEPTH * 2;  // of shared memory per thread
  constexpr auto kernel = &fwd_ring_kernel<T, VEC, 16 / VEC, DEPTH, OUT, THREADS, ANY>;
  const Groups gr = ring_groups(wide(p.cols, VEC, ANY), 16, THREADS);
  const int threads = gr.warps * gr.groups * 32, fit = ring_blocks<std::remove_const_t<decltype(kernel)>, kernel>(sms, gr, BYTES, p.rows);
  const int64_t blocks = even_blocks(fit, gr.groups, p, VEC, ANY);
  return fit > 0 && lm::launch(kernel, dim3((unsigned)blocks), dim3(threads), (size_t)threads * BYTES / (p.R ? 1 : 2), 1, stream, p, gr);
}
template <typename T, int OUT, int THREADS, bool ANY>
bool launch_fwd_again(int sms, const Params& p, cudaStream_t stream) {
  constexpr int VEC = 16 / (int)sizeof(T), BYTES = 32 * (int)sizeof(T) * 2 * 2;  // of shared memory per thread
  constexpr auto kernel = &fwd_again_kernel<T, VEC, 32 / VEC, OUT, THREADS, ANY>;
  const Groups gr = ring_groups(wide(p.cols, VEC, ANY), 32, THREADS);
  const int threads = gr.warps * gr.groups * 32, fit = ring_blocks<std::remove_const_t<decltype(kernel)>, kernel>(sms, gr, BYTES, p.rows);
  const int64_t blocks = even_blocks(fit, gr.groups, p, VEC, ANY);
  return fit > 0 && lm::launch(kernel, dim3((unsigned)blocks), dim3(threads), (size_t)threads * BYTES / (p.R ? 1 : 2), 1, stream, p, gr);
}
template <typename T, int VEC, int VALUES, bool ANY, typename F>
int launch_bwd_ring(int sms, Params& p, cudaStream_t stream, F partial) {
  constexpr int DEPTH = 2, BYTES = VALUES * (int)sizeof(T) * DEPTH;  // per stream
  constexpr auto kernel = &bwd_ring_kernel<T, VEC, VALUES / VEC, DEPTH, ANY>;
  const Groups gr = ring_groups(wide(p.cols, VEC, ANY), VALUES);
  const int threads = gr.warps * gr.groups * 32, fit = ring_blocks<std::remove_const_t<decltype(kernel)>, kernel>(sms, gr, 3 * BYTES, p.rows);
  const int blocks = (int)even_blocks(fit, gr.groups, p, VEC, ANY);
  if (fit == 0 || !partial(blocks)) return 0;
  return lm::launch(kernel, dim3(blocks), dim3(threads), (size_t)threads * BYTES * (p.R && p.out ? 3 : 2), 1, stream, p, gr) ? blocks : 0;
}

template <typename T, int VEC, int ITEMS, int OUT, bool ANY>
bool launch_fwd(int sms, const Shape& s, const Params& p, cudaStream_t stream) {
  const auto go = [&](auto k, int threads, int64_t need) {
    constexpr auto kernel = decltype(k)::value;
    const int64_t fit = resident_blocks<std::remove_const_t<decltype(kernel)>, kernel>(sms, threads, 0, need);
    return fit > 0 && lm::launch(kernel, dim3((unsigned)even_blocks(fit, s.threads == 32 ? 4 : 1, p, VEC, ANY)), dim3(threads), 0, 1, stream, p);
  };
  if (s.threads == 32) {
    if constexpr (VEC * ITEMS <= 16)
      return go(std::integral_constant<void (*)(const Params), &fwd_kernel<T, VEC, ITEMS, true, OUT, ANY>>(), 128, (p.rows + 3) / 4);
    return false;
  }
  return go(std::integral_constant<void (*)(const Params), &fwd_kernel<T, VEC, ITEMS, false, OUT, ANY>>(), s.threads, p.rows);
}
template <typename T, int VEC, int OUT, bool ANY>
bool run_fwd_vec(int sms, const Params& p, cudaStream_t stream) {
  const int64_t cols = wide(p.cols, VEC, ANY);
  const Shape s = fwd_shape(p.rows, cols, VEC, sms, OUT == OUT_ROWS);
  // 16-bit rows through shared memory, where there are many. Rows of up to 512 columns (unless misaligned), few rows, single precision
  // and rows to 8 bits without norm: level or slower.
  if constexpr (VEC == 8 && OUT != OUT_ROWS) {
    // (1500 x 1152 Y with residual 4.0 us, in registers 4.6, 700 x 1152 level; misaligned 1000 x 4089 8.2 and 11.3, 500 x 4089 5.8 and 5.1)
    const bool many = p.rows > 2 * (int64_t)sms && p.rows * cols >= (ANY ? 3ll << 20 : 1ll << 20);
    // Beyond 8192 columns, and from 4096 on, 32 values per thread (2000 x 16384 Y with residual 50.0 -> 46.6 us, to 8 bits 44.8 -> 38.0; 6000 x
    // 5120 to 8 bits 36.2, by 16 values about 50; 8192 x 4097 Y 37.9 -> 30.3); aligned and with residual Y is better off with 16
    // (8192 x 4600 49.4, about 53), 8 bits too where 16 leave no warp of a block idle (4097 x 8192 40.0, 41.7), and 8 bits without
    // residual in registers (8192 x 5000 31.2, 39.6).
    if (many && cols > RING_COLS && cols <= 2 * RING_COLS) return launch_fwd_again<T, OUT, RING_THREADS, ANY>(sms, p, stream);
    if (many && cols > RING_COLS / 2 && cols <= RING_COLS && (ANY || (p.R ? OUT == OUT_E4M3 && cols <= RING_COLS - 512 : OUT == OUT_Y)))
      return p.R ? launch_fwd_again<T, OUT, RING_THREADS, ANY>(sms, p, stream) : launch_fwd_again<T, OUT, SMALL_RING_THREADS, ANY>(sms, p, stream);
    // Blocks of 256 threads (8192 x 4096 without a residual: Y 29.1 -> 24.2 us, to 8 bits 27.3 -> 24.1; 1500 x 4000 with one 10.9 -> 9.7 and
    // 10.5 -> 9.2); but with a residual beyond L2 so many streams of reads and writes slow each other down (8192 x 4096: 47.1, 16384 x 2048
    // 46.5), and one block of 512 (42.3), or for shorter rows the registers (42.9), are better.
    if (many && cols > (ANY ? 128 : 512) && cols <= RING_COLS) {
      const bool large = p.R && p.rows * p.cols > 16ll << 20;
      if ((!large || ANY) && cols <= RING_COLS / 2) return launch_fwd_ring<T, OUT, SMALL_RING_THREADS, ANY>(sms, p, stream);
      if (p.R && cols > 2048 && p.rows >= 8 * (int64_t)sms) return launch_fwd_ring<T, OUT, RING_THREADS, ANY>(sms, p, stream);
    }
  }
  if (s.longer) return lm::launch(fwd_long_kernel<T, ANY ? 1 : VEC, OUT>, dim3((unsigned)p.rows), dim3(1024), 0, 1, stream, p);
  if (s.items == 1) return launch_fwd<T, VEC, 1, OUT, ANY>(sms, s, p, stream);
  if (s.items == 2) return launch_fwd<T, VEC, 2, OUT, ANY>(sms, s, p, stream);
  if (s.items == 4) return launch_fwd<T, VEC, 4, OUT, ANY>(sms, s, p, stream);
  if constexpr (VEC <= 4)
    if (s.items == 8) return launch_fwd<T, VEC, 8, OUT, ANY>(sms, s, p, stream);
  if constexpr (VEC == 1)
    return s.items == 16 ? launch_fwd<T, 1, 16, OUT, ANY>(sms, s, p, stream) : launch_fwd<T, 1, 32, OUT, ANY>(sms, s, p, stream);
  return false;
}
// How the matrices of a call lie: rows all 16-byte aligned, all misaligned alike, or each in its own way.
enum class Lie { ALIGNED, ALIKE, MIXED };

template <typename T, int OUT>
bool run_fwd_type(Lie lie, const Params& p, int sms, cudaStream_t stream) {
  constexpr int VEC = 16 / (int)sizeof(T);
  // rows of vectors for less than half a warp: single values keep more lanes busy (16384 x 100, bf16: Y with residual 6.5 us, by vectors 7.3)
  if (p.cols <= 16 * VEC) lie = Lie::MIXED;
  if (lie == Lie::ALIGNED) return run_fwd_vec<T, VEC, OUT, false>(sms, p, stream);
  return lie == Lie::ALIKE ? run_fwd_vec<T, VEC, OUT, true>(sms, p, stream) : run_fwd_vec<T, 1, OUT, false>(sms, p, stream);
}
template <int OUT>
bool run_fwd(int type, Lie lie, const Params& p, const lm::DeviceState* st, cudaStream_t stream) {
  if (type == HGEMM_TYPE_F32) return run_fwd_type<float, OUT>(lie, p, st->sm_count, stream);
  if (type == HGEMM_TYPE_F16) return run_fwd_type<__half, OUT>(lie, p, st->sm_count, stream);
  return run_fwd_type<__nv_bfloat16, OUT>(lie, p, st->sm_count, stream);
}

// How the matrices lie, added one after the other.
class Rows {
 public:
  Rows(int vec, int64_t rows) : vec_(vec), one_(rows == 1) {}
  // (of `bytes` per value; NULL: not there)
  void add(const void* ptr, int64_t ld, int bytes) {
    if (!ptr) return;
    const int s = (int)((uintptr_t)ptr / bytes % vec_), l = one_ ? 0 : (int)(ld % vec_);
    alike_ = alike_ && (!any_ || (s == shift_ && l == ld_));
    any_ = true;
    shift_ = s;
    ld_ = l;
  }
  Lie lie(bool gamma_aligned, Params* p) const {
    p->shift = shift_;
    p->shift_ld = ld_;
    return !alike_ ? Lie::MIXED : shift_ == 0 && ld_ == 0 && gamma_aligned ? Lie::ALIGNED : Lie::ALIKE;
  }

 private:
  int vec_, shift_ = 0, ld_ = 0;
  bool one_, any_ = false, alike_ = true;  // one_: a single row
};

// Blocks of the backward pass: as many as fit at once, but for few rows at least two rows each (every block leaves
// its own sums to be added; 721 x 816, binary32: with eight each 8.5 us, with two 7.4), down to one per SM.
template <typename K, K kernel>
int bwd_blocks(int sms, int threads, size_t smem, int64_t rows, int rows_per_block) {
  const int64_t need = (rows + rows_per_block - 1) / rows_per_block;
  const int64_t some = (int)resident_blocks<K, kernel>(sms, threads, smem, need);
  const int64_t half = (rows + 2 * rows_per_block - 1) / (2 * rows_per_block);
  const int64_t want = half > sms ? half : sms;
  return (int)(some < want ? some : want);
}

// Runs the row kernel; `partial` is asked for the matrix of the blocks' sums. Returns the number of blocks, 0 on failure.
template <typename T, int VEC, int ITEMS, bool WARP_ROW, bool WIDE, bool ANY, typename F>
int launch_bwd(int sms, int threads, Params& p, cudaStream_t stream, F partial) {
  constexpr auto kernel = &bwd_kernel<T, VEC, ITEMS, WARP_ROW, WIDE, ANY>;
  const size_t smem = WIDE ? (size_t)threads * ITEMS * VEC * 8 : WARP_ROW && p.want_params ? (size_t)threads * ITEMS * 4 : 0;
  if (WIDE && !allow_smem<decltype(kernel), kernel>(BWD_THREADS * ITEMS * VEC * 8)) return 0;
  const size_t most = WIDE ? smem : WARP_ROW ? (size_t)threads * ITEMS * 4 : 0;
  const int fit = bwd_blocks<decltype(kernel), kernel>(sms, threads, most, p.rows, WARP_ROW ? 8 : 1);
  const int blocks = (int)even_blocks(fit, WARP_ROW ? 8 : 1, p, VEC, ANY);
  if (fit == 0 || !partial(blocks)) return 0;
  return lm::launch(kernel, dim3(blocks), dim3(threads), smem, 1, stream, p) ? blocks : 0;
}
template <typename T, int VEC, bool ANY, typename F>
int run_bwd_vec(int sms, Params& p, cudaStream_t stream, F partial) {
  const int64_t cols = wide(p.cols, VEC, ANY);
  if constexpr (VEC == 8)
    if (cols > (!ANY && p.rows > 2 * (int64_t)sms ? RING_COLS / 2 : RING_COLS) && cols <= RING_COLS * 2) return launch_bwd_ring<T, VEC, 32, ANY>(sms, p, stream, partial);
  if constexpr (VEC > 1) {
    if constexpr (!ANY)  // (misaligned rows of up to 256 columns go by single values)
      if (cols <= 256) return launch_bwd_ring<T, VEC, 8, false>(sms, p, stream, partial);
    if (cols <= RING_COLS) return launch_bwd_ring<T, VEC, 16, ANY>(sms, p, stream, partial);
  }
  const Shape s = bwd_shape(cols, VEC);
  if (s.longer) {
    const int chunks = (int)((p.rows + 15) / 16 < sms * 2 ? (p.rows + 15) / 16 : sms * 2);
    if (!partial(chunks)) return 0;
    if (p.out && !lm::launch(bwd_long_kernel<T, ANY ? 1 : VEC>, dim3((unsigned)p.rows), dim3(1024), 0, 1, stream, p)) return 0;
    if (p.want_params && !lm::launch(bwd_long_params_kernel<T>, dim3((unsigned)((p.cols + 255) / 256), chunks), dim3(256), 0, 1, stream, p))
      return 0;
    return chunks;
  }
  if constexpr (VEC == 1) {
    if (s.threads == 32) {
      if (s.items == 1) return launch_bwd<T, 1, 1, true, false, false>(sms, 256, p, stream, partial);
      if (s.items == 2) return launch_bwd<T, 1, 2, true, false, false>(sms, 256, p, stream, partial);
      if (s.items == 4) return launch_bwd<T, 1, 4, true, false, false>(sms, 256, p, stream, partial);
      if (s.items == 8) return launch_bwd<T, 1, 8, true, false, false>(sms, 256, p, stream, partial);
      return launch_bwd<T, 1, 16, true, false, false>(sms, 256, p, stream, partial);
    }
    if (s.items == 8) return launch_bwd<T, 1, 8, false, false, false>(sms, s.threads, p, stream, partial);
    if (s.items == 16) return launch_bwd<T, 1, 16, false, false, false>(sms, s.threads, p, stream, partial);
  }
  if constexpr (VEC != 8) return launch_bwd<T, VEC, 32 / VEC, false, true, ANY>(sms, s.threads, p, stream, partial);
  return 0;
}
template <typename T, typename F>
int run_bwd(int sms, Lie lie, Params& p, cudaStream_t stream, F partial) {
  constexpr int VEC = 16 / (int)sizeof(T);
  // misaligned rows: short ones or little of them by single values (16384 x 99, bf16: 10.0 us, by vectors 14.3; 721 x 816, binary32: 7.0 and 7.7; 64 x
  // 4097 5.9 and 6.9)
  if (lie == Lie::ALIKE && p.cols <= RING_COLS && (p.cols <= 256 || p.rows * p.cols < 1ll << 20)) lie = Lie::MIXED;
  if (lie == Lie::ALIGNED) return run_bwd_vec<T, VEC, false>(sms, p, stream, partial);
  return lie == Lie::ALIKE ? run_bwd_vec<T, VEC, true>(sms, p, stream, partial) : run_bwd_vec<T, 1, false>(sms, p, stream, partial);
}

struct Range {
  const void* ptr;
  int64_t bytes;
};
// Outputs must not overlap inputs or one another; the first `nout` ranges are the outputs.
bool aliased(const Range* r, int nout, int n) {
  for (int i = 0; i < nout; ++i)
    for (int j = i + 1; j < n; ++j)
      if (r[i].ptr && r[j].ptr && r[i].bytes > 0 && r[j].bytes > 0 && lm::ranges_overlap(r[i].ptr, r[i].bytes, r[j].ptr, r[j].bytes))
        return true;
  return false;
}

// The forward pass in its three forms.
template <int OUT>
int forward(int type, int64_t rows, int64_t cols, const void* X, int64_t ldx, const void* R, int64_t ldr, const void* gamma, float eps,
            void* S, int64_t lds, void* out, int64_t ldo, float* scale, float* rstd, cudaStream_t stream) {
  constexpr bool EIGHT = OUT != OUT_Y;
  if (bad_type(type) || !std::isfinite(eps) || eps < 0.f) return DGEMM_ERR_VARIANT;
  if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return DGEMM_ERR_BAD_DIM;
  if (rows == 0 || cols == 0) return DGEMM_OK;
  int rc = check(type, X, rows, cols, ldx);
  if (rc == DGEMM_OK && R) rc = check(type, R, rows, cols, ldr);
  if (rc == DGEMM_OK && S) rc = check(type, S, rows, cols, lds);
  if (rc != DGEMM_OK) return rc;
  if (EIGHT) {
    if (ldo < cols || ldo > (int64_t)1 << 38) return DGEMM_ERR_BAD_LD;
    if (!out || !scale) return DGEMM_ERR_NULL;
  } else if ((rc = check(type, out, rows, cols, ldo)) != DGEMM_OK) {
    return rc;
  }
  if (((uintptr_t)gamma & (elem_bytes(type) - 1)) || (((uintptr_t)scale | (uintptr_t)rstd) & 3)) return DGEMM_ERR_ALIGN;
  // S in the place of an input: the same values in the same places
  const bool on_x = S && S == X && lds == ldx, on_r = S && R && S == R && lds == ldr;
  const int64_t nx = span(type, rows, cols, ldx), nr = R ? span(type, rows, cols, ldr) : 0, ns = S ? span(type, rows, cols, lds) : 0;
  const int64_t no = EIGHT ? (rows - 1) * ldo + cols : span(type, rows, cols, ldo);
  const Range r[] = {{S, ns}, {out, no}, {rstd, rows * 4}, {scale, rows * 4}, {gamma, cols * elem_bytes(type)}, {on_x ? nullptr : X, nx}, {on_r ? nullptr : R, nr}};
  if (aliased(r, 4, 7)) return DGEMM_ERR_ALIAS;
  lm::DeviceState* st = nullptr;
  if ((rc = lm::device_state(&st)) != DGEMM_OK) return rc;
  Params p;
  memset(&p, 0, sizeof(p));
  p.rows = rows;
  p.cols = (int)cols;
  p.X = X;
  p.ldx = ldx;
  p.R = R;
  p.ldr = R ? ldr : 0;
  p.gamma = gamma;
  p.eps = eps;
  p.S = S;
  p.lds = S ? lds : 0;
  p.out = out;
  p.ldo = ldo;
  p.scale = scale;
  p.rstd = rstd;
  const int e = elem_bytes(type);
  Rows lies(16 / e, rows);
  lies.add(X, ldx, e);
  lies.add(R, ldr, e);
  lies.add(S, lds, e);
  lies.add(out, ldo, EIGHT ? 1 : e);
  return run_fwd<OUT>(type, lies.lie(((uintptr_t)gamma & 15) == 0, &p), p, st, stream) ? DGEMM_OK : lm::cuda_failed();
}

}  // namespace

extern "C" {

int rmsnorm_fwd(int type, int64_t rows, int64_t cols, const void* X, int64_t ldx, const void* R, int64_t ldr, const void* gamma, float eps,
                void* S, int64_t lds, void* Y, int64_t ldy, float* rstd, void* stream) {
  return forward<OUT_Y>(type, rows, cols, X, ldx, R, ldr, gamma, eps, S, lds, Y, ldy, nullptr, rstd, static_cast<cudaStream_t>(stream));
}

int rmsnorm_fwd_e4m3(int type, int64_t rows, int64_t cols, const void* X, int64_t ldx, const void* R, int64_t ldr, const void* gamma,
                     float eps, void* S, int64_t lds, void* Q, int64_t ldq, float* scale, float* rstd, void* stream) {
  return forward<OUT_E4M3>(type, rows, cols, X, ldx, R, ldr, gamma, eps, S, lds, Q, ldq, scale, rstd, static_cast<cudaStream_t>(stream));
}

int quantize_rows_e4m3(int type, int64_t rows, int64_t cols, const void* X, int64_t ldx, void* Q, int64_t ldq, float* scale, void* stream) {
  return forward<OUT_ROWS>(type, rows, cols, X, ldx, nullptr, 0, nullptr, 0.f, nullptr, 0, Q, ldq, scale, nullptr,
                           static_cast<cudaStream_t>(stream));
}

int rmsnorm_bwd(int type, int64_t rows, int64_t cols, const void* S, int64_t lds, const void* gamma, const float* rstd, const void* dY,
                int64_t lddy, const void* dS, int64_t ldds, void* dX, int64_t lddx, float* dgamma, void* stream) {
  if (bad_type(type)) return DGEMM_ERR_VARIANT;
  if (rows < 0 || cols < 0 || rows > kMaxDim || cols > kMaxDim) return DGEMM_ERR_BAD_DIM;
  if (cols == 0) return DGEMM_OK;
  int rc = check(type, S, rows, cols, lds);
  if (rc == DGEMM_OK) rc = check(type, dY, rows, cols, lddy);
  if (rc == DGEMM_OK && dS) rc = check(type, dS, rows, cols, ldds);
  if (rc == DGEMM_OK && dX) rc = check(type, dX, rows, cols, lddx);
  if (rc != DGEMM_OK) return rc;
  if (rows > 0 && !rstd) return DGEMM_ERR_NULL;
  if (((uintptr_t)gamma & (elem_bytes(type) - 1)) || (((uintptr_t)rstd | (uintptr_t)dgamma) & 3)) return DGEMM_ERR_ALIGN;
  const bool in_place = dX && dX == dS && lddx == ldds;
  const Range r[] = {{dX, span(type, rows, cols, lddx)}, {dgamma, cols * 4}, {S, span(type, rows, cols, lds)}, {gamma, cols * elem_bytes(type)},
                     {rstd, rows * 4}, {dY, span(type, rows, cols, lddy)}, {in_place ? nullptr : dS, span(type, rows, cols, ldds)}};
  if (aliased(r, 2, 7) || (in_place && dgamma && lm::ranges_overlap(dgamma, cols * 4, dS, span(type, rows, cols, ldds)))) return DGEMM_ERR_ALIAS;
  lm::DeviceState* st = nullptr;
  if ((rc = lm::device_state(&st)) != DGEMM_OK) return rc;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    if (dgamma && cudaMemsetAsync(dgamma, 0, (size_t)cols * 4, s) != cudaSuccess) return lm::cuda_failed();
    return DGEMM_OK;
  }
  if (!dX && !dgamma) return DGEMM_OK;
  Params p;
  memset(&p, 0, sizeof(p));
  p.rows = rows;
  p.cols = (int)cols;
  p.X = S;
  p.ldx = lds;
  p.gamma = gamma;
  p.dY = dY;
  p.ldy = lddy;
  p.R = dX ? dS : nullptr;
  p.ldr = p.R ? ldds : 0;
  p.out = dX;
  p.ldo = dX ? lddx : 0;
  p.rstd = const_cast<float*>(rstd);
  p.want_params = dgamma != nullptr;
  p.ldp = (cols + 3) / 4 * 4;
  const int e = elem_bytes(type);
  Rows lies(16 / e, rows);
  lies.add(S, lds, e);
  lies.add(dY, lddy, e);
  lies.add(p.R, p.ldr, e);
  lies.add(dX, lddx, e);
  const Lie lie = lies.lie(((uintptr_t)gamma & 15) == 0, &p);
  scratch::Hold hold(st->scratch, s);
  const auto partial = [&](int blocks) {
    if (p.want_params) p.partial = static_cast<float*>(hold.workspace((size_t)blocks * p.ldp * 4));
    return !p.want_params || p.partial != nullptr;
  };
  const int blocks = type == HGEMM_TYPE_F32   ? run_bwd<float>(st->sm_count, lie, p, s, partial)
                     : type == HGEMM_TYPE_F16 ? run_bwd<__half>(st->sm_count, lie, p, s, partial)
                                              : run_bwd<__nv_bfloat16>(st->sm_count, lie, p, s, partial);
  if (blocks == 0) return lm::cuda_failed();
  const bool many = blocks > lnorm::MANY_BLOCKS;
  if (p.want_params && !lm::launch(many ? lnorm::bwd_reduce_kernel<32> : lnorm::bwd_reduce_kernel<16>, dim3((unsigned)((cols + 31) / 32)),
                                   dim3(many ? 1024 : 512), 0, 1, s, (const float*)p.partial, blocks, (int)cols, (int)p.ldp, dgamma,
                                   (float*)nullptr))
    return lm::cuda_failed();
  return DGEMM_OK;
}

}  // extern "C"
