// C ABI of the 16-bit products (include/hgemm.h) and those of 8-bit operands (include/qgemm.h): validation, packing of
// operands TMA cannot address, choice of tile and work decomposition, tensor maps, launches.
#include <atomic>
#include <cstdint>
#include <cstring>
#include <mutex>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/hgemm.h"
#include "../../include/qgemm.h"
#include "hgemm_aux.cuh"
#include "hgemm_kernels.h"
#include "lm_state.h"

namespace {

using namespace hgemm;

constexpr int kMaxDevices = 64;
constexpr unsigned long long kWaitLimitNs = 4000000000ull;  // bounded device-side waits give up after 4 s
constexpr int64_t kMaxDim = (int64_t)INT32_MAX - 1024;

__device__ int g_hgemm_status_word;
__device__ int g_hgemm_counters[scratch::kMaxLeases * lm::kCounters];

lm::DeviceState g_dev[kMaxDevices];
std::mutex g_mutex;
lm::EncodeTiledFn g_encode = nullptr;
std::atomic<int> g_drop_limit_us{0};

// ---- kernels by type --------------------------------------------------------------------------------

bool launch_tc(int type, bool eight, bool gated, int act, int config, int clusters, cudaStream_t stream, const Params& p) {
  if (eight) {
    if (type == HGEMM_TYPE_BF16)
      return gated ? launch_gated8_bf16(act, config, clusters, stream, p) : launch_plain8_bf16(act, config, clusters, stream, p);
    return gated ? launch_gated8_f16(act, config, clusters, stream, p) : launch_plain8_f16(act, config, clusters, stream, p);
  }
  if (type == HGEMM_TYPE_BF16)
    return gated ? launch_gated_bf16(act, config, clusters, stream, p) : launch_plain_bf16(act, config, clusters, stream, p);
  return gated ? launch_gated_f16(act, config, clusters, stream, p) : launch_plain_f16(act, config, clusters, stream, p);
}

// ---- work decomposition -------------------------------------------------------------------------------

// Sizes of one product: output columns N (lanes) and rows M, k-blocks, and the clocks a CTA's epilogue takes per
// row of the output.
struct Size {
  int64_t N, M;
  int kblocks;
  double epilogue;
};
// Clocks per output row of a tile's epilogue in one CTA: a plain store, what the activation adds, each further
// matrix with 16-byte aligned rows, and what a matrix that moves value by value adds (outputs; the residual). For the
// last two the time of 1000 x 1536 x 64 rises by 0.9 us; 13 to 25 clocks give the same time within 0.4 % over 99 ragged sizes.
// GELU's exact form takes 1.4 of what its tanh form adds (4096 x 9472 x 64: 34.6 us without activation, 59.5, 52.8), SiLU 0.83;
// as an estimate 60 serves it better than 30 (15 shapes with GELU: 16.70 us in the geometric mean against 16.86, 45 16.77).
double epilogue_clocks(int act, int matrices, int unaligned_out, bool unaligned_res) {
  const double f = act == HGEMM_ACT_NONE || act == HGEMM_ACT_RELU ? 0.0 : act == HGEMM_ACT_GELU ? 60.0 : 20.0;
  return 10.0 + f + 10.0 * (matrices - 1) + 16.0 * unaligned_out + (unaligned_res ? 13.0 : 0.0);
}

struct Plan {
  int config = 0;
  int clusters = 0;
  int nt = 0;
  struct Part {
    int tiles_n, tiles_m, rounds, rest, skip, span_len;
  } part[MAX_PROBLEMS];
  int rounds = 0, rest = 0;
  int span = 0, span_total = 0;  // positions per cluster and in all of the tiles left over; span 0: run whole
  size_t workspace = 0;          // bytes
};

// The model of a launch's time in clocks. Its constants were fitted to 20 shapes in every configuration and cut that
// could win (M 1 .. 4096, N 128 .. 16384, K 64 .. 8192): the pick's time is 1.3 % above the best one's in the
// geometric mean.
constexpr double kL2BytesPerClock = 43.5;  // operand bytes into one SM
constexpr double kKBlockClocks = 510.0;    // least time of a k-block
constexpr double kUnitClocks = 1700.0;     // start and end of a unit of work
constexpr double kLaunchClocks = 6700.0;
constexpr double kRoundColumn = 10.0;      // what an epilogue takes more while other tiles are on their way, per row
                                           // (one k-block per tile: 2800, 4100, 6500 clocks a round for 64, 128, 256 rows)
constexpr double kPartColumn = 20.0;       // a part's sums to the workspace, per row of the output
constexpr double kJoinColumn = 8.0;        // adding one part, per row of the output
constexpr double kJoinClocks = 4500.0;     // publishing the parts and finding the last one

constexpr double kWideKBlockClocks = 1270.0;  // of a 512 x 256 tile
// A 512 x 256 tile's two accumulators fill TMEM: its epilogue stands beside little of the next tile's MMAs. Per row of
// the output: a part of its own and most of an ordinary epilogue, for each of the two.
constexpr double kWideEpilogue = 20.0, kWideShare = 0.85;

// Clocks of one k-block in a CTA: its MMAs (8192 flop per clock), or its operand bytes.
double step_clocks(const Config& c) {
  if (c.nb == 2) return kWideKBlockClocks;
  const double mma = 2.16 * c.bm, bytes = (16384.0 + 128.0 * (c.bm / c.cg < 64 ? 64 : c.bm / c.cg)) / kL2BytesPerClock;
  const double t = mma > bytes ? mma : bytes;
  return t > kKBlockClocks ? t : kKBlockClocks;
}

// Decomposes the problems (longest contraction first) for one configuration and returns the estimated clocks: whole
// rounds of tiles, then the tiles left over, whole or as spans of `span` positions per cluster. -1: too many tiles.
// A position is a k-block; where products of unlike lengths share a launch, a tile whose k-blocks take less time than its
// epilogue has positions for the rest of that time (`skip`, before its k-blocks), or a cluster's span would be a dozen
// epilogues long and another's none (gated gradients 1 x 4485 x 1312: 91 -> 39 us, linear
// gradients 16 x 4096 x 4096: 80 -> 30, 5451 x 280 x 7032: 128 -> 79).
struct Layout {
  int64_t tiles[MAX_PROBLEMS], rounds[MAX_PROBLEMS], rest[MAX_PROBLEMS];
  int64_t left, left_positions;
  int skip[MAX_PROBLEMS], most_skip;
  int clusters, nt, longest;  // longest: positions of the longest tile left over
  double step, epi, fixed;    // fixed: all but the tiles left over
};
bool lay_out(const Size* sz, int n, bool gated, int sms, int config, Layout* out) {
  const Config& c = kConfigs[config];
  Layout l;
  l.clusters = sms / c.cg;
  l.nt = (gated ? 64 : 128) * c.cg * c.nb;
  l.step = step_clocks(c);
  l.epi = 0.0;
  l.left = l.left_positions = 0;
  l.longest = l.most_skip = 0;
  for (int i = 0; i < n; ++i)
    if (sz[i].epilogue * c.bm > l.epi) l.epi = sz[i].epilogue * c.bm;
  l.fixed = kLaunchClocks + l.epi;
  l.epi += kRoundColumn * c.bm;
  for (int i = 0; i < n; ++i) {
    l.tiles[i] = ((sz[i].N + l.nt - 1) / l.nt) * ((sz[i].M + c.bm - 1) / c.bm);
    if (l.tiles[i] > INT32_MAX / 64) return false;
    l.rounds[i] = l.tiles[i] / l.clusters;
    l.rest[i] = l.tiles[i] % l.clusters;
    l.left += l.rest[i];
    const int least = (int)(((sz[i].epilogue + kRoundColumn) * c.bm + kUnitClocks) / l.step);
    l.skip[i] = n > 1 && sz[i].kblocks < least ? least - sz[i].kblocks : 0;
    l.left_positions += l.rest[i] * (sz[i].kblocks + l.skip[i]);
    if (l.rest[i] > 0 && sz[i].kblocks + l.skip[i] > l.longest) l.longest = sz[i].kblocks + l.skip[i];
    if (l.skip[i] > l.most_skip) l.most_skip = l.skip[i];
    // a round is as long as a tile's MMAs, or as an epilogue (which runs beside the next tile's MMAs)
    const double mma = sz[i].kblocks * l.step;
    if (c.nb == 2) l.fixed += (double)l.rounds[i] * (mma + 2 * c.bm * (kWideEpilogue + kWideShare * sz[i].epilogue));
    else l.fixed += (double)l.rounds[i] * ((mma > l.epi ? mma : l.epi) + kUnitClocks);
  }
  *out = l;
  return true;
}
// Whether 512 x 256 tiles are worth a thought: they move a quarter less from L2 per product, which pays where the power
// limit holds the clock down for long, and lose where tiles are few or short. Sustained, against 256 x 256: 8192 x
// 4096 x 8192 466 -> 447 us, gated gradients 4096 x 8192 x 2048 548 -> 503, gated 8192 x 4096 x 8192 880 -> 755; but
// 4096 x 9472 x 4096 (64 k-blocks) 243 -> 297, 2048 x 2048 x 8192 (half a round) 60 -> 93. Between 64 and 128 k-blocks, over
// three shapes, where the estimate takes them (sustained): 8192 x 8192 at 88 650 -> 621, 96 708 -> 666, 128 938 -> 870; 4096 x
// 7168 at 112 390 -> 368, 128 444 -> 420; gated 8192 x 4096 at 72 505 -> 466, 96 670 -> 624, 128 906 -> 831; below those the
// estimate leaves them aside (level within 0.5 %). So they would already pay from 72 on, by 4 to 8 %, where the rule waits for 96.
bool wide_tiles(const Layout& l, const Size* sz, int n) {
  int64_t tiles = 0, kblocks = 0;
  for (int i = 0; i < n; ++i) {
    tiles += l.tiles[i];
    kblocks += l.tiles[i] * sz[i].kblocks;
  }
  return tiles >= 3 * (int64_t)l.clusters && kblocks >= 96 * tiles;
}
// The tiles left over, run whole: rounds over the clusters, each as long as its longest tile.
double whole_clocks(const Layout& l, const Size* sz, int n) {
  double clocks = 0.0;
  int64_t at = 0;
  int i = 0;
  int64_t end = l.rest[0];
  while (at < l.left) {
    while (at >= end) end += l.rest[++i];
    const double mma = sz[i].kblocks * l.step;
    clocks += (mma > l.epi || at + l.clusters >= l.left ? mma : l.epi) + kUnitClocks;
    at += l.clusters;
  }
  return clocks;
}
// ... or in spans. `even`: every tile is cut alike, each part by a cluster of its own; otherwise a span holds the end of
// one tile, whole ones and the beginning of another.
double span_clocks(const Layout& l, const Config& c, int64_t span, bool even) {
  const double write = kPartColumn * c.bm, mma = span * l.step;
  const int64_t parts = (l.longest + span - 1) / span + (even ? 0 : 1);
  const int64_t pieces = even ? 1 : 1 + (span * l.left + l.left_positions - 1) / l.left_positions;
  return (mma > write ? mma : write) + pieces * kUnitClocks + write + kJoinColumn * c.bm * parts + kJoinClocks;
}

// The configuration and cut with the smallest estimate.
bool make_plan(const Size* sz, int n, bool gated, int sms, Plan* best) {
  double best_clocks = -1.0;
  int64_t max_m = 0;
  for (int i = 0; i < n; ++i)
    if (sz[i].M > max_m) max_m = sz[i].M;
  Layout pick;
  int config = -1;
  int64_t pick_span = 0;
  bool pick_even = false;
  for (int c = 0; c < kNumConfigs; ++c) {
    if (c > 0 && kConfigs[c - 1].cg == 1 && kConfigs[c - 1].bm >= max_m) break;  // only more padding
    Layout l;
    if (!lay_out(sz, n, gated, sms, c, &l) || (kConfigs[c].nb == 2 && !wide_tiles(l, sz, n))) continue;
    const auto consider = [&](double t, int64_t span, bool even) {
      if (best_clocks >= 0.0 && t >= best_clocks) return;
      best_clocks = t;
      pick = l;
      config = c;
      pick_span = span;
      pick_even = even;
    };
    consider(l.fixed + (l.left > 0 ? whole_clocks(l, sz, n) : 0.0), 0, false);
    if (l.left == 0 || l.left * kConfigs[c].cg * kConfigs[c].nb > lm::kCounters || l.left_positions > INT32_MAX / 2) continue;
    // equal spans over all clusters, or over half or a quarter of them where joining many parts costs more
    for (int divide = 1; divide <= 4; divide *= 2) {
      int64_t span = (l.left_positions * divide + l.clusters - 1) / l.clusters;
      if (span >= l.longest) break;
      if (span > l.most_skip)  // (no span without a k-block)
        consider(l.fixed + span_clocks(l, kConfigs[c], span, false), span, false);
    }
    const int64_t cut = l.clusters / l.left;
    if (n == 1 && cut > 1 && l.longest > 1) {
      const int64_t span = (l.longest + cut - 1) / cut;
      if (span < l.longest) consider(l.fixed + span_clocks(l, kConfigs[c], span, true), span, true);
    }
  }
  if (config < 0) return false;
  const Config& c = kConfigs[config];
  Plan pl;
  pl.config = config;
  pl.nt = pick.nt;
  for (int i = 0; i < n; ++i) {
    Plan::Part& q = pl.part[i];
    q.tiles_n = (int)((sz[i].N + pick.nt - 1) / pick.nt);
    q.tiles_m = (int)((sz[i].M + c.bm - 1) / c.bm);
    q.rounds = (int)pick.rounds[i];
    q.rest = (int)pick.rest[i];
    q.skip = pick_even ? 0 : pick.skip[i];
    q.span_len = (int)(pick_even ? (sz[i].kblocks + pick_span - 1) / pick_span * pick_span : q.skip + sz[i].kblocks);
    pl.rounds += q.rounds;
    pl.rest += q.rest;
    if (pick_span > 0) pl.span_total += q.rest * q.span_len;
  }
  pl.span = (int)pick_span;
  const int64_t used = pick_span > 0 ? (pl.span_total + pick_span - 1) / pick_span : pick.left;
  pl.clusters = pl.rounds > 0 || used > pick.clusters ? pick.clusters : (int)used;
  if (pick_span > 0) pl.workspace = (size_t)2 * pl.clusters * c.cg * c.nb * c.bm * 128 * sizeof(float);
  *best = pl;
  return true;
}

// ---- operands -----------------------------------------------------------------------------------------

// A matrix as it is stored: rows x cols values of 16 bits, or of 8, row-major.
struct Matrix {
  const void* ptr;
  int64_t rows, cols, ld;
  bool eight = false;
  int64_t bytes() const { return eight ? 1 : 2; }                   // of a value
  int64_t padded_ld() const { return eight ? (cols + 127) / 128 * 128 : (cols + 63) / 64 * 64; }  // whole 128-byte rows
};

// TMA takes 16-byte aligned rows. A single row has no stride that matters.
bool addressable(const Matrix& m) { return ((uintptr_t)m.ptr & 15) == 0 && (m.ld * m.bytes() % 16 == 0 || m.rows == 1); }

bool make_map(CUtensorMap* map, int type, const Matrix& m, int box_rows) {
  const int64_t ld = m.rows == 1 ? m.padded_ld() : m.ld;
  const cuuint64_t dims[2] = {(cuuint64_t)m.cols, (cuuint64_t)m.rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(ld * m.bytes())};
  const cuuint32_t box[2] = {(cuuint32_t)(m.eight ? TK8 : TK), (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return g_encode(map, m.eight ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : type == HGEMM_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                  2, const_cast<void*>(m.ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int64_t padded(int64_t cols) { return (cols + 63) / 64 * 64; }
inline unsigned capped(int64_t n) { return (unsigned)(n < 65535 ? n : 65535); }

// Operands that need rewriting (all of 16 bits, or all of 8), collected so that one launch and one buffer serve them all.
class Packer {
 public:
  explicit Packer(int sms, size_t first_free = 0) : most_(8u * sms), bytes_(first_free) {}
  void add(Matrix* m) {
    if (addressable(*m)) return;
    for (int i = 0; i < n_; ++i)
      if (src_[i].ptr == m->ptr && src_[i].ld == m->ld && src_[i].rows == m->rows && src_[i].cols == m->cols) {
        users_[nu_] = m;
        of_[nu_++] = i;
        return;
      }
    src_[n_] = *m;
    at_[n_] = bytes_;
    bytes_ += (size_t)m->rows * m->padded_ld() * m->bytes();
    users_[nu_] = m;
    of_[nu_++] = n_++;
  }
  size_t bytes() const { return bytes_; }
  // The copies into `buf`, a block for 256 vectors each up to eight blocks per SM; from here on the operands are the copies.
  PackOps finish(char* buf) {
    PackOps ops;
    memset(&ops, 0, sizeof(ops));
    for (int i = 0; i < n_; ++i) {
      const Matrix& m = src_[i];
      ops.op[i] = PackOp{m.ptr, m.ld, (int)m.rows, (int)m.cols, buf + at_[i], m.padded_ld()};
      const int64_t vec = 16 / m.bytes(), blocks = ((m.cols + vec - 1) / vec * m.rows + 255) / 256;
      blocks_ += (unsigned)(blocks < most_ ? blocks : most_);
      ops.end[i] = blocks_;
    }
    for (int i = 0; i < nu_; ++i) *users_[i] = Matrix{buf + at_[of_[i]], users_[i]->rows, users_[i]->cols, users_[i]->padded_ld(), users_[i]->eight};
    return ops;
  }
  unsigned blocks() const { return blocks_; }  // after finish()
  bool launch(char* buf, cudaStream_t stream) {
    const PackOps ops = finish(buf);
    const bool eight = n_ > 0 && src_[0].eight;
    return blocks_ == 0 || lm::launch(eight ? hgemm_pack8_kernel : hgemm_pack_kernel, dim3(blocks_), dim3(256), 0, 1, stream, ops);
  }

 private:
  unsigned most_;  // blocks per operand
  size_t bytes_;
  unsigned blocks_ = 0;
  int n_ = 0, nu_ = 0;
  Matrix src_[3];
  size_t at_[3];
  Matrix* users_[6];
  int of_[6];
};

// One product for the tensor-core kernel: out (M x N, rows m, columns n) from lane operand P and column
// operand Q, over one or two contraction segments.
struct Product {
  int64_t N, M;
  int nseg;
  int64_t K[2];
  Matrix p[2], q[2];
  bool p_mn, q_mn;
  int act = HGEMM_ACT_NONE;  // (the same in all products of a launch)
  const void* bias = nullptr;
  const void* R = nullptr;
  int64_t ldr = 0;
  void* D = nullptr;
  int64_t ldd = 0;
  void* Z = nullptr;
  int64_t ldz = 0;
  void* U = nullptr;
  int64_t ldu = 0;
  bool eight = false;  // operands of 8 bits, with the scales of op(A)'s rows and of op(B)'s columns (gated: of both)
  const float* row_scale = nullptr;
  const float* col_scale[2] = {nullptr, nullptr};
  int step() const { return eight ? TK8 : TK; }  // values of a k-block
  Size size() const {
    int64_t kb = 0;
    for (int i = 0; i < nseg; ++i) kb += (K[i] + step() - 1) / step();
    int count = R ? 1 : 0, unaligned = 0;
    const auto add = [&](const void* p, int64_t ld) {
      if (!p) return;
      ++count;
      if (!addressable(Matrix{p, M, N, ld})) ++unaligned;
    };
    add(D, ldd);
    add(Z, ldz);
    add(U, ldu);
    return Size{N, M, (int)kb, epilogue_clocks(act, count, unaligned, R && !addressable(Matrix{R, M, N, ldr}))};
  }
};

// The element-wise gradient kernel's strips: 64 columns, so that its bias gradient has fewer partial sums in a row to add
// (bias gradient alone, GELU's tanh form, 256 and 64 columns: 5451 x 280 11.6 and 7.1 us, 20000 x 128 11.3 and 9.5, 4096 x 1024
// 10.2 and 8.8), or, from this many values on, 256, as memory likes it better (2088 x 4096 13.9 and 20.9, 8192 x 4096 35.5 and 59.4).
constexpr int64_t kWideStrips = 6ll << 20;

// Longest contraction first (the schedule assumes it), stable.
void order(Product** pr, int n) {
  for (int i = 1; i < n; ++i)
    for (int j = i; j > 0 && pr[j]->size().kblocks > pr[j - 1]->size().kblocks; --j) {
      Product* t = pr[j];
      pr[j] = pr[j - 1];
      pr[j - 1] = t;
    }
}

bool plan_products(Product** pr, int n, bool gated, int sms, Plan* pl) {
  Size sz[MAX_PROBLEMS];
  for (int i = 0; i < n; ++i) sz[i] = pr[i]->size();
  return make_plan(sz, n, gated, sms, pl);
}

int run_products(int type, bool gated, Product** pr, int n, const Plan& pl, lm::DeviceState* st, float* ws, int* counters,
                 cudaStream_t stream, const float* unscale = nullptr) {
  const Config& c = kConfigs[pl.config];
  Params p;
  memset(&p, 0, sizeof(p));
  const int qrows = c.bm / c.cg;
  for (int i = 0; i < n; ++i) {
    const Product& s = *pr[i];
    Problem& d = p.prob[i];
    const Plan::Part& q = pl.part[i];
    const int np = gated ? 2 : s.nseg, nq = s.nseg;
    for (int j = 0; j < np; ++j)
      if (!make_map(&d.p[j], type, s.p[j], s.p_mn || gated || c.nb == 1 ? 64 : 128)) return lm::cuda_failed();
    for (int j = 0; j < nq; ++j)
      if (!make_map(&d.q[j], type, s.q[j], s.q_mn ? 64 : qrows)) return lm::cuda_failed();
    d.N = (int)s.N;
    d.M = (int)s.M;
    d.tiles_n = q.tiles_n;
    d.tiles_m = q.tiles_m;
    d.kblocks = s.size().kblocks;
    d.kb_seg0 = (int)((s.K[0] + s.step() - 1) / s.step());
    d.p_mn = s.p_mn;
    d.q_mn = s.q_mn;
    d.rounds = q.rounds;
    d.rest = q.rest;
    d.skip = q.skip;
    d.span_len = q.span_len;
    d.vec = (addressable(Matrix{s.D, s.M, s.N, s.ldd}) ? VEC_D : 0) | (addressable(Matrix{s.Z, s.M, s.N, s.ldz}) ? VEC_Z : 0) |
            (addressable(Matrix{s.U, s.M, s.N, s.ldu}) ? VEC_U : 0) | (addressable(Matrix{s.R, s.M, s.N, s.ldr}) ? VEC_R : 0);
    d.bias = s.bias;
    d.R = s.R;
    d.D = s.D;
    d.Z = s.Z;
    d.U = s.U;
    d.ldr = s.ldr;
    d.ldd = s.ldd;
    d.ldz = s.ldz;
    d.ldu = s.ldu;
    d.row_scale = s.row_scale;
    d.col_scale[0] = s.col_scale[0];
    d.col_scale[1] = s.col_scale[1];
  }
  p.nprob = n;
  p.rounds = pl.rounds;
  p.rest = pl.rest;
  p.span = pl.span;
  p.span_total = pl.span_total;
  p.ws = ws;
  p.counters = counters;
  const int drop = g_drop_limit_us.load();
  p.wait_limit_ns = drop > 0 ? (unsigned long long)drop * 1000ull : kWaitLimitNs;
  p.drop = drop > 0;
  p.status = st->status;
  p.unscale = unscale;
  return launch_tc(type, pr[0]->eight, gated, pr[0]->act, pl.config, pl.clusters, stream, p) ? DGEMM_OK : lm::cuda_failed();
}

// ---- validation -----------------------------------------------------------------------------------------

bool bad_type(int type) { return type != HGEMM_TYPE_F16 && type != HGEMM_TYPE_BF16; }
bool bad_op(int op) { return op != DGEMM_OP_N && op != DGEMM_OP_T; }
bool bad_act(int act) { return act < 0 || act >= HGEMM_ACT_COUNT; }

int64_t span(int64_t rows, int64_t cols, int64_t ld) { return rows > 0 && cols > 0 ? ((rows - 1) * ld + cols) * 2 : 0; }

// A matrix argument: NULL only where it is empty or optional, element-aligned, ld >= max(1, cols).
int check(const void* ptr, int64_t rows, int64_t cols, int64_t ld, bool optional = false) {
  if (optional && !ptr) return DGEMM_OK;
  if (ld < (cols > 0 ? cols : 1)) return DGEMM_ERR_BAD_LD;
  if (rows == 0 || cols == 0) return DGEMM_OK;
  if (!ptr) return DGEMM_ERR_NULL;
  if ((uintptr_t)ptr & 1) return DGEMM_ERR_ALIGN;
  if (ld > (int64_t)1 << 38) return DGEMM_ERR_BAD_LD;
  return DGEMM_OK;
}

// The same of 8-bit values: any address, ld in bytes.
int check8(const void* ptr, int64_t rows, int64_t cols, int64_t ld) {
  if (ld < (cols > 0 ? cols : 1) || ld > (int64_t)1 << 38) return DGEMM_ERR_BAD_LD;
  return ptr || rows == 0 || cols == 0 ? (int)DGEMM_OK : (int)DGEMM_ERR_NULL;
}
int64_t span8(int64_t rows, int64_t cols, int64_t ld) { return rows > 0 && cols > 0 ? (rows - 1) * ld + cols : 0; }

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

#define HGEMM_TRY(expr)             \
  do {                              \
    const int rc_ = (expr);         \
    if (rc_ != DGEMM_OK) return rc_; \
  } while (0)

template <typename T>
bool launch_empty(int64_t M, int64_t N, const void* bias, int act, const void* R, int64_t ldr, void* D, int64_t ldd, void* Z, int64_t ldz,
                  cudaStream_t stream) {
  return lm::launch(hgemm_empty_kernel<T>, dim3((unsigned)((N + 255) / 256), capped(M)), dim3(256), 0, 1, stream, (int)M, (int)N,
                    static_cast<const T*>(bias), act, static_cast<const T*>(R), (long long)ldr, static_cast<T*>(D), (long long)ldd,
                    static_cast<T*>(Z), (long long)ldz);
}
int run_empty(int type, int64_t M, int64_t N, const void* bias, int act, const void* R, int64_t ldr, void* D, int64_t ldd, void* Z,
              int64_t ldz, cudaStream_t stream) {
  const bool ok = type == HGEMM_TYPE_BF16 ? launch_empty<__nv_bfloat16>(M, N, bias, act, R, ldr, D, ldd, Z, ldz, stream)
                                          : launch_empty<__half>(M, N, bias, act, R, ldr, D, ldd, Z, ldz, stream);
  return ok ? DGEMM_OK : lm::cuda_failed();
}

// Whether a product runs on the kernels for one or two rows (16-bit operands) or up to eight (8-bit).
//
// 8 bits, time of the token kernel over that of the tensor-core kernel, for K from 512 to 8192 (the tensor-core kernel's time rises where its tiles
// begin another round, at 32 and at 64 columns per SM):
//   several rows     N = 4096: 0.58 to 0.91, gated 0.70 to 0.91   6144: 0.95 to 1.3, 1.03 to 1.19   16384: 1.25 to 2.0, 1.05 to 1.7
//   one row          N = 4096: 0.57 to 0.79, gated 0.63 to 0.85   8192: 0.82 to 0.96, 0.95 to 1.01  16384: 1.15 to 1.5, 0.98 to 1.3
// and gated over the wider N: several rows 0.92 to 1.08 where K >= 4096, one row 0.81 to 1.07 where K >= 2048.
bool by_token(const Product& s, bool gated, int sms) {
  if (s.eight) {
    const bool one = s.M == 1, narrow = s.N <= (int64_t)(one ? 64 : 32) * sms, deep = gated && s.K[0] >= (one ? 2048 : 4096);
    return s.M <= TOKEN8_ROWS && (narrow || deep) && addressable(s.p[0]) && (!gated || addressable(s.p[1])) && g_drop_limit_us.load() == 0;
  }
  return s.M <= TOKEN_ROWS && !s.p_mn && addressable(s.p[0]) && (!gated || addressable(s.p[1])) &&
         s.M * ((s.K[0] + 7) / 8 * 8) * 2 <= (int64_t)TOKEN_SMEM && g_drop_limit_us.load() == 0;
}
int run_token(int type, bool gated, const Product& s, int sms, cudaStream_t stream) {
  TokenParams p;
  memset(&p, 0, sizeof(p));
  p.M = (int)s.M;
  p.N = (int)s.N;
  p.K = (int)s.K[0];
  p.X = s.q[0].ptr;
  p.ldx = s.q[0].ld;
  p.x_trans = s.q_mn;
  p.x_vec = !s.q_mn && addressable(s.q[0]);
  p.W[0] = s.p[0].ptr;
  p.ldw[0] = s.p[0].ld;
  if (gated) {
    p.W[1] = s.p[1].ptr;
    p.ldw[1] = s.p[1].ld;
  }
  p.act = s.act;
  p.bias = s.bias;
  p.R = s.R;
  p.D = s.D;
  p.Z = s.Z;
  p.U = s.U;
  p.ldr = s.ldr;
  p.ldd = s.ldd;
  p.ldz = s.ldz;
  p.ldu = s.ldu;
  if (!s.eight) return launch_token(type, gated, sms, stream, p) ? DGEMM_OK : lm::cuda_failed();
  Token8Params e;
  memset(&e, 0, sizeof(e));
  e.M = p.M;
  e.N = p.N;
  e.K = p.K;
  e.X = static_cast<const uint8_t*>(s.q[0].ptr);
  e.ldx = s.q[0].ld;
  e.x_vec = p.x_vec;
  e.row_scale = s.row_scale;
  for (int i = 0; i < (gated ? 2 : 1); ++i) {
    e.W[i] = static_cast<const uint8_t*>(s.p[i].ptr);
    e.ldw[i] = s.p[i].ld;
    e.col_scale[i] = s.col_scale[i];
  }
  e.out = p;
  return launch_token8(type, gated, sms, stream, e) ? DGEMM_OK : lm::cuda_failed();
}

// The range of a binary16 gradient part stored by `blocks` blocks takes range_bytes of scratch at the 4-byte aligned `at`.
size_t range_bytes(int64_t blocks) { return (size_t)(blocks + 1) * 4; }
PartRange range_at(char* at) { return PartRange{reinterpret_cast<float*>(at), reinterpret_cast<unsigned*>(at) + 1}; }
// Blocks of the kernel that scales it.
unsigned rescale_blocks(const lm::DeviceState* st, int64_t rows, int64_t cols) {
  const int64_t need = ((cols + 7) / 8 * rows + 255) / 256, most = (int64_t)st->sm_count * 4;
  return (unsigned)(need < most ? need : most);
}

// Packs what needs it and runs the products: the whole of a forward call.
int forward(int type, bool gated, Product* prod, cudaStream_t stream) {
  lm::DeviceState* st = nullptr;
  HGEMM_TRY(lm::device_state(&st));
  if (by_token(*prod, gated, st->sm_count)) return run_token(type, gated, *prod, st->sm_count, stream);
  Plan pl;
  if (!plan_products(&prod, 1, gated, st->sm_count, &pl)) return DGEMM_ERR_BAD_DIM;
  scratch::Hold hold(st->scratch, stream);
  Packer pack(st->sm_count);
  pack.add(&prod->p[0]);
  if (gated) pack.add(&prod->p[1]);
  pack.add(&prod->q[0]);
  if (pack.bytes() > 0) {
    char* buf = static_cast<char*>(hold.pack_buffer(pack.bytes()));
    if (!buf || !pack.launch(buf, stream)) return lm::cuda_failed();
  }
  float* ws = nullptr;
  if (pl.workspace > 0) {
    ws = static_cast<float*>(hold.workspace(pl.workspace));
    if (!ws) return lm::cuda_failed();
  }
  return run_products(type, gated, &prod, 1, pl, st, ws, st->counters + hold.lease_index() * lm::kCounters, stream);
}

}  // namespace

namespace lm {

bool release_scratch() {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return false;
  return !g_dev[dev].ready || scratch::release_all(g_dev[dev].scratch);
}

int device_state(DeviceState** out) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
    (void)cudaGetLastError();
    return DGEMM_ERR_DEVICE;
  }
  std::lock_guard<std::mutex> lock(g_mutex);
  DeviceState& st = g_dev[dev];
  if (!st.ready) {
    int major = 0, sms = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
      (void)cudaGetLastError();
      return DGEMM_ERR_DEVICE;
    }
    if (major != 10) return DGEMM_ERR_DEVICE;
    if (cudaGetSymbolAddress(reinterpret_cast<void**>(&st.status), g_hgemm_status_word) != cudaSuccess ||
        cudaGetSymbolAddress(reinterpret_cast<void**>(&st.counters), g_hgemm_counters) != cudaSuccess)
      return lm::cuda_failed();
    if (!configure_plain_f16() || !configure_gated_f16() || !configure_plain_bf16() || !configure_gated_bf16() || !configure_plain8_f16() ||
        !configure_gated8_f16() || !configure_plain8_bf16() || !configure_gated8_bf16())
      return lm::cuda_failed();
    if (!g_encode) {
      void* fn = nullptr;
      cudaDriverEntryPointQueryResult qres;
      if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess || !fn ||
          qres != cudaDriverEntryPointSuccess)
        return lm::cuda_failed();
      g_encode = reinterpret_cast<EncodeTiledFn>(fn);
    }
    st.sm_count = sms;
    st.ready = true;
  }
  *out = &st;
  return DGEMM_OK;
}

}  // namespace lm

extern "C" {

int hgemm_epilogue(int type, int transa, int transb, int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* B,
                   int64_t ldb, const void* bias, int act, const void* R, int64_t ldr, void* D, int64_t ldd, void* Z, int64_t ldz,
                   void* stream) {
  if (bad_type(type) || bad_act(act)) return DGEMM_ERR_VARIANT;
  if (bad_op(transa) || bad_op(transb)) return DGEMM_ERR_BAD_DIM;
  if (M < 0 || N < 0 || K < 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim) return DGEMM_ERR_BAD_DIM;
  if (M == 0 || N == 0) return DGEMM_OK;
  const int64_t ar = transa ? K : M, ac = transa ? M : K, br = transb ? N : K, bc = transb ? K : N;
  HGEMM_TRY(check(A, ar, ac, lda));
  HGEMM_TRY(check(B, br, bc, ldb));
  HGEMM_TRY(check(R, M, N, ldr, true));
  HGEMM_TRY(check(D, M, N, ldd));
  HGEMM_TRY(check(Z, M, N, ldz, true));
  if ((uintptr_t)bias & 1) return DGEMM_ERR_ALIGN;
  const bool in_place = R == D && ldr == ldd;
  const Range rg[6] = {{D, span(M, N, ldd)},   {Z, span(M, N, ldz)}, {A, span(ar, ac, lda)},
                       {B, span(br, bc, ldb)}, {bias, N * 2},        {R, span(M, N, ldr)}};
  if (aliased(rg, 2, in_place ? 5 : 6)) return DGEMM_ERR_ALIAS;
  if (in_place && Z && lm::ranges_overlap(Z, span(M, N, ldz), R, span(M, N, ldr))) return DGEMM_ERR_ALIAS;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (K == 0) {
    lm::DeviceState* st = nullptr;
    HGEMM_TRY(lm::device_state(&st));
    return run_empty(type, M, N, bias, act, R, ldr, D, ldd, Z, ldz, s);
  }
  Product pr;
  pr.N = N;
  pr.M = M;
  pr.nseg = 1;
  pr.K[0] = K;
  pr.p[0] = Matrix{B, br, bc, ldb};
  pr.p_mn = !transb;
  pr.q[0] = Matrix{A, ar, ac, lda};
  pr.q_mn = transa != 0;
  pr.act = act;
  pr.bias = bias;
  pr.R = R;
  pr.ldr = ldr;
  pr.D = D;
  pr.ldd = ldd;
  pr.Z = Z;
  pr.ldz = ldz;
  return forward(type, false, &pr, s);
}

int hgemm_epilogue_bwd(int type, int transa, int transb, int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const void* B,
                       int64_t ldb, int act, const void* Z, int64_t ldz, const void* dD, int64_t lddd, void* dA, int64_t ldda, void* dB,
                       int64_t lddb, float* dbias, void* stream) {
  if (bad_type(type) || bad_act(act)) return DGEMM_ERR_VARIANT;
  if (bad_op(transa) || bad_op(transb)) return DGEMM_ERR_BAD_DIM;
  if (M < 0 || N < 0 || K < 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim) return DGEMM_ERR_BAD_DIM;
  const int64_t ar = transa ? K : M, ac = transa ? M : K, br = transb ? N : K, bc = transb ? K : N;
  if (dB) HGEMM_TRY(check(A, ar, ac, lda));
  if (dA) HGEMM_TRY(check(B, br, bc, ldb));
  if (act != HGEMM_ACT_NONE) HGEMM_TRY(check(Z, M, N, ldz));
  HGEMM_TRY(check(dD, M, N, lddd));
  HGEMM_TRY(check(dA, ar, ac, ldda, true));
  HGEMM_TRY(check(dB, br, bc, lddb, true));
  if ((uintptr_t)dbias & 3) return DGEMM_ERR_ALIGN;
  const Range rg[7] = {{dA, span(ar, ac, ldda)}, {dB, span(br, bc, lddb)}, {dbias, N * 4},
                       {dB ? A : nullptr, span(ar, ac, lda)}, {dA ? B : nullptr, span(br, bc, ldb)},
                       {act != HGEMM_ACT_NONE ? Z : nullptr, span(M, N, ldz)}, {dD, span(M, N, lddd)}};
  if (aliased(rg, 3, 7)) return DGEMM_ERR_ALIAS;
  lm::DeviceState* st = nullptr;
  HGEMM_TRY(lm::device_state(&st));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // empty sums
  if (dA && N == 0 && M > 0 && K > 0) HGEMM_TRY(run_empty(type, ar, ac, nullptr, HGEMM_ACT_NONE, nullptr, 0, dA, ldda, nullptr, 0, s));
  if (dB && M == 0 && N > 0 && K > 0) HGEMM_TRY(run_empty(type, br, bc, nullptr, HGEMM_ACT_NONE, nullptr, 0, dB, lddb, nullptr, 0, s));
  if (dbias && M == 0 && N > 0 && cudaMemsetAsync(dbias, 0, (size_t)N * 4, s) != cudaSuccess) return lm::cuda_failed();
  if (M == 0 || N == 0) return DGEMM_OK;
  const bool want_a = dA && K > 0, want_b = dB && K > 0;
  if (!want_a && !want_b && !dbias) return DGEMM_OK;

  Product pa, pb;
  Product* list[2];
  int n = 0;
  Matrix dz{dD, M, N, lddd};
  const bool want_dz = (want_a || want_b) && (act != HGEMM_ACT_NONE || !addressable(dz));
  const Matrix a{A, ar, ac, lda}, b{B, br, bc, ldb};
  if (want_a) {
    pa.N = ac;
    pa.M = ar;
    pa.nseg = 1;
    pa.K[0] = N;
    pa.D = dA;
    pa.ldd = ldda;
    pa.p[0] = transa ? dz : b;
    pa.q[0] = transa ? b : dz;
    (transa ? pa.p_mn : pa.q_mn) = false;          // dZ: contraction over its columns
    (transa ? pa.q_mn : pa.p_mn) = transb != 0;    // B stored N x K: contraction over its rows
    list[n++] = &pa;
  }
  if (want_b) {
    pb.N = bc;
    pb.M = br;
    pb.nseg = 1;
    pb.K[0] = M;
    pb.D = dB;
    pb.ldd = lddb;
    pb.p[0] = transb ? a : dz;
    pb.q[0] = transb ? dz : a;
    (transb ? pb.q_mn : pb.p_mn) = true;           // dZ: contraction over its rows
    (transb ? pb.p_mn : pb.q_mn) = transa == 0;    // A stored M x K: contraction over its rows
    list[n++] = &pb;
  }
  Plan pl;
  order(list, n);
  if (n > 0 && !plan_products(list, n, false, st->sm_count, &pl)) return DGEMM_ERR_BAD_DIM;

  scratch::Hold hold(st->scratch, s);
  const int64_t lddz = padded(N);
  Packer pack(st->sm_count, want_dz ? (size_t)M * lddz * 2 : 0);
  if (want_a) pack.add(transa ? &pa.q[0] : &pa.p[0]);
  if (want_b) pack.add(transb ? &pb.p[0] : &pb.q[0]);

  // dZ and dbias
  const bool want_act = want_dz || dbias;
  ActBwdParams ap;
  memset(&ap, 0, sizeof(ap));
  int64_t strips = 0, chunks = 1;
  if (want_act) {
    const int most = M * N >= kWideStrips ? 5 : 3;
    while (ap.lane_bits < most && (8 << ap.lane_bits) < N) ++ap.lane_bits;
    strips = (N + (8 << ap.lane_bits) - 1) >> (3 + ap.lane_bits);
    ap.vec_d = addressable(dz);
    ap.vec_z = addressable(Matrix{Z, M, N, ldz});
    // four blocks per SM, at least two sweeps of rows each
    const int64_t sweep = 2 * (256 >> ap.lane_bits);
    chunks = ((int64_t)st->sm_count * 4 + strips - 1) / strips;
    if (chunks > (M + sweep - 1) / sweep) chunks = (M + sweep - 1) / sweep;
    if (chunks > 1 && strips > lm::kCounters) chunks = 1;
    if (chunks > 256) chunks = 256;
    ap.rows_per_chunk = (int)((M + chunks - 1) / chunks);
    chunks = (M + ap.rows_per_chunk - 1) / ap.rows_per_chunk;
    ap.M = (int)M;
    ap.N = (int)N;
    ap.Z = act != HGEMM_ACT_NONE ? Z : nullptr;
    ap.dD = dD;
    ap.dbias = dbias;
    ap.ldz = ldz;
    ap.lddd = lddd;
    ap.lddz = lddz;
    ap.act = act;
  }
  // (without activation or with ReLU dZ's values are dD's own or zero)
  const bool ranged = want_dz && type == HGEMM_TYPE_F16 && act != HGEMM_ACT_NONE && act != HGEMM_ACT_RELU;
  const size_t pack_bytes = pack.bytes() + (ranged ? range_bytes(strips * chunks) : 0);
  char* buf = nullptr;
  if (pack_bytes > 0 && !(buf = static_cast<char*>(hold.pack_buffer(pack_bytes)))) return lm::cuda_failed();
  if (want_dz) ap.dZ = buf;
  if (ranged) ap.range = range_at(buf + pack.bytes());
  size_t ws_bytes = n > 0 ? pl.workspace : 0;
  if (dbias && chunks > 1 && (size_t)chunks * (N + 7) * 4 > ws_bytes) ws_bytes = (size_t)chunks * (N + 7) * 4;
  float* ws = nullptr;
  if (ws_bytes > 0 && !(ws = static_cast<float*>(hold.workspace(ws_bytes)))) return lm::cuda_failed();
  int* counters = st->counters + hold.lease_index() * lm::kCounters;
  if (want_act) {
    ap.partial = ws;
    ap.counters = counters;
    // the operands that TMA cannot address are copied by further blocks of the same launch
    ap.strips = (unsigned)strips;
    ap.chunks = (unsigned)chunks;
    const PackOps ops = pack.finish(buf);
    const dim3 grid((unsigned)(strips * chunks) + pack.blocks());
    const bool ok = type == HGEMM_TYPE_BF16 ? lm::launch(hgemm_act_bwd_kernel<__nv_bfloat16>, grid, dim3(256), 0, 1, s, ap, ops)
                                            : lm::launch(hgemm_act_bwd_kernel<__half>, grid, dim3(256), 0, 1, s, ap, ops);
    if (!ok) return lm::cuda_failed();
    if (ranged && !lm::launch(hgemm_act_rescale_kernel, dim3(rescale_blocks(st, M, N)), dim3(256), 0, 1, s, ap)) return lm::cuda_failed();
  }
  if (n == 0) return DGEMM_OK;
  if (want_dz) {
    const Matrix packed{buf, M, N, lddz};
    if (want_a) (transa ? pa.p[0] : pa.q[0]) = packed;
    if (want_b) (transb ? pb.q[0] : pb.p[0]) = packed;
  }
  if (!want_act && !pack.launch(buf, s)) return lm::cuda_failed();
  return run_products(type, false, list, n, pl, st, ws, counters, s, ap.range.inverse);
}

int hgemm_gated(int type, int transw, int64_t M, int64_t F, int64_t K, const void* X, int64_t ldx, const void* Wg, int64_t ldwg,
                const void* Wu, int64_t ldwu, int act, void* H, int64_t ldh, void* G, int64_t ldg, void* U, int64_t ldu, void* stream) {
  if (bad_type(type) || bad_act(act)) return DGEMM_ERR_VARIANT;
  if (bad_op(transw)) return DGEMM_ERR_BAD_DIM;
  if (M < 0 || F < 0 || K < 0 || M > kMaxDim || F > kMaxDim || K > kMaxDim) return DGEMM_ERR_BAD_DIM;
  if (M == 0 || F == 0) return DGEMM_OK;
  const int64_t wr = transw ? F : K, wc = transw ? K : F;
  HGEMM_TRY(check(X, M, K, ldx));
  HGEMM_TRY(check(Wg, wr, wc, ldwg));
  HGEMM_TRY(check(Wu, wr, wc, ldwu));
  HGEMM_TRY(check(H, M, F, ldh));
  HGEMM_TRY(check(G, M, F, ldg, true));
  HGEMM_TRY(check(U, M, F, ldu, true));
  if ((G == nullptr) != (U == nullptr)) return DGEMM_ERR_NULL;
  const Range rg[6] = {{H, span(M, F, ldh)}, {G, span(M, F, ldg)},    {U, span(M, F, ldu)},
                       {X, span(M, K, ldx)}, {Wg, span(wr, wc, ldwg)}, {Wu, span(wr, wc, ldwu)}};
  if (aliased(rg, 3, 6)) return DGEMM_ERR_ALIAS;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (K == 0) {  // G = U = 0, H = act(0) 0
    lm::DeviceState* st = nullptr;
    HGEMM_TRY(lm::device_state(&st));
    HGEMM_TRY(run_empty(type, M, F, nullptr, HGEMM_ACT_NONE, nullptr, 0, H, ldh, G, ldg, s));
    return U ? run_empty(type, M, F, nullptr, HGEMM_ACT_NONE, nullptr, 0, U, ldu, nullptr, 0, s) : (int)DGEMM_OK;
  }
  Product pr;
  pr.N = F;
  pr.M = M;
  pr.nseg = 1;
  pr.K[0] = K;
  pr.p[0] = Matrix{Wg, wr, wc, ldwg};
  pr.p[1] = Matrix{Wu, wr, wc, ldwu};
  pr.p_mn = !transw;
  pr.q[0] = Matrix{X, M, K, ldx};
  pr.q_mn = false;
  pr.act = act;
  pr.D = H;
  pr.ldd = ldh;
  pr.Z = G;
  pr.ldz = ldg;
  pr.U = U;
  pr.ldu = ldu;
  return forward(type, true, &pr, s);
}

int hgemm_gated_bwd(int type, int transw, int64_t M, int64_t F, int64_t K, const void* X, int64_t ldx, const void* Wg, int64_t ldwg,
                    const void* Wu, int64_t ldwu, int act, const void* G, int64_t ldg, const void* U, int64_t ldu, const void* dH,
                    int64_t lddh, void* dX, int64_t lddx, void* dWg, int64_t lddwg, void* dWu, int64_t lddwu, void* stream) {
  if (bad_type(type) || bad_act(act)) return DGEMM_ERR_VARIANT;
  if (bad_op(transw)) return DGEMM_ERR_BAD_DIM;
  if (M < 0 || F < 0 || K < 0 || M > kMaxDim || F > kMaxDim || K > kMaxDim) return DGEMM_ERR_BAD_DIM;
  const int64_t wr = transw ? F : K, wc = transw ? K : F;
  const bool need_x = dWg || dWu;
  if (need_x) HGEMM_TRY(check(X, M, K, ldx));
  if (dX) {
    HGEMM_TRY(check(Wg, wr, wc, ldwg));
    HGEMM_TRY(check(Wu, wr, wc, ldwu));
  }
  HGEMM_TRY(check(G, M, F, ldg));
  HGEMM_TRY(check(U, M, F, ldu));
  HGEMM_TRY(check(dH, M, F, lddh));
  HGEMM_TRY(check(dX, M, K, lddx, true));
  HGEMM_TRY(check(dWg, wr, wc, lddwg, true));
  HGEMM_TRY(check(dWu, wr, wc, lddwu, true));
  const Range rg[9] = {{dX, span(M, K, lddx)}, {dWg, span(wr, wc, lddwg)}, {dWu, span(wr, wc, lddwu)},
                       {need_x ? X : nullptr, span(M, K, ldx)}, {dX ? Wg : nullptr, span(wr, wc, ldwg)},
                       {dX ? Wu : nullptr, span(wr, wc, ldwu)}, {G, span(M, F, ldg)}, {U, span(M, F, ldu)}, {dH, span(M, F, lddh)}};
  if (aliased(rg, 3, 9)) return DGEMM_ERR_ALIAS;
  lm::DeviceState* st = nullptr;
  HGEMM_TRY(lm::device_state(&st));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (K == 0) return DGEMM_OK;  // every output is empty
  if (dX && F == 0 && M > 0) HGEMM_TRY(run_empty(type, M, K, nullptr, HGEMM_ACT_NONE, nullptr, 0, dX, lddx, nullptr, 0, s));
  for (int i = 0; i < 2; ++i) {
    void* w = i ? dWu : dWg;
    if (w && M == 0 && F > 0)
      HGEMM_TRY(run_empty(type, wr, wc, nullptr, HGEMM_ACT_NONE, nullptr, 0, w, i ? lddwu : lddwg, nullptr, 0, s));
  }
  if (M == 0 || F == 0 || (!dX && !dWg && !dWu)) return DGEMM_OK;

  // dG and dU, rounded, in scratch rows of a multiple of 128 bytes
  const int64_t ldo = padded(F);
  const size_t half_bytes = (size_t)M * ldo * 2;
  Product px, pw[2];
  Product* list[3];
  int n = 0;
  Matrix dgu[2] = {Matrix{nullptr, M, F, ldo}, Matrix{nullptr, M, F, ldo}};
  Matrix x{X, M, K, ldx}, w[2] = {Matrix{Wg, wr, wc, ldwg}, Matrix{Wu, wr, wc, ldwu}};
  if (dX) {
    px.N = K;
    px.M = M;
    px.nseg = 2;
    px.K[0] = px.K[1] = F;
    px.p_mn = transw != 0;
    px.q_mn = false;
    px.D = dX;
    px.ldd = lddx;
    list[n++] = &px;
  }
  for (int i = 0; i < 2; ++i) {
    void* out = i ? dWu : dWg;
    if (!out) continue;
    pw[i].N = wc;
    pw[i].M = wr;
    pw[i].nseg = 1;
    pw[i].K[0] = M;
    pw[i].p_mn = pw[i].q_mn = true;
    pw[i].D = out;
    pw[i].ldd = i ? lddwu : lddwg;
    list[n++] = &pw[i];
  }
  Plan pl;
  order(list, n);
  if (!plan_products(list, n, false, st->sm_count, &pl)) return DGEMM_ERR_BAD_DIM;

  scratch::Hold hold(st->scratch, s);
  Packer pack(st->sm_count, 2 * half_bytes);
  if (need_x) pack.add(&x);
  if (dX) {
    pack.add(&w[0]);
    pack.add(&w[1]);
  }
  int64_t blocks = ((F + 7) / 8 * M + 255) / 256;
  if (blocks > (int64_t)st->sm_count * 16) blocks = (int64_t)st->sm_count * 16;
  const bool ranged = type == HGEMM_TYPE_F16;
  char* buf = static_cast<char*>(hold.pack_buffer(pack.bytes() + (ranged ? range_bytes(blocks) : 0)));
  if (!buf) return lm::cuda_failed();
  float* ws = nullptr;
  if (pl.workspace > 0 && !(ws = static_cast<float*>(hold.workspace(pl.workspace)))) return lm::cuda_failed();
  GatedBwdParams gp;
  memset(&gp, 0, sizeof(gp));
  gp.M = (int)M;
  gp.F = (int)F;
  gp.G = G;
  gp.U = U;
  gp.dH = dH;
  gp.dG = buf;
  gp.dU = buf + half_bytes;
  gp.ldg = ldg;
  gp.ldu = ldu;
  gp.lddh = lddh;
  gp.ldo = ldo;
  gp.act = act;
  dgu[0].ptr = gp.dG;
  dgu[1].ptr = gp.dU;
  gp.vec_g = addressable(Matrix{G, M, F, ldg});
  gp.vec_u = addressable(Matrix{U, M, F, ldu});
  gp.vec_h = addressable(Matrix{dH, M, F, lddh});
  gp.blocks = (unsigned)blocks;
  if (ranged) gp.range = range_at(buf + pack.bytes());
  const PackOps ops = pack.finish(buf);  // copied by further blocks of the same launch
  const dim3 grid((unsigned)blocks + pack.blocks());
  const bool ok = type == HGEMM_TYPE_BF16 ? lm::launch(hgemm_gated_bwd_kernel<__nv_bfloat16>, grid, dim3(256), 0, 1, s, gp, ops)
                                          : lm::launch(hgemm_gated_bwd_kernel<__half>, grid, dim3(256), 0, 1, s, gp, ops);
  if (!ok) return lm::cuda_failed();
  if (ranged && !lm::launch(hgemm_gated_rescale_kernel, dim3(rescale_blocks(st, M, F)), dim3(256), 0, 1, s, gp)) return lm::cuda_failed();
  for (int i = 0; i < 2; ++i) {
    px.p[i] = w[i];
    px.q[i] = dgu[i];
    pw[i].p[0] = transw ? x : dgu[i];
    pw[i].q[0] = transw ? dgu[i] : x;
  }
  return run_products(type, false, list, n, pl, st, ws, st->counters + hold.lease_index() * lm::kCounters, s,
                      gp.range.inverse);
}

int qgemm_epilogue(int type, int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const float* a_scale, const void* B, int64_t ldb,
                   const float* b_scale, const void* bias, int act, const void* R, int64_t ldr, void* D, int64_t ldd, void* Z, int64_t ldz,
                   void* stream) {
  if (bad_type(type) || bad_act(act)) return DGEMM_ERR_VARIANT;
  if (M < 0 || N < 0 || K < 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim) return DGEMM_ERR_BAD_DIM;
  if (M == 0 || N == 0) return DGEMM_OK;
  HGEMM_TRY(check8(A, M, K, lda));
  HGEMM_TRY(check8(B, N, K, ldb));
  HGEMM_TRY(check(R, M, N, ldr, true));
  HGEMM_TRY(check(D, M, N, ldd));
  HGEMM_TRY(check(Z, M, N, ldz, true));
  if (((uintptr_t)bias & 1) || (((uintptr_t)a_scale | (uintptr_t)b_scale) & 3)) return DGEMM_ERR_ALIGN;
  const bool in_place = R == D && ldr == ldd;
  const Range rg[8] = {{D, span(M, N, ldd)},   {Z, span(M, N, ldz)}, {A, span8(M, K, lda)}, {B, span8(N, K, ldb)},
                       {a_scale, M * 4}, {b_scale, N * 4}, {bias, N * 2}, {in_place ? nullptr : R, span(M, N, ldr)}};
  if (aliased(rg, 2, 8)) return DGEMM_ERR_ALIAS;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (K == 0) {
    lm::DeviceState* st = nullptr;
    HGEMM_TRY(lm::device_state(&st));
    return run_empty(type, M, N, bias, act, R, ldr, D, ldd, Z, ldz, s);
  }
  Product pr;
  pr.eight = true;
  pr.row_scale = a_scale;
  pr.col_scale[0] = b_scale;
  pr.N = N;
  pr.M = M;
  pr.nseg = 1;
  pr.K[0] = K;
  pr.p[0] = Matrix{B, N, K, ldb, true};
  pr.q[0] = Matrix{A, M, K, lda, true};
  pr.p_mn = pr.q_mn = false;
  pr.act = act;
  pr.bias = bias;
  pr.R = R;
  pr.ldr = ldr;
  pr.D = D;
  pr.ldd = ldd;
  pr.Z = Z;
  pr.ldz = ldz;
  return forward(type, false, &pr, s);
}

int qgemm_gated(int type, int64_t M, int64_t F, int64_t K, const void* X, int64_t ldx, const float* x_scale, const void* Wg, int64_t ldwg,
                const float* g_scale, const void* Wu, int64_t ldwu, const float* u_scale, int act, void* H, int64_t ldh, void* G, int64_t ldg,
                void* U, int64_t ldu, void* stream) {
  if (bad_type(type) || bad_act(act)) return DGEMM_ERR_VARIANT;
  if (M < 0 || F < 0 || K < 0 || M > kMaxDim || F > kMaxDim || K > kMaxDim) return DGEMM_ERR_BAD_DIM;
  if (M == 0 || F == 0) return DGEMM_OK;
  HGEMM_TRY(check8(X, M, K, ldx));
  HGEMM_TRY(check8(Wg, F, K, ldwg));
  HGEMM_TRY(check8(Wu, F, K, ldwu));
  HGEMM_TRY(check(H, M, F, ldh));
  HGEMM_TRY(check(G, M, F, ldg, true));
  HGEMM_TRY(check(U, M, F, ldu, true));
  if ((G == nullptr) != (U == nullptr)) return DGEMM_ERR_NULL;
  if (((uintptr_t)x_scale | (uintptr_t)g_scale | (uintptr_t)u_scale) & 3) return DGEMM_ERR_ALIGN;
  const Range rg[9] = {{H, span(M, F, ldh)}, {G, span(M, F, ldg)}, {U, span(M, F, ldu)}, {X, span8(M, K, ldx)}, {Wg, span8(F, K, ldwg)},
                       {Wu, span8(F, K, ldwu)}, {x_scale, M * 4}, {g_scale, F * 4}, {u_scale, F * 4}};
  if (aliased(rg, 3, 9)) return DGEMM_ERR_ALIAS;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (K == 0) {  // G = U = 0, H = act(0) 0
    lm::DeviceState* st = nullptr;
    HGEMM_TRY(lm::device_state(&st));
    HGEMM_TRY(run_empty(type, M, F, nullptr, HGEMM_ACT_NONE, nullptr, 0, H, ldh, G, ldg, s));
    return U ? run_empty(type, M, F, nullptr, HGEMM_ACT_NONE, nullptr, 0, U, ldu, nullptr, 0, s) : (int)DGEMM_OK;
  }
  Product pr;
  pr.eight = true;
  pr.row_scale = x_scale;
  pr.col_scale[0] = g_scale;
  pr.col_scale[1] = u_scale;
  pr.N = F;
  pr.M = M;
  pr.nseg = 1;
  pr.K[0] = K;
  pr.p[0] = Matrix{Wg, F, K, ldwg, true};
  pr.p[1] = Matrix{Wu, F, K, ldwu, true};
  pr.q[0] = Matrix{X, M, K, ldx, true};
  pr.p_mn = pr.q_mn = false;
  pr.act = act;
  pr.D = H;
  pr.ldd = ldh;
  pr.Z = G;
  pr.ldz = ldg;
  pr.U = U;
  pr.ldu = ldu;
  return forward(type, true, &pr, s);
}

int hgemm_last_device_status(void* stream) {
  lm::DeviceState* st = nullptr;
  HGEMM_TRY(lm::device_state(&st));
  if (cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) != cudaSuccess) {
    return lm::cuda_failed();
  }
  int v = 0;
  if (cudaMemcpy(&v, st->status, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess) return lm::cuda_failed();
  // The word alone: the counters of cut tiles belong to calls that may be in flight on other streams, and a kernel that gave
  // up has still counted every part (its epilogue walks through all units), so they are zero after it like after any other.
  if (v != 0 && cudaMemset(st->status, 0, sizeof(int)) != cudaSuccess) return lm::cuda_failed();
  return v;
}

int hgemm_plan(int64_t M, int64_t N, int64_t K, int gated, int sm_count, int* out) {
  if (!out) return DGEMM_ERR_NULL;
  if (M <= 0 || N <= 0 || K <= 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim || sm_count < 0 || sm_count == 1) return DGEMM_ERR_BAD_DIM;
  const Size sz{N, M, (int)((K + TK - 1) / TK), epilogue_clocks(HGEMM_ACT_NONE, 1, 0, false)};
  Plan pl;
  if (!make_plan(&sz, 1, gated != 0, sm_count ? sm_count : 148, &pl)) return DGEMM_ERR_BAD_DIM;
  const Config& c = kConfigs[pl.config];
  const Plan::Part& q = pl.part[0];
  const int v[8] = {c.cg, c.bm, pl.nt, pl.clusters, sz.kblocks, q.rounds, q.rest, pl.span};
  memcpy(out, v, sizeof(v));
  return DGEMM_OK;
}

int hgemm_set_test_drop_loads(int limit_us) {
  if (limit_us < 0 || limit_us > 4000000) return DGEMM_ERR_VARIANT;
  g_drop_limit_us.store(limit_us);
  return DGEMM_OK;
}

}  // extern "C"
