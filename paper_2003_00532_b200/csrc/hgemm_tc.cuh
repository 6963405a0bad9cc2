// 16-bit matrix products on the fifth-generation tensor cores, with what follows the product in
// the epilogue: bias, activation, residual, or the gated pair act(G) * U.
//
// Orientation. The tile's 128 TMEM lanes (256 over a CTA pair) run along the output's columns n and
// its BM TMEM columns along the output's rows m: D^T = P Q^T with P = op(B)^T ("lane operand", the
// weights) and Q = op(A) ("column operand", the tokens). Few rows (single tokens) then need a small
// BM, not a 128-row tile: BM = 16 .. 256.
//
// Epilogue. A warp takes 32 lanes x CH columns at a time, in the register layout of 8 x 8 matrices. Results
// are packed in pairs and turned into row pieces of 32 values by transposing matrix stores into a small
// buffer of the warp's own, from which they leave as 16-byte vectors (rows that are 16-byte aligned)
// or value by value (any other alignment, ragged last columns); a residual comes in the same way
// backwards. Storing each lane's column directly, 2 bytes per lane, made the store instructions the
// limit: 4096 x 9472 x 1024 took 94 us (125 with bias and GELU) where the MMAs take 54.
//
// Operands. Either may be stored with its contraction index contiguous ("K-major") or with its
// outer index contiguous ("MN-major"): both are staged by TMA in boxes of 64 x 64 values (rows of 128
// bytes, 128-byte swizzle, 8 KB) and the MMA descriptors say which of the two a box holds, so all four
// transpositions run the same code without a transposing pass.
//
// Work. One launch covers up to three problems (the gradients of one operator). Of each problem's tiles as many as make
// whole rounds over the clusters run whole. The tiles left over, of all problems together, are either dealt out whole
// as well, or their k-blocks are laid end to end and cut into equal spans, one per cluster: then a tile may be
// computed in parts, whose binary32 sums go to a workspace, and the CTA that finishes the last part of a tile (a
// counter per tile) adds all parts in order and runs the epilogue: one launch, no CTA waits for another, same bits
// every time.
//
// Operands of 8 bits (e4m3, with a scale per row of each) run the same code: a 128-byte row of a box then holds 128 values, an MMA
// instruction takes 32 of them in the time of 16 values of 16 bits, and the epilogue multiplies the sums by the two scales before
// anything else. K-major only.
//
// The activation is a template argument of the whole kernel: with a switch over the five of them in it, the
// registers of all shared one allocation and the epilogue without activation spilled (4096 x 9472 x 256: 50 us,
// 40 alone).
//
// Roles (384 threads): warps 0 and 2 stage halves of P, warp 3 stages Q (one thread that issued all copies was the
// limit: 479 ns per 64-wide k-block with four copies, against 366 ns for its MMAs), warp 1 issues the MMAs, warp 2 also
// owns the TMEM allocation, warps 4-11 run the epilogue of one accumulator while the MMAs fill the other. In a
// pair the MMAs of both CTAs are issued by the leader; each CTA stages its own lanes and its half of Q.
#pragma once

#include <cstdint>
#include <type_traits>
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/dgemm.h"
#include "../../include/hgemm.h"
#include "hgemm_act.cuh"
#include "hgemm_ptx.cuh"
#include "layernorm.cuh"

namespace hgemm {

constexpr int TK = 64;           // k-block: 64 values of 16 bits = one 128-byte swizzled row
constexpr int TK8 = 128;         // ... of 8 bits
constexpr int BOX_BYTES = 8192;  // 64 x 64 values
constexpr int PITCH = 80;  // bytes per patch row in shared memory: 64 + 16, no two of 8 rows on the same banks
constexpr int MAX_SMEM = 232448;  // 227 KB
constexpr int MAX_PROBLEMS = 3;

// A kernel's element type: T for operands and outputs of that type, Eight<T> for operands in e4m3 and outputs of type T.
template <typename T>
struct Eight {};
template <typename T>
struct Kind {
  using Out = T;
  static constexpr bool EIGHT = false;
  static constexpr int TK = hgemm::TK;
  static constexpr uint32_t FORMAT = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;  // in the instruction descriptor
};
template <typename T>
struct Kind<Eight<T>> {
  using Out = T;
  static constexpr bool EIGHT = true;
  static constexpr int TK = TK8;
  static constexpr uint32_t FORMAT = 0u;
};

// CG: CTAs per tile (1, or a pair); BM: TMEM columns of the tile (rows of the output); NB: blocks of 128 lanes per CTA.
// With NB = 1 the two accumulators are two tiles', filled and drained in turn; with NB = 2 they are the two lane
// blocks of one tile, which share each staged Q.
template <int CG_, int BM_, int NB_, bool GATED_, bool EIGHT_>
struct Cfg {
  static constexpr int CG = CG_, BM = BM_, NB = NB_;
  // The epilogue is a chain of latencies: for 8-bit operands, whose products are done in half the time, more warps (4096 x 8192 x 512 with
  // tanh-GELU 59.9 -> 52.5 us, with residual 71.7 -> 60.8; with 16 of them, and 96 registers each, 56.8 and 70.8; before RowScales). Not the gated one, whose
  // partners would wait for one another more often (4097 x 8192 x 2048 116.3 us, with 12 warps 119.0).
  static constexpr int EPI_WARPS = EIGHT_ && !GATED_ && BM >= 128 ? 12 : 8;
  static constexpr int THREADS = 128 + 32 * EPI_WARPS;
  static constexpr bool GATED = GATED_;
  static constexpr int QROWS = BM / CG;  // rows of Q that one CTA stages
  static constexpr int QBOXES = (QROWS + 63) / 64;
  static constexpr int P_BYTES = NB * 2 * BOX_BYTES;
  static constexpr int STAGE_BYTES = P_BYTES + QBOXES * BOX_BYTES;
  static constexpr int CH = GATED ? (BM < 32 ? 8 : 16) : 16;  // TMEM columns one warp takes at a time
  // Each epilogue warp's buffer: a patch of the output or, before that, the values it hands to its partner.
  static constexpr int BUF_BYTES = GATED ? CH * 128 : CH * PITCH;
  static constexpr int BUFS_BYTES = EPI_WARPS * BUF_BYTES;
  static constexpr int CTRL_BYTES = 512;
  static constexpr int FIT = (MAX_SMEM - 1024 - BUFS_BYTES - CTRL_BYTES) / STAGE_BYTES;
  static constexpr int STAGES = FIT < 8 ? FIT : 8;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + BUFS_BYTES + CTRL_BYTES + 1024;
  static constexpr int TMEM_COLS = 2 * BM < 32 ? 32 : 2 * BM;  // two accumulators (a power of two)
  static constexpr int BLOCK = GATED ? 64 : 128;               // output columns of one accumulator
  static constexpr int NT = BLOCK * CG * NB;                   // output columns per tile
};

struct alignas(64) Problem {
  CUtensorMap p[2], q[2];  // [segment] of the contraction; gated: p[0] = gate weights, p[1] = up weights
  int N, M;                // output columns (lanes) and rows
  int tiles_n, tiles_m;
  int kblocks, kb_seg0;    // k-blocks in all, and of the first segment
  int p_mn, q_mn;          // operand stored MN-major
  int rounds;              // tiles run whole in rounds over all clusters; the first `rounds` x clusters tiles
  int rest;                // tiles left over
  int skip;                // positions before such a tile's k-blocks in the spans, which stand for its epilogue's time
  int span_len;            // positions that it takes in all: skip + its k-blocks, or a multiple of the span
  int vec;                 // which of D, Z, U, R have 16-byte aligned rows (VEC_*)
  const void* bias;
  const void* R;
  void* D;
  void* Z;                 // pre-activation; gated: gate pre-activation
  void* U;                 // gated: up pre-activation
  long long ldr, ldd, ldz, ldu;
  const float* row_scale;     // operands of 8 bits: of op(A)'s rows and of op(B)'s columns (gated: gate, up), NULL: ones
  const float* col_scale[2];
};

struct Params {
  Problem prob[MAX_PROBLEMS];
  int nprob;
  int rounds;              // of all problems
  int span;                // positions per cluster of the tiles left over, 0: they run whole
  int span_total;          // positions of all tiles left over
  int rest;                // tiles left over
  float* ws;               // two slots of CG x NB x BM x 128 sums per cluster
  int* counters;           // CG x NB per tile left over; zero between launches
  unsigned long long wait_limit_ns;
  int* status;
  const float* unscale;  // gradients in binary16: what the sums are multiplied by (a power of two), or NULL
  int drop;  // testing aid: the producers skip their copies
};

// One unit of work: k-blocks kb0 .. kb1 of a tile. For a part of a cut tile: its slot in the workspace, the tile's index
// among those left over, the clusters that share it and the first one's slot.
struct Work {
  int prob, tile, kb0, kb1;
  int slot;  // -1: the whole tile
  int left, parts, first_slot, next_slot;
};

// Unit number j of `cluster`; false after its last one.
__device__ __forceinline__ bool get_work(const Params& p, int cluster, int clusters, int j, Work& w) {
  w.slot = -1;
  if (j < p.rounds) {
    w.prob = 0;
    while (j >= p.prob[w.prob].rounds) j -= p.prob[w.prob++].rounds;
    w.tile = j * clusters + cluster;
    w.kb0 = 0;
    w.kb1 = p.prob[w.prob].kblocks;
    return true;
  }
  j -= p.rounds;
  if (p.span == 0) {
    int left = j * clusters + cluster;
    if (left >= p.rest) return false;
    w.prob = 0;
    while (left >= p.prob[w.prob].rest) left -= p.prob[w.prob++].rest;
    w.tile = p.prob[w.prob].rounds * clusters + left;
    w.kb0 = 0;
    w.kb1 = p.prob[w.prob].kblocks;
    return true;
  }
  // the span's pieces: up to the end of a tile each
  int pos = cluster * p.span;
  const int end = min(pos + p.span, p.span_total);
  for (;;) {
    if (pos >= end) return false;
    int base = 0, left = 0;  // position and index of the problem's first tile left over
    w.prob = 0;
    while (pos >= base + p.prob[w.prob].rest * p.prob[w.prob].span_len) {
      base += p.prob[w.prob].rest * p.prob[w.prob].span_len;
      left += p.prob[w.prob++].rest;
    }
    const int kb = p.prob[w.prob].kblocks, len = p.prob[w.prob].span_len, t = (pos - base) / len;
    const int lo = base + t * len, hi = lo + len;
    const int k0 = lo + p.prob[w.prob].skip, stop = min(hi, end);
    if (stop > k0 && j-- == 0) {
      w.tile = p.prob[w.prob].rounds * clusters + t;
      w.kb0 = max(pos - k0, 0);
      w.kb1 = min(stop - k0, kb);
      if (w.kb1 - w.kb0 < kb) {
        const int c0 = k0 / p.span;
        w.left = left + t;
        w.parts = (hi - 1) / p.span - c0 + 1;
        // a cluster whose span begins inside the tile uses its first slot, the one whose span runs into it the second
        w.first_slot = 2 * c0 + (c0 * p.span >= lo ? 0 : 1);
        w.next_slot = 2 * c0 + 2;
        w.slot = cluster == c0 ? w.first_slot : 2 * cluster;
      }
      return true;
    }
    pos = stop;
  }
}

// Grouped raster: 8 tile rows of lanes (n) at a time, so that the tiles in flight share operands in L2.
__device__ __forceinline__ void tile_to_mn(const Problem& pr, int tile, int& tm, int& tn) {
  constexpr int GROUP = 8;
  const int per = GROUP * pr.tiles_m;
  const int g = tile / per, r = tile - g * per;
  const int h = min(GROUP, pr.tiles_n - g * GROUP);
  tm = r / h;
  tn = g * GROUP + r % h;
}

// Polls an mbarrier phase; gives up after the limit, records the timeout and raises the CTA's abort
// flag. Never spins without a limit.
__device__ __noinline__ static bool wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit_ns, int* status) {
  using namespace dgemm::ptx;
  const unsigned long long t0 = globaltimer_ns();
  for (;;) {
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    if (globaltimer_ns() - t0 > limit_ns) {
      atomicExch(status, (int)DGEMM_ERR_TIMEOUT);
      *abort_flag = 1;
      return false;
    }
  }
}
__device__ __forceinline__ bool wait_bounded(uint32_t bar, uint32_t parity, volatile int* abort_flag, const Params& p) {
  if (dgemm::ptx::mbar_try_wait(bar, parity)) return true;
  return wait_slow(bar, parity, abort_flag, p.wait_limit_ns, p.status);
}

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }

// Two values rounded to T, `lo` in the lower half.
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t v);
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

// A warp's patch of the output: CH rows from m0, 32 columns from n0. A thread's CH values of it, v[i]:
// i = 4 (h MB + b) + r (h: half of the 32 lanes, b: block of 8 rows, MB = CH / 8) is column
// 16 h + 8 (r / 2) + lane / 4 and row 8 b + 2 (lane % 4) + r % 2 of the patch; the pair (v[i], v[i + 1]), i even, is
// one register of an 8 x 8 matrix.
template <int CH>
struct Patch {
  static constexpr int MB = CH / 8;

  // A matrix as one lane sees it: the address of its piece of the tile's first row(s), and whether the warp moves
  // 16-byte vectors (lane -> row lane / 4, columns 8 (lane % 4)) or single values (lane -> column).
  struct View {
    char* p;
    long long ld;  // bytes
    bool vec;
  };

  int rows;  // rows of the matrix from the tile's first one
  int cols;  // columns of the matrix from the patch's first one
  int lane;
  uint32_t buf;     // this warp's buffer
  uint32_t matrix;  // this lane's row address for the matrix instructions: row lane % 8, columns 8 (lane / 8)

  __device__ __forceinline__ View view(const void* ptr, long long ld, bool aligned, int m_base, int n0) const {
    View w;
    w.ld = ld * 2;
    w.vec = aligned && cols >= 32;
    w.p = static_cast<char*>(const_cast<void*>(ptr)) + m_base * w.ld + n0 * 2ll + (w.vec ? (lane >> 2) * w.ld + (lane & 3) * 16 : lane * 2);
    return w;
  }

  // Stores the patch that begins at row m of the tile, given as packed pairs: q[i / 2].
  __device__ __forceinline__ void store(const View& out, int m, const uint32_t* q) const {
#pragma unroll
    for (int b = 0; b < MB; ++b)
      ptx5::stmatrix_x4_trans(matrix + b * 8 * PITCH, q[2 * b], q[2 * b + 1], q[2 * (MB + b)], q[2 * (MB + b) + 1]);
    __syncwarp();
    char* o = out.p + m * out.ld;
    if (out.vec) {
      uint4 x[MB];
#pragma unroll
      for (int i = 0; i < MB; ++i) x[i] = ptx5::lds128(buf + (8 * i + (lane >> 2)) * PITCH + (lane & 3) * 16);
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        if (m + 8 * i + (lane >> 2) < rows) *reinterpret_cast<uint4*>(o) = x[i];
        o += 8 * out.ld;
      }
    } else if (lane < cols) {
      uint16_t x[CH];
#pragma unroll
      for (int r = 0; r < CH; ++r) x[r] = ptx5::lds16(buf + r * PITCH + lane * 2);
#pragma unroll
      for (int r = 0; r < CH; ++r) {
        if (m + r < rows) *reinterpret_cast<uint16_t*>(o) = x[r];
        o += out.ld;
      }
    }
    __syncwarp();
  }

  // The patch of a 16-bit matrix on its way into registers: fetch() issues the global loads, take() turns
  // them into packed pairs.
  struct Raw {
    uint32_t w[CH / 2];
  };
  __device__ __forceinline__ void fetch(Raw& raw, const View& view, int m) const {
    const long long in_ld = view.ld;
    if (view.vec) {
      const char* s = view.p + m * in_ld;
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (m + 8 * i + (lane >> 2) < rows) x = *reinterpret_cast<const uint4*>(s);
        s += 8 * in_ld;
        raw.w[4 * i] = x.x;
        raw.w[4 * i + 1] = x.y;
        raw.w[4 * i + 2] = x.z;
        raw.w[4 * i + 3] = x.w;
      }
    } else {
      // Rows beyond the matrix read its last row (a warp's first patch may begin there): no condition between the
      // loads, or they would wait for one another.
      const char* s = view.p + min(m, rows - 1) * in_ld;
      uint16_t x[CH];
      const bool in = lane < cols;
#pragma unroll
      for (int r = 0; r < CH; ++r) {
        x[r] = in ? *reinterpret_cast<const uint16_t*>(s) : (uint16_t)0;
        if (m + r + 1 < rows) s += in_ld;
      }
#pragma unroll
      for (int r = 0; r < CH; r += 2) raw.w[r / 2] = (uint32_t)x[r] | (uint32_t)x[r + 1] << 16;
    }
  }
  __device__ __forceinline__ void take(const Raw& raw, bool vec, uint32_t* q) const {
    if (vec) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
        ptx5::sts128(buf + (8 * i + (lane >> 2)) * PITCH + (lane & 3) * 16,
                     make_uint4(raw.w[4 * i], raw.w[4 * i + 1], raw.w[4 * i + 2], raw.w[4 * i + 3]));
    } else {
#pragma unroll
      for (int r = 0; r < CH; r += 2) {
        ptx5::sts16(buf + r * PITCH + lane * 2, (uint16_t)raw.w[r / 2]);
        ptx5::sts16(buf + (r + 1) * PITCH + lane * 2, (uint16_t)(raw.w[r / 2] >> 16));
      }
    }
    __syncwarp();
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      uint32_t r[4];
      ptx5::ldmatrix_x4_trans(matrix + b * 8 * PITCH, r);
      q[2 * b] = r[0];
      q[2 * b + 1] = r[1];
      q[2 * (MB + b)] = r[2];
      q[2 * (MB + b) + 1] = r[3];
    }
    __syncwarp();
  }
};

// `vec` bits of a problem: 16-byte rows of D, Z, U, R.
constexpr int VEC_D = 1, VEC_Z = 2, VEC_U = 4, VEC_R = 8;

// What a warp needs of a problem for one tile.
template <int CH>
struct Epilogue {
  Patch<CH> pt;
  typename Patch<CH>::View d, z, u, r;
  bool has_z, has_r;
  float unscale;  // see Params (read by the binary16 kernel without activation alone)
  float bias[4];  // bias[j]: of column 8 j + lane / 4 of the patch
  const float* row_scale;  // operands of 8 bits: of the tile's rows, or NULL; and of the columns, as `bias`
  float col[4], col_up[4];
};

// The scales of a patch's rows. Lane l holds that of row l % CH: one load, which is on its way since the patch before; a thread's rows,
// 8 b + 2 (lane % 4) and the next, come from the lanes that hold them. (With loads of its own in every thread, products value by value and
// eight epilogue warps, 4096 x 8192 x 512 took 44.5 us without activation, 58.1 with tanh-GELU and 78.6 with residual; now 37, 48.5 and 62.
// Twelve warps with loads of their own: 52.5 with tanh-GELU, 60.8 with residual, so that the residual's form gains nothing from this.)
template <int CH>
struct RowScales {
  float mine;
  __device__ __forceinline__ void fetch(const Epilogue<CH>& ep, int m) {
    mine = ep.row_scale ? __ldg(ep.row_scale + min(m + (ep.pt.lane & (CH - 1)), ep.pt.rows - 1)) : 1.f;
  }
  // Those of this thread.
  struct Own {
    float2 row[CH / 8];
  };
  __device__ __forceinline__ Own own() const {
    Own o;
    const int from = 2 * (threadIdx.x & 3);
#pragma unroll
    for (int b = 0; b < CH / 8; ++b) o.row[b] = make_float2(__shfl_sync(0xffffffffu, mine, 8 * b + from), __shfl_sync(0xffffffffu, mine, 8 * b + from + 1));
    return o;
  }
  // v row col + bias
  static __device__ __forceinline__ void apply(const Own& o, const float* col, const float* bias, float* v) {
    constexpr int MB = CH / 8;
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // columns
        float* x = v + 4 * ((j >> 1) * MB + b) + 2 * (j & 1);
        const float2 y = lnorm::fma2(lnorm::mul2(make_float2(x[0], x[1]), o.row[b]), lnorm::both(col[j]), lnorm::both(bias ? bias[j] : 0.f));
        x[0] = y.x;
        x[1] = y.y;
      }
  }
};

// The gradients' products, whose operand may have been scaled, run without activation; bfloat16 needs no scaling.
template <typename T, int ACT>
constexpr bool UNSCALED = std::is_same<T, __half>::value && ACT == HGEMM_ACT_NONE;

// next: the row whose residual is fetched in the place of this one's, or -1.
template <typename K, int CH, int ACT>
__device__ __forceinline__ void emit_plain(const Epilogue<CH>& ep, int m, float* v, typename Patch<CH>::Raw& raw, const RowScales<CH>& rs, int next) {
  using T = typename Kind<K>::Out;
  constexpr int MB = CH / 8;
  if constexpr (Kind<K>::EIGHT) rs.apply(rs.own(), ep.col, ep.bias, v);
  const auto bias = [&](int i) { return Kind<K>::EIGHT ? 0.f : ep.bias[2 * (i / (4 * MB)) + ((i >> 1) & 1)]; };  // still to be added to v[i]
  if (UNSCALED<K, ACT> && ep.unscale != 1.f) {
#pragma unroll
    for (int i = 0; i < CH; ++i) v[i] *= ep.unscale;
  }
  uint32_t q[CH / 2], r[CH / 2];
  if (ep.has_r) {
    ep.pt.take(raw, ep.r.vec, r);
    if (next >= 0) ep.pt.fetch(raw, ep.r, next);
  }
  if (ep.has_z) {
#pragma unroll
    for (int i = 0; i < CH; i += 2) {
      const float b = bias(i);
      q[i / 2] = pack2<T>(v[i] + b, v[i + 1] + b);
    }
    ep.pt.store(ep.z, m, q);
  }
#pragma unroll
  for (int i = 0; i < CH; i += 2) {
    const float b = bias(i);
    float x = act_fwd<ACT>(v[i] + b), y = act_fwd<ACT>(v[i + 1] + b);
    if (ep.has_r) {
      const float2 a = unpack2<T>(r[i / 2]);
      x += a.x;
      y += a.y;
    }
    q[i / 2] = pack2<T>(x, y);
  }
  ep.pt.store(ep.d, m, q);
}

template <typename K, int CH, int ACT>
__device__ __forceinline__ void emit_gated(const Epilogue<CH>& ep, int m, float* g, float* u, const RowScales<CH>& rs) {
  using T = typename Kind<K>::Out;
  if constexpr (Kind<K>::EIGHT) {
    const typename RowScales<CH>::Own own = rs.own();
    rs.apply(own, ep.col, nullptr, g);
    rs.apply(own, ep.col_up, nullptr, u);
  }
  uint32_t q[CH / 2];
  if (ep.has_z) {
#pragma unroll
    for (int i = 0; i < CH; i += 2) q[i / 2] = pack2<T>(g[i], g[i + 1]);
    ep.pt.store(ep.z, m, q);
#pragma unroll
    for (int i = 0; i < CH; i += 2) q[i / 2] = pack2<T>(u[i], u[i + 1]);
    ep.pt.store(ep.u, m, q);
  }
#pragma unroll
  for (int i = 0; i < CH; i += 2) q[i / 2] = pack2<T>(act_fwd<ACT>(g[i]) * u[i], act_fwd<ACT>(g[i + 1]) * u[i + 1]);
  ep.pt.store(ep.d, m, q);
}

// CH columns of a warp's 32 lanes, in the patch's order, from the lane and column in `addr`.
template <int CH>
__device__ __forceinline__ void tmem_load(uint32_t addr, float* v) {
  ptx5::tmem_ld_16x256b<CH / 8>(addr, v);
  ptx5::tmem_ld_16x256b<CH / 8>(addr + (16u << 16), v + CH / 2);
}

// The sum of a cut tile's parts, in order, for one thread's CH values: the first at `first`, the others `stride` apart
// from `ws`; the loads of four parts are in flight.
template <int CH>
__device__ __forceinline__ void add_parts(const float4* first, const float4* ws, int others, long long stride, float* v) {
#pragma unroll
  for (int j = 0; j < CH / 4; ++j) *reinterpret_cast<float4*>(v + 4 * j) = __ldcg(first + j * 32);
  int s = 0;
  for (; s + 4 <= others; s += 4) {
    float4 x[4][CH / 4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int j = 0; j < CH / 4; ++j) x[q][j] = __ldcg(ws + (s + q) * stride + j * 32);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int j = 0; j < CH / 4; ++j) {
        v[4 * j] += x[q][j].x;
        v[4 * j + 1] += x[q][j].y;
        v[4 * j + 2] += x[q][j].z;
        v[4 * j + 3] += x[q][j].w;
      }
  }
  for (; s < others; ++s)
#pragma unroll
    for (int j = 0; j < CH / 4; ++j) {
      const float4 x = __ldcg(ws + s * stride + j * 32);
      v[4 * j] += x.x;
      v[4 * j + 1] += x.y;
      v[4 * j + 2] += x.z;
      v[4 * j + 3] += x.w;
    }
}

// One epilogue warp: its accumulator quarter, buffers and place.
struct EpiWarp {
  uint32_t acc, bufs, last_flag, acc_empty;
  int e, quad, group, lane, block;  // block: of 128 lanes among the tile's CG x NB
};

__device__ __forceinline__ void sts32(uint32_t addr, int v) { asm volatile("st.shared.s32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ int lds32(uint32_t addr) {
  int v;
  asm volatile("ld.shared.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// The epilogue of one unit for one warp.
template <typename T, typename C, int ACT>
__device__ __forceinline__ void epilogue_unit(const Params& p, const Problem& pr, const Work& w, const Epilogue<C::CH>& ep,
                                              typename Patch<C::CH>::Raw& raw, const EpiWarp& ew, int rows, bool n_in) {
  using namespace dgemm::ptx;
  constexpr int CG = C::CG, BM = C::BM, CH = C::CH, BLOCKS = C::CG * C::NB, EPI_WARPS = C::EPI_WARPS, GROUPS = EPI_WARPS / 4;
  constexpr bool GATED = C::GATED, EIGHT = Kind<T>::EIGHT;
  // a part's sums in the workspace: [slot][block][quarter][chunk][CH / 4][lane] of float4
  constexpr long long WS_SLOT = (long long)BLOCKS * BM * 32;  // float4 per slot
  constexpr int WS_CHUNK = CH / 4 * 32;                   // float4 per quarter and chunk
  float4* const ws_cta = reinterpret_cast<float4*>(p.ws) + ew.block * (BM * 32) + ew.lane;
  // the accumulator may be overwritten: called once this warp's last load of it has been waited for
  bool released = false;
  const auto release = [&]() {
    ptx5::fence_before_sync();
    __syncwarp();
    if (ew.lane == 0) {
      if (CG == 1) mbar_arrive(ew.acc_empty);
      else ptx5::mbar_arrive_cluster_relaxed(map_to_cta(ew.acc_empty, 0));
    }
    released = true;
  };
  if (w.slot < 0) {
    if constexpr (EIGHT && !GATED) {
      // the next chunk's scales and residual are on their way while this one is computed
      RowScales<CH> rs;
      if (ew.group * CH < rows) rs.fetch(ep, ew.group * CH);
      for (int c = ew.group; c * CH < rows; c += GROUPS) {
        float v[CH];
        tmem_load<CH>(ew.acc + c * CH, v);
        ptx5::tmem_ld_wait<CH>(v);
        const RowScales<CH> rows_now = rs;
        const int next = (c + GROUPS) * CH;
        if (next < rows) rs.fetch(ep, next);
        else release();
        if (n_in) emit_plain<T, CH, ACT>(ep, c * CH, v, raw, rows_now, next < rows ? next : -1);
      }
    } else if constexpr (!GATED) {
      for (int c = ew.group; c * CH < rows; c += GROUPS) {
        float v[CH];
        tmem_load<CH>(ew.acc + c * CH, v);
        ptx5::tmem_ld_wait<CH>(v);
        if ((c + GROUPS) * CH >= rows) release();
        if (n_in) {
          typename Patch<CH>::Raw now = raw;
          // the next chunk's residual is on its way while this one is computed
          if (ep.has_r && (c + GROUPS) * CH < rows) ep.pt.fetch(raw, ep.r, (c + GROUPS) * CH);
          emit_plain<T, CH, ACT>(ep, c * CH, v, now, RowScales<CH>{1.f}, -1);
        }
      }
    } else {
      // Lanes 0-63 hold g, lanes 64-127 hold u of the same 64 columns. Two chunks at a time: the
      // g warp takes u of the first from its partner, the u warp takes g of the second.
      const bool is_g = ew.quad < 2;
      const uint32_t mine = ew.bufs + ew.e * C::BUF_BYTES + ew.lane * 16, theirs = ew.bufs + (ew.e ^ 2) * C::BUF_BYTES + ew.lane * 16;
      for (int c = 2 * ew.group; c * CH < rows; c += 2 * GROUPS) {
        float v[CH], o[CH];
        RowScales<CH> rs;
        const int m = (is_g ? c : c + 1) * CH;
        if (EIGHT) rs.fetch(ep, m);
        tmem_load<CH>(ew.acc + (is_g ? c + 1 : c) * CH, o);  // what the partner needs
        tmem_load<CH>(ew.acc + (is_g ? c : c + 1) * CH, v);  // what stays here
        ptx5::tmem_ld_wait<CH>(o);
        ptx5::tmem_ld_wait<CH>(v);
        if ((c + 2 * GROUPS) * CH >= rows) release();
#pragma unroll
        for (int j = 0; j < CH / 4; ++j) ptx5::sts128(mine + j * 512, *reinterpret_cast<const uint4*>(o + 4 * j));
        named_barrier_sync(1 + ew.group * 2 + (ew.quad & 1), 64);
#pragma unroll
        for (int j = 0; j < CH / 4; ++j) *reinterpret_cast<uint4*>(o + 4 * j) = ptx5::lds128(theirs + j * 512);
        named_barrier_sync(1 + ew.group * 2 + (ew.quad & 1), 64);
        if (n_in && m < rows) {
          if (is_g) emit_gated<T, CH, ACT>(ep, m, v, o, rs);
          else emit_gated<T, CH, ACT>(ep, m, o, v, rs);
        }
      }
    }
  } else {
    float4* ws = ws_cta + w.slot * WS_SLOT + (ew.quad * (BM / CH)) * WS_CHUNK;
    for (int c = ew.group; c * CH < rows; c += GROUPS) {
      float v[CH];
      tmem_load<CH>(ew.acc + c * CH, v);
      ptx5::tmem_ld_wait<CH>(v);
#pragma unroll
      for (int j = 0; j < CH / 4; ++j) __stcg(ws + c * WS_CHUNK + j * 32, make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
    }
  }
  if (!released) release();
  if (w.slot >= 0) {
    int* counter = p.counters + w.left * BLOCKS + ew.block;
    __threadfence();
    named_barrier_sync(15, EPI_WARPS * 32);
    if (ew.e == 0 && ew.lane == 0) {
      const int old = atomicAdd(counter, 1);
      sts32(ew.last_flag, old == w.parts - 1);
      if (old == w.parts - 1) *counter = 0;  // ready for the next launch
    }
    named_barrier_sync(15, EPI_WARPS * 32);
    if (lds32(ew.last_flag)) {
      __threadfence();
      if (!GATED) {
        const float4* first = ws_cta + w.first_slot * WS_SLOT + (ew.quad * (BM / CH)) * WS_CHUNK;
        const float4* next = ws_cta + w.next_slot * WS_SLOT + (ew.quad * (BM / CH)) * WS_CHUNK;
        for (int c = ew.group; c * CH < rows; c += GROUPS) {
          if (ep.has_r && n_in) ep.pt.fetch(raw, ep.r, c * CH);
          float v[CH];
          RowScales<CH> rs;
          if (EIGHT) rs.fetch(ep, c * CH);
          add_parts<CH>(first + c * WS_CHUNK, next + c * WS_CHUNK, w.parts - 1, 2 * WS_SLOT, v);
          if (n_in) emit_plain<T, CH, ACT>(ep, c * CH, v, raw, rs, -1);
        }
      } else {
        const float4* first = ws_cta + w.first_slot * WS_SLOT + ((ew.quad & 1) * (BM / CH)) * WS_CHUNK;
        const float4* next = ws_cta + w.next_slot * WS_SLOT + ((ew.quad & 1) * (BM / CH)) * WS_CHUNK;
        constexpr int UP = 2 * (BM / CH) * WS_CHUNK;  // the up projection's quarters
        for (int c = 2 * ew.group + (ew.quad >> 1); c * CH < rows; c += 2 * GROUPS) {
          float g[CH], uu[CH];
          RowScales<CH> rs;
          if (EIGHT) rs.fetch(ep, c * CH);
          add_parts<CH>(first + c * WS_CHUNK, next + c * WS_CHUNK, w.parts - 1, 2 * WS_SLOT, g);
          add_parts<CH>(first + UP + c * WS_CHUNK, next + UP + c * WS_CHUNK, w.parts - 1, 2 * WS_SLOT, uu);
          if (n_in) emit_gated<T, CH, ACT>(ep, c * CH, g, uu, rs);
        }
      }
    }
    named_barrier_sync(15, EPI_WARPS * 32);  // last_flag may be rewritten
  }
}

// Shared-memory descriptor of an operand tile made of 64 x 64 boxes with 128-byte swizzle. K-major:
// 8-row groups are 1024 bytes apart. MN-major: the 64-value chunks of the outer index are one
// box apart, groups of 8 k are 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, bool mn_major) {
  const uint64_t lbo = mn_major ? BOX_BYTES >> 4 : 1, sbo = 1024 >> 4;
  return (uint64_t)((addr & 0x3FFFF) >> 4) | (lbo << 16) | (sbo << 32) | (1ull << 46) | (2ull << 61);
}

template <typename T, int CG, int BM, int NB, bool GATED, int ACT>
__global__ void __launch_bounds__(Cfg<CG, BM, NB, GATED, Kind<T>::EIGHT>::THREADS, 1) hgemm_tc_kernel(const __grid_constant__ Params p) {
  using namespace dgemm::ptx;
  using C = Cfg<CG, BM, NB, GATED, Kind<T>::EIGHT>;
  using Out = typename Kind<T>::Out;
  constexpr bool EIGHT = Kind<T>::EIGHT;
  constexpr int STAGES = C::STAGES, CH = C::CH;

  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t pad = (1024 - (raw & 1023)) & 1023;
  const uint32_t base = raw + pad;  // the same offset in both CTAs of a pair (same kernel, same launch)
  uint8_t* gen = smem_raw + pad;
  const uint32_t bufs = base + STAGES * C::STAGE_BYTES;
  uint8_t* ctrl = gen + STAGES * C::STAGE_BYTES + C::BUFS_BYTES;
  const uint32_t bars = bufs + C::BUFS_BYTES;
  const uint32_t full_bar = bars, empty_bar = bars + 8 * STAGES;        // stage s at + 8 s
  const uint32_t acc_full = bars + 16 * STAGES, acc_empty = acc_full + 16;  // accumulator a at + 8 a
  const uint32_t drain_bar = acc_empty + 16;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctrl + 16 * STAGES + 48);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + 16 * STAGES + 52);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = CG == 1 ? 0 : (int)cluster_ctarank();
  const int cluster = (int)blockIdx.x / CG, clusters = (int)gridDim.x / CG;

  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full_bar + 8 * s, 1);
      mbar_init(empty_bar + 8 * s, 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full + 8 * a, 1);
      mbar_init(acc_empty + 8 * a, C::EPI_WARPS * CG);
    }
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 2) ptx5::tmem_alloc<CG>(bars + 16 * STAGES + 48, C::TMEM_COLS);
  ptx5::fence_before_sync();
  if (CG == 1) {
    __syncthreads();
  } else {
    cluster_arrive_release();
    cluster_wait_acquire();
  }
  ptx5::fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  ptx5::launch_dependents();
  grid_dependency_wait();
  if ((warp == 0 || warp == 2 || warp == 3) && lane == 0) {
    // ---- stages: warps 0 and 2 copy half of the P boxes each, warp 3 the Q boxes: one stream of copies brings about 35
    // bytes per clock. Zero fill outside the matrices ----
    const bool is_p = warp != 3;
    const int half = warp == 2 ? 1 : 0;
    uint32_t it = 0;
    bool ok = !p.drop;
    Work w;
    for (int j = 0; ok && get_work(p, cluster, clusters, j, w); ++j) {
      const Problem& pr = p.prob[w.prob];
      int tm, tn;
      tile_to_mn(pr, w.tile, tm, tn);
      const int n0 = tn * C::NT + rank * NB * C::BLOCK, m0 = tm * BM + rank * C::QROWS;
      const uint32_t bytes = CG * (C::P_BYTES + (pr.q_mn ? C::QBOXES * BOX_BYTES : C::QROWS * 128));
      for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
        const uint32_t s = it % STAGES, ph = (it / STAGES) & 1u;
        if (!wait_bounded(empty_bar + 8 * s, ph ^ 1u, abort_flag, p)) {
          ok = false;
          break;
        }
        const uint32_t fb = CG == 1 ? full_bar + 8 * s : map_to_cta(full_bar + 8 * s, 0);
        if (warp == 0 && rank == 0) mbar_arrive_expect_tx(full_bar + 8 * s, bytes);
        const int seg = kb >= pr.kb_seg0 ? 1 : 0;
        const int k0 = (kb - (seg ? pr.kb_seg0 : 0)) * Kind<T>::TK;
        const uint32_t dst = base + s * C::STAGE_BYTES;
        const auto load_p = [&](int i) {
          const CUtensorMap* map = &pr.p[GATED ? i & 1 : seg];
          const int n = n0 + 64 * (GATED ? i >> 1 : i);
          ptx5::tma_load_2d<CG>(dst + i * BOX_BYTES, map, pr.p_mn ? n : k0, pr.p_mn ? k0 : n, fb);
        };
        if (is_p) {
          load_p(NB * half);
          if (NB == 2 && (GATED || pr.p_mn)) load_p(NB * half + 1);
        } else {
          const CUtensorMap* map = &pr.q[GATED ? 0 : seg];
          if (pr.q_mn) {
#pragma unroll
            for (int i = 0; i < C::QBOXES; ++i) ptx5::tma_load_2d<CG>(dst + C::P_BYTES + i * BOX_BYTES, map, m0 + 64 * i, k0, fb);
          } else {
            ptx5::tma_load_2d<CG>(dst + C::P_BYTES, map, k0, m0, fb);
          }
        }
      }
    }
    // After a normal run every copy has been consumed. After an abort let the copies in flight land
    // (bounded); the leader's barriers count the bytes of both CTAs of a pair.
    if (!ok && !p.drop && warp == 0 && rank == 0) {
      const uint32_t n_inflight = it < (uint32_t)STAGES ? it : (uint32_t)STAGES;
      for (uint32_t j = it - n_inflight; j < it; ++j) {
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try_wait(full_bar + 8 * (j % STAGES), (j / STAGES) & 1u))
          if (globaltimer_ns() - t0 > 500000000ull) break;
      }
    }
  } else if (warp == 1 && lane == 0 && rank == 0) {
    // ---- MMAs ----
    constexpr uint32_t fmt = Kind<T>::FORMAT;
    constexpr uint32_t idesc0 = (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)(BM >> 3) << 17) | ((uint32_t)((128 * CG) >> 4) << 24);
    uint32_t it = 0, acc_it = 0;
    bool ok = true;
    Work w;
    for (; ok && get_work(p, cluster, clusters, (int)acc_it, w); ++acc_it) {
      const Problem& pr = p.prob[w.prob];
      const uint32_t idesc = idesc0 | ((uint32_t)pr.p_mn << 15) | ((uint32_t)pr.q_mn << 16);
      const uint32_t p_step = pr.p_mn ? 2048 >> 4 : 32 >> 4, q_step = pr.q_mn ? 2048 >> 4 : 32 >> 4;
      const auto mmas = [&](uint32_t stage, uint32_t d, int block, bool first) {
        const uint32_t src = base + stage * C::STAGE_BYTES;
        const uint64_t pd = smem_desc(src + block * 2 * BOX_BYTES, pr.p_mn), qd = smem_desc(src + C::P_BYTES, pr.q_mn);
#pragma unroll
        for (int k = 0; k < 4; ++k) ptx5::mma<CG, EIGHT>(d, pd + k * p_step, qd + k * q_step, idesc, !first || k > 0);
      };
      const auto staged = [&](uint32_t i) {
        if (!wait_bounded(full_bar + 8 * (i % STAGES), (i / STAGES) & 1u, abort_flag, p)) return false;
        ptx5::fence_after_sync();
        return true;
      };
      if constexpr (NB == 1) {
        const uint32_t a = acc_it & 1u;
        if (!wait_bounded(acc_empty + 8 * a, ((acc_it >> 1) & 1u) ^ 1u, abort_flag, p)) {
          ok = false;
          break;
        }
        ptx5::fence_after_sync();
        for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
          if (!staged(it)) {
            ok = false;
            break;
          }
          mmas(it % STAGES, tmem + a * BM, 0, kb == w.kb0);
          ptx5::mma_commit<CG>(empty_bar + 8 * (it % STAGES));
        }
        if (ok) ptx5::mma_commit<CG>(acc_full + 8 * a);
      } else {
        // The first block's accumulator is drained first: its MMAs on all staged k-blocks run while the second one's is
        // still being read; then the second block catches up.
        const int nkb = w.kb1 - w.kb0, ahead = min(nkb, STAGES);
        if (!wait_bounded(acc_empty, (acc_it & 1u) ^ 1u, abort_flag, p)) ok = false;
        ptx5::fence_after_sync();
        for (int i = 0; ok && i < ahead; ++i) {
          if (!(ok = staged(it + i))) break;
          mmas((it + i) % STAGES, tmem, 0, i == 0);
        }
        if (ok && ahead == nkb) ptx5::mma_commit<CG>(acc_full);
        if (ok && !wait_bounded(acc_empty + 8, (acc_it & 1u) ^ 1u, abort_flag, p)) ok = false;
        ptx5::fence_after_sync();
        for (int i = 0; ok && i < ahead; ++i) {
          mmas((it + i) % STAGES, tmem + BM, 1, i == 0);
          ptx5::mma_commit<CG>(empty_bar + 8 * ((it + i) % STAGES));
        }
        for (int i = ahead; ok && i < nkb; ++i) {
          if (!(ok = staged(it + i))) break;
          mmas((it + i) % STAGES, tmem, 0, false);
          if (i == nkb - 1) ptx5::mma_commit<CG>(acc_full);
          mmas((it + i) % STAGES, tmem + BM, 1, false);
          ptx5::mma_commit<CG>(empty_bar + 8 * ((it + i) % STAGES));
        }
        if (ok) ptx5::mma_commit<CG>(acc_full + 8);
        it += nkb;
      }
    }
    if (!ok) {  // leave no MMA in flight (bounded)
      ptx5::mma_commit<CG>(drain_bar);
      const unsigned long long t0 = globaltimer_ns();
      while (!mbar_try_wait(drain_bar, 0))
        if (globaltimer_ns() - t0 > 500000000ull) break;
    }
  } else if (warp >= 4) {
    // ---- epilogue: warp e takes TMEM quarter e % 4 and every GROUPS-th chunk (pair of chunks if gated) ----
    const int e = warp - 4, quad = warp & 3, group = e >> 2;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const uint32_t buf = bufs + e * C::BUF_BYTES;
    uint32_t acc_it = 0;
    // After a wait has given up, the warps still walk through the rest of the units together (without
    // waiting again), so that every named barrier below is met by all of its warps.
    bool dead = false;
    const float unscale = !GATED && UNSCALED<T, ACT> && p.unscale ? __ldcg(p.unscale) : 1.f;
    Work w;
    for (; get_work(p, cluster, clusters, (int)acc_it, w); ++acc_it) {
      const Problem& pr = p.prob[w.prob];
      int tm, tn;
      tile_to_mn(pr, w.tile, tm, tn);
      const int m_base = tm * BM, rows = min(pr.M - m_base, BM);
      for (int h = 0; h < NB; ++h) {
        const int n0 = tn * C::NT + (rank * NB + h) * C::BLOCK + (GATED ? (quad & 1) * 32 : quad * 32);
        const bool n_in = n0 < pr.N;  // (the whole warp: a patch beyond the last column has nothing to do)
        Epilogue<CH> ep;
        ep.pt = Patch<CH>{rows, pr.N - n0, lane, buf, buf + (lane & 7) * PITCH + (lane >> 3) * 16};
        ep.unscale = unscale;
        ep.has_z = pr.Z != nullptr;
        ep.has_r = !GATED && pr.R != nullptr;
        ep.d = ep.pt.view(pr.D, pr.ldd, pr.vec & VEC_D, m_base, n0);
        if (ep.has_z) ep.z = ep.pt.view(pr.Z, pr.ldz, pr.vec & VEC_Z, m_base, n0);
        if (GATED && ep.has_z) ep.u = ep.pt.view(pr.U, pr.ldu, pr.vec & VEC_U, m_base, n0);
        if (ep.has_r) ep.r = ep.pt.view(pr.R, pr.ldr, pr.vec & VEC_R, m_base, n0);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int n = n0 + 8 * j + (lane >> 2);
          ep.bias[j] = !GATED && pr.bias && n < pr.N ? to_f32(static_cast<const Out*>(pr.bias)[n]) : 0.f;
          if (EIGHT) {
            ep.col[j] = pr.col_scale[0] && n < pr.N ? __ldg(pr.col_scale[0] + n) : 1.f;
            if (GATED) ep.col_up[j] = pr.col_scale[1] && n < pr.N ? __ldg(pr.col_scale[1] + n) : 1.f;
          }
        }
        if (EIGHT) ep.row_scale = pr.row_scale ? pr.row_scale + m_base : nullptr;
        typename Patch<CH>::Raw raw;
        if (ep.has_r && n_in && w.slot < 0) ep.pt.fetch(raw, ep.r, group * CH);
        const uint32_t a = NB == 1 ? acc_it & 1u : (uint32_t)h;
        if (!dead) dead = !wait_bounded(acc_full + 8 * a, (NB == 1 ? acc_it >> 1 : acc_it) & 1u, abort_flag, p);
        __syncwarp();
        ptx5::fence_after_sync();
        const EpiWarp ew{tmem + a * BM + lane_addr, bufs, bars + 16 * STAGES + 56, acc_empty + 8 * a, e, quad, group, lane, rank * NB + h};
        epilogue_unit<T, C, ACT>(p, pr, w, ep, raw, ew, rows, n_in);
      }
    }
  }
  __syncwarp();

  // Leaving: both CTAs of a pair together (the leader's MMAs read both shared memories).
  ptx5::fence_before_sync();
  if (CG == 1) {
    __syncthreads();
  } else {
    cluster_arrive_release();
    cluster_wait_acquire();
  }
  ptx5::fence_after_sync();
  if (warp == 2) ptx5::tmem_dealloc<CG>(tmem, C::TMEM_COLS);
}

}  // namespace hgemm
