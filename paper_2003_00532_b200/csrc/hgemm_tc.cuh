// 16-bit matrix products on the fifth-generation tensor cores, with what follows the product in
// the epilogue: bias, activation, residual, or the gated pair act(G) * U.
//
// Orientation. The tile's 128 TMEM lanes (256 over a CTA pair) run along the output's columns n and
// its BM TMEM columns along the output's rows m: D^T = P Q^T with P = op(B)^T ("lane operand", the
// weights) and Q = op(A) ("column operand", the tokens). Then
//   - a warp of the epilogue holds 32 consecutive n of one row m in its 32 lanes, so that every load
//     and store of D, Z, R is one contiguous 64-byte piece of a row, whatever the alignment or leading
//     dimension: no staging through shared memory and no aligned / unaligned variants;
//   - a bias is one register per thread;
//   - few rows (single tokens) need a small BM, not a 128-row tile: BM = 16 .. 256.
//
// Operands. Either may be stored with its contraction index contiguous ("K-major") or with its
// outer index contiguous ("MN-major"): both are staged by TMA in boxes of 64 x 64 values (rows of 128
// bytes, 128-byte swizzle, 8 KB) and the MMA descriptors say which of the two a box holds, so all four
// transpositions run the same code without a transposing pass.
//
// Work. One launch covers up to three problems (the gradients of one operator), each cut into tiles;
// tiles beyond the whole waves may have their k-blocks cut into parts, whose binary32 sums go to
// a workspace; the CTA that finishes the last part of a tile (a counter per tile) adds all parts in
// order and runs the epilogue: one launch, no CTA waits for another, same bits every time.
//
// Roles (384 threads): warps 0 and 3 stage P and Q (one thread that issued all copies was the limit:
// 479 ns per 64-wide k-block with four copies, against 366 ns for its MMAs; two threads with one or
// two copies each are not), warp 1 issues the MMAs, warp 2 owns the TMEM allocation, warps 4-11 run the epilogue of one accumulator while the MMAs fill the other. In a pair the MMAs of
// both CTAs are issued by the leader; each CTA stages its own 128 lanes and its half of Q.
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

namespace hgemm {

constexpr int TK = 64;           // k-block: 64 values of 16 bits = one 128-byte swizzled row
constexpr int BOX_BYTES = 8192;  // 64 x 64 values
constexpr int THREADS = 384;
constexpr int EPI_WARPS = 8;
constexpr int MAX_SMEM = 232448;  // 227 KB
constexpr int MAX_PROBLEMS = 3;

// CG: CTAs per tile (1, or a pair); BM: TMEM columns of the tile (rows of the output).
template <int CG_, int BM_, bool GATED_>
struct Cfg {
  static constexpr int CG = CG_, BM = BM_;
  static constexpr bool GATED = GATED_;
  static constexpr int QROWS = BM / CG;  // rows of Q that one CTA stages
  static constexpr int QBOXES = (QROWS + 63) / 64;
  static constexpr int P_BYTES = 2 * BOX_BYTES;
  static constexpr int STAGE_BYTES = P_BYTES + QBOXES * BOX_BYTES;
  static constexpr int CH = GATED ? (BM < 32 ? 8 : 16) : 16;  // TMEM columns one warp takes at a time
  static constexpr int XCHG_BYTES = GATED ? EPI_WARPS * CH * 128 : 0;  // g / u exchange between warps
  static constexpr int CTRL_BYTES = 512;
  static constexpr int FIT = (MAX_SMEM - 1024 - XCHG_BYTES - CTRL_BYTES) / STAGE_BYTES;
  static constexpr int STAGES = FIT < 8 ? FIT : 8;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + XCHG_BYTES + CTRL_BYTES + 1024;
  static constexpr int TMEM_COLS = 2 * BM < 32 ? 32 : 2 * BM;  // two accumulators (a power of two)
  static constexpr int NT = (GATED ? 64 : 128) * CG;           // output columns per tile
};

struct alignas(64) Problem {
  CUtensorMap p[2], q[2];  // [segment] of the contraction; gated: p[0] = gate weights, p[1] = up weights
  int N, M;                // output columns (lanes) and rows
  int tiles_n, tiles_m;
  int kblocks, kb_seg0;    // k-blocks in all, and of the first segment
  int p_mn, q_mn;          // operand stored MN-major
  int dp_tiles;            // tiles run whole; the others are cut into `split` parts of kb_per_split k-blocks
  int split, kb_per_split;
  int units;               // dp_tiles + (tiles - dp_tiles) * split
  int slot0, counter0;     // first workspace slot and tile counter of the cut tiles
  int act;
  const void* bias;
  const void* R;
  void* D;
  void* Z;                 // pre-activation; gated: gate pre-activation
  void* U;                 // gated: up pre-activation
  long long ldr, ldd, ldz, ldu;
};

struct Params {
  Problem prob[MAX_PROBLEMS];
  int nprob;
  int units;
  float* ws;
  int* counters;
  unsigned long long wait_limit_ns;
  int* status;
  int drop;  // testing aid: the producers skip their copies
};

struct Work {
  int prob, tile, kb0, kb1, part;  // part: -1 = whole tile
};

__device__ __forceinline__ Work get_work(const Params& p, int u) {
  Work w;
  w.prob = 0;
  while (w.prob + 1 < p.nprob && u >= p.prob[w.prob].units) u -= p.prob[w.prob++].units;
  const Problem& pr = p.prob[w.prob];
  if (u < pr.dp_tiles) {
    w.tile = u;
    w.kb0 = 0;
    w.kb1 = pr.kblocks;
    w.part = -1;
  } else {
    const int v = u - pr.dp_tiles;
    w.tile = pr.dp_tiles + v / pr.split;
    w.part = v % pr.split;
    w.kb0 = w.part * pr.kb_per_split;
    w.kb1 = min(pr.kblocks, w.kb0 + pr.kb_per_split);
  }
  return w;
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
__device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit_ns, int* status) {
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

// Rows m0 .. m0 + CH - 1 of column n: v[j] is the sum of row m0 + j. WHOLE: all of them are inside the
// matrix; otherwise those below M. All loads are issued before the first store (R may be D).
template <typename T, int CH, int ACT, bool WHOLE>
__device__ __forceinline__ void emit_plain(const Problem& pr, const float* v, float bias, int m0, int n) {
  const int rows = pr.M - m0;
  T r[CH];
  if (pr.R) {
    const T* src = static_cast<const T*>(pr.R) + (long long)m0 * pr.ldr + n;
#pragma unroll
    for (int j = 0; j < CH; ++j) r[j] = src[(WHOLE || j < rows ? j : 0) * pr.ldr];
  }
  if (pr.Z) {
    T* dst = static_cast<T*>(pr.Z) + (long long)m0 * pr.ldz + n;
#pragma unroll
    for (int j = 0; j < CH; ++j)
      if (WHOLE || j < rows) dst[j * pr.ldz] = from_f32<T>(v[j] + bias);
  }
  T* dst = static_cast<T*>(pr.D) + (long long)m0 * pr.ldd + n;
  if (pr.R) {
#pragma unroll
    for (int j = 0; j < CH; ++j)
      if (WHOLE || j < rows) dst[j * pr.ldd] = from_f32<T>(act_fwd<ACT>(v[j] + bias) + to_f32(r[j]));
  } else {
#pragma unroll
    for (int j = 0; j < CH; ++j)
      if (WHOLE || j < rows) dst[j * pr.ldd] = from_f32<T>(act_fwd<ACT>(v[j] + bias));
  }
}

template <typename T, int CH, int ACT, bool WHOLE>
__device__ __forceinline__ void emit_gated(const Problem& pr, const float* g, const float* u, int m0, int n) {
  const int rows = pr.M - m0;
  if (pr.Z) {
    T* zg = static_cast<T*>(pr.Z) + (long long)m0 * pr.ldz + n;
    T* zu = static_cast<T*>(pr.U) + (long long)m0 * pr.ldu + n;
#pragma unroll
    for (int j = 0; j < CH; ++j)
      if (WHOLE || j < rows) {
        zg[j * pr.ldz] = from_f32<T>(g[j]);
        zu[j * pr.ldu] = from_f32<T>(u[j]);
      }
  }
  T* dst = static_cast<T*>(pr.D) + (long long)m0 * pr.ldd + n;
#pragma unroll
  for (int j = 0; j < CH; ++j)
    if (WHOLE || j < rows) dst[j * pr.ldd] = from_f32<T>(act_fwd<ACT>(g[j]) * u[j]);
}

template <typename T, int CH, bool WHOLE>
__device__ __forceinline__ void emit_plain_act(const Problem& pr, const float* v, float bias, int m0, int n) {
  switch (pr.act) {
    case HGEMM_ACT_NONE: emit_plain<T, CH, HGEMM_ACT_NONE, WHOLE>(pr, v, bias, m0, n); break;
    case HGEMM_ACT_RELU: emit_plain<T, CH, HGEMM_ACT_RELU, WHOLE>(pr, v, bias, m0, n); break;
    case HGEMM_ACT_GELU: emit_plain<T, CH, HGEMM_ACT_GELU, WHOLE>(pr, v, bias, m0, n); break;
    case HGEMM_ACT_GELU_TANH: emit_plain<T, CH, HGEMM_ACT_GELU_TANH, WHOLE>(pr, v, bias, m0, n); break;
    default: emit_plain<T, CH, HGEMM_ACT_SILU, WHOLE>(pr, v, bias, m0, n); break;
  }
}
template <typename T, int CH>
__device__ __forceinline__ void emit_plain_any(const Problem& pr, const float* v, float bias, int m0, int n) {
  if (m0 + CH <= pr.M) emit_plain_act<T, CH, true>(pr, v, bias, m0, n);
  else emit_plain_act<T, CH, false>(pr, v, bias, m0, n);
}
template <typename T, int CH, bool WHOLE>
__device__ __forceinline__ void emit_gated_act(const Problem& pr, const float* g, const float* u, int m0, int n) {
  switch (pr.act) {
    case HGEMM_ACT_NONE: emit_gated<T, CH, HGEMM_ACT_NONE, WHOLE>(pr, g, u, m0, n); break;
    case HGEMM_ACT_RELU: emit_gated<T, CH, HGEMM_ACT_RELU, WHOLE>(pr, g, u, m0, n); break;
    case HGEMM_ACT_GELU: emit_gated<T, CH, HGEMM_ACT_GELU, WHOLE>(pr, g, u, m0, n); break;
    case HGEMM_ACT_GELU_TANH: emit_gated<T, CH, HGEMM_ACT_GELU_TANH, WHOLE>(pr, g, u, m0, n); break;
    default: emit_gated<T, CH, HGEMM_ACT_SILU, WHOLE>(pr, g, u, m0, n); break;
  }
}
template <typename T, int CH>
__device__ __forceinline__ void emit_gated_any(const Problem& pr, const float* g, const float* u, int m0, int n) {
  if (m0 + CH <= pr.M) emit_gated_act<T, CH, true>(pr, g, u, m0, n);
  else emit_gated_act<T, CH, false>(pr, g, u, m0, n);
}

template <int CH>
__device__ __forceinline__ void tmem_load(uint32_t addr, float* v) {
  if (CH == 8) ptx5::tmem_ld_x8(addr, v);
  else ptx5::tmem_ld_x16(addr, v);
}

// Shared-memory descriptor of an operand tile made of 64 x 64 boxes with 128-byte swizzle. K-major:
// 8-row groups are 1024 bytes apart. MN-major: the 64-value chunks of the outer index are one
// box apart, groups of 8 k are 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, bool mn_major) {
  const uint64_t lbo = mn_major ? BOX_BYTES >> 4 : 1, sbo = 1024 >> 4;
  return (uint64_t)((addr & 0x3FFFF) >> 4) | (lbo << 16) | (sbo << 32) | (1ull << 46) | (2ull << 61);
}

template <typename T, int CG, int BM, bool GATED>
__global__ void __launch_bounds__(THREADS, 1) hgemm_tc_kernel(const __grid_constant__ Params p) {
  using namespace dgemm::ptx;
  using C = Cfg<CG, BM, GATED>;
  constexpr int STAGES = C::STAGES, CH = C::CH;

  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t pad = (1024 - (raw & 1023)) & 1023;
  const uint32_t base = raw + pad;  // the same offset in both CTAs of a pair (same kernel, same launch)
  uint8_t* gen = smem_raw + pad;
  float* xchg = reinterpret_cast<float*>(gen + STAGES * C::STAGE_BYTES);
  uint8_t* ctrl = gen + STAGES * C::STAGE_BYTES + C::XCHG_BYTES;
  const uint32_t bars = base + STAGES * C::STAGE_BYTES + C::XCHG_BYTES;
  const uint32_t full_bar = bars, empty_bar = bars + 8 * STAGES;        // stage s at + 8 s
  const uint32_t acc_full = bars + 16 * STAGES, acc_empty = acc_full + 16;  // accumulator a at + 8 a
  const uint32_t drain_bar = acc_empty + 16;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(ctrl + 16 * STAGES + 48);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(ctrl + 16 * STAGES + 52);
  volatile int* last_flag = reinterpret_cast<volatile int*>(ctrl + 16 * STAGES + 56);

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
      mbar_init(acc_empty + 8 * a, EPI_WARPS * CG);
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

  if ((warp == 0 || warp == 3) && lane == 0) {
    // ---- stages: warp 0 copies the P boxes, warp 3 the Q boxes; zero fill outside the matrices ----
    const bool is_p = warp == 0;
    uint32_t it = 0;
    bool ok = !p.drop;
    for (int u = cluster; u < p.units && ok; u += clusters) {
      const Work w = get_work(p, u);
      const Problem& pr = p.prob[w.prob];
      int tm, tn;
      tile_to_mn(pr, w.tile, tm, tn);
      const bool mn = is_p ? pr.p_mn : pr.q_mn;
      // first outer index of this CTA's rows of the operand
      const int o0 = is_p ? tn * C::NT + rank * (GATED ? 64 : 128) : tm * BM + rank * C::QROWS;
      const int boxes = is_p ? (GATED || mn ? 2 : 1) : (mn ? C::QBOXES : 1);
      const int o_step = is_p && GATED ? 0 : 64;
      const CUtensorMap* maps = is_p ? pr.p : pr.q;
      const uint32_t bytes = CG * (C::P_BYTES + (pr.q_mn ? C::QBOXES * BOX_BYTES : C::QROWS * 128));
      for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
        const uint32_t s = it % STAGES, ph = (it / STAGES) & 1u;
        if (!wait_bounded(empty_bar + 8 * s, ph ^ 1u, abort_flag, p)) {
          ok = false;
          break;
        }
        const uint32_t fb = CG == 1 ? full_bar + 8 * s : map_to_cta(full_bar + 8 * s, 0);
        if (is_p && rank == 0) mbar_arrive_expect_tx(full_bar + 8 * s, bytes);
        const int seg = kb >= pr.kb_seg0 ? 1 : 0;
        const int k0 = (kb - (seg ? pr.kb_seg0 : 0)) * TK;
        const uint32_t dst = base + s * C::STAGE_BYTES + (is_p ? 0 : C::P_BYTES);
        for (int i = 0; i < boxes; ++i) {
          const CUtensorMap* map = maps + (GATED ? (is_p ? i : 0) : seg);
          const int o = o0 + i * o_step;
          ptx5::tma_load_2d<CG>(dst + i * BOX_BYTES, map, mn ? o : k0, mn ? k0 : o, fb);
        }
      }
    }
    // After a normal run every copy has been consumed. After an abort let the copies in flight land
    // (bounded); the leader's barriers count the bytes of both CTAs of a pair.
    if (!ok && !p.drop && is_p && rank == 0) {
      const uint32_t n_inflight = it < (uint32_t)STAGES ? it : (uint32_t)STAGES;
      for (uint32_t j = it - n_inflight; j < it; ++j) {
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try_wait(full_bar + 8 * (j % STAGES), (j / STAGES) & 1u))
          if (globaltimer_ns() - t0 > 500000000ull) break;
      }
    }
  } else if (warp == 1 && lane == 0 && rank == 0) {
    // ---- MMAs ----
    constexpr uint32_t fmt = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
    constexpr uint32_t idesc0 = (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)(BM >> 3) << 17) | ((uint32_t)((128 * CG) >> 4) << 24);
    uint32_t it = 0, acc_it = 0;
    bool ok = true;
    for (int u = cluster; u < p.units && ok; u += clusters, ++acc_it) {
      const Work w = get_work(p, u);
      const Problem& pr = p.prob[w.prob];
      const uint32_t idesc = idesc0 | ((uint32_t)pr.p_mn << 15) | ((uint32_t)pr.q_mn << 16);
      const uint32_t p_step = pr.p_mn ? 2048 >> 4 : 32 >> 4, q_step = pr.q_mn ? 2048 >> 4 : 32 >> 4;
      const uint32_t a = acc_it & 1u;
      if (!wait_bounded(acc_empty + 8 * a, ((acc_it >> 1) & 1u) ^ 1u, abort_flag, p)) {
        ok = false;
        break;
      }
      ptx5::fence_after_sync();
      const uint32_t d = tmem + a * BM;
      for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
        const uint32_t s = it % STAGES, ph = (it / STAGES) & 1u;
        if (!wait_bounded(full_bar + 8 * s, ph, abort_flag, p)) {
          ok = false;
          break;
        }
        ptx5::fence_after_sync();
        const uint32_t src = base + s * C::STAGE_BYTES;
        const uint64_t pd = smem_desc(src, pr.p_mn), qd = smem_desc(src + C::P_BYTES, pr.q_mn);
#pragma unroll
        for (int k = 0; k < TK / 16; ++k) ptx5::mma_f16<CG>(d, pd + k * p_step, qd + k * q_step, idesc, kb > w.kb0 || k > 0);
        ptx5::mma_commit<CG>(empty_bar + 8 * s);
      }
      if (ok) ptx5::mma_commit<CG>(acc_full + 8 * a);
    }
    if (!ok) {  // leave no MMA in flight (bounded)
      ptx5::mma_commit<CG>(drain_bar);
      const unsigned long long t0 = globaltimer_ns();
      while (!mbar_try_wait(drain_bar, 0))
        if (globaltimer_ns() - t0 > 500000000ull) break;
    }
  } else if (warp >= 4) {
    // ---- epilogue ----
    const int e = warp - 4, quad = warp & 3, half = e >> 2;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const int l = quad * 32 + lane;  // this thread's TMEM lane
    uint32_t acc_it = 0;
    // After a wait has given up, the warps still walk through the rest of the units together (without
    // waiting again), so that every named barrier below is met by all of its warps.
    bool dead = false;
    for (int u = cluster; u < p.units; u += clusters, ++acc_it) {
      const Work w = get_work(p, u);
      const Problem& pr = p.prob[w.prob];
      int tm, tn;
      tile_to_mn(pr, w.tile, tm, tn);
      const int m_base = tm * BM;
      const int n = GATED ? tn * C::NT + rank * 64 + (l & 63) : tn * C::NT + rank * 128 + l;
      const bool n_in = n < pr.N;
      const uint32_t a = acc_it & 1u;
      const float bias = !GATED && pr.bias && n_in ? to_f32(static_cast<const T*>(pr.bias)[n]) : 0.f;
      if (!dead) dead = !wait_bounded(acc_full + 8 * a, (acc_it >> 1) & 1u, abort_flag, p);
      ptx5::fence_after_sync();
      const uint32_t t_acc = tmem + a * BM + lane_addr;
      if (w.part < 0) {
        if (!GATED) {
          for (int c = half; c < BM / CH; c += 2) {
            if (m_base + c * CH >= pr.M) break;
            float v[CH];
            tmem_load<CH>(t_acc + c * CH, v);
            ptx5::tmem_ld_wait<CH>(v);
            if (n_in) emit_plain_any<T, CH>(pr, v, bias, m_base + c * CH, n);
          }
        } else {
          // Lanes 0-63 hold g, lanes 64-127 hold u of the same 64 columns. Two chunks at a time: the
          // g warp takes u of the first from its partner, the u warp takes g of the second.
          const bool is_g = quad < 2;
          float* mine = xchg + e * (CH * 32);
          const float* theirs = xchg + (e ^ 2) * (CH * 32);
          for (int c = 2 * half; c < BM / CH; c += 4) {
            if (m_base + c * CH >= pr.M) break;
            float v[CH], o[CH];
            tmem_load<CH>(t_acc + (is_g ? c + 1 : c) * CH, o);  // what the partner needs
            tmem_load<CH>(t_acc + (is_g ? c : c + 1) * CH, v);  // what stays here
            ptx5::tmem_ld_wait<CH>(o);
            ptx5::tmem_ld_wait<CH>(v);
#pragma unroll
            for (int j = 0; j < CH; ++j) mine[j * 32 + lane] = o[j];
            named_barrier_sync(1 + half * 2 + (quad & 1), 64);
#pragma unroll
            for (int j = 0; j < CH; ++j) o[j] = theirs[j * 32 + lane];
            named_barrier_sync(1 + half * 2 + (quad & 1), 64);
            const int m0 = m_base + (is_g ? c : c + 1) * CH;
            if (n_in && m0 < pr.M) emit_gated_any<T, CH>(pr, is_g ? v : o, is_g ? o : v, m0, n);
          }
        }
      } else {
        // a part of a tile: its sums go to the workspace as [m][128 lanes]
        const int rel = w.tile - pr.dp_tiles;
        float* ws = p.ws + ((long long)(pr.slot0 + rel * pr.split + w.part) * CG + rank) * (BM * 128) + l;
        for (int c = half; c < BM / CH; c += 2) {
          if (m_base + c * CH >= pr.M) break;
          float v[CH];
          tmem_load<CH>(t_acc + c * CH, v);
          ptx5::tmem_ld_wait<CH>(v);
#pragma unroll
          for (int j = 0; j < CH; ++j) __stcg(ws + (c * CH + j) * 128, v[j]);
        }
      }
      // the accumulator may be overwritten
      ptx5::fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        if (CG == 1) mbar_arrive(acc_empty + 8 * a);
        else ptx5::mbar_arrive_cluster(map_to_cta(acc_empty + 8 * a, 0));
      }
      if (w.part >= 0) {
        const int rel = w.tile - pr.dp_tiles;
        int* counter = p.counters + (pr.counter0 + rel) * CG + rank;
        __threadfence();
        named_barrier_sync(8, EPI_WARPS * 32);
        if (e == 0 && lane == 0) {
          const int old = atomicAdd(counter, 1);
          *last_flag = old == pr.split - 1;
          if (old == pr.split - 1) *counter = 0;  // ready for the next launch
        }
        named_barrier_sync(8, EPI_WARPS * 32);
        if (*last_flag) {
          __threadfence();
          const float* ws = p.ws + ((long long)(pr.slot0 + rel * pr.split) * CG + rank) * (BM * 128);
          const long long stride = (long long)CG * BM * 128;
          if (!GATED) {
            for (int c = half; c < BM / CH; c += 2) {
              if (m_base + c * CH >= pr.M) break;
              float v[CH];
#pragma unroll
              for (int j = 0; j < CH; ++j) v[j] = 0.f;
              for (int s = 0; s < pr.split; ++s)
#pragma unroll
                for (int j = 0; j < CH; ++j) v[j] += __ldcg(ws + s * stride + (c * CH + j) * 128 + l);
              if (n_in) emit_plain_any<T, CH>(pr, v, bias, m_base + c * CH, n);
            }
          } else {
            for (int c = 2 * half + (quad >> 1); c < BM / CH; c += 4) {
              if (m_base + c * CH >= pr.M) break;
              float g[CH], uu[CH];
#pragma unroll
              for (int j = 0; j < CH; ++j) g[j] = uu[j] = 0.f;
              for (int s = 0; s < pr.split; ++s)
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                  g[j] += __ldcg(ws + s * stride + (c * CH + j) * 128 + (l & 63));
                  uu[j] += __ldcg(ws + s * stride + (c * CH + j) * 128 + 64 + (l & 63));
                }
              if (n_in) emit_gated_any<T, CH>(pr, g, uu, m_base + c * CH, n);
            }
          }
        }
        named_barrier_sync(8, EPI_WARPS * 32);  // last_flag may be rewritten
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
