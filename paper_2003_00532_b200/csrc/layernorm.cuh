// Layer norm, forward and backward. Bound by memory: each kernel reads its rows once, holds them in
// registers through all sums, and writes once.
//
// A row belongs to one warp (short rows: no block barrier at all) or to one block; a thread holds ITEMS
// vectors of VEC values (VEC = 16 bytes where the rows are 16-byte aligned, else single values) at
// columns (item * threads + thread) * VEC. Blocks are persistent: a thread keeps its columns' gamma and beta in
// registers from row to row, and the next row's loads are in flight while a row is computed.
//
// Forward: mean and variance in one block barrier. Each warp takes the mean and the sum of squares about that
// mean of its own part of the row (both from registers); the parts are then combined as
// M2 = sum_w M2_w + n_w (mean_w - mean)^2, so no large sums are ever subtracted.
//
// Backward: while a block walks over its rows, each thread also keeps dgamma and dbeta of its own columns
// in registers. The blocks' sums go to a partial matrix [block][column] that a second kernel adds in
// order of the blocks: no atomics, same bits every time.
//
// Rows too long for the registers are streamed (later passes mostly from L2).
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hgemm_ptx.cuh"

namespace lnorm {

struct Params {
  long long rows;
  int cols;
  const void* X;
  const void* gamma;
  const void* beta;
  const void* dY;
  void* out;  // Y, or dX
  long long ldx, ldy, ldo;  // ldy: of dY
  float* mean;
  float* rstd;
  float* partial;  // backward: [2][blocks][ldp]: dgamma's, dbeta's
  long long ldp;   // cols rounded up to 4: every row can be written as vectors
  float eps;
  int want_params;
};

__device__ __forceinline__ float cvt(float x) { return x; }
__device__ __forceinline__ float cvt(__half x) { return __half2float(x); }
__device__ __forceinline__ float cvt(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T rnd(float x);
template <> __device__ __forceinline__ float rnd<float>(float x) { return x; }
template <> __device__ __forceinline__ __half rnd<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 rnd<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// VEC values as one access of VEC * sizeof(T) bytes (16, or one value).
template <int BYTES> struct Bits;
template <> struct Bits<16> { using type = uint4; };
template <> struct Bits<4> { using type = uint32_t; };
template <> struct Bits<2> { using type = uint16_t; };
template <typename T, int VEC>
struct Vec {
  typename Bits<sizeof(T) * VEC>::type bits;
  __device__ __forceinline__ T get(int i) const { return reinterpret_cast<const T*>(&bits)[i]; }
  __device__ __forceinline__ void set(int i, T x) { reinterpret_cast<T*>(&bits)[i] = x; }
};

// VEC values at column c; beyond `cols` they read as `fill`.
template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> load(const T* row, int c, int cols, float fill) {
  Vec<T, VEC> r;
  if (c + VEC <= cols) {
    r.bits = *reinterpret_cast<const decltype(r.bits)*>(row + c);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.set(i, c + i < cols ? row[c + i] : rnd<T>(fill));
  }
  return r;
}
template <typename T, int VEC>
__device__ __forceinline__ void store(T* row, int c, int cols, const Vec<T, VEC>& r) {
  if (c + VEC <= cols) {
    *reinterpret_cast<typename Bits<sizeof(T) * VEC>::type*>(row + c) = r.bits;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (c + i < cols) row[c + i] = r.get(i);
  }
}

// Two binary32 values per instruction.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long&>(r)) : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long&>(r)) : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)), "l"(reinterpret_cast<unsigned long long&>(c)));
  return r;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// A thread's VEC * ITEMS values as pairs, in order of their columns (an odd count is padded with 0): pair k is
// values 2 k and 2 k + 1, value f belongs to item f / VEC.
template <typename T, int VEC, int ITEMS>
struct Pairs {
  static constexpr int N = (VEC * ITEMS + 1) / 2;
  float2 v[N];
  __device__ __forceinline__ void unpack(const Vec<T, VEC> (&raw)[ITEMS]) {
    if constexpr (VEC == 8 && sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const uint32_t w[4] = {raw[i].bits.x, raw[i].bits.y, raw[i].bits.z, raw[i].bits.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * i + j] = unpack_pair(w[j], T());
      }
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        v[k].x = cvt(raw[2 * k / VEC].get(2 * k % VEC));
        v[k].y = 2 * k + 1 < VEC * ITEMS ? cvt(raw[(2 * k + 1 < VEC * ITEMS ? 2 * k + 1 : 0) / VEC].get((2 * k + 1) % VEC)) : 0.f;
      }
    }
  }
  // Item i rounded to T.
  __device__ __forceinline__ Vec<T, VEC> pack(int i) const {
    Vec<T, VEC> o;
    if constexpr (VEC == 8 && sizeof(T) == 2) {
      o.bits = make_uint4(pack_pair(v[4 * i], T()), pack_pair(v[4 * i + 1], T()), pack_pair(v[4 * i + 2], T()), pack_pair(v[4 * i + 3], T()));
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int f = i * VEC + j;
        o.set(j, rnd<T>(f % 2 ? v[f / 2].y : v[f / 2].x));
      }
    }
    return o;
  }
  static __device__ __forceinline__ float2 unpack_pair(uint32_t w, __nv_bfloat16) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ float2 unpack_pair(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
  static __device__ __forceinline__ uint32_t pack_pair(float2 x, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x.x, x.y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint32_t pack_pair(float2 x, __half) {
    const __half2 h = __floats2half2_rn(x.x, x.y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};

// A thread's part of a row: ITEMS vectors 32 vectors apart, so that a warp covers 32 ITEMS vectors and every offset
// from the thread's first one is a constant. `full`: all of them lie inside the row.
template <typename T, int VEC, int ITEMS>
__device__ __forceinline__ void load_row(Vec<T, VEC> (&raw)[ITEMS], const T* at, int c0, int cols, bool full) {
  if (full) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) raw[i].bits = *reinterpret_cast<const decltype(raw[i].bits)*>(at + i * 32 * VEC);
  } else {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) raw[i] = load<T, VEC>(at + i * 32 * VEC, 0, cols - c0 - i * 32 * VEC, 0.f);
  }
}
template <typename T, int VEC, int ITEMS>
__device__ __forceinline__ void store_row(T* at, const Pairs<T, VEC, ITEMS>& v, int c0, int cols, bool full) {
  if (full) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) *reinterpret_cast<decltype(v.pack(0).bits)*>(at + i * 32 * VEC) = v.pack(i).bits;
  } else {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) store<T, VEC>(at + i * 32 * VEC, 0, cols - c0 - i * 32 * VEC, v.pack(i));
  }
}
// Values per vector and plane of a parameter kept in shared memory as binary32: value j of vector v at
// [plane j / 4][v][j % 4], so that 16-byte accesses are free of conflicts.
template <int VEC>
__device__ __forceinline__ int plane_at(int c, int nv) {
  constexpr int LOW = VEC < 4 ? VEC : 4;
  return ((c % VEC / LOW) * nv + c / VEC) * LOW + c % VEC % LOW;
}

// 1 / sqrt(x): the approximation (2 units in the last place) and one Newton step. x = 0 gives infinity.
__device__ __forceinline__ float inv_sqrt(float x) {
  const float r = rsqrtf(x);
  return x > 0.f && r < __int_as_float(0x7f800000) && r > 0.f ? r * fmaf(-0.5f * x * r, r, 1.5f) : r;
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
// Two sums over the warp with six shuffles instead of ten: the halves of the warp each take one of them.
__device__ __forceinline__ float2 warp_sum_pair(float a, float b) {
  const bool low = (threadIdx.x & 16) == 0;
  float x = (low ? a : b) + __shfl_xor_sync(0xffffffffu, low ? b : a, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  const float y = __shfl_xor_sync(0xffffffffu, x, 16);
  return low ? make_float2(x, y) : make_float2(y, x);
}
// Sum over the block; `red` holds one value per warp and may be reused after the next barrier.
__device__ __forceinline__ float block_sum(float x, float* red) {
  x = warp_sum(x);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  const int warps = (blockDim.x + 31) >> 5, lane = threadIdx.x & 31;
  return warp_sum(lane < warps ? red[lane] : 0.f);
}

// ---- forward ----------------------------------------------------------------------------------------

// Most threads per row, by the values a thread holds.
constexpr int fwd_threads(int values) { return values <= 8 ? 1024 : 512; }

// WARP_ROW: four rows per block of 128 threads, one warp each; otherwise one row per block. gamma and beta wait in
// shared memory. What the shuffles, the barrier and the combination of the warps' parts cost per row is shared by 16
// values per thread; 8 leave them half of all instructions, with 32 too few warps fit on an SM.
template <typename T, int VEC, int ITEMS, bool WARP_ROW>
__global__ void __launch_bounds__(WARP_ROW ? 128 : fwd_threads(VEC* ITEMS)) fwd_kernel(const __grid_constant__ Params p) {
  constexpr int PLANES = (VEC + 3) / 4, LOW = VEC < 4 ? VEC : 4;
  extern __shared__ uint4 smem[];
  __shared__ float2 red[2][32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int v0 = (WARP_ROW ? 0 : warp * ITEMS * 32) + lane, c0 = v0 * VEC;  // first vector and column of this thread
  const bool full = c0 + (ITEMS - 1) * 32 * VEC + VEC <= p.cols;
  const long long step = WARP_ROW ? (long long)gridDim.x * 4 : (long long)gridDim.x;
  long long row = WARP_ROW ? (long long)blockIdx.x * 4 + warp : (long long)blockIdx.x;
  const T* x_at = static_cast<const T*>(p.X) + row * p.ldx + c0;
  T* y_at = static_cast<T*>(p.out) + row * p.ldo + c0;
  using P = Pairs<T, VEC, ITEMS>;
  constexpr int N = P::N;
  Vec<T, VEC> raw[ITEMS];
  const int nv = (int)(WARP_ROW ? 1 : blockDim.x >> 5) * ITEMS * 32;  // vectors of the whole block, inside the row or not
  float* sg = reinterpret_cast<float*>(smem);
  float* sb = sg + nv * VEC;
  {
    // every thread puts down what it will read itself (WARP_ROW: the four warps the same values)
    Vec<T, VEC> raw_b[ITEMS];
    if (p.gamma) load_row<T, VEC, ITEMS>(raw, static_cast<const T*>(p.gamma) + c0, c0, p.cols, full);
    if (p.beta) load_row<T, VEC, ITEMS>(raw_b, static_cast<const T*>(p.beta) + c0, c0, p.cols, full);
    P g, b;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      g.v[k] = both(1.f);
      b.v[k] = both(0.f);
    }
    if (p.gamma) g.unpack(raw);
    if (p.beta) b.unpack(raw_b);
    if (row < p.rows) load_row<T, VEC, ITEMS>(raw, x_at, c0, p.cols, full);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int v = v0 + i * 32;
      if constexpr (VEC > 1) {
#pragma unroll
        for (int h = 0; h < PLANES; ++h) {
          const int k = i * VEC / 2 + 2 * h;
          *reinterpret_cast<float4*>(sg + (h * nv + v) * LOW) = make_float4(g.v[k].x, g.v[k].y, g.v[k + 1].x, g.v[k + 1].y);
          *reinterpret_cast<float4*>(sb + (h * nv + v) * LOW) = make_float4(b.v[k].x, b.v[k].y, b.v[k + 1].x, b.v[k + 1].y);
        }
      } else {
        sg[v] = i % 2 ? g.v[i / 2].y : g.v[i / 2].x;
        sb[v] = i % 2 ? b.v[i / 2].y : b.v[i / 2].x;
      }
    }
  }
  const bool plain = full && VEC * ITEMS % 2 == 0;
  const float inv_n = 1.f / (float)p.cols;
  // columns of this warp, and of warp number `lane`
  const auto columns = [&](int w) { return (float)max(0, min(32 * ITEMS * VEC, p.cols - w * 32 * ITEMS * VEC)); };
  const float n_warp = WARP_ROW ? (float)p.cols : columns(warp), inv_warp = n_warp > 0.f ? 1.f / n_warp : 0.f;
  const float n_lane = !WARP_ROW && lane < (int)(blockDim.x >> 5) ? columns(lane) : 0.f;
  int parity = 0;
  for (; row < p.rows; parity ^= 1) {
    P x;
    x.unpack(raw);
    const long long at = row;
    row += step;
    x_at += step * p.ldx;
    if (row < p.rows) load_row<T, VEC, ITEMS>(raw, x_at, c0, p.cols, full);
    float2 s = both(0.f);
#pragma unroll
    for (int k = 0; k < N; ++k) s = add2(s, x.v[k]);
    float mean = warp_sum(s.x + s.y) * inv_warp;
    s = both(0.f);
    const float2 minus = both(-mean);
    if (plain) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        x.v[k] = add2(x.v[k], minus);
        s = fma2(x.v[k], x.v[k], s);
      }
    } else {
#pragma unroll
      for (int f = 0; f < VEC * ITEMS; ++f) {
        float& d = f % 2 ? x.v[f / 2].y : x.v[f / 2].x;
        d -= mean;
        if (c0 + f / VEC * 32 * VEC + f % VEC < p.cols) s.x += d * d;
      }
    }
    float m2 = warp_sum(s.x + s.y);
    float shift = 0.f;  // row mean minus the mean that x is centred by
    if (!WARP_ROW) {
      if (lane == 0) red[parity][warp] = make_float2(mean, m2);
      __syncthreads();  // one per row: a warp can be one row ahead, and writes the other half of `red` then
      const float2 part = lane < (int)(blockDim.x >> 5) ? red[parity][lane] : make_float2(0.f, 0.f);
      const float warp_mean = mean;
      mean = warp_sum(part.x * n_lane) * inv_n;
      const float off = part.x - mean;
      m2 = warp_sum(part.y + n_lane * off * off);
      shift = mean - warp_mean;
    }
    const float rstd = inv_sqrt(m2 * inv_n + p.eps);
    if (lane == 0 && (WARP_ROW || warp == 0)) {
      if (p.mean) p.mean[at] = mean;
      if (p.rstd) p.rstd[at] = rstd;
    }
    // x was centred before it is scaled: a mean far above the deviation costs no accuracy
    const float bias = -shift * rstd;
#pragma unroll
    for (int k = 0; k < N; ++k) x.v[k] = fma2(x.v[k], both(rstd), both(bias));
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int v = v0 + i * 32;
      if constexpr (VEC > 1) {
#pragma unroll
        for (int h = 0; h < PLANES; ++h) {
          const float4 g = *reinterpret_cast<const float4*>(sg + (h * nv + v) * LOW), b = *reinterpret_cast<const float4*>(sb + (h * nv + v) * LOW);
          const int k = i * VEC / 2 + 2 * h;
          x.v[k] = fma2(x.v[k], make_float2(g.x, g.y), make_float2(b.x, b.y));
          x.v[k + 1] = fma2(x.v[k + 1], make_float2(g.z, g.w), make_float2(b.z, b.w));
        }
      } else {
        float& d = i % 2 ? x.v[i / 2].y : x.v[i / 2].x;
        d = d * sg[v] + sb[v];
      }
    }
    store_row<T, VEC, ITEMS>(y_at, x, c0, p.cols, full);
    y_at += step * p.ldo;
  }
}

// Rows of any length: one block per row, three passes.
template <typename T>
__global__ void __launch_bounds__(1024) fwd_long_kernel(const __grid_constant__ Params p) {
  __shared__ float red[2][32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const T* x = static_cast<const T*>(p.X) + (long long)blockIdx.x * p.ldx;
  T* y = static_cast<T*>(p.out) + (long long)blockIdx.x * p.ldo;
  float s = 0.f;
  for (int c = threadIdx.x; c < p.cols; c += blockDim.x) s += cvt(x[c]);
  const float mean = block_sum(s, red[0]) / (float)p.cols;
  s = 0.f;
  for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
    const float d = cvt(x[c]) - mean;
    s += d * d;
  }
  const float rstd = inv_sqrt(block_sum(s, red[1]) / (float)p.cols + p.eps);
  if (threadIdx.x == 0) {
    if (p.mean) p.mean[blockIdx.x] = mean;
    if (p.rstd) p.rstd[blockIdx.x] = rstd;
  }
  const T* gamma = static_cast<const T*>(p.gamma);
  const T* beta = static_cast<const T*>(p.beta);
  for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
    float a = (cvt(x[c]) - mean) * rstd;
    if (gamma) a *= cvt(gamma[c]);
    if (beta) a += cvt(beta[c]);
    y[c] = rnd<T>(a);
  }
}

// ---- backward ---------------------------------------------------------------------------------------

// Most threads per row: 512 with 16 values each in 128 registers.
constexpr int BWD_THREADS = 512;

// WARP_ROW: eight rows per block, one warp each; otherwise one row per block. WIDE: 32 values per thread, gamma and the
// sums for dgamma and dbeta in shared memory (each thread's own entries) instead of registers.
template <typename T, int VEC, int ITEMS, bool WARP_ROW, bool WIDE>
__global__ void __launch_bounds__(WARP_ROW ? 256 : BWD_THREADS) bwd_kernel(const __grid_constant__ Params p) {
  constexpr int LOW = VEC < 4 ? VEC : 4;
  extern __shared__ uint4 smem[];  // WARP_ROW with parameter gradients: [cols] twice; WIDE: gamma, dgamma, dbeta
  __shared__ float2 red[2][32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int v0 = (WARP_ROW ? 0 : warp * ITEMS * 32) + lane, c0 = v0 * VEC;  // first vector and column of this thread
  const bool full = c0 + (ITEMS - 1) * 32 * VEC + VEC <= p.cols;
  const long long step = WARP_ROW ? (long long)gridDim.x * 8 : (long long)gridDim.x;
  long long row = WARP_ROW ? (long long)blockIdx.x * 8 + warp : (long long)blockIdx.x;
  const T* x_at = static_cast<const T*>(p.X) + row * p.ldx + c0;
  const T* d_at = static_cast<const T*>(p.dY) + row * p.ldy + c0;
  T* o_at = static_cast<T*>(p.out) + row * p.ldo + c0;
  const T* gamma = static_cast<const T*>(p.gamma);
  const float inv_n = 1.f / (float)p.cols;
  using P = Pairs<T, VEC, ITEMS>;
  constexpr int N = P::N;
  const int nv = (int)(blockDim.x >> 5) * ITEMS * 32;  // WIDE: vectors of the whole block, inside the row or not
  float* sums = reinterpret_cast<float*>(smem);
  float* w_g = sums;
  float* w_dg = sums + nv * VEC;
  float* w_db = sums + 2 * nv * VEC;
  Vec<T, VEC> xr[ITEMS], dr[ITEMS];
  P g, dg, db;
  if (WIDE) {
    for (int c = threadIdx.x; c < nv * VEC; c += blockDim.x) {
      const int at = plane_at<VEC>(c, nv);
      w_g[at] = gamma && c < p.cols ? cvt(gamma[c]) : 1.f;
      w_dg[at] = w_db[at] = 0.f;
    }
    __syncthreads();
  }
  // gamma's loads and the first row's are in flight together
  Vec<T, VEC> gr[ITEMS];
  if (!WIDE && gamma) load_row<T, VEC, ITEMS>(gr, gamma + c0, c0, p.cols, full);
  float mean = 0.f, rstd = 0.f;
  if (row < p.rows) {
    load_row<T, VEC, ITEMS>(xr, x_at, c0, p.cols, full);
    load_row<T, VEC, ITEMS>(dr, d_at, c0, p.cols, full);
    mean = p.mean[row];
    rstd = p.rstd[row];
  }
  if (!WIDE) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      g.v[k] = both(1.f);
      dg.v[k] = db.v[k] = both(0.f);
    }
    if (gamma) g.unpack(gr);
  }
  int parity = 0;
  for (; row < p.rows; parity ^= 1) {
    // xh and w = dy gamma of this row. Beyond `cols` dy is 0, and so is every term of the sums: t2 adds w (x - mean) and is
    // scaled at the end, because (0 - mean) rstd may be infinite there
    P xh, w;
    xh.unpack(xr);
    w.unpack(dr);
    const float rs = rstd, mu = mean;
    row += step;
    x_at += step * p.ldx;
    d_at += step * p.ldy;
    if (row < p.rows) {
      load_row<T, VEC, ITEMS>(xr, x_at, c0, p.cols, full);
      load_row<T, VEC, ITEMS>(dr, d_at, c0, p.cols, full);
      mean = p.mean[row];
      rstd = p.rstd[row];
    }
    float2 t1 = both(0.f), t2 = both(0.f);
    if (!WIDE) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float2 d = add2(xh.v[k], both(-mu));
        xh.v[k] = mul2(d, both(rs));
        dg.v[k] = fma2(w.v[k], xh.v[k], dg.v[k]);
        db.v[k] = add2(db.v[k], w.v[k]);
        w.v[k] = mul2(w.v[k], g.v[k]);
        t1 = add2(t1, w.v[k]);
        t2 = fma2(w.v[k], d, t2);
      }
    } else {
      // LOW values at a time; with VEC == 1 the pairs span two vectors, so single values are used
#pragma unroll
      for (int q = 0; q < VEC * ITEMS / LOW; ++q) {
        const int at = ((q % (VEC / LOW)) * nv + v0 + q / (VEC / LOW) * 32) * LOW;
        if constexpr (LOW == 4) {
          float4 a = *reinterpret_cast<float4*>(w_dg + at), b = *reinterpret_cast<float4*>(w_db + at);
          const float4 gg = *reinterpret_cast<const float4*>(w_g + at);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int k = 2 * q + h;
            float2& da = reinterpret_cast<float2*>(&a)[h];
            float2& dbb = reinterpret_cast<float2*>(&b)[h];
            const float2 d = add2(xh.v[k], both(-mu));
            xh.v[k] = mul2(d, both(rs));
            da = fma2(w.v[k], xh.v[k], da);
            dbb = add2(dbb, w.v[k]);
            w.v[k] = mul2(w.v[k], reinterpret_cast<const float2*>(&gg)[h]);
            t1 = add2(t1, w.v[k]);
            t2 = fma2(w.v[k], d, t2);
          }
          *reinterpret_cast<float4*>(w_dg + at) = a;
          *reinterpret_cast<float4*>(w_db + at) = b;
        } else {
          float& h = q % 2 ? xh.v[q / 2].y : xh.v[q / 2].x;
          float& d = q % 2 ? w.v[q / 2].y : w.v[q / 2].x;
          const float off = h - mu;
          h = off * rs;
          w_dg[at] += d * h;
          w_db[at] += d;
          d *= w_g[at];
          t1.x += d;
          t2.x += d * off;
        }
      }
    }
    if (p.out) {
      float2 both_sums = warp_sum_pair(t1.x + t1.y, t2.x + t2.y);
      if (!WARP_ROW) {
        if (lane == 0) red[parity][warp] = both_sums;
        __syncthreads();  // one barrier per row: the other parity's values are read before the next one
        both_sums = lane < (int)(blockDim.x >> 5) ? red[parity][lane] : both(0.f);
        both_sums = warp_sum_pair(both_sums.x, both_sums.y);
      }
      const float s1 = both_sums.x * inv_n, s2 = both_sums.y * rs * inv_n;
#pragma unroll
      for (int k = 0; k < N; ++k) w.v[k] = mul2(add2(fma2(xh.v[k], both(-s2), w.v[k]), both(-s1)), both(rs));
      store_row<T, VEC, ITEMS>(o_at, w, c0, p.cols, full);
      o_at += step * p.ldo;
    }
  }
  if (!p.want_params) return;
  float* out = p.partial + blockIdx.x * p.ldp;
  const long long half = gridDim.x * p.ldp;
  const auto value = [](const P& x, int f) { return f % 2 ? x.v[f / 2].y : x.v[f / 2].x; };
  if (WIDE) {
    __syncthreads();
    for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
      out[c] = w_dg[plane_at<VEC>(c, nv)];
      out[half + c] = w_db[plane_at<VEC>(c, nv)];
    }
  } else if (!WARP_ROW && VEC >= 4) {
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      const int c = c0 + 2 * k / VEC * 32 * VEC + 2 * k % VEC;
      const int l = k + 1 < N ? k + 1 : k;
      if (c >= p.cols) continue;
      *reinterpret_cast<float4*>(out + c) = make_float4(dg.v[k].x, dg.v[k].y, dg.v[l].x, dg.v[l].y);
      *reinterpret_cast<float4*>(out + half + c) = make_float4(db.v[k].x, db.v[k].y, db.v[l].x, db.v[l].y);
    }
  } else if (!WARP_ROW) {
#pragma unroll
    for (int f = 0; f < VEC * ITEMS; ++f) {
      const int c = c0 + f / VEC * 32 * VEC + f % VEC;
      if (c < p.cols) {
        out[c] = value(dg, f);
        out[half + c] = value(db, f);
      }
    }
  } else {
    // the eight warps add their sums one after the other, in order
    for (int k = 0; k < 8; ++k) {
      if (warp == k) {
#pragma unroll
        for (int f = 0; f < VEC * ITEMS; ++f) {
          const int c = c0 + f / VEC * 32 * VEC + f % VEC;
          if (c < p.cols) {
            const float a = value(dg, f), b = value(db, f);
            sums[c] = k ? sums[c] + a : a;
            sums[p.cols + c] = k ? sums[p.cols + c] + b : b;
          }
        }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
      out[c] = sums[c];
      out[half + c] = sums[p.cols + c];
    }
  }
}

// Rows of any length, dx: one block per row, two passes.
template <typename T>
__global__ void __launch_bounds__(1024) bwd_long_kernel(const __grid_constant__ Params p) {
  __shared__ float red[2][32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const long long row = blockIdx.x;
  const T* x = static_cast<const T*>(p.X) + row * p.ldx;
  const T* dy = static_cast<const T*>(p.dY) + row * p.ldy;
  const T* gamma = static_cast<const T*>(p.gamma);
  const float mean = p.mean[row], rstd = p.rstd[row];
  float s1 = 0.f, s2 = 0.f;
  for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
    const float w = cvt(dy[c]) * (gamma ? cvt(gamma[c]) : 1.f);
    s1 += w;
    s2 += w * ((cvt(x[c]) - mean) * rstd);
  }
  s1 = block_sum(s1, red[0]) / (float)p.cols;
  s2 = block_sum(s2, red[1]) / (float)p.cols;
  T* dx = static_cast<T*>(p.out) + row * p.ldo;
  for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
    const float w = cvt(dy[c]) * (gamma ? cvt(gamma[c]) : 1.f);
    dx[c] = rnd<T>(rstd * (w - s1 - (cvt(x[c]) - mean) * rstd * s2));
  }
}
// Rows of any length, parameter gradients: a thread per column, gridDim.y chunks of rows.
template <typename T>
__global__ void __launch_bounds__(256) bwd_long_params_kernel(const __grid_constant__ Params p) {
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= p.cols) return;
  const long long per = (p.rows + gridDim.y - 1) / gridDim.y;
  const long long r0 = blockIdx.y * per, r1 = r0 + per < p.rows ? r0 + per : p.rows;
  float dg = 0.f, db = 0.f;
  for (long long r = r0; r < r1; ++r) {
    const float dy = cvt(static_cast<const T*>(p.dY)[r * p.ldy + c]);
    dg += dy * ((cvt(static_cast<const T*>(p.X)[r * p.ldx + c]) - p.mean[r]) * p.rstd[r]);
    db += dy;
  }
  p.partial[blockIdx.y * p.ldp + c] = dg;
  p.partial[(gridDim.y + blockIdx.y) * p.ldp + c] = db;
}

// Adds the blocks' sums in an order that depends on the sizes alone: blockIdx.y 0 = dgamma, 1 = dbeta. 32 columns per
// block; its warps take a part of the rows each, eight loads in flight. With 16 warps the last rows of a part are read one
// after the other; with 32, which are for many rows (MANY_BLOCKS), eight at a time without a condition between them (those
// that are not the part's are read again and dropped), and the parts are added by shuffles. With all outputs: 592 rows of
// sums (4097 x 1537 binary32) 25.3 us with 16 warps, 22.8 with 32; 296 (8192 x 4096) 43.2 and 42.5; but 61 (1224 x 248)
// 9.3 and 10.4, one 3.7 and 4.1.
constexpr int MANY_BLOCKS = 256;
template <int WARPS>
__global__ void __launch_bounds__(32 * WARPS) bwd_reduce_kernel(const float* partial, int blocks, int cols, int ldp, float* dgamma, float* dbeta) {
  __shared__ float red[WARPS][33];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  float* out = blockIdx.y ? dbeta : dgamma;
  if (!out) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  const float* src = partial + (long long)blockIdx.y * blocks * ldp + min(c, cols - 1);
  const int per = (blocks + WARPS - 1) / WARPS;
  const int b1 = min(blocks, (warp + 1) * per);
  float s = 0.f;
  int b = warp * per;
  if (WARPS == 32) {
    for (; b < b1; b += 8) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __ldcg(src + (long long)min(b + j, b1 - 1) * ldp);
#pragma unroll
      for (int j = 0; j < 8; ++j) s += b + j < b1 ? v[j] : 0.f;
    }
  } else {
    for (; b + 8 <= b1; b += 8) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __ldcg(src + (long long)(b + j) * ldp);
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[j];
    }
    for (; b < b1; ++b) s += __ldcg(src + (long long)b * ldp);
  }
  red[warp][lane] = s;
  __syncthreads();
  if (WARPS == 32) {
    s = red[lane][warp];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0 && blockIdx.x * 32 + warp < cols) out[blockIdx.x * 32 + warp] = s;
  } else if (warp == 0 && c < cols) {
    s = red[0][lane];
    for (int w = 1; w < WARPS; ++w) s += red[w][lane];
    out[c] = s;
  }
}

}  // namespace lnorm
