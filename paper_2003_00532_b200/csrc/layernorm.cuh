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
  float* partial;  // backward: [2][blocks][cols]: dgamma's, dbeta's
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

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
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

// Most threads per row, by the values a thread holds: 1024 x 64 registers, 512 x 128.
constexpr int fwd_threads(int values) { return values <= 8 ? 1024 : 512; }

template <typename T, int VEC, int ITEMS, bool WARP_ROW>
__global__ void __launch_bounds__(WARP_ROW ? 256 : fwd_threads(VEC* ITEMS)) fwd_kernel(const __grid_constant__ Params p) {
  __shared__ float2 red[2][32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int threads = WARP_ROW ? 32 : blockDim.x;
  const int t = WARP_ROW ? threadIdx.x & 31 : threadIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long first = WARP_ROW ? (long long)blockIdx.x * 8 + warp : (long long)blockIdx.x;
  const long long step = WARP_ROW ? (long long)gridDim.x * 8 : (long long)gridDim.x;
  if (first >= p.rows) return;
  const T* X = static_cast<const T*>(p.X);
  const T* gamma = static_cast<const T*>(p.gamma);
  const T* beta = static_cast<const T*>(p.beta);
  Vec<T, VEC> g[ITEMS], b[ITEMS], raw[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) raw[i] = load<T, VEC>(X + first * p.ldx, (i * threads + t) * VEC, p.cols, 0.f);
  int mine = 0;  // columns of this thread
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int c = (i * threads + t) * VEC;
    mine += max(0, min(VEC, p.cols - c));
    if (gamma) g[i] = load<T, VEC>(gamma, c, p.cols, 1.f);
    if (beta) b[i] = load<T, VEC>(beta, c, p.cols, 0.f);
  }
  const float inv_n = 1.f / (float)p.cols;
  // columns of this warp, and of warp number `lane` (exact in binary32: at most 2^15)
  const float n_warp = WARP_ROW ? (float)p.cols : warp_sum((float)mine);
  const float inv_warp = n_warp > 0.f ? 1.f / n_warp : 0.f;
  float n_lane = 0.f;
  if (!WARP_ROW) {
    if (lane == 0) red[1][warp].x = n_warp;
    __syncthreads();
    if (lane < (int)(blockDim.x >> 5)) n_lane = red[1][lane].x;
    __syncthreads();
  }
  int parity = 0;
  for (long long row = first; row < p.rows; row += step, parity ^= 1) {
    float v[ITEMS][VEC], s = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        v[i][j] = cvt(raw[i].get(j));
        s += v[i][j];
      }
    if (row + step < p.rows) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) raw[i] = load<T, VEC>(X + (row + step) * p.ldx, (i * threads + t) * VEC, p.cols, 0.f);
    }
    float mean = warp_sum(s) * inv_warp;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float d = v[i][j] - mean;
        if ((i * threads + t) * VEC + j < p.cols) s += d * d;
      }
    float m2 = warp_sum(s);
    if (!WARP_ROW) {
      if (lane == 0) red[parity][warp] = make_float2(mean, m2);
      __syncthreads();  // one per row: a warp can be one row ahead, and writes the other half of `red` then
      const float2 part = lane < (int)(blockDim.x >> 5) ? red[parity][lane] : make_float2(0.f, 0.f);
      mean = warp_sum(part.x * n_lane) * inv_n;
      const float d = part.x - mean;
      m2 = warp_sum(part.y + n_lane * d * d);
    }
    const float rstd = 1.f / sqrtf(m2 * inv_n + p.eps);
    if (t == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
    T* y = static_cast<T*>(p.out) + row * p.ldo;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = (i * threads + t) * VEC;
      if (c >= p.cols) continue;
      Vec<T, VEC> o;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        float a = (v[i][j] - mean) * rstd;
        if (gamma) a *= cvt(g[i].get(j));
        if (beta) a += cvt(b[i].get(j));
        o.set(j, rnd<T>(a));
      }
      store<T, VEC>(y, c, p.cols, o);
    }
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
  const float rstd = 1.f / sqrtf(block_sum(s, red[1]) / (float)p.cols + p.eps);
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

constexpr int BWD_THREADS = 512;  // most threads per row: 128 registers each hold 16 columns and their sums

template <typename T, int VEC, int ITEMS, bool WARP_ROW>
__global__ void __launch_bounds__(WARP_ROW ? 256 : BWD_THREADS) bwd_kernel(const __grid_constant__ Params p) {
  extern __shared__ float sums[];  // WARP_ROW with parameter gradients: [cols] twice
  __shared__ float red[2][2][32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int threads = WARP_ROW ? 32 : blockDim.x;
  const int t = WARP_ROW ? threadIdx.x & 31 : threadIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long first = WARP_ROW ? (long long)blockIdx.x * 8 + warp : (long long)blockIdx.x;
  const long long step = WARP_ROW ? (long long)gridDim.x * 8 : (long long)gridDim.x;
  const T* X = static_cast<const T*>(p.X);
  const T* dY = static_cast<const T*>(p.dY);
  const T* gamma = static_cast<const T*>(p.gamma);
  const float inv_n = 1.f / (float)p.cols;
  Vec<T, VEC> g[ITEMS], xr[ITEMS], dr[ITEMS];
  float dg[ITEMS][VEC], db[ITEMS][VEC];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int c = (i * threads + t) * VEC;
    if (gamma) {
      g[i] = load<T, VEC>(gamma, c, p.cols, 0.f);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) g[i].set(j, rnd<T>(1.f));
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) dg[i][j] = db[i][j] = 0.f;
  }
  float mean = 0.f, rstd = 0.f;
  if (first < p.rows) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = (i * threads + t) * VEC;
      xr[i] = load<T, VEC>(X + first * p.ldx, c, p.cols, 0.f);
      dr[i] = load<T, VEC>(dY + first * p.ldy, c, p.cols, 0.f);
    }
    mean = p.mean[first];
    rstd = p.rstd[first];
  }
  int parity = 0;
  for (long long row = first; row < p.rows; row += step, parity ^= 1) {
    // xh and w = dy gamma of this row; beyond `cols` dy is 0 and so is every sum's term
    float xh[ITEMS][VEC], w[ITEMS][VEC], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float dy = cvt(dr[i].get(j));
        xh[i][j] = (cvt(xr[i].get(j)) - mean) * rstd;
        // a column beyond the row takes no part, whatever mean and rstd are
        if ((i * threads + t) * VEC + j >= p.cols) xh[i][j] = 0.f;
        w[i][j] = dy * cvt(g[i].get(j));
        dg[i][j] += dy * xh[i][j];
        db[i][j] += dy;
        s1 += w[i][j];
        s2 += w[i][j] * xh[i][j];
      }
    const float rs = rstd;
    const long long next = row + step;
    if (next < p.rows) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * threads + t) * VEC;
        xr[i] = load<T, VEC>(X + next * p.ldx, c, p.cols, 0.f);
        dr[i] = load<T, VEC>(dY + next * p.ldy, c, p.cols, 0.f);
      }
      mean = p.mean[next];
      rstd = p.rstd[next];
    }
    if (!p.out) continue;
    s1 = warp_sum(s1);
    s2 = warp_sum(s2);
    if (!WARP_ROW) {
      if (lane == 0) {
        red[parity][0][warp] = s1;
        red[parity][1][warp] = s2;
      }
      __syncthreads();  // one barrier per row: the other parity's values are read before the next one
      const int warps = (blockDim.x + 31) >> 5;
      s1 = warp_sum(lane < warps ? red[parity][0][lane] : 0.f);
      s2 = warp_sum(lane < warps ? red[parity][1][lane] : 0.f);
    }
    s1 *= inv_n;
    s2 *= inv_n;
    T* dx = static_cast<T*>(p.out) + row * p.ldo;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = (i * threads + t) * VEC;
      if (c >= p.cols) continue;
      Vec<T, VEC> o;
#pragma unroll
      for (int j = 0; j < VEC; ++j) o.set(j, rnd<T>(rs * (w[i][j] - s1 - xh[i][j] * s2)));
      store<T, VEC>(dx, c, p.cols, o);
    }
  }
  if (!p.want_params) return;
  if (!WARP_ROW) {
    float* out = p.partial + (long long)blockIdx.x * p.cols;
    const long long half = (long long)gridDim.x * p.cols;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int c = (i * threads + t) * VEC + j;
        if (c < p.cols) {
          out[c] = dg[i][j];
          out[half + c] = db[i][j];
        }
      }
  } else {
    // the eight warps add their sums one after the other, in order
    for (int k = 0; k < 8; ++k) {
      if (warp == k) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const int c = (i * 32 + t) * VEC + j;
            if (c < p.cols) {
              sums[c] = k ? sums[c] + dg[i][j] : dg[i][j];
              sums[p.cols + c] = k ? sums[p.cols + c] + db[i][j] : db[i][j];
            }
          }
      }
      __syncthreads();
    }
    float* out = p.partial + (long long)blockIdx.x * p.cols;
    const long long half = (long long)gridDim.x * p.cols;
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
  p.partial[(long long)blockIdx.y * p.cols + c] = dg;
  p.partial[((long long)gridDim.y + blockIdx.y) * p.cols + c] = db;
}

// Adds the blocks' sums in order: blockIdx.y 0 = dgamma, 1 = dbeta. 32 columns per block; eight warps
// take an eighth of the blocks each.
__global__ void __launch_bounds__(256) bwd_reduce_kernel(const float* partial, int blocks, int cols, float* dgamma, float* dbeta) {
  __shared__ float red[8][32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  float* out = blockIdx.y ? dbeta : dgamma;
  if (!out) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  const float* src = partial + (long long)blockIdx.y * blocks * cols;
  const int per = (blocks + 7) / 8;
  float s = 0.f;
  if (c < cols)
    for (int b = warp * per; b < min(blocks, (warp + 1) * per); ++b) s += __ldcg(src + (long long)b * cols + c);
  red[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < cols) {
    s = red[0][lane];
    for (int w = 1; w < 8; ++w) s += red[w][lane];
    out[c] = s;
  }
}

}  // namespace lnorm
