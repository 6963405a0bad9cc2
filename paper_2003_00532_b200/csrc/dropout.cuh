// Dropout with the residual's addition, and its backward pass (the same kernel without a residual): one pass over
// the matrices, the mask from a counter-based generator.
//
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC 2011) turns a counter of four words and a key of two into four random words
// by ten rounds of two 32 x 32 -> 64 bit products. The counter is (column / 4, row, offset), so that any thread makes the words of any
// four columns by itself.
//
// A thread takes vectors of VEC columns (16 bytes where all rows are 16-byte aligned, else the four columns of one counter,
// value by value), UNROLL at a time so that their loads are in flight together and the rounds of several counters overlap.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hgemm_ptx.cuh"
#include "layernorm.cuh"

namespace drop {

struct Params {
  long long rows;
  int cols;
  int nv;             // vectors per row
  int none;           // p = 1: nothing is kept
  uint32_t threshold; // p 2^32
  float scale;        // 1 / (1 - p)
  uint32_t key0, key1;
  unsigned long long offset;
  const long long* step;
  const void* X;
  const void* R;
  void* Y;
  long long ldx, ldr, ldy;
};

__device__ __forceinline__ uint4 philox4x32_10(uint4 c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const unsigned long long a = (unsigned long long)c.x * 0xD2511F53u, b = (unsigned long long)c.z * 0xCD9E8D57u;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k1, (uint32_t)a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

template <typename T, int VEC, bool ALIGNED>
struct Access {
  using V = lnorm::Vec<T, ALIGNED ? VEC : 1>;
  V v[ALIGNED ? 1 : VEC];
  __device__ __forceinline__ float get(int j) const { return lnorm::cvt(ALIGNED ? v[0].get(j) : v[ALIGNED ? 0 : j].get(0)); }
  __device__ __forceinline__ void set(int j, float x) {
    if (ALIGNED) v[0].set(j, lnorm::rnd<T>(x));
    else v[ALIGNED ? 0 : j].set(0, lnorm::rnd<T>(x));
  }
  __device__ __forceinline__ void read(const T* row, int c, int cols) {
    if (ALIGNED) {
      v[0] = lnorm::load<T, ALIGNED ? VEC : 1>(row, c, cols, 0.f);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[ALIGNED ? 0 : j] = lnorm::load<T, ALIGNED ? VEC : 1>(row, c + j, cols, 0.f);
    }
  }
  __device__ __forceinline__ void write(T* row, int c, int cols) const {
    if (ALIGNED) {
      lnorm::store<T, ALIGNED ? VEC : 1>(row, c, cols, v[0]);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) lnorm::store<T, ALIGNED ? VEC : 1>(row, c + j, cols, v[ALIGNED ? 0 : j]);
    }
  }
};

constexpr int THREADS = 256;

template <typename T, int VEC, bool ALIGNED, int UNROLL>
__global__ void __launch_bounds__(THREADS) dropout_kernel(const __grid_constant__ Params p) {
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const unsigned long long offset = p.offset + (p.step ? (unsigned long long)*p.step : 0ull);
  const uint32_t o0 = (uint32_t)offset, o1 = (uint32_t)(offset >> 32);
  // this thread's place, and how far a sweep of the grid moves it: rows and vectors of a row
  const long long first = (long long)blockIdx.x * THREADS + threadIdx.x, sweep = (long long)gridDim.x * THREADS;
  long long row = first / p.nv;
  int v = (int)(first - row * p.nv);
  const long long rows_on = sweep / p.nv;
  const int v_on = (int)(sweep - rows_on * p.nv);
  while (row < p.rows) {
    Access<T, VEC, ALIGNED> x[UNROLL], r[UNROLL];
    long long at[UNROLL];
    int c[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      at[u] = row;
      c[u] = v * VEC;
      if (row < p.rows) {
        x[u].read(static_cast<const T*>(p.X) + row * p.ldx, c[u], p.cols);
        if (p.R) r[u].read(static_cast<const T*>(p.R) + row * p.ldr, c[u], p.cols);
      }
      row += rows_on;
      v += v_on;
      if (v >= p.nv) {
        v -= p.nv;
        ++row;
      }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (at[u] >= p.rows) break;
      Access<T, VEC, ALIGNED> y;
#pragma unroll
      for (int q = 0; q < VEC; q += 4) {
        const uint4 w = philox4x32_10(make_uint4((uint32_t)(c[u] + q) >> 2, (uint32_t)at[u], o0, o1), p.key0, p.key1);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float kept = word[j] >= p.threshold && !p.none ? x[u].get(q + j) * p.scale : 0.f;
          y.set(q + j, p.R ? kept + r[u].get(q + j) : kept);
        }
      }
      y.write(static_cast<T*>(p.Y) + at[u] * p.ldy, c[u], p.cols);
    }
  }
}

}  // namespace drop
