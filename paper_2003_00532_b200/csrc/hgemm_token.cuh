// Products of one or two rows (new tokens) with weights stored N x K: bound by reading the weights once. Plain binary32
// fused multiply-adds from registers; no tensor cores, no TMEM set-up, no workspace.
//
// A warp takes two weight rows (gated: the gate and the up row of one column), a lane 8 consecutive k (16 bytes) of
// each, in turns of up to eight steps without a condition between their loads. A turn of eight would need 64 registers for its
// loads alone; the kernels are compiled to 54 (one row; gated 48, with 12 bytes of spills) and 64 (two rows, 8 bytes), so its loads
// leave in two or more portions, each a trip to memory. WK warps of a block share the rows' k where there are too few rows for
// all SMs. The tokens wait in shared memory. Sums are binary32: per lane in ascending k, then over the lanes by
// shuffles, then over the warps in order: the same bits every time.
//
// Measured against the tensor-core kernel (4096 x 4096 bf16, bias and residual, calls back to back, weights rotating through
// more than L2): 10.0 to 10.3 us for one row, 11.0 for two, against 12; four rows 23 us (bound by the arithmetic), and a kernel of
// this kind for weights stored K x N 13.4 us against 12.6, so that those and rows that are not 16-byte aligned go to the
// tensor-core kernel.
#pragma once

#include <cstdint>

#include "hgemm_act.cuh"
#include "hgemm_tc.cuh"

namespace hgemm {

constexpr int TOKEN_ROWS = 2;  // most rows

struct TokenParams {
  int M, N, K;
  const void* X;         // M x K, or K x M if x_trans
  const void* W[2];      // weights; gated: gate, up
  long long ldx, ldw[2];
  int x_trans, x_vec;    // x_vec: rows of X may be read as 16-byte vectors
  int act;
  int wk;                // warps that share a row
  const void* bias;
  const void* R;
  void* D;
  void* Z;
  void* U;
  long long ldr, ldd, ldz, ldu;
};

__device__ __forceinline__ float act_any(int act, float z) {
  switch (act) {
    case HGEMM_ACT_RELU: return act_fwd<HGEMM_ACT_RELU>(z);
    case HGEMM_ACT_GELU: return act_fwd<HGEMM_ACT_GELU>(z);
    case HGEMM_ACT_GELU_TANH: return act_fwd<HGEMM_ACT_GELU_TANH>(z);
    case HGEMM_ACT_SILU: return act_fwd<HGEMM_ACT_SILU>(z);
    default: return z;
  }
}

// The epilogue of one value (gated: of the pair g, u).
template <typename T, bool GATED>
__device__ __forceinline__ void token_emit(const TokenParams& p, int m, int n, float a, float u) {
  if (GATED) {
    if (p.Z) {
      static_cast<T*>(p.Z)[m * p.ldz + n] = from_f32<T>(a);
      static_cast<T*>(p.U)[m * p.ldu + n] = from_f32<T>(u);
    }
    static_cast<T*>(p.D)[m * p.ldd + n] = from_f32<T>(act_any(p.act, a) * u);
  } else {
    const float z = a + (p.bias ? to_f32(static_cast<const T*>(p.bias)[n]) : 0.f);
    const float r = p.R ? to_f32(static_cast<const T*>(p.R)[m * p.ldr + n]) : 0.f;
    if (p.Z) static_cast<T*>(p.Z)[m * p.ldz + n] = from_f32<T>(z);
    static_cast<T*>(p.D)[m * p.ldd + n] = from_f32<T>(act_any(p.act, z) + r);
  }
}

__device__ __forceinline__ float2 fma_pair(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<unsigned long long&>(r))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)), "l"(reinterpret_cast<unsigned long long&>(c)));
  return r;
}

// The tokens into shared memory as [row][k], k padded with zeros to a multiple of 8; rows beyond M (up to MT) are zero.
template <typename T, int MT>
__device__ __forceinline__ void stage_tokens(const TokenParams& p, T* xs, int kp) {
  const T* X = static_cast<const T*>(p.X);
  if (p.x_vec) {
    const int nv = kp / 8;
    for (int i = threadIdx.x; i < MT * nv; i += blockDim.x) {
      const int m = i / nv, v = i - m * nv;
      uint4 x = make_uint4(0, 0, 0, 0);
      if (m < p.M) {
        if (v * 8 + 8 <= p.K) {
          x = *reinterpret_cast<const uint4*>(X + m * p.ldx + v * 8);
        } else {
          T* e = reinterpret_cast<T*>(&x);
          for (int j = 0; v * 8 + j < p.K; ++j) e[j] = X[m * p.ldx + v * 8 + j];
        }
      }
      reinterpret_cast<uint4*>(xs)[i] = x;
    }
  } else {
    for (int i = threadIdx.x; i < MT * kp; i += blockDim.x) {
      const int m = i / kp, k = i - m * kp;
      xs[i] = m < p.M && k < p.K ? (p.x_trans ? X[k * p.ldx + m] : X[m * p.ldx + k]) : from_f32<T>(0.f);
    }
  }
  __syncthreads();
}

template <typename T, int MT, bool GATED>
__global__ void __launch_bounds__(256) hgemm_token_kernel(const __grid_constant__ TokenParams p) {
  extern __shared__ uint4 smem[];
  __shared__ float red[8][2 * MT];
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int kp = (p.K + 7) / 8 * 8;
  T* xs = reinterpret_cast<T*>(smem);
  stage_tokens<T, MT>(p, xs, kp);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int slice = warp % p.wk, group = warp / p.wk, groups = 8 / p.wk;
  const int cols = GATED ? 1 : 2;  // output columns of a warp
  const int nfull = p.K / 8, step = 32 * p.wk;  // whole vectors of a row
  for (long long base = (long long)blockIdx.x * groups * cols; base < p.N; base += (long long)gridDim.x * groups * cols) {
    const int n = (int)base + group * cols;
    const bool in0 = n < p.N, in1 = GATED ? in0 : n + 1 < p.N;
    const T* w0 = static_cast<const T*>(p.W[0]) + (long long)(in0 ? n : 0) * p.ldw[0];
    const T* w1 = GATED ? static_cast<const T*>(p.W[1]) + (long long)(in0 ? n : 0) * p.ldw[1]
                        : static_cast<const T*>(p.W[0]) + (long long)(in1 ? n + 1 : 0) * p.ldw[0];
    float2 acc[2][MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[0][m] = acc[1][m] = make_float2(0.f, 0.f);
    int v = slice * 32 + lane;
    const auto add = [&](const uint4& a, const uint4& b, int k) {
      const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
      float2 fa[4], fb[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        fa[j] = unpack2<T>(wa[j]);
        fb[j] = unpack2<T>(wb[j]);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const uint4 x = *reinterpret_cast<const uint4*>(xs + m * kp + k);
        const uint32_t wx[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 fx = unpack2<T>(wx[j]);
          acc[0][m] = fma_pair(fa[j], fx, acc[0][m]);
          acc[1][m] = fma_pair(fb[j], fx, acc[1][m]);
        }
      }
    };
    // U steps at a time, with no condition between their loads, or they would wait for one another
    const auto turns = [&](auto unroll) {
      constexpr int U = decltype(unroll)::value;
      for (; v + (U - 1) * step < nfull; v += U * step) {
        uint4 a[U], b[U];
#pragma unroll
        for (int q = 0; q < U; ++q) {
          a[q] = __ldcs(reinterpret_cast<const uint4*>(w0 + (v + q * step) * 8));
          b[q] = __ldcs(reinterpret_cast<const uint4*>(w1 + (v + q * step) * 8));
        }
#pragma unroll
        for (int q = 0; q < U; ++q) add(a[q], b[q], (v + q * step) * 8);
      }
    };
    turns(std::integral_constant<int, 8>());
    turns(std::integral_constant<int, 4>());
    turns(std::integral_constant<int, 2>());
    turns(std::integral_constant<int, 1>());
    if (v == nfull && nfull * 8 < p.K) {  // the row's last, partial vector
      uint4 a = make_uint4(0, 0, 0, 0), b = a;
      for (int j = 0; v * 8 + j < p.K; ++j) {
        reinterpret_cast<T*>(&a)[j] = w0[v * 8 + j];
        reinterpret_cast<T*>(&b)[j] = w1[v * 8 + j];
      }
      add(a, b, v * 8);
    }
    // lane i keeps the sum of pair i / MT, row i % MT
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) {
      float s = acc[i / MT][i % MT].x + acc[i / MT][i % MT].y;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (lane == i) mine = s;
    }
    if (p.wk > 1) {
      if (lane < 2 * MT) red[warp][lane] = mine;
      __syncthreads();
      if (slice == 0 && lane < 2 * MT)
        for (int k = 1; k < p.wk; ++k) mine += red[warp + k][lane];
      __syncthreads();
    }
    const float other = __shfl_down_sync(0xffffffffu, mine, MT);
    if (slice == 0) {
      const int m = lane % MT;
      if (GATED) {
        if (lane < MT && m < p.M && in0) token_emit<T, true>(p, m, n, mine, other);
      } else if (lane < 2 * MT && m < p.M && (lane < MT ? in0 : in1)) {
        token_emit<T, false>(p, m, n + lane / MT, mine, 0.f);
      }
    }
  }
}

}  // namespace hgemm
