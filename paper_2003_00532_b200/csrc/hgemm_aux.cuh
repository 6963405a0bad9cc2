// The element-wise kernels around the 16-bit products: rewriting of operands the copy engine cannot
// address, the gradients at the activation, and the constant result of an empty sum. All are bound by
// memory; all wait for the kernel before them before they touch global memory.
#pragma once

#include <cstdint>

#include "hgemm_act.cuh"
#include "hgemm_tc.cuh"

namespace hgemm {

// ---- packing --------------------------------------------------------------------------------------

struct PackOp {
  const uint16_t* src;
  long long ld_src;
  int rows, cols;
  uint16_t* dst;
  long long ld_dst;
};
struct PackOps {
  PackOp op[3];
};

// Copies up to three matrices (blockIdx.y) into 16-byte aligned rows. A thread writes 8 values as one vector; it reads
// them as five aligned words shifted by the row's misalignment, or, where those would reach beyond the row, one by one.
// (One value per thread and block row: 17 us for 1000 x 777 and 777 x 1537.)
__global__ void __launch_bounds__(256) hgemm_pack_kernel(const __grid_constant__ PackOps ops) {
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const PackOp& o = ops.op[blockIdx.y];
  const int per_row = (o.cols + 7) / 8;
  const long long total = (long long)per_row * o.rows;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
    const int r = (int)(i / per_row), c = (int)(i - (long long)r * per_row) * 8;
    const uint16_t* src = o.src + r * o.ld_src + c;
    uint4 v;
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
    const bool half = (reinterpret_cast<uintptr_t>(src) & 2) != 0;  // the first value is the upper half of its word
    if (c + 9 <= o.cols && (!half || c > 0)) {
      const uint32_t* p = reinterpret_cast<const uint32_t*>(src - (half ? 1 : 0));
      uint32_t x[5];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = p[j];
      x[4] = half ? p[4] : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = half ? __funnelshift_r(x[j], x[j + 1], 16) : x[j];
    } else {
      uint16_t e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = c + j < o.cols ? src[j] : (uint16_t)0;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = (uint32_t)e[2 * j] | (uint32_t)e[2 * j + 1] << 16;
    }
    *reinterpret_cast<uint4*>(o.dst + r * o.ld_dst + c) = v;
  }
}

// ---- empty sums -----------------------------------------------------------------------------------

// D = act(bias) + R, Z = bias: the product over no terms.
template <typename T>
__global__ void hgemm_empty_kernel(int M, int N, const T* bias, int act, const T* R, long long ldr, T* D, long long ldd, T* Z, long long ldz) {
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int n = blockIdx.x * blockDim.x + threadIdx.x;
  if (n >= N) return;
  const float z = bias ? to_f32(bias[n]) : 0.f;
  float a = z;
  switch (act) {
    case HGEMM_ACT_RELU: a = act_fwd<HGEMM_ACT_RELU>(z); break;
    case HGEMM_ACT_GELU: a = act_fwd<HGEMM_ACT_GELU>(z); break;
    case HGEMM_ACT_GELU_TANH: a = act_fwd<HGEMM_ACT_GELU_TANH>(z); break;
    case HGEMM_ACT_SILU: a = act_fwd<HGEMM_ACT_SILU>(z); break;
    default: break;
  }
  for (int m = blockIdx.y; m < M; m += gridDim.y) {
    if (Z) Z[m * ldz + n] = from_f32<T>(z);
    const float r = R ? to_f32(R[m * ldr + n]) : 0.f;
    D[m * ldd + n] = from_f32<T>(a + r);
  }
}

// ---- gradient at the activation -------------------------------------------------------------------

// VEC consecutive 16-bit values as one access.
template <int VEC> struct Raw;
template <> struct Raw<8> { using type = uint4; };
template <> struct Raw<1> { using type = uint16_t; };

template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T* p, float* v) {
  typename Raw<VEC>::type raw = *reinterpret_cast<const typename Raw<VEC>::type*>(p);
  const T* t = reinterpret_cast<const T*>(&raw);
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = to_f32(t[i]);
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* p, const float* v) {
  typename Raw<VEC>::type raw;
  T* t = reinterpret_cast<T*>(&raw);
#pragma unroll
  for (int i = 0; i < VEC; ++i) t[i] = from_f32<T>(v[i]);
  *reinterpret_cast<typename Raw<VEC>::type*>(p) = raw;
}

struct ActBwdParams {
  int M, N;
  int rows_per_chunk;
  const void* Z;
  const void* dD;
  void* dZ;         // or NULL
  float* dbias;     // or NULL
  float* partial;   // [chunks][N]
  int* counters;    // one per strip
  long long ldz, lddd, lddz;
  int act;
};

// dZ = dD act'(Z) (rounded) and dbias = column sums of the unrounded products. A block takes a strip of
// 32 VEC columns and a chunk of rows; its eight warps take every eighth row. The blocks' column sums go
// to `partial`; the block that finishes a strip last adds them in order of the chunks.
template <typename T, int VEC, int ACT>
__device__ __forceinline__ void act_bwd_body(const ActBwdParams& p, float (*red)[32 * VEC], int* last) {
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int n = (blockIdx.x * 32 + tx) * VEC;
  const int r0 = blockIdx.y * p.rows_per_chunk, r1 = min(p.M, r0 + p.rows_per_chunk);
  const bool whole = n + VEC <= p.N;
  float sum[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
  if (n < p.N) {
    for (int r = r0 + ty; r < r1; r += 8) {
      const T* pd = static_cast<const T*>(p.dD) + r * p.lddd + n;
      const T* pz = static_cast<const T*>(p.Z) + r * p.ldz + n;
      T* po = static_cast<T*>(p.dZ) + r * p.lddz + n;
      float d[VEC], z[VEC];
      if (whole) {
        load_vec<T, VEC>(pd, d);
        if (ACT != HGEMM_ACT_NONE) load_vec<T, VEC>(pz, z);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          d[i] = n + i < p.N ? to_f32(pd[i]) : 0.f;
          z[i] = ACT != HGEMM_ACT_NONE && n + i < p.N ? to_f32(pz[i]) : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        if (ACT != HGEMM_ACT_NONE) {
          float f, df;
          act_both<ACT>(z[i], f, df);
          d[i] *= df;
        }
        sum[i] += d[i];
      }
      if (p.dZ) {
        if (whole) {
          store_vec<T, VEC>(po, d);
        } else {
#pragma unroll
          for (int i = 0; i < VEC; ++i)
            if (n + i < p.N) po[i] = from_f32<T>(d[i]);
        }
      }
    }
  }
  if (!p.dbias) return;
#pragma unroll
  for (int i = 0; i < VEC; ++i) red[ty][tx * VEC + i] = sum[i];
  __syncthreads();
  const int c0 = blockIdx.x * 32 * VEC;
  for (int c = threadIdx.x; c < 32 * VEC && c0 + c < p.N; c += blockDim.x) {
    float s = 0.f;
    for (int w = 0; w < 8; ++w) s += red[w][c];
    if (gridDim.y == 1) p.dbias[c0 + c] = s;
    else __stcg(p.partial + (long long)blockIdx.y * p.N + c0 + c, s);
  }
  if (gridDim.y == 1) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    const int old = atomicAdd(p.counters + blockIdx.x, 1);
    *last = old == (int)gridDim.y - 1;
    if (*last) p.counters[blockIdx.x] = 0;
  }
  __syncthreads();
  if (!*last) return;
  __threadfence();
  for (int c = threadIdx.x; c < 32 * VEC && c0 + c < p.N; c += blockDim.x) {
    float s = 0.f;
    for (int k = 0; k < (int)gridDim.y; ++k) s += __ldcg(p.partial + (long long)k * p.N + c0 + c);
    p.dbias[c0 + c] = s;
  }
}

template <typename T, int VEC>
__global__ void __launch_bounds__(256) hgemm_act_bwd_kernel(const __grid_constant__ ActBwdParams p) {
  __shared__ float red[8][32 * VEC];
  __shared__ int last;
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  switch (p.act) {
    case HGEMM_ACT_RELU: act_bwd_body<T, VEC, HGEMM_ACT_RELU>(p, red, &last); break;
    case HGEMM_ACT_GELU: act_bwd_body<T, VEC, HGEMM_ACT_GELU>(p, red, &last); break;
    case HGEMM_ACT_GELU_TANH: act_bwd_body<T, VEC, HGEMM_ACT_GELU_TANH>(p, red, &last); break;
    case HGEMM_ACT_SILU: act_bwd_body<T, VEC, HGEMM_ACT_SILU>(p, red, &last); break;
    default: act_bwd_body<T, VEC, HGEMM_ACT_NONE>(p, red, &last); break;
  }
}

struct GatedBwdParams {
  int M, F;
  const void* G;
  const void* U;
  const void* dH;
  void* dG;
  void* dU;
  long long ldg, ldu, lddh, ldo;  // ldo: of dG and dU
  int act;
};

// dG = dH U act'(G), dU = dH act(G); both rounded. One thread per VEC columns of a row.
template <typename T, int VEC, int ACT>
__device__ __forceinline__ void gated_bwd_body(const GatedBwdParams& p) {
  const int per_row = (p.F + VEC - 1) / VEC;
  const long long total = (long long)per_row * p.M;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
    const int r = (int)(i / per_row), f = (int)(i - (long long)r * per_row) * VEC;
    const T* pg = static_cast<const T*>(p.G) + r * p.ldg + f;
    const T* pu = static_cast<const T*>(p.U) + r * p.ldu + f;
    const T* pd = static_cast<const T*>(p.dH) + r * p.lddh + f;
    T* og = static_cast<T*>(p.dG) + r * p.ldo + f;
    T* ou = static_cast<T*>(p.dU) + r * p.ldo + f;
    float g[VEC], u[VEC], d[VEC];
    const bool whole = f + VEC <= p.F;
    if (whole) {
      load_vec<T, VEC>(pg, g);
      load_vec<T, VEC>(pu, u);
      load_vec<T, VEC>(pd, d);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const bool in = f + j < p.F;
        g[j] = in ? to_f32(pg[j]) : 0.f;
        u[j] = in ? to_f32(pu[j]) : 0.f;
        d[j] = in ? to_f32(pd[j]) : 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      float a, da;
      act_both<ACT>(g[j], a, da);
      g[j] = d[j] * u[j] * da;
      u[j] = d[j] * a;
    }
    if (whole) {
      store_vec<T, VEC>(og, g);
      store_vec<T, VEC>(ou, u);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (f + j < p.F) {
          og[j] = from_f32<T>(g[j]);
          ou[j] = from_f32<T>(u[j]);
        }
    }
  }
}

template <typename T, int VEC>
__global__ void __launch_bounds__(256) hgemm_gated_bwd_kernel(const __grid_constant__ GatedBwdParams p) {
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  switch (p.act) {
    case HGEMM_ACT_RELU: gated_bwd_body<T, VEC, HGEMM_ACT_RELU>(p); break;
    case HGEMM_ACT_GELU: gated_bwd_body<T, VEC, HGEMM_ACT_GELU>(p); break;
    case HGEMM_ACT_GELU_TANH: gated_bwd_body<T, VEC, HGEMM_ACT_GELU_TANH>(p); break;
    case HGEMM_ACT_SILU: gated_bwd_body<T, VEC, HGEMM_ACT_SILU>(p); break;
    default: gated_bwd_body<T, VEC, HGEMM_ACT_NONE>(p); break;
  }
}

}  // namespace hgemm
