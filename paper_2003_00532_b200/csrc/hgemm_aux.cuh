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
  const void* src;  // 16-bit or 8-bit values
  long long ld_src;
  int rows, cols;
  void* dst;
  long long ld_dst;
};
struct PackOps {
  PackOp op[3];
  unsigned end[3];  // the first block that is not op i's (nor an earlier one's)
};

// 8 values of 16 bits at src[0 .. 8), the columns c .. of a row of `cols`; those beyond the row are zero. An aligned vector
// where it can be one (`vec`); else five aligned words shifted by the row's misalignment, or, where those would
// reach beyond the row, one value after the other.
__device__ __forceinline__ uint4 load8(const uint16_t* src, int c, int cols, bool vec) {
  if (vec && c + 8 <= cols) return *reinterpret_cast<const uint4*>(src);
  uint4 v;
  uint32_t* w = reinterpret_cast<uint32_t*>(&v);
  const bool half = (reinterpret_cast<uintptr_t>(src) & 2) != 0;  // the first value is the upper half of its word
  if (c + 9 <= cols && (!half || c > 0)) {
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
    for (int j = 0; j < 8; ++j) e[j] = c + j < cols ? src[j] : (uint16_t)0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (uint32_t)e[2 * j] | (uint32_t)e[2 * j + 1] << 16;
  }
  return v;
}
template <typename T>
__device__ __forceinline__ void unpack8(const uint4& raw, float* v) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = unpack2<T>(w[j]);
    v[2 * j] = f.x;
    v[2 * j + 1] = f.y;
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float* v) {
  return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}

// Copies up to three matrices into 16-byte aligned rows, a vector of 8 values per thread; `block` counts the blocks of all of
// them. (One value per thread and block row: 17 us for 1000 x 777 and 777 x 1537, this 4 us.)
__device__ __forceinline__ void pack_body(const PackOps& ops, unsigned block) {
  int k = 0;
  while (block >= ops.end[k]) ++k;
  const unsigned first = k ? ops.end[k - 1] : 0;
  const PackOp& o = ops.op[k];
  const int per_row = (o.cols + 7) / 8;
  const long long total = (long long)per_row * o.rows, step = (long long)(ops.end[k] - first) * blockDim.x;
  for (long long i = (long long)(block - first) * blockDim.x + threadIdx.x; i < total; i += step) {
    const int r = (int)(i / per_row), c = (int)(i - (long long)r * per_row) * 8;
    const uint16_t* src = static_cast<const uint16_t*>(o.src) + r * o.ld_src + c;
    const uint4 v = load8(src, c, o.cols, false);
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(o.dst) + r * o.ld_dst + c) = v;
  }
}
// (Forward. The gradients' copies are blocks of the element-wise kernels below: a launch of their own cost 2 to 3 us,
// 333 x 1537 x 1000 29.1 -> 27.2, 24 x 138 x 512 9.5 -> 7.1.)
__global__ void __launch_bounds__(256) hgemm_pack_kernel(const __grid_constant__ PackOps ops) {
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  pack_body(ops, blockIdx.x);
}

// The same copies for matrices of 8-bit values, 16 of them per thread.
__global__ void __launch_bounds__(256) hgemm_pack8_kernel(const __grid_constant__ PackOps ops) {
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const unsigned block = blockIdx.x;
  int k = 0;
  while (block >= ops.end[k]) ++k;
  const unsigned first = k ? ops.end[k - 1] : 0;
  const PackOp& o = ops.op[k];
  const int per_row = (o.cols + 15) / 16;
  const long long total = (long long)per_row * o.rows, step = (long long)(ops.end[k] - first) * blockDim.x;
  for (long long i = (long long)(block - first) * blockDim.x + threadIdx.x; i < total; i += step) {
    const int r = (int)(i / per_row), c = (int)(i - (long long)r * per_row) * 16;
    *reinterpret_cast<uint4*>(static_cast<uint8_t*>(o.dst) + r * o.ld_dst + c) = load16(static_cast<const uint8_t*>(o.src) + r * o.ld_src + c, c, o.cols);
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

// ---- range of the gradients' element-wise part ------------------------------------------------------

// dZ, dG and dU enter the products in 16 bits. bfloat16 has binary32's range; binary16 has not: dH = 1500 and U = 50 make
// 75000, beyond its largest number, where the products' results may lie well inside, and gradients without loss scaling
// fall below its smallest. So the binary16 kernels also leave the largest finite magnitude of what each block stores, and
// a second kernel looks at the largest of all: where it lies outside [2^-4, 65520) it stores the part once more, times the
// power of two that brings it into [2^14, 2^15), and the products' sums are multiplied by the inverse (both exact). One power
// serves the whole part, because each product sums over another of its dimensions; values below 2^-28 of the largest lose
// bits to it. Down to a largest value of 2^-4 the part stays as it is: there bits are lost below 2^-10 of the largest, in
// steps of 2^-20 of it, under the rounding of the larger ones.
// Where the part stays as it is this costs 2 to 3 us, the second kernel's launch (64 x 512 x 512 with SiLU 9.3 -> 11.4 us,
// 2088 x 4096 x 2088 101.4 -> 104.5); a pass that takes the largest magnitude first would read every call's inputs twice.
struct PartRange {
  float* inverse;   // what the products' sums are multiplied by: written by the second kernel
  unsigned* top;    // bits of each block's largest magnitude
};
__device__ __forceinline__ unsigned finite_magnitude(float x) {
  const unsigned m = __float_as_uint(x) & 0x7fffffffu;
  return m < 0x7f800000u ? m : 0u;
}
// The largest of the block's values, in every thread (256 of them).
__device__ __forceinline__ unsigned block_max(unsigned top) {
  __shared__ unsigned most[8];
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) top = max(top, most[w]);
  return top;
}
// Second kernel: the power of two that the part is to be multiplied by, from the `blocks` blocks of the first.
__device__ __forceinline__ float part_scale(const PartRange& r, unsigned blocks) {
  unsigned top = 0;
#pragma unroll 4
  for (unsigned i = threadIdx.x; i < blocks; i += 256) top = max(top, __ldcg(r.top + i));
  top = block_max(top);
  const float t = __uint_as_float(top);
  int e = 0;
  if (top != 0 && !(t >= 0.0625f && t < 65520.f)) e = min(14 + 127 - (int)(top >> 23), 100);
  if (blockIdx.x == 0 && threadIdx.x == 0) *r.inverse = __int_as_float((127 - e) << 23);
  return __int_as_float((127 + e) << 23);
}

// ---- gradient at the activation -------------------------------------------------------------------

struct ActBwdParams {
  int M, N;
  int rows_per_chunk;
  int lane_bits;    // 2^lane_bits threads to a row, 32 at most
  unsigned strips, chunks;  // one block each; the blocks beyond copy operands
  const void* Z;
  const void* dD;
  void* dZ;         // rows of 16-byte vectors (padding columns are written); or NULL
  float* dbias;     // or NULL
  float* partial;   // [chunks][N rounded up to 8]
  int* counters;    // one per strip
  long long ldz, lddd, lddz;
  int act;
  int vec_z, vec_d;  // 16-byte aligned rows
  PartRange range;   // of a binary16 dZ; or NULLs
};

// dZ = dD act'(Z) (rounded) and dbias = column sums of the unrounded products. A block takes a strip of 64 or 256 columns
// (a thread 8 of them; of fewer columns, fewer threads to a row and more rows at a time) and a chunk of rows. The blocks'
// column sums go to `partial`; the block that finishes a strip last adds them up, its threads every R-th chunk each, in an
// order that depends on the sizes alone (one thread per column for all chunks, eight rows at a time: 5451 x 280 15.4 us
// for 8.3 now, 7269 x 70 18.6 for 9.1). Large ones stand near half of the copy rate (2088 x 4096: 18 us), held by the
// activation's arithmetic, small ones wait for the chain load - sum - partial - join. The rounding of dZ is what the products
// cannot do without: the tensor cores take 16-bit operands, and dZ in two 16-bit parts would double their MMAs. It makes the error
// of dA and dB against 64 bits 2.35e-3 in bfloat16 (2-norm), where a binary32 dZ leaves the outputs' own rounding, 1.66e-3.
template <typename T, int ACT>
__device__ __forceinline__ void act_bwd_body(const ActBwdParams& p, float (*red)[256], int* last) {
  const unsigned strip = blockIdx.x % p.strips, chunk = blockIdx.x / p.strips;
  const int W = 1 << p.lane_bits, R = 256 >> p.lane_bits;
  const int tx = threadIdx.x & (W - 1), ty = threadIdx.x >> p.lane_bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n = ((strip << p.lane_bits) + tx) * 8;
  const int r0 = chunk * p.rows_per_chunk, r1 = min(p.M, r0 + p.rows_per_chunk);
  constexpr bool RANGED = std::is_same<T, __half>::value && ACT != HGEMM_ACT_NONE && ACT != HGEMM_ACT_RELU;
  unsigned top = 0;
  float sum[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] = 0.f;
  if (n < p.N) {
    const uint16_t* pd = static_cast<const uint16_t*>(p.dD) + n;
    const uint16_t* pz = static_cast<const uint16_t*>(p.Z) + n;
    uint16_t* po = static_cast<uint16_t*>(p.dZ) + n;
    const auto one = [&](const uint4& raw_d, const uint4& raw_z, int r) {
      float d[8];
      unpack8<T>(raw_d, d);
      if (ACT != HGEMM_ACT_NONE) {
        float z[8];
        unpack8<T>(raw_z, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float f, df;
          act_both<ACT>(z[i], f, df);
          d[i] *= df;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum[i] += d[i];
        if (RANGED) top = max(top, finite_magnitude(d[i]));
      }
      if (p.dZ) *reinterpret_cast<uint4*>(po + r * p.lddz) = pack8<T>(d);
    };
    int r = r0 + ty;
    // two rows at a time where both are aligned vectors: no condition between the loads, or they would wait for one
    // another (four rows made so much straight code that fetching it was the limit)
    if (n + 8 <= p.N && p.vec_d && (ACT == HGEMM_ACT_NONE || p.vec_z)) {
#pragma unroll 1
      for (; r + R < r1; r += 2 * R) {
        uint4 d[2], z[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          d[i] = *reinterpret_cast<const uint4*>(pd + (r + R * i) * p.lddd);
          if (ACT != HGEMM_ACT_NONE) z[i] = *reinterpret_cast<const uint4*>(pz + (r + R * i) * p.ldz);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) one(d[i], z[i], r + R * i);
      }
    }
#pragma unroll 1
    for (; r < r1; r += R) {
      const uint4 d = load8(pd + r * p.lddd, n, p.N, p.vec_d);
      uint4 z = d;
      if (ACT != HGEMM_ACT_NONE) z = load8(pz + r * p.ldz, n, p.N, p.vec_z);
      one(d, z, r);
    }
  }
  if (RANGED && p.range.top) {
    top = block_max(top);
    if (threadIdx.x == 0) p.range.top[blockIdx.x] = top;
  }
  if (!p.dbias) return;
  // the sum over the rows of threads, of column threadIdx.x of the strip
  const auto over_rows = [&]() {
    for (int o = W; o < 32; o *= 2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
    }
    if (lane < W) {
      *reinterpret_cast<float4*>(&red[warp][8 * lane]) = make_float4(sum[0], sum[1], sum[2], sum[3]);
      *reinterpret_cast<float4*>(&red[warp][8 * lane + 4]) = make_float4(sum[4], sum[5], sum[6], sum[7]);
    }
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += red[w][threadIdx.x];
    return t;
  };
  const int c0 = (strip << p.lane_bits) * 8 + threadIdx.x;
  const bool in = (int)threadIdx.x < 8 * W && c0 < p.N;
  const long long ld = (p.N + 7) / 8 * 8;
  const float t = over_rows();
  if (p.chunks == 1) {
    if (in) p.dbias[c0] = t;
    return;
  }
  if (in) __stcg(p.partial + chunk * ld + c0, t);
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    const int old = atomicAdd(p.counters + strip, 1);
    *last = old == (int)p.chunks - 1;
    if (*last) p.counters[strip] = 0;
  }
  __syncthreads();
  if (!*last) return;
  __threadfence();
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] = 0.f;
  if (n < p.N) {  // (the columns beyond N, of the last 8, hold anything and are dropped)
#pragma unroll 8
    for (int k = ty; k < (int)p.chunks; k += R) {
      const float4 a = __ldcg(reinterpret_cast<const float4*>(p.partial + k * ld + n));
      const float4 b = __ldcg(reinterpret_cast<const float4*>(p.partial + k * ld + n + 4));
      sum[0] += a.x, sum[1] += a.y, sum[2] += a.z, sum[3] += a.w;
      sum[4] += b.x, sum[5] += b.y, sum[6] += b.z, sum[7] += b.w;
    }
  }
  const float s = over_rows();
  if (in) p.dbias[c0] = s;
}

template <typename T>
__global__ void __launch_bounds__(256) hgemm_act_bwd_kernel(const __grid_constant__ ActBwdParams p, const __grid_constant__ PackOps ops) {
  __shared__ __align__(16) float red[8][256];
  __shared__ int last;
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  if (blockIdx.x >= p.strips * p.chunks) {
    pack_body(ops, blockIdx.x - p.strips * p.chunks);
    return;
  }
  switch (p.act) {
    case HGEMM_ACT_RELU: act_bwd_body<T, HGEMM_ACT_RELU>(p, red, &last); break;
    case HGEMM_ACT_GELU: act_bwd_body<T, HGEMM_ACT_GELU>(p, red, &last); break;
    case HGEMM_ACT_GELU_TANH: act_bwd_body<T, HGEMM_ACT_GELU_TANH>(p, red, &last); break;
    case HGEMM_ACT_SILU: act_bwd_body<T, HGEMM_ACT_SILU>(p, red, &last); break;
    default: act_bwd_body<T, HGEMM_ACT_NONE>(p, red, &last); break;
  }
}

struct GatedBwdParams {
  int M, F;
  const void* G;
  const void* U;
  const void* dH;
  void* dG;  // rows of 16-byte vectors (padding columns are written)
  void* dU;
  long long ldg, ldu, lddh, ldo;  // ldo: of dG and dU
  int act;
  int vec_g, vec_u, vec_h;  // 16-byte aligned rows
  unsigned blocks;          // the blocks beyond copy operands
  PartRange range;          // of a binary16 dG and dU; or NULLs
};

// dG = dH U act'(G), dU = dH act(G); both rounded, AGAIN: times `scale` first. One thread per 8 columns of a row.
template <typename T, int ACT, bool AGAIN = false>
__device__ __forceinline__ void gated_bwd_body(const GatedBwdParams& p, float scale = 1.f) {
  constexpr bool RANGED = std::is_same<T, __half>::value && !AGAIN;
  unsigned top = 0;
  const int per_row = (p.F + 7) / 8;
  const bool vec = p.vec_g && p.vec_u && p.vec_h;
  const long long total = (long long)per_row * p.M;
  const unsigned blocks = AGAIN ? gridDim.x : p.blocks;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)blocks * blockDim.x) {
    const int r = (int)(i / per_row), f = (int)(i - (long long)r * per_row) * 8;
    const uint16_t* pg = static_cast<const uint16_t*>(p.G) + r * p.ldg + f;
    const uint16_t* pu = static_cast<const uint16_t*>(p.U) + r * p.ldu + f;
    const uint16_t* pd = static_cast<const uint16_t*>(p.dH) + r * p.lddh + f;
    uint4 rg, ru, rd;
    if (vec && f + 8 <= p.F) {  // one condition for the three loads, or they would wait for one another
      rg = *reinterpret_cast<const uint4*>(pg);
      ru = *reinterpret_cast<const uint4*>(pu);
      rd = *reinterpret_cast<const uint4*>(pd);
    } else {
      rg = load8(pg, f, p.F, p.vec_g);
      ru = load8(pu, f, p.F, p.vec_u);
      rd = load8(pd, f, p.F, p.vec_h);
    }
    float g[8], u[8], d[8];
    unpack8<T>(rg, g);
    unpack8<T>(ru, u);
    unpack8<T>(rd, d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float a, da;
      act_both<ACT>(g[j], a, da);
      g[j] = d[j] * u[j] * da;
      u[j] = d[j] * a;
      if (RANGED) top = max(top, max(finite_magnitude(g[j]), finite_magnitude(u[j])));
      if (AGAIN) {
        g[j] *= scale;
        u[j] *= scale;
      }
    }
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.dG) + r * p.ldo + f) = pack8<T>(g);
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.dU) + r * p.ldo + f) = pack8<T>(u);
  }
  if (RANGED && p.range.top) {
    top = block_max(top);
    if (threadIdx.x == 0) p.range.top[blockIdx.x] = top;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) hgemm_gated_bwd_kernel(const __grid_constant__ GatedBwdParams p, const __grid_constant__ PackOps ops) {
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  if (blockIdx.x >= p.blocks) {
    pack_body(ops, blockIdx.x - p.blocks);
    return;
  }
  switch (p.act) {
    case HGEMM_ACT_RELU: gated_bwd_body<T, HGEMM_ACT_RELU>(p); break;
    case HGEMM_ACT_GELU: gated_bwd_body<T, HGEMM_ACT_GELU>(p); break;
    case HGEMM_ACT_GELU_TANH: gated_bwd_body<T, HGEMM_ACT_GELU_TANH>(p); break;
    case HGEMM_ACT_SILU: gated_bwd_body<T, HGEMM_ACT_SILU>(p); break;
    default: gated_bwd_body<T, HGEMM_ACT_NONE>(p); break;
  }
}

// The second pass over a binary16 part outside the range: the same values times the chosen power of two.
__global__ void __launch_bounds__(256) hgemm_gated_rescale_kernel(const __grid_constant__ GatedBwdParams p) {
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const float scale = part_scale(p.range, p.blocks);
  if (scale == 1.f) return;
  switch (p.act) {
    case HGEMM_ACT_RELU: gated_bwd_body<__half, HGEMM_ACT_RELU, true>(p, scale); break;
    case HGEMM_ACT_GELU: gated_bwd_body<__half, HGEMM_ACT_GELU, true>(p, scale); break;
    case HGEMM_ACT_GELU_TANH: gated_bwd_body<__half, HGEMM_ACT_GELU_TANH, true>(p, scale); break;
    case HGEMM_ACT_SILU: gated_bwd_body<__half, HGEMM_ACT_SILU, true>(p, scale); break;
    default: gated_bwd_body<__half, HGEMM_ACT_NONE, true>(p, scale); break;
  }
}
template <int ACT>
__device__ __forceinline__ void act_rescale_body(const ActBwdParams& p, float scale) {
  const int per_row = (p.N + 7) / 8;
  const long long total = (long long)per_row * p.M;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
    const int r = (int)(i / per_row), n = (int)(i - (long long)r * per_row) * 8;
    float d[8], z[8];
    unpack8<__half>(load8(static_cast<const uint16_t*>(p.dD) + r * p.lddd + n, n, p.N, p.vec_d), d);
    unpack8<__half>(load8(static_cast<const uint16_t*>(p.Z) + r * p.ldz + n, n, p.N, p.vec_z), z);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float f, df;
      act_both<ACT>(z[j], f, df);
      d[j] = d[j] * df * scale;
    }
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.dZ) + r * p.lddz + n) = pack8<__half>(d);
  }
}
__global__ void __launch_bounds__(256) hgemm_act_rescale_kernel(const __grid_constant__ ActBwdParams p) {
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const float scale = part_scale(p.range, p.strips * p.chunks);
  if (scale == 1.f) return;
  switch (p.act) {
    case HGEMM_ACT_GELU: act_rescale_body<HGEMM_ACT_GELU>(p, scale); break;
    case HGEMM_ACT_GELU_TANH: act_rescale_body<HGEMM_ACT_GELU_TANH>(p, scale); break;
    default: act_rescale_body<HGEMM_ACT_SILU>(p, scale); break;
  }
}

}  // namespace hgemm
