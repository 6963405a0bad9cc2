// Root-mean-square norm with the residual's addition, forward (to the operands' type or to 8 bits with a scale per row)
// and backward. Bound by memory: each kernel reads its rows once and holds them through all sums, in registers or, with 32 values of 16 bits
// per thread, in shared memory (from where they are taken twice), and writes once.
//
// A row belongs to one warp (short rows: no block barrier at all) or to one block; a thread holds ITEMS vectors of VEC
// values (VEC = 16 bytes where all rows are 16-byte aligned, else single values). Blocks are persistent: a thread keeps its
// columns' gamma in registers from row to row, and the next row's loads are in flight while a row is computed.
//
// Forward: one reduction per row. For 8 bits the sum of squares and the largest |s gamma| go through it together:
// y = s rstd gamma, so max |y| = rstd max |s gamma|, and q = s gamma (rstd / scale). Rows in which these products could leave binary32's range
// take two or three more, with rstd before gamma (out_of_range()).
//
// Backward: while a block walks over its rows, each thread also keeps dgamma of its own columns in registers. The blocks'
// sums go to a partial matrix [block][column] that a second kernel (layer norm's) adds in order of the blocks: no atomics,
// same bits every time.
//
// Rows that are not 16-byte aligned (ANY), as long as all matrices are misaligned alike (which they are where a program's matrices have
// the same odd number of columns): a thread's vectors begin at the aligned address before the row, `shift` columns to the left of it, and only
// the two vectors at the row's ends are taken value by value. Every VEC-th row has the same shift, so rows are dealt out by multiples
// of VEC and a thread has the same columns for good, as with aligned rows. Matrices of different alignment are read and
// written value by value (VEC = 1). 8192 x 4089 bfloat16, with residual and by single values: Y 70 -> 47.4 us, to 8 bits 73 -> 41.9,
// gradients 108 -> 54.5; 4097 x 1537 binary32, gradients without residual 22.7 -> 19.4.
//
// Rows too long for the registers are streamed twice (the second time mostly from L2).
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hgemm_ptx.cuh"
#include "layernorm.cuh"

namespace rmsn {

using lnorm::both;
using lnorm::cvt;
using lnorm::fma2;
using lnorm::load;
using lnorm::load_row;
using lnorm::mul2;
using lnorm::add2;
using lnorm::Pairs;
using lnorm::rnd;
using lnorm::store;
using lnorm::store_row;
using lnorm::Vec;
using lnorm::warp_sum;

struct Params {
  long long rows;
  int cols;
  const void* X;      // backward: S
  const void* R;      // backward: dS
  const void* gamma;
  const void* dY;
  void* S;
  void* out;          // Y, Q or dX
  long long ldx, ldr, lds, ldo, ldy;  // ldy: of dY
  float* rstd;
  float* scale;       // of Q's rows
  float* partial;     // backward: [blocks][ldp], dgamma's
  long long ldp;      // cols rounded up to 4: every row can be written as vectors
  float eps;
  int want_params;
  int shift, shift_ld;  // ANY: columns from the aligned address to the first row; what a row adds to them (modulo VEC)
};

// Columns between the row and the aligned address before it.
template <int VEC, bool ANY>
__device__ __forceinline__ int shift_of(const Params& p, long long row) {
  return ANY ? (p.shift + (int)(row % VEC) * p.shift_ld) % VEC : 0;
}
// Items of a row whose first vector may begin before its first column (c0 < 0); values outside the row are 0, and not read or written.
template <typename T, int VEC, int ITEMS, bool ANY>
__device__ __forceinline__ void take_row(Vec<T, VEC> (&raw)[ITEMS], const T* at, int c0, int cols, bool full) {
  if constexpr (ANY) {
    if (!full) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int c = c0 + i * 32 * VEC;
        const T* src = at + i * 32 * VEC;
        if (c >= 0 && c + VEC <= cols) {
          raw[i].bits = *reinterpret_cast<const decltype(raw[i].bits)*>(src);
        } else {
#pragma unroll
          for (int j = 0; j < VEC; ++j) raw[i].set(j, (unsigned)(c + j) < (unsigned)cols ? src[j] : rnd<T>(0.f));
        }
      }
      return;
    }
  }
  load_row<T, VEC, ITEMS>(raw, at, c0, cols, full);
}
template <typename T, int VEC, int ITEMS, bool ANY>
__device__ __forceinline__ void put_row(T* at, const Pairs<T, VEC, ITEMS>& v, int c0, int cols, bool full) {
  if constexpr (ANY) {
    if (!full) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int c = c0 + i * 32 * VEC;
        T* dst = at + i * 32 * VEC;
        const Vec<T, VEC> o = v.pack(i);
        if (c >= 0 && c + VEC <= cols) {
          *reinterpret_cast<decltype(v.pack(0).bits)*>(dst) = o.bits;
        } else {
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if ((unsigned)(c + j) < (unsigned)cols) dst[j] = o.get(j);
        }
      }
      return;
    }
  }
  store_row<T, VEC, ITEMS>(at, v, c0, cols, full);
}
// gamma in the columns of a thread, at any address.
template <typename T, int VEC, int ITEMS, bool ANY>
__device__ __forceinline__ void take_gamma(Vec<T, VEC> (&raw)[ITEMS], const T* gamma, int c0, int cols, bool full) {
  if constexpr (ANY) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int c = c0 + i * 32 * VEC + j;
        raw[i].set(j, (unsigned)c < (unsigned)cols ? gamma[c] : rnd<T>(0.f));
      }
  } else {
    load_row<T, VEC, ITEMS>(raw, gamma + c0, c0, cols, full);
  }
}

// What the forward kernel makes of a row: y, y in 8 bits, or x itself in 8 bits.
constexpr int OUT_Y = 0, OUT_E4M3 = 1, OUT_ROWS = 2;

constexpr float E4M3_TOP = 448.f;          // largest finite e4m3 value
constexpr float LEAST_MAX = 0x1p-100f;     // rows that are smaller are scaled as if this were their largest value
// Sums of squares from here on (or below, with an eps that is not above) are taken again from scaled values.
constexpr float SUM_TOP = 0x1p+120f, SUM_LOW = 0x1p-90f;

// y is taken as (s gamma) rstd: the product with gamma then lies in front of the row's reduction (behind it: 8192 x 4089 bfloat16 60.3 us instead
// of 47.4, 6000 x 5120 46.4 instead of 41.7). So that it stays in binary32's range, rows whose sum of squares is Y_SUM_TOP or more (below it
// |s| < 2^27: enough for weights up to 2^100) or whose rstd is above Y_RSTD_TOP (below it what s gamma loses under 2^-149 is below 2^-130 in y) are
// taken again with rstd first. A choice by each thread's own weights cost registers in every row: 8192 x 4089 58.7 us, 16384 x 500 16.3 instead of 14.4.
constexpr float Y_SUM_TOP = 0x1p+54f, Y_RSTD_TOP = 0x1p+20f;

// For 8 bits y / scale is taken as (s gamma) (rstd 448 / max|y|). With an eps that lets rstd become large beside a row of zeros or of very small
// values that factor leaves binary32's range (max|y| is not taken below 2^-100: from rstd = 2^19 on), and s gamma loses the bits below
// 2^-149. Up to rstd = RSTD_TOP, or from max|s gamma| = WEIGHED_LOW on, the factor is at most 2^119 and what s gamma has lost stays below 2^-30
// in q; beyond them, as where s gamma overflows, the row is taken again with rstd before gamma.
constexpr float RSTD_TOP = 0x1p+10f, WEIGHED_LOW = 0x1p-110f;

// Whether a row's values have to be scaled before they are squared or multiplied by gamma; `top`: for 8 bits, the magnitude of max|s gamma|.
template <bool EIGHT>
__device__ __forceinline__ bool out_of_range(float sum, float eps, float rstd, uint32_t top) {
  if (!EIGHT) return !(sum < Y_SUM_TOP) || rstd > Y_RSTD_TOP;
  return !(sum < SUM_TOP) || (sum < SUM_LOW && eps < SUM_LOW) ||
         (EIGHT && (top >= 0x7f800000u || (rstd > RSTD_TOP && top < __float_as_uint(WEIGHED_LOW))));
}

// max(x, least) that keeps a NaN.
__device__ __forceinline__ float at_least(float x, float least) { return x < least ? least : x; }

// Two values in e4m3, `lo` in the lower byte; to nearest, ties to even, beyond 448 to 448, NaN to NaN.
__device__ __forceinline__ uint16_t e4m3_pair(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// Magnitudes as integers: their order is that of the values, with infinity above them all and NaN above infinity.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
// The largest of three magnitudes, NaN if one is: one instruction.
__device__ __forceinline__ float max_abs(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
template <int N>
__device__ __forceinline__ uint32_t magnitude_max(const float2 (&v)[N]) {
  float m = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) m = max_abs(m, v[k].x, v[k].y);
  return __float_as_uint(m);
}
template <int N>
__device__ __forceinline__ float squares(const float2 (&v)[N]) {
  float2 s = both(0.f);
#pragma unroll
  for (int k = 0; k < N; ++k) s = fma2(v[k], v[k], s);
  return s.x + s.y;
}

// A row's sum and largest magnitude, for one warp per row or for the whole block (one barrier). `red` is one of two
// buffers that are used in turn: a warp can be one reduction ahead of another.
template <bool WARP_ROW, bool SUM, bool MAX>
__device__ __forceinline__ void reduce(float& sum, uint32_t& top, uint2* red) {
  if (SUM) sum = warp_sum(sum);
  if (MAX) top = __reduce_max_sync(0xffffffffu, top);
  if (WARP_ROW) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) red[warp] = make_uint2(__float_as_uint(sum), top);
  __syncthreads();
  const uint2 part = lane < (int)(blockDim.x >> 5) ? red[lane] : make_uint2(0u, 0u);
  if (SUM) sum = warp_sum(__uint_as_float(part.x));
  if (MAX) top = __reduce_max_sync(0xffffffffu, part.y);
}

// 2^-k, k the exponent of the larger one of the row's largest magnitude and sqrt(eps); 1 where that is 0 or not finite.
__device__ __forceinline__ float row_unit(uint32_t top, float eps) {
  const uint32_t bits = max(top, magnitude(sqrtf(eps)));
  if (top == 0 || top >= 0x7f800000u) return 1.f;
  const int k = max(-126, min(126, (int)(bits >> 23) - 127));
  return __uint_as_float((uint32_t)(127 - k) << 23);
}

// By what rows are multiplied that are brought to 8 bits as they are: 448 / most in two parts. f is a quotient that is too small by 2^-22 to 2^-20 of
// itself (an approximate division is within 2^-22; scaled by 16, because it gives 0 for divisors above 2^126), rest is what its remainder
// stands for, known to 2^-40 of f and not negative, so that a zero keeps its sign. x f + x rest is rounded once: a quotient
// of 16-bit values that lies half-way between two e4m3 values is met exactly (with one rounded factor 2861 of 2088 x 8192 bfloat16 values went
// to the odd neighbour).
struct Factor {
  float f, rest;
};
__device__ __forceinline__ Factor top_over(float most) {
  const float f = __fdividef(E4M3_TOP / 16, most / 16) * (1.f - 0x1p-21f);
  return Factor{f, f > 0.f ? fmaf(-f, most, E4M3_TOP) * (1.f / E4M3_TOP) * f : 0.f};
}

// Item i times f (ROWS: times f + rest) in 8 bits, at `at` + its columns.
template <bool ROWS, typename T, int VEC, int ITEMS>
__device__ __forceinline__ void store_e4m3(uint8_t* at, const Pairs<T, VEC, ITEMS>& v, float f, float rest, int c0, int cols, bool full) {
  Pairs<T, VEC, ITEMS> w;
#pragma unroll
  for (int k = 0; k < Pairs<T, VEC, ITEMS>::N; ++k) w.v[k] = ROWS ? fma2(v.v[k], both(f), mul2(v.v[k], both(rest))) : mul2(v.v[k], both(f));
  const auto value = [&](int j) { return j % 2 ? w.v[j / 2].y : w.v[j / 2].x; };
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    uint8_t* o = at + i * 32 * VEC;
    const int c = c0 + i * 32 * VEC;
    if constexpr (VEC == 1) {
      if (c < cols) *o = (uint8_t)e4m3_pair(value(i), 0.f);
    } else {
      uint16_t q[VEC / 2];
#pragma unroll
      for (int j = 0; j < VEC / 2; ++j) q[j] = e4m3_pair(value(i * VEC + 2 * j), value(i * VEC + 2 * j + 1));
      if (full || (c >= 0 && c + VEC <= cols)) {
        if constexpr (VEC == 8) *reinterpret_cast<uint2*>(o) = make_uint2((uint32_t)q[0] | (uint32_t)q[1] << 16, (uint32_t)q[2] | (uint32_t)q[3] << 16);
        else *reinterpret_cast<uint32_t*>(o) = (uint32_t)q[0] | (uint32_t)q[1] << 16;
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if ((unsigned)(c + j) < (unsigned)cols) o[j] = (uint8_t)(q[j / 2] >> 8 * (j % 2));
      }
    }
  }
}

// ---- forward ----------------------------------------------------------------------------------------

// Most threads per row, by the values a thread holds.
constexpr int fwd_threads(int values) { return values <= 8 ? 1024 : 512; }

// WARP_ROW: four rows per block of 128 threads, one warp each; otherwise one row per block.
template <typename T, int VEC, int ITEMS, bool WARP_ROW, int OUT, bool ANY>
__global__ void __launch_bounds__(WARP_ROW ? 128 : fwd_threads(VEC* ITEMS)) fwd_kernel(const __grid_constant__ Params p) {
  __shared__ uint2 red[2][32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  using P = Pairs<T, VEC, ITEMS>;
  constexpr int N = P::N;
  constexpr bool NORM = OUT != OUT_ROWS, EIGHT = OUT != OUT_Y;
  // y with 32 values per thread: gamma behind rstd, because s gamma beside s does not fit in the registers (2000 x 16384 binary32 99.5 us, the
  // other way round 120)
  constexpr bool BEHIND = !EIGHT && VEC * ITEMS > 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long step = WARP_ROW ? (long long)gridDim.x * 4 : (long long)gridDim.x;
  long long row = WARP_ROW ? (long long)blockIdx.x * 4 + warp : (long long)blockIdx.x;
  const int c0 = ((WARP_ROW ? 0 : warp * ITEMS * 32) + lane) * VEC - shift_of<VEC, ANY>(p, row);  // first column of this thread
  const bool full = c0 >= 0 && c0 + (ITEMS - 1) * 32 * VEC + VEC <= p.cols;
  const T* x_at = static_cast<const T*>(p.X) + row * p.ldx + c0;
  const T* r_at = static_cast<const T*>(p.R) + row * p.ldr + c0;
  T* s_at = static_cast<T*>(p.S) + row * p.lds + c0;
  Vec<T, VEC> xr[ITEMS], rr[ITEMS], gr[ITEMS];
  if (NORM && p.gamma) take_gamma<T, VEC, ITEMS, ANY>(gr, static_cast<const T*>(p.gamma), c0, p.cols, full);
  if (row < p.rows) {
    take_row<T, VEC, ITEMS, ANY>(xr, x_at, c0, p.cols, full);
    if (NORM && p.R) take_row<T, VEC, ITEMS, ANY>(rr, r_at, c0, p.cols, full);
  }
  if (NORM && !p.gamma) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) gr[i].set(j, rnd<T>(1.f));
  }
  P g;
  if (NORM) g.unpack(gr);
  const float inv_n = 1.f / (float)p.cols;
  int parity = 0;
  const auto next = [&]() {  // the buffer of the next reduction
    parity ^= 1;
    return red[parity];
  };
  for (; row < p.rows;) {
    P x;
    x.unpack(xr);
    if (NORM && p.R) {
      P r;
      r.unpack(rr);
#pragma unroll
      for (int k = 0; k < N; ++k) x.v[k] = add2(x.v[k], r.v[k]);
    }
    const long long at = row;
    row += step;
    x_at += step * p.ldx;
    r_at += step * p.ldr;
    if (row < p.rows) {
      take_row<T, VEC, ITEMS, ANY>(xr, x_at, c0, p.cols, full);
      if (NORM && p.R) take_row<T, VEC, ITEMS, ANY>(rr, r_at, c0, p.cols, full);
    }
    float f = 1.f;  // what is left to multiply by
    uint32_t top = 0;
    if (NORM) {
      if (p.S) {
        put_row<T, VEC, ITEMS, ANY>(s_at, x, c0, p.cols, full);
        s_at += step * p.lds;
      }
      float sum = squares(x.v), unit = 1.f;
      P z;
      const auto weigh = [&]() {
#pragma unroll
        for (int k = 0; k < N; ++k) z.v[k] = BEHIND ? x.v[k] : mul2(x.v[k], g.v[k]);
        if (EIGHT) top = magnitude_max(z.v);
      };
      weigh();
      reduce<WARP_ROW, true, EIGHT>(sum, top, next());
      f = lnorm::inv_sqrt(sum * inv_n + p.eps);
      // (the same for all threads of a row)
      if (out_of_range<EIGHT>(sum, p.eps, f, top)) {
        uint32_t most = magnitude_max(x.v);
        float none = 0.f;
        reduce<WARP_ROW, false, true>(none, most, next());
        unit = row_unit(most, p.eps);
#pragma unroll
        for (int k = 0; k < N; ++k) x.v[k] = mul2(x.v[k], both(unit));
        sum = squares(x.v);
        uint32_t no = 0;
        reduce<WARP_ROW, true, false>(sum, no, next());
        f = lnorm::inv_sqrt(sum * inv_n + p.eps * unit * unit);
#pragma unroll
        for (int k = 0; k < N; ++k) x.v[k] = mul2(x.v[k], both(f));
        unit *= f;  // rstd
        f = 1.f;
        weigh();
        if (EIGHT) reduce<WARP_ROW, false, true>(none, top, next());
      } else {
        unit = f;
      }
      if (lane == 0 && (WARP_ROW || warp == 0) && p.rstd) p.rstd[at] = unit;
      x = z;
    } else {
      top = magnitude_max(x.v);
      float none = 0.f;
      reduce<WARP_ROW, false, true>(none, top, next());
    }
    if constexpr (EIGHT) {
      const float most = at_least(f * __uint_as_float(top), LEAST_MAX);
      if (lane == 0 && (WARP_ROW || warp == 0)) p.scale[at] = most / E4M3_TOP;
      const Factor q = NORM ? Factor{f * (E4M3_TOP / most), 0.f} : top_over(most);
      store_e4m3<!NORM>(static_cast<uint8_t*>(p.out) + at * p.ldo + c0, x, q.f, q.rest, c0, p.cols, full);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) x.v[k] = BEHIND ? mul2(mul2(x.v[k], both(f)), g.v[k]) : mul2(x.v[k], both(f));
      put_row<T, VEC, ITEMS, ANY>(static_cast<T*>(p.out) + at * p.ldo + c0, x, c0, p.cols, full);
    }
  }
}

// Rows of any length: one block per row, two passes. Sums in binary64, whose range the squares cannot leave.
template <typename T, int VEC, int OUT>
__global__ void __launch_bounds__(1024) fwd_long_kernel(const __grid_constant__ Params p) {
  __shared__ double red_sum[32];
  __shared__ uint32_t red_top[32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  constexpr bool NORM = OUT != OUT_ROWS, EIGHT = OUT != OUT_Y;
  const long long row = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const T* X = static_cast<const T*>(p.X) + row * p.ldx;
  const T* R = NORM && p.R ? static_cast<const T*>(p.R) + row * p.ldr : nullptr;
  const T* G = NORM ? static_cast<const T*>(p.gamma) : nullptr;
  const auto sum_at = [&](int c, float* v) {  // s in the VEC columns from c
    const Vec<T, VEC> x = load<T, VEC>(X, c, p.cols, 0.f);
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[j] = cvt(x.get(j));
    if (R) {
      const Vec<T, VEC> r = load<T, VEC>(R, c, p.cols, 0.f);
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[j] += cvt(r.get(j));
    }
  };
  double sum = 0.0, rstd = 1.0;
  for (int c = threadIdx.x * VEC; NORM && c < p.cols; c += blockDim.x * VEC) {
    float v[VEC];
    sum_at(c, v);
    double part = 0.0;
#pragma unroll
    for (int j = 0; j < VEC; ++j) part += (double)v[j] * v[j];
    sum += part;
  }
  if (NORM) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) red_sum[warp] = sum;
    __syncthreads();
    sum = red_sum[lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    rstd = 1.0 / sqrt(sum / p.cols + (double)p.eps);
    if (threadIdx.x == 0 && p.rstd) p.rstd[row] = (float)rstd;
  }
  // s rstd as (s a) b, both factors in range whatever rstd is
  const float b = NORM ? (float)fmin(fmax(rstd, 0x1p-100), 0x1p+100) : 1.f, a = NORM ? (float)(rstd / b) : 1.f;
  const auto value = [&](const float* v, const Vec<T, VEC>& g, int j) {
    const float y = NORM ? v[j] * b * a : v[j];
    return G ? y * cvt(g.get(j)) : y;
  };
  Factor f{1.f, 0.f};
  if (EIGHT) {
    uint32_t top = 0;
    for (int c = threadIdx.x * VEC; c < p.cols; c += blockDim.x * VEC) {
      float v[VEC];
      sum_at(c, v);
      Vec<T, VEC> g;
      if (G) g = load<T, VEC>(G, c, p.cols, 0.f);
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (c + j < p.cols) top = max(top, magnitude(value(v, g, j)));
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) red_top[warp] = top;
    __syncthreads();
    const float most = at_least(__uint_as_float(__reduce_max_sync(0xffffffffu, red_top[lane])), LEAST_MAX);
    if (threadIdx.x == 0) p.scale[row] = most / E4M3_TOP;
    f = NORM ? Factor{E4M3_TOP / most, 0.f} : top_over(most);
  }
  for (int c = threadIdx.x * VEC; c < p.cols; c += blockDim.x * VEC) {
    float v[VEC];
    sum_at(c, v);
    Vec<T, VEC> g, o;
    if (G) g = load<T, VEC>(G, c, p.cols, 0.f);
    if (NORM && p.S) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) o.set(j, rnd<T>(v[j]));
      store<T, VEC>(static_cast<T*>(p.S) + row * p.lds, c, p.cols, o);
    }
    if constexpr (EIGHT) {
      Pairs<T, VEC, 1> q;
#pragma unroll
      for (int j = 0; j < VEC; ++j) (j % 2 ? q.v[j / 2].y : q.v[j / 2].x) = value(v, g, j);
      store_e4m3<!NORM>(static_cast<uint8_t*>(p.out) + row * p.ldo + c, q, f.f, f.rest, c, p.cols, false);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) o.set(j, rnd<T>(value(v, g, j)));
      store<T, VEC>(static_cast<T*>(p.out) + row * p.ldo, c, p.cols, o);
    }
  }
}

__device__ __forceinline__ bool finite(float x) { return magnitude(x) < 0x7f800000u; }

// ---- backward ---------------------------------------------------------------------------------------

// Most threads per row: 512 with 16 values each in 128 registers.
constexpr int BWD_THREADS = 512;

// WARP_ROW: eight rows per block, one warp each; otherwise one row per block. WIDE: 32 values per thread, gamma and the
// sums for dgamma in shared memory (each thread's own entries) instead of registers.
template <typename T, int VEC, int ITEMS, bool WARP_ROW, bool WIDE, bool ANY>
__global__ void __launch_bounds__(WARP_ROW ? 256 : BWD_THREADS) bwd_kernel(const __grid_constant__ Params p) {
  static_assert(!WARP_ROW || VEC == 1, "rows of any alignment");
  extern __shared__ float sums[];  // WARP_ROW with dgamma: [value][thread]; WIDE: gamma, dgamma as [pair][thread] of float2
  __shared__ uint2 red[2][32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  using P = Pairs<T, VEC, ITEMS>;
  constexpr int N = P::N;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long step = WARP_ROW ? (long long)gridDim.x * 8 : (long long)gridDim.x;
  long long row = WARP_ROW ? (long long)blockIdx.x * 8 + warp : (long long)blockIdx.x;
  const int c0 = ((WARP_ROW ? 0 : warp * ITEMS * 32) + lane) * VEC - shift_of<VEC, ANY>(p, row);  // first column of this thread
  const bool full = c0 >= 0 && c0 + (ITEMS - 1) * 32 * VEC + VEC <= p.cols;
  const T* x_at = static_cast<const T*>(p.X) + row * p.ldx + c0;
  const T* d_at = static_cast<const T*>(p.dY) + row * p.ldy + c0;
  const T* r_at = static_cast<const T*>(p.R) + row * p.ldr + c0;
  T* o_at = static_cast<T*>(p.out) + row * p.ldo + c0;
  const T* gamma = static_cast<const T*>(p.gamma);
  const bool add = p.R && p.out;  // dS joins
  float2* w_g = reinterpret_cast<float2*>(sums) + threadIdx.x;
  float2* w_dg = w_g + N * blockDim.x;
  const float inv_n = 1.f / (float)p.cols;
  // gamma's loads and the first row's are in flight together
  Vec<T, VEC> xr[ITEMS], dr[ITEMS], gr[ITEMS];
  if (gamma) take_gamma<T, VEC, ITEMS, ANY>(gr, gamma, c0, p.cols, full);
  float rstd = 0.f;
  if (row < p.rows) {
    take_row<T, VEC, ITEMS, ANY>(xr, x_at, c0, p.cols, full);
    take_row<T, VEC, ITEMS, ANY>(dr, d_at, c0, p.cols, full);
    rstd = p.rstd[row];
  }
  P g, dg;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    g.v[k] = both(1.f);
    dg.v[k] = both(0.f);
  }
  if (gamma) g.unpack(gr);
  if (WIDE) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      w_g[k * blockDim.x] = g.v[k];
      w_dg[k * blockDim.x] = both(0.f);
    }
  }
  int parity = 0;
  for (; row < p.rows; parity ^= 1) {
    // xh and w = dy gamma of this row; beyond `cols` all are 0 (rstd may be infinite: 0 rstd is not taken there)
    P xh, w;
    xh.unpack(xr);
    w.unpack(dr);
    const float rs = rstd;
    Vec<T, VEC> rr[ITEMS];
    if (add) take_row<T, VEC, ITEMS, ANY>(rr, r_at, c0, p.cols, full);
    row += step;
    x_at += step * p.ldx;
    d_at += step * p.ldy;
    r_at += step * p.ldr;
    if (row < p.rows) {
      take_row<T, VEC, ITEMS, ANY>(xr, x_at, c0, p.cols, full);
      take_row<T, VEC, ITEMS, ANY>(dr, d_at, c0, p.cols, full);
      rstd = p.rstd[row];
    }
    if ((full || finite(rs)) && VEC * ITEMS % 2 == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) xh.v[k] = mul2(xh.v[k], both(rs));
    } else {
#pragma unroll
      for (int f = 0; f < VEC * ITEMS; ++f) {
        float& h = f % 2 ? xh.v[f / 2].y : xh.v[f / 2].x;
        h = (unsigned)(c0 + f / VEC * 32 * VEC + f % VEC) < (unsigned)p.cols ? h * rs : 0.f;
      }
    }
    float2 t = both(0.f);
    if (!WIDE) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        dg.v[k] = fma2(w.v[k], xh.v[k], dg.v[k]);
        w.v[k] = mul2(w.v[k], g.v[k]);
        t = fma2(w.v[k], xh.v[k], t);
      }
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        w_dg[k * blockDim.x] = fma2(w.v[k], xh.v[k], w_dg[k * blockDim.x]);
        w.v[k] = mul2(w.v[k], w_g[k * blockDim.x]);
        t = fma2(w.v[k], xh.v[k], t);
      }
    }
    if (p.out) {
      float sum = t.x + t.y;
      uint32_t none = 0;
      reduce<WARP_ROW, true, false>(sum, none, red[parity]);
      const float minus = -sum * inv_n;
#pragma unroll
      for (int k = 0; k < N; ++k) w.v[k] = mul2(fma2(xh.v[k], both(minus), w.v[k]), both(rs));
      if (add) {
        P r;
        r.unpack(rr);
#pragma unroll
        for (int k = 0; k < N; ++k) w.v[k] = add2(w.v[k], r.v[k]);
      }
      put_row<T, VEC, ITEMS, ANY>(o_at, w, c0, p.cols, full);
      o_at += step * p.ldo;
    }
  }
  if (!p.want_params) return;
  float* out = p.partial + blockIdx.x * p.ldp;
  if (WIDE) {
#pragma unroll
    for (int k = 0; k < N; ++k) dg.v[k] = w_dg[k * blockDim.x];
  }
  const auto value = [&](int f) { return f % 2 ? dg.v[f / 2].y : dg.v[f / 2].x; };
  const auto column = [&](int f) { return c0 + f / VEC * 32 * VEC + f % VEC; };
  if (!WARP_ROW) {
    if constexpr (VEC >= 4 && !ANY) {
#pragma unroll
      for (int f = 0; f < VEC * ITEMS; f += 4)
        if (column(f) < p.cols) *reinterpret_cast<float4*>(out + column(f)) = make_float4(value(f), value(f + 1), value(f + 2), value(f + 3));
    } else {
#pragma unroll
      for (int f = 0; f < VEC * ITEMS; ++f)
        if ((unsigned)column(f) < (unsigned)p.cols) out[column(f)] = value(f);
    }
  } else {
    // all warps' sums side by side, then added over the warps in order
#pragma unroll
    for (int f = 0; f < VEC * ITEMS; ++f) sums[f * blockDim.x + threadIdx.x] = value(f);
    __syncthreads();
    for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
      const float* at = sums + c / 32 * blockDim.x + c % 32;  // (VEC = 1: column c is value c / 32 of lane c % 32)
      float a = at[0];
      for (int k = 1; k < 8; ++k) a += at[32 * k];
      out[c] = a;
    }
  }
}

// ---- rows through shared memory ---------------------------------------------------------------------

// The kernels for many rows. A block is `groups` groups of `warps` warps, each on a row of its own; a thread holds ITEMS vectors
// of VEC values, 32 vectors apart. The next DEPTH - 1 rows are on their way into shared memory by asynchronous copies of every thread's own
// vectors (no barrier: a thread reads only what it has copied), so that what is in flight takes no registers.
struct Groups {
  int warps, groups;
};

// One vector of 16 bytes: `bytes` of it from `src`, zeros behind them.
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory");
}

__device__ __forceinline__ void copy_word_async(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void sts32(uint32_t dst, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst), "r"(v) : "memory"); }
__device__ __forceinline__ uint32_t upper(__half x) { return (uint32_t)__half_as_ushort(x) << 16; }
__device__ __forceinline__ uint32_t upper(__nv_bfloat16 x) { return (uint32_t)__bfloat16_as_ushort(x) << 16; }
__device__ __forceinline__ uint32_t upper(float) { return 0; }

// One thread's vectors of the rows on their way: [row % DEPTH][stream][item][thread].
//
// ANY: of the vector that begins before the row (`skip` bytes of it) the words inside the row are copied one by one. Where the row begins
// in the middle of a word (16-bit values), its first value goes through a register: load_odd() with the copies, put_odd() any time before
// the row is taken.
template <typename T, int VEC, int ITEMS, int DEPTH, bool ANY>
struct Ring {
  static constexpr int SIZE = 16;
  static_assert(VEC * sizeof(T) == SIZE, "vectors of 16 bytes");
  uint32_t base;     // of this thread
  int pitch;         // bytes between items
  int streams;
  int bytes[ITEMS];  // of each vector up to the row's end
  int skip;
  bool odd;          // the row begins in the middle of a word of this thread's
  __device__ __forceinline__ Ring(void* smem, int streams_, int c0, int cols) : streams(streams_) {
    base = dgemm::ptx::smem_u32(smem) + threadIdx.x * SIZE;
    pitch = blockDim.x * SIZE;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) bytes[i] = max(0, min(SIZE, (cols - c0 - i * 32 * VEC) * (int)sizeof(T)));
    skip = ANY && c0 < 0 ? -c0 * (int)sizeof(T) : 0;
    odd = ANY && skip % 4 != 0;
    if (skip > 0)  // the words outside the row stay 0
      for (int k = 0; k < DEPTH * streams; ++k)
        for (int w = 0; w < 4; ++w)
          if (4 * w < skip || 4 * w >= bytes[0]) sts32(base + k * ITEMS * pitch + 4 * w, 0);
  }
  __device__ __forceinline__ uint32_t at(int slot, int stream) const { return base + (slot * streams + stream) * ITEMS * pitch; }
  __device__ __forceinline__ void copy(int slot, int stream, const T* src) const {
    const uint32_t dst = at(slot, stream);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (ANY && i == 0 && skip > 0) {
#pragma unroll
        for (int w = 1; w < 4; ++w)
          if (4 * w >= skip && 4 * w < bytes[0]) copy_word_async(dst + 4 * w, src + 4 * w / (int)sizeof(T), min(4, bytes[0] - 4 * w));
      } else {
        copy_async(dst + i * pitch, bytes[i] > 0 ? src + i * 32 * VEC : src, bytes[i]);
      }
    }
  }
  __device__ __forceinline__ Pairs<T, VEC, 1> item(int slot, int stream, int i) const {
    Vec<T, VEC> raw[1];
    raw[0].bits = hgemm::ptx5::lds128(at(slot, stream) + i * pitch);
    Pairs<T, VEC, 1> v;
    v.unpack(raw);
    return v;
  }
  __device__ __forceinline__ T load_odd(const T* src) const { return src[skip / (int)sizeof(T)]; }
  __device__ __forceinline__ void put_odd(int slot, int stream, T v) const { sts32(at(slot, stream) + skip / 4 * 4, upper(v)); }
  __device__ __forceinline__ void take(int slot, int stream, Vec<T, VEC> (&raw)[ITEMS]) const {
    const uint32_t src = at(slot, stream);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) raw[i].bits = hgemm::ptx5::lds128(src + i * pitch);
  }
};

// Sum and largest magnitude of a row over the warps of its group; `red` as in reduce(), a part per group.
template <bool SUM, bool MAX>
__device__ __forceinline__ void reduce_group(float& sum, uint32_t& top, uint2* red, const Groups& gr, int group, int warp) {
  if (SUM) sum = warp_sum(sum);
  if (MAX) top = __reduce_max_sync(0xffffffffu, top);
  if (gr.warps == 1) return;
  const int lane = threadIdx.x & 31;
  red += group * gr.warps;
  if (lane == 0) red[warp] = make_uint2(__float_as_uint(sum), top);
  dgemm::ptx::named_barrier_sync(1 + group, gr.warps * 32);
  const uint2 part = lane < gr.warps ? red[lane] : make_uint2(0u, 0u);
  if (SUM) sum = warp_sum(__uint_as_float(part.x));
  if (MAX) top = __reduce_max_sync(0xffffffffu, part.y);
}

constexpr int RING_THREADS = 512, SMALL_RING_THREADS = 256;

// THREADS: most of a block; three blocks of 256 fit on an SM, one of 512.
template <typename T, int VEC, int ITEMS, int DEPTH, int OUT, int THREADS, bool ANY>
__global__ void __launch_bounds__(THREADS, THREADS == SMALL_RING_THREADS ? 3 : 1) fwd_ring_kernel(const __grid_constant__ Params p, const Groups gr) {
  extern __shared__ uint4 ring_smem[];
  __shared__ uint2 red[2][16];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  using P = Pairs<T, VEC, ITEMS>;
  constexpr int N = P::N;
  constexpr bool EIGHT = OUT == OUT_E4M3;
  const int lane = threadIdx.x & 31, group = (threadIdx.x >> 5) / gr.warps, warp = (threadIdx.x >> 5) - group * gr.warps;
  const long long step = (long long)gridDim.x * gr.groups;
  long long row = (long long)blockIdx.x * gr.groups + group;
  const int c0 = (warp * ITEMS * 32 + lane) * VEC - shift_of<VEC, ANY>(p, row);
  const bool full = c0 >= 0 && c0 + (ITEMS - 1) * 32 * VEC + VEC <= p.cols;
  const bool add = p.R != nullptr;
  const Ring<T, VEC, ITEMS, DEPTH, ANY> ring(ring_smem, add ? 2 : 1, c0, p.cols);
  const T* x_at = static_cast<const T*>(p.X) + row * p.ldx + c0;
  const T* r_at = static_cast<const T*>(p.R) + row * p.ldr + c0;
  long long ahead = row;
  T odd_x, odd_r;
  int late = -1;  // the slot that waits for them
  const auto send = [&](int slot) {
    if (ahead < p.rows) {
      ring.copy(slot, 0, x_at);
      if (add) ring.copy(slot, 1, r_at);
      if (ANY && ring.odd) {
        odd_x = ring.load_odd(x_at);
        if (add) odd_r = ring.load_odd(r_at);
        late = slot;
      }
    }
    copies_commit();
    ahead += step;
    x_at += step * p.ldx;
    r_at += step * p.ldr;
  };
  const auto settle = [&]() {
    if (ANY && late >= 0) {
      ring.put_odd(late, 0, odd_x);
      if (add) ring.put_odd(late, 1, odd_r);
      late = -1;
    }
  };
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d) {
    if (d > 0) settle();
    send(d);
  }
  Vec<T, VEC> g_raw[ITEMS];
  if (p.gamma) {
    take_gamma<T, VEC, ITEMS, ANY>(g_raw, static_cast<const T*>(p.gamma), c0, p.cols, full);
  } else {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) g_raw[i].set(j, rnd<T>(1.f));
  }
  settle();  // (behind gamma's loads)
  const float inv_n = 1.f / (float)p.cols;
  int parity = 0, slot = 0;
  const auto next = [&]() {  // the buffer of the next reduction
    parity ^= 1;
    return red[parity];
  };
  for (; row < p.rows; row += step) {
    send(slot == 0 ? DEPTH - 1 : slot - 1);
    copies_wait<DEPTH - 1>();
    P x;
    const auto take = [&]() {  // s
      Vec<T, VEC> raw[ITEMS];
      ring.take(slot, 0, raw);
      x.unpack(raw);
      if (add) {
        P r;
        ring.take(slot, 1, raw);
        r.unpack(raw);
#pragma unroll
        for (int k = 0; k < N; ++k) x.v[k] = add2(x.v[k], r.v[k]);
      }
    };
    take();
    float f = 1.f;  // what is left to multiply by
    uint32_t top = 0;
    float none = 0.f;
    if (p.S) put_row<T, VEC, ITEMS, ANY>(static_cast<T*>(p.S) + row * p.lds + c0, x, c0, p.cols, full);
    float sum = squares(x.v), rstd;
    const auto weigh = [&]() {
      P g;
      g.unpack(g_raw);
#pragma unroll
      for (int k = 0; k < N; ++k) x.v[k] = mul2(x.v[k], g.v[k]);
      if (EIGHT) top = magnitude_max(x.v);
    };
    weigh();
    reduce_group<true, EIGHT>(sum, top, next(), gr, group, warp);
    f = rstd = lnorm::inv_sqrt(sum * inv_n + p.eps);
    // (the same for all threads of a row)
    if (out_of_range<EIGHT>(sum, p.eps, f, top)) {
      take();
      uint32_t most = magnitude_max(x.v);
      reduce_group<false, true>(none, most, next(), gr, group, warp);
      const float unit = row_unit(most, p.eps);
#pragma unroll
      for (int k = 0; k < N; ++k) x.v[k] = mul2(x.v[k], both(unit));
      sum = squares(x.v);
      reduce_group<true, false>(sum, top, next(), gr, group, warp);
      f = lnorm::inv_sqrt(sum * inv_n + p.eps * unit * unit);
#pragma unroll
      for (int k = 0; k < N; ++k) x.v[k] = mul2(x.v[k], both(f));
      rstd = unit * f;
      f = 1.f;
      weigh();
      if (EIGHT) reduce_group<false, true>(none, top, next(), gr, group, warp);
    }
    if (lane == 0 && warp == 0 && p.rstd) p.rstd[row] = rstd;
    if constexpr (EIGHT) {
      const float most = at_least(f * __uint_as_float(top), LEAST_MAX);
      if (lane == 0 && warp == 0) p.scale[row] = most / E4M3_TOP;
      store_e4m3<false>(static_cast<uint8_t*>(p.out) + row * p.ldo + c0, x, f * (E4M3_TOP / most), 0.f, c0, p.cols, full);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) x.v[k] = mul2(x.v[k], both(f));
      put_row<T, VEC, ITEMS, ANY>(static_cast<T*>(p.out) + row * p.ldo + c0, x, c0, p.cols, full);
    }
    settle();
    slot = slot == DEPTH - 1 ? 0 : slot + 1;
  }
  copies_wait<0>();
}

// The same for longer rows, 32 values per thread: too many to be kept in registers through the reduction beside gamma, so they are read from
// shared memory once for the sums and once for the outputs.
template <typename T, int VEC, int ITEMS, int OUT, int THREADS, bool ANY>
__global__ void __launch_bounds__(THREADS, THREADS == SMALL_RING_THREADS ? 3 : 1) fwd_again_kernel(const __grid_constant__ Params p, const Groups gr) {
  extern __shared__ uint4 ring_smem[];
  __shared__ uint2 red[2][16];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  using Item = Pairs<T, VEC, 1>;
  constexpr int DEPTH = 2;
  constexpr bool EIGHT = OUT == OUT_E4M3;
  const int lane = threadIdx.x & 31, group = (threadIdx.x >> 5) / gr.warps, warp = (threadIdx.x >> 5) - group * gr.warps;
  const long long step = (long long)gridDim.x * gr.groups;
  long long row = (long long)blockIdx.x * gr.groups + group;
  const int c0 = (warp * ITEMS * 32 + lane) * VEC - shift_of<VEC, ANY>(p, row);
  const bool full = c0 >= 0 && c0 + (ITEMS - 1) * 32 * VEC + VEC <= p.cols, add = p.R != nullptr;
  const Ring<T, VEC, ITEMS, DEPTH, ANY> ring(ring_smem, add ? 2 : 1, c0, p.cols);
  const T* x_at = static_cast<const T*>(p.X) + row * p.ldx + c0;
  const T* r_at = static_cast<const T*>(p.R) + row * p.ldr + c0;
  long long ahead = row;
  T odd_x, odd_r;
  int late = -1;  // the slot that waits for them
  const auto send = [&](int slot) {
    if (ahead < p.rows) {
      ring.copy(slot, 0, x_at);
      if (add) ring.copy(slot, 1, r_at);
      if (ANY && ring.odd) {
        odd_x = ring.load_odd(x_at);
        if (add) odd_r = ring.load_odd(r_at);
        late = slot;
      }
    }
    copies_commit();
    ahead += step;
    x_at += step * p.ldx;
    r_at += step * p.ldr;
  };
  const auto settle = [&]() {
    if (ANY && late >= 0) {
      ring.put_odd(late, 0, odd_x);
      if (add) ring.put_odd(late, 1, odd_r);
      late = -1;
    }
  };
  send(0);
  Vec<T, VEC> g_raw[ITEMS];
  if (p.gamma) {
    take_gamma<T, VEC, ITEMS, ANY>(g_raw, static_cast<const T*>(p.gamma), c0, p.cols, full);
  } else {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) g_raw[i].set(j, rnd<T>(1.f));
  }
  settle();  // (behind gamma's loads)
  const float inv_n = 1.f / (float)p.cols;
  int parity = 0, slot = 0;
  const auto next = [&]() {  // the buffer of the next reduction
    parity ^= 1;
    return red[parity];
  };
  for (; row < p.rows; row += step) {
    send(slot ^ 1);
    copies_wait<1>();
    const auto item = [&](int i) {  // s
      Item x = ring.item(slot, 0, i);
      if (add) {
        const Item r = ring.item(slot, 1, i);
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) x.v[k] = add2(x.v[k], r.v[k]);
      }
      return x;
    };
    const auto times = [&](Item& x, float f) {
#pragma unroll
      for (int k = 0; k < VEC / 2; ++k) x.v[k] = mul2(x.v[k], both(f));
    };
    const auto weigh = [&](Item& x, int i) {
      Vec<T, VEC> raw[1] = {g_raw[i]};
      Item g;
      g.unpack(raw);
#pragma unroll
      for (int k = 0; k < VEC / 2; ++k) x.v[k] = mul2(x.v[k], g.v[k]);
    };
    float2 part = both(0.f);
    float most = 0.f, none = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      Item x = item(i);
      if (p.S) put_row<T, VEC, 1, ANY>(static_cast<T*>(p.S) + row * p.lds + c0 + i * 32 * VEC, x, c0 + i * 32 * VEC, p.cols, full);
#pragma unroll
      for (int k = 0; k < VEC / 2; ++k) part = fma2(x.v[k], x.v[k], part);
      if (EIGHT) {
        weigh(x, i);
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) most = max_abs(most, x.v[k].x, x.v[k].y);
      }
    }
    float sum = part.x + part.y, rstd;
    uint32_t top = __float_as_uint(most);
    reduce_group<true, EIGHT>(sum, top, next(), gr, group, warp);
    float f = rstd = lnorm::inv_sqrt(sum * inv_n + p.eps), unit = 1.f, g = 1.f;  // s unit g gamma f: y
    // (the same for all threads of a row)
    const bool rescale = out_of_range<EIGHT>(sum, p.eps, rstd, top);
    if (rescale) {
      most = 0.f;
#pragma unroll 1
      for (int i = 0; i < ITEMS; ++i) {
        const Item x = item(i);
        most = max_abs(most, __uint_as_float(magnitude_max(x.v)), 0.f);
      }
      uint32_t all = __float_as_uint(most);
      reduce_group<false, true>(none, all, next(), gr, group, warp);
      unit = row_unit(all, p.eps);
      sum = 0.f;
#pragma unroll 1
      for (int i = 0; i < ITEMS; ++i) {
        Item x = item(i);
        times(x, unit);
        sum += squares(x.v);
      }
      reduce_group<true, false>(sum, all, next(), gr, group, warp);
      g = lnorm::inv_sqrt(sum * inv_n + p.eps * unit * unit);
      rstd = unit * g;
      f = 1.f;
      if (EIGHT) {
        most = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          Item x = item(i);
          times(x, unit);
          times(x, g);
          weigh(x, i);
          most = max_abs(most, __uint_as_float(magnitude_max(x.v)), 0.f);
        }
        top = __float_as_uint(most);
        reduce_group<false, true>(none, top, next(), gr, group, warp);
      }
    }
    if (lane == 0 && warp == 0 && p.rstd) p.rstd[row] = rstd;
    if (EIGHT) {
      const float largest = at_least(f * __uint_as_float(top), LEAST_MAX);
      if (lane == 0 && warp == 0) p.scale[row] = largest / E4M3_TOP;
      f *= E4M3_TOP / largest;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      Item x = item(i);
      if (rescale) {
        times(x, unit);
        times(x, g);
      }
      weigh(x, i);
      const int c = c0 + i * 32 * VEC;
      if constexpr (EIGHT) {
        store_e4m3<false>(static_cast<uint8_t*>(p.out) + row * p.ldo + c, x, f, 0.f, c, p.cols, full);
      } else {
        times(x, f);
        put_row<T, VEC, 1, ANY>(static_cast<T*>(p.out) + row * p.ldo + c, x, c, p.cols, full);
      }
    }
    settle();
    slot ^= 1;
  }
  copies_wait<0>();
}

// dgamma: each thread keeps the sums of its own columns in registers; the block's groups add theirs up at the end, in order.
template <typename T, int VEC, int ITEMS, int DEPTH, bool ANY>
__global__ void __launch_bounds__(RING_THREADS) bwd_ring_kernel(const __grid_constant__ Params p, const Groups gr) {
  extern __shared__ float4 ring_smem4[];
  __shared__ uint2 red[2][16];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  using P = Pairs<T, VEC, ITEMS>;
  constexpr int N = P::N;
  constexpr bool AGAIN = VEC * ITEMS > 16;  // rows are read twice, because two of their matrices do not fit in registers beside dgamma
  const int lane = threadIdx.x & 31, group = (threadIdx.x >> 5) / gr.warps, warp = (threadIdx.x >> 5) - group * gr.warps;
  const long long step = (long long)gridDim.x * gr.groups;
  long long row = (long long)blockIdx.x * gr.groups + group;
  const int c0 = (warp * ITEMS * 32 + lane) * VEC - shift_of<VEC, ANY>(p, row);
  const bool full = c0 >= 0 && c0 + (ITEMS - 1) * 32 * VEC + VEC <= p.cols;
  const bool add = p.R && p.out;  // dS joins
  const Ring<T, VEC, ITEMS, DEPTH, ANY> ring(ring_smem4, add ? 3 : 2, c0, p.cols);
  const T* x_at = static_cast<const T*>(p.X) + row * p.ldx + c0;
  const T* d_at = static_cast<const T*>(p.dY) + row * p.ldy + c0;
  const T* r_at = static_cast<const T*>(p.R) + row * p.ldr + c0;
  long long ahead = row;
  T odd_x, odd_d, odd_r;
  int late = -1;  // the slot that waits for them
  const auto send = [&](int slot) {
    if (ahead < p.rows) {
      ring.copy(slot, 0, x_at);
      ring.copy(slot, 1, d_at);
      if (add) ring.copy(slot, 2, r_at);
      if (ANY && ring.odd) {
        odd_x = ring.load_odd(x_at);
        odd_d = ring.load_odd(d_at);
        if (add) odd_r = ring.load_odd(r_at);
        late = slot;
      }
    }
    copies_commit();
    ahead += step;
    x_at += step * p.ldx;
    d_at += step * p.ldy;
    r_at += step * p.ldr;
  };
  const auto settle = [&]() {
    if (ANY && late >= 0) {
      ring.put_odd(late, 0, odd_x);
      ring.put_odd(late, 1, odd_d);
      if (add) ring.put_odd(late, 2, odd_r);
      late = -1;
    }
  };
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d) {
    if (d > 0) settle();
    send(d);
  }
  Vec<T, VEC> g_raw[ITEMS];
  if (p.gamma) {
    take_gamma<T, VEC, ITEMS, ANY>(g_raw, static_cast<const T*>(p.gamma), c0, p.cols, full);
  } else {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) g_raw[i].set(j, rnd<T>(1.f));
  }
  const float inv_n = 1.f / (float)p.cols;
  P dg;
#pragma unroll
  for (int k = 0; k < N; ++k) dg.v[k] = both(0.f);
  float rstd = row < p.rows ? p.rstd[row] : 0.f;
  settle();  // (behind gamma's loads)
  int parity = 0, slot = 0;
  for (; row < p.rows; row += step, parity ^= 1) {
    send(slot == 0 ? DEPTH - 1 : slot - 1);
    const float rs = rstd;
    if (row + step < p.rows) rstd = p.rstd[row + step];
    copies_wait<DEPTH - 1>();
    if constexpr (AGAIN) {
      // item by item, both times out of shared memory
      const auto scaled = [&](int i) {  // xh
        Pairs<T, VEC, 1> v = ring.item(slot, 0, i);
        if (full || finite(rs)) {
#pragma unroll
          for (int k = 0; k < VEC / 2; ++k) v.v[k] = mul2(v.v[k], both(rs));
        } else {
#pragma unroll
          for (int f = 0; f < VEC; ++f) {
            float& h = f % 2 ? v.v[f / 2].y : v.v[f / 2].x;
            h = (unsigned)(c0 + i * 32 * VEC + f) < (unsigned)p.cols ? h * rs : 0.f;
          }
        }
        return v;
      };
      const auto weight = [&](int i) {
        Vec<T, VEC> raw[1] = {g_raw[i]};
        Pairs<T, VEC, 1> g;
        g.unpack(raw);
        return g;
      };
      float2 t = both(0.f);
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const Pairs<T, VEC, 1> xh = scaled(i), d = ring.item(slot, 1, i), g = weight(i);
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) {
          dg.v[i * VEC / 2 + k] = fma2(d.v[k], xh.v[k], dg.v[i * VEC / 2 + k]);
          t = fma2(mul2(d.v[k], g.v[k]), xh.v[k], t);
        }
      }
      if (p.out) {
        float sum = t.x + t.y;
        uint32_t none = 0;
        reduce_group<true, false>(sum, none, red[parity], gr, group, warp);
        const float minus = -sum * inv_n;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          const Pairs<T, VEC, 1> xh = scaled(i), g = weight(i);
          Pairs<T, VEC, 1> w = ring.item(slot, 1, i);
#pragma unroll
          for (int k = 0; k < VEC / 2; ++k) w.v[k] = mul2(fma2(xh.v[k], both(minus), mul2(w.v[k], g.v[k])), both(rs));
          if (add) {
            const Pairs<T, VEC, 1> r = ring.item(slot, 2, i);
#pragma unroll
            for (int k = 0; k < VEC / 2; ++k) w.v[k] = add2(w.v[k], r.v[k]);
          }
          put_row<T, VEC, 1, ANY>(static_cast<T*>(p.out) + row * p.ldo + c0 + i * 32 * VEC, w, c0 + i * 32 * VEC, p.cols, full);
        }
      }
    } else {
      // xh and w = dy gamma; beyond `cols` all are 0 (rstd may be infinite: 0 rstd is not taken there)
      P xh, w;
      {
        Vec<T, VEC> raw[ITEMS];
        ring.take(slot, 0, raw);
        xh.unpack(raw);
        ring.take(slot, 1, raw);
        w.unpack(raw);
      }
      if (full || finite(rs)) {
#pragma unroll
        for (int k = 0; k < N; ++k) xh.v[k] = mul2(xh.v[k], both(rs));
      } else {
#pragma unroll
        for (int f = 0; f < VEC * ITEMS; ++f) {
          float& h = f % 2 ? xh.v[f / 2].y : xh.v[f / 2].x;
          h = (unsigned)(c0 + f / VEC * 32 * VEC + f % VEC) < (unsigned)p.cols ? h * rs : 0.f;
        }
      }
      float2 t = both(0.f);
      {
        P g;
        g.unpack(g_raw);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          dg.v[k] = fma2(w.v[k], xh.v[k], dg.v[k]);
          w.v[k] = mul2(w.v[k], g.v[k]);
          t = fma2(w.v[k], xh.v[k], t);
        }
      }
      if (p.out) {
        float sum = t.x + t.y;
        uint32_t none = 0;
        reduce_group<true, false>(sum, none, red[parity], gr, group, warp);
        const float minus = -sum * inv_n;
#pragma unroll
        for (int k = 0; k < N; ++k) w.v[k] = mul2(fma2(xh.v[k], both(minus), w.v[k]), both(rs));
        if (add) {
          Vec<T, VEC> raw[ITEMS];
          ring.take(slot, 2, raw);
          P r;
          r.unpack(raw);
#pragma unroll
          for (int k = 0; k < N; ++k) w.v[k] = add2(w.v[k], r.v[k]);
        }
        put_row<T, VEC, ITEMS, ANY>(static_cast<T*>(p.out) + row * p.ldo + c0, w, c0, p.cols, full);
      }
    }
    settle();
    slot = slot == DEPTH - 1 ? 0 : slot + 1;
  }
  copies_wait<0>();
  if (!p.want_params) return;
  // All groups' sums side by side in shared memory, then added over the groups in order.
  __syncthreads();
  float* out = p.partial + blockIdx.x * p.ldp;
  if constexpr (ANY) {
    // by columns, which lie elsewhere in every group's threads; a word is left out behind every 32, so that eight columns per
    // lane do not meet in the same banks
    float* sums = reinterpret_cast<float*>(ring_smem4);
    const int pitch = p.cols + p.cols / 32 + 1;
#pragma unroll
    for (int f = 0; f < VEC * ITEMS; ++f) {
      const int c = c0 + f / VEC * 32 * VEC + f % VEC;
      if ((unsigned)c < (unsigned)p.cols) sums[group * pitch + c + c / 32] = f % 2 ? dg.v[f / 2].y : dg.v[f / 2].x;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.cols; c += blockDim.x) {
      const float* at = sums + c + c / 32;
      float a = at[0];
      for (int g = 1; g < gr.groups; ++g) a += at[g * pitch];
      out[c] = a;
    }
  } else {
    // four columns at a time
    static_assert(VEC % 4 == 0, "four columns at a time");
    float4* sums = ring_smem4;
    const int per = gr.warps * 32;  // threads of a group
#pragma unroll
    for (int q = 0; q < N / 2; ++q) sums[q * blockDim.x + threadIdx.x] = make_float4(dg.v[2 * q].x, dg.v[2 * q].y, dg.v[2 * q + 1].x, dg.v[2 * q + 1].y);
    __syncthreads();
    for (int e = threadIdx.x; e < per * (N / 2); e += blockDim.x) {
      const int q = e / per, t = e - q * per;
      const int c = ((t >> 5) * ITEMS * 32 + 4 * q / VEC * 32 + (t & 31)) * VEC + 4 * q % VEC;
      if (c >= p.cols) continue;
      float4 a = sums[q * blockDim.x + t];
      for (int g = 1; g < gr.groups; ++g) {
        const float4 b = sums[q * blockDim.x + g * per + t];
        a = make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
      }
      *reinterpret_cast<float4*>(out + c) = a;
    }
  }
}

// Rows of any length, dx: one block per row, two passes.
template <typename T, int VEC>
__global__ void __launch_bounds__(1024) bwd_long_kernel(const __grid_constant__ Params p) {
  __shared__ float red[32];
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const long long row = blockIdx.x;
  const T* X = static_cast<const T*>(p.X) + row * p.ldx;
  const T* D = static_cast<const T*>(p.dY) + row * p.ldy;
  const T* R = p.R ? static_cast<const T*>(p.R) + row * p.ldr : nullptr;
  const T* G = static_cast<const T*>(p.gamma);
  const float rstd = p.rstd[row];
  const auto pass = [&](auto body) {
    for (int c = threadIdx.x * VEC; c < p.cols; c += blockDim.x * VEC) {
      const Vec<T, VEC> x = load<T, VEC>(X, c, p.cols, 0.f), d = load<T, VEC>(D, c, p.cols, 0.f);
      Vec<T, VEC> g;
      if (G) g = load<T, VEC>(G, c, p.cols, 0.f);
      float xh[VEC], w[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        xh[j] = c + j < p.cols ? cvt(x.get(j)) * rstd : 0.f;
        w[j] = G ? cvt(d.get(j)) * cvt(g.get(j)) : cvt(d.get(j));
      }
      body(c, xh, w);
    }
  };
  float sum = 0.f;
  pass([&](int, const float* xh, const float* w) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum += w[j] * xh[j];
  });
  sum = lnorm::block_sum(sum, red) / (float)p.cols;
  pass([&](int c, const float* xh, const float* w) {
    Vec<T, VEC> r, o;
    if (R) r = load<T, VEC>(R, c, p.cols, 0.f);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float dx = rstd * (w[j] - xh[j] * sum);
      o.set(j, rnd<T>(R ? dx + cvt(r.get(j)) : dx));
    }
    store<T, VEC>(static_cast<T*>(p.out) + row * p.ldo, c, p.cols, o);
  });
}
// Rows of any length, dgamma: a thread per column, gridDim.y chunks of rows.
template <typename T>
__global__ void __launch_bounds__(256) bwd_long_params_kernel(const __grid_constant__ Params p) {
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int c = blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= p.cols) return;
  const long long per = (p.rows + gridDim.y - 1) / gridDim.y;
  const long long r0 = blockIdx.y * per, r1 = r0 + per < p.rows ? r0 + per : p.rows;
  float dg = 0.f;
  for (long long r = r0; r < r1; ++r)
    dg += cvt(static_cast<const T*>(p.dY)[r * p.ldy + c]) * (cvt(static_cast<const T*>(p.X)[r * p.ldx + c]) * p.rstd[r]);
  p.partial[blockIdx.y * p.ldp + c] = dg;
}

}  // namespace rmsn
