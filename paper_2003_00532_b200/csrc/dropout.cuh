// Dropout with the residual's addition, and its backward pass (the same kernel without a residual): one pass over
// the matrices, the mask from a counter-based generator.
//
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC 2011) turns a counter of four words and a key of two into four random words
// by ten rounds of two 32 x 32 -> 64 bit products. The counter is (column / 4, row, offset), so that any thread makes the words of any
// four columns by itself.
//
// Rows that are 16-byte aligned: a thread takes vectors of 16 bytes. Any other: a warp takes 128 columns, lane l makes the words of columns
// 4 l to 4 l + 3 and votes on each, and loads and stores the columns l, l + 32, ..., whose bits it picks from the votes.
//
// With a residual bound by memory once the arithmetic is short enough: 8192 x 4096 bfloat16 35 to 38 us (82 to 89 % of the copy rate), where words
// made anew for every four values, converted and rounded one by one, took 47 us. Without one (the gradient) 32 to 33 us, 65 %: the same words
// are made beside two thirds of the bytes. Rows that are not aligned, by two-byte accesses in 16 bits: 8192 x 4097 53 and 52 us (binary32, whose
// single values are words: 64 and 55, aligned 66 and 45.5).
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
  int nv;             // vectors (rows of any alignment: chunks of 128 columns) per row
  int none;           // p = 1: nothing is kept
  uint32_t threshold; // p 2^32
  float scale;        // 1 / (1 - p)
  uint32_t key[2][10]; // of every round, first and second word
  unsigned long long offset;
  const long long* step;
  const void* X;
  const void* R;
  void* Y;
  long long ldx, ldr, ldy;
};

// A block covers `tx` vectors of `ty` rows; a thread keeps its vector and walks down the rows, so that whatever in the generator's first
// rounds depends on the column or on the offset alone is computed once, and addresses advance by additions: 16 of the 20 products are left
// per four values.
struct Shape {
  int tx, ty;
};

constexpr int MAX_THREADS = 256, MIN_BLOCKS = 4;

constexpr uint32_t M0 = 0xD2511F53u, M1 = 0xCD9E8D57u, W0 = 0x9E3779B9u, W1 = 0xBB67AE85u;  // multipliers; what the key grows by

// What is fixed for a counter's column: words after the second round, and products of the third.
struct Column {
  uint32_t y3, z1, hi, lo;
};

// The words of a row in the columns of `col`; a2: the row's product of the second round.
__device__ __forceinline__ uint4 words(const Params& p, const Column& col, unsigned long long a2) {
  // round 3 from z = (z0, z1, z2, z3), of which z0's product is known
  const uint32_t z2 = (uint32_t)(a2 >> 32) ^ col.y3 ^ p.key[1][1];
  const unsigned long long b3 = (unsigned long long)z2 * M1;
  uint4 w = make_uint4((uint32_t)(b3 >> 32) ^ col.z1 ^ p.key[0][2], (uint32_t)b3, col.hi ^ (uint32_t)a2 ^ p.key[1][2], col.lo);
#pragma unroll
  for (int i = 3; i < 10; ++i) {
    const unsigned long long a = (unsigned long long)w.x * M0, b = (unsigned long long)w.z * M1;
    w = make_uint4((uint32_t)(b >> 32) ^ w.y ^ p.key[0][i], (uint32_t)b, (uint32_t)(a >> 32) ^ w.w ^ p.key[1][i], (uint32_t)a);
  }
  return w;
}
// Rounds 1 and 2 for counter column `x0`, x1 = row, x2 and x3 = offset; and what they give for every row (y0, to be combined with the row).
struct Offset {
  uint32_t o1, y0;
  unsigned long long b1;
};
__device__ __forceinline__ Offset offset_of(const Params& p) {
  const unsigned long long offset = p.offset + (p.step ? (unsigned long long)*p.step : 0ull), b1 = (unsigned long long)(uint32_t)offset * M1;
  return Offset{(uint32_t)(offset >> 32), (uint32_t)(b1 >> 32) ^ p.key[0][0], b1};
}
__device__ __forceinline__ Column column_of(const Params& p, const Offset& o, uint32_t x0) {
  const unsigned long long a1 = (unsigned long long)x0 * M0;
  const uint32_t y2 = (uint32_t)(a1 >> 32) ^ o.o1 ^ p.key[1][0];
  const unsigned long long b2 = (unsigned long long)y2 * M1;  // round 2: y0 depends on the row alone, y1 = low word of b1
  const uint32_t z0 = (uint32_t)(b2 >> 32) ^ (uint32_t)o.b1 ^ p.key[0][1];
  const unsigned long long a3 = (unsigned long long)z0 * M0;
  return Column{(uint32_t)a1, (uint32_t)b2, (uint32_t)(a3 >> 32), (uint32_t)a3};
}

// One thread's rows: `row`, and every `sweep`-th after it; the vector in the `left` columns from x_at and so on. WHOLE: all of it lies
// inside the row.
template <typename T, int VEC, bool RES, bool WHOLE>
__device__ __forceinline__ void walk(const Params& p, const Column (&col)[VEC / 4], uint32_t y0, long long row, long long sweep, const T* x_at,
                                     const T* r_at, T* y_at, int left) {
  using P = lnorm::Pairs<T, VEC, 1>;
  const uint32_t t = p.threshold;
  const bool none = p.none;
  int rows = (int)((p.rows - row + sweep - 1) / sweep);  // of this thread
  uint32_t at = (uint32_t)row;
  const long long x_on = sweep * p.ldx, r_on = sweep * p.ldr, y_on = sweep * p.ldy;
  lnorm::Vec<T, VEC> x[1], r[1];
  const auto fetch = [&]() {
    if (WHOLE) {
      x[0].bits = *reinterpret_cast<const uint4*>(x_at);
      if (RES) r[0].bits = *reinterpret_cast<const uint4*>(r_at);
    } else {
      x[0] = lnorm::load<T, VEC>(x_at, 0, left, 0.f);
      if (RES) r[0] = lnorm::load<T, VEC>(r_at, 0, left, 0.f);
    }
  };
  fetch();
  for (; rows > 0; --rows) {
    P y, add;
    y.unpack(x);
    if (RES) add.unpack(r);
    if (rows > 1) {  // the next row's loads are in flight while this one's words are made
      x_at += x_on;
      r_at += r_on;
      fetch();
    }
    const unsigned long long a2 = (unsigned long long)(y0 ^ at) * M0;
#pragma unroll
    for (int q = 0; q < VEC / 4; ++q) {
      const uint4 w = words(p, col[q], a2);
      float2& lo = y.v[2 * q];
      float2& hi = y.v[2 * q + 1];
      lo = make_float2(w.x >= t && !none ? lo.x : 0.f, w.y >= t && !none ? lo.y : 0.f);
      hi = make_float2(w.z >= t && !none ? hi.x : 0.f, w.w >= t && !none ? hi.y : 0.f);
    }
#pragma unroll
    for (int k = 0; k < VEC / 2; ++k)
      y.v[k] = RES ? lnorm::fma2(y.v[k], lnorm::both(p.scale), add.v[k]) : lnorm::mul2(y.v[k], lnorm::both(p.scale));
    if (WHOLE) *reinterpret_cast<uint4*>(y_at) = y.pack(0).bits;
    else lnorm::store<T, VEC>(y_at, 0, left, y.pack(0));
    at += (uint32_t)sweep;
    y_at += y_on;
  }
}

template <typename T, int VEC, bool RES>
__global__ void __launch_bounds__(MAX_THREADS, MIN_BLOCKS) dropout_kernel(const __grid_constant__ Params p, const Shape shape) {
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int ty = threadIdx.x / shape.tx, tx = threadIdx.x - ty * shape.tx;
  const int v = blockIdx.x * shape.tx + tx, c = v * VEC;
  const long long row = (long long)blockIdx.y * shape.ty + ty, sweep = (long long)gridDim.y * shape.ty;
  if (ty >= shape.ty || v >= p.nv || row >= p.rows) return;
  const Offset o = offset_of(p);
  Column col[VEC / 4];
#pragma unroll
  for (int q = 0; q < VEC / 4; ++q) col[q] = column_of(p, o, (uint32_t)c / 4 + q);
  const T* x = static_cast<const T*>(p.X) + row * p.ldx + c;
  const T* r = static_cast<const T*>(p.R) + row * p.ldr + c;
  T* y = static_cast<T*>(p.Y) + row * p.ldy + c;
  if (c + VEC <= p.cols) walk<T, VEC, RES, true>(p, col, o.y0, row, sweep, x, r, y, VEC);
  else walk<T, VEC, RES, false>(p, col, o.y0, row, sweep, x, r, y, p.cols - c);
}

// Rows of any alignment: warp number w of the grid takes chunk w % nv of 128 columns in row w / nv and every `sweep`-th after it, AHEAD
// rows in flight.
template <typename T, bool RES>
__global__ void __launch_bounds__(256) dropout_any_kernel(const __grid_constant__ Params p, int sweep) {
  constexpr int AHEAD = 2;
  hgemm::ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int lane = threadIdx.x & 31;
  const unsigned w = blockIdx.x * 8 + (threadIdx.x >> 5), first = w / p.nv;
  if (first >= (unsigned)sweep || first >= p.rows) return;
  const int c = (int)(w - first * p.nv) * 128 + lane;  // the lane's first column
  const Offset o = offset_of(p);
  const Column col = column_of(p, o, (uint32_t)(c - lane) / 4 + lane);
  long long row = first;
  const T* x_at = static_cast<const T*>(p.X) + row * p.ldx + c;
  const T* r_at = static_cast<const T*>(p.R) + row * p.ldr + c;
  T* y_at = static_cast<T*>(p.Y) + row * p.ldy + c;
  const long long x_on = sweep * p.ldx, r_on = sweep * p.ldr, y_on = sweep * p.ldy;
  const uint32_t t = p.threshold;
  const bool none = p.none;
  T x[AHEAD][4], r[AHEAD][4];
  const auto fetch = [&](int u, bool in) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (in && c + 32 * i < p.cols) {
        x[u][i] = x_at[32 * i];
        if (RES) r[u][i] = r_at[32 * i];
      }
    }
    x_at += x_on;
    r_at += r_on;
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) fetch(u, row + u * (long long)sweep < p.rows);
  while (row < p.rows) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (row >= p.rows) break;
      const uint4 word = words(p, col, (unsigned long long)(o.y0 ^ (uint32_t)row) * M0);
      // bit l of votes j: column 4 l + j of the chunk; the lane's column 32 i + lane is bit 8 i + lane / 4 of votes lane % 4
      const uint32_t v0 = __ballot_sync(0xffffffffu, word.x >= t && !none), v1 = __ballot_sync(0xffffffffu, word.y >= t && !none);
      const uint32_t v2 = __ballot_sync(0xffffffffu, word.z >= t && !none), v3 = __ballot_sync(0xffffffffu, word.w >= t && !none);
      const uint32_t votes = (lane & 2 ? (lane & 1 ? v3 : v2) : (lane & 1 ? v1 : v0)) >> (lane >> 2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float kept = votes >> 8 * i & 1 ? lnorm::cvt(x[u][i]) : 0.f;
        const float y = RES ? fmaf(kept, p.scale, lnorm::cvt(r[u][i])) : kept * p.scale;
        if (c + 32 * i < p.cols) y_at[32 * i] = lnorm::rnd<T>(y);
      }
      fetch(u, row + AHEAD * (long long)sweep < p.rows);
      row += sweep;
      y_at += y_on;
    }
  }
}

}  // namespace drop
