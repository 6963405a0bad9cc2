// Products of up to eight rows of 8-bit operands (new tokens): bound by reading the weights once. No TMEM set-up, no staging,
// no workspace.
//
// A warp takes 16 weight rows (gated: of both matrices), 64 bytes of k at a time. Every lane takes 16 consecutive bytes of rows
// lane / 4 and lane / 4 + 8 and of token lane / 4 into the registers of the warp-wide matrix instruction m16n8k16: which k a
// register holds does not matter as long as it is the same in both operands, so lane t of four simply keeps bytes 16 t to 16 t + 15,
// four instructions' worth. The values are widened to binary16, which is exact; products and sums are binary32. Eight tokens cost what
// one does.
//
// The bytes come through shared memory by asynchronous copies of every lane's own vectors, DEPTH - 1 steps ahead and across the rows
// that a warp takes one after the other: loads into registers the compiler keeps in flight one or two steps at a time, whatever the
// source says (4096 x 4096, one token: 10.0 us).
//
// WK warps of a block share the rows' k. Sums are binary32: per warp in ascending k, then
// over the warps in order: the same bits every time.
#pragma once

#include <cstdint>

#include "hgemm_act.cuh"
#include "hgemm_kernels.h"
#include "hgemm_token.cuh"

namespace hgemm {

// 16 e4m3 values as 8 pairs of binary16, in order.
struct Wide {
  uint32_t v[8];
  __device__ __forceinline__ explicit Wide(const uint4& x) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
          : "=r"(v[2 * i]), "=r"(v[2 * i + 1])
          : "r"(w[i]));
  }
};
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void copy_16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// Shared memory of a block: [warp][slot][vector][lane] of 16 bytes; vectors: two of each weight matrix, one of the tokens. As many slots as
// leave room for two blocks on an SM.
template <bool GATED>
struct TokenRing {
  static constexpr int NW = GATED ? 2 : 1, VECS = 2 * NW + 1, DEPTH = GATED ? 5 : 8;
  static constexpr int BYTES = 8 * DEPTH * VECS * 512;
};

template <typename T, bool GATED>
__global__ void __launch_bounds__(256) qgemm_token_kernel(const __grid_constant__ Token8Params p) {
  using R = TokenRing<GATED>;
  constexpr int NW = R::NW, DEPTH = R::DEPTH;
  extern __shared__ uint4 ring[];
  __shared__ float red[8][NW * 4][32];
  ptx5::launch_dependents();
  dgemm::ptx::grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int slice = warp % p.wk, group = warp / p.wk, groups = 8 / p.wk;
  const int all = (p.K + 63) / 64, steps = slice < all ? (all - slice + p.wk - 1) / p.wk : 0;  // of 64 bytes: all, and this warp's
  const int first = slice * 64 + 16 * t, step = p.wk * 64;                                      // the lane's bytes of a row
  const long long on = (long long)gridDim.x * groups * 16;
  const uint32_t mine = dgemm::ptx::smem_u32(ring) + (warp * DEPTH * R::VECS * 32 + lane) * 16;
  // ---- copies: `left` steps still to copy of the 16 rows from `rows`, the next one at byte k ----
  long long rows = (long long)blockIdx.x * groups * 16 + group * 16;
  int left = rows < p.N ? steps : 0, k = first;
  uint32_t to = mine;
  const uint8_t* w_at[NW][2];
  const bool x_in = g < p.M;
  const uint8_t* const x_row = p.X + (x_in ? g : 0) * p.ldx;
  const auto aim = [&]() {  // rows beyond the last read the last
#pragma unroll
    for (int q = 0; q < NW; ++q)
#pragma unroll
      for (int h = 0; h < 2; ++h) w_at[q][h] = p.W[q] + min(rows + g + 8 * h, (long long)p.N - 1) * p.ldw[q] + first;
    k = first;
  };
  aim();
  const auto send = [&]() {
    if (left > 0) {
      const int bytes = max(0, min(16, p.K - k));
#pragma unroll
      for (int q = 0; q < NW; ++q)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          copy_16(to + (2 * q + h) * 512, bytes > 0 ? w_at[q][h] : p.W[q], bytes);
          w_at[q][h] += step;
        }
      if (p.x_vec) copy_16(to + 2 * NW * 512, bytes > 0 ? x_row + k : p.X, x_in ? bytes : 0);
      else ptx5::sts128(to + 2 * NW * 512, x_in && bytes > 0 ? load16(x_row + k, k, p.K) : make_uint4(0, 0, 0, 0));
      k += step;
      to = to == mine + (DEPTH - 1) * R::VECS * 512 ? mine : to + R::VECS * 512;
      if (--left == 0) {
        rows += on;
        if (rows < p.N) {
          left = steps;
          aim();
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d) send();
  uint32_t src = mine;
  for (long long base = (long long)blockIdx.x * groups * 16; base < p.N; base += on) {
    float acc[NW][4];
#pragma unroll
    for (int q = 0; q < NW; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[q][j] = 0.f;
    for (int s = 0; s < steps; ++s) {
      send();
      asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
      const Wide xw(ptx5::lds128(src + 2 * NW * 512));
#pragma unroll
      for (int q = 0; q < NW; ++q) {
        const Wide lo(ptx5::lds128(src + 2 * q * 512)), hi(ptx5::lds128(src + (2 * q + 1) * 512));
#pragma unroll
        for (int c = 0; c < 8; c += 2) mma_16x8x16(acc[q], lo.v[c], hi.v[c], lo.v[c + 1], hi.v[c + 1], xw.v[c], xw.v[c + 1]);
      }
      src = src == mine + (DEPTH - 1) * R::VECS * 512 ? mine : src + R::VECS * 512;
    }
    if (p.wk > 1) {
#pragma unroll
      for (int q = 0; q < NW; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) red[warp][q * 4 + j][lane] = acc[q][j];
      __syncthreads();
    }
    // register j: row g + 8 (j / 2), token 2 t + j % 2
    if (slice == 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const long long n = base + group * 16 + g + 8 * (j >> 1);
        const int m = 2 * t + (j & 1);
        if (m >= p.M || n >= p.N) continue;
        float a = acc[0][j], u = GATED ? acc[NW - 1][j] : 0.f;
        for (int i = 1; i < p.wk; ++i) {
          a += red[warp + i][j][lane];
          if (GATED) u += red[warp + i][(NW - 1) * 4 + j][lane];
        }
        const float rs = p.row_scale ? p.row_scale[m] : 1.f;
        a = a * rs * (p.col_scale[0] ? p.col_scale[0][n] : 1.f);
        if (GATED) u = u * rs * (p.col_scale[1] ? p.col_scale[1][n] : 1.f);
        token_emit<T, GATED>(p.out, m, (int)n, a, u);
      }
    }
    if (p.wk > 1) __syncthreads();
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

}  // namespace hgemm
