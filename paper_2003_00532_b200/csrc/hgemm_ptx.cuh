// Inline-PTX wrappers for the fifth-generation tensor cores: TMEM allocation, tcgen05 MMA, commit
// and TMEM loads, and the CTA-pair forms of barrier arrivals and tile loads. Device code only.
#pragma once

#include <cstdint>
#include <cuda.h>

#include "ptx.cuh"

namespace hgemm {
namespace ptx5 {

// ---- TMEM allocation: one whole warp; for a CTA pair, one warp of each CTA -------------------------

template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t smem_dst, uint32_t cols) {
  if (CG == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
}
template <int CG>
__device__ __forceinline__ void tmem_dealloc(uint32_t addr, uint32_t cols) {
  if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
  else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}

__device__ __forceinline__ void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// ---- MMA: D (TMEM, binary32) (+)= A (smem) B (smem), 32 bytes of K (16 values of 16 bits, or 32 of 8: EIGHT); issued by one
// thread ----

template <int CG, bool EIGHT>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
#define HGEMM_MMA(form)                                                                                                            \
  asm volatile(                                                                                                                    \
      "{\n\t.reg .pred p;\n\t"                                                                                                    \
      "setp.ne.b32 p, %4, 0;\n\t"                                                                                                  \
      "tcgen05.mma." form " [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)             \
      : "memory")
  if (CG == 1 && !EIGHT) HGEMM_MMA("cta_group::1.kind::f16");
  if (CG == 2 && !EIGHT) HGEMM_MMA("cta_group::2.kind::f16");
  if (CG == 1 && EIGHT) HGEMM_MMA("cta_group::1.kind::f8f6f4");
  if (CG == 2 && EIGHT) HGEMM_MMA("cta_group::2.kind::f8f6f4");
#undef HGEMM_MMA
}

// Arrives on `bar` (for a pair: on the barrier at that offset in both CTAs) when all MMAs this
// thread has issued so far are complete.
template <int CG>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  if (CG == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)3)
                 : "memory");
}

// ---- TMEM loads ------------------------------------------------------------------------------------
// One warp reads 16 lanes (the first or second half of its own quarter) x 8 X columns. Thread t gets, for
// each block b of 8 columns, v[4 b + r]: lane t / 4 + 8 (r / 2), column 8 b + 2 (t % 4) + r % 2 -- the layout of
// the 8 x 8 matrices that stmatrix and ldmatrix move.
template <int X>
__device__ __forceinline__ void tmem_ld_16x256b(uint32_t addr, float* v);
template <>
__device__ __forceinline__ void tmem_ld_16x256b<1>(uint32_t addr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
template <>
__device__ __forceinline__ void tmem_ld_16x256b<2>(uint32_t addr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(addr));
}
// Waits for this warp's TMEM loads. The loaded registers are operands, so no use of them can move
// ahead of the wait.
template <int N>
__device__ __forceinline__ void tmem_ld_wait(float* v);
template <>
__device__ __forceinline__ void tmem_ld_wait<8>(float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])
               :
               : "memory");
}
template <>
__device__ __forceinline__ void tmem_ld_wait<16>(float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}

// ---- 8 x 8 matrices of 16-bit values between registers and shared memory, transposed ---------------------
// Lane l gives the address of row l % 8 (16 bytes) of matrix l / 8; register i of thread t holds row values
// t / 4 of rows 2 (t % 4) and 2 (t % 4) + 1 of matrix i.
__device__ __forceinline__ void stmatrix_x4_trans(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t* v) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint16_t lds16(uint32_t addr) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts16(uint32_t addr, uint16_t v) { asm volatile("st.shared.u16 [%0], %1;" ::"r"(addr), "h"(v) : "memory"); }

// ---- barriers and tile loads of a CTA pair -------------------------------------------------------------

// Arrival on a barrier in the shared memory of any CTA of the cluster (`addr` from map_to_cta). Relaxed: it
// publishes no memory, only that this warp's TMEM loads are done (they have been waited for, and
// tcgen05.fence::before_thread_sync orders them). A release at cluster scope would wait for all of the
// warp's stores to global memory: measured, 4 us per tile.
__device__ __forceinline__ void mbar_arrive_cluster_relaxed(uint32_t addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}

// Tile load into the issuing CTA's shared memory. For a pair, `bar` may be the leader's barrier
// (an address from map_to_cta): the bytes are counted there.
template <int CG>
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if (CG == 1)
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

// Lets the next kernel in the stream start its set-up while this one runs (it still waits for this
// one's completion before it touches global memory).
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace ptx5
// 16 values of 8 bits at src[0 .. 16), the columns c .. of a row of `cols`; those beyond the row are zero. Five aligned words
// shifted by the row's misalignment, or, where those would reach beyond the row, one value after the other.
__device__ __forceinline__ uint4 load16(const uint8_t* src, int c, int cols) {
  uint4 v;
  uint32_t* w = reinterpret_cast<uint32_t*>(&v);
  const int off = (int)(reinterpret_cast<uintptr_t>(src) & 3);  // bytes of the first word before the first value
  if (c >= off && c + 20 - off <= cols) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(src - off);
    uint32_t x[5];
#pragma unroll
    for (int j = 0; j < 5; ++j) x[j] = p[j];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __funnelshift_r(x[j], x[j + 1], 8 * off);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = 0;
#pragma unroll
      for (int b = 0; b < 4; ++b)
        if (c + 4 * j + b < cols) w[j] |= (uint32_t)src[4 * j + b] << 8 * b;
    }
  }
  return v;
}

}  // namespace hgemm
