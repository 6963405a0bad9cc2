// What the C entry points of the operators on rows share (layernorm.cu, rmsnorm.cu, dropout.cu): checks of matrix arguments,
// threads per row, blocks on the device.
#pragma once

#include <atomic>
#include <cstdint>

#include <cuda_runtime.h>

#include "../../include/hgemm.h"

namespace rowop {

constexpr int64_t kMaxDim = (int64_t)INT32_MAX - 65536;

inline int elem_bytes(int type) { return type == HGEMM_TYPE_F32 ? 4 : 2; }

// A matrix argument: NULL only where it is empty, element-aligned, ld >= max(1, cols).
inline int check(int type, const void* ptr, int64_t rows, int64_t cols, int64_t ld) {
  if (ld < (cols > 0 ? cols : 1) || ld > (int64_t)1 << 38) return DGEMM_ERR_BAD_LD;
  if (rows == 0 || cols == 0) return DGEMM_OK;
  if (!ptr) return DGEMM_ERR_NULL;
  if ((uintptr_t)ptr & (elem_bytes(type) - 1)) return DGEMM_ERR_ALIGN;
  return DGEMM_OK;
}

// Bytes from its first value to its last.
inline int64_t span(int type, int64_t rows, int64_t cols, int64_t ld) { return rows > 0 && cols > 0 ? ((rows - 1) * ld + cols) * elem_bytes(type) : 0; }

// Whether its rows are 16-byte aligned.
inline bool rows_aligned(int type, const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld * elem_bytes(type) % 16 == 0; }

inline bool bad_type(int type) { return type != HGEMM_TYPE_F32 && type != HGEMM_TYPE_F16 && type != HGEMM_TYPE_BF16; }

// Smallest power of two >= n.
inline int pow2(int64_t n) {
  int p = 1;
  while (p < n) p *= 2;
  return p;
}
// Threads of a block that covers nv vectors with `items` per thread (a warp covers 32 items vectors).
inline int threads_for(int64_t nv, int items) { return (int)((nv + 32 * items - 1) / (32 * items) * 32); }


// Raises the kernel's limit of dynamic shared memory to `bytes`, the most that any call asks for, once per device and before
// its first launch or occupancy query whatever that one asks for: without it static and dynamic memory together stop at 48 KB.
template <typename K, K kernel>
bool allow_smem(int bytes) {
  static std::atomic<bool> done[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
  if (!done[dev].load()) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    done[dev].store(true);
  }
  return true;
}

// Blocks of one kernel (one instance of this function per kernel) that fit on the device at once, or fewer
// for few rows; 0 on failure. `smem` is the most that the kernel is launched with.
template <typename K, K kernel>
unsigned resident_blocks(int sms, int threads, size_t smem, int64_t need) {
  static std::atomic<int> known[33];  // by warps per block; the same on every device of this kind
  int per_sm = known[threads / 32].load();
  if (per_sm == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem) != cudaSuccess || per_sm < 1) return 0;
    known[threads / 32].store(per_sm);
  }
  return (unsigned)(need < (int64_t)sms * per_sm ? need : (int64_t)sms * per_sm);
}

}  // namespace rowop
