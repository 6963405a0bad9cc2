// Host state shared by the 16-bit products (hgemm_api.cu) and layer norm (layernorm.cu): per-device
// scratch, tile counters and status word, and the launch helper. Not part of the C ABI.
#pragma once

#include <cstddef>
#include <cstdint>
#include <utility>

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/hgemm.h"
#include "scratch_pool.h"

namespace lm {

constexpr int kCounters = 4096;  // per lease; zero between launches (the last arrival resets its counter)

struct DeviceState {
  bool ready = false;
  int sm_count = 0;
  int* status = nullptr;
  int* counters = nullptr;  // [scratch::kMaxLeases][kCounters]
  scratch::Pool scratch;
};

// The current device's state, set up on first use. DGEMM_OK or an error code.
int device_state(DeviceState** out);

// DGEMM_ERR_CUDA, with the runtime's last error cleared: the next call, of any part of the library, must not find it.
inline int cuda_failed() {
  (void)cudaGetLastError();
  return DGEMM_ERR_CUDA;
}

// Frees the current device's scratch leases (it has been synchronised). False if a free failed.
bool release_scratch();

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Launch with programmatic stream serialization (every kernel of these files waits for its
// predecessor before its first global access); `cluster` CTAs per cluster.
template <typename... KArgs, typename... Args>
bool launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t stream, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...) == cudaSuccess;
}

inline bool ranges_overlap(const void* p, int64_t pbytes, const void* q, int64_t qbytes) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return a < b + (uintptr_t)qbytes && b < a + (uintptr_t)pbytes;
}

}  // namespace lm
