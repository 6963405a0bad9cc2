// Launch and set-up of every configuration and activation of the tensor-core kernel for one element type.
#pragma once

#include "hgemm_kernels.h"
#include "lm_state.h"

namespace hgemm {

template <typename T, bool GATED, int I, int ACT>
bool launch_one(int clusters, cudaStream_t stream, const Params& p) {
  constexpr int CG = kConfigs[I].cg, BM = kConfigs[I].bm, NB = kConfigs[I].nb;
  using C = Cfg<CG, BM, NB, GATED, Kind<T>::EIGHT>;
  return lm::launch(hgemm_tc_kernel<T, CG, BM, NB, GATED, ACT>, dim3(clusters * CG), dim3(C::THREADS), (size_t)C::SMEM_BYTES, CG, stream, p);
}
template <typename T, bool GATED, int I>
bool launch_act(int act, int clusters, cudaStream_t stream, const Params& p) {
  switch (act) {
    case HGEMM_ACT_NONE: return launch_one<T, GATED, I, HGEMM_ACT_NONE>(clusters, stream, p);
    case HGEMM_ACT_RELU: return launch_one<T, GATED, I, HGEMM_ACT_RELU>(clusters, stream, p);
    case HGEMM_ACT_GELU: return launch_one<T, GATED, I, HGEMM_ACT_GELU>(clusters, stream, p);
    case HGEMM_ACT_GELU_TANH: return launch_one<T, GATED, I, HGEMM_ACT_GELU_TANH>(clusters, stream, p);
    default: return launch_one<T, GATED, I, HGEMM_ACT_SILU>(clusters, stream, p);
  }
}
template <typename T, bool GATED, int I = 0>
bool launch_config(int act, int config, int clusters, cudaStream_t stream, const Params& p) {
  if (config == I) return launch_act<T, GATED, I>(act, clusters, stream, p);
  if constexpr (I + 1 < kNumConfigs) return launch_config<T, GATED, I + 1>(act, config, clusters, stream, p);
  return false;
}

template <typename T, bool GATED, int I, int ACT = 0>
bool configure_config() {
  constexpr int CG = kConfigs[I].cg, BM = kConfigs[I].bm, NB = kConfigs[I].nb;
  if (cudaFuncSetAttribute(hgemm_tc_kernel<T, CG, BM, NB, GATED, ACT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           Cfg<CG, BM, NB, GATED, Kind<T>::EIGHT>::SMEM_BYTES) != cudaSuccess)
    return false;
  if constexpr (ACT + 1 < HGEMM_ACT_COUNT) return configure_config<T, GATED, I, ACT + 1>();
  return true;
}
template <typename T, bool GATED, int I = 0>
bool configure_all() {
  if (!configure_config<T, GATED, I>()) return false;
  if constexpr (I + 1 < kNumConfigs) return configure_all<T, GATED, I + 1>();
  return true;
}

}  // namespace hgemm
