// Launches of the kernels for products of one or two rows.
#include <atomic>

#include "hgemm_kernels.h"
#include "hgemm_token.cuh"
#include "lm_state.h"

namespace hgemm {

namespace {

// Raises the kernel's limit of dynamic shared memory to the most that a call asks for, once per device and before its first
// launch whatever that one asks for: without it static and dynamic memory together stop at 48 KB.
template <typename K, K kernel>
bool allow_smem() {
  static std::atomic<bool> done[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
  if (!done[dev].load()) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TOKEN_SMEM) != cudaSuccess) return false;
    done[dev].store(true);
  }
  return true;
}

template <typename T, int MT, bool GATED>
bool run(TokenParams p, int sms, cudaStream_t stream) {
  constexpr auto kernel = &hgemm_token_kernel<T, MT, GATED>;
  const size_t smem = (size_t)MT * ((p.K + 7) / 8 * 8) * sizeof(T);
  if (!allow_smem<decltype(kernel), kernel>()) return false;
  // enough warps for 16 per SM; a warp's share of k is at least one load of every lane
  const int cols = GATED ? 1 : 2;
  const long long pairs = (p.N + cols - 1) / cols;
  p.wk = 1;
  while (p.wk < 8 && pairs * p.wk < (long long)sms * 16 && p.K > 256 * p.wk) p.wk *= 2;
  const long long blocks = (pairs + 8 / p.wk - 1) / (8 / p.wk), most = (long long)sms * 4;
  return lm::launch(kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), smem, 1, stream, p);
}
template <typename T>
bool run_type(const TokenParams& p, bool gated, int sms, cudaStream_t stream) {
  if (p.M == 1) return gated ? run<T, 1, true>(p, sms, stream) : run<T, 1, false>(p, sms, stream);
  return gated ? run<T, 2, true>(p, sms, stream) : run<T, 2, false>(p, sms, stream);
}

}  // namespace

bool launch_token(int type, bool gated, int sms, cudaStream_t stream, const TokenParams& p) {
  return type == HGEMM_TYPE_BF16 ? run_type<__nv_bfloat16>(p, gated, sms, stream) : run_type<__half>(p, gated, sms, stream);
}

}  // namespace hgemm
