// Gated projections in bfloat16 on the tensor cores.
#include "hgemm_kernels.cuh"

namespace hgemm {

bool launch_gated_bf16(int act, int config, int clusters, cudaStream_t stream, const Params& p) {
  return launch_config<__nv_bfloat16, true>(act, config, clusters, stream, p);
}
bool configure_gated_bf16() { return configure_all<__nv_bfloat16, true>(); }

}  // namespace hgemm
