// Gated projections in binary16 on the tensor cores.
#include "hgemm_kernels.cuh"

namespace hgemm {

bool launch_gated_f16(int act, int config, int clusters, cudaStream_t stream, const Params& p) {
  return launch_config<__half, true>(act, config, clusters, stream, p);
}
bool configure_gated_f16() { return configure_all<__half, true>(); }

}  // namespace hgemm
