// Products in binary16 on the tensor cores.
#include "hgemm_kernels.cuh"

namespace hgemm {

bool launch_plain_f16(int act, int config, int clusters, cudaStream_t stream, const Params& p) {
  return launch_config<__half, false>(act, config, clusters, stream, p);
}
bool configure_plain_f16() { return configure_all<__half, false>(); }

}  // namespace hgemm
