// Launches of the kernels for products of up to eight rows of 8-bit operands.
#include <type_traits>

#include "hgemm_kernels.h"
#include "lm_state.h"
#include "qgemm_token.cuh"
#include "row_launch.h"

namespace hgemm {

namespace {

template <typename T, bool GATED>
bool run(Token8Params p, int sms, cudaStream_t stream) {
  constexpr auto kernel = &qgemm_token_kernel<T, GATED>;
  // all eight warps share the rows' k, as far as each gets 64 bytes of a row: also where there are rows enough for all (28672 x 8192:
  // 45 us, with rows of their own 54), because then a warp's copies run ahead across fewer rows
  const int64_t rows = (p.N + 15) / 16;
  p.wk = 1;
  while (p.wk < 8 && p.K > 64 * p.wk) p.wk *= 2;
  const int64_t blocks = (rows + 8 / p.wk - 1) / (8 / p.wk);
  constexpr int bytes = TokenRing<GATED>::BYTES;
  using K = std::remove_const_t<decltype(kernel)>;
  if (!rowop::allow_smem<K, kernel>(bytes)) return false;
  const unsigned fit = rowop::resident_blocks<K, kernel>(sms, 256, bytes, blocks);
  return fit > 0 && lm::launch(kernel, dim3(fit), dim3(256), bytes, 1, stream, p);
}

}  // namespace

bool launch_token8(int type, bool gated, int sms, cudaStream_t stream, const Token8Params& p) {
  if (type == HGEMM_TYPE_BF16) return gated ? run<__nv_bfloat16, true>(p, sms, stream) : run<__nv_bfloat16, false>(p, sms, stream);
  return gated ? run<__half, true>(p, sms, stream) : run<__half, false>(p, sms, stream);
}

}  // namespace hgemm
