// The tensor-core kernels by element type and kind: launchers and set-up, one source file each (they are
// most of the library's compile time).
#pragma once

#include <cuda_runtime.h>

#include "hgemm_tc.cuh"
#include "hgemm_token.cuh"

namespace hgemm {

// Tile configurations: CTAs per tile, TMEM columns (rows of the output), blocks of 128 lanes per CTA.
struct Config {
  int cg, bm, nb;
};
constexpr Config kConfigs[] = {{1, 16, 1}, {1, 32, 1}, {1, 64, 1}, {1, 128, 1}, {2, 128, 1}, {2, 256, 1}, {2, 256, 2}};
constexpr int kNumConfigs = sizeof(kConfigs) / sizeof(kConfigs[0]);

// Launches configuration `config` for activation `act` on `clusters` tiles' worth of CTAs.
bool launch_plain_f16(int act, int config, int clusters, cudaStream_t stream, const Params& p);
bool launch_plain_bf16(int act, int config, int clusters, cudaStream_t stream, const Params& p);
bool launch_gated_f16(int act, int config, int clusters, cudaStream_t stream, const Params& p);
bool launch_gated_bf16(int act, int config, int clusters, cudaStream_t stream, const Params& p);

// Products of at most TOKEN_ROWS rows with 16-byte aligned weights stored N x K (hgemm_token.cuh). The tokens must fit in
// TOKEN_SMEM bytes of shared memory.
constexpr size_t TOKEN_SMEM = 160 * 1024;
bool launch_token(int type, bool gated, int sms, cudaStream_t stream, const TokenParams& p);

// Once per device: shared-memory limits.
bool configure_plain_f16();
bool configure_plain_bf16();
bool configure_gated_f16();
bool configure_gated_bf16();

}  // namespace hgemm
