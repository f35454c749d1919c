// Host-visible launchers of the product in 8-bit floating point (internal; the public ABI is
// include/subspec.h).
#pragma once

#include "kernels_rows.h"

namespace subspec {

struct Fp8Args {
  const void* x;          // codes [M][K], or bf16 [M][K] where xs is null
  const uint32_t* xs;     // [fp8_words(K)][M]
  const uint8_t* w;       // weight tiles of [N][K]
  const uint32_t* ws;     // [fp8_words(K)][N]
  int M, N, K;
  uint16_t* y;            // bf16 [M][N]
};

struct Fp8Plan {
  size_t workspace_bytes;  // completion counters, then x's codes and scales where the call makes them
};
Fp8Plan fp8_plan(int M, int N, int K, bool rows8);
hipError_t launch_fp8_linear(const Fp8Plan& p, Fp8Args a, void* workspace, hipStream_t st);
hipError_t launch_fp8_pack(const uint8_t* codes, int N, int K, uint8_t* tiles, hipStream_t st);

}  // namespace subspec
