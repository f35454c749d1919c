// Host-visible launchers of the row operators between two projections and of 8-bit rows
// (internal; the public ABI is include/subspec.h).
#pragma once

#include "kernels.h"

namespace subspec {

constexpr int kFp8Block = 128;  // values of a row that share a scale

// 32-bit words of four scale bytes that a row has, one after every `rows` words.
inline int fp8_words(int K) { return (K + 4 * kFp8Block - 1) / (4 * kFp8Block); }

constexpr int kNormMostK = 65536;  // a row stays in one workgroup's registers

struct NormArgs {
  const uint16_t* x;         // bf16 [M][K]
  const uint16_t* residual;  // bf16 [M][K] or null
  const uint16_t* weight;    // bf16 [K]
  float eps;
  int M, K;
  uint16_t* sum;             // bf16 [M][K] or null
  uint16_t* y;               // bf16 [M][K] or null
  uint8_t* codes;            // [M][K] or null, with
  uint8_t* scales;           // bytes of [fp8_words(K)][M] words
};
hipError_t launch_add_norm(const NormArgs& a, hipStream_t st);

struct ActArgs {
  const uint16_t* gu;        // bf16 [M][2 I]
  int M, I;
  uint16_t* y;               // bf16 [M][I] or null
  uint8_t* codes;            // [M][I] or null, with
  uint8_t* scales;
};
hipError_t launch_silu_mul(const ActArgs& a, hipStream_t st);

hipError_t launch_fp8_rows(const uint16_t* x, int M, int K, uint8_t* codes, uint8_t* scales, hipStream_t st);
hipError_t launch_fp8_read(const uint8_t* codes, const uint8_t* scales, int M, int K, uint16_t* y, hipStream_t st);

}  // namespace subspec
