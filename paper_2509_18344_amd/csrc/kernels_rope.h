// Host-visible launcher of the preparation of queries, keys and values from the fused
// q|k|v projection (internal; the public ABI is include/subspec.h).
#pragma once

#include "kernels.h"

namespace subspec {

struct RopeArgs {
  const uint16_t* qkv;       // bf16 [M][ld]: Hq query, Hkv key, Hkv value heads of 128
  const uint16_t* bias;      // bf16 [(Hq + 2 Hkv) * 128] or null
  const uint16_t* q_weight;  // bf16 [128] or null
  const uint16_t* k_weight;  // bf16 [128] or null
  const int* positions;      // [M]
  const double* inv_freq;    // [rot / 2]
  int ld, rot, interleaved, M, Hq, Hkv;
  float eps;
  uint16_t* q;               // bf16 [M][Hq][128]
  uint16_t* k;               // bf16 [M][Hkv][128]
  uint16_t* v;               // bf16 [M][Hkv][128]
};

hipError_t launch_qkv_rope(const RopeArgs& a, hipStream_t st);

}  // namespace subspec
