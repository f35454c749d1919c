// Bias, norm and position rotation of one head row, 16 lanes of 8 dimensions each: shared
// by the kernels that prepare queries, keys and values.
#pragma once

#include "device_common.h"
#include "kernels_rope.h"

namespace subspec {

constexpr int kRopeD = 128;
constexpr int kRopeHalf = kRopeD / 2;

__device__ __forceinline__ float rope_bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float rope_bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ void unpack8(uint4 w, float (&x)[8]) {
  const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = rope_bf16_lo(a[i]);
    x[2 * i + 1] = rope_bf16_hi(a[i]);
  }
}

__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  uint32_t a[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    a[i] = static_cast<uint32_t>(float_to_bf16_bits(x[2 * i])) |
           (static_cast<uint32_t>(float_to_bf16_bits(x[2 * i + 1])) << 16);
  return make_uint4(a[0], a[1], a[2], a[3]);
}

// Sum over the 16 lanes of a DPP row, in every lane.
template <int CTRL>
__device__ __forceinline__ float rope_dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float row_sum16(float v) {
  v = rope_dpp_add<0xB1>(v);   // quad_perm [1,0,3,2]
  v = rope_dpp_add<0x4E>(v);   // quad_perm [2,3,0,1]
  v = rope_dpp_add<0x141>(v);  // row_half_mirror
  return rope_dpp_add<0x140>(v);  // row_mirror
}

// cos and sin of position * inv_freq.  The angle is formed in 64 bits and reduced there to
// a fraction of a turn (a position of 10^6 times a frequency of 1 has lost 5 bits of its
// fraction in 32), then 32 bits hold the fraction to 2^-25 of a turn.
__device__ __forceinline__ float2 rope_cos_sin(int position, double inv_freq) {
  const double turns = static_cast<double>(position) * (inv_freq * 0.15915494309189535);  // 1 / (2 pi)
  const float f = static_cast<float>(turns - rint(turns));
  float s, c;
  sincospif(2.f * f, &s, &c);
  return make_float2(c, s);
}

// One head row, dimensions 8 col .. 8 col + 7 in x (bias already added): x / sqrt(mean x^2
// + eps) * w if `w` is not null, then the rotation of the first `rot` dimensions (a
// multiple of 16).  cs: cos and sin of the rot / 2 frequencies.  Every lane of a row's 16 calls
// it.
__device__ __forceinline__ void rope_row(float (&x)[8], int col, const uint16_t* w, float eps, int rot, int interleaved,
                                         const float2* cs) {
  if (w) {
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sq += x[i] * x[i];
    const float r = 1.f / sqrtf(row_sum16(sq) * (1.f / kRopeD) + eps);
    float wf[8];
    unpack8(*reinterpret_cast<const uint4*>(w + 8 * col), wf);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * wf[i];
  }
  const int chunks = rot / 8;  // lanes that hold rotated dimensions
  if (interleaved) {
    if (col < chunks) {
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const float2 t = cs[4 * col + p];
        const float a = x[2 * p], b = x[2 * p + 1];
        x[2 * p] = a * t.x - b * t.y;
        x[2 * p + 1] = b * t.x + a * t.y;
      }
    }
  } else if (rot) {
    // pairs (d, d + rot / 2): the partner's dimensions are rot / 16 lanes away
    const int h = chunks / 2;
    const bool first = col < h;
    const int lane = threadIdx.x % kWave;
    const int from = col < chunks ? (first ? lane + h : lane - h) : lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float other = __shfl(x[i], from);
      if (col < chunks) {
        const float2 t = cs[8 * (first ? col : col - h) + i];
        x[i] = first ? x[i] * t.x - other * t.y : x[i] * t.x + other * t.y;
      }
    }
  }
}

}  // namespace subspec
