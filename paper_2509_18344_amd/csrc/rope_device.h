// Norm and position rotation of one head row, 16 lanes of 8 dimensions, and the rows'
// packing that the 4-bit cache's kernels use too.
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

// What a lane needs of its token's angles: for its 8 dimensions x the rotated value is
// x cos + partner sin, where the partner's sign is in sin.
struct RopeTurn {
  float c[8], s[8];
};

// cs: cos and sin of the rot / 2 frequencies.  Pairs are (d, d + rot / 2), the partner rot / 16
// lanes away, or (interleaved) neighbours in the lane.  Lanes past `rot` have no turn (rope_rotate
// leaves them alone: a turn by nothing would make NaN of infinities).
__device__ __forceinline__ RopeTurn rope_turn(int col, int rot, int interleaved, const float2* cs) {
  RopeTurn t;
  const int chunks = rot / 8, h = chunks / 2;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool turned = col < chunks;
    const bool first = interleaved ? i % 2 == 0 : col < h;
    const int f = interleaved ? 4 * col + i / 2 : 8 * (first ? col : col - h) + i;
    const float2 v = cs[turned ? f : 0];
    t.c[i] = turned ? v.x : 1.f;
    t.s[i] = turned ? (first ? -v.y : v.y) : 0.f;
  }
  return t;
}

// x / sqrt(mean x^2 + eps) * w over a head row, 16 lanes of 8 dimensions; w: this lane's weights.
__device__ __forceinline__ void rope_norm(float (&x)[8], const float (&w)[8], float eps) {
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sq = __builtin_fmaf(x[i], x[i], sq);
  const float r = rsqrtf(row_sum16(sq) * (1.f / kRopeD) + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
}

// The rotation of a head row; the dimensions past `rot`, whole lanes, stay as they are.  FULL: all 128
// dimensions in pairs (d, d + 64), whose partner is eight lanes away in the row of 16 (a DPP move
// instead of one through LDS).
template <bool FULL>
__device__ __forceinline__ void rope_rotate(float (&x)[8], int col, int rot, int interleaved, const RopeTurn& t) {
  float other[8];
  if constexpr (FULL) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      other[i] = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x[i]), 0x128, 0xF, 0xF, true));  // row_ror:8
  } else if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) other[i] = x[i ^ 1];
  } else {
    const int chunks = rot / 8, h = chunks / 2, lane = threadIdx.x % kWave;
    const int from = col < chunks ? (col < h ? lane + h : lane - h) : lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) other[i] = __shfl(x[i], from);
  }
  const bool turned = FULL || 8 * col < rot;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = turned ? __builtin_fmaf(x[i], t.c[i], other[i] * t.s[i]) : x[i];
}

}  // namespace subspec
