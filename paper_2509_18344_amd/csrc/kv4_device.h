// The key/value cache held in 4 bits: a position's row into its tile.
//
// A row of 128 dimensions is stored per group of 64 or 128 dimensions as
//   m = fp16(min x), s = fp16((max x - min x) / 15), c = clamp(rint((x - m) / s), 0, 15)
// (s = 0: c = 0) and stands for m + s c.  The layout of a tile of 32 positions is
// declared in include/subspec.h; its two halves serve the two products of attention: keys
// as rows of dimensions (what K Q^T contracts), values as rows of positions (what P V
// contracts), each as the matrix instruction's operand in registers, so that attention
// moves no code between lanes.
#pragma once

#include "device_common.h"
#include "kernels_kv4.h"
#include "rope_device.h"

namespace subspec {

// (x - m) / s correctly rounded, so that a tie of the rounding to a code falls as in exact
// arithmetic: the product with the rounded reciprocal is off by an ulp or two, one step with
// the residual (exact in an fma) corrects it.
__device__ __forceinline__ float kv4_quotient(float a, float s, float inv) {
  const float q = a * inv;
  return __builtin_fmaf(__builtin_fmaf(-q, s, a), inv, q);
}

// min (max) over the 8 or 16 lanes that hold a group of dimensions, in every lane
template <int CTRL>
__device__ __forceinline__ float kv4_dpp(float v) {
  const int b = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CTRL, 0xF, 0xF, false));
}
template <int G>
__device__ __forceinline__ void kv4_range(float& lo, float& hi) {
  lo = fminf(lo, kv4_dpp<0xB1>(lo));  // quad_perm [1,0,3,2]
  hi = fmaxf(hi, kv4_dpp<0xB1>(hi));
  lo = fminf(lo, kv4_dpp<0x4E>(lo));  // quad_perm [2,3,0,1]
  hi = fmaxf(hi, kv4_dpp<0x4E>(hi));
  lo = fminf(lo, kv4_dpp<0x141>(lo));  // row_half_mirror
  hi = fmaxf(hi, kv4_dpp<0x141>(hi));
  if constexpr (G == 1) {
    lo = fminf(lo, kv4_dpp<0x140>(lo));  // row_mirror
    hi = fmaxf(hi, kv4_dpp<0x140>(hi));
  }
}

struct Kv4Meta {
  _Float16 s, m;
};

// The group's scale and minimum and this lane's 8 codes as bytes (dimension 8 col + i in
// byte i).  NaN counts as 0 and a value past fp16's range as its largest.
template <int G>
__device__ __forceinline__ uint2 kv4_quantize(float (&x)[8], Kv4Meta& meta) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] == x[i] ? fminf(fmaxf(x[i], -65504.f), 65504.f) : 0.f;
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
  }
  kv4_range<G>(lo, hi);
  meta.m = static_cast<_Float16>(lo);
  meta.s = static_cast<_Float16>((hi - lo) / 15.f);
  const float m = static_cast<float>(meta.m), s = static_cast<float>(meta.s);
  const float inv = s > 0.f ? 1.f / s : 0.f;
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = fminf(fmaxf(rintf(kv4_quotient(x[i] - m, s, inv)), 0.f), 15.f);
    w[i / 4] |= static_cast<uint32_t>(c) << (8 * (i % 4));
  }
  return make_uint2(w[0], w[1]);
}

// Byte offsets within a tile.  Position w = 0 .. 31, dimension chunk col (8 dimensions).
__device__ __forceinline__ int kv4_key_word(int w, int col) {  // its 8 codes of a key
  return (w / 16) * 1024 + (16 * (col % 4) + w % 16) * 16 + 4 * (col / 4);
}
__device__ __forceinline__ int kv4_slot(int w) { return (w & 3) + 4 * (w / 16); }  // within a quarter
template <int G>
__device__ __forceinline__ int kv4_meta(int w, int g) {  // its scale; the minimum 16 bytes on
  return kKv4CodeBytes + (((w % 16) / 4 * G + g) * 2) * 16 + 2 * kv4_slot(w);
}

constexpr int kKv4LdsRow = kKv4D + 16;  // bytes of a position's codes in LDS

// One tile of one head: 256 threads write the positions that are live.  `load(w, col, value, x)`
// puts dimensions 8 col .. of position w's key or value into x and says whether the position
// is written; the 16 lanes of a row agree.  Codes of other positions keep their bits: a
// value's word holds the codes of 8 positions, so a tile belongs to one workgroup and a
// word to one thread, which merges.
template <int G, typename Load>
__device__ __forceinline__ void kv4_store_tile(uint8_t* kt, uint8_t* vt, uint8_t (*lds)[kKv4LdsRow], uint32_t* live_bits,
                                               Load load) {
  const int col = threadIdx.x % 16, r = threadIdx.x / 16;
  if (threadIdx.x == 0) *live_bits = 0;
  __syncthreads();
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int w = 16 * b + r;
    float x[8];
    Kv4Meta meta;
    if (load(w, col, false, x)) {
      const uint2 c = kv4_quantize<G>(x, meta);
      // byte i -> nibble: even dimensions in the low half word, odd ones in the high
      const uint32_t e = (c.x & 0xFu) | ((c.x >> 12) & 0xF0u) | ((c.y & 0xFu) << 8) | ((c.y >> 4) & 0xF000u);
      const uint32_t o = ((c.x >> 8) & 0xFu) | ((c.x >> 20) & 0xF0u) | (c.y & 0xF00u) | ((c.y >> 12) & 0xF000u);
      *reinterpret_cast<uint32_t*>(kt + kv4_key_word(w, col)) = e | (o << 16);
      if (col % (16 / G) == 0) {
        const int at = kv4_meta<G>(w, col / (16 / G));
        *reinterpret_cast<_Float16*>(kt + at) = meta.s;
        *reinterpret_cast<_Float16*>(kt + at + 16) = meta.m;
      }
    }
    if (load(w, col, true, x)) {
      const uint2 c = kv4_quantize<G>(x, meta);
      *reinterpret_cast<uint2*>(&lds[w][8 * col]) = c;
      if (col % (16 / G) == 0) {
        const int at = kv4_meta<G>(w, col / (16 / G));
        *reinterpret_cast<_Float16*>(vt + at) = meta.s;
        *reinterpret_cast<_Float16*>(vt + at + 16) = meta.m;
      }
      if (col == 0) atomicOr(live_bits, 1u << w);
    }
  }
  __syncthreads();
  const uint32_t live = *live_bits;
  if (threadIdx.x < 128) {
    const int half = threadIdx.x / 64, lane = threadIdx.x % 64;
    const int vc = lane % 16, quarter = lane / 16;
    // the quarter's 8 positions: 4 quarter + 0..3 and 16 + 4 quarter + 0..3
    uint32_t keep = 0;  // bits of a word that stay
    uint32_t word[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int w = 4 * quarter + (e & 3) + 16 * (e >> 2);
      const int shift = 4 * (e / 2) + 16 * (e % 2);
      if ((live >> w) & 1u) {
#pragma unroll
        for (int d = 0; d < 4; ++d) word[d] |= static_cast<uint32_t>(lds[w][64 * half + 16 * d + vc]) << shift;
      } else {
        keep |= 0xFu << shift;
      }
    }
    uint4* p = reinterpret_cast<uint4*>(vt + half * 1024 + lane * 16);
    if (keep != ~0u) {
      uint4 old = make_uint4(0, 0, 0, 0);
      if (keep) old = *p;
      *p = make_uint4(word[0] | (old.x & keep), word[1] | (old.y & keep), word[2] | (old.z & keep),
                      word[3] | (old.w & keep));
    }
  }
}

}  // namespace subspec
