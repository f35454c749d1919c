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

// 1 / s correctly rounded: the hardware's reciprocal (1 ulp) and one Newton step; checked for every
// significand of an fp16 s.
__device__ __forceinline__ float kv4_reciprocal(float s) {
  const float y = __builtin_amdgcn_rcpf(s);
  return __builtin_fmaf(__builtin_fmaf(-s, y, 1.f), y, y);
}

// a / s correctly rounded, given 1 / s, so that a tie of the rounding to a code falls as in
// exact arithmetic: the product is off by an ulp or two, one step with its residual (exact
// in an fma) corrects it.
__device__ __forceinline__ float kv4_quotient(float a, float s, float inv) {
  const float q = a * inv;
  return __builtin_fmaf(__builtin_fmaf(-q, s, a), inv, q);
}

// min and max over the 8 or 16 lanes that hold a group of dimensions, in every lane
template <int CTRL>
__device__ __forceinline__ int kv4_dpp(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true);
}
template <int G>
__device__ __forceinline__ void kv4_range(int& lo, int& hi) {
  lo = min(lo, kv4_dpp<0xB1>(lo));  // quad_perm [1,0,3,2]
  hi = max(hi, kv4_dpp<0xB1>(hi));
  lo = min(lo, kv4_dpp<0x4E>(lo));  // quad_perm [2,3,0,1]
  hi = max(hi, kv4_dpp<0x4E>(hi));
  lo = min(lo, kv4_dpp<0x141>(lo));  // row_half_mirror
  hi = max(hi, kv4_dpp<0x141>(hi));
  if constexpr (G == 1) {
    lo = min(lo, kv4_dpp<0x140>(lo));  // row_mirror
    hi = max(hi, kv4_dpp<0x140>(hi));
  }
}

// Numbers in an integer form that orders them (-0 below 0); the same function turns it back.
__device__ __forceinline__ int kv4_order(int bits) { return bits ^ ((bits >> 31) & 0x7FFFFFFF); }

typedef int16_t i16x2_t __attribute__((ext_vector_type(2)));

struct Kv4Meta {
  _Float16 s, m;
};

// The group's scale and minimum and this lane's 8 codes as bytes (dimension 8 col + i in
// byte i), of 8 bf16 values.  NaN counts as 0 and a value past fp16's range as its largest.
template <int G>
__device__ __forceinline__ uint2 kv4_quantize(uint4 raw, Kv4Meta& meta) {
  float x[8];
  unpack8(raw, x);
  // the range of pairs of bf16 values in their ordered 16-bit form (half the instructions of floats')
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  i16x2_t plo, phi;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const i16x2_t v = __builtin_bit_cast(i16x2_t, w[i]);
    const i16x2_t k = v ^ ((v >> 15) & static_cast<int16_t>(0x7FFF));
    plo = i == 0 ? k : __builtin_elementwise_min(plo, k);
    phi = i == 0 ? k : __builtin_elementwise_max(phi, k);
  }
  int ilo = min(static_cast<int>(plo[0]), static_cast<int>(plo[1])), ihi = max(static_cast<int>(phi[0]), static_cast<int>(phi[1]));
  kv4_range<G>(ilo, ihi);
  float lo = __uint_as_float(static_cast<uint32_t>(ilo ^ ((ilo >> 31) & 0x7FFF)) << 16);
  float hi = __uint_as_float(static_cast<uint32_t>(ihi ^ ((ihi >> 31) & 0x7FFF)) << 16);
  // 0x477F is the largest bf16 within fp16's range; larger ones, infinities and NaN lie past it
  if (__builtin_amdgcn_ballot_w64(ihi > 0x477F || ilo < -0x4780)) {
    int flo = 0x7FFFFFFF, fhi = -0x7FFFFFFF;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = x[i] == x[i] ? fminf(fmaxf(x[i], -65504.f), 65504.f) : 0.f;
      const int k = kv4_order(__float_as_int(x[i]));
      flo = min(flo, k);
      fhi = max(fhi, k);
    }
    kv4_range<G>(flo, fhi);
    lo = __int_as_float(kv4_order(flo));
    hi = __int_as_float(kv4_order(fhi));
  }
  meta.m = static_cast<_Float16>(lo);
  meta.s = static_cast<_Float16>(kv4_quotient(hi - lo, 15.f, 0x1.111112p-4f));  // 1 / 15 rounded
  const float m = static_cast<float>(meta.m), s = static_cast<float>(meta.s);
  const float inv = s > 0.f ? kv4_reciprocal(s) : 0.f;
  uint32_t code[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)  // (the conversion takes negative numbers to 0)
    code[i / 4] = __builtin_amdgcn_cvt_pk_u8_f32(fminf(rintf(kv4_quotient(x[i] - m, s, inv)), 15.f), i % 4, code[i / 4]);
  return make_uint2(code[0], code[1]);
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

struct Kv4TileLds {
  alignas(16) uint8_t key[kv4_tile_bytes(2)];    // the tiles as they are in memory
  alignas(16) uint8_t value[kv4_tile_bytes(2)];
  alignas(16) uint8_t code[kKv4Tile][kKv4D + 16];  // the values' codes, one a byte
  uint32_t live;                                 // positions that are written
};

// One tile of one head: 256 threads write the positions that are live.  `load(w, col, value, x)`
// puts dimensions 8 col .. of position w's key or value (bf16) into x and says whether the
// position is written; the 16 lanes of a row agree.  The tile is put together in LDS and written
// 16 bytes a thread; where only some positions are live, their parts of it, and words that
// hold codes of other positions too (a value's hold 8) are merged with what they held: a
// tile belongs to one workgroup and a word to one thread.
template <int G, typename Load>
__device__ __forceinline__ void kv4_store_tile(uint8_t* kt, uint8_t* vt, Kv4TileLds& L, Load load) {
  const int t = threadIdx.x, col = t % 16, r = t / 16;
  if (t == 0) L.live = 0;
  uint4 x[2][2];
  bool live[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {  // all of the workgroup's rows in flight
    live[b] = load(16 * b + r, col, false, x[b][0]);
    (void)load(16 * b + r, col, true, x[b][1]);
  }
  __syncthreads();
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int w = 16 * b + r;
    if (!live[b]) continue;
    Kv4Meta meta;
    const bool head = col % (16 / G) == 0;
    const int at = kv4_meta<G>(w, col / (16 / G));
    uint2 c = kv4_quantize<G>(x[b][0], meta);
    // byte i -> nibble: even dimensions in the low half word, odd ones in the high
    const uint32_t p = c.x | (c.x >> 12), q = c.y | (c.y >> 12);  // bytes 0, 1: codes 0, 1 and 2, 3 above them
    *reinterpret_cast<uint32_t*>(L.key + kv4_key_word(w, col)) = __builtin_amdgcn_perm(q, p, 0x05010400u);
    if (head) {
      *reinterpret_cast<_Float16*>(L.key + at) = meta.s;
      *reinterpret_cast<_Float16*>(L.key + at + 16) = meta.m;
    }
    c = kv4_quantize<G>(x[b][1], meta);
    *reinterpret_cast<uint2*>(&L.code[w][8 * col]) = c;
    if (head) {
      *reinterpret_cast<_Float16*>(L.value + at) = meta.s;
      *reinterpret_cast<_Float16*>(L.value + at + 16) = meta.m;
    }
    if (col == 0) atomicOr(&L.live, 1u << w);
  }
  __syncthreads();
  const uint32_t all = L.live;
  if (t < 128) {
    // four adjacent columns of one of a lane's words: dimensions 64 half + 16 dl + vc .. + 3
    const int vc = 4 * (t % 4), quarter = t / 4 % 4, dl = t / 16 % 4, half = t / 64;
    // the quarter's 8 positions, 4 quarter + 0..3 and 16 + 4 quarter + 0..3 (codes of positions that
    // are not live are whatever LDS held)
    uint32_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      c[e] = *reinterpret_cast<const uint32_t*>(&L.code[4 * quarter + (e & 3) + 16 * (e >> 2)][64 * half + 16 * dl + vc]) & 0x0F0F0F0Fu;
    // bytes of pairs of nibbles, then the four words out of their bytes
    const uint32_t b0 = c[0] | (c[2] << 4), b1 = c[4] | (c[6] << 4), b2 = c[1] | (c[3] << 4), b3 = c[5] | (c[7] << 4);
    const uint32_t lo01 = __builtin_amdgcn_perm(b1, b0, 0x05010400u), hi01 = __builtin_amdgcn_perm(b1, b0, 0x07030602u);
    const uint32_t lo23 = __builtin_amdgcn_perm(b3, b2, 0x05010400u), hi23 = __builtin_amdgcn_perm(b3, b2, 0x07030602u);
    uint32_t* p = reinterpret_cast<uint32_t*>(L.value + half * 1024 + (16 * quarter + vc) * 16 + 4 * dl);
    p[0] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u);
    p[4] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
    p[8] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100u);
    p[12] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302u);
  }
  __syncthreads();
  constexpr int kPieces = kv4_tile_bytes(G) / 16;
  for (int i = t; i < 2 * kPieces; i += 256) {
    const bool value = i >= kPieces;
    const int at = value ? i - kPieces : i;
    uint4 w = *reinterpret_cast<const uint4*>((value ? L.value : L.key) + 16 * at);
    uint4* dst = reinterpret_cast<uint4*>(value ? vt : kt) + at;
    if (all != ~0u) {
      // which bits of the piece belong to live positions: a key's codes to one, a value's word
      // to its quarter's 8, 4 bits each, of scales or minima 16 bits each
      uint32_t mask[4];
      if (!value && at < kKv4CodeBytes / 16) {
        const bool on = (all >> (16 * (at / 64) + at % 16)) & 1u;
        mask[0] = mask[1] = mask[2] = mask[3] = on ? ~0u : 0u;
      } else {
        const int quarter = at < kKv4CodeBytes / 16 ? at % 64 / 16 : (at - kKv4CodeBytes / 16) / (2 * G);
        const uint32_t mine = ((all >> (4 * quarter)) & 0xFu) | (((all >> (16 + 4 * quarter)) & 0xFu) << 4);
        if (at < kKv4CodeBytes / 16) {
          uint32_t m = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if ((mine >> e) & 1u) m |= 0xFu << (4 * (e / 2) + 16 * (e % 2));
          mask[0] = mask[1] = mask[2] = mask[3] = m;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            mask[e] = ((mine >> (2 * e)) & 1u ? 0xFFFFu : 0u) | ((mine >> (2 * e + 1)) & 1u ? 0xFFFF0000u : 0u);
        }
      }
      if (!(mask[0] | mask[1] | mask[2] | mask[3])) continue;
      const uint4 old = *dst;
      w.x = (w.x & mask[0]) | (old.x & ~mask[0]);
      w.y = (w.y & mask[1]) | (old.y & ~mask[1]);
      w.z = (w.z & mask[2]) | (old.z & ~mask[2]);
      w.w = (w.w & mask[3]) | (old.w & ~mask[3]);
    }
    *dst = w;
  }
}

}  // namespace subspec
