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

// a / s correctly rounded, so that a tie of the rounding to a code falls as in exact arithmetic, given
// 1 / s as the sum of two numbers: the hardware's reciprocal and what it leaves.  With a of 24 bits
// and s of 11 no quotient lies nearer to the middle of two numbers than 2^-36 of itself, the
// sum is within 2^-45 of 1 / s and the fma rounds once.
struct Kv4Reciprocal {
  float hi, lo;
};
__device__ __forceinline__ Kv4Reciprocal kv4_reciprocal(float s) {
  const float hi = __builtin_amdgcn_rcpf(s);
  return {hi, __builtin_fmaf(-s, hi, 1.f) * hi};
}
__device__ __forceinline__ float kv4_quotient(float a, Kv4Reciprocal r) { return __builtin_fmaf(a, r.hi, a * r.lo); }

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

struct Kv4Meta {
  _Float16 s, m;
};

// The group's scale and minimum and this lane's 8 codes as bytes (dimension 8 col + i in
// byte i), of 8 bf16 values.  NaN counts as 0 and a value past fp16's range as its largest.
template <int G>
__device__ __forceinline__ uint2 kv4_quantize(uint4 raw, Kv4Meta& meta) {
  float x[8];
  unpack8(raw, x);
  float lo = x[0], hi = x[0];  // NaN wins, -0 lies below 0
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = __builtin_elementwise_minimum(lo, x[i]);
    hi = __builtin_elementwise_maximum(hi, x[i]);
  }
  int ilo = kv4_order(__float_as_int(lo)), ihi = kv4_order(__float_as_int(hi));
  kv4_range<G>(ilo, ihi);
  // past fp16's range (as the bounds' next bf16 values are), infinities and NaN
  if (__builtin_amdgcn_ballot_w64(ihi >= 0x47800000 || ilo <= kv4_order(static_cast<int>(0xC7800000u)))) {
    ilo = 0x7FFFFFFF;
    ihi = -0x7FFFFFFF;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = x[i] == x[i] ? fminf(fmaxf(x[i], -65504.f), 65504.f) : 0.f;
      const int k = kv4_order(__float_as_int(x[i]));
      ilo = min(ilo, k);
      ihi = max(ihi, k);
    }
    kv4_range<G>(ilo, ihi);
  }
  lo = __int_as_float(kv4_order(ilo));
  hi = __int_as_float(kv4_order(ihi));
  meta.m = static_cast<_Float16>(lo);
  constexpr Kv4Reciprocal kFifteenth{0x1.111112p-4f, -0x1.dddddep-29f};
  meta.s = static_cast<_Float16>(kv4_quotient(hi - lo, kFifteenth));
  const float m = static_cast<float>(meta.m), s = static_cast<float>(meta.s);
  const Kv4Reciprocal r = kv4_reciprocal(s);
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = kv4_quotient(x[i] - m, r);
  // A scale that fp16 holds to 11 bits keeps every quotient below 15.5; below, and for 0, they may be anything.
  if (__builtin_amdgcn_ballot_w64(s < 0x1p-14f)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = s == 0.f ? 0.f : fminf(q[i], 15.f);
  }
  uint32_t code[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)  // (the conversion rounds to nearest-even and takes negative numbers to 0)
    code[i / 4] = __builtin_amdgcn_cvt_pk_u8_f32(q[i], i % 4, code[i / 4]);
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
  alignas(16) uint32_t live[8];                    // positions that are written: 4 i + bit
};

// One tile of one head: 256 threads write the positions that are live.  `source(w)` is where
// position w's row of 128 starts in k and v (bf16), or negative where the position is not written.  The tile is put together in LDS and written
// 16 bytes a thread; where only some positions are live, their parts of it, and words that
// hold codes of other positions too (a value's hold 8) are merged with what they held: a
// tile belongs to one workgroup and a word to one thread.
template <int G, typename Source>
__device__ __forceinline__ void kv4_store_tile(uint8_t* kt, uint8_t* vt, const uint16_t* k, const uint16_t* v, Kv4TileLds& L,
                                               Source source) {
  const int t = threadIdx.x, col = t % 16, r = t / 16;
  uint4 x[2][2];
  bool live[2];
  const long long at[2] = {source(r), source(16 + r)};
#pragma unroll
  for (int b = 0; b < 2; ++b) {  // all of the workgroup's rows in flight
    live[b] = at[b] >= 0;
    if (live[b]) {
      x[b][0] = *reinterpret_cast<const uint4*>(k + at[b] + 8 * col);
      x[b][1] = *reinterpret_cast<const uint4*>(v + at[b] + 8 * col);
    }
  }
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int w = 16 * b + r;
    // a wavefront's four rows
    const unsigned long long rows = __builtin_amdgcn_ballot_w64(live[b]) & 0x0001000100010001ull;
    if (t % kWave == 0) L.live[4 * b + t / kWave] = static_cast<uint32_t>((rows * 0x0001000200040008ull) >> 48) & 0xFu;
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
  }
  __syncthreads();
  uint32_t all = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) all |= L.live[i] << (4 * i);
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
