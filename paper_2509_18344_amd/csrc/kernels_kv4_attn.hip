// Tree attention over the key/value cache held in 4 bits.
//
// M new tree tokens with Hq query heads grouped onto Hkv key/value heads attend, with
// scores q.k scale and a softmax, to the P committed positions and to the tree positions
// P + j (j < T + M) that their mask rows allow.  A position's key is m_g + s_g c per group g
// of dimensions (fp16 minimum m, scale s, codes c of 4 bits), its value the same with its own.
//
// Neither product forms those numbers.  With x the sum over a group g of dimensions,
//   q.k = sum_g s_g (q.c)_g + m_g (sum q)_g
//   sum_j p_j v_j = sum_j (p_j s_jg) c_j + sum_j p_j m_jg
// where q.c and (p s) c are fp16 matrix products: a code in a byte is an fp8 number, so unpacking a word
// of eight is two ands, a shift and four conversions.  bf16 q fits fp16 once its row is scaled by a power
// of two.  The sum of the weights and the minima's share come from one more product against rows of
// ones and of minima, so that the numerator's and the denominator's weights are the same numbers.
//
// A weight p, and its product with the scale, go into the products as sums of two fp16 numbers each:
// the number rounded and what the rounding left (of the product an fma returns it exactly), 21 bits
// and more.  With one number each and the codes left as subnormals a call at 131138 positions took 42.8 us
// instead of 49.4 and one at 2336 10.8 instead of 11.0, but 8 to 24 % of the outputs were not the bf16
// number next to the exact one, where now 0.1 to 0.2 % are not, as of a plain form in 32 bits.
// Everything else is exact or in 32 bits.  fp16 spans 2^-24 .. 65504, so weights are
// relative to a reference that covers score + log2 of the tile's largest scale where that passes 1: p
// and p s stay below 2^15, and the heaviest position's p is at least 2^8 while scales lie below 1.
// Scales below 1 are raised by the power of two that brings the largest of the wavefront's so far to
// 1/2 .. 1, and its sums lowered when a larger one comes: values of any size keep the same bits.  The
// reference moves only when a weight would pass 2^14 (a few times in a row's life), so most
// tiles scale nothing.
//
// Kernel 1 (k_kv4_partial): workgroup (range s, key/value head g); its wavefronts take the
// range's tiles of 32 positions in turn, each for up to two tiles of 16 query rows (row =
// local head * M + token; with more rows two or four wavefronts share a tile of positions).
// The cache holds both operands in register order: no code moves between lanes, and no wavefront
// waits for another until the end, when their outputs are scaled to a common reference and added in
// wavefront order.
//   S^T = K Q^T     16x16x32 fp16, 2 blocks of 16 positions x 4 steps of 32 dimensions
//   O^T += V^T P^T  16x16x32 fp16, 8 tiles of 16 dimensions; P is in the operand layout
//                   where the scores are
// Kernel 2 (k_kv4_combine) combines the ranges in a fixed order; a single range writes the
// output itself.
//
// Measured (a call, both kernels): 131138 positions of 8 heads in groups of 64, 30 query rows a head:
// 151 MB of cache in 49.4 us, 3.1 TB/s.  The first kernel takes 46 to 49 us, 28 with nothing but its loads:
// unpacking, softmax and products bound it (508 vector instructions a tile of 32 positions x 32 query rows, 52 of
// them matrix products; the vector ALUs issue two thirds of the time).  8407 positions of 8 heads in groups of
// 128, 64 rows a head: 9 MB in 17.8 us, a chain of the launch with the first loads (3.4 us), five tiles a
// wavefront, the merge (1 to 2.5) and the second kernel (2.5 to 3.3).  2336 positions of 4 heads, 42 rows:
// 10.9 us, the same chain with one tile; 16385 of 8 heads with 5 rows 11.0 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device_common.h"
#include "kernels_kv4.h"

namespace subspec {

namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

// Visibility of the 32 positions key0 .. for one query row (bit k: key0 + k): committed
// positions always, tree positions P + j by bit j of the row's mask (its W words in device
// memory), nothing at or past `end`.
__device__ __forceinline__ uint32_t kv4_visibility(const uint32_t* row_mask, int W, int P, int key0, int end) {
  uint32_t vis;
  if (key0 + kKv4Tile <= P) {
    vis = ~0u;
  } else if (key0 >= P) {
    const int jb = key0 - P, w = jb >> 5, sh = jb & 31;
    const uint64_t lo = row_mask[w];
    const uint64_t hi = w + 1 < W ? row_mask[w + 1] : 0u;
    vis = static_cast<uint32_t>(((hi << 32) | lo) >> sh);
  } else {  // the tile straddles P: committed positions, then the first tree bits
    const int n = P - key0;  // 1 .. 31
    vis = (row_mask[0] << n) | ((1u << n) - 1u);
  }
  const int live = end - key0;  // >= 1
  return live >= kKv4Tile ? vis : vis & ((1u << live) - 1u);
}

// One lane's share of a tile: codes, and of its quarter's 8 positions (4 quarter + r and 16 +
// 4 quarter + r) the scales per group; the keys' minima the same; of the values' minima one
// row of the auxiliary product's operand (group 0 in the lanes of column 1, group 1 in column 2).
template <int G>
struct Kv4Keys {
  u32x4_t c[2], s[G], m[G];
};
template <int G>
struct Kv4Values {
  u32x4_t c[2], s[G], m;
};

template <int G>
__device__ __forceinline__ void kv4_load(const uint8_t* tile, int lane, Kv4Keys<G>& r) {
#pragma unroll
  for (int u = 0; u < 2; ++u) r.c[u] = *reinterpret_cast<const u32x4_t*>(tile + u * 1024 + lane * 16);
  const uint8_t* meta = tile + kKv4CodeBytes + (lane / 16) * (32 * G);
#pragma unroll
  for (int g = 0; g < G; ++g) {
    r.s[g] = *reinterpret_cast<const u32x4_t*>(meta + 32 * g);
    r.m[g] = *reinterpret_cast<const u32x4_t*>(meta + 32 * g + 16);
  }
}

template <int G>
__device__ __forceinline__ void kv4_load(const uint8_t* tile, int lane, Kv4Values<G>& r) {
  const uint8_t* meta = tile + kKv4CodeBytes + (lane / 16) * (32 * G);
#pragma unroll
  for (int g = 0; g < G; ++g) r.s[g] = *reinterpret_cast<const u32x4_t*>(meta + 32 * g);
  r.m = *reinterpret_cast<const u32x4_t*>(meta + (lane % 16 == 2 ? 32 * (G - 1) : 0) + 16);
#pragma unroll
  for (int u = 0; u < 2; ++u) r.c[u] = *reinterpret_cast<const u32x4_t*>(tile + u * 1024 + lane * 16);
}

// Counts the registers of `r` as written.  Where a branch leaves them alone because nothing
// reads them again, the compiler may otherwise take them as undefined on that path, and has then
// dropped parts of them on the other (three of four registers of a tile's minima).
template <int G>
__device__ __forceinline__ void kv4_keep(Kv4Values<G>& r) {
#pragma unroll
  for (int u = 0; u < 2; ++u) asm volatile("" : "+v"(r.c[u]));
#pragma unroll
  for (int g = 0; g < G; ++g) asm volatile("" : "+v"(r.s[g]));
  asm volatile("" : "+v"(r.m));
}
template <int G>
__device__ __forceinline__ void kv4_keep(Kv4Keys<G>& r) {
#pragma unroll
  for (int u = 0; u < 2; ++u) asm volatile("" : "+v"(r.c[u]));
#pragma unroll
  for (int g = 0; g < G; ++g) asm volatile("" : "+v"(r.s[g]), "+v"(r.m[g]));
}

__device__ __forceinline__ uint32_t kv4_pack(float lo, float hi) {
  return static_cast<uint32_t>(float_to_bf16_bits(lo)) | (static_cast<uint32_t>(float_to_bf16_bits(hi)) << 16);
}

// Eight codes of a word as fp16 numbers 2^-9 c, code e of the word at place kv4_place(e): a code in a byte is
// the fp8 number (three bits of mantissa, exponents from 2^-6) 2^-9 c, subnormal below 8 and normal from 8
// on, and the conversion takes two bytes at a time.  Masked alone, a code is the mantissa of an fp16
// subnormal, which the matrix instruction takes as it is; but it aligns a group of eight products by
// the exponents of their operands, a subnormal's counting as 2^-14, and drops what lies 24 bits below the
// largest: of that all but 14 bits would be the leading zeros of the codes, and a weight of 2^-14 of
// its neighbour's, or a dimension of q beside a large one, was lost.
__device__ __forceinline__ f16x8_t kv4_codes(uint32_t d) {
  const uint32_t even = d & 0x0F0F0F0Fu, odd = (d >> 4) & 0x0F0F0F0Fu;  // codes 0, 4, 1, 5 and 2, 6, 3, 7
  return __builtin_bit_cast(f16x8_t, u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(even, 1.f, false)),
                                             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(even, 1.f, true)),
                                             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(odd, 1.f, false)),
                                             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(odd, 1.f, true))});
}
constexpr int kv4_place(int e) { return 2 * (e % 4) + e / 4; }

// Halves in the order of codes (a position's scales or minima) to those places.
__device__ __forceinline__ u32x4_t kv4_to_places(u32x4_t h) {
  return u32x4_t{__builtin_amdgcn_perm(h[2], h[0], 0x05040100u), __builtin_amdgcn_perm(h[2], h[0], 0x07060302u),
                 __builtin_amdgcn_perm(h[3], h[1], 0x05040100u), __builtin_amdgcn_perm(h[3], h[1], 0x07060302u)};
}

// One load straight into LDS: lane l's SIZE bytes at base + offset (the lane's) land at byte
// dst + SIZE * l.  Written as assembly because the compiler, where it sees such loads, waits for all
// of them before it reads the ring again; it has no register result, and the ring's own waits order
// it (a wait state after the write of m0 included).  m0 is named as written, for whatever the compiler may
// keep there (it warns that m0 is not for it to allocate, which nothing asks of it).
template <int SIZE>
__device__ __forceinline__ void kv4_to_lds(const uint8_t* base, uint32_t offset, uint32_t dst) {
  if constexpr (SIZE == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(offset), "s"(base)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(dst), "v"(offset), "s"(base)
                 : "memory", "m0");
}

// The halves of a metadata word, two positions', of which bits 0 and 1 of `seen` say which stay; the
// others become zero.
__device__ __forceinline__ uint32_t kv4_seen_halves(uint32_t seen) {
  return (seen & 1u ? 0xFFFFu : 0u) | (seen & 2u ? 0xFFFF0000u : 0u);
}

// OR over the 16 lanes of a DPP row, in every lane.
template <int CTRL>
__device__ __forceinline__ uint32_t kv4_dpp_or(uint32_t v) {
  return v | static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ uint32_t kv4_row_or(uint32_t v) {
  v = kv4_dpp_or<0xB1>(v);     // quad_perm [1,0,3,2]
  v = kv4_dpp_or<0x4E>(v);     // quad_perm [2,3,0,1]
  v = kv4_dpp_or<0x141>(v);    // row_half_mirror
  return kv4_dpp_or<0x140>(v); // row_mirror
}

// A lane and its partners 16, 32 and 48 lanes away (the four quarters that share a query):
// the swaps put a row's and its neighbour's values side by side.
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2_t kv4_swap16(uint32_t v) { return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_permlane16_swap(v, v, false, false)); }
__device__ __forceinline__ u32x2_t kv4_swap32(uint32_t v) { return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_permlane32_swap(v, v, false, false)); }
__device__ __forceinline__ float kv4_cross_max(float v) {
  u32x2_t w = kv4_swap16(__float_as_uint(v));
  v = fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
  w = kv4_swap32(__float_as_uint(v));
  return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float kv4_cross_sum(float v) {
  u32x2_t w = kv4_swap16(__float_as_uint(v));
  v = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  w = kv4_swap32(__float_as_uint(v));
  return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}

// Larger of two pairs of fp16 numbers that are not negative (their bits order them).
__device__ __forceinline__ uint32_t kv4_max_halves(uint32_t a, uint32_t b) {
  const u16x2_t x = __builtin_bit_cast(u16x2_t, a), y = __builtin_bit_cast(u16x2_t, b);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}

// The largest half of the four quarters that share a column (the halves not negative).
__device__ __forceinline__ uint32_t kv4_row_max(uint32_t v) {
  u32x2_t w = kv4_swap16(v);
  w = kv4_swap32(kv4_max_halves(w[0], w[1]));
  v = kv4_max_halves(w[0], w[1]);
  return max(v & 0xFFFFu, v >> 16);
}

// -1, unknown to the compiler: the difference of an fp32 number and an fp16 one stays one fma that takes
// both as they are (otherwise a conversion and a subtraction).
__device__ __forceinline__ float kv4_minus_one() {
  float m = -1.f;
  asm("" : "+v"(m));
  return m;
}

// 2^n, n in -126 .. 127.
__device__ __forceinline__ float kv4_exp2i(int n) { return __uint_as_float(static_cast<uint32_t>(n + 127) << 23); }

// Orders a wavefront's LDS accesses to each other's words, for the compiler (the hardware keeps
// them in order).
__device__ __forceinline__ void kv4_wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// row / M for a row below 64, from 1 / M: the quotient's distance to a whole number is at least
// half of 1 / M before the 32-bit product's rounding.
__device__ __forceinline__ int kv4_row_head(int row, float inv_m) { return static_cast<int>((static_cast<float>(row) + 0.5f) * inv_m); }

// From this reference on a row's scores are rounded before the reference is taken from them.  Below,
// the rounding of the reference (2^-5) is a common factor of the row's weights.  Above, the exact
// product and the rounded reference may lie further apart than fp16's range, while fp32 holds no
// score more closely than that; the rounded ones of equal positions are equal, and the reference is
// the largest itself, so that no weight passes 1.
constexpr float kVast = 0x1p20f;

// Query rows of one wavefront (QW tiles of 16) and what it has summed for them.
template <int QW, int G>
struct Kv4Rows {
  // Per lane the query row's fragments of q times 2^(15 - e), where the row's largest value
  // lies below 2^e, as fp16 (bf16's 8 bits fit, down to 2^-29 of the largest), their sums per group times
  // 2^-9, and the factor that takes a score to log2.
  f16x8_t qf[QW][4];
  float qs[QW][G], factor[QW];
  bool live[QW];
  int qi[QW];
  float ref[QW];              // what weights are relative to: 2^(score - ref)
  f32x4_t o[QW][8], aux[QW];  // aux: in quarter 0 the sum of weights, and of weights times minima
  int field;                  // the largest fp16 exponent field of a scale so far, at most 14: o stands for 2^(14 - field) of its sums
  u32x4_t raw[QW][4];

  __device__ __forceinline__ void request(const Kv4AttnArgs& a, int g, int row0, int lane) {
#pragma unroll
    for (int t = 0; t < QW; ++t) {
      const int row = row0 + 16 * t + (lane & 15);
      live[t] = row < a.Gq * a.M;
      const int hl = live[t] ? kv4_row_head(row, a.inv_m) : 0;  // (a row past the last repeats the first)
      qi[t] = live[t] ? row - hl * a.M : 0;
      const uint16_t* q = a.q + (static_cast<size_t>(qi[t]) * a.Hq + g * a.Gq + hl) * kKv4D + 8 * (lane >> 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) raw[t][j] = *reinterpret_cast<const u32x4_t*>(q + 32 * j);
    }
  }

  __device__ __forceinline__ void begin(const Kv4AttnArgs& a) {
    field = 0;
#pragma unroll
    for (int t = 0; t < QW; ++t) {
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        raw[t][j] ^= a.q_sign;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = kv4_max_halves(top, raw[t][j][i] & 0x7FFF7FFFu);
      }
      const int e = static_cast<int>(kv4_row_max(top) >> 7) - 126;  // bf16's exponent field
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          qf[t][j][kv4_place(2 * i)] = static_cast<_Float16>(ldexpf(__uint_as_float(raw[t][j][i] << 16), 15 - e));
          qf[t][j][kv4_place(2 * i + 1)] = static_cast<_Float16>(ldexpf(__uint_as_float(raw[t][j][i] & 0xFFFF0000u), 15 - e));
        }
#pragma unroll
      for (int gg = 0; gg < G; ++gg) {
        float sum = 0.f;
#pragma unroll
        for (int j = gg * (4 / G); j < (gg + 1) * (4 / G); ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) sum += static_cast<float>(qf[t][j][i]);
        qs[t][gg] = kv4_cross_sum(sum) * 0x1p-9f;
      }
      // |x| stays below 2^31, so no score overflows; a factor of 2^95 has long left one position alone.
      factor[t] = fminf(fmaxf(ldexpf(a.scale_log2, e - 6), 0x1p-126f), 0x1p95f);
      ref[t] = -INFINITY;
      aux[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) o[t][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Scores times 2^(6 - e): lane holds positions 16u + 4 quarter + e of its query.
  __device__ __forceinline__ void scores(const Kv4Keys<G>& k, f32x4_t (&x)[QW][2]) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4_t st[QW][G];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f16x8_t kf = kv4_codes(k.c[u][j]);
#pragma unroll
        for (int t = 0; t < QW; ++t)
          st[t][j * G / 4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
              kf, qf[t][j], j % (4 / G) == 0 ? f32x4_t{0.f, 0.f, 0.f, 0.f} : st[t][j * G / 4], 0, 0, 0);
      }
#pragma unroll
      for (int t = 0; t < QW; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float y = 0.f;
#pragma unroll
          for (int gg = 0; gg < G; ++gg)
            y = __builtin_fmaf(static_cast<float>(__builtin_bit_cast(f16x8_t, k.m[gg])[4 * u + e]), qs[t][gg], y);
#pragma unroll
          for (int gg = 0; gg < G; ++gg)
            y = __builtin_fmaf(static_cast<float>(__builtin_bit_cast(f16x8_t, k.s[gg])[4 * u + e]), st[t][gg][e], y);
          x[t][u][e] = y;
        }
    }
  }

  // The tile's positions that each row sees, and (returned) that any of the wavefront's rows does.
  __device__ __forceinline__ uint32_t look(const Kv4AttnArgs& a, const uint32_t* words, int key0, int total, uint32_t (&vis)[QW]) const {
    uint32_t any = 0;
#pragma unroll
    for (int t = 0; t < QW; ++t) {
      vis[t] = live[t] ? kv4_visibility(words + qi[t] * a.W, a.W, a.P, key0, total) : 0u;
      any |= vis[t];
    }
    return kv4_row_or(any);
  }

  __device__ __forceinline__ void mask(const uint32_t (&vis)[QW], int quarter, f32x4_t (&x)[QW][2]) const {
#pragma unroll
    for (int t = 0; t < QW; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!((vis[t] >> (16 * u + 4 * quarter + e)) & 1u)) x[t][u][e] = -INFINITY;
  }

  // Weights of the tile's positions, and their products with the values.  keep, ones: the
  // auxiliary operand's first row is ones.
  __device__ __forceinline__ void values(const Kv4Values<G>& v, const f32x4_t (&x)[QW][2], uint32_t keep, uint32_t ones) {
    // The largest scale's exponent (fp16's field: s < 2^(field - 14)).  Scales from 1 on lower the weights;
    // of smaller ones all are raised by the same power of two (exact), so that neither they nor their
    // products with weights fall to fp16's subnormals before a weight does by itself.
    uint32_t top = 0;
#pragma unroll
    for (int gg = 0; gg < G; ++gg)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = kv4_max_halves(top, v.s[gg][e]);
    const int most = __builtin_amdgcn_readfirstlane(static_cast<int>((kv4_row_max(top) & 0x7FFFu) >> 10));
    const float lift = static_cast<float>(max(most - 14, 0) - 8);
    if (min(most, 14) > field) {  // the largest so far
      const float down = kv4_exp2i(field - min(most, 14));
      field = min(most, 14);
#pragma unroll
      for (int t = 0; t < QW; ++t)
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[t][dt] *= down;
    }
    const _Float16 raise = __builtin_bit_cast(_Float16, static_cast<uint16_t>((29 - field) << 10));  // 2^(14 - field)
    f16x2_t sc[G][4];
#pragma unroll
    for (int gg = 0; gg < G; ++gg) {
      const u32x4_t h = kv4_to_places(v.s[gg]);
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[gg][e] = __builtin_bit_cast(f16x2_t, static_cast<uint32_t>(h[e])) * raise;
    }

    const float minus = kv4_minus_one();
    u32x4_t ps[QW][2], pf[QW][G][2];  // weights, and their products with the scales, as sums of two
#pragma unroll
    for (int t = 0; t < QW; ++t) {
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, x[t][u][e]);
      const float most_score = kv4_cross_max(mx) * factor[t];
      const bool vast = fabsf(most_score) >= kVast;
      const float cand = vast ? most_score : most_score + lift;
      const bool move = cand - ref[t] > (vast ? 0.f : 6.f);
      if (__builtin_amdgcn_ballot_w64(move)) {  // some row's weights would pass 2^14
        const float r = move ? cand : ref[t];
        const float alpha = ref[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref[t] - r);
        ref[t] = r;
        aux[t] *= alpha;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[t][dt] *= alpha;
      }
      const float base = ref[t] == -INFINITY ? 0.f : ref[t];  // nothing visible yet: every weight is 2^-inf
      f32x4_t y[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[u][e] = __builtin_fmaf(x[t][u][e], factor[t], -base);
      if (__builtin_amdgcn_ballot_w64(fabsf(base) >= kVast)) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) y[u][e] = fabsf(base) >= kVast ? x[t][u][e] * factor[t] - base : y[u][e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x2_t w{__builtin_amdgcn_exp2f(y[0][e]), __builtin_amdgcn_exp2f(y[1][e])};
        const f16x2_t hi = __builtin_convertvector(w, f16x2_t);
        const f16x2_t lo = __builtin_convertvector(f32x2_t{__builtin_fmaf(static_cast<float>(hi[0]), minus, w[0]),
                                                           __builtin_fmaf(static_cast<float>(hi[1]), minus, w[1])}, f16x2_t);
        ps[t][0][e] = __builtin_bit_cast(uint32_t, hi);
        ps[t][1][e] = __builtin_bit_cast(uint32_t, lo);
        // Times the scales: the first product's rounding, which an fma returns exactly, goes to the second.
#pragma unroll
        for (int gg = 0; gg < G; ++gg) {
          const f16x2_t c = sc[gg][e], h = hi * c;
          pf[t][gg][0][e] = __builtin_bit_cast(uint32_t, h);
          pf[t][gg][1][e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(lo, c, __builtin_elementwise_fma(hi, c, -h)));
        }
      }
    }
    u32x4_t w = kv4_to_places(v.m);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = and_or(w[e], keep, ones);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int t = 0; t < QW; ++t)
        aux[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, w), __builtin_bit_cast(f16x8_t, ps[t][i]),
                                                       aux[t], 0, 0, 0);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      const f16x8_t vf = kv4_codes(v.c[dt / 4][dt % 4]);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < QW; ++t)
          o[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, __builtin_bit_cast(f16x8_t, pf[t][dt * G / 8][i]), o[t][dt], 0, 0, 0);
    }
  }

  // Codes back from 2^-9, scales from their raise, minima added.
  __device__ __forceinline__ void finish(int col) {
    const float back = kv4_exp2i(field - 5);
#pragma unroll
    for (int t = 0; t < QW; ++t)
#pragma unroll
      for (int gg = 0; gg < G; ++gg) {
        const float z = __shfl(aux[t][1 + gg], col);
#pragma unroll
        for (int dt = gg * (8 / G); dt < (gg + 1) * (8 / G); ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[t][dt][e] = __builtin_fmaf(o[t][dt][e], back, z);
      }
  }
};

constexpr int kWaves = 8;
constexpr int kRing = 4;  // tiles of a wavefront's ring in LDS, all but one in flight

// s_waitcnt immediate: at most `vm` vector memory operations outstanding, nothing said of others.
constexpr int kv4_wait_vm(int vm) { return (vm & 15) | (7 << 4) | (15 << 8) | ((vm >> 4) << 14); }

constexpr int kKv4WaitLds = 15 | (7 << 4) | (3 << 14);  // no LDS operation outstanding

// A wavefront takes QW query tiles of 16 rows, QG wavefronts share a tile of positions.  G:
// groups of dimensions (1 or 2).
//
// RING: a wavefront's tiles go from memory into a ring of four in LDS of its own (no register is
// held by a load in flight, so three tiles are, 14 KB a wavefront); otherwise into registers, for
// ranges of few tiles per wavefront, which a ring could not get ahead of (kv4_shape has the line).
template <int QW, int QG, int G, bool RING>
__global__ __launch_bounds__(kWaves* kWave) __attribute__((amdgpu_waves_per_eu(2))) void k_kv4_partial(Kv4AttnArgs a) {
  constexpr int KW = kWaves / QG;  // tiles of positions at a time
  constexpr int kThreads = kWaves * kWave;
  constexpr int kSlot = (2 * kv4_tile_bytes(G)) / 16;  // of a wavefront, in 16 bytes: key codes, value codes, their scales and minima
  constexpr int kMergeRow = kKv4D + 4;                 // floats of an output row in the merge
  constexpr int kMerge = kWaves * 16 * kMergeRow / 4;  // the wavefronts' outputs of a query tile, in 16 bytes
  static_assert(kRing * kWaves * kSlot >= kMerge, "the merge fits the ring");
  __shared__ u32x4_t lds[RING ? kRing * kWaves * kSlot : kMerge];
  __shared__ float2 stat[kWaves][16 * QW];  // reference and sum of weights
  __shared__ uint32_t words[kKv4MaskWords];
  const int s = blockIdx.x, g = blockIdx.y;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x / kWave));
  const int qg = wave % QG, kw = wave / QG;
  const int col = lane & 15, quarter = lane >> 4;
  const int total = a.P + a.T + a.M;
  const int first = s * a.tiles_per_split;
  const int last = min((total + kKv4Tile - 1) / kKv4Tile, first + a.tiles_per_split);
  const size_t head = static_cast<size_t>(g) * (a.S / kKv4Tile) * kv4_tile_bytes(G);
  const uint8_t* kbase = a.k_cache + head;
  const uint8_t* vbase = a.v_cache + head;
  // the auxiliary product's first row is ones
  const uint32_t keep = col == 0 ? 0u : ~0u, ones = col == 0 ? 0x3C003C00u : 0u;
  Kv4Rows<QW, G> rows;
  int n = first + kw;
  // The masks, where the range has a tile that they have a say in: in LDS, since a load from
  // memory in the loop would wait for every load before it.
  const bool any_masked = last * kKv4Tile > a.P;  // the same for the whole workgroup
  constexpr int kWords = kKv4MaskWords / kThreads;  // a thread
  uint32_t own_words[kWords];
  auto request_masks = [&]() __attribute__((always_inline)) {
    if (any_masked)
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const int w = static_cast<int>(threadIdx.x) + i * kThreads;
        own_words[i] = w < a.M * a.W ? a.mask[w] : 0u;
      }
  };
  auto keep_masks = [&]() __attribute__((always_inline)) {
    if (any_masked) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) words[threadIdx.x + i * kThreads] = own_words[i];
      __syncthreads();
    }
  };

  if constexpr (RING) {
    constexpr int VM = 6;  // vector memory operations of a tile's loads
    u32x4_t* ring = lds + wave * (kRing * kSlot);
    const uint32_t ring_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)ring));
    // Tile `tile` into slot `slot`.  A tile past the range's last is one word of that one over
    // and over: the count of loads in flight stays what the waits assume, and memory sees one
    // line.
    const uint32_t l16 = 16 * lane, l4 = 4 * lane;
    auto request = [&](int slot, int tile) __attribute__((always_inline)) {
      const uint32_t to = __builtin_amdgcn_readfirstlane(ring_at + slot * (16 * kSlot));
      if (tile < last) {
        const size_t at = static_cast<size_t>(tile) * kv4_tile_bytes(G);
        const uint8_t* kt = kbase + at;
        const uint8_t* vt = vbase + at;
        kv4_to_lds<16>(kt, l16, to);
        kv4_to_lds<16>(kt + 1024, l16, to + 1024);
        if (G == 2 || lane < 32) {  // scales and minima: 128 G bytes a side
          kv4_to_lds<4>(kt + kKv4CodeBytes, l4, to + 4 * 1024);
          kv4_to_lds<4>(vt + kKv4CodeBytes, l4, to + 4 * 1024 + 128 * G);
        }
        kv4_to_lds<16>(vt, l16, to + 2 * 1024);
        kv4_to_lds<16>(vt + 1024, l16, to + 3 * 1024);
      } else {
        const uint8_t* kt = kbase + static_cast<size_t>(last - 1) * kv4_tile_bytes(G);
#pragma unroll
        for (int i = 0; i < VM; ++i) kv4_to_lds<4>(kt, 0, to);
      }
    };
    rows.request(a, g, 16 * QW * qg, lane);
    request_masks();
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) request(i, n + i * KW);
    rows.begin(a);
    keep_masks();
    for (int slot = 0; n < last; n += KW, slot = (slot + 1) % kRing) {
      // Into the slot whose tile the last step was done with, once that step's reads are back.
      __builtin_amdgcn_s_waitcnt(kKv4WaitLds);
      request((slot + kRing - 1) % kRing, n + (kRing - 1) * KW);
      // Loads complete in order: when the later tiles' are all that is outstanding, this tile
      // is in LDS.
      __builtin_amdgcn_s_waitcnt(kv4_wait_vm((kRing - 1) * VM));
      asm volatile("" ::: "memory");
      const int key0 = n * kKv4Tile;
      const bool masked = key0 + kKv4Tile > a.P;  // the same for the whole wavefront
      u32x4_t* p = ring + slot * kSlot;
      uint32_t vis[QW] = {};
      if (masked) {
        // Scales and minima of values that no row sees become zero: they may be anything, and a large
        // scale among them would cost the others' weights bits.
        const uint32_t any = rows.look(a, words, key0, total, vis);
        if (lane < 32 * G) {
          const int e = lane % 4, at = 4 * (lane / (8 * G)) + 16 * (e / 2) + 2 * (e % 2);  // the word's first position
          reinterpret_cast<uint32_t*>(p + 256)[32 * G + lane] &= kv4_seen_halves(any >> at);
        }
      }
      if (masked) kv4_wave_fence();
      Kv4Keys<G> k;
      Kv4Values<G> v;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        k.c[u] = p[64 * u + lane];
        v.c[u] = p[128 + 64 * u + lane];
      }
      const u32x4_t* meta = p + 256 + 2 * G * quarter;
#pragma unroll
      for (int gg = 0; gg < G; ++gg) {
        k.s[gg] = meta[2 * gg];
        k.m[gg] = meta[2 * gg + 1];
        v.s[gg] = meta[8 * G + 2 * gg];
      }
      v.m = meta[8 * G + (col == 2 ? 2 * (G - 1) : 0) + 1];
      f32x4_t x[QW][2];
      rows.scores(k, x);
      if (masked) rows.mask(vis, quarter, x);
      rows.values(v, x, keep, ones);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);  // nothing may land in the ring once it is used for the merge
    __syncthreads();
  } else {
    Kv4Keys<G> k{};
    Kv4Values<G> v{};
    if (n < last) {
      kv4_load<G>(kbase + static_cast<size_t>(n) * kv4_tile_bytes(G), lane, k);
      kv4_load<G>(vbase + static_cast<size_t>(n) * kv4_tile_bytes(G), lane, v);
    }
    rows.request(a, g, 16 * QW * qg, lane);
    request_masks();
    rows.begin(a);
    keep_masks();
    auto one_tile = [&](auto masked) __attribute__((always_inline)) {
      f32x4_t x[QW][2];
      rows.scores(k, x);
      const int next = n + KW;
      if (next < last)
        kv4_load<G>(kbase + static_cast<size_t>(next) * kv4_tile_bytes(G), lane, k);
      else
        kv4_keep(k);
      if constexpr (decltype(masked)::value) {
        uint32_t vis[QW];
        const uint32_t any = rows.look(a, words, n * kKv4Tile, total, vis);
        rows.mask(vis, quarter, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {  // scales and minima of values that no row sees become zero, as in the ring
          const uint32_t stay = kv4_seen_halves(any >> (4 * quarter + 16 * (e / 2) + 2 * (e % 2)));
#pragma unroll
          for (int gg = 0; gg < G; ++gg) v.s[gg][e] &= stay;
          v.m[e] &= stay;
        }
      }
      rows.values(v, x, keep, ones);
      if (next < last)
        kv4_load<G>(vbase + static_cast<size_t>(next) * kv4_tile_bytes(G), lane, v);
      else
        kv4_keep(v);
      n = next;
    };
    // tiles of committed positions alone, then those that the masks have a say in
    for (const int plain = min(last, a.P / kKv4Tile); n < plain;) one_tile(std::false_type{});
    while (n < last) one_tile(std::true_type{});
  }

  // The wavefronts' outputs, references and sums in LDS; then the workgroup scales and adds them in
  // wavefront order, four dimensions of a row a thread.
  rows.finish(col);
  float* merge = reinterpret_cast<float*>(lds);
  const int nrows = a.Gq * a.M;
#pragma unroll
  for (int t = 0; t < QW; ++t) {
    if (t > 0) __syncthreads();
    if (quarter == 0) stat[wave][16 * t + col] = make_float2(rows.ref[t], rows.aux[t][0]);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
      *reinterpret_cast<f32x4_t*>(merge + (wave * 16 + col) * kMergeRow + 16 * dt + 4 * quarter) = rows.o[t][dt];
    __syncthreads();
    for (int i = threadIdx.x; i < QG * 16 * (kKv4D / 4); i += kThreads) {
      const int qw = i / (16 * (kKv4D / 4)), rr = i / (kKv4D / 4) % 16, d4 = 4 * (i % (kKv4D / 4));
      const int row = 16 * (QW * qw + t) + rr;
      if (row >= nrows) continue;  // padding rows are never read
      float2 st[KW];
      f32x4_t v[KW];
      float top = -INFINITY, ls = 0.f;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        st[w] = stat[w * QG + qw][16 * t + rr];
        v[w] = *reinterpret_cast<const f32x4_t*>(merge + ((w * QG + qw) * 16 + rr) * kMergeRow + d4);
        top = fmaxf(top, st[w].x);
      }
      const float base = top == -INFINITY ? 0.f : top;
      f32x4_t sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float f = __builtin_amdgcn_exp2f(st[w].x - base);
        sum += v[w] * f;
        ls += st[w].y * f;
      }
      if (a.splits == 1) {
        const float inv = ls == 0.f ? 0.f : 1.f / ls;
        const int hl = kv4_row_head(row, a.inv_m), token = row - hl * a.M;
        *reinterpret_cast<uint2*>(a.out + (static_cast<size_t>(token) * a.Hq + g * a.Gq + hl) * kKv4D + d4) =
            make_uint2(kv4_pack(sum[0] * inv, sum[1] * inv), kv4_pack(sum[2] * inv, sum[3] * inv));
        continue;
      }
      const size_t at = (static_cast<size_t>(g) * a.splits + s) * a.rows_pad + row;
      *reinterpret_cast<f32x4_t*>(a.part_o + at * kKv4D + d4) = sum;
      if (d4 == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(top, ls);
    }
  }
}

// The wavefront's largest value, in every lane: within rows of 16 lanes by DPP moves, then across
// them.
template <int CTRL>
__device__ __forceinline__ float kv4_dpp_max(float v) {
  const int b = __float_as_int(v);
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(b, b, CTRL, 0xF, 0xF, false)));
}
__device__ __forceinline__ float kv4_wave_max(float v) {
  v = kv4_dpp_max<0xB1>(v);   // quad_perm [1,0,3,2]
  v = kv4_dpp_max<0x4E>(v);   // quad_perm [2,3,0,1]
  v = kv4_dpp_max<0x141>(v);  // row_half_mirror
  v = kv4_dpp_max<0x140>(v);  // row_mirror
  return kv4_cross_max(v);
}

constexpr int kCombineThreads = 256;

// One workgroup per (token i, query head h): 8 teams of 32 threads, four dimensions a thread,
// team c takes the ranges c, c + 8, ...  Every wavefront reads the ranges' (max, sum) pairs
// itself, one a lane, so the outputs are requested with them and the only barrier is
// the one in front of the teams' sum, which runs in team order.
__global__ __launch_bounds__(kCombineThreads) void k_kv4_combine(Kv4AttnArgs a) {
  constexpr int kTeams = kCombineThreads / 32, kBatch = 8;
  __shared__ f32x4_t num[kTeams][32];
  __shared__ float den[kTeams];
  const int i = blockIdx.y, h = blockIdx.x;
  const int team = threadIdx.x / 32, d4 = 4 * (threadIdx.x % 32);
  const int lane = threadIdx.x % kWave;
  const int g = h / a.Gq, row = (h - g * a.Gq) * a.M + i;
  const int ns = a.splits;
  const size_t base = static_cast<size_t>(g) * ns * a.rows_pad + row;
  const float* po = a.part_o + base * kKv4D + d4;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + base;
  const size_t step = static_cast<size_t>(a.rows_pad);
  f32x4_t sum{0.f, 0.f, 0.f, 0.f};
  float total = 0.f, mmax = -INFINITY;
  for (int s0 = 0; s0 < ns; s0 += kWave) {  // 64 ranges at a time: a lane's pair each
    f32x4_t v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int s = s0 + team + kTeams * u;
      v[u] = s < ns ? *reinterpret_cast<const f32x4_t*>(po + s * step * kKv4D) : f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const float2 own = s0 + lane < ns ? ml[(s0 + lane) * step] : make_float2(-INFINITY, 0.f);
    const float mx = fmaxf(mmax, kv4_wave_max(own.x));
    const float w = own.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(own.x - mx);
    const float keep = mmax == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mmax - mx);
    mmax = mx;
    sum *= keep;
    total *= keep;
    const float wl = w * own.y;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int s = team + kTeams * u;
      sum += v[u] * __shfl(w, s);
      total += __shfl(wl, s);
    }
  }
  num[team][d4 / 4] = sum;
  if (d4 == 0) den[team] = total;
  __syncthreads();
  if (threadIdx.x < 32) {
    total = den[0];
#pragma unroll
    for (int c = 1; c < kTeams; ++c) {
      sum += num[c][d4 / 4];
      total += den[c];
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    *reinterpret_cast<uint2*>(a.out + (static_cast<size_t>(i) * a.Hq + h) * kKv4D + d4) =
        make_uint2(kv4_pack(sum[0] * inv, sum[1] * inv), kv4_pack(sum[2] * inv, sum[3] * inv));
  }
}

// How a call is cut: wavefronts of QW query tiles, QG of them on a tile of positions, and ranges of
// `tiles` tiles.
struct Kv4Shape {
  int qw, qg, tiles;
  bool ring;
};

// A range has a workgroup, and there are as many as CUs (16385 positions of eight heads with 5 rows
// 11.0 us; with ranges of whole turns of a workgroup's wavefronts, 171 workgroups, 11.7; 8407 with 64
// rows 18.0 against 19.3), but no wavefront goes without a tile.
// Up to three and a half tiles a wavefront one workgroup takes a whole head, and the second kernel is
// saved (four heads of 7 rows: 20 tiles 7.8 us a call against 10.0, 28 9.2 against 10.0, 32 10.3 against
// 9.9; of 21 rows, four wavefronts side by side: 12 9.2 against 9.9, 14 9.8 against 9.7).
// Two query tiles a wavefront share the unpacking, and from kRingFrom tiles on the ring in LDS gets ahead
// of it (five tiles: 20 rows a head 24.3 us against 24.4 with one query tile from registers, 64 rows 24.3
// against 25.5; 131138 positions of eight heads with 30 rows, 17 tiles, 49.7 against 65.7, and 60.0 in a
// ring with one query tile).  One query tile a wavefront is faster from registers up to kRingFromOne (5 rows,
// five tiles 15.4 against 17.6, eight 19.9 against 21.4, ten 24.0 both, twelve 28.0 against 27.4).
constexpr int kRingFrom = 5, kRingFromOne = 9;
static_assert(kRingFromOne - 1 >= 2 * (kRingFrom - 1), "a ring of one query tile only where no wavefronts share positions");

Kv4Shape kv4_shape(int M, int Hq, int Hkv, int P, int T) {
  const int tiles = (P + T + M + kKv4Tile - 1) / kKv4Tile;
  const int qt = (Hq / Hkv * M + 15) / 16;
  const int ranges = (256 + Hkv - 1) / Hkv;  // per head: one workgroup a CU
  auto cut = [&](int qw) {
    const int qg = qt <= qw ? 1 : qt <= 2 * qw ? 2 : 4;
    const int at_once = kWaves / qg;
    int tiles_a_split = std::max((tiles + ranges - 1) / ranges, at_once);
    if (2 * tiles <= 7 * at_once) tiles_a_split = tiles;
    return Kv4Shape{qw, qg, tiles_a_split, (tiles_a_split + at_once - 1) / at_once >= (qw == 2 ? kRingFrom : kRingFromOne)};
  };
  if (qt > 1) {
    const Kv4Shape wide = cut(2);
    if (wide.ring) return wide;
  }
  return cut(1);
}

template <int QW, int QG, bool RING>
void launch_shape(const Kv4AttnArgs& a, int groups, hipStream_t st) {
  const dim3 grid(a.splits, a.Hkv), block(kWaves * kWave);
  if (groups == 1)
    hipLaunchKernelGGL((k_kv4_partial<QW, QG, 1, RING>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_kv4_partial<QW, QG, 2, RING>), grid, block, 0, st, a);
}

}  // namespace

void kv4_attn_plan(int M, int Hq, int Hkv, int P, int T, int* splits, int* tiles_per_split) {
  const int tiles = (P + T + M + kKv4Tile - 1) / kKv4Tile;
  const Kv4Shape sh = kv4_shape(M, Hq, Hkv, P, T);
  *tiles_per_split = sh.tiles;
  *splits = (tiles + *tiles_per_split - 1) / *tiles_per_split;
}

size_t kv4_attn_workspace_bytes(int M, int Hq, int Hkv, int P, int T) {
  int splits = 0, tps = 0;
  kv4_attn_plan(M, Hq, Hkv, P, T, &splits, &tps);
  if (splits == 1) return 0;
  const int rows_pad = 16 * ((Hq / Hkv * M + 15) / 16);
  const size_t n = static_cast<size_t>(Hkv) * splits * rows_pad;
  // The partials follow the split-K completion counters at the workspace's start.
  return kSplitCounterBytes + n * kKv4D * sizeof(float) + n * 2 * sizeof(float);
}

hipError_t launch_kv4_attention(const Kv4AttnArgs& a, int groups, hipStream_t st) {
  const Kv4Shape sh = kv4_shape(a.M, a.Hq, a.Hkv, a.P, a.T);
  if (sh.qw == 2 && sh.qg == 1)
    launch_shape<2, 1, true>(a, groups, st);
  else if (sh.qw == 2)
    launch_shape<2, 2, true>(a, groups, st);
  else if (sh.ring)
    launch_shape<1, 1, true>(a, groups, st);
  else if (sh.qg == 1)
    launch_shape<1, 1, false>(a, groups, st);
  else if (sh.qg == 2)
    launch_shape<1, 2, false>(a, groups, st);
  else
    launch_shape<1, 4, false>(a, groups, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  hipLaunchKernelGGL(k_kv4_combine, dim3(a.Hq, a.M), dim3(kCombineThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace subspec
