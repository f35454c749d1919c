// The product in 8-bit floating point for few rows, where the weights' bytes are all that counts:
// scaled codes become bf16 numbers on the way (exactly) and meet in the 16-bit matrix instruction, whose
// products are exact and whose sums are in fp32.  (The 8-bit matrix instruction would cut products to 13 bits, and its rate is not
// needed here: at 5 TB/s a SIMD has about 1000 cycles for a tile of 16 columns and 128 k.)
//
// A wavefront takes CT tiles of 16 columns and a run of K, its weights straight from memory to registers, a
// unit of two blocks ahead; the wavefronts of a workgroup share the columns and cut K among them, as do
// `splits` workgroups where K is long.  bf16 rows become codes on the way: the block's largest magnitude by
// packed 16-bit maxima, then one conversion for two values, which divides by the power of two too.
//
// Measured in a trace, of bf16 rows: 1 row, 3584 x 3584 6.3 us (12.8 MB; a launch that does nothing takes 2; 6.6 a call in
// a graph of them, 5.6 of 8-bit rows); 7 rows, 5120 x 27648 29.0 us, 4.9 TB/s of weights, where a copy moves 5.2; 1 row,
// 37888 x 3584 30 us (26 of 8-bit rows, 5.2 TB/s).
#include <algorithm>

#include "fp8_device.h"
#include "kernels_fp8.h"

namespace subspec {

namespace {

constexpr int kUnit = 2;    // blocks that a wavefront loads at once, one unit ahead of the products
constexpr int kAgent = 16;  // sc1: coherent at agent scope

__device__ __forceinline__ uint32_t max_across_rows(uint32_t v) {  // over the lanes l, l ^ 16, l ^ 32, l ^ 48
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(b[0], b[1]);
}

// What a lane holds of a block of x: row lane % 16, k = 16 q .. and 64 + 16 q .. (q = lane / 16), 16 each, the
// places that a weight tile gives it too.
template <bool FUSED>
struct XBlock {
  u32x4_t v[FUSED ? 4 : 2];
};

template <bool FUSED>
__device__ __forceinline__ XBlock<FUSED> load_x(const uint8_t* row, int kb) {
  XBlock<FUSED> b;
  if constexpr (FUSED) {
    const u32x4_t* p = reinterpret_cast<const u32x4_t*>(row + 256ll * kb);
    b.v[0] = p[0];
    b.v[1] = p[1];
    b.v[2] = p[8];
    b.v[3] = p[9];
  } else {
    const u32x4_t* p = reinterpret_cast<const u32x4_t*>(row + 128ll * kb);
    b.v[0] = p[0];
    b.v[1] = p[4];
  }
  return b;
}

// The block's codes, 32 a lane, and (of bf16 rows) its scale byte.
struct Codes {
  uint32_t v[8];
};
template <bool FUSED>
__device__ __forceinline__ Codes x_codes(const XBlock<FUSED>& b, uint32_t* byte) {
  Codes out;
  if constexpr (FUSED) {
    // Magnitudes of pairs as 16-bit whole numbers, which order as the numbers do.
    typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
    u16x2_t top = {0, 0};
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, b.v[u][i] & 0x7FFF7FFFu));
    const uint32_t most = max_across_rows(max(static_cast<uint32_t>(top[0]), static_cast<uint32_t>(top[1])));
    if (__any(most >= 0x7F80u)) {  // infinities or NaN in some row's block
      float x[4][8], finite = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        unpack8(make_uint4(b.v[u][0], b.v[u][1], b.v[u][2], b.v[u][3]), x[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float m = fabsf(x[u][i]);
          finite = fmaxf(finite, m < __builtin_inff() ? m : 0.f);
        }
      }
      *byte = fp8_scale_byte(__uint_as_float(max_across_rows(__float_as_uint(finite))));
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint2 c = fp8_codes(x[u], *byte);
        out.v[2 * u] = c.x;
        out.v[2 * u + 1] = c.y;
      }
      return out;
    }
    *byte = fp8_scale_byte(__uint_as_float(most << 16));
    const float scale = fp8_power(*byte);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      typedef short s16x2_t __attribute__((ext_vector_type(2)));
      const uint32_t w[2] = {b.v[u / 2][2 * (u % 2)], b.v[u / 2][2 * (u % 2) + 1]};
      s16x2_t c = {0, 0};
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2_t, w[0]), scale, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2_t, w[1]), scale, true);
      out.v[u] = __builtin_bit_cast(uint32_t, c);
    }
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u) out.v[u] = b.v[u / 4][u % 4];
  }
  return out;
}

__device__ __forceinline__ void operands(const Codes& c, float scale, bf16x8_t (&out)[4]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) out[u] = fp8_as_bf16(c.v[2 * u], c.v[2 * u + 1], scale);
}

// MT tiles of 16 rows, CT of 16 columns a wavefront.
template <int WAVES, int MT, int CT, bool FUSED>
__global__ __launch_bounds__(WAVES * kWave) void k_fp8_few(Fp8Args a) {
  constexpr int TILES = MT * CT;
  __shared__ f32x4_t sums[WAVES][TILES][kWave];
  __shared__ int last;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, q = lane / 16;
  const int KB = a.K / 128, units = (KB + kUnit - 1) / kUnit;
  const int set = blockIdx.x / a.splits, split = blockIdx.x % a.splits, parts = a.splits * WAVES, part = split * WAVES + wave;
  const int g0 = static_cast<int>(static_cast<long long>(part) * units / parts), g1 = static_cast<int>(static_cast<long long>(part + 1) * units / parts);
  const int kb1 = min(kUnit * g1, KB);
  const uint8_t* xrow[MT];
  const uint32_t* xsrow[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = min(16 * t + lane % 16, a.M - 1);  // (rows past the last: that one again)
    xrow[t] = static_cast<const uint8_t*>(a.x) + (FUSED ? 2 : 1) * (static_cast<size_t>(m) * a.K + 16 * q);
    xsrow[t] = a.xs + m;
  }
  const uint8_t* wt[CT];
  const uint32_t* wst[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int tile = min(set * CT + c, a.N / 16 - 1);
    wt[c] = a.w + static_cast<size_t>(tile) * KB * 2048 + 16 * lane;
    wst[c] = a.ws + 16 * tile + lane % 16;
  }
  struct Weights {
    u32x4_t w[CT][kUnit][2];
    uint32_t s[CT];
  };
  struct Rows {
    XBlock<FUSED> b[MT];
    uint32_t s[MT];
  };
  auto load_w = [&](int g, Weights& r) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const u32x4_t* p = reinterpret_cast<const u32x4_t*>(wt[c] + 2048ll * min(kUnit * g + j, KB - 1));
        r.w[c][j][0] = __builtin_nontemporal_load(p);
        r.w[c][j][1] = __builtin_nontemporal_load(p + 64);
      }
      r.s[c] = wst[c][static_cast<size_t>(kUnit * g / 4) * a.N];
    }
  };
  auto load_rows = [&](int kb, Rows& r) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      r.b[t] = load_x<FUSED>(xrow[t], kb);
      if constexpr (!FUSED) r.s[t] = xsrow[t][static_cast<size_t>(kb / 4) * a.M];
    }
  };
  f32x4_t acc[MT][CT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[t][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  Weights next;
  Rows rows;
  if (g0 < g1) {
    load_rows(kUnit * g0, rows);
    load_w(g0, next);
  }
  for (int g = g0; g < g1; ++g) {
    const Weights now = next;
    if (g + 1 < g1) load_w(g + 1, next);
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
      const int kb = kUnit * g + j;
      if (kb >= kb1) break;
      const Rows x = rows;
      if (kb + 1 < kb1) load_rows(kb + 1, rows);
      const int shift = 8 * (kb % 4);
      Codes xc[MT];
      uint32_t xb[MT], wb[CT];
      bool plain = true;
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        xb[t] = FUSED ? 0u : x.s[t] >> shift & 255u;
        xc[t] = x_codes<FUSED>(x.b[t], &xb[t]);
        plain &= fp8_plain(xb[t]);
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        wb[c] = now.s[c] >> shift & 255u;
        plain &= fp8_plain(wb[c]);
      }
      plain = __all(plain);
      if (!plain) {  // once more without the scales of zeros
        bool p = true;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          uint32_t any = 0;
#pragma unroll
          for (int u = 0; u < 8; ++u) any |= xc[t].v[u];
          p &= fp8_plain(xb[t]) || fp8_zeros(any);
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          uint32_t any = 0;
#pragma unroll
          for (int u = 0; u < 8; ++u) any |= now.w[c][j][u / 4][u % 4];
          p &= fp8_plain(wb[c]) || fp8_zeros(any);
        }
        plain = __all(p);
      }
      bf16x8_t w[CT][4];
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        Codes wc;
#pragma unroll
        for (int u = 0; u < 8; ++u) wc.v[u] = now.w[c][j][u / 4][u % 4];
        operands(wc, plain ? fp8_power(wb[c]) : 1.f, w[c]);
      }
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        bf16x8_t xo[4];
        operands(xc[t], plain ? fp8_power(xb[t]) : 1.f, xo);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          f32x4_t s = plain ? acc[t][c] : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int u = 0; u < 4; ++u) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[c][u], xo[u], s, 0, 0, 0);
          if (plain) {
            acc[t][c] = s;
          } else {  // a scale so far from 1 that bf16 would not hold the codes: this lane's row of x and four columns afterwards
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[t][c][e] += ldexpf(s[e], static_cast<int>(xb[t] + __shfl(wb[c], 4 * q + e)) - 254);
          }
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int c = 0; c < CT; ++c) sums[wave][t * CT + c][lane] = acc[t][c];
  __syncthreads();
  // The runs of K are added in their order, tile i by wavefront i % WAVES.
  constexpr int MINE = (TILES + WAVES - 1) / WAVES;
  f32x4_t v[MINE];
#pragma unroll
  for (int o = 0; o < MINE; ++o) {
    const int i = min(wave + o * WAVES, TILES - 1);
    v[o] = sums[0][i][lane];
#pragma unroll
    for (int u = 1; u < WAVES; ++u) v[o] += sums[u][i][lane];
  }
  if (a.splits > 1) {
    // Agent-scope stores, counted in once they are acknowledged; the last workgroup of the columns adds all.
    const uint32_t bytes = static_cast<uint32_t>(a.splits) * TILES * kWave * 16;
    const __amdgpu_buffer_rsrc_t part_of = buffer_rsrc(reinterpret_cast<const uint8_t*>(a.part) + static_cast<size_t>(set) * bytes, bytes);
#pragma unroll
    for (int o = 0; o < MINE; ++o) {
      const int i = min(wave + o * WAVES, TILES - 1);
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v[o]), part_of, ((split * TILES + i) * kWave + lane) * 16, 0, kAgent);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __syncthreads();
    if (threadIdx.x == 0)
      last = __hip_atomic_fetch_add(a.count + set, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<unsigned>(a.splits - 1);
    __syncthreads();
    if (!last) return;
#pragma unroll
    for (int o = 0; o < MINE; ++o) v[o] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; s += 4) {
      f32x4_t p[MINE][4];
#pragma unroll
      for (int o = 0; o < MINE; ++o)
#pragma unroll
        for (int u = 0; u < 4; ++u) {  // (past the last part: zeros, past the buffer)
          const int i = min(wave + o * WAVES, TILES - 1);
          const int at = s + u < a.splits ? (((s + u) * TILES + i) * kWave + lane) * 16 : -16;
          p[o][u] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(part_of, at, 0, kAgent));
        }
#pragma unroll
      for (int o = 0; o < MINE; ++o)
#pragma unroll
        for (int u = 0; u < 4; ++u) v[o] += p[o][u];
    }
    if (threadIdx.x == 0) __hip_atomic_store(a.count + set, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
#pragma unroll
  for (int o = 0; o < MINE; ++o) {
    const int i = wave + o * WAVES, tile = set * CT + i % CT, m = 16 * (i / CT) + lane % 16;
    if (i >= TILES || tile >= a.N / 16 || m >= a.M) continue;
    const uint32_t lo = float_to_bf16_bits(v[o][0]) | static_cast<uint32_t>(float_to_bf16_bits(v[o][1])) << 16;
    const uint32_t hi = float_to_bf16_bits(v[o][2]) | static_cast<uint32_t>(float_to_bf16_bits(v[o][3])) << 16;
    *reinterpret_cast<uint2*>(a.y + static_cast<size_t>(m) * a.N + 16 * tile + 4 * q) = make_uint2(lo, hi);
  }
}

template <int WAVES, int MT, int CT, bool FUSED>
void few_at(const Fp8Args& a, hipStream_t st) {
  hipLaunchKernelGGL((k_fp8_few<WAVES, MT, CT, FUSED>), dim3((a.N / 16 + CT - 1) / CT * a.splits), dim3(WAVES * kWave), 0, st, a);
}

}  // namespace

hipError_t launch_fp8_few(const Fp8Args& a, int columns, int waves, hipStream_t st) {
  const int rows = (a.M + 15) / 16;
  const bool fused = !a.xs;
  if (rows == 1) {
    if (columns == 2 && waves == 8) fused ? few_at<8, 1, 2, true>(a, st) : few_at<8, 1, 2, false>(a, st);
    else if (columns == 2) fused ? few_at<4, 1, 2, true>(a, st) : few_at<4, 1, 2, false>(a, st);
    else if (waves == 16) fused ? few_at<16, 1, 1, true>(a, st) : few_at<16, 1, 1, false>(a, st);
    else fused ? few_at<8, 1, 1, true>(a, st) : few_at<8, 1, 1, false>(a, st);
  } else if (rows == 2) {
    fused ? few_at<4, 2, 1, true>(a, st) : few_at<4, 2, 1, false>(a, st);
  } else if (rows == 3) {
    few_at<4, 3, 1, false>(a, st);
  } else {
    few_at<4, 4, 1, false>(a, st);
  }
  return hipGetLastError();
}

}  // namespace subspec
