// Tree attention over the key/value cache held in 4 bits.
//
// M new tree tokens with Hq query heads grouped onto Hkv key/value heads attend, with
// scores q.k scale and a softmax, to the P committed positions and to the tree positions
// P + j (j < T + M) that their mask rows allow.  A position's key is m_g + s_g c per group g
// of dimensions (fp16 minimum m, scale s, codes c of 4 bits), its value the same with its own.
//
// Neither product forms those numbers.  With codes as exact 16-bit floats (16 + c: the code
// or-ed into the mantissa of 16),
//   q.k = sum_g s_g (q.(16 + c))_g + (m_g - 16 s_g) (sum q)_g
//       = sum_g s_g ((q.(16 + c))_g - 16 (sum q)_g) + m_g (sum q)_g
// where the bracket is a bf16 matrix product whose accumulator starts at -16 (sum q)_g, and
//   sum_j p_j v_j = sum_j (p_j s_jg) (16 + c_j) - 16 sum_j (p_j s_jg) + sum_j p_j m_jg
// where the first term is an fp16 matrix product, the second the same weights against a row
// of 16s, and the third stays in 32-bit lanes.  The weight p s is rounded to fp16 (2^-12
// relative: a sixteenth of what rounding the bf16 output costs, and the roundings of
// different positions are independent); everything else is exact or in 32 bits.  fp16
// spans 2^-24 .. 65504, so the running maximum is that of score + log2 of the tile's
// largest scale: then p s is at most 2^14 for the heaviest position and keeps its
// 11 bits down to 2^-28 of it.
//
// Kernel 1 (k_kv4_partial): workgroup (range s, key/value head g); its wavefronts take the
// range's tiles of 32 positions in turn, each for up to two tiles of 16 query rows (row =
// local head * M + token; with more than 32 rows two wavefronts share a tile of positions).
// The cache holds both operands in register order: a lane's share of a tile is five or six
// 16-byte loads a side, no code passes through LDS and no wavefront waits for another until
// the end, when their outputs are scaled to a common maximum and added in wavefront order.
//   S^T = K Q^T     16x16x32 bf16, 2 blocks of 16 positions x 4 steps of 32 dimensions
//   O^T += V^T P^T  16x16x32 fp16, 8 tiles of 16 dimensions; P is in the operand layout
//                   where the scores are
// Kernel 2 (k_kv4_combine) combines the ranges in a fixed order; a single range writes the
// output itself.
#include <cmath>

#include "device_common.h"
#include "kernels_kv4.h"

namespace subspec {

namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));

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

// One lane's share of a tile: codes, and of its quarter's 8 positions (4 quarter + r and
// 16 + 4 quarter + r) the scales and minima per group.
template <int G>
struct Kv4Regs {
  u32x4_t kc[2], vc[2];
  u32x4_t ks[G], km[G], vs[G], vm[G];
};

template <int G>
__device__ __forceinline__ void kv4_load(const uint8_t* kt, const uint8_t* vt, int lane, Kv4Regs<G>& r) {
#pragma unroll
  for (int u = 0; u < 2; ++u) r.kc[u] = *reinterpret_cast<const u32x4_t*>(kt + u * 1024 + lane * 16);
  const int meta = kKv4CodeBytes + (lane / 16) * (32 * G);
#pragma unroll
  for (int g = 0; g < G; ++g) {
    r.ks[g] = *reinterpret_cast<const u32x4_t*>(kt + meta + 32 * g);
    r.km[g] = *reinterpret_cast<const u32x4_t*>(kt + meta + 32 * g + 16);
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) r.vc[u] = *reinterpret_cast<const u32x4_t*>(vt + u * 1024 + lane * 16);
#pragma unroll
  for (int g = 0; g < G; ++g) {
    r.vs[g] = *reinterpret_cast<const u32x4_t*>(vt + meta + 32 * g);
    r.vm[g] = *reinterpret_cast<const u32x4_t*>(vt + meta + 32 * g + 16);
  }
}

// Eight codes of a word as bf16 (fp16) numbers 16 + c, in order.
__device__ __forceinline__ bf16x8_t kv4_bf16(uint32_t d) {
  const uint32_t bias = 0x41804180u, mask = 0x00780078u;
  return __builtin_bit_cast(bf16x8_t, u32x4_t{and_or(d << 3, mask, bias), and_or(d >> 1, mask, bias),
                                              and_or(d >> 5, mask, bias), and_or(d >> 9, mask, bias)});
}
__device__ __forceinline__ f16x8_t kv4_f16(uint32_t d) {
  const uint32_t bias = 0x4C004C00u, mask = 0x03C003C0u;
  return __builtin_bit_cast(f16x8_t, u32x4_t{and_or(d << 6, mask, bias), and_or(d << 2, mask, bias),
                                             and_or(d >> 2, mask, bias), and_or(d >> 6, mask, bias)});
}

// Infinite and NaN halves become zero (rows that nothing has written, seen by no query).
__device__ __forceinline__ uint32_t kv4_finite(uint32_t w) {
  uint32_t r = w;
  if ((w & 0x7C00u) == 0x7C00u) r &= 0xFFFF0000u;
  if ((w & 0x7C000000u) == 0x7C000000u) r &= 0x0000FFFFu;
  return r;
}

__device__ __forceinline__ float kv4_cross_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float kv4_cross_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

constexpr int kMergeRow = kKv4D + 4;  // floats per query row of a wavefront's merged output

template <int WAVES>
struct Kv4Lds {
  alignas(16) float o[WAVES][16][kMergeRow];
  float m[WAVES][32], l[WAVES][32];
};

// QT: query tiles of 16 rows (1 .. 4); a wavefront takes up to two of them.  G: groups of
// dimensions (1 or 2).
template <int QT, int G, int WAVES>
__global__ __launch_bounds__(WAVES* kWave) void k_kv4_partial(Kv4AttnArgs a) {
  constexpr int QW = QT < 2 ? 1 : 2;
  constexpr int QG = (QT + 1) / 2;   // wavefronts that share a tile of positions
  constexpr int KW = WAVES / QG;     // tiles of positions at a time
  constexpr int kThreads = WAVES * kWave;
  __shared__ Kv4Lds<WAVES> L;
  const int s = blockIdx.x, g = blockIdx.y;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x / kWave));
  const int qg = wave % QG, kw = wave / QG;
  const int col = lane & 15, quarter = lane >> 4;
  const int Gq = a.Hq / a.Hkv;
  const int rows = Gq * a.M;
  const int total = a.P + a.T + a.M;
  const int first = s * a.tiles_per_split;
  const int last = min((total + kKv4Tile - 1) / kKv4Tile, first + a.tiles_per_split);
  const size_t head = static_cast<size_t>(g) * (a.S / kKv4Tile) * kv4_tile_bytes(G);
  const uint8_t* kbase = a.k_cache + head;
  const uint8_t* vbase = a.v_cache + head;

  Kv4Regs<G> r;
  int n = first + kw;
  if (n < last) kv4_load<G>(kbase + static_cast<size_t>(n) * kv4_tile_bytes(G), vbase + static_cast<size_t>(n) * kv4_tile_bytes(G), lane, r);

  // this lane's query row in each query tile, its fragments of q and their sums per group
  bool live[QW];
  int qi[QW];
  bf16x8_t qf[QW][4];
  float qs[QW][G];
#pragma unroll
  for (int t = 0; t < QW; ++t) {
    const int row = 16 * (QW * qg + t) + col;
    live[t] = row < rows;
    qi[t] = live[t] ? row % a.M : 0;
    const int hl = live[t] ? row / a.M : 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u32x4_t w{0, 0, 0, 0};
      if (live[t])
        w = *reinterpret_cast<const u32x4_t*>(a.q + (static_cast<size_t>(qi[t]) * a.Hq + g * Gq + hl) * kKv4D + 32 * j +
                                              8 * quarter) ^ a.q_sign;
      qf[t][j] = __builtin_bit_cast(bf16x8_t, w);
    }
#pragma unroll
    for (int gg = 0; gg < G; ++gg) {
      float sum = 0.f;
#pragma unroll
      for (int j = gg * (4 / G); j < (gg + 1) * (4 / G); ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += static_cast<float>(qf[t][j][e]);
      qs[t][gg] = kv4_cross_sum(sum);
    }
  }

  float m[QW], lsum[QW], zsum[QW][G];
  f32x4_t o[QW][8], osum[QW][G];
#pragma unroll
  for (int t = 0; t < QW; ++t) {
    m[t] = -INFINITY;
    lsum[t] = 0.f;
#pragma unroll
    for (int gg = 0; gg < G; ++gg) {
      zsum[t][gg] = 0.f;
      osum[t][gg] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) o[t][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const _Float16 h16 = static_cast<_Float16>(16.f);
  const f16x8_t sixteen{h16, h16, h16, h16, h16, h16, h16, h16};

  for (; n < last; n += KW) {
    const int key0 = n * kKv4Tile;
    const bool masked = key0 + kKv4Tile > a.P;  // the same for the whole wavefront
    // scores: lane holds positions 16u + 4 quarter + e of its query
    f32x4_t x[QW][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4_t st[QW][G];
#pragma unroll
      for (int t = 0; t < QW; ++t)
#pragma unroll
        for (int gg = 0; gg < G; ++gg) {
          const float c = -16.f * qs[t][gg];
          st[t][gg] = f32x4_t{c, c, c, c};
        }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x8_t kf = kv4_bf16(r.kc[u][j]);
#pragma unroll
        for (int t = 0; t < QW; ++t)
          st[t][j * G / 4] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][j], st[t][j * G / 4], 0, 0, 0);
      }
#pragma unroll
      for (int t = 0; t < QW; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = 0.f;
#pragma unroll
          for (int gg = 0; gg < G; ++gg) {
            const f16x8_t ks = __builtin_bit_cast(f16x8_t, r.ks[gg]), km = __builtin_bit_cast(f16x8_t, r.km[gg]);
            v = __builtin_fmaf(static_cast<float>(km[4 * u + e]), qs[t][gg], v);
            v = __builtin_fmaf(static_cast<float>(ks[4 * u + e]), st[t][gg][e], v);
          }
          x[t][u][e] = v;
        }
    }
    Kv4Regs<G> c;
#pragma unroll
    for (int u = 0; u < 2; ++u) c.vc[u] = r.vc[u];
#pragma unroll
    for (int gg = 0; gg < G; ++gg) {
      c.vs[gg] = r.vs[gg];
      c.vm[gg] = r.vm[gg];
    }
    if (n + KW < last)
      kv4_load<G>(kbase + static_cast<size_t>(n + KW) * kv4_tile_bytes(G), vbase + static_cast<size_t>(n + KW) * kv4_tile_bytes(G), lane, r);
    if (masked) {
#pragma unroll
      for (int t = 0; t < QW; ++t) {
        const uint32_t vis = live[t] ? kv4_visibility(a.mask + static_cast<size_t>(qi[t]) * a.W, a.W, a.P, key0, total) : 0u;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!((vis >> (16 * u + 4 * quarter + e)) & 1u)) x[t][u][e] = -INFINITY;
      }
#pragma unroll
      for (int gg = 0; gg < G; ++gg)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          c.vs[gg][e] = kv4_finite(c.vs[gg][e]);
          c.vm[gg][e] = kv4_finite(c.vm[gg][e]);
        }
    }
    // the exponent of the tile's largest scale of a value (scales are not negative), at least 2^-14
    float smax = 0x1p-14f;
#pragma unroll
    for (int gg = 0; gg < G; ++gg) {
      const f16x8_t vs = __builtin_bit_cast(f16x8_t, c.vs[gg]);
#pragma unroll
      for (int e = 0; e < 8; ++e) smax = fmaxf(smax, static_cast<float>(vs[e]));
    }
    smax = kv4_cross_max(smax);
    const float shift = static_cast<float>(__builtin_amdgcn_frexp_expf(smax) - 14);

    f16x8_t pf[QW][G];
#pragma unroll
    for (int t = 0; t < QW; ++t) {
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, x[t][u][e]);
      mx = kv4_cross_max(mx);
      const float mn = mx == -INFINITY ? m[t] : fmaxf(m[t], mx * a.scale_log2 + shift);
      const float ref = mn == -INFINITY ? 0.f : mn;  // nothing visible yet: every weight is 2^-inf
      const float alpha = __builtin_amdgcn_exp2f(m[t] - ref);
      m[t] = mn;
      float add = 0.f, z[G];
#pragma unroll
      for (int gg = 0; gg < G; ++gg) z[gg] = 0.f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][u][e], a.scale_log2, -ref));
          add += p;
#pragma unroll
          for (int gg = 0; gg < G; ++gg) {
            const f16x8_t vs = __builtin_bit_cast(f16x8_t, c.vs[gg]), vm = __builtin_bit_cast(f16x8_t, c.vm[gg]);
            pf[t][gg][4 * u + e] = static_cast<_Float16>(p * static_cast<float>(vs[4 * u + e]));
            z[gg] = __builtin_fmaf(p, static_cast<float>(vm[4 * u + e]), z[gg]);
          }
        }
      lsum[t] = lsum[t] * alpha + add;
#pragma unroll
      for (int gg = 0; gg < G; ++gg) zsum[t][gg] = zsum[t][gg] * alpha + z[gg];
      if (__builtin_amdgcn_ballot_w64(alpha != 1.f)) {  // some row's maximum moved
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[t][dt] *= alpha;
#pragma unroll
        for (int gg = 0; gg < G; ++gg) osum[t][gg] *= alpha;
      }
#pragma unroll
      for (int gg = 0; gg < G; ++gg)
        osum[t][gg] = __builtin_amdgcn_mfma_f32_16x16x32_f16(sixteen, pf[t][gg], osum[t][gg], 0, 0, 0);
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      const f16x8_t vf = kv4_f16(c.vc[dt / 4][dt % 4]);
#pragma unroll
      for (int t = 0; t < QW; ++t)
        o[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[t][dt * G / 8], o[t][dt], 0, 0, 0);
    }
  }

  // minima added, biases taken off; then the workgroup's maximum per row
#pragma unroll
  for (int t = 0; t < QW; ++t) {
    lsum[t] = kv4_cross_sum(lsum[t]);
#pragma unroll
    for (int gg = 0; gg < G; ++gg) {
      const float z = kv4_cross_sum(zsum[t][gg]) - osum[t][gg][0];
#pragma unroll
      for (int dt = gg * (8 / G); dt < (gg + 1) * (8 / G); ++dt) o[t][dt] += z;
    }
    if (quarter == 0) L.m[wave][16 * t + col] = m[t];
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < QW; ++t) {
    float mall = -INFINITY;
#pragma unroll
    for (int w = 0; w < KW; ++w) mall = fmaxf(mall, L.m[w * QG + qg][16 * t + col]);
    const float sc = m[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[t] - mall);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) o[t][dt] *= sc;
    if (quarter == 0) L.l[wave][16 * t + col] = lsum[t] * sc;
  }
  // One query tile of every wavefront at a time: outputs [row][dimension] in LDS, then the
  // workgroup adds the wavefronts' in order, four dimensions a thread.
#pragma unroll
  for (int t = 0; t < QW; ++t) {
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
      *reinterpret_cast<f32x4_t*>(&L.o[wave][col][16 * dt + 4 * quarter]) = o[t][dt];
    __syncthreads();
    for (int i = threadIdx.x; i < QG * 16 * (kKv4D / 4); i += kThreads) {
      const int qw = i / (16 * (kKv4D / 4)), rr = i / (kKv4D / 4) % 16, d4 = 4 * (i % (kKv4D / 4));
      const int row = 16 * (QW * qw + t) + rr;
      if (row >= rows) continue;  // padding rows are never read
      f32x4_t sum = *reinterpret_cast<const f32x4_t*>(&L.o[qw][rr][d4]);
      float ls = L.l[qw][16 * t + rr];
#pragma unroll
      for (int w = 1; w < KW; ++w) {
        sum += *reinterpret_cast<const f32x4_t*>(&L.o[w * QG + qw][rr][d4]);
        ls += L.l[w * QG + qw][16 * t + rr];
      }
      if (a.splits == 1) {
        const float inv = ls == 0.f ? 0.f : 1.f / ls;
        const int token = row % a.M, h = g * Gq + row / a.M;
        uint2 w2;
        w2.x = static_cast<uint32_t>(float_to_bf16_bits(sum[0] * inv)) | (static_cast<uint32_t>(float_to_bf16_bits(sum[1] * inv)) << 16);
        w2.y = static_cast<uint32_t>(float_to_bf16_bits(sum[2] * inv)) | (static_cast<uint32_t>(float_to_bf16_bits(sum[3] * inv)) << 16);
        *reinterpret_cast<uint2*>(a.out + (static_cast<size_t>(token) * a.Hq + h) * kKv4D + d4) = w2;
        continue;
      }
      const size_t base = (static_cast<size_t>(g) * a.splits + s) * a.rows_pad + row;
      *reinterpret_cast<f32x4_t*>(a.part_o + base * kKv4D + d4) = sum;
      if (d4 == 0) {
        float mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < KW; ++w) mm = fmaxf(mm, L.m[w * QG + qw][16 * t + rr]);
        a.part_ml[2 * base] = mm;
        a.part_ml[2 * base + 1] = ls;
      }
    }
    if (t + 1 < QW) __syncthreads();
  }
}

// One workgroup per (token i, query head h), one thread per dimension; the ranges' outputs
// are summed in range order, the first kBatch requested together with the (max, sum) pairs.
__global__ __launch_bounds__(kKv4D) void k_kv4_combine(Kv4AttnArgs a) {
  __shared__ float sm[kKv4MaxSplits], sl[kKv4MaxSplits];
  constexpr int kBatch = 32, kMore = 16;
  const int i = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq;
  const int d = threadIdx.x;
  const int Gq = a.Hq / a.Hkv;
  const int g = h / Gq, row = h % Gq * a.M + i;
  const int ns = a.splits;
  const size_t base = static_cast<size_t>(g) * ns * a.rows_pad + row;
  const float* po = a.part_o + base * kKv4D + d;
  const size_t step = static_cast<size_t>(a.rows_pad) * kKv4D;
  for (int s = d; s < ns; s += kKv4D) {
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * (base + static_cast<size_t>(s) * a.rows_pad));
    sm[s] = ml.x;
    sl[s] = ml.y;
  }
  float v[kBatch];
#pragma unroll
  for (int u = 0; u < kBatch; ++u) v[u] = u < ns ? po[u * step] : 0.f;
  __syncthreads();
  float mmax = -INFINITY;
  for (int s = 0; s < ns; ++s) mmax = fmaxf(mmax, sm[s]);
  __syncthreads();
  for (int s = d; s < ns; s += kKv4D) sm[s] = sm[s] == -INFINITY ? 0.f : exp2f(sm[s] - mmax);
  __syncthreads();
  float den = 0.f, num = 0.f;
#pragma unroll
  for (int u = 0; u < kBatch; ++u)
    if (u < ns) {
      den += sm[u] * sl[u];
      num += sm[u] * v[u];
    }
  for (int s0 = kBatch; s0 < ns; s0 += kMore) {
#pragma unroll
    for (int u = 0; u < kMore; ++u) v[u] = s0 + u < ns ? po[(s0 + u) * step] : 0.f;
#pragma unroll
    for (int u = 0; u < kMore; ++u)
      if (s0 + u < ns) {
        den += sm[s0 + u] * sl[s0 + u];
        num += sm[s0 + u] * v[u];
      }
  }
  a.out[(static_cast<size_t>(i) * a.Hq + h) * kKv4D + d] = float_to_bf16_bits(den == 0.f ? 0.f : num / den);
}

constexpr int kPartialWaves = 4;

template <int G>
void launch_partial(const Kv4AttnArgs& a, hipStream_t st) {
  const dim3 grid(a.splits, a.Hkv), block(kPartialWaves * kWave);
  switch (a.rows_pad / 16) {
    case 1: hipLaunchKernelGGL((k_kv4_partial<1, G, kPartialWaves>), grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL((k_kv4_partial<2, G, kPartialWaves>), grid, block, 0, st, a); break;
    case 3: hipLaunchKernelGGL((k_kv4_partial<3, G, kPartialWaves>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_kv4_partial<4, G, kPartialWaves>), grid, block, 0, st, a); break;
  }
}

}  // namespace

void kv4_attn_plan(int M, int Hq, int Hkv, int P, int T, int* splits, int* tiles_per_split) {
  const int tiles = (P + T + M + kKv4Tile - 1) / kKv4Tile;
  const int rows_pad = 16 * ((Hq / Hkv * M + 15) / 16);
  const int at_once = kPartialWaves / (rows_pad > 32 ? 2 : 1);  // tiles a workgroup works on at a time
  // two workgroups a CU of the 256, every wavefront with a tile
  const int most = (512 + Hkv - 1) / Hkv;  // ranges per head
  int tps = (tiles + most - 1) / most;
  tps = (tps + at_once - 1) / at_once * at_once;
  *tiles_per_split = tps;
  *splits = (tiles + tps - 1) / tps;
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
  if (groups == 1)
    launch_partial<1>(a, st);
  else
    launch_partial<2>(a, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  hipLaunchKernelGGL(k_kv4_combine, dim3(a.M * a.Hq), dim3(kKv4D), 0, st, a);
  return hipGetLastError();
}

}  // namespace subspec
