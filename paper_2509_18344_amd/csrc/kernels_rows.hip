// The row operators between two projections: residual addition with the RMS norm, the gated
// activation, and rows to and from 8 bits.
//
//   norm  s = x + residual,  y = s / sqrt(mean s^2 + eps) * w
//   act   y = g / (1 + exp(-g)) * u
//   rows  a block of 128 values: e = the smallest whole number >= -126 with max |x| <= 448 * 2^e,
//         codes e4m3(x * 2^-e)
//
// All are bound by memory; a few rows by a launch.  A thread holds 8 neighbouring values (16 bytes of
// bf16), so a block of 128 is a DPP row of 16 lanes.
//
// Measured: norm of 4096 rows of 5120 with the addition 32.3 us, 168 MB at 5.2 TB/s, which is a large copy's rate;
// activation of 4096 rows of 27648 132 us, 679 MB at 5.1 TB/s (112 into 8-bit rows, 567 MB); 8-bit rows of 4096 x 5120
// 14.8 us and back 14.1, 63 MB at 4.3 and 4.5 TB/s, of 4096 x 27648 67 us and 68, 5.0 TB/s.
// One row 2.4 us, of which a launch that does nothing is about 2; a call from Python costs 4.2 to 5.9.
#include "fp8_device.h"

namespace subspec {

namespace {

__device__ __forceinline__ uint4 load16(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }

__device__ __forceinline__ void store_codes(const float (&v)[8], uint8_t* codes, uint8_t* scales, int c, int m, int M, int K) {
  uint32_t byte;
  const uint2 q = fp8_block(v, &byte);
  *reinterpret_cast<uint2*>(codes + static_cast<size_t>(m) * K + 8 * c) = q;
  if (threadIdx.x % 16 == 0) scales[fp8_scale_at(c / 16, m, M)] = static_cast<uint8_t>(byte);
}

template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float* part) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off /= 2) v += __shfl_xor(v, off);
  if constexpr (THREADS == kWave) return v;
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  float s = part[0];
#pragma unroll
  for (int w = 1; w < THREADS / kWave; ++w) s += part[w];
  return s;
}

// A workgroup takes one row and holds it in registers, CHUNKS times 8 values a thread.
template <int THREADS, int CHUNKS>
__global__ __launch_bounds__(THREADS) void k_add_norm(NormArgs a) {
  __shared__ float part[2][THREADS / kWave];
  const int m = blockIdx.x, n = a.K / 8;
  const size_t row = static_cast<size_t>(m) * a.K;
  uint4 xr[CHUNKS], rr[CHUNKS], wr[CHUNKS];
#pragma unroll
  for (int u = 0; u < CHUNKS; ++u) {
    const int c = threadIdx.x + u * THREADS;
    xr[u] = rr[u] = wr[u] = make_uint4(0, 0, 0, 0);
    if (c < n) {
      xr[u] = load16(a.x + row + 8 * c);
      if (a.residual) rr[u] = load16(a.residual + row + 8 * c);
      wr[u] = load16(a.weight + 8 * c);
    }
  }
  float s[CHUNKS][8];
  float sq = 0.f;
#pragma unroll
  for (int u = 0; u < CHUNKS; ++u) {
    float r[8];
    unpack8(xr[u], s[u]);
    unpack8(rr[u], r);
    if (a.residual) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[u][i] += r[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sq = __builtin_fmaf(s[u][i], s[u][i], sq);
    const int c = threadIdx.x + u * THREADS;
    if (a.sum && c < n) *reinterpret_cast<uint4*>(a.sum + row + 8 * c) = pack8(s[u]);
  }
  float total = block_sum<THREADS>(sq, part[0]), eps = a.eps;
  // Squares past fp32's range, or lost below it (next to an eps as small): once more with the row scaled.
  const float f = total > 0x1p126f ? 0x1p-80f : total < 0x1p-80f && eps < 0x1p-60f ? 0x1p80f : 1.f;
  if (f != 1.f) {
    sq = 0.f;
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[u][i] *= f;
        sq = __builtin_fmaf(s[u][i], s[u][i], sq);
      }
    }
    total = block_sum<THREADS>(sq, part[1]);
    eps = eps * f * f;
  }
  const float r = 1.f / sqrtf(total / static_cast<float>(a.K) + eps);
#pragma unroll
  for (int u = 0; u < CHUNKS; ++u) {
    const int c = threadIdx.x + u * THREADS;
    if (c >= n) continue;  // (of 8-bit rows the 16 lanes of a block agree)
    float w[8], v[8];
    unpack8(wr[u], w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = s[u][i] * r * w[i];
    if (a.y) *reinterpret_cast<uint4*>(a.y + row + 8 * c) = pack8(v);
    if (a.codes) store_codes(v, a.codes, a.scales, c, m, a.M, a.K);
  }
}

constexpr int kRowThreads = 256;

// g * sigmoid(g) * u.  With p = exp(-|g| / 2), sigmoid(|g|) = 1 / (1 + p^2) and sigmoid(-|g|) = p^2 times
// that: no exponential overflows, and p's second factor comes last, so that a small sigmoid keeps its bits
// next to a large u.  The hardware's exponential has no numbers below 2^-126, which p passes at g = -174.7, while
// next to bf16's largest u the result lasts until g = -187: FAR moves 2^64 out of a small p (p^2 next to 1 counts
// for nothing either way) and back, exactly, once u is in.  Other gates come out the same with it or without.
template <bool FAR>
__device__ __forceinline__ float silu_mul(float g, float u) {
  const float t = -0.72134752044448170f * fabsf(g);  // log2(e) / 2
  const bool far = FAR && t < -100.f;
  const float p = __builtin_amdgcn_exp2f(far ? t + 64.f : t);
  const float q = g < 0.f ? p : 1.f;
  const float h = g * q * __builtin_amdgcn_rcpf(__builtin_fmaf(p, p, 1.f)) * u * q;
  return far && g < 0.f ? h * 0x1p-64f * 0x1p-64f : h;
}

__global__ __launch_bounds__(kRowThreads) void k_silu_mul(ActArgs a) {
  const int m = blockIdx.x, c = blockIdx.y * kRowThreads + threadIdx.x;
  if (8 * c >= a.I) return;
  const uint16_t* src = a.gu + static_cast<size_t>(m) * 2 * a.I + 8 * c;
  const uint4 gr = load16(src), ur = load16(src + a.I);
  float g[8], u[8], v[8];
  unpack8(gr, g);
  unpack8(ur, u);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = silu_mul<false>(g[i], u[i]);
  float least = g[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) least = fminf(least, g[i]);
  if (least < -170.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = silu_mul<true>(g[i], u[i]);
  }
  if (a.y) *reinterpret_cast<uint4*>(a.y + static_cast<size_t>(m) * a.I + 8 * c) = pack8(v);
  if (a.codes) store_codes(v, a.codes, a.scales, c, m, a.M, a.I);
}

__global__ __launch_bounds__(kRowThreads) void k_fp8_rows(const uint16_t* x, int M, int K, uint8_t* codes, uint8_t* scales) {
  const int m = blockIdx.x, c = blockIdx.y * kRowThreads + threadIdx.x;
  if (8 * c >= K) return;
  float v[8];
  unpack8(load16(x + static_cast<size_t>(m) * K + 8 * c), v);
  store_codes(v, codes, scales, c, m, M, K);
}

__global__ __launch_bounds__(kRowThreads) void k_fp8_read(const uint8_t* codes, const uint8_t* scales, int M, int K, uint16_t* y) {
  const int m = blockIdx.x, c = blockIdx.y * kRowThreads + threadIdx.x;
  if (8 * c >= K) return;
  const size_t at = static_cast<size_t>(m) * K + 8 * c;
  const uint2 q = *reinterpret_cast<const uint2*>(codes + at);
  const int e = static_cast<int>(scales[fp8_scale_at(c / 16, m, M)]) - 127;
  float v[8];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int w = static_cast<int>(i ? q.y : q.x);
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    v[4 * i] = ldexpf(lo[0], e);
    v[4 * i + 1] = ldexpf(lo[1], e);
    v[4 * i + 2] = ldexpf(hi[0], e);
    v[4 * i + 3] = ldexpf(hi[1], e);
  }
  *reinterpret_cast<uint4*>(y + at) = pack8(v);
}

dim3 row_grid(int M, int K) { return dim3(M, (K / 8 + kRowThreads - 1) / kRowThreads); }

template <int THREADS, int CHUNKS>
void add_norm_at(const NormArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_add_norm<THREADS, CHUNKS>), dim3(a.M), dim3(THREADS), 0, st, a);
}

}  // namespace

// Few rows: 8 values a thread, so that a row's loads, squares and sums spread widest (49 rows of 3584: 2.93 us,
// 3.11 with 16 values a thread; of 5120 3.13 and 3.24).  Many: 16, for fewer wavefronts at the sum (4096 rows of 512:
// 4.4 us, 4.7 with 8; of 3584 18.4 and 18.9).  More where a workgroup of 1024 needs them (64 for rows past 32768, which
// spill 28 bytes a lane).
hipError_t launch_add_norm(const NormArgs& a, hipStream_t st) {
  const int n = a.K / 8;
  const bool few = a.M < 512;
  if (n > 4096) add_norm_at<1024, 8>(a, st);
  else if (n > 2048) add_norm_at<1024, 4>(a, st);
  else if (n > 1024) add_norm_at<1024, 2>(a, st);
  else if (few && n > 512) add_norm_at<1024, 1>(a, st);
  else if (few && n > 256) add_norm_at<512, 1>(a, st);
  else if (few && n > 128) add_norm_at<256, 1>(a, st);
  else if (few) add_norm_at<128, 1>(a, st);
  else if (n > 512) add_norm_at<512, 2>(a, st);
  else if (n > 256) add_norm_at<256, 2>(a, st);
  else if (n > 128) add_norm_at<128, 2>(a, st);
  else add_norm_at<64, 2>(a, st);
  return hipGetLastError();
}

hipError_t launch_silu_mul(const ActArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(k_silu_mul, row_grid(a.M, a.I), dim3(kRowThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_fp8_rows(const uint16_t* x, int M, int K, uint8_t* codes, uint8_t* scales, hipStream_t st) {
  hipLaunchKernelGGL(k_fp8_rows, row_grid(M, K), dim3(kRowThreads), 0, st, x, M, K, codes, scales);
  return hipGetLastError();
}

hipError_t launch_fp8_read(const uint8_t* codes, const uint8_t* scales, int M, int K, uint16_t* y, hipStream_t st) {
  hipLaunchKernelGGL(k_fp8_read, row_grid(M, K), dim3(kRowThreads), 0, st, codes, scales, M, K, y);
  return hipGetLastError();
}

}  // namespace subspec
