// The product in 8-bit floating point:
//   y[m][n] = sum over blocks b of 2^(ex[m][b] + ew[n][b]) * sum over the block's k of x[m][k] w[n][k]
// with e4m3 codes and fp32 sums.  The scales are powers of two, so that the matrix instruction takes
// them as operands (a byte for each row of either side) and the sum over k never leaves it.
#include "fp8_device.h"
#include "kernels_fp8.h"

namespace subspec {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8_t codes32(const uint8_t* lo, const uint8_t* hi) {
  const int4 a = *reinterpret_cast<const int4*>(lo), b = *reinterpret_cast<const int4*>(hi);
  return i32x8_t{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}

// Byte J of the scale words; weights are the left operand, so a lane ends up with four columns of one row.
template <int J>
__device__ __forceinline__ f32x4_t mfma16(i32x8_t w, i32x8_t x, f32x4_t c, uint32_t ws, uint32_t xs) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 0, 0, J, static_cast<int>(ws), J, static_cast<int>(xs));
}

// A wavefront takes 16 rows and 16 columns, all of K.
__global__ __launch_bounds__(256) void k_fp8_tile(Fp8Args a) {
  const int lane = threadIdx.x % kWave, nt = blockIdx.y * 4 + threadIdx.x / kWave, KB = a.K / 128;
  if (nt >= a.N / 16) return;
  const int m = min(static_cast<int>(blockIdx.x) * 16 + lane % 16, a.M - 1);  // (rows past the last: that one again)
  const uint8_t* x = static_cast<const uint8_t*>(a.x) + static_cast<size_t>(m) * a.K + 16 * (lane / 16);
  const uint8_t* w = a.w + static_cast<size_t>(nt) * KB * 2048 + 16 * lane;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  for (int g = 0; 4 * g < KB; ++g) {
    const uint32_t xs = a.xs[static_cast<size_t>(g) * a.M + m], ws = a.ws[static_cast<size_t>(g) * a.N + 16 * nt + lane % 16];
    auto block = [&](auto j) __attribute__((always_inline)) {
      constexpr int J = decltype(j)::value;
      const int kb = 4 * g + J;
      if (kb >= KB) return;
      acc = mfma16<J>(codes32(w + 2048ll * kb, w + 2048ll * kb + 1024), codes32(x + 128ll * kb, x + 128ll * kb + 64), acc, ws, xs);
    };
    block(std::integral_constant<int, 0>{});
    block(std::integral_constant<int, 1>{});
    block(std::integral_constant<int, 2>{});
    block(std::integral_constant<int, 3>{});
  }
  const int row = blockIdx.x * 16 + lane % 16;
  if (row >= a.M) return;
  uint2 v;
  v.x = float_to_bf16_bits(acc[0]) | static_cast<uint32_t>(float_to_bf16_bits(acc[1])) << 16;
  v.y = float_to_bf16_bits(acc[2]) | static_cast<uint32_t>(float_to_bf16_bits(acc[3])) << 16;
  *reinterpret_cast<uint2*>(a.y + static_cast<size_t>(row) * a.N + 16 * nt + 4 * (lane / 16)) = v;
}

// A thread moves 16 codes of one column: slice `lane` of half h of tile (nt, kb).
__global__ __launch_bounds__(256) void k_fp8_pack(const uint8_t* codes, int N, int K, uint8_t* tiles) {
  const size_t t = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
  if (16 * t >= static_cast<size_t>(N) * K) return;
  const int lane = t % 64, half = t / 64 % 2;
  const size_t tile = t / 128;
  const int KB = K / 128;
  const size_t n = tile / KB * 16 + lane % 16, k = tile % KB * 128 + 64 * half + 16 * (lane / 16);
  *reinterpret_cast<uint4*>(tiles + 16 * t) = *reinterpret_cast<const uint4*>(codes + n * K + k);
}

}  // namespace

Fp8Plan fp8_plan(int M, int N, int K, bool rows8) {
  Fp8Plan p{};
  if (!rows8) p.workspace_bytes = kSplitCounterBytes + static_cast<size_t>(M) * K + static_cast<size_t>(fp8_words(K)) * M * 4;
  return p;
}

hipError_t launch_fp8_linear(const Fp8Plan& p, Fp8Args a, void* workspace, hipStream_t st) {
  if (!a.xs) {
    uint8_t* codes = static_cast<uint8_t*>(workspace) + kSplitCounterBytes;
    uint8_t* scales = codes + static_cast<size_t>(a.M) * a.K;
    const hipError_t e = launch_fp8_rows(static_cast<const uint16_t*>(a.x), a.M, a.K, codes, scales, st);
    if (e != hipSuccess) return e;
    a.x = codes;
    a.xs = reinterpret_cast<const uint32_t*>(scales);
  }
  hipLaunchKernelGGL(k_fp8_tile, dim3((a.M + 15) / 16, (a.N / 16 + 3) / 4), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_fp8_pack(const uint8_t* codes, int N, int K, uint8_t* tiles, hipStream_t st) {
  const size_t threads = static_cast<size_t>(N) * K / 16;
  hipLaunchKernelGGL(k_fp8_pack, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, st, codes, N, K, tiles);
  return hipGetLastError();
}

}  // namespace subspec
