// Preparation of one layer's queries, keys and values from the rows of the fused q|k|v
// projection: bias, an RMS norm of every query and key head and the position rotation, in
// one pass over the row.
//
//   x = row + bias;  q, k heads: x <- x / sqrt(mean(x^2) + eps) * w;  then each pair
//   (a, b) of rotated dimensions i: (a cos t - b sin t, b cos t + a sin t),
//   t = position * inv_freq[i].
//
// A workgroup takes one token and 16 heads, 16 lanes of 8 dimensions (16 bytes) a head: a
// norm is four DPP additions within a row of lanes, and the partner of a pair is a lane of
// the same row.  Its first rot / 2 threads compute the token's angles once, in LDS for all
// heads.
#include "rope_device.h"

namespace subspec {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeHeads = kRopeThreads / 16;

__global__ __launch_bounds__(kRopeThreads) void k_qkv_rope(RopeArgs a) {
  __shared__ float2 cs[kRopeHalf];
  const int i = blockIdx.x;
  const int col = threadIdx.x % 16, h = blockIdx.y * kRopeHeads + threadIdx.x / 16;
  const int heads = a.Hq + 2 * a.Hkv;
  const bool live = h < heads;
  uint4 row = make_uint4(0, 0, 0, 0), bias = make_uint4(0, 0, 0, 0);
  if (live) {
    row = *reinterpret_cast<const uint4*>(a.qkv + static_cast<size_t>(i) * a.ld + h * kRopeD + 8 * col);
    if (a.bias) bias = *reinterpret_cast<const uint4*>(a.bias + h * kRopeD + 8 * col);
  }
  if (static_cast<int>(threadIdx.x) < a.rot / 2) cs[threadIdx.x] = rope_cos_sin(a.positions[i], a.inv_freq[threadIdx.x]);
  __syncthreads();
  float x[8];
  unpack8(row, x);
  if (a.bias) {
    float b[8];
    unpack8(bias, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += b[e];
  }
  const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
  // the 16 lanes of a head agree on every branch
  if (is_q || is_k) rope_row(x, col, is_q ? a.q_weight : a.k_weight, a.eps, a.rot, a.interleaved, cs);
  if (!live) return;
  uint16_t* dst = is_q ? a.q + (static_cast<size_t>(i) * a.Hq + h) * kRopeD
                 : is_k ? a.k + (static_cast<size_t>(i) * a.Hkv + (h - a.Hq)) * kRopeD
                        : a.v + (static_cast<size_t>(i) * a.Hkv + (h - a.Hq - a.Hkv)) * kRopeD;
  *reinterpret_cast<uint4*>(dst + 8 * col) = pack8(x);
}

}  // namespace

hipError_t launch_qkv_rope(const RopeArgs& a, hipStream_t st) {
  const int heads = a.Hq + 2 * a.Hkv;
  hipLaunchKernelGGL(k_qkv_rope, dim3(a.M, (heads + kRopeHeads - 1) / kRopeHeads), dim3(kRopeThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace subspec
