// Preparation of one layer's queries, keys and values from the rows of the fused q|k|v
// projection: bias, an RMS norm of every query and key head and the position rotation, in
// one pass over the row.
//
//   x = row + bias;  q, k heads: x <- x / sqrt(mean(x^2) + eps) * w;  then each pair
//   (a, b) of rotated dimensions i: (a cos t - b sin t, b cos t + a sin t),
//   t = position * inv_freq[i].
//
// A workgroup takes one token: 16 lanes of 8 dimensions (16 bytes) a head, 16 heads at a time, so
// a norm is four DPP additions within a row of lanes and the partner of a pair a lane of the
// same row.  Its first rot / 2 threads compute the token's angles once, in LDS, and a lane holds
// those of its dimensions for all heads.  Few tokens: a workgroup for every 16 heads
// instead, so that their loads are all in flight.
//
// Measured: 4096 tokens of 56 heads with bias and norms 25.2 us, 117 MB at 4.7 TB/s, where a large
// copy moves 5.5: bound by memory.  One token 2.4 us, of which a launch that does nothing is about
// 2; a call from Python costs 6.6.
#include "rope_device.h"

namespace subspec {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeHeads = kRopeThreads / 16;
// Tokens from which a workgroup takes all heads of its token (56 heads: 128 tokens 3.6 us against 3.1 in
// workgroups of 16 heads, 256 4.1 against 4.0, 400 5.0 against 5.5, 4096 24 against 40).
constexpr int kRopeWhole = 320;
constexpr int kRopeAhead = 4;  // head rows of a thread in flight

template <bool FULL>
__global__ __launch_bounds__(kRopeThreads) void k_qkv_rope(RopeArgs a) {
  __shared__ float2 cs[kRopeHalf];
  const int i = blockIdx.x;
  const int col = threadIdx.x % 16, h0 = blockIdx.y * kRopeHeads + threadIdx.x / 16, step = gridDim.y * kRopeHeads;
  const int heads = a.Hq + 2 * a.Hkv;
  const uint16_t* src = a.qkv + static_cast<size_t>(i) * a.ld + 8 * col;
  uint4 row[kRopeAhead], bias[kRopeAhead];
  auto request = [&](int h) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kRopeAhead; ++u) {
      const int at = min(h + u * step, heads - 1) * kRopeD;  // (past the last head: that one again)
      row[u] = *reinterpret_cast<const uint4*>(src + at);
      bias[u] = a.bias ? *reinterpret_cast<const uint4*>(a.bias + at + 8 * col) : make_uint4(0, 0, 0, 0);
    }
  };
  request(h0);
  uint4 qw = make_uint4(0, 0, 0, 0), kw = qw;
  if (a.q_weight) qw = *reinterpret_cast<const uint4*>(a.q_weight + 8 * col);
  if (a.k_weight) kw = *reinterpret_cast<const uint4*>(a.k_weight + 8 * col);
  if (static_cast<int>(threadIdx.x) < a.rot / 2) cs[threadIdx.x] = rope_cos_sin(a.positions[i], a.inv_freq[threadIdx.x]);
  __syncthreads();
  RopeTurn turn{};
  if (a.rot) turn = rope_turn(col, a.rot, FULL ? 0 : a.interleaved, cs);
  for (int h1 = h0; h1 < heads; h1 += kRopeAhead * step) {
    if (h1 > h0) request(h1);
#pragma unroll
    for (int u = 0; u < kRopeAhead; ++u) {
      const int h = h1 + u * step;
      if (h >= heads) break;
      float x[8];
      unpack8(row[u], x);
      if (a.bias) {
        float b[8];
        unpack8(bias[u], b);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += b[e];
      }
      // the 16 lanes of a head agree on every branch
      const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
      if (is_q ? a.q_weight != nullptr : is_k && a.k_weight != nullptr) {
        float w[8];
        unpack8(is_q ? qw : kw, w);
        rope_norm(x, w, a.eps);
      }
      if (is_q || is_k) {
        if (FULL || a.rot) rope_rotate<FULL>(x, col, a.rot, a.interleaved, turn);
      }
      uint16_t* dst = is_q ? a.q + (static_cast<size_t>(i) * a.Hq + h) * kRopeD
                     : is_k ? a.k + (static_cast<size_t>(i) * a.Hkv + (h - a.Hq)) * kRopeD
                            : a.v + (static_cast<size_t>(i) * a.Hkv + (h - a.Hq - a.Hkv)) * kRopeD;
      *reinterpret_cast<uint4*>(dst + 8 * col) = pack8(x);
    }
  }
}

}  // namespace

hipError_t launch_qkv_rope(const RopeArgs& a, hipStream_t st) {
  const int blocks = (a.Hq + 2 * a.Hkv + kRopeHeads - 1) / kRopeHeads;
  const dim3 grid(a.M, a.M < kRopeWhole ? blocks : 1);
  if (a.rot == kRopeD && !a.interleaved)
    hipLaunchKernelGGL(k_qkv_rope<true>, grid, dim3(kRopeThreads), 0, st, a);
  else
    hipLaunchKernelGGL(k_qkv_rope<false>, grid, dim3(kRopeThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace subspec
