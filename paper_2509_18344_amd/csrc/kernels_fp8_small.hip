// The product in 8-bit floating point where tiles are few: a workgroup takes one smaller tile, or a run of its
// K, and its wavefronts cut every stage's blocks of k among them too, so that a short tile still keeps all its
// wavefronts busy and most of the sums over K meet in LDS.
//
// A step costs a round trip of its copies (0.6 us) while few compute units have one, then their bytes: 66 KB
// a compute unit in 1.4 us, 12 TB/s out of L2 (64 x 64); with exact products (up to 64 rows) the conversion
// of codes to bf16, 1.5 us for 64 x 128 x 256.  Measured: 289 rows, 7168 x 5120: 24.6 us in 224 workgroups of
// 96 x 128, where 128 x 128 takes 30 in 168 and large tiles of 128 x 256 with K in two 30; 49 rows, 3584 x 18944:
// 22.7 us in 224 workgroups of 64 x 64, four a tile (37 in large tiles); 32 rows, 55296 x 5120: 52.5 us, 5.4 TB/s
// of weights, with two workgroups a compute unit, whose starts and ends overlap (59 with one).
#include <algorithm>

#include "fp8_tile.h"

namespace subspec {

namespace {

// WM by WN by WK wavefronts, four or eight: MF blocks of 32 rows and NF of 32 columns each, one of WK blocks of k of a stage.
template <int MF, int NF, int WM, int WN, int WK, int STAGES>
struct SmallTile {
  static constexpr int WAVES = WM * WN * WK, THREADS = WAVES * kWave;
  static constexpr int BM = 32 * MF * WM, BN = 32 * NF * WN;
  static constexpr int kXBytes = BM * 128, kWBytes = BN * 128, kWords = (BM + BN + kWave - 1) / kWave;
  static constexpr int kBlock = kXBytes + kWBytes + 256 * kWords;  // codes and scale words of a block of k
  static constexpr int kStage = WK * kBlock;
  static constexpr int kRuns = BM / 8 + BN / 8;  // 1024-byte copies of a block
  static constexpr int kCopies = WK * kRuns / WAVES, kWordCopies = (WK * kWords + WAVES - 1) / WAVES;
  static_assert(WK * kRuns % WAVES == 0, "copies of a stage");
  static constexpr int kLoads = kCopies + kWordCopies, kAhead = STAGES - 1;
  static_assert(kAhead * kLoads < 64, "vmcnt has six bits");
  static constexpr size_t kSums = static_cast<size_t>(WK - 1) * BM * BN * 4;
  static constexpr size_t kLds = (static_cast<size_t>(STAGES) * kStage > kSums ? static_cast<size_t>(STAGES) * kStage : kSums) + 16;
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
};

template <int MF, int NF, int WM, int WN, int WK, int STAGES, bool EXACT>
__global__ __launch_bounds__(WM * WN * WK * kWave) __attribute__((amdgpu_waves_per_eu(2, 4))) void k_fp8_small(Fp8Args a) {
  using T = SmallTile<MF, NF, WM, WN, WK, STAGES>;
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int KB = a.K / 128, units = (KB + WK - 1) / WK;
  // Workgroups b, b + 8, .. run on one XCD: it takes neighbouring tiles.
  const int b = blockIdx.x, count = gridDim.x, at = count % 8 ? b : b % 8 * (count / 8) + b / 8;
  const int tile = at / a.splits, split = at % a.splits;
  const int m0 = tile % a.tiles_m * T::BM, n0 = tile / a.tiles_m * T::BN;
  const int u0 = static_cast<int>(static_cast<long long>(split) * units / a.splits), u1 = static_cast<int>(static_cast<long long>(split + 1) * units / a.splits);
  const int steps = u1 - u0;

  // --- copies into the ring of stages.  Rows, columns and blocks past the last: that one again.
  const uint32_t ring = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)lds));
  const uint8_t* xbase = static_cast<const uint8_t*>(a.x) + static_cast<size_t>(m0) * a.K;
  const uint8_t* wbase = a.w + static_cast<size_t>(n0) * a.K;
  uint32_t offset[T::kCopies];
#pragma unroll
  for (int j = 0; j < T::kCopies; ++j) {
    const int i = (wave + T::WAVES * j) % T::kRuns;
    if (i < T::BM / 8) {
      offset[j] = static_cast<uint32_t>(min(8 * i + lane / 8, a.M - 1 - m0)) * a.K + fp8_chunk(lane, i);
    } else {
      const int u = i - T::BM / 8;
      offset[j] = static_cast<uint32_t>(min(u / 2, a.N / 16 - 1 - n0 / 16)) * 16 * a.K + 1024 * (u % 2) + 16 * lane;
    }
  }
  const uint32_t* sbase[T::kWordCopies];
  uint32_t sstep[T::kWordCopies];
#pragma unroll
  for (int j = 0; j < T::kWordCopies; ++j) {
    const int v = kWave * (min(wave + T::WAVES * j, WK * T::kWords - 1) % T::kWords) + lane;
    const bool of_x = v < T::BM;
    sbase[j] = of_x ? a.xs + min(m0 + v, a.M - 1) : a.ws + min(n0 + min(v - T::BM, T::BN - 1), a.N - 1);
    sstep[j] = of_x ? a.M : a.N;
  }
  auto issue = [&](int unit, uint32_t slot) __attribute__((always_inline)) {
    const uint32_t to = ring + slot * T::kStage;
#pragma unroll
    for (int j = 0; j < T::kCopies; ++j) {
      const int c = wave + T::WAVES * j, k = c / T::kRuns, i = c % T::kRuns, kb = min(unit * WK + k, KB - 1);
      if (i < T::BM / 8) copy16<false>(xbase + 128ll * kb, offset[j], to + k * T::kBlock + 1024 * i);
      else copy16<(EXACT && MF == 1)>(wbase + 2048ll * kb, offset[j], to + k * T::kBlock + 1024 * i);
    }
#pragma unroll
    for (int j = 0; j < T::kWordCopies; ++j) {
      const int c = min(wave + T::WAVES * j, WK * T::kWords - 1), k = c / T::kWords, kb = min(unit * WK + k, KB - 1);
      copy4(sbase[j] + static_cast<size_t>(kb / 4) * sstep[j], to + k * T::kBlock + T::kXBytes + T::kWBytes + 256 * (c % T::kWords));
    }
  };
  int issued = 0;
  for (; issued < T::kAhead && issued < steps; ++issued) issue(u0 + issued, issued);

  // --- products
  const Fp8Lane l = fp8_lane(lane);
  const int half = lane / 32, team = wave % (WM * WN), wk = wave / (WM * WN), wm = team % WM, wn = team / WM;
  f32x16_t acc[NF][MF];
  fp8_clear(acc);
  uint32_t slot = 0;
  for (int t = 0; t < steps; ++t) {
    if (t + T::kAhead <= steps) wait_and_meet<(T::kAhead - 1) * T::kLoads>();
    else wait_and_meet<0>();
    if (issued < steps) {
      issue(u0 + issued, slot == 0 ? STAGES - 1 : slot - 1);  // the stage that everyone has read
      ++issued;
    }
    const int kb = (u0 + t) * WK + wk;
    if (kb < KB) {
      const uint8_t* st = lds + slot * T::kStage + wk * T::kBlock;
      const uint8_t* words = st + T::kXBytes + T::kWBytes;
      fp8_block_products<MF, NF, EXACT>(acc, st + 4096 * MF * wm, st + T::kXBytes + 4096 * NF * wn, words + 128 * MF * wm,
                                        words + 4 * T::BM + 128 * NF * wn, l, half, kb % 4);
    }
    slot = slot + 1 == STAGES ? 0 : slot + 1;
  }

  // --- the wavefronts' sums in the order of their blocks
  if constexpr (WK > 1) {
    f32x4_t* sums = reinterpret_cast<f32x4_t*>(lds);
    __syncthreads();
    if (wk > 0) {
#pragma unroll
      for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int j = 0; j < MF; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            sums[((((wk - 1) * WM * WN + team) * NF * MF + i * MF + j) * 4 + q) * kWave + lane] =
                f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    }
    __syncthreads();
    if (wk == 0) {
#pragma unroll
      for (int k = 0; k < WK - 1; ++k)
#pragma unroll
        for (int i = 0; i < NF; ++i)
#pragma unroll
          for (int j = 0; j < MF; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x4_t v = sums[(((k * WM * WN + team) * NF * MF + i * MF + j) * 4 + q) * kWave + lane];
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += v[e];
            }
    }
  }
  if (a.splits > 1) {
    // Agent-scope stores, counted in once they are acknowledged; the tile's last workgroup adds all of K in order.
    constexpr uint32_t kPart = T::BM * T::BN * 4, kThreads = kWave * WM * WN;
    auto part = [&](int k) __attribute__((always_inline)) {
      return buffer_rsrc(reinterpret_cast<const uint8_t*>(a.part) + (static_cast<size_t>(tile) * a.splits + k) * kPart, kPart);
    };
    int* last = reinterpret_cast<int*>(lds + T::kLds - 16);
    if (wk == 0) fp8_store_part(acc, part(split), kWave * team + lane, kThreads);
    wait_and_meet<0>();
    if (threadIdx.x == 0)
      *last = __hip_atomic_fetch_add(a.count + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<unsigned>(a.splits - 1);
    __syncthreads();
    if (!*last) return;
    if (wk == 0) fp8_add_parts(acc, a.splits, part, kWave * team + lane, kThreads);
    if (threadIdx.x == 0) __hip_atomic_store(a.count + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (wk == 0) fp8_results(acc, a, m0 + 32 * MF * wm, n0 + 32 * NF * wn, lane);
}

template <int MF, int NF, int WM, int WN, int WK, int STAGES, bool EXACT>
hipError_t small_at(Fp8Args a, hipStream_t st) {
  using T = SmallTile<MF, NF, WM, WN, WK, STAGES>;
  a.tiles_m = (a.M + T::BM - 1) / T::BM;
  a.tiles_n = (a.N + T::BN - 1) / T::BN;
  hipLaunchKernelGGL((k_fp8_small<MF, NF, WM, WN, WK, STAGES, EXACT>), dim3(a.tiles_m * a.tiles_n * a.splits), dim3(T::THREADS), T::kLds, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_fp8_small(const Fp8Args& a, int kind, hipStream_t st) {
  switch (kind) {
    case 1: return small_at<1, 1, 1, 2, 4, 3, true>(a, st);   // 32 x 64
    case 2: return small_at<2, 1, 1, 2, 4, 2, true>(a, st);   // 64 x 64
    case 3: return small_at<2, 1, 1, 4, 2, 3, true>(a, st);   // 64 x 128
    case 4: return small_at<2, 1, 1, 2, 4, 2, false>(a, st);  // 64 x 64
    case 5: return small_at<2, 1, 1, 4, 2, 3, false>(a, st);  // 64 x 128
    case 6: return small_at<3, 1, 1, 4, 2, 2, false>(a, st);  // 96 x 128
    case 7: return small_at<2, 1, 2, 4, 1, 4, false>(a, st);  // 128 x 128
    default: return small_at<1, 1, 1, 2, 2, 3, true>(a, st);   // 32 x 64, four wavefronts, two workgroups a compute unit
  }
}

}  // namespace subspec
