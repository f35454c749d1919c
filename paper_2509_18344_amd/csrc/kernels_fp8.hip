// The product in 8-bit floating point:
//   y[m][n] = sum over blocks b of 2^(ex[m][b] + ew[n][b]) * sum over the block's k of x[m][k] w[n][k]
// with e4m3 codes and fp32 sums.  The scales are powers of two, so that the matrix instruction takes
// them as operands (a byte for each row of either side) and the sum over k never leaves it.
//
// The matrix units cut the products of eight neighbouring k to a grid of 2^-13 of the largest before they
// add them in fp32 (measured: 16x16x128 and 32x32x64 with scales, 16x16x32 without, all the same).  On
// rows of ordinary values that is a few 2^-14 of a result's size, a sixteenth of its rounding to bf16;
// the only way around it is 16-bit products, at half the rate and with every code converted.
#include <algorithm>

#include "fp8_device.h"
#include "kernels_fp8.h"

namespace subspec {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kFp8Waves = 8, kFp8Threads = kFp8Waves * kWave;
constexpr int kAgent = 16;  // sc1: coherent at agent scope

// A tile of MF * WM blocks of 32 rows and NF * WN blocks of 32 columns; a wavefront takes MF by NF of them.
template <int MF, int NF, int WM, int WN, int STAGES>
struct Tile {
  static_assert(WM * WN == kFp8Waves, "wavefronts of a workgroup");
  static constexpr int BM = 32 * MF * WM, BN = 32 * NF * WN;
  static constexpr int kXBytes = BM * 128, kWBytes = BN * 128;
  static constexpr int kScaleCopies = (BM + BN + kWave - 1) / kWave;
  static constexpr int kStage = kXBytes + kWBytes + 256 * kScaleCopies;  // codes and scale words of a block of k
  static constexpr int kCopies = (BM / 8 + BN / 8 + kFp8Waves - 1) / kFp8Waves;  // 1024-byte copies a wavefront
  static constexpr int kLoads = kCopies + 1;                                    // and one of scale words
  static constexpr int kAhead = STAGES - 1;
  static_assert(kScaleCopies <= kFp8Waves, "scale words of a block");
  static_assert(kAhead * kLoads < 64, "vmcnt has six bits");
  static constexpr size_t kLds = static_cast<size_t>(STAGES) * kStage + 16;
  static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
};

// One load straight into LDS: lane l's SIZE bytes land at byte dst + SIZE * l.  Written as assembly because
// the compiler, where it sees such loads, waits for all of them before it reads LDS again; it has no register
// result, and the kernel's own waits order it (a wait state after the write of m0 included).
__device__ __forceinline__ void copy16(const uint8_t* base, uint32_t offset, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void copy4(const uint32_t* from, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(dst), "v"(from) : "memory", "m0");
}

// s_waitcnt: at most `vm` vector memory operations outstanding, no LDS one.
constexpr int wait_vm_lds(int vm) { return (vm & 15) | (7 << 4) | ((vm >> 4) << 14); }
template <int VM>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(wait_vm_lds(VM));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ i32x8_t codes32(const uint8_t* lo, const uint8_t* hi) {
  const int4 a = *reinterpret_cast<const int4*>(lo), b = *reinterpret_cast<const int4*>(hi);
  return i32x8_t{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return float_to_bf16_bits(lo) | static_cast<uint32_t>(float_to_bf16_bits(hi)) << 16;
}

// Which worker has block p of the left tiles' `total` blocks: worker w's run starts at floor(w total / sharers).
__device__ __forceinline__ int sharer_of(long long p, long long total, int sharers) {
  return static_cast<int>(((p + 1) * sharers - 1) / total);
}

template <int MF, int NF, int WM, int WN, int STAGES>
__global__ __launch_bounds__(kFp8Threads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_fp8_tiles(Fp8Args a) {
  using T = Tile<MF, NF, WM, WN, STAGES>;
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int KB = a.K / 128;
  // Workgroups b, b + 8, .. run on one XCD: it takes neighbouring workers, so that its L2 serves tiles of the
  // same rows and columns.
  const int b = blockIdx.x, per = a.workers / 8, w = a.workers % 8 ? b : (b % 8) * per + b / 8;

  // --- this worker's segments: up to two cut tiles, then whole ones
  const long long total = static_cast<long long>(a.left) * KB;
  long long from = 0, to = 0;
  if (w < a.sharers) from = w * total / a.sharers, to = (w + 1) * total / a.sharers;
  const int first = static_cast<int>(from / KB), cut = to == from ? 0 : (to - 1) / KB > first ? 2 : 1;
  const int segments = cut + a.rounds;
  struct Segment {
    int tile, kb0, kb1;
  };
  auto segment = [&](int s) __attribute__((always_inline)) {
    Segment g;
    if (s >= cut) {
      g = {w + (s - cut) * a.workers, 0, KB};
    } else {
      const int t = first + s;
      const long long at = static_cast<long long>(t) * KB;
      g = {a.rounds * a.workers + t, static_cast<int>(max(from, at) - at), static_cast<int>(min(to, at + KB) - at)};
    }
    return g;
  };
  // Tiles in bands of eight along the rows, columns inside: neighbouring workers share either.
  auto place = [&](int tile, int* m0, int* n0) __attribute__((always_inline)) {
    const int band = tile / (8 * a.tiles_n), rest = tile - band * 8 * a.tiles_n, high = min(8, a.tiles_m - 8 * band);
    *n0 = rest / high * T::BN;
    *m0 = (8 * band + rest % high) * T::BM;
  };
  int steps = 0;
  for (int s = 0; s < segments; ++s) {
    const Segment g = segment(s);
    steps += g.kb1 - g.kb0;
  }
  if (!steps) return;

  // --- copies into the ring of stages
  const uint32_t ring = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)lds));
  int iseg = -1, ikb = 0, iend = 0;
  uint32_t islot = 0;
  const uint8_t *xbase = nullptr, *wbase = nullptr;
  const uint32_t* sbase = nullptr;
  long long sstep = 0;
  uint32_t offset[T::kCopies];
  auto open = [&]() __attribute__((always_inline)) {
    const Segment g = segment(++iseg);
    ikb = g.kb0;
    iend = g.kb1;
    int m0, n0;
    place(g.tile, &m0, &n0);
    xbase = static_cast<const uint8_t*>(a.x) + static_cast<size_t>(m0) * a.K + 128ll * ikb;
    wbase = a.w + static_cast<size_t>(n0) * a.K + 2048ll * ikb;
    // Rows and columns past the last: that one again (their results go nowhere).
#pragma unroll
    for (int j = 0; j < T::kCopies; ++j) {
      const int i = min(wave + kFp8Waves * j, T::BM / 8 + T::BN / 8 - 1);
      if (i < T::BM / 8) {  // eight rows of 128 codes, 16 bytes c of row r at place c ^ r: no bank twice when read
        const int r = lane / 8;
        offset[j] = static_cast<uint32_t>(min(8 * i + r, a.M - 1 - m0)) * a.K + 16 * (lane % 8 ^ r);
      } else {
        const int u = i - T::BM / 8;
        offset[j] = static_cast<uint32_t>(min(u / 2, a.N / 16 - 1 - n0 / 16)) * 16 * a.K + 1024 * (u % 2) + 16 * lane;
      }
    }
    const int v = kWave * min(wave, T::kScaleCopies - 1) + lane;
    const bool of_x = v < T::BM;
    sbase = of_x ? a.xs + min(m0 + v, a.M - 1) : a.ws + min(n0 + min(v - T::BM, T::BN - 1), a.N - 1);
    sstep = of_x ? a.M : a.N;
    sbase += sstep * (ikb / 4);
  };
  auto issue = [&]() __attribute__((always_inline)) {
    if (ikb == iend) open();
    const uint32_t at = ring + islot * T::kStage;
#pragma unroll
    for (int j = 0; j < T::kCopies; ++j) {
      const int i = min(wave + kFp8Waves * j, T::BM / 8 + T::BN / 8 - 1);
      copy16(i < T::BM / 8 ? xbase : wbase, offset[j], at + 1024 * i);
    }
    copy4(sbase, at + T::kXBytes + T::kWBytes + 256 * min(wave, T::kScaleCopies - 1));
    xbase += 128;
    wbase += 2048;
    if (++ikb % 4 == 0) sbase += sstep;
    islot = islot + 1 == STAGES ? 0 : islot + 1;
  };
  int issued = 0;
  for (; issued < T::kAhead && issued < steps; ++issued) issue();

  // --- products
  const int r = lane % 32, half = lane / 32, wm = wave % WM, wn = wave / WM;
  uint32_t xat[4];  // 16 bytes 4 s + 2 half + t of row r
#pragma unroll
  for (int u = 0; u < 4; ++u) xat[u] = (32 * MF * wm + r) * 128 + 16 * ((4 * (u / 2) + 2 * half + u % 2) ^ (r % 8));
  const uint32_t wat = T::kXBytes + 32 * NF * wn * 128 + r / 16 * 2048 + 512 * half + 16 * (r % 16);
  const uint32_t xsat = T::kXBytes + T::kWBytes + 4 * (32 * MF * wm + r), wsat = T::kXBytes + T::kWBytes + 4 * (T::BM + 32 * NF * wn + r);
  f32x16_t acc[NF][MF];
  int step = 0;
  uint32_t slot = 0;
  for (int s = 0; s < segments; ++s) {
    const Segment g = segment(s);
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
      for (int j = 0; j < MF; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    for (int kb = g.kb0; kb < g.kb1; ++kb, ++step) {
      // Loads complete in order: once the later stages' are all that is outstanding, this stage is in LDS; the
      // stage before it is read by everyone and takes the next copies.
      if (step + T::kAhead <= steps) wait_and_meet<(T::kAhead - 1) * T::kLoads>();
      else wait_and_meet<0>();
      if (issued < steps) issue(), ++issued;
      const uint8_t* st = lds + slot * T::kStage;
      uint32_t xs[MF], ws[NF];
#pragma unroll
      for (int j = 0; j < MF; ++j) xs[j] = st[xsat + 128 * j + kb % 4];
#pragma unroll
      for (int i = 0; i < NF; ++i) ws[i] = st[wsat + 128 * i + kb % 4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        i32x8_t wf[NF], xf[MF];
#pragma unroll
        for (int i = 0; i < NF; ++i) wf[i] = codes32(st + wat + 4096 * i + 1024 * h, st + wat + 4096 * i + 1024 * h + 256);
#pragma unroll
        for (int j = 0; j < MF; ++j) xf[j] = codes32(st + xat[2 * h] + 4096 * j, st + xat[2 * h + 1] + 4096 * j);
#pragma unroll
        for (int j = 0; j < MF; ++j)
#pragma unroll
          for (int i = 0; i < NF; ++i)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[i], xf[j], acc[i][j], 0, 0, 0, static_cast<int>(ws[i]), 0,
                                                                       static_cast<int>(xs[j]));
      }
      slot = slot + 1 == STAGES ? 0 : slot + 1;
    }

    int m0, n0;
    place(g.tile, &m0, &n0);
    if (g.kb1 - g.kb0 < KB) {
      // Partial sums in the accumulators' order.  Every worker of the tile stores its own with agent-scope
      // stores and counts itself in once they are acknowledged; the last adds them in the order of k.
      const int t = g.tile - a.rounds * a.workers;
      constexpr uint32_t kPart = T::BM * T::BN * 4;
      auto part = [&](int who, int seg) __attribute__((always_inline)) {
        return buffer_rsrc(reinterpret_cast<const uint8_t*>(a.part) + static_cast<size_t>(2 * who + seg) * kPart, kPart);
      };
      const __amdgpu_buffer_rsrc_t mine = part(w, s);
#pragma unroll
      for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int j = 0; j < MF; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            __builtin_amdgcn_raw_buffer_store_b128(
                __builtin_bit_cast(u32x4_t, f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]}), mine,
                16 * threadIdx.x, ((i * MF + j) * 4 + q) * 16 * kFp8Threads, kAgent);
      int* last = reinterpret_cast<int*>(lds + static_cast<size_t>(STAGES) * T::kStage);
      wait_and_meet<0>();
      const int w0 = sharer_of(static_cast<long long>(t) * KB, total, a.sharers);
      const int w1 = sharer_of(static_cast<long long>(t) * KB + KB - 1, total, a.sharers);
      if (threadIdx.x == 0)
        *last = __hip_atomic_fetch_add(a.count + t, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<unsigned>(w1 - w0);
      __syncthreads();
      if (!*last) continue;
      for (int who = w0; who <= w1; ++who) {
        // the tile is the first of a worker's run or its second
        const __amdgpu_buffer_rsrc_t from_part = part(who, static_cast<int>(who * total / a.sharers / KB) == t ? 0 : 1);
#pragma unroll
        for (int i = 0; i < NF; ++i)
#pragma unroll
          for (int j = 0; j < MF; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x4_t v = __builtin_bit_cast(
                  f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from_part, 16 * threadIdx.x, ((i * MF + j) * 4 + q) * 16 * kFp8Threads, kAgent));
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] = who == w0 ? v[e] : acc[i][j][4 * q + e] + v[e];
            }
      }
      if (threadIdx.x == 0) __hip_atomic_store(a.count + t, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // A lane holds columns 8 q + 4 half + 0 .. 3 of one row; swapped with the other half's, 8 in a row.
#pragma unroll
    for (int j = 0; j < MF; ++j) {
      const int m = m0 + 32 * (MF * wm + j) + r;
#pragma unroll
      for (int i = 0; i < NF; ++i) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const int n = n0 + 32 * (NF * wn + i) + 16 * p;
          const f32x16_t& c = acc[i][j];
          const auto lo = __builtin_amdgcn_permlane32_swap(pack_bf16(c[8 * p], c[8 * p + 1]), pack_bf16(c[8 * p + 4], c[8 * p + 5]), false, false);
          const auto hi = __builtin_amdgcn_permlane32_swap(pack_bf16(c[8 * p + 2], c[8 * p + 3]), pack_bf16(c[8 * p + 6], c[8 * p + 7]), false, false);
          if (m < a.M && n < a.N)
            *reinterpret_cast<uint4*>(a.y + static_cast<size_t>(m) * a.N + n + 8 * half) = make_uint4(lo[0], hi[0], lo[1], hi[1]);
        }
      }
    }
  }
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

constexpr int kFewRows = 64;   // up to here kernels_fp8_few.hip
constexpr int kColumns = 256;  // of every tile

template <int MF, int NF, int WM, int WN, int STAGES>
hipError_t tiles_at(const Fp8Args& a, hipStream_t st) {
  using T = Tile<MF, NF, WM, WN, STAGES>;
  static_assert(T::BN == kColumns, "columns of a tile");
  static const hipError_t set = hipFuncSetAttribute(reinterpret_cast<const void*>(&k_fp8_tiles<MF, NF, WM, WN, STAGES>),
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, T::kLds);
  if (set != hipSuccess) return set;
  hipLaunchKernelGGL((k_fp8_tiles<MF, NF, WM, WN, STAGES>), dim3(a.workers), dim3(kFp8Threads), T::kLds, st, a);
  return hipGetLastError();
}

size_t fp8_row_bytes(int M, int K) {
  return (static_cast<size_t>(M) * K + static_cast<size_t>(fp8_words(K)) * M * 4 + 255) & ~size_t(255);
}

}  // namespace

Fp8Plan fp8_plan(int M, int N, int K, bool rows8, int cus) {
  Fp8Plan p{};
  if (M <= kFewRows) {
    const int tiles = N / 16, units = (K + 255) / 256;
    p.few = tiles >= 4 * cus ? 2 : 1;
    p.waves = M > 16 || tiles > cus ? 4 : 8;
    const int sets = (tiles + p.few - 1) / p.few, rows = (M + 15) / 16;
    p.splits = std::max(1, std::min({(p.waves == 4 ? 4 : 1) * cus / sets, units / (4 * p.waves), 64}));
    size_t at = kSplitCounterBytes;
    if (!rows8 && M > 16) at += p.code_bytes = fp8_row_bytes(M, K);
    if (p.splits > 1) at += static_cast<size_t>(sets) * p.splits * rows * p.few * kWave * 16;
    p.workspace_bytes = at > kSplitCounterBytes ? at : 0;
    return p;
  }
  p.rows = M <= 128 ? 128 : 256;
  const long long tiles = static_cast<long long>((M + p.rows - 1) / p.rows) * ((N + kColumns - 1) / kColumns);
  const long long KB = K / 128;
  p.rounds = static_cast<int>(tiles / cus);
  p.left = static_cast<int>(tiles % cus);
  p.sharers = static_cast<int>(std::min<long long>(cus, p.left * KB));
  p.workers = p.rounds ? cus : p.sharers;
  size_t at = kSplitCounterBytes;
  if (!rows8) at += p.code_bytes = fp8_row_bytes(M, K);
  if (p.sharers > p.left) at += static_cast<size_t>(p.sharers) * 2 * p.rows * kColumns * 4;
  p.workspace_bytes = at > kSplitCounterBytes ? at : 0;
  return p;
}

hipError_t launch_fp8_linear(const Fp8Plan& p, Fp8Args a, void* workspace, hipStream_t st) {
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  if (p.code_bytes) {
    uint8_t* codes = ws + kSplitCounterBytes;
    uint8_t* scales = codes + static_cast<size_t>(a.M) * a.K;
    const hipError_t e = launch_fp8_rows(static_cast<const uint16_t*>(a.x), a.M, a.K, codes, scales, st);
    if (e != hipSuccess) return e;
    a.x = codes;
    a.xs = reinterpret_cast<const uint32_t*>(scales);
  }
  if (ws) {
    a.count = reinterpret_cast<unsigned*>(ws);
    a.part = reinterpret_cast<float*>(ws + kSplitCounterBytes + p.code_bytes);
  }
  if (p.few) {
    a.splits = p.splits;
    return launch_fp8_few(a, p.few, p.waves, st);
  }
  a.tiles_m = (a.M + p.rows - 1) / p.rows;
  a.tiles_n = (a.N + kColumns - 1) / kColumns;
  a.workers = p.workers;
  a.rounds = p.rounds;
  a.left = p.left;
  a.sharers = p.sharers;
  switch (p.rows) {
    case 128: return tiles_at<4, 1, 1, 8, 3>(a, st);
    default: return tiles_at<4, 2, 2, 4, 2>(a, st);
  }
}

hipError_t launch_fp8_pack(const uint8_t* codes, int N, int K, uint8_t* tiles, hipStream_t st) {
  const size_t threads = static_cast<size_t>(N) * K / 16;
  hipLaunchKernelGGL(k_fp8_pack, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, st, codes, N, K, tiles);
  return hipGetLastError();
}

}  // namespace subspec
