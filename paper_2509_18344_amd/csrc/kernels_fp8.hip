// The product in 8-bit floating point:
//   y[m][n] = sum over blocks b of 2^(ex[m][b] + ew[n][b]) * sum over the block's k of x[m][k] w[n][k]
// with e4m3 codes and fp32 sums.  The scales are powers of two, so that the matrix instruction takes
// them as operands (a byte for each row of either side) and the sum over k never leaves it.
//
// The matrix units cut the products of eight neighbouring k to a grid of 2^-13 of the largest before they
// add them in fp32 (measured: 16x16x128 and 32x32x64 with scales, 16x16x32 without, all the same).  On
// rows of ordinary values that moves sums by 1.6e-5 of their size (2-norm; by 7e-5 to 1e-4 where every 8th to 1024th
// channel of x is 100 to 10000 times larger), so that one result in 80 rounds to the neighbouring bf16 number: 2.2e-4
// to 3.3e-4 of the results' size, next to 1.7e-3 of the rounding itself.  The only way around it is 16-bit products, at half
// the rate and with every code converted.  Up to 64 rows, where the weights' bytes bound the call, that is what runs
// (EXACT; 64 rows, 55296 x 5120: 67 us, 4.2 TB/s of weights); more rows run so on request, in the same tiles: 128 rows
// 116 us (65 with 8-bit products), 289 rows, 7168 x 5120, 46 (28), 4096 rows, 55296 x 5120, 2918 (1033).
//
// This file: large tiles, by workgroups that take several each.  Both sides go through a ring in LDS, copied
// straight from memory: a tile of 256 x 256 reads 64 KB for 16.8 MFLOP, eight wavefronts of 128 x 64.  4096
// rows, 55296 x 5120: 1043 to 1059 us in a trace, 2190 to 2220 TFLOP/s (1030 to 1080 a call, over several machines), where
// a large library product of these sizes runs at 2290 to 2340; the matrix units are busy 53 % of the cycles.  A step takes
// 1.9 us, without its copies 1.4 (769 us in all), without its reads of LDS as long as with them.  LDS holds two stages,
// so that one step's 64 KB a compute unit are on their way at a time and are waited for whole: their latency is not
// hidden.  (12 TB/s, what smaller tiles draw from L2, would move them in 1.4 us.)  Tried against 1055: half blocks of k,
// four in flight, reads and copies spread between the products by hand 1048 to 1084; lines brought into L2
// ahead of their copies 1036 to 1067; bands of 2, 4 and 16 tiles of rows 1100, 1078 and 1069.
#include <algorithm>

#include "fp8_tile.h"

namespace subspec {

namespace {

// A tile of MF * WM blocks of 32 rows and NF * WN blocks of 32 columns; a wavefront takes MF by NF of them.
// STAGES blocks of k are in LDS or on their way.
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

template <int MF, int NF, int WM, int WN, int STAGES, bool EXACT>
__global__ __launch_bounds__(kFp8Threads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_fp8_tiles(Fp8Args a) {
  using T = Tile<MF, NF, WM, WN, STAGES>;
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const Fp8Work work(a);
  const int steps = work.blocks();
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
    const Fp8Segment g = work.segment(++iseg);
    ikb = g.kb0;
    iend = g.kb1;
    int m0, n0;
    fp8_place(a, g.tile, T::BM, T::BN, &m0, &n0);
    xbase = static_cast<const uint8_t*>(a.x) + static_cast<size_t>(m0) * a.K + 128ll * ikb;
    wbase = a.w + static_cast<size_t>(n0) * a.K + 2048ll * ikb;
    // Rows and columns past the last: that one again (their results go nowhere).
#pragma unroll
    for (int j = 0; j < T::kCopies; ++j) {
      const int i = min(wave + kFp8Waves * j, T::BM / 8 + T::BN / 8 - 1);
      if (i < T::BM / 8) {
        offset[j] = static_cast<uint32_t>(min(8 * i + lane / 8, a.M - 1 - m0)) * a.K + fp8_chunk(lane, i);
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
      if (i < T::BM / 8) copy16<false>(xbase, offset[j], at + 1024 * i);
      else copy16<(EXACT && MF == 1)>(wbase, offset[j], at + 1024 * i);
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
  const Fp8Lane at = fp8_lane(lane);
  const int half = lane / 32, wm = wave % WM, wn = wave / WM;
  f32x16_t acc[NF][MF];
  int step = 0;
  uint32_t slot = 0;
  for (int s = 0; s < work.segments; ++s) {
    const Fp8Segment g = work.segment(s);
    fp8_clear(acc);
    for (int kb = g.kb0; kb < g.kb1; ++kb, ++step) {
      // Loads complete in order: once the later stages' are all that is outstanding, this stage is in LDS; the
      // stage before it is read by everyone and takes the next copies.
      if (step + T::kAhead <= steps) wait_and_meet<(T::kAhead - 1) * T::kLoads>();
      else wait_and_meet<0>();
      if (issued < steps) issue(), ++issued;
      const uint8_t* st = lds + slot * T::kStage;
      const uint8_t* words = st + T::kXBytes + T::kWBytes;
      fp8_block_products<MF, NF, EXACT>(acc, st + 4096 * MF * wm, st + T::kXBytes + 4096 * NF * wn, words + 128 * MF * wm,
                                        words + 4 * T::BM + 128 * NF * wn, at, half, kb % 4);
      slot = slot + 1 == STAGES ? 0 : slot + 1;
    }

    int m0, n0;
    fp8_place(a, g.tile, T::BM, T::BN, &m0, &n0);
    if (g.kb1 - g.kb0 < work.KB &&
        !fp8_join(acc, a, work, s, g.tile, T::BM * T::BN * 4, reinterpret_cast<int*>(lds + static_cast<size_t>(STAGES) * T::kStage)))
      continue;
    fp8_results(acc, a, m0 + 32 * MF * wm, n0 + 32 * NF * wn, lane);
  }
}

// A thread moves 16 codes of one column: slice `lane` of half h of tile (nt, kb), two tiles a workgroup.  5120 x 27648:
// 56.5 us, 5.0 TB/s read and written, a copy's rate; with the rows to codes before it 139 us a weight.
__global__ __launch_bounds__(256) void k_fp8_pack(const uint8_t* codes, int K, uint8_t* tiles) {
  const int nt = blockIdx.x, KB = K / 128, kb = blockIdx.y * 2 + threadIdx.x / 128;
  if (kb >= KB) return;
  const int lane = threadIdx.x % 64, half = threadIdx.x / 64 % 2;
  const size_t n = static_cast<size_t>(nt) * 16 + lane % 16, k = static_cast<size_t>(kb) * 128 + 64 * half + 16 * (lane / 16);
  *reinterpret_cast<uint4*>(tiles + (static_cast<size_t>(nt) * KB + kb) * 2048 + 1024 * half + 16 * lane) =
      *reinterpret_cast<const uint4*>(codes + n * K + k);
}

constexpr int kColumns = 256;  // of every tile

template <int MF, int NF, int WM, int WN, int STAGES, bool EXACT>
hipError_t tiles_at(const Fp8Args& a, hipStream_t st) {
  using T = Tile<MF, NF, WM, WN, STAGES>;
  static_assert(T::BN == kColumns, "columns of a tile");
  hipLaunchKernelGGL((k_fp8_tiles<MF, NF, WM, WN, STAGES, EXACT>), dim3(a.workers), dim3(kFp8Threads), T::kLds, st, a);
  return hipGetLastError();
}

// What the launches cost, in microseconds: a call; a workgroup's stage of k when few compute units have one and
// when all do, its end, and a start after another's end; joining parts of K, first in a launch or ahead of whole
// tiles: trips to memory one after the other, and bytes, written and read, cheaper while they stay in the last
// cache; a kind's bytes of weights from memory, and of weights that two tiles of rows read one after the other.
// Fitted to sweeps of every shape: the choice below, the cheapest by them, lost 3.9 % to the best over 105 other
// sizes (geometric mean; over 10 % at nine of them, 39 % at most: 1298 rows, 1696 x 13312, 68 us where large tiles of 128
// rows take 49).
constexpr float kCall = 4.f, kTurn = 2.f, kEnd = 1.f, kJoin = 0.5f, kJoinAhead = 2.f, kTrip = 0.8f, kJoinBytes = 7e6f, kJoinCached = 1e8f,
                kAgain = 6.7e6f;
float join_cost(float bytes, int sharing, int at_once, int passes, bool ahead) {
  return (ahead ? kJoinAhead : kJoin) + kTrip * passes * ((sharing + at_once - 1) / at_once) + (bytes + std::max(0.f, bytes - kJoinCached)) / kJoinBytes;
}
struct SmallCost {
  int kind, rows, columns, blocks;  // launch_fp8_small's kind; a workgroup's tile and blocks of k a stage
  float few, all, rate;
  bool exact;
  int resident;                     // workgroups a compute unit
  int at_once;                      // parts that are added at once
};
constexpr SmallCost kSmall[] = {
    {1, 32, 64, 4, 0.6f, 0.95f, 4.9e6f, true, 1, 8},  {2, 64, 64, 4, 1.45f, 1.6f, 4.9e6f, true, 1, 4},  {3, 64, 128, 2, 1.4f, 1.5f, 4.9e6f, true, 1, 4},
    {8, 32, 64, 2, 0.6f, 1.f, 5.4e6f, true, 2, 8},    {4, 64, 64, 4, 0.65f, 1.4f, 4.9e6f, false, 1, 4}, {5, 64, 128, 2, 0.6f, 0.85f, 4.9e6f, false, 1, 4},
    {6, 96, 128, 2, 0.9f, 1.1f, 4.9e6f, false, 1, 2}, {7, 128, 128, 1, 0.56f, 0.66f, 4.9e6f, false, 1, 4},
};
struct LargeCost {
  int rows;
  float step;
  bool exact;
  int at_once, passes;  // parts that are added at once, passes over them
};
constexpr float kLargeRate = 5.2e6f;
constexpr LargeCost kLarge[] = {{32, 1.0f, true, 8, 1}, {64, 1.5f, true, 4, 1}, {128, 1.05f, false, 1, 2}, {192, 1.4f, false, 1, 2}, {256, 1.8f, false, 1, 2}};

// At most 16 rows, or little work: wavefronts straight from memory.  One tile of 16 columns a wavefront where
// that already spreads over the compute units, else two, which share the rows' conversion.  K is cut over the eight
// wavefronts of a workgroup where it is short, over sixteen where eight would load twice one after the other and
// sixteen need no more than that, else over four and over workgroups too, no more than two a compute unit, which is
// what stays resident.
// (Sixteen against eight, in graphs, 1 to 16 rows: 17 to 32 blocks 0.90 to 1.00 of the time of 8-bit rows and 0.94 to 1.03 of
// bf16 rows, which convert; 33 to 64 blocks 0.90 to 1.09 and 1.00 to 1.19; below 17, 1.06 to 1.10.  1 row: 3584 x 3584 5.6
// and 5.9 us of 8 bits, 6.6 both of bf16; 3584 x 5120 7.8 and 7.6, 9.6 and 8.1.  7 bf16 rows, 5120 x 27648: 480 workgroups
// 29.0 us, 640 35.5.  1 row of 8 bits, 3584 x 18944: 17.6 with two tiles, four wavefronts and four workgroups, 19.6 with
// one tile and one workgroup.)  The same for bf16 rows, so that they give the bits of their 8-bit rows.
void few_plan(int M, int N, int K, int cus, Fp8Plan* p) {
  const int tiles = N / 16, KB = K / 128;
  const bool longer = KB > 64;
  p->few = M > 16 || (tiles <= cus && !longer) ? 1 : 2;
  const int sets = (tiles + p->few - 1) / p->few;
  p->waves = M > 16 || longer || sets > cus ? 4 : p->few == 1 && KB > 16 && KB <= 32 ? 16 : 8;
  p->splits = longer || M > 16 ? std::max(1, std::min(2 * cus / sets, std::min(KB / 16, 64))) : 1;
}

}  // namespace

Fp8Plan fp8_plan(int M, int N, int K, bool rows8, bool exact, int cus) {
  Fp8Plan p{};
  const int KB = K / 128;
  const bool few = M <= kFp8ExactRows;
  exact = exact || few;
  size_t parts = 0;
  if (M <= 16 || (few && static_cast<long long>(N) * K <= 1 << 21)) {
    few_plan(M, N, K, cus, &p);
    p.tile_rows = 16 * ((M + 15) / 16);
    p.tile_columns = 16 * p.few;
    p.groups = (N / 16 + p.few - 1) / p.few * p.splits;
    p.sharing = p.splits;
    if (p.splits > 1) parts = static_cast<size_t>((N / 16 + p.few - 1) / p.few) * p.splits * ((M + 15) / 16) * p.few * kWave * 16;
  } else {
    const float weights = static_cast<float>(N) * K;
    float best = 1e30f;
    for (const SmallCost& c : kSmall) {
      if (c.exact != exact) continue;
      const long long tiles = static_cast<long long>((M + c.rows - 1) / c.rows) * ((N + c.columns - 1) / c.columns);
      if (tiles > 64ll * cus) continue;
      const int units = (KB + c.blocks - 1) / c.blocks;
      const int splits = std::max(1, std::min(cus / static_cast<int>(tiles), units));
      const long long groups = tiles * splits;
      // (of two workgroups a compute unit the one goes on while the other starts or ends)
      const float turns = c.resident == 1 ? static_cast<float>((groups + cus - 1) / cus) : std::max(1.f, groups / (2.f * cus));
      const float step = std::max(c.few, c.all * std::min<long long>(groups, cus) / cus);
      const size_t bytes = splits > 1 ? static_cast<size_t>(groups) * c.rows * c.columns * 4 : 0;
      const float memory = weights / (exact && M > c.rows ? kAgain / 2 : c.rate);
      const float cost = kCall + std::max(memory, turns * ((units + splits - 1) / splits * step) + (turns - 1) * kTurn + kEnd) +
                         (bytes ? join_cost(2.f * bytes, splits, c.at_once, 1, false) : 0.f);
      if (cost < best) {
        best = cost;
        p.small = c.kind;
        p.splits = splits;
        p.tile_rows = c.rows;
        p.tile_columns = c.columns;
        p.groups = static_cast<int>(groups);
        p.sharing = splits;
        parts = bytes;
      }
    }
    for (const LargeCost& c : kLarge) {
      if (c.exact != exact || (few && c.rows < M)) continue;
      const long long tiles = static_cast<long long>((M + c.rows - 1) / c.rows) * ((N + kColumns - 1) / kColumns);
      const int rounds = static_cast<int>(tiles / cus), left = static_cast<int>(tiles % cus);
      // The tiles left over whole, in as many equal runs each as there are compute units for, or in runs of all
      // tiles over all compute units.
      for (int way = 0; way < (left ? 3 : 1); ++way) {
        const int sharers = static_cast<int>(std::min<long long>(way == 0 ? left : way == 1 ? cus / left * left : cus, static_cast<long long>(left) * KB));
        if (way && sharers <= left) continue;
        const long long steps = static_cast<long long>(rounds) * KB + (left ? (static_cast<long long>(left) * KB + sharers - 1) / sharers : 0);
        const int places = left && sharers % left ? 2 : 1;
        const size_t runs = sharers > left ? static_cast<size_t>(sharers) * places : 0;  // their places in the workspace
        const float moved = sharers <= left ? 0.f : (sharers % left ? sharers + left : sharers) * 2.f * c.rows * kColumns * 4;
        const int sharing = runs ? (sharers + left - 1) / left + (sharers % left != 0) : 1;
        const int ends = rounds + (left ? 1 + (sharers % left != 0) : 0);
        // (with compute units idle the others run faster: 220 of 256 took 1.32 us a step of 192 rows)
        const float step = rounds ? c.step : c.step * (0.8f + 0.2f * sharers / cus);
        const float cost = kCall + std::max(weights / kLargeRate, steps * step) + ends * kEnd + (runs ? join_cost(moved, sharing, c.at_once, c.passes, rounds > 0) : 0.f);
        if (cost < best) {
          best = cost;
          p.small = 0;
          p.rows = c.rows;
          p.rounds = rounds;
          p.left = left;
          p.sharers = sharers;
          p.places = places;
          p.workers = rounds ? cus : sharers;
          p.tile_rows = c.rows;
          p.tile_columns = kColumns;
          p.groups = p.workers;
          p.sharing = sharing;
          parts = runs * c.rows * kColumns * 4;
        }
      }
    }
  }
  // bf16 rows: up to 32 the few rows' kernel turns them into codes itself (30 rows, 4096 x 512: 5.7 us, 8.2 with
  // a launch that does; of 49 rows, 1024 x 2048, 10.8 and 9.0: every workgroup turns them all).
  if (!rows8 && !(p.few && M <= 32)) p.code_bytes = (static_cast<size_t>(M) * K + static_cast<size_t>(fp8_words(K)) * M * 4 + 255) & ~size_t(255);
  if (p.code_bytes + parts) p.workspace_bytes = kSplitCounterBytes + p.code_bytes + parts;
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
  if (p.small) {
    a.splits = p.splits;
    return launch_fp8_small(a, p.small, st);
  }
  a.tiles_m = (a.M + p.rows - 1) / p.rows;
  a.tiles_n = (a.N + kColumns - 1) / kColumns;
  a.workers = p.workers;
  a.rounds = p.rounds;
  a.left = p.left;
  a.sharers = p.sharers;
  a.places = p.places;
  switch (p.rows) {
    case 32: return tiles_at<1, 1, 1, 8, 4, true>(a, st);
    case 64: return tiles_at<2, 1, 1, 8, 3, true>(a, st);
    case 128: return tiles_at<2, 2, 2, 4, 3, false>(a, st);
    case 192: return tiles_at<3, 2, 2, 4, 2, false>(a, st);
    default: return tiles_at<4, 2, 2, 4, 2, false>(a, st);
  }
}

hipError_t launch_fp8_pack(const uint8_t* codes, int N, int K, uint8_t* tiles, hipStream_t st) {
  hipLaunchKernelGGL(k_fp8_pack, dim3(N / 16, (K / 128 + 1) / 2), dim3(256), 0, st, codes, K, tiles);
  return hipGetLastError();
}

}  // namespace subspec
