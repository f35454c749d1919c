// Host-visible launchers of the product in 8-bit floating point (internal; the public ABI is
// include/subspec.h).
#pragma once

#include "kernels_rows.h"

namespace subspec {

constexpr int kFp8ExactRows = 64;  // up to here products are exact

struct Fp8Args {
  const void* x;          // codes [M][K], or bf16 [M][K] where xs is null
  const uint32_t* xs;     // [fp8_words(K)][M]
  const uint8_t* w;       // weight tiles of [N][K]
  const uint32_t* ws;     // [fp8_words(K)][N]
  int M, N, K;
  uint16_t* y;            // bf16 [M][N]
  // Work of the tiles' kernel.  Its workgroups ("workers") take tiles whole in `rounds` rounds of one
  // each; the tiles left over are cut along K among the first `sharers` workers, in equal runs of
  // blocks.
  int tiles_m, tiles_n;
  int workers, rounds, left, sharers;
  int places;             // tiles that a sharer's run may touch: 1 where each left tile has equally many, else 2
  float* part;            // [sharers][places] tiles of partial sums; few rows: [columns][splits]
  unsigned* count;        // per left tile, or columns: workers done (zero between launches)
  int splits;             // few rows: workgroups that share columns
};

struct Fp8Plan {
  int few;                 // few rows: tiles of 16 columns a wavefront; 0: the tiles' kernel
  int waves, splits;       // wavefronts of a workgroup and workgroups that share columns then
  int small;               // which of the small tiles; 0: the large ones
  int rows;                // rows of a large tile
  int workers, rounds, left, sharers, places;
  int tile_rows, tile_columns, groups, sharing;  // the launch described: tile, workgroups, most that share a tile's K
  size_t code_bytes;       // x's codes and scales, where the call makes them
  size_t workspace_bytes;  // completion counters, codes and scales, partial sums; 0: none
};
Fp8Plan fp8_plan(int M, int N, int K, bool rows8, bool exact, int cus);  // exact: at any number of rows
hipError_t launch_fp8_linear(const Fp8Plan& p, Fp8Args a, void* workspace, hipStream_t st);
hipError_t launch_fp8_few(const Fp8Args& a, int columns, int waves, hipStream_t st);
hipError_t launch_fp8_small(const Fp8Args& a, int kind, hipStream_t st);
hipError_t launch_fp8_pack(const uint8_t* codes, int N, int K, uint8_t* tiles, hipStream_t st);

}  // namespace subspec
