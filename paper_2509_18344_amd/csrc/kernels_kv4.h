// Host-visible launchers of the key/value cache held in 4 bits and of the tree attention
// that reads it (internal; the public ABI is include/subspec.h).
#pragma once

#include "kernels.h"

namespace subspec {

constexpr int kKv4D = 128;           // head dimension
constexpr int kKv4Tile = 32;         // positions per tile
constexpr int kKv4CodeBytes = kKv4Tile * kKv4D / 2;
constexpr int kKv4MaxRows = 64;      // attention: query rows per key/value head
constexpr int kKv4MaskWords = 2048;  // attention: M * ceil((T + M) / 32)

// Bytes of a tile: the codes, and per 64 or 128 dimensions a scale and a minimum of each position.
constexpr int kv4_tile_bytes(int groups) { return kKv4CodeBytes + kKv4Tile * 4 * groups; }

struct Kv4RowsArgs {
  const uint16_t* k;  // append: bf16 [src_rows][Hkv][128]
  const uint16_t* v;
  const int* rows;    // append: source row of each position, or null (row i)
  const int* count;   // append: positions written (at most n), or null (n)
  int src_rows, n, pos, Hkv, S;
  uint8_t* k_cache;
  uint8_t* v_cache;
  uint16_t* k_out;    // read: bf16 [n][Hkv][128]
  uint16_t* v_out;
  bool heads_first;   // grid (heads, tiles); set by the launchers
};

hipError_t launch_kv4_append(Kv4RowsArgs a, int groups, hipStream_t st);
hipError_t launch_kv4_read(Kv4RowsArgs a, int groups, hipStream_t st);

struct Kv4AttnArgs {
  const uint16_t* q;       // bf16 [M][Hq][128]
  const uint8_t* k_cache;  // [Hkv][S / 32] tiles
  const uint8_t* v_cache;
  const uint32_t* mask;    // [M][W] bit rows over the tree positions
  int M, Hq, Hkv, S, P, T, W;
  int Gq;                  // Hq / Hkv
  float inv_m;             // 1 / M
  float scale_log2;        // |scale| * log2(e)
  uint32_t q_sign;         // 0x80008000 where the scale is negative: flips q's signs
  int splits;              // key ranges per key/value head
  int tiles_per_split;
  int rows_pad;            // 16 * ceil((Hq / Hkv) * M / 16)
  float* part_o;           // [Hkv][splits][rows_pad][128] unnormalised partial outputs
  float* part_ml;          // [Hkv][splits][rows_pad][2] running maximum (log2 domain), sum
  uint16_t* out;           // bf16 [M][Hq][128]
};

void kv4_attn_plan(int M, int Hq, int Hkv, int P, int T, int* splits, int* tiles_per_split);
size_t kv4_attn_workspace_bytes(int M, int Hq, int Hkv, int P, int T);
hipError_t launch_kv4_attention(const Kv4AttnArgs& a, int groups, hipStream_t st);

}  // namespace subspec
