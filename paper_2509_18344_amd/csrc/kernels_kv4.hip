// Rows into and out of the key/value cache held in 4 bits (kv4_device.h has the arithmetic,
// include/subspec.h the layout).
//
// A workgroup takes one tile of 32 positions of one key/value head, 16 lanes of 8 dimensions
// a row: a row's range is three or four DPP steps, a key's 8 codes are one word, and the
// values' codes turn in LDS into words of 8 positions each.
//
// Measured, 16384 positions of 8 heads in groups of 128: append 22.7 us for 67 MB read and 18 written,
// 3.7 TB/s, issuing vector instructions 70 % of the time (455 a wavefront, 95 of them for a lane's 8
// values), with no load in flight while a workgroup quantizes and turns its tile; read 15.5 us for the
// same bytes, 5.5 TB/s, as a large copy: bound by memory.  A few rows
// 3.9 and 3.4 us, the launch and one chain of loads.
#include "kv4_device.h"

namespace subspec {

namespace {

constexpr int kKv4Threads = 256;

template <int G>
__global__ __launch_bounds__(kKv4Threads) void k_kv4_append(Kv4RowsArgs a) {
  __shared__ Kv4TileLds lds;
  const int tile = a.pos / kKv4Tile + (a.heads_first ? blockIdx.y : blockIdx.x), g = a.heads_first ? blockIdx.x : blockIdx.y;
  const int n = a.count ? min(max(*a.count, 0), a.n) : a.n;
  if (tile * kKv4Tile - a.pos >= n) return;  // no position of this tile is written
  const size_t at = (static_cast<size_t>(g) * (a.S / kKv4Tile) + tile) * kv4_tile_bytes(G);
  kv4_store_tile<G>(a.k_cache + at, a.v_cache + at, a.k, a.v, lds, [&](int w) {
    const int i = tile * kKv4Tile + w - a.pos;
    if (i < 0 || i >= n) return -1ll;
    const int src = a.rows ? a.rows[i] : i;
    if (src < 0 || src >= a.src_rows) return -1ll;
    return (static_cast<long long>(src) * a.Hkv + g) * kKv4D;
  });
}

__device__ __forceinline__ uint4 kv4_values8(const uint32_t (&code)[8], float s, float m) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = m + s * static_cast<float>(code[i]);
  return pack8(x);
}

template <int G>
__global__ __launch_bounds__(kKv4Threads) void k_kv4_read(Kv4RowsArgs a) {
  __shared__ alignas(16) uint8_t lds[kKv4Tile][kKv4D + 16];
  const int tile = a.pos / kKv4Tile + (a.heads_first ? blockIdx.y : blockIdx.x), g = a.heads_first ? blockIdx.x : blockIdx.y;
  const size_t at = (static_cast<size_t>(g) * (a.S / kKv4Tile) + tile) * kv4_tile_bytes(G);
  const uint8_t* kt = a.k_cache + at;
  const uint8_t* vt = a.v_cache + at;
  if (threadIdx.x < 128) {
    const int half = threadIdx.x / 64, lane = threadIdx.x % 64;
    const int vc = lane % 16, quarter = lane / 16;
    const uint4 p = *reinterpret_cast<const uint4*>(vt + half * 1024 + lane * 16);
    const uint32_t word[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int w = 4 * quarter + (e & 3) + 16 * (e >> 2);
#pragma unroll
      for (int d = 0; d < 4; ++d)
        lds[w][64 * half + 16 * d + vc] = (word[d] >> (4 * (e / 2) + 16 * (e % 2))) & 0xFu;
    }
  }
  __syncthreads();
  const int col = threadIdx.x % 16, r = threadIdx.x / 16;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int w = 16 * b + r, i = tile * kKv4Tile + w - a.pos;
    if (i < 0 || i >= a.n) continue;
    const int meta = kv4_meta<G>(w, col / (16 / G));
    const size_t dst = (static_cast<size_t>(i) * a.Hkv + g) * kKv4D + 8 * col;
    uint32_t code[8];
    const uint32_t kw = *reinterpret_cast<const uint32_t*>(kt + kv4_key_word(w, col));
#pragma unroll
    for (int e = 0; e < 8; ++e) code[e] = (kw >> (4 * (e / 2) + 16 * (e % 2))) & 0xFu;
    *reinterpret_cast<uint4*>(a.k_out + dst) = kv4_values8(code, static_cast<float>(*reinterpret_cast<const _Float16*>(kt + meta)),
                                                          static_cast<float>(*reinterpret_cast<const _Float16*>(kt + meta + 16)));
    const uint2 vw = *reinterpret_cast<const uint2*>(&lds[w][8 * col]);
#pragma unroll
    for (int e = 0; e < 8; ++e) code[e] = ((e < 4 ? vw.x : vw.y) >> (8 * (e % 4))) & 0xFu;
    *reinterpret_cast<uint4*>(a.v_out + dst) = kv4_values8(code, static_cast<float>(*reinterpret_cast<const _Float16*>(vt + meta)),
                                                          static_cast<float>(*reinterpret_cast<const _Float16*>(vt + meta + 16)));
  }
}

// The heads of a tile next to each other in the order of launch, where the grid allows: their
// rows of k and v are neighbours in memory.
dim3 kv4_grid(Kv4RowsArgs* a) {
  const unsigned tiles = (a->pos + a->n - 1) / kKv4Tile - a->pos / kKv4Tile + 1;
  a->heads_first = tiles <= 65535;
  return a->heads_first ? dim3(a->Hkv, tiles) : dim3(tiles, a->Hkv);
}

}  // namespace

hipError_t launch_kv4_append(Kv4RowsArgs a, int groups, hipStream_t st) {
  const dim3 grid = kv4_grid(&a);
  if (groups == 1)
    hipLaunchKernelGGL(k_kv4_append<1>, grid, dim3(kKv4Threads), 0, st, a);
  else
    hipLaunchKernelGGL(k_kv4_append<2>, grid, dim3(kKv4Threads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_kv4_read(Kv4RowsArgs a, int groups, hipStream_t st) {
  const dim3 grid = kv4_grid(&a);
  if (groups == 1)
    hipLaunchKernelGGL(k_kv4_read<1>, grid, dim3(kKv4Threads), 0, st, a);
  else
    hipLaunchKernelGGL(k_kv4_read<2>, grid, dim3(kKv4Threads), 0, st, a);
  return hipGetLastError();
}

}  // namespace subspec
