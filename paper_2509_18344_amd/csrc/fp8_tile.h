// What the kernels of the product in 8-bit floating point share: copies into LDS, the products of a
// block of 128 k out of it, and results to memory.
#pragma once

#include "fp8_device.h"
#include "kernels_fp8.h"

namespace subspec {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kFp8Waves = 8, kFp8Threads = kFp8Waves * kWave;
constexpr int kAgent = 16;  // sc1: coherent at agent scope

// One load straight into LDS: lane l's SIZE bytes land at byte dst + SIZE * l.  Written as assembly because
// the compiler, where it sees such loads, waits for all of them before it reads LDS again; it has no register
// result, and the kernel's own waits order it (a wait state after the write of m0 included).
template <bool ONCE>
__device__ __forceinline__ void copy16(const uint8_t* base, uint32_t offset, uint32_t dst) {
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(dst), "v"(offset), "s"(base) : "memory", "m0");
  else
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

// Sixteen scaled codes as two operands of the 16-bit matrix instruction.
__device__ __forceinline__ void sixteen_bf16(u32x4_t c, float scale, bf16x8_t (&out)[2]) {
  out[0] = fp8_as_bf16(c[0], c[1], scale);
  out[1] = fp8_as_bf16(c[2], c[3], scale);
}
__device__ __forceinline__ u32x4_t sixteen_codes(const uint8_t* p) { return *reinterpret_cast<const u32x4_t*>(p); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return float_to_bf16_bits(lo) | static_cast<uint32_t>(float_to_bf16_bits(hi)) << 16;
}

// A block of k in LDS: eight rows of x in 1024 bytes, 16 bytes c of row r at place c ^ (r / 2 % 8) of its 128 (no
// bank twice in the 16 rows that are read at once), the weight tiles as they are in memory, and the scale words.
// What lane `lane` of copy i (rows 8 i ..) takes to place lane % 8 of row lane / 8.
__device__ __forceinline__ uint32_t fp8_chunk(int lane, int i) { return 16 * (lane % 8 ^ (4 * (i % 2) + lane / 16)); }

// Where a lane reads: 32 rows of either side start at `x` and `w`, words at `xs` and `ws`.
struct Fp8Lane {
  uint32_t x[4];  // 16 bytes 4 h + 2 half + t of row lane % 32, at [2 h + t]
  uint32_t w, s;
};
__device__ __forceinline__ Fp8Lane fp8_lane(int lane) {
  const int r = lane % 32, half = lane / 32;
  Fp8Lane l;
#pragma unroll
  for (int u = 0; u < 4; ++u) l.x[u] = r * 128 + 16 * ((4 * (u / 2) + 2 * half + u % 2) ^ (r / 2 % 8));
  l.w = r / 16 * 2048 + 512 * half + 16 * (r % 16);
  l.s = 4 * r;
  return l;
}

// A lane's sixteen codes of every block of 32 rows and columns: a quarter of what it has of a block of k.  (The first
// are read ahead of the branches on the scales: 49 rows, 3584 x 18944: 22.9 us, 23.5 behind them.)
template <int MF, int NF>
struct Fp8Quarter {
  u32x4_t w[NF], x[MF];
};
template <int MF, int NF>
__device__ __forceinline__ Fp8Quarter<MF, NF> fp8_quarter(const uint8_t* x, const uint8_t* w, const Fp8Lane& l, int u) {
  Fp8Quarter<MF, NF> c;
#pragma unroll
  for (int i = 0; i < NF; ++i) c.w[i] = sixteen_codes(w + l.w + 4096 * i + 1024 * (u / 2) + 256 * (u % 2));
#pragma unroll
  for (int j = 0; j < MF; ++j) c.x[j] = sixteen_codes(x + l.x[u] + 4096 * j);
  return c;
}
// acc[i][j] += the block's products of columns 32 i .. and rows 32 j .. (weights are the left operand: a lane
// ends up with columns 8 q + 4 half + 0 .. 3 of one row).  `byte` is the block's place in its scale words.
// EXACT: scaled codes become bf16 numbers, whose products the 16-bit instruction adds in fp32.  Where a scale
// is so far from 1 that bf16 would not hold them, the bare codes do, and the block's sum is scaled afterwards.
template <int MF, int NF>
__device__ __forceinline__ void fp8_block_sums(f32x16_t (&acc)[NF][MF], const Fp8Quarter<MF, NF>& first, const uint8_t* x, const uint8_t* w,
                                               const Fp8Lane& l, const float (&xp)[MF], const float (&wp)[NF]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const Fp8Quarter<MF, NF> c = u ? fp8_quarter<MF, NF>(x, w, l, u) : first;
    bf16x8_t wf[NF][2], xf[MF][2];
#pragma unroll
    for (int i = 0; i < NF; ++i) sixteen_bf16(c.w[i], wp[i], wf[i]);
#pragma unroll
    for (int j = 0; j < MF; ++j) sixteen_bf16(c.x[j], xp[j], xf[j]);
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
      for (int j = 0; j < MF; ++j)
#pragma unroll
        for (int i = 0; i < NF; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[i][v], xf[j][v], acc[i][j], 0, 0, 0);
  }
}

template <int MF, int NF>
__device__ __forceinline__ void fp8_clear(f32x16_t (&acc)[NF][MF]) {
#pragma unroll
  for (int i = 0; i < NF; ++i)
#pragma unroll
    for (int j = 0; j < MF; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
}

// The bits that are set in any of a lane's 64 codes of a block.
__device__ __forceinline__ uint32_t fp8_any(const uint8_t* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const u32x4_t v = *reinterpret_cast<const u32x4_t*>(p + a) | *reinterpret_cast<const u32x4_t*>(p + b) |
                    *reinterpret_cast<const u32x4_t*>(p + c) | *reinterpret_cast<const u32x4_t*>(p + d);
  return v[0] | v[1] | v[2] | v[3];
}

template <int MF, int NF, bool EXACT>
__device__ __forceinline__ void fp8_block_products(f32x16_t (&acc)[NF][MF], const uint8_t* x, const uint8_t* w, const uint8_t* xs, const uint8_t* ws,
                                                   const Fp8Lane& l, int half, int byte) {
  uint32_t xb[MF], wb[NF];
#pragma unroll
  for (int j = 0; j < MF; ++j) xb[j] = xs[l.s + 128 * j + byte];
#pragma unroll
  for (int i = 0; i < NF; ++i) wb[i] = ws[l.s + 128 * i + byte];
  if constexpr (EXACT) {
    float xp[MF], wp[NF];
    bool plain = true;
    const Fp8Quarter<MF, NF> first = fp8_quarter<MF, NF>(x, w, l, 0);
#pragma unroll
    for (int j = 0; j < MF; ++j) plain &= fp8_plain(xb[j]), xp[j] = fp8_power(xb[j]);
#pragma unroll
    for (int i = 0; i < NF; ++i) plain &= fp8_plain(wb[i]), wp[i] = fp8_power(wb[i]);
    plain = __all(plain);
    if (!plain) {  // once more without the scales of zeros
      bool p = true;
#pragma unroll
      for (int j = 0; j < MF; ++j) p &= fp8_plain(xb[j]) || fp8_zeros(fp8_any(x + 4096 * j, l.x[0], l.x[1], l.x[2], l.x[3]));
#pragma unroll
      for (int i = 0; i < NF; ++i) p &= fp8_plain(wb[i]) || fp8_zeros(fp8_any(w + 4096 * i, l.w, l.w + 256, l.w + 1024, l.w + 1280));
      plain = __all(p);
    }
    if (plain) {
      fp8_block_sums(acc, first, x, w, l, xp, wp);
      return;
    }
    f32x16_t part[NF][MF];
    fp8_clear(part);
#pragma unroll
    for (int j = 0; j < MF; ++j) xp[j] = 1.f;
#pragma unroll
    for (int i = 0; i < NF; ++i) wp[i] = 1.f;
    fp8_block_sums(part, first, x, w, l, xp, wp);
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const u32x4_t words = *reinterpret_cast<const u32x4_t*>(ws + 4 * (32 * i + 8 * q + 4 * half));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int n = static_cast<int>(words[e] >> (8 * byte) & 255u) - 254;
#pragma unroll
          for (int j = 0; j < MF; ++j) acc[i][j][4 * q + e] += ldexpf(part[i][j][4 * q + e], n + static_cast<int>(xb[j]));
        }
      }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      i32x8_t wf[NF], xf[MF];
#pragma unroll
      for (int i = 0; i < NF; ++i) wf[i] = codes32(w + l.w + 4096 * i + 1024 * h, w + l.w + 4096 * i + 1024 * h + 256);
#pragma unroll
      for (int j = 0; j < MF; ++j) xf[j] = codes32(x + l.x[2 * h] + 4096 * j, x + l.x[2 * h + 1] + 4096 * j);
#pragma unroll
      for (int j = 0; j < MF; ++j)
#pragma unroll
        for (int i = 0; i < NF; ++i)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[i], xf[j], acc[i][j], 0, 0, 0, static_cast<int>(wb[i]), 0,
                                                                     static_cast<int>(xb[j]));
    }
  }
}

// Which worker has block p of the left tiles' `total` blocks: worker w's run starts at floor(w total / sharers).
__device__ __forceinline__ int sharer_of(long long p, long long total, int sharers) {
  return static_cast<int>(((p + 1) * sharers - 1) / total);
}

// A worker's segments: up to two cut tiles, then whole ones.
struct Fp8Segment {
  int tile, kb0, kb1;
};
struct Fp8Work {
  long long total, from, to;  // blocks of the left tiles; this worker's
  int KB, w, first, cut, segments, left0, step;

  __device__ __forceinline__ explicit Fp8Work(const Fp8Args& a) : KB(a.K / 128), left0(a.rounds * a.workers), step(a.workers) {
    // Workgroups b, b + 8, .. run on one XCD: it takes neighbouring workers, so that its L2 serves tiles of the
    // same rows and columns.
    const int b = blockIdx.x, per = a.workers / 8;
    w = a.workers % 8 ? b : (b % 8) * per + b / 8;
    total = static_cast<long long>(a.left) * KB;
    from = to = 0;
    if (w < a.sharers) from = w * total / a.sharers, to = (w + 1) * total / a.sharers;
    first = static_cast<int>(from / KB);
    cut = to == from ? 0 : (to - 1) / KB > first ? 2 : 1;
    segments = cut + a.rounds;
  }
  __device__ __forceinline__ Fp8Segment segment(int s) const {
    if (s >= cut) return {w + (s - cut) * step, 0, KB};
    const int t = first + s;
    const long long at = static_cast<long long>(t) * KB;
    return {left0 + t, static_cast<int>(max(from, at) - at), static_cast<int>(min(to, at + KB) - at)};
  }
  __device__ __forceinline__ int blocks() const {
    return static_cast<int>(to - from) + (segments - cut) * KB;
  }
};

// Tiles in bands of eight along the rows, columns inside: neighbouring workers share either.
__device__ __forceinline__ void fp8_place(const Fp8Args& a, int tile, int rows, int columns, int* m0, int* n0) {
  const int band = tile / (8 * a.tiles_n), rest = tile - band * 8 * a.tiles_n, high = min(8, a.tiles_m - 8 * band);
  *n0 = rest / high * columns;
  *m0 = (8 * band + rest % high) * rows;
}

// Results of rows m0 .. and columns n0 .. : a lane's four columns of a row, swapped with the other half's, are
// eight in a row.
template <int MF, int NF>
__device__ __forceinline__ void fp8_results(const f32x16_t (&acc)[NF][MF], const Fp8Args& a, int m0, int n0, int lane) {
  const int half = lane / 32;
#pragma unroll
  for (int j = 0; j < MF; ++j) {
    const int m = m0 + 32 * j + lane % 32;
#pragma unroll
    for (int i = 0; i < NF; ++i) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int n = n0 + 32 * i + 16 * p;
        const f32x16_t& c = acc[i][j];
        const auto lo = __builtin_amdgcn_permlane32_swap(pack_bf16(c[8 * p], c[8 * p + 1]), pack_bf16(c[8 * p + 4], c[8 * p + 5]), false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap(pack_bf16(c[8 * p + 2], c[8 * p + 3]), pack_bf16(c[8 * p + 6], c[8 * p + 7]), false, false);
        if (m < a.M && n < a.N)
          *reinterpret_cast<uint4*>(a.y + static_cast<size_t>(m) * a.N + n + 8 * half) = make_uint4(lo[0], hi[0], lo[1], hi[1]);
      }
    }
  }
}

// Partial sums of a workgroup, in the accumulators' order: quad e of block (i, j) of every thread in turn.
template <int MF, int NF>
__device__ __forceinline__ void fp8_store_part(const f32x16_t (&acc)[NF][MF], __amdgpu_buffer_rsrc_t to, uint32_t thread, uint32_t threads) {
#pragma unroll
  for (int i = 0; i < NF; ++i)
#pragma unroll
    for (int j = 0; j < MF; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        __builtin_amdgcn_raw_buffer_store_b128(
            __builtin_bit_cast(u32x4_t, f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]}), to, 16 * thread,
            ((i * MF + j) * 4 + q) * 16 * threads, kAgent);
}

// acc = the sum of `count` workgroups' partial sums in their order; from(k) is the buffer of the k-th.
template <int MF, int NF, class From>
__device__ __forceinline__ void fp8_add_parts(f32x16_t (&acc)[NF][MF], int count, From from, uint32_t thread, uint32_t threads) {
  constexpr int AT_ONCE = NF == 1 && MF < 8 ? 8 / MF : 1;  // sums in flight
  fp8_clear(acc);
#pragma unroll
  for (int i = 0; i < NF; ++i) {
    for (int k = 0; k < count; k += AT_ONCE) {
      f32x4_t v[AT_ONCE][MF][4];
#pragma unroll
      for (int o = 0; o < AT_ONCE; ++o) {
        const __amdgpu_buffer_rsrc_t p = from(min(k + o, count - 1));
        const uint32_t at = k + o < count ? 16 * thread : 0x80000000u;  // past the last: zeros, from past the buffer
#pragma unroll
        for (int j = 0; j < MF; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            v[o][j][q] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(p, at, ((i * MF + j) * 4 + q) * 16 * threads, kAgent));
      }
#pragma unroll
      for (int o = 0; o < AT_ONCE; ++o)
#pragma unroll
        for (int j = 0; j < MF; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[i][j][e] += v[o][j][e / 4][e % 4];
    }
  }
}

// A cut tile's sums, called by the whole workgroup.  Every worker of the tile stores its own with agent-scope
// stores and counts itself in once they are acknowledged; the last, for which this returns true, has the sum in
// the order of k.
template <int MF, int NF>
__device__ __forceinline__ bool fp8_join(f32x16_t (&acc)[NF][MF], const Fp8Args& a, const Fp8Work& work, int s, int tile, uint32_t part_bytes, int* last) {
  const int t = tile - work.left0;
  auto part = [&](int who, int seg) __attribute__((always_inline)) {
    return buffer_rsrc(reinterpret_cast<const uint8_t*>(a.part) + static_cast<size_t>(a.places * who + seg) * part_bytes, part_bytes);
  };
  fp8_store_part(acc, part(work.w, s), threadIdx.x, kFp8Threads);
  wait_and_meet<0>();
  const int w0 = sharer_of(static_cast<long long>(t) * work.KB, work.total, a.sharers);
  const int w1 = sharer_of(static_cast<long long>(t) * work.KB + work.KB - 1, work.total, a.sharers);
  if (threadIdx.x == 0)
    *last = __hip_atomic_fetch_add(a.count + t, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<unsigned>(w1 - w0);
  __syncthreads();
  if (!*last) return false;
  // (the tile is the first of a worker's run or its second)
  fp8_add_parts(acc, w1 - w0 + 1, [&](int k) { return part(w0 + k, static_cast<int>((w0 + k) * work.total / a.sharers / work.KB) == t ? 0 : 1); },
                threadIdx.x, kFp8Threads);
  if (threadIdx.x == 0) __hip_atomic_store(a.count + t, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}

}  // namespace subspec
