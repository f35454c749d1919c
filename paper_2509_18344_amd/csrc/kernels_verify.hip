// Verification of a drafted tree against the target's logits with given uniform numbers.
//
// Row 0 of the logits belongs to the context's last token, row 1 + j to drafted token j.
// In row i, p_i = softmax(l_i / T); the row's children c_1, c_2, ... (tokens whose parent it
// is, in index order, a repeated token counting once) hold the first part of [0, 1) in
// that order, every other token of the vocabulary the rest in token order.  The number u_i
// picks one of them, so the pick is a sample of p_i: a child continues the path, any other
// token ends it.  At temperature 0 the pick is the row's largest logit, the lowest token of
// equals.
//
// All rows are read at once, although only those on the path matter, because the path is
// known only at its end: a row needs its maximum and its sum of exponentials to say which
// child it picks, not the whole distribution.
// Up to 1750 to 2200 slices of 2048 logits in all (verify_small) one kernel does everything in 64 bits
// (k_verify_small: a slice its maximum and its sum without the row's children, the last workgroup of a
// row the row's pick and, where that ends the path, its token, the last of all the path: a chain of 4 at
// V = 32000 9.8 us a call against 15.3 with two kernels).  Beyond, two, since 64-bit exponentials of all
// logits would bound them:
//   k_verify_rows      per (row, slice) workgroup a reference and the sum, of exponentials in 32 bits; the
//                      last of a row finds the child that the row picks, the last of all the path
//   k_verify_residual  the last row's other tokens in 64 bits: with V = 152064 tokens the
//                      borders lie 10^-5 apart, and a sum in 32 bits, 10^-7 off, would pick a
//                      neighbour in one call of a hundred; the last workgroup finds the token
// Measured, 288 tokens at V = 152064, 88 MB: k_verify_rows 21.2 us (greedy 20.6), of which reading
// alone takes 15 (5.9 TB/s) and the chain from a row's sum over its pick to the path 4.5;
// k_verify_residual 7.8, a chain of dependent loads and two reductions; 29 us a call, greedy 20.5.
#include <algorithm>
#include <climits>
#include <cmath>

#include "device_common.h"
#include "kernels_verify.h"

namespace subspec {

namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / kWave;
constexpr int kRowOwn = kVerifyMaxTokens / kRowThreads;  // drafted tokens a thread looks at
// Rows' completion counters lie 60 bytes apart, the most that the workspace has for 1024 tokens: arrivals
// at one line take turns, 17 ns each, and a line holds one or two rows' this way.
constexpr int kCounterStep = 15;
static_assert(kCounterStep * (kVerifyMaxTokens + 2) <= kSplitCounters, "the workspace's counters");

constexpr int kRowLoads = 2;               // 16-byte loads in flight per thread (four: 22.8 us against 21.2)
constexpr int kRowTile = 8 * kRowThreads;  // logits that the workgroup's threads load at a time

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ void split8(uint4 w, float (&x)[8]) {
  const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf_lo(a[i]);
    x[2 * i + 1] = bf_hi(a[i]);
  }
}

__device__ __forceinline__ float wave_top(float v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// Greedy: the larger logit and of equals the lower token; a NaN (the row has none) stays.
__device__ __forceinline__ void best_of(float& m, int& i, float m2, int i2) {
  const bool take = m != m ? false : m2 != m2 ? true : m2 > m || (m2 == m && i2 < i);
  m = take ? m2 : m;
  i = take ? i2 : i;
}

// What is kept of logits seen: (reference, sum of 2^(c (l - reference))), or greedy (maximum, the first
// token of the eight that it was found in).  The reference is a logit that the largest one passes by less
// than 2^kAhead: it moves so far that what the move's rounding costs the sum so far is nothing
// beside what comes.  A thread adds its sums of eight in 64 bits (`sum`, one addition in eight terms): bf16
// logits repeat, and in 32 bits the roundings of 4096 equal terms were off by 2^-14 together.
constexpr float kAhead = 16.f;

template <bool GREEDY>
struct Seen {
  float m = -INFINITY;
  float s = GREEDY ? __int_as_float(INT_MAX) : 0.f;
  double sum = 0.0;

  __device__ __forceinline__ void add(float c, const float (&x)[8], int v0) {
    if constexpr (GREEDY) {
      float mx = x[0];  // a NaN stays
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = __builtin_elementwise_maximum(mx, x[e]);
      // a thread's tokens come in order: later equal ones do not replace
      const bool take = m == m && !(mx <= m);
      m = take ? mx : m;
      s = take ? __int_as_float(v0) : s;
    } else {
      float mx = x[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
      const bool move = c * (mx - m) > kAhead;
      if (__builtin_amdgcn_ballot_w64(move)) {
        sum = move && m != -INFINITY ? sum * static_cast<double>(__builtin_amdgcn_exp2f(c * (m - mx))) : sum;
        m = move ? mx : m;
      }
      const float base = m == -INFINITY ? 0.f : m;  // (2^-inf of -inf, and a NaN that the sum has to show)
      float t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = __builtin_amdgcn_exp2f(c * (x[e] - base));
      sum += static_cast<double>(((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7])));
    }
  }

  // The thread's logits are all added.
  __device__ __forceinline__ void close() {
    if constexpr (!GREEDY) s = static_cast<float>(sum);
  }

  // What the wavefront's lanes have seen, in every lane.
  __device__ __forceinline__ void across_wave(float c) {
    if constexpr (GREEDY) {
      int i = __float_as_int(s);
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) best_of(m, i, __shfl_xor(m, d), __shfl_xor(i, d));
      s = __int_as_float(i);
    } else {
      const float top = wave_top(m);
      s = m == -INFINITY ? s : s * __builtin_amdgcn_exp2f(c * (m - top));  // (a sum of nothing, or a NaN, stays)
      m = top;
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) s += __shfl_xor(s, d);
    }
  }

  // What `n` wavefronts or slices have seen, the pairs from `at`.
  template <typename At>
  __device__ __forceinline__ static Seen all(float c, int n, At at) {
    Seen own;
    for (int i = threadIdx.x % kWave; i < n; i += kWave) own.join(c, at(i));
    own.across_wave(c);
    return own;
  }
  __device__ __forceinline__ void join(float c, float2 o) {
    if constexpr (GREEDY) {
      int i = __float_as_int(s);
      best_of(m, i, o.x, __float_as_int(o.y));
      s = __int_as_float(i);
    } else {
      const float top = fmaxf(m, o.x);
      s = (m == -INFINITY ? s : s * __builtin_amdgcn_exp2f(c * (m - top))) +
          (o.x == -INFINITY ? o.y : o.y * __builtin_amdgcn_exp2f(c * (o.x - top)));
      m = top;
    }
  }
};

// Stores that other XCDs' coherent loads see once they are acknowledged.
__device__ __forceinline__ void put(int* p, int v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void put(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void put(double* p, double v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void put(float2* p, float x, float y) {
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p),
                     (static_cast<unsigned long long>(__float_as_uint(y)) << 32) | __float_as_uint(x), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ __forceinline__ T get(const T* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get(const float2* p) {
  const unsigned long long w =
      __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float(static_cast<uint32_t>(w)), __uint_as_float(static_cast<uint32_t>(w >> 32)));
}

// Whether the calling workgroup is the `of`-th to arrive; it then clears the counter.  Every
// wavefront's stores are acknowledged before it arrives.  (All threads call it.)
__device__ __forceinline__ bool last_to_arrive(unsigned* cnt, unsigned of, int* flag) {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool last = __hip_atomic_fetch_add(cnt, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == of - 1;
    if (last) __hip_atomic_store(cnt, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = last;
  }
  __syncthreads();
  return *flag != 0;
}

// Token j continues `row` (a parent p that does not come before it, or a token k outside the
// vocabulary, continues nothing).
__device__ __forceinline__ bool continues(const VerifyArgs& a, int j, int p, int k, int row) {
  return p >= -1 && p < j && p + 1 == row && k >= 0 && k < a.V;
}

struct Children {
  int j[kVerifyMaxTokens];
  int token[kVerifyMaxTokens];
  float p[kVerifyMaxTokens];  // logits
};
struct Ordered {  // by index; a repeated token's share is 0
  int j[kVerifyMaxTokens];
  float p[kVerifyMaxTokens];
};

template <bool GREEDY>
__global__ __launch_bounds__(kRowThreads) void k_verify_rows(VerifyArgs a) {
  __shared__ Children kids;
  __shared__ union {
    Ordered order;
    int next[kVerifyMaxTokens + 1];
  } u;
  __shared__ float2 waves[kRowWaves];
  __shared__ int n, flag, pick;
  const int t = threadIdx.x;
  const int row = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int lo = chunk * a.chunk_len, hi = min(a.V, lo + a.chunk_len);
  const uint16_t* l = a.logits + static_cast<size_t>(row) * a.V;
  // A thread's drafted tokens, then the slice's whole tiles, kRowLoads of them in flight; the row's
  // children's logits come among them.
  int token[kRowOwn], parent[kRowOwn];
#pragma unroll
  for (int k = 0; k < kRowOwn; ++k) {
    const int j = t + k * kRowThreads;
    token[k] = j < a.N ? a.token[j] : -1;
    parent[k] = j < a.N ? a.parent[j] : -1;
  }
  const int tiles = (hi - lo) / kRowTile;
  auto tile = [&](int i) __attribute__((always_inline)) {
    return *reinterpret_cast<const uint4*>(l + lo + i * kRowTile + 8 * t);
  };
  Seen<GREEDY> seen;
  auto take = [&](uint4 w, int i) __attribute__((always_inline)) {
    float x[8];
    split8(w, x);
    seen.add(a.c, x, lo + i * kRowTile + 8 * t);
  };
  uint4 w[kRowLoads] = {};
#pragma unroll
  for (int j = 0; j < kRowLoads; ++j)
    if (j < tiles) w[j] = tile(j);
  if (t == 0) {
    n = 0;
    pick = INT_MAX;
  }
  bool child[kRowOwn];
  uint16_t own[kRowOwn];
#pragma unroll
  for (int k = 0; k < kRowOwn; ++k) {
    child[k] = continues(a, t + k * kRowThreads, parent[k], token[k], row);
    own[k] = child[k] ? l[token[k]] : 0;
  }
  int i = 0;
  for (; i + 2 * kRowLoads <= tiles; i += kRowLoads)
#pragma unroll
    for (int j = 0; j < kRowLoads; ++j) {
      const uint4 now = w[j];
      w[j] = tile(i + kRowLoads + j);
      take(now, i + j);
    }
  for (; i < tiles; i += kRowLoads)
#pragma unroll
    for (int j = 0; j < kRowLoads; ++j)
      if (i + j < tiles) {
        const uint4 now = w[j];
        if (i + kRowLoads + j < tiles) w[j] = tile(i + kRowLoads + j);
        take(now, i + j);
      }
  if (lo + tiles * kRowTile + 8 * t < hi) take(tile(tiles), tiles);  // its last, partial tile
  seen.close();
  seen.across_wave(a.c);
  if (t % kWave == 0) waves[t / kWave] = make_float2(seen.m, seen.s);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kRowOwn; ++k)
    if (child[k]) {  // the row's children, in any order
      const int at = atomicAdd(&n, 1);
      kids.j[at] = t + k * kRowThreads;
      kids.token[at] = token[k];
      kids.p[at] = __uint_as_float(static_cast<uint32_t>(own[k]) << 16);
    }
  seen = Seen<GREEDY>::all(a.c, kRowWaves, [&](int k) { return waves[k]; });
  __syncthreads();
  if (a.chunks > 1) {
    if (t == 0) put(a.stat + blockIdx.x, seen.m, seen.s);
    if (!last_to_arrive(a.cnt + kCounterStep * (1 + row), a.chunks, &flag)) return;
    // every wavefront merges the row's slices, in the same order
    seen = Seen<GREEDY>::all(a.c, a.chunks, [&](int k) { return get(a.stat + static_cast<size_t>(row) * a.chunks + k); });
  }

  // The row's pick among its children.
  const int nk = n;
  const bool ok = fabsf(seen.m) < INFINITY && (GREEDY || (seen.s > 0.f && seen.s < INFINITY));
  int best = -1;  // greedy: the first of its eight
  if (GREEDY && ok) {
    float x[8];
    split8(*reinterpret_cast<const uint4*>(l + __float_as_int(seen.s)), x);
#pragma unroll
    for (int e = 7; e >= 0; --e) best = x[e] == seen.m ? __float_as_int(seen.s) + e : best;
  }
  if (ok) {
    for (int k = t; k < nk; k += kRowThreads) {
      const int j = kids.j[k], token = kids.token[k];
      if constexpr (GREEDY) {
        if (token == best) atomicMin(&pick, j);  // of equal siblings the first
      } else {
        int rank = 0;
        bool repeat = false;
        for (int i = 0; i < nk; ++i) {
          const bool before = kids.j[i] < j;
          rank += before;
          repeat |= before && kids.token[i] == token;
        }
        u.order.j[rank] = j;
        u.order.p[rank] = repeat ? 0.f : __builtin_amdgcn_exp2f(a.c * (kids.p[k] - seen.m)) / seen.s;
      }
    }
    __syncthreads();
    if (!GREEDY && t == 0) {
      const double at = static_cast<double>(a.uniform[row]);
      double f = 0.0;  // (a thousand shares in a row)
      for (int k = 0; k < nk; ++k) {
        const double f2 = f + static_cast<double>(u.order.p[k]);
        if (f <= at && at < f2) {
          pick = u.order.j[k];
          break;
        }
        f = f2;
      }
    }
  }
  if (t == 0) {
    put(a.next + row, pick == INT_MAX ? -1 : pick);
    // a row without a distribution: no sum, or no token
    put(a.row_stat + row, seen.m, GREEDY ? __int_as_float(best) : ok ? seen.s : 0.f);
  }
  if (!last_to_arrive(a.cnt, a.N + 1, &flag)) return;

  // The path.
  for (int r = t; r <= a.N; r += kRowThreads) u.next[r] = get(a.next + r);
  __syncthreads();
  if (t == 0) {
    int r = 0, len = 0;
    for (int j; (j = u.next[r]) >= 0; r = j + 1) a.path[len++] = j;  // j >= r: it ends
    *a.accepted = len;
    n = len;
    const float2 st = get(a.row_stat + r);
    if constexpr (GREEDY) {
      *a.next_token = __float_as_int(st.y);
    } else {
      *a.last_row = r;
      *a.last_stat = st;
    }
  }
  __syncthreads();
  for (int i = n + t; i < a.N; i += kRowThreads) a.path[i] = -1;
}

constexpr int kResThreads = 256;
constexpr int kResWaves = kResThreads / kWave;
static_assert(kVerifySlice == 8 * kResThreads, "eight logits a thread");
constexpr int kSlices = kVerifyMaxV / kVerifySlice / kWave;  // sums of slices a lane
constexpr int kRowSlices = (kVerifyMaxV / kVerifySlice + kResThreads - 1) / kResThreads;  // and a thread

__device__ __forceinline__ double wave_add(double v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// Within a wavefront whose lanes hold K terms each, in order, the first of which has number
// `first` in lane 0: the number of the first term whose running sum (on top of `start`)
// passes `target`, or of the last positive one if none does (-1 if none is); in *before the
// sum in front of it.  The same in every lane.
template <int K>
__device__ __forceinline__ int find_term(const double (&e)[K], int first, double start, double target, double* before) {
  const int lane = threadIdx.x % kWave;
  double own = 0.0;
#pragma unroll
  for (int i = 0; i < K; ++i) own += e[i];
  double run = own;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const double o = __shfl_up(run, d);
    if (lane >= d) run += o;
  }
  run = start + (run - own);
  int hit = -1, any = -1;
  double hit_before = 0.0, any_before = 0.0;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const double up = run + e[i];
    if (e[i] > 0.0) {
      any = first + K * lane + i;
      any_before = run;
      if (up > target && hit < 0) {
        hit = any;
        hit_before = run;
      }
    }
    run = up;
  }
  const unsigned long long hits = __ballot(hit >= 0), some = __ballot(any >= 0);
  if (hits == 0 && some == 0) return -1;
  const int from = hits ? __ffsll(hits) - 1 : 63 - __clzll(static_cast<long long>(some));
  *before = __shfl(hits ? hit_before : any_before, from);
  return __shfl(hits ? hit : any, from);
}

// Zeroes the terms of tokens v0 .. v0 + 7 that are among `kids`.
__device__ __forceinline__ void drop_tokens(const int* kids, int n, int v0, double (&e)[8]) {
  for (int k = 0; k < n; ++k) {
    const int d = kids[k] - v0;
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = d == i ? 0.0 : e[i];
  }
}

// 8 logits at v0, or -inf past the vocabulary.
__device__ __forceinline__ uint4 load_logits(const VerifyArgs& a, const uint16_t* l, int v0) {
  return v0 < a.V ? *reinterpret_cast<const uint4*>(l + v0) : make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
}

// e^((l - m) / T) of 8 logits at v0, drafted tokens zero.
__device__ __forceinline__ void residual_terms(const VerifyArgs& a, const int* kids, int n, uint4 raw, float m, int v0,
                                               double (&e)[8]) {
  float x[8];
  split8(raw, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = exp((static_cast<double>(x[i]) - static_cast<double>(m)) * a.inv_t);
  drop_tokens(kids, n, v0, e);
}

// The token that the residual of `row` gives to its uniform number, into *out by the calling
// workgroup.  x: a lane's kSlices slice sums (the same in every wavefront), `rest` their sum,
// `drafted` the drafted tokens' share, all relative to the maximum m; kid: the drafted tokens.
__device__ __forceinline__ void pick_residual(const VerifyArgs& a, int row, float m, const double (&x)[kSlices], double rest,
                                              double drafted, const int* kid, int n, double* part, int* out) {
  const int t = threadIdx.x, wave = t / kWave;
  const uint16_t* l = a.logits + static_cast<size_t>(row) * a.V;
  int token = -1;
  if (rest > 0.0) {
    const double target = fmax(static_cast<double>(a.uniform[row]) * (rest + drafted) - drafted, 0.0);
    double before = 0.0, unused, e[8];
    const int slice = find_term(x, 0, 0.0, target, &before);
    const int v0 = slice * kVerifySlice + 8 * t;
    residual_terms(a, kid, n, load_logits(a, l, v0), m, v0, e);
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += e[i];
    s = wave_add(s);
    if (t % kWave == 0) part[wave] = s;
    __syncthreads();
    // The wavefront in whose share the target falls, or the last with a share.
    double start = before;
    int owner = 0;  // (with no share anywhere find_term gives -1)
    double owner_start = 0.0;
    for (int w = 0; w < kResWaves; ++w) {
      const double up = start + part[w];
      if (part[w] > 0.0) {
        owner = w;
        owner_start = start;
        if (up > target) break;
      }
      start = up;
    }
    if (wave != owner) return;
    token = find_term(e, slice * kVerifySlice + 8 * kWave * wave, owner_start, target, &unused);
    if (t % kWave == 0) put(out, token);
    return;
  }
  // The drafted tokens hold everything, and rounding kept u from all of them: the last of them.
  if (t == 0) {
    for (int i = 0; i < n; ++i)
      if (__uint_as_float(static_cast<uint32_t>(l[kid[i]]) << 16) > -INFINITY) token = max(token, kid[i]);
    put(out, token);
  }
}

__global__ __launch_bounds__(kResThreads) void k_verify_residual(VerifyArgs a) {
  constexpr int kOwn = kVerifyMaxTokens / kResThreads;  // drafted tokens a thread looks at
  __shared__ int kid_j[kVerifyMaxTokens], kid[kVerifyMaxTokens];  // the row's drafted tokens
  __shared__ float kid_l[kVerifyMaxTokens];                       // and their logits
  __shared__ double part[2][kResWaves], share[kVerifyMaxTokens];
  __shared__ int n, flag;
  const int t = threadIdx.x, wave = t / kWave;
  // The tree's loads before the row's, which wait for the path's end.
  int parent[kOwn], token[kOwn];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int j = t + i * kResThreads;
    parent[i] = j < a.N ? a.parent[j] : INT_MAX - 1;
    token[i] = j < a.N ? a.token[j] : 0;
  }
  const int row = *a.last_row;
  const float2 st = *a.last_stat;
  if (!(st.y > 0.f)) {  // no distribution (the same for every workgroup)
    if (blockIdx.x == 0 && t == 0) *a.next_token = -1;
    return;
  }
  const uint16_t* l = a.logits + static_cast<size_t>(row) * a.V;
  const int v0 = blockIdx.x * kVerifySlice + 8 * t;
  const uint4 raw = load_logits(a, l, v0);
  if (t == 0) n = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int j = t + i * kResThreads;
    if (continues(a, j, parent[i], token[i], row)) {
      const int at = atomicAdd(&n, 1);
      kid_j[at] = j;
      kid[at] = token[i];
      kid_l[at] = __uint_as_float(static_cast<uint32_t>(l[token[i]]) << 16);
    }
  }
  __syncthreads();
  double e[8];
  residual_terms(a, kid, n, raw, st.x, v0, e);
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) s += e[i];
  s = wave_add(s);
  if (t % kWave == 0) part[0][wave] = s;
  __syncthreads();
  if (t == 0) {
    s = part[0][0];
#pragma unroll
    for (int w = 1; w < kResWaves; ++w) s += part[0][w];
    put(a.slice_sum + blockIdx.x, s);
  }
  if (!last_to_arrive(a.cnt, gridDim.x, &flag)) return;

  // The last workgroup: the drafted tokens' share (each token once, summed in index order),
  // the slice, the token.  Every wavefront finds the slice itself.
  double x[kSlices], rest = 0.0;
#pragma unroll
  for (int i = 0; i < kSlices; ++i) {
    const int at = kSlices * (t % kWave) + i;
    x[i] = at < static_cast<int>(gridDim.x) ? get(a.slice_sum + at) : 0.0;
    rest += x[i];
  }
  rest = wave_add(rest);
  // in index order, whatever order they were found in
  for (int k = t; k < n; k += kResThreads) {
    int rank = 0;
    bool repeat = false;
    for (int i = 0; i < n; ++i) {
      const bool first = kid_j[i] < kid_j[k];
      rank += first;
      repeat |= first && kid[i] == kid[k];
    }
    share[rank] = repeat ? 0.0
                         : exp((static_cast<double>(kid_l[k]) - static_cast<double>(st.x)) * a.inv_t);
  }
  __syncthreads();
  double drafted = 0.0;
  for (int k = t % kWave; k < n; k += kWave) drafted += share[k];
  drafted = wave_add(drafted);
  pick_residual(a, row, st.x, x, rest, drafted, kid, n, part[1], a.next_token);
}

// Everything in one kernel, workgroup (row, slice of 2048 logits); the last workgroup of a row finds
// the row's pick, its residual's too, the last of all the path.
__global__ __launch_bounds__(kResThreads) void k_verify_small(VerifyArgs a) {
  __shared__ double sums[kSlices * kWave], share[kResThreads], part[2][kResWaves];
  __shared__ float wm[2][kResWaves];
  __shared__ int kid_j[kResThreads], kid[kResThreads], order[kResThreads], next[kResThreads], end_token[kResThreads];
  __shared__ float kid_l[kResThreads];
  __shared__ int n, flag;
  const int t = threadIdx.x, wave = t / kWave, lane = t % kWave;
  const int slices = (a.V + kVerifySlice - 1) / kVerifySlice;
  const int row = blockIdx.x / slices, slice = blockIdx.x % slices;
  const uint16_t* l = a.logits + static_cast<size_t>(row) * a.V;
  const int v0 = slice * kVerifySlice + 8 * t;
  uint4 raw = make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);  // -inf
  if (v0 < a.V) raw = *reinterpret_cast<const uint4*>(l + v0);
  if (t == 0) n = 0;
  __syncthreads();
  const int token = t < a.N ? a.token[t] : -1, parent = t < a.N ? a.parent[t] : -1;
  if (continues(a, t, parent, token, row)) {  // the row's children, in any order
    const int at = atomicAdd(&n, 1);
    kid_j[at] = t;
    kid[at] = token;
    kid_l[at] = __uint_as_float(static_cast<uint32_t>(l[token]) << 16);
  }
  // the slice's maximum; a NaN or +inf in it makes the sum NaN
  float x[8], m = -INFINITY;
  split8(raw, x);
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    m = fmaxf(m, x[i]);
    bad |= !(x[i] < INFINITY);
  }
  m = wave_top(m);
  if (lane == 0) wm[0][wave] = m;
  const int any_bad = __syncthreads_or(bad);
#pragma unroll
  for (int w = 0; w < kResWaves; ++w) m = fmaxf(m, wm[0][w]);
  double e[8], s = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = x[i] == -INFINITY ? 0.0 : exp((static_cast<double>(x[i]) - static_cast<double>(m)) * a.inv_t);
  drop_tokens(kid, n, v0, e);
#pragma unroll
  for (int i = 0; i < 8; ++i) s += e[i];
  s = wave_add(s);
  if (lane == 0) part[0][wave] = s;
  __syncthreads();
  if (t == 0) {
    s = part[0][0];
#pragma unroll
    for (int w = 1; w < kResWaves; ++w) s += part[0][w];
    put(a.slice_sum + blockIdx.x, any_bad ? __longlong_as_double(0x7FF8000000000000ll) : s);
    put(a.slice_max + blockIdx.x, m);
  }
  if (!last_to_arrive(a.cnt + kCounterStep * (1 + row), slices, &flag)) return;

  // The row: its maximum, its slices' sums relative to it, and their sum.
  double v[kRowSlices];
  float vm[kRowSlices], rm = -INFINITY;
#pragma unroll
  for (int i = 0; i < kRowSlices; ++i) {
    const int c = t + i * kResThreads;
    v[i] = c < slices ? get(a.slice_sum + row * slices + c) : 0.0;
    vm[i] = c < slices ? get(a.slice_max + row * slices + c) : -INFINITY;
    rm = fmaxf(rm, vm[i]);
  }
  rm = wave_top(rm);
  if (lane == 0) wm[1][wave] = rm;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kResWaves; ++w) rm = fmaxf(rm, wm[1][w]);
#pragma unroll
  for (int i = 0; i < kRowSlices; ++i) {
    // (a slice of -inf alone has nothing; a NaN stays one)
    if (v[i] != 0.0) v[i] *= exp((static_cast<double>(vm[i]) - static_cast<double>(rm)) * a.inv_t);
    sums[t + i * kResThreads] = v[i];
  }
  // its children's shares in index order, a repeated token's 0
  const int nk = n;
  if (t < nk) {
    int rank = 0;
    bool repeat = false;
    for (int i = 0; i < nk; ++i) {
      const bool before = kid_j[i] < kid_j[t];
      rank += before;
      repeat |= before && kid[i] == kid[t];
    }
    order[rank] = kid_j[t];
    share[rank] = repeat || kid_l[t] == -INFINITY ? 0.0 : exp((static_cast<double>(kid_l[t]) - static_cast<double>(rm)) * a.inv_t);
  }
  __syncthreads();
  // Every thread's own, in the same order: the sums, and the first child whose interval holds u.
  double y[kSlices], rest = 0.0, drafted = 0.0;
#pragma unroll
  for (int i = 0; i < kSlices; ++i) {
    y[i] = sums[kSlices * lane + i];
    rest += y[i];
  }
  rest = wave_add(rest);
  for (int k = 0; k < nk; ++k) drafted += share[k];
  const bool ok = fabsf(rm) < INFINITY && rest == rest;
  int own = -1;
  if (ok) {
    const double target = static_cast<double>(a.uniform[row]) * (rest + drafted);
    double f = 0.0;
    for (int k = 0; k < nk && own < 0; ++k) {
      const double f2 = f + share[k];
      if (f <= target && target < f2) own = order[k];
      f = f2;
    }
  }
  if (t == 0) {
    put(a.next + row, own);
    if (!ok) put(a.row_token + row, -1);  // no distribution
  }
  if (ok && own < 0) pick_residual(a, row, rm, y, rest, drafted, kid, nk, part[1], a.row_token + row);
  if (!last_to_arrive(a.cnt, a.N + 1, &flag)) return;

  // The path.
  for (int r = t; r <= a.N; r += kResThreads) {
    next[r] = get(a.next + r);
    end_token[r] = get(a.row_token + r);  // (of a row that goes on, whatever was there)
  }
  __syncthreads();
  if (t == 0) {
    int r = 0, len = 0;
    for (int j; (j = next[r]) >= 0; r = j + 1) a.path[len++] = j;  // j >= r: it ends
    *a.accepted = len;
    *a.next_token = end_token[r];
    n = len;
  }
  __syncthreads();
  for (int i = n + t; i < a.N; i += kResThreads) a.path[i] = -1;
}

}  // namespace

void verify_plan(int N, int V, int* chunks, int* chunk_len) {
  // about 640 workgroups, each with at least two tiles (a call at V = 152064 against 320 and 1280 of them:
  // 34 rows 18.5 us, 19.4 and 18.7; 101 rows 20.7, 21.4 and 21.2; 289 rows 29.0, 29.3 and 29.2; 1025
  // rows 73.5, 74.1 and 83.3; greedy 61 rows 10.1, 10.7 and 10.6)
  int c = (640 + N) / (N + 1);
  const int most = (V + 2 * kRowTile - 1) / (2 * kRowTile);
  if (c > most) c = most;
  if (c < 1) c = 1;
  *chunk_len = ((V + c - 1) / c + 7) / 8 * 8;
  *chunks = (V + *chunk_len - 1) / *chunk_len;
}

// One kernel against two, us a call.  16 slices a row: 1456 in all 14.7 against 15.9, 1776 16.1 against 16.1,
// 2016 17.2 against 16.3 (8 a row: 1024 13.6 against 16.6, 2048 18.9 against 17.5).  63 a row: 2142 16.4
// against 17.8, 75 a row: 2175 16.2 against 18.2; the two kernels take longer there, a row being longer.
bool verify_small(int N, int V) {
  const long long slices = (V + kVerifySlice - 1) / kVerifySlice;
  return N < kResThreads && (N + 1) * slices <= (slices < 32 ? 1750 : 2200);
}

// After the completion counters, small calls: the slices' sums and maxima, the rows' picks and the
// tokens of those that end the path.  Others: the last row
// and its (reference, sum), its slices' sums, the rows' (reference, sum) pairs, the slices' of
// rows, the rows' picks.
size_t verify_workspace_bytes(int N, int V) {
  int chunks = 0, len = 0;
  verify_plan(N, V, &chunks, &len);
  const size_t slices = (V + kVerifySlice - 1) / kVerifySlice, rows = N + 1;
  const size_t small = verify_small(N, V) ? rows * (slices * (sizeof(double) + sizeof(float)) + 2 * sizeof(int)) : 0;
  const size_t large = 16 + slices * sizeof(double) + rows * (1 + chunks) * sizeof(float2) + rows * sizeof(int);
  return kSplitCounterBytes + std::max(small, large);
}

void verify_workspace(VerifyArgs* a, void* ws) {
  char* p = static_cast<char*>(ws);
  a->cnt = reinterpret_cast<unsigned*>(p);
  p += kSplitCounterBytes;
  const int slices = (a->V + kVerifySlice - 1) / kVerifySlice;
  if (!a->greedy && verify_small(a->N, a->V)) {
    a->slice_sum = reinterpret_cast<double*>(p);
    a->slice_max = reinterpret_cast<float*>(a->slice_sum + static_cast<size_t>(a->N + 1) * slices);
    a->next = reinterpret_cast<int*>(a->slice_max + static_cast<size_t>(a->N + 1) * slices);
    a->row_token = a->next + (a->N + 1);
    return;
  }
  a->last_row = reinterpret_cast<int*>(p);
  a->last_stat = reinterpret_cast<float2*>(p + 8);
  a->slice_sum = reinterpret_cast<double*>(p + 16);
  a->row_stat = reinterpret_cast<float2*>(a->slice_sum + slices);
  a->stat = a->row_stat + (a->N + 1);
  a->next = reinterpret_cast<int*>(a->stat + static_cast<size_t>(a->N + 1) * a->chunks);
}

hipError_t launch_tree_verify(const VerifyArgs& a, hipStream_t st) {
  const int slices = (a.V + kVerifySlice - 1) / kVerifySlice;
  if (!a.greedy && verify_small(a.N, a.V)) {
    hipLaunchKernelGGL(k_verify_small, dim3((a.N + 1) * slices), dim3(kResThreads), 0, st, a);
    return hipGetLastError();
  }
  const dim3 rows((a.N + 1) * a.chunks);
  if (a.greedy)
    hipLaunchKernelGGL(k_verify_rows<true>, rows, dim3(kRowThreads), 0, st, a);
  else
    hipLaunchKernelGGL(k_verify_rows<false>, rows, dim3(kRowThreads), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.greedy) return e;
  hipLaunchKernelGGL(k_verify_residual, dim3(slices), dim3(kResThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace subspec
