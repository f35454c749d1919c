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
//   k_verify_rows     per (row, slice) workgroup the maximum and the sum, 32 bits
//   k_verify_walk     one workgroup: every token's interval, then the path
//   k_verify_residual the last row's other tokens in 64 bits: with V = 152064 tokens the
//                     borders lie 10^-5 apart, and a sum in 32 bits, 10^-7 off, would pick a
//                     neighbour in one call of a hundred; the last workgroup to finish finds
//                     the token.
#include <climits>
#include <cmath>

#include "device_common.h"
#include "kernels_verify.h"

namespace subspec {

namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / kWave;
constexpr int kRowLoads = 4;  // 16-byte loads in flight per thread

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

// A row's (m, s): s = sum of 2^(c (l - m)); -inf (nothing seen yet, or masked logits) adds
// nothing.  NaN and +inf in a row leave m or s not finite.
__device__ __forceinline__ void merge(float c, float& m, float& s, float m2, float s2) {
  const float mx = fmaxf(m, m2);
  if (mx == -INFINITY) {
    s += s2;  // zeros, or a NaN to be shown
    return;
  }
  s = (m == -INFINITY ? s : s * __builtin_amdgcn_exp2f(c * (m - mx))) +
      (m2 == -INFINITY ? s2 : s2 * __builtin_amdgcn_exp2f(c * (m2 - mx)));
  m = mx;
}

__global__ __launch_bounds__(kRowThreads) void k_verify_rows(VerifyArgs a) {
  __shared__ float wm[kRowWaves], ws[kRowWaves];
  const int row = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int lo = chunk * a.chunk_len, hi = min(a.V, lo + a.chunk_len);
  const uint16_t* l = a.logits + static_cast<size_t>(row) * a.V;
  float m = -INFINITY, s = 0.f;
  for (int v0 = lo + 8 * static_cast<int>(threadIdx.x); v0 < hi; v0 += 8 * kRowThreads * kRowLoads) {
    uint4 w[kRowLoads];
#pragma unroll
    for (int j = 0; j < kRowLoads; ++j) {
      const int v = v0 + 8 * kRowThreads * j;
      w[j] = v < hi ? *reinterpret_cast<const uint4*>(l + v) : make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
    }
#pragma unroll
    for (int j = 0; j < kRowLoads; ++j) {
      float x[8];
      split8(w[j], x);
      float mx = m;
#pragma unroll
      for (int e = 0; e < 8; ++e) mx = fmaxf(mx, x[e]);
      if (mx == -INFINITY) {  // nothing but -inf (or NaN, which the sum has to show)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += x[e] == x[e] ? 0.f : x[e];
        continue;
      }
      s = m == -INFINITY ? s : s * __builtin_amdgcn_exp2f(a.c * (m - mx));
      m = mx;
#pragma unroll
      for (int e = 0; e < 8; ++e) s += __builtin_amdgcn_exp2f(a.c * (x[e] - mx));
    }
  }
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) merge(a.c, m, s, __shfl_xor(m, d), __shfl_xor(s, d));
  if (threadIdx.x % kWave == 0) {
    wm[threadIdx.x / kWave] = m;
    ws[threadIdx.x / kWave] = s;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    m = wm[0];
    s = ws[0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) merge(a.c, m, s, wm[w], ws[w]);
    a.stat[blockIdx.x] = make_float2(m, s);
  }
}

// Greedy: the slice's largest logit and its lowest token; a NaN makes the row have none
// (stored as NaN).
__device__ __forceinline__ void best_of(float& m, int& i, float m2, int i2) {
  const bool take = m != m ? false : m2 != m2 ? true : m2 > m || (m2 == m && i2 < i);
  m = take ? m2 : m;
  i = take ? i2 : i;
}

__global__ __launch_bounds__(kRowThreads) void k_verify_best(VerifyArgs a) {
  __shared__ float wm[kRowWaves];
  __shared__ int wi[kRowWaves];
  const int row = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int lo = chunk * a.chunk_len, hi = min(a.V, lo + a.chunk_len);
  const uint16_t* l = a.logits + static_cast<size_t>(row) * a.V;
  float m = -INFINITY;
  int i = INT_MAX;
  for (int v0 = lo + 8 * static_cast<int>(threadIdx.x); v0 < hi; v0 += 8 * kRowThreads * kRowLoads) {
    uint4 w[kRowLoads];
#pragma unroll
    for (int j = 0; j < kRowLoads; ++j) {
      const int v = v0 + 8 * kRowThreads * j;
      w[j] = v < hi ? *reinterpret_cast<const uint4*>(l + v) : make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
    }
#pragma unroll
    for (int j = 0; j < kRowLoads; ++j) {
      float x[8];
      split8(w[j], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        // within a thread the tokens come in order: a later equal one does not replace
        const bool take = x[e] > m || x[e] != x[e];
        m = take && m == m ? x[e] : m;
        i = take ? v0 + 8 * kRowThreads * j + e : i;
      }
    }
  }
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) best_of(m, i, __shfl_xor(m, d), __shfl_xor(i, d));
  if (threadIdx.x % kWave == 0) {
    wm[threadIdx.x / kWave] = m;
    wi[threadIdx.x / kWave] = i;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    m = wm[0];
    i = wi[0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) best_of(m, i, wm[w], wi[w]);
    a.stat[blockIdx.x] = make_float2(m, __int_as_float(i));
  }
}

constexpr int kWalkThreads = 1024;

__global__ __launch_bounds__(kWalkThreads) void k_verify_walk(VerifyArgs a) {
  __shared__ float rm[kVerifyMaxTokens + 1], rs[kVerifyMaxTokens + 1];  // rows' maxima and sums (greedy: tokens)
  __shared__ float pj[kVerifyMaxTokens];
  __shared__ int par[kVerifyMaxTokens], tok[kVerifyMaxTokens], next[kVerifyMaxTokens + 1];
  const int t = threadIdx.x;
  for (int r = t; r <= a.N; r += kWalkThreads) {
    float2 st = a.stat[static_cast<size_t>(r) * a.chunks];
    if (a.greedy) {
      int i = __float_as_int(st.y);
      for (int c = 1; c < a.chunks; ++c) {
        const float2 o = a.stat[static_cast<size_t>(r) * a.chunks + c];
        best_of(st.x, i, o.x, __float_as_int(o.y));
      }
      // no finite largest logit: nothing is picked
      rs[r] = __int_as_float(fabsf(st.x) < INFINITY ? i : -1);
    } else {
      for (int c = 1; c < a.chunks; ++c) {
        const float2 o = a.stat[static_cast<size_t>(r) * a.chunks + c];
        merge(a.c, st.x, st.y, o.x, o.y);
      }
      const bool ok = fabsf(st.x) < INFINITY && st.y > 0.f && st.y < INFINITY;
      rm[r] = st.x;
      rs[r] = ok ? st.y : 0.f;
    }
    next[r] = -1;
  }
  if (t < a.N) {
    const int p = a.parent[t], k = a.token[t];
    // a parent that does not come before its child, or a token outside the vocabulary: never accepted
    const bool ok = p >= -1 && p < t && k >= 0 && k < a.V;
    par[t] = ok ? p : -2;
    tok[t] = k;
  }
  __syncthreads();
  const bool ok = t < a.N && par[t] != -2;
  const int row = ok ? par[t] + 1 : 0;
  if (a.greedy) {
    if (ok && tok[t] == __float_as_int(rs[row])) {
      bool first = true;  // of equal siblings the first
      for (int i = 0; i < t; ++i) first &= !(par[i] == par[t] && tok[i] == tok[t]);
      if (first) next[row] = t;
    }
    __syncthreads();
  } else {
    float p = 0.f;
    if (ok && rs[row] > 0.f) {
      const uint32_t bits = a.logits[static_cast<size_t>(row) * a.V + tok[t]];
      p = __builtin_amdgcn_exp2f(a.c * (__uint_as_float(bits << 16) - rm[row])) / rs[row];
    }
    if (t < a.N) {
      for (int i = 0; i < t; ++i)
        if (ok && par[i] == par[t] && tok[i] == tok[t]) p = 0.f;
      pj[t] = p;
    }
    __syncthreads();
    if (p > 0.f) {
      float f = 0.f;
      for (int i = 0; i < t; ++i)
        if (par[i] == par[t]) f += pj[i];
      const float u = a.uniform[row];
      if (f <= u && u < f + p) next[row] = t;
    }
    __syncthreads();
  }
  if (t == 0) {
    int r = 0, n = 0;
    for (int j; (j = next[r]) >= 0; r = j + 1) a.path[n++] = j;  // j >= r: it ends
    *a.accepted = n;
    par[0] = n;
    if (a.greedy) {
      *a.next_token = __float_as_int(rs[r]);
    } else {
      *a.last_row = r;
      *a.row_stat = make_float2(rm[r], rs[r]);
    }
  }
  __syncthreads();
  for (int i = t; i < a.N; i += kWalkThreads)
    if (i >= par[0]) a.path[i] = -1;
}

constexpr int kResThreads = 256;
static_assert(kVerifySlice == 8 * kResThreads, "eight logits a thread");

struct Residual {
  int kids[kVerifyMaxTokens];  // the last row's drafted tokens
  int n, last;
  double sum[kResThreads / kWave];
};

// e^((l - m) / T) of this thread's 8 logits of a slice, drafted tokens and logits past the
// vocabulary zero.
__device__ __forceinline__ void residual_terms(const VerifyArgs& a, const Residual& sh, const uint16_t* l, float m, int v0,
                                               double (&e)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = 0.0;
  if (v0 >= a.V) return;
  float x[8];
  split8(*reinterpret_cast<const uint4*>(l + v0), x);
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = exp((static_cast<double>(x[i]) - static_cast<double>(m)) * a.inv_t);
  for (int k = 0; k < sh.n; ++k) {
    const int d = sh.kids[k] - v0;
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = d == i ? 0.0 : e[i];
  }
}

__device__ __forceinline__ double wave_add(double v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// The first of the workgroup's terms (K a thread, in order, the first of thread 0's with
// number `first`) whose running sum passes `target`; if none does, the last positive one; -1 if
// no term is positive.  Every thread gets the number, and in *before the sum of the terms in
// front of it.
template <int K>
__device__ int find_term(const double (&e)[K], int first, double target, double* wsum, int* found, double* before) {
  const int t = threadIdx.x;
  double own = 0.0;
#pragma unroll
  for (int i = 0; i < K; ++i) own += e[i];
  double incl = own;  // inclusive sum over the wavefront's lanes
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const double o = __shfl_up(incl, d);
    if (t % kWave >= d) incl += o;
  }
  if (t % kWave == kWave - 1) wsum[t / kWave] = incl;
  if (t < 2) found[t] = t == 0 ? INT_MAX : -1;
  __syncthreads();
  double run = incl - own;
  for (int w = 0; w < t / kWave; ++w) run += wsum[w];
  const double start = run;
  int hit = INT_MAX, any = -1;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    run += e[i];
    if (e[i] > 0.0) {
      any = first + K * t + i;
      if (run > target && hit == INT_MAX) hit = any;
    }
  }
  if (hit != INT_MAX) atomicMin(&found[0], hit);
  if (any >= 0) atomicMax(&found[1], any);
  __syncthreads();
  const int r = found[0] != INT_MAX ? found[0] : found[1];
  const int mine = r - (first + K * t);
  if (mine >= 0 && mine < K) {
    run = start;
#pragma unroll
    for (int i = 0; i < K; ++i)
      if (i < mine) run += e[i];
    wsum[0] = run;
  }
  __syncthreads();
  *before = wsum[0];
  __syncthreads();
  return r;
}

// The threads' sum, in a fixed order, in every thread.
__device__ double block_add(double v, double* wsum) {
  v = wave_add(v);
  if (threadIdx.x % kWave == 0) wsum[threadIdx.x / kWave] = v;
  __syncthreads();
  v = wsum[0];
#pragma unroll
  for (int w = 1; w < kResThreads / kWave; ++w) v += wsum[w];
  __syncthreads();
  return v;
}

__device__ __forceinline__ bool is_child(const VerifyArgs& a, int j, int row) {
  const int p = a.parent[j], k = a.token[j];
  return p + 1 == row && p >= -1 && p < j && k >= 0 && k < a.V;
}

__global__ __launch_bounds__(kResThreads) void k_verify_residual(VerifyArgs a) {
  __shared__ Residual sh;
  __shared__ int found[2];
  const int t = threadIdx.x;
  const int row = *a.last_row;
  const float2 st = *a.row_stat;
  if (!(st.y > 0.f)) {  // no distribution (the same for every workgroup)
    if (blockIdx.x == 0 && t == 0) *a.next_token = -1;
    return;
  }
  if (t == 0) sh.n = 0;
  __syncthreads();
  for (int j = t; j < a.N; j += kResThreads)
    if (is_child(a, j, row)) sh.kids[atomicAdd(&sh.n, 1)] = a.token[j];  // in any order
  __syncthreads();
  const uint16_t* l = a.logits + static_cast<size_t>(row) * a.V;
  double e[8];
  residual_terms(a, sh, l, st.x, blockIdx.x * kVerifySlice + 8 * t, e);
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) s += e[i];
  s = block_add(s, sh.sum);
  if (t == 0) {
    __hip_atomic_store(a.slice_sum + blockIdx.x, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // the sum is out before the counter says so
    sh.last = __hip_atomic_fetch_add(a.cnt, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (!sh.last) return;

  // The last workgroup: the drafted tokens' share (each once), the slice, the token.
  double drafted = 0.0;
  for (int j = t; j < a.N; j += kResThreads) {
    if (!is_child(a, j, row)) continue;
    const int k = a.token[j];
    bool once = true;
    for (int i = 0; i < j && once; ++i) once = !(is_child(a, i, row) && a.token[i] == k);
    if (once)
      drafted += exp((static_cast<double>(__uint_as_float(static_cast<uint32_t>(l[k]) << 16)) - static_cast<double>(st.x)) * a.inv_t);
  }
  drafted = block_add(drafted, sh.sum);
  constexpr int kSlices = kVerifyMaxV / kVerifySlice / kResThreads;  // a thread
  double x[kSlices], mine = 0.0;
#pragma unroll
  for (int i = 0; i < kSlices; ++i) {
    const int at = kSlices * t + i;
    x[i] = at < static_cast<int>(gridDim.x) ? __hip_atomic_load(a.slice_sum + at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
    mine += x[i];
  }
  const double rest = block_add(mine, sh.sum);
  int token = -1;
  if (rest > 0.0) {
    const double target = fmax(static_cast<double>(a.uniform[row]) * (rest + drafted) - drafted, 0.0);
    double before = 0.0, unused;
    const int slice = find_term(x, 0, target, sh.sum, found, &before);
    residual_terms(a, sh, l, st.x, slice * kVerifySlice + 8 * t, e);
    token = find_term(e, slice * kVerifySlice, target - before, sh.sum, found, &unused);
  } else {
    // the drafted tokens hold everything, and rounding kept u from all of them: the last of them
    for (int i = 0; i < sh.n; ++i)
      if (__uint_as_float(static_cast<uint32_t>(l[sh.kids[i]]) << 16) > -INFINITY) token = max(token, sh.kids[i]);
  }
  if (t == 0) {
    *a.next_token = token;
    __hip_atomic_store(a.cnt, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

}  // namespace

void verify_plan(int N, int V, int* chunks, int* chunk_len) {
  // about 1024 workgroups, each with at least one round of loads
  int c = (1024 + N) / (N + 1);
  const int most = (V + 8 * kRowThreads * kRowLoads - 1) / (8 * kRowThreads * kRowLoads);
  if (c > most) c = most;
  if (c < 1) c = 1;
  *chunk_len = ((V + c - 1) / c + 7) / 8 * 8;
  *chunks = (V + *chunk_len - 1) / *chunk_len;
}

// After the completion counters: the last row and its (maximum, sum), the slices' sums,
// the rows' pairs.
size_t verify_workspace_bytes(int N, int V) {
  int chunks = 0, len = 0;
  verify_plan(N, V, &chunks, &len);
  const size_t slices = (V + kVerifySlice - 1) / kVerifySlice;
  return kSplitCounterBytes + 16 + slices * sizeof(double) + static_cast<size_t>(N + 1) * chunks * sizeof(float2);
}

hipError_t launch_tree_verify(const VerifyArgs& a, hipStream_t st) {
  const dim3 rows((a.N + 1) * a.chunks);
  if (a.greedy)
    hipLaunchKernelGGL(k_verify_best, rows, dim3(kRowThreads), 0, st, a);
  else
    hipLaunchKernelGGL(k_verify_rows, rows, dim3(kRowThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_verify_walk, dim3(1), dim3(kWalkThreads), 0, st, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.greedy) return e;
  hipLaunchKernelGGL(k_verify_residual, dim3((a.V + kVerifySlice - 1) / kVerifySlice), dim3(kResThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace subspec
