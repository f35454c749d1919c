// Host-visible launcher of the verification of a drafted tree (internal; the public ABI is
// include/subspec.h).
#pragma once

#include "kernels.h"

namespace subspec {

constexpr int kVerifyMaxTokens = 1024;
constexpr int kVerifyMaxV = 1 << 20;
constexpr int kVerifySlice = 2048;  // logits per workgroup of the kernels in 64 bits

struct VerifyArgs {
  const uint16_t* logits;  // bf16 [N + 1][V]
  const int* parent;       // [N]: -1 (the context) or an earlier token
  const int* token;        // [N]
  const float* uniform;    // [N + 1]; greedy: unused
  int N, V, greedy;
  float c;                 // log2(e) / T
  double inv_t;            // 1 / T
  int chunks, chunk_len;   // workgroups per row and the logits each one covers
  // workspace
  unsigned* cnt;           // completion counters (zero between launches): the residual's slices, rows, slices of each row
  float2* stat;            // [N + 1][chunks] reference, and sum of 2^(c (l - reference)) (greedy: the maximum and its token)
  float2* row_stat;        // [N + 1] the same of whole rows
  int* next;               // [N + 1] the drafted token that a row picks, or -1
  float2* last_stat;       // [1] row_stat of the path's last row
  int* last_row;           // [1]
  double* slice_sum;       // [ceil(V / kVerifySlice)] the last row's sums without its children (small calls: every row's)
  float* slice_max;        // small calls: [N + 1][ceil(V / kVerifySlice)] the slices' maxima
  int* row_token;          // small calls: [N + 1] the token of a row that ends the path
  int* path;               // [N]
  int* accepted;           // [1]
  int* next_token;         // [1]
};

void verify_plan(int N, int V, int* chunks, int* chunk_len);
size_t verify_workspace_bytes(int N, int V);
void verify_workspace(VerifyArgs* a, void* ws);  // fills the workspace's pointers; N, V and chunks are set
hipError_t launch_tree_verify(const VerifyArgs& a, hipStream_t st);

}  // namespace subspec
