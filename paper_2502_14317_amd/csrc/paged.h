// Drafted trees over a paged cache: internal declarations of the append (paged_append.hip), the attention (tree_attn.hip),
// the log probabilities (logprobs.hip) and the acceptance (tree_accept.hip), and what they share on the device.
#pragma once
#include "pc_common.h"
#include "page_row.h"

#define PC_TREE_NODES 64          // a node a lane

__device__ __forceinline__ int pc_tree_rows(const int32_t* n_rows, long long b, int n) {
  return n_rows ? min(max(n_rows[b], 0), n) : n;
}
// Nodes above lane t's node and itself, as bits: pointers jump twice as far each time, so that six times reach 64 nodes.
// parent: of the lane's node (anything outside [0, lane): a root)
__device__ __forceinline__ unsigned long long pc_tree_above(int parent, int lane) {
  int up = parent >= 0 && parent < lane ? parent : -1;
  unsigned long long above = 1ull << lane;
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    const int from = up < 0 ? lane : up;
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)above, from), hi = (uint32_t)__shfl((int)(uint32_t)(above >> 32), from);
    above |= (unsigned long long)hi << 32 | lo;
    const int next = __shfl(up, from);
    up = up < 0 ? -1 : next;
  }
  return above;
}
// ... of sequence b's tree (up to 64 nodes of n)
__device__ __forceinline__ unsigned long long pc_tree_above(const int32_t* parent, long long b, int n, int lane) {
  if (!parent) return ~0ull >> (63 - lane);
  return pc_tree_above(lane < n ? parent[b * n + lane] : -1, lane);
}

// ---- append
struct PcPagedAppend {
  const uint16_t* k_new;
  const uint16_t* v_new;
  long long batch_stride, row_stride, head_stride;
  const int32_t* parent;
  const int32_t* n_rows;
  const int32_t* pos;
  int pos0;
  float rope_base;
  int batch, n_new, n_kv_heads, head_dim;
  PcPages pages;
  const int32_t* len_in;
  int32_t* len_out;
};
int pc_launch_append_paged(const PcPagedAppend& c, hipStream_t st);

// ---- attention
struct PcTreeCall {
  const uint16_t* q;
  long long batch_stride, row_stride;
  const int32_t* parent;
  const int32_t* n_rows;
  const int32_t* pos;
  int pos0;
  float rope_base, scale;
  PcPages pages;
  const int32_t* len;
  int batch, n, n_q_heads, n_kv_heads, head_dim;
  uint16_t* out;           // [B, n, H_q, D]
  float* lse;              // [B, H_q, n] or nullptr
};
struct PcTreePlan { int rows, tiles, shares; };      // query rows a workgroup, tiles of them a KV head, cuts of the batch's keys (0: one launch)
PcTreePlan pc_tree_plan(const PcTreeCall& c);
bool pc_tree_fits(const PcTreeCall& c, const PcTreePlan& p);
size_t pc_tree_ws_bytes(const PcTreeCall& c, const PcTreePlan& p);
int pc_launch_tree_attn(const PcTreeCall& c, const PcTreePlan& p, void* ws, hipStream_t st);

// ---- log probabilities
#define PC_TOP_MOST 64
struct PcLogprobs {
  const void* logits;
  int fp32;
  long long row_stride;
  const int32_t* tokens;   // [rows, n_tokens]
  int n_tokens, n_top, rows, vocab;
  float* token_logprob;
  float* entropy;          // [rows] or nullptr
  int32_t* top_idx;        // [rows, n_top]
  float* top_logprob;      // or nullptr
};
size_t pc_logprobs_ws_bytes(int rows, int vocab, int n_top);
int pc_launch_logprobs(const PcLogprobs& c, void* ws, hipStream_t st);

// ---- acceptance
struct PcTreeAccept {
  const int32_t* tokens;
  const int32_t* parent;
  const int32_t* choice;
  int choice_stride;
  const int32_t* n_rows;
  int batch, n;
  PcPages pages;
  int moves;               // is there a cache
  int n_kv_heads, head_dim;
  const int32_t* len_in;
  int32_t* len_out;
  int32_t* pos;
  int32_t* path;
  int32_t* n_kept;
  int32_t* next_token;
};
int pc_launch_tree_accept(const PcTreeAccept& c, hipStream_t st);
