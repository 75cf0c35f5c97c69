// The path of a drafted tree that the target follows, and its rows moved to where they stay.  A wavefront holds the tree, a
// node a lane: a step down is one ballot.  Every wavefront walks for itself (some 20 cycles a step) and then moves the rows of
// one KV head's keys or values: the rows of a path ascend, so place j lies at or before row path[j], and a row that
// has not been read yet is never written over: later rows of the path come from behind every place that is filled.
// Bound by latency: a chain of the tree's loads, the walk, the table, the rows.
#include "paged.h"

#define ACCEPT_WAVES 4

template <int LPR>                 // lanes a row: a row is LPR pieces of 16 bytes
__device__ __forceinline__ void accept_move(uint8_t* rows, float* scales, long long from, long long to, int count) {
  constexpr int AT_ONCE = PC_WAVE / LPR;
  const int lane = threadIdx.x % PC_WAVE;
  for (int j0 = 1; j0 < count; j0 += AT_ONCE) {             // (row 0 stays; lane j has path row j's places)
    const int j = j0 + lane / LPR, src = min(j, PC_WAVE - 1);
    const long long f = __shfl(from, src), t = __shfl(to, src);
    const bool moves = j < count && f >= 0 && t >= 0 && f != t;
    u32x4 x = {0, 0, 0, 0};
    float s = 0.f;
    if (moves) {
      x = *(const u32x4*)(rows + f * (16 * LPR) + lane % LPR * 16);
      if (scales) s = scales[f];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // the round's rows are read before any of them is written over
    if (moves) {
      *(u32x4*)(rows + t * (16 * LPR) + lane % LPR * 16) = x;
      if (scales && lane % LPR == 0) scales[t] = s;
    }
  }
}

__global__ __launch_bounds__(ACCEPT_WAVES* PC_WAVE) void tree_accept_kernel(PcTreeAccept c, int parts, PcDiv parts_div) {
  const int lane = threadIdx.x % PC_WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PC_WAVE);
  const int b = pc_div((int)blockIdx.x, parts_div), part = (int)blockIdx.x - b * parts;
  const int n_rows = pc_tree_rows(c.n_rows, b, c.n);
  const long long at = (long long)b * c.n + min(lane, c.n - 1);
  const int token = c.tokens[at], choice = c.choice[at * c.choice_stride], up = c.parent ? c.parent[at] : lane - 1;
  const int base = c.moves ? c.len_in[b] - n_rows : 0;
  int path = -1, count = 0, next = -1;
  if (n_rows > 0) {
    int cur = 0;
    for (;;) {                                              // (cur grows: 64 steps at most)
      if (lane == count) path = cur;
      ++count;
      next = __builtin_amdgcn_readlane(choice, cur);
      const unsigned long long hit = __ballot(lane < n_rows && lane > cur && up == cur && token == next);
      if (!hit) break;
      cur = __ffsll((long long)hit) - 1;
    }
  }
  if (part == 0 && wave == 0) {
    if (lane < c.n) c.path[(long long)b * c.n + lane] = path;
    if (lane == 0) {
      c.n_kept[b] = count;
      c.next_token[b] = next;
      if (c.moves && c.len_out) c.len_out[b] = base + count;
      if (c.pos) c.pos[b] += count;
    }
  }
  const int which = part * ACCEPT_WAVES + wave;             // (KV head, keys or values)
  if (!c.moves || which >= 2 * c.n_kv_heads || count < 2) return;
  const int g = which / 2;
  const long long from = lane < count ? pc_page_row(c.pages, b, (long long)base + path, g, c.n_kv_heads) : -1;
  const long long to = lane < count ? pc_page_row(c.pages, b, (long long)base + lane, g, c.n_kv_heads) : -1;
  uint8_t* rows = (uint8_t*)(which % 2 ? c.pages.v : c.pages.k);
  float* scales = which % 2 ? c.pages.v_scale : c.pages.k_scale;
  const int lanes = c.head_dim * (scales ? 1 : 2) / 16;
  if (lanes == 16) accept_move<16>(rows, scales, from, to, count);
  else if (lanes == 8) accept_move<8>(rows, scales, from, to, count);
  else accept_move<4>(rows, scales, from, to, count);
}

int pc_launch_tree_accept(const PcTreeAccept& c, hipStream_t st) {
  const int parts = c.moves ? (2 * c.n_kv_heads + ACCEPT_WAVES - 1) / ACCEPT_WAVES : 1;
  PcProfScope prof(PC_KERNEL_TREE_ACCEPT, st);
  hipLaunchKernelGGL(tree_accept_kernel, dim3((unsigned)(c.batch * parts)), dim3(ACCEPT_WAVES * PC_WAVE), 0, st, c, parts, pc_div_by(parts));
  PC_LAUNCH_CHECK();
  return PC_OK;
}
