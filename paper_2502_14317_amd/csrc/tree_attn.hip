// Attention of drafted trees over a paged cache.
//
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q . k_j,  over the rows in front of the tree and the
//   node's own ancestors (itself among them).
//
// The rows (node, head of the group) of a sequence and KV head are the columns of S^T = K Q^T.  A node's ancestors are the
// bits of one 64-bit word, which a wavefront finds with six exchanges (a node a lane) and a lane keeps for its columns: the
// mask of a tree costs a shift where a block holds rows of it, and nothing elsewhere.
// The keys of all sequences, laid end to end in blocks of 32, are cut into equal shares, a workgroup each for a KV head and a
// tile of query rows: so a batch of very unequal lengths keeps every CU busy, whatever the table's width.  A share is a
// piece of one sequence or of several; each piece leaves a partial (o, lse) a row at place share + sequence (both
// only grow along the keys, so a place is taken once), and tree_join_kernel joins a sequence's.
#include "paged.h"
#include "shared_core.h"
#include "serve.h"

#define TREE_WAVES 4
#define TREE_THREADS (TREE_WAVES * PC_WAVE)

struct TreeArgs {
  PcTreeCall c;
  PcRope rope;
  int group, n_tiles, n_shares, per_xcd;
  PcDiv group_div, tiles_div, heads_div;
  float scale_log2;
  float* part_o;           // [n_shares + B][H_kv][n group][D]
  float* part_lse;         // [n_shares + B][H_kv][n group]
  int2* span;              // [B] first and last share of a sequence
};

// 32-key blocks that sequence b has: none where it has no nodes
__device__ __forceinline__ int tree_len(const PcTreeCall& c, int b) {
  const long long cap = (long long)c.pages.max_pages << c.pages.shift;
  return (int)min((long long)max(c.len[b], 0), cap);
}
__device__ __forceinline__ int tree_blocks(const PcTreeCall& c, int b) {
  return pc_tree_rows(c.n_rows, b, c.n) > 0 ? (tree_len(c, b) + 31) / 32 : 0;
}

// Which of four keys a column sees: bit j is node first + j of the tree (a row in front of it where that is negative), of which
// `there` follow from the first one on.  No branches (a vector shift by the lane's own number costs as much as a test).
__device__ __forceinline__ uint32_t tree_sight(unsigned long long above, int first, int there) {
  const int up = min(max(first, 0), 63), down = min(max(-first, 0), 4);
  const uint32_t nodes = (uint32_t)(above >> up) << down | ((1u << down) - 1u);
  return nodes & ((1u << min(max(there, 0), 4)) - 1u);
}

// What a piece is about
struct TreePiece {
  int b, g, row0, n_here;  // query rows row0 .. row0 + n_here - 1 of (node, head)
  int len, base;           // rows that are there, the first of the tree's
};

// A 32-key block: its two halves of 16 keys, each inside a page
struct TreeBlock {
  int blk;
  long long row[2];        // of the pool
  int keys[2];             // that are there
};

template <int D, int NC, int WK, bool Q8>
struct TreeWalk {
  static constexpr int KSTEPS = D / 32, VE = D / 16, ELEM = Q8 ? 1 : 2, ROW = D * ELEM;
  static constexpr int KP = Q8 ? D / 64 : KSTEPS;
  typedef uint32_t vpiece __attribute__((ext_vector_type(VE * ELEM / 4)));
  u32x4 kbuf[2][KP];
  vpiece vbuf[8];
  float sbuf;
  TreeBlock cur;
  int end;                                                   // the run's last block is in front of it
  int tab, tab_next, tab0;                                   // 64 entries of the table from tab0 on, and the 64 behind them

  __device__ __forceinline__ int entries(const TreeArgs& a, const TreePiece& x, int at) const {
    const int i = min(at + (int)(threadIdx.x % PC_WAVE), a.c.pages.max_pages - 1);
    return a.c.pages.table[(long long)x.b * a.c.pages.max_pages + i];
  }
  __device__ __forceinline__ TreeBlock block(const TreeArgs& a, const TreePiece& x, int blk) {
    TreeBlock t;
    t.blk = blk;
    const int shift = a.c.pages.shift;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      t.row[h] = 0; t.keys[h] = 0;
      const int key = 32 * blk + 16 * h;
      if (blk >= end || key >= x.len) continue;
      const int at = key >> shift;
      if (at >= tab0 + PC_WAVE) {                            // (entries are taken in order)
        tab = tab_next; tab0 += PC_WAVE;
        tab_next = entries(a, x, tab0 + PC_WAVE);
      }
      const long long row = pc_pool_row(a.c.pages, __builtin_amdgcn_readlane(tab, at - tab0), key, x.g, a.c.n_kv_heads);
      if (row < 0) continue;
      t.row[h] = row;
      t.keys[h] = min(16, x.len - key);
    }
    return t;
  }
  __device__ __forceinline__ void keys(const TreeArgs& a, const TreeBlock& t) {
    const int lane = threadIdx.x % PC_WAVE, kk = lane / 16, c16 = lane % 16;
    if constexpr (Q8) {                                      // (every lane reads a row that the pool has)
      const int h = lane % 32 / 16;
      const long long row = (h ? t.row[1] : t.row[0]) + max(min(c16, (h ? t.keys[1] : t.keys[0]) - 1), 0);
      sbuf = (lane < 32 ? a.c.pages.k_scale : a.c.pages.v_scale)[row];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)a.c.pages.k + t.row[h] * ROW), 0, t.keys[h] * ROW, 0x00020000);
#pragma unroll
      for (int p = 0; p < KP; ++p) kbuf[h][p] = __builtin_amdgcn_raw_buffer_load_b128(r, c16 * ROW + 16 * kk, 64 * p, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ void values(const TreeArgs& a, const TreeBlock& t) {
    const int lane = threadIdx.x % PC_WAVE, kk = lane / 16, c16 = lane % 16;
    const int off = (4 * kk * D + VE * c16) * ELEM;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)a.c.pages.v + t.row[h] * ROW), 0, t.keys[h] * ROW, 0x00020000);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(vpiece) == 16) vbuf[4 * h + i] = __builtin_amdgcn_raw_buffer_load_b128(r, off, i * ROW, 0);
        else if constexpr (sizeof(vpiece) == 8) vbuf[4 * h + i] = __builtin_amdgcn_raw_buffer_load_b64(r, off, i * ROW, 0);
        else vbuf[4 * h + i] = __builtin_amdgcn_raw_buffer_load_b32(r, off, i * ROW, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // the wk-th of the piece's WK runs of blocks
  __device__ __forceinline__ void begin(const TreeArgs& a, const TreePiece& x, int blk0, int n_blk, int wk) {
    const int first = blk0 + (int)((long long)n_blk * wk / WK);
    end = blk0 + (int)((long long)n_blk * (wk + 1) / WK);
    tab0 = (32 * first) >> a.c.pages.shift;
    tab = entries(a, x, tab0);
    tab_next = entries(a, x, tab0 + PC_WAVE);
    cur = block(a, x, first);
    keys(a, cur);
    values(a, cur);
  }
  // One block.  MASKED: some of its keys are not there, or rows of the tree; few blocks are, so that the query operands come from
  // LDS there and leave their registers to the masks (in registers throughout, 128 values a row and 32 columns, 89 to 126
  // registers spilled, and every block waited for its own: 16 sequences of 11000 rows, 64 query rows a KV head, 363 us)
  template <bool MASKED>
  __device__ __forceinline__ void step(const TreeArgs& a, const TreePiece& x, SharedColumns<D, NC>& c, const unsigned long long (&above)[NC], float (*scale)[32],
                                       const uint16_t (*hi)[D + 8], const uint16_t (*lo)[D + 8], int col0) {
    const int lane = threadIdx.x % PC_WAVE, kk = lane / 16;
    const TreeBlock nx = block(a, x, cur.blk + 1);
    if constexpr (Q8) scale[lane / 32][lane % 32] = sbuf;
    floatx4 s[NC][1][2];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc)
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) s[nc][0][bi] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) {
        u32x4 ka;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if constexpr (Q8) ka[w] = shared_widen(kbuf[bi][ks / 2][2 * (ks % 2) + w / 2], w % 2);
          else ka[w] = kbuf[bi][ks][w];
        }
#pragma unroll
        for (int h = 1; h >= 0; --h)
#pragma unroll
          for (int nc = 0; nc < NC; ++nc) {
            bf16x8 q;
            if constexpr (MASKED) q = *(const bf16x8*)&(h ? lo : hi)[col0 + 16 * nc + lane % 16][shared_query_at(Q8, ks, kk)];
            else q = c.q[h][nc][ks];
            s[nc][0][bi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(bf16x8*)&ka, q, s[nc][0][bi], 0, 0, 0);
          }
      }
    __builtin_amdgcn_sched_barrier(0);
    keys(a, nx);
    SharedScales sc[1];
    if constexpr (Q8) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) {
        sc[0].k[bi] = *(const floatx4*)&scale[0][16 * bi + 4 * kk];
        sc[0].v[bi] = *(const floatx4*)&scale[1][16 * bi + 4 * kk];
      }
    }
    const int rel = 32 * cur.blk - x.base;                   // the block's first key as a node of the tree
    const auto hidden = [&](int nc, int, int bi, int j) { return !(tree_sight(above[nc], rel + 16 * bi + 4 * kk, cur.keys[bi] - 4 * kk) >> j & 1); };
    u32x4 p[NC][1];
    shared_softmax<NC, 1, VE, Q8>(s, sc, MASKED, hidden, a.scale_log2, c.ref, c.sub, c.l, c.o, p);
    shared_values<NC, 1, VE, MASKED>([&](int, int e) { return shared_value_operand<Q8>(vbuf, e); }, rel + 32 > 0, p, c.o);
    __builtin_amdgcn_sched_barrier(0);
    values(a, nx);
    cur = nx;
  }
  // above: the nodes that the lane's columns see, as bits.  The blocks that every column sees whole come first.
  __device__ __forceinline__ void run(const TreeArgs& a, const TreePiece& x, SharedColumns<D, NC>& c, const unsigned long long (&above)[NC], float (*scale)[32],
                                      const uint16_t (*hi)[D + 8], const uint16_t (*lo)[D + 8], int col0) {
    while (cur.keys[0] == 16 && cur.keys[1] == 16 && 32 * cur.blk + 32 <= x.base) step<false>(a, x, c, above, scale, hi, lo, col0);
    while (cur.blk < end) step<true>(a, x, c, above, scale, hi, lo, col0);
  }
};

template <int D, int NC, int WR>
struct TreeLds {
  SharedFewLds<D, NC, WR, TREE_WAVES> few;
  unsigned long long above[PC_TREE_NODES];
  int sums[TREE_WAVES];    // of the lengths' scan
  int begin[2];
};

// Query rows -> LDS as two bf16 parts, rotated at their nodes' positions (rows behind the last one: zeros).  D / 16 threads a
// row, 8 values of each half.
template <int D, int N>
__device__ __forceinline__ void tree_query_rows(const TreeArgs& a, const TreePiece& x, const unsigned long long* above, uint16_t (*hi)[D + 8],
                                                uint16_t (*lo)[D + 8]) {
  constexpr int HALF = D / 2, TPR = HALF / 8, PASS = TREE_THREADS / TPR, PASSES = (N + PASS - 1) / PASS;
  const int i0 = threadIdx.x % TPR * 8;
  u32x4 lo_half[PASSES], hi_half[PASSES];
#pragma unroll
  for (int n = 0; n < PASSES; ++n) {
    const int r = x.row0 + min((int)threadIdx.x / TPR + n * PASS, x.n_here - 1);
    const int t = pc_div(r, a.group_div), h = r - t * a.group;
    const uint16_t* src = a.c.q + x.b * a.c.batch_stride + t * a.c.row_stride + (x.g * a.group + h) * D + i0;
    lo_half[n] = *(const u32x4*)src; hi_half[n] = *(const u32x4*)(src + HALF);
  }
  double theta[8];
  double first = 0.0;
  if (a.c.pos) {
    first = (double)a.c.pos0 + a.c.pos[x.b];
#pragma unroll
    for (int e = 0; e < 8; ++e) theta[e] = pc_rope_theta(a.rope, i0 + e);
  }
#pragma unroll
  for (int n = 0; n < PASSES; ++n) {
    const int r = threadIdx.x / TPR + n * PASS;
    if (r >= N) break;
    u32x4 u = lo_half[n], v = hi_half[n], ul = {0, 0, 0, 0}, vl = {0, 0, 0, 0};
    if (r >= x.n_here) u = v = u32x4{0, 0, 0, 0};
    if (a.c.pos) {
      const int t = pc_div(x.row0 + min(r, x.n_here - 1), a.group_div);
      const double at = first + (__popcll(above[t]) - 1);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float y1[2], y2[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float x1 = b ? bf16_hi_to_f32(u[w]) : bf16_lo_to_f32(u[w]), x2 = b ? bf16_hi_to_f32(v[w]) : bf16_lo_to_f32(v[w]);
          float sn, cs;
          pc_sincos_f32(at * theta[2 * w + b], sn, cs);
          y1[b] = x1 * cs - x2 * sn; y2[b] = x2 * cs + x1 * sn;
        }
        u[w] = pack_bf16x2(y1[0], y1[1]); v[w] = pack_bf16x2(y2[0], y2[1]);
        ul[w] = pack_bf16x2(y1[0] - bf16_lo_to_f32(u[w]), y1[1] - bf16_hi_to_f32(u[w]));
        vl[w] = pack_bf16x2(y2[0] - bf16_lo_to_f32(v[w]), y2[1] - bf16_hi_to_f32(v[w]));
      }
    }
    *(u32x4*)&hi[r][i0] = u; *(u32x4*)&hi[r][i0 + HALF] = v;
    *(u32x4*)&lo[r][i0] = ul; *(u32x4*)&lo[r][i0 + HALF] = vl;
  }
}

// Blocks blk0 .. of a sequence for its query rows -> a partial at `place`
template <int D, int NC, int WR, bool Q8>
__device__ __forceinline__ void tree_piece(const TreeArgs& a, const TreePiece& x, int blk0, int n_blk, int place, TreeLds<D, NC, WR>& sm) {
  constexpr int WK = TREE_WAVES / WR;
  const int lane = threadIdx.x % PC_WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PC_WAVE);
  const int wk = wave / WR, col0 = 16 * NC * (wave % WR);
  const unsigned long long mine = pc_tree_above(a.c.parent, x.b, a.c.n, lane);
  __syncthreads();                                           // (the piece before this one is done with LDS)
  if (wave == 0) sm.above[lane] = mine;
  __syncthreads();
  TreeWalk<D, NC, WK, Q8> walk;
  walk.begin(a, x, blk0, n_blk, wk);
  tree_query_rows<D, 16 * NC * WR>(a, x, sm.above, sm.few.q[0], sm.few.q[1]);
  __syncthreads();
  SharedColumns<D, NC> c;
  c.clear();
  shared_query_operands<D, NC, Q8>(c, sm.few.q[0], sm.few.q[1], col0);
  unsigned long long above[NC];
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) above[nc] = sm.above[pc_div(x.row0 + min(col0 + 16 * nc + lane % 16, x.n_here - 1), a.group_div)];
  walk.run(a, x, c, above, sm.few.scale[wave], sm.few.q[0], sm.few.q[1], col0);
  __syncthreads();                                           // (the query rows are written over)
  shared_columns_out<D, NC>(c, sm.few, wk, col0, x.n_here);
  __syncthreads();
  for (int idx = threadIdx.x; idx < x.n_here * (D / 4); idx += TREE_THREADS) {
    const int r = idx / (D / 4), d4 = idx % (D / 4) * 4;
    SharedRowSum sum;
    sum.clear();
#pragma unroll
    for (int w = 0; w < WK; ++w) sum.add(sm.few.m[w][r], sm.few.l[w][r], *(const floatx4*)&sm.few.o[w][r][d4]);
    const long long row = ((long long)place * a.c.n_kv_heads + x.g) * (a.c.n * a.group) + x.row0 + r;
    *(floatx4*)(a.part_o + row * D + d4) = sum.mean();
    if (d4 == 0) a.part_lse[row] = sum.lse();
  }
}

// A share's first block: of sequence begin[0], at its block begin[1].  Every thread counts the blocks of a run of sequences.
template <typename Lds>
__device__ __forceinline__ int tree_scan(const TreeArgs& a, int share, Lds& sm) {
  const int lane = threadIdx.x % PC_WAVE, wave = threadIdx.x / PC_WAVE;
  const int per = (a.c.batch + TREE_THREADS - 1) / TREE_THREADS, b0 = min((int)threadIdx.x * per, a.c.batch), b1 = min(b0 + per, a.c.batch);
  int mine = 0;
  for (int b = b0; b < b1; ++b) mine += tree_blocks(a.c, b);
  const int incl = pc_wave_scan(mine);
  if (lane == PC_WAVE - 1) sm.sums[wave] = incl;
  __syncthreads();
  int before = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < TREE_WAVES; ++w) {
    if (w < wave) before += sm.sums[w];
    total += sm.sums[w];
  }
  // shares as equal as possible, of 8 blocks at least
  const int n_eff = max(1, min(a.n_shares, total / 8));
  if (share >= n_eff) return 0;
  const int each = total / n_eff, extra = total - each * n_eff;
  const int lo = share * each + min(share, extra), n = each + (share < extra);
  if (n == 0) return 0;
  if (lo >= before && lo < before + mine) {
    int off = lo - before, b = b0;
    for (; b < b1; ++b) {
      const int nb = tree_blocks(a.c, b);
      if (off < nb) break;
      off -= nb;
    }
    sm.begin[0] = b; sm.begin[1] = off;
  }
  __syncthreads();
  return n;
}

template <int D, int NC, int WR, bool Q8>
__global__ __launch_bounds__(TREE_THREADS, 2) void tree_rows_kernel(TreeArgs a) {
  extern __shared__ __align__(16) unsigned char lds[];
  TreeLds<D, NC, WR>& sm = *(TreeLds<D, NC, WR>*)lds;
  constexpr int ROWS = 16 * NC * WR;
  // an XCD (number mod 8) has an eighth of (share, head, tile), the tiles behind each other: its L2 serves the keys to them
  const int at = (int)(blockIdx.x % 8) * a.per_xcd + (int)(blockIdx.x / 8);
  if (at >= a.n_shares * a.c.n_kv_heads * a.n_tiles) return;
  const int sg = pc_div(at, a.tiles_div), tile = at - sg * a.n_tiles;
  const int share = pc_div(sg, a.heads_div), g = sg - share * a.c.n_kv_heads;
  int left = tree_scan(a, share, sm);
  if (left == 0) return;
  int b = __builtin_amdgcn_readfirstlane(sm.begin[0]), off = __builtin_amdgcn_readfirstlane(sm.begin[1]);
  for (; left > 0 && b < a.c.batch; ++b, off = 0) {
    const int nb = __builtin_amdgcn_readfirstlane(tree_blocks(a.c, b));
    const int take = min(left, nb - off);
    if (take <= 0) continue;
    left -= take;
    if (g == 0 && tile == 0 && threadIdx.x == 0) {
      if (off == 0) a.span[b].x = share;
      if (off + take == nb) a.span[b].y = share;
    }
    TreePiece x;
    x.b = b; x.g = g; x.row0 = tile * ROWS;
    const int n_rows = __builtin_amdgcn_readfirstlane(pc_tree_rows(a.c.n_rows, b, a.c.n));
    x.n_here = min(ROWS, n_rows * a.group - x.row0);
    if (x.n_here <= 0) continue;
    x.len = __builtin_amdgcn_readfirstlane(tree_len(a.c, b)); x.base = __builtin_amdgcn_readfirstlane(max(a.c.len[b], 0)) - n_rows;
    tree_piece<D, NC, WR, Q8>(a, x, off, take, share + b, sm);
  }
}

// The partials of a row, joined: D / 4 threads take 4 values each
template <int D>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a, long long n_out, PcDiv heads_div, PcDiv nodes_div) {
  constexpr int TPR = D / 4, U = 4;
  const int d4 = threadIdx.x % TPR * 4;
  const long long row = (long long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;          // (b, t, h)
  if (row >= n_out) return;
  const int bt = pc_div((int)row, heads_div), h = (int)row - bt * a.c.n_q_heads;
  const int b = pc_div(bt, nodes_div), t = bt - b * a.c.n;
  if (t >= pc_tree_rows(a.c.n_rows, b, a.c.n)) return;
  const int g = pc_div(h, a.group_div), r = t * a.group + h - g * a.group;
  float m = -INFINITY, den = 0.f;
  floatx4 num = {0.f, 0.f, 0.f, 0.f};
  if (tree_blocks(a.c, b) > 0) {
    const int2 span = a.span[b];
    for (int s0 = span.x; s0 <= span.y; s0 += U) {
      float l[U];
      floatx4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long at = ((long long)(min(s0 + u, span.y) + b) * a.c.n_kv_heads + g) * (a.c.n * a.group) + r;
        l[u] = a.part_lse[at];
        x[u] = *(const floatx4*)(a.part_o + at * D + d4);
      }
      float top = m;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (s0 + u > span.y) l[u] = -INFINITY;
        top = fmaxf(top, l[u]);
      }
      const float ref = top == -INFINITY ? 0.f : top;
      const float w0 = expf(m - ref);
      m = top; den *= w0;
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] *= w0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = expf(l[u] - ref);
        den += w;
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] += l[u] == -INFINITY ? 0.f : w * x[u][e];
      }
    }
  }
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = den == 0.f ? 0.f : num[e] / den;
  *(uint2*)(a.c.out + row * D + d4) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
  if (a.c.lse && d4 == 0) a.c.lse[((long long)b * a.c.n_q_heads + h) * a.c.n + t] = den == 0.f ? -INFINITY : m + logf(den);
}

// ---- host
PcTreePlan pc_tree_plan(const PcTreeCall& c) {
  PcTreePlan p;
  const int rows = c.n * (c.n_q_heads / c.n_kv_heads);
  p.rows = rows <= 16 ? 16 : (rows <= 32 ? 32 : 64);
  p.tiles = (rows + p.rows - 1) / p.rows;
  const long long blocks = (long long)c.batch * ((((long long)c.pages.max_pages << c.pages.shift) + 31) / 32);
  long long shares = 512 / ((long long)c.n_kv_heads * p.tiles);
  if (shares > blocks / 8) shares = blocks / 8;
  p.shares = shares < 1 ? 1 : (int)shares;
  return p;
}
static long long workgroups(const PcTreeCall& c, const PcTreePlan& p) { return (long long)p.shares * c.n_kv_heads * p.tiles; }
bool pc_tree_fits(const PcTreeCall& c, const PcTreePlan& p) {
  const long long blocks = (((long long)c.pages.max_pages << c.pages.shift) + 31) / 32;
  return workgroups(c, p) < (1LL << 32) / TREE_THREADS - 8 && c.batch * blocks < (1LL << 31);
}
static size_t part_rows(const PcTreeCall& c, const PcTreePlan& p) { return (size_t)(p.shares + c.batch) * c.n * c.n_q_heads; }
size_t pc_tree_ws_bytes(const PcTreeCall& c, const PcTreePlan& p) {
  const size_t rows = part_rows(c, p);
  return pc_align_up(rows * c.head_dim * 4, 256) + pc_align_up(rows * 4, 256) + pc_align_up((size_t)c.batch * sizeof(int2), 256);
}

template <int D, int NC, int WR, bool Q8>
static int launch_rows(const TreeArgs& a, hipStream_t st) {
  static std::atomic<uint64_t> raised{0};
  constexpr int LDS = sizeof(TreeLds<D, NC, WR>);
  const int rc = pc_raise_dynamic_lds((const void*)tree_rows_kernel<D, NC, WR, Q8>, LDS, raised);
  if (rc != PC_OK) return rc;
  PcProfScope prof(PC_KERNEL_TREE_ATTN, st);
  hipLaunchKernelGGL((tree_rows_kernel<D, NC, WR, Q8>), dim3((unsigned)(8 * a.per_xcd)), dim3(TREE_THREADS), LDS, st, a);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
template <int D, bool Q8>
static int launch_body(const TreeArgs& a, const PcTreePlan& p, hipStream_t st) {
  if (p.rows == 16) return launch_rows<D, 1, 1, Q8>(a, st);
  return p.rows == 32 ? launch_rows<D, 2, 1, Q8>(a, st) : launch_rows<D, 2, 2, Q8>(a, st);
}
template <int D>
static int launch_all(const PcTreeCall& c, const PcTreePlan& p, void* ws, hipStream_t st) {
  TreeArgs a;
  a.c = c;
  a.rope = pc_rope_factors(c.pos ? c.rope_base : 2.0f, c.head_dim);
  a.group = c.n_q_heads / c.n_kv_heads; a.n_tiles = p.tiles; a.n_shares = p.shares;
  a.per_xcd = (int)((workgroups(c, p) + 7) / 8);
  a.group_div = pc_div_by(a.group); a.tiles_div = pc_div_by(p.tiles); a.heads_div = pc_div_by(c.n_kv_heads);
  a.scale_log2 = c.scale * SHARED_LOG2E;
  const size_t rows = part_rows(c, p);
  a.part_o = (float*)ws;
  a.part_lse = (float*)((char*)ws + pc_align_up(rows * D * 4, 256));
  a.span = (int2*)((char*)a.part_lse + pc_align_up(rows * 4, 256));
  const int rc = c.pages.k_scale ? launch_body<D, true>(a, p, st) : launch_body<D, false>(a, p, st);
  if (rc != PC_OK) return rc;
  const long long n_out = (long long)c.batch * c.n * c.n_q_heads;
  PcProfScope prof(PC_KERNEL_TREE_MERGE, st);
  hipLaunchKernelGGL(tree_join_kernel<D>, dim3((unsigned)((n_out * (D / 4) + 255) / 256)), dim3(256), 0, st, a, n_out, pc_div_by(c.n_q_heads),
                     pc_div_by(c.n));
  PC_LAUNCH_CHECK();
  return PC_OK;
}
int pc_launch_tree_attn(const PcTreeCall& c, const PcTreePlan& p, void* ws, hipStream_t st) {
  return c.head_dim == 128 ? launch_all<128>(c, p, ws, st) : launch_all<64>(c, p, ws, st);
}
