// Attention of drafted trees over a paged cache.
//
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q . k_j,  over the rows in front of the tree and the
//   node's own ancestors (itself among them).
//
// The rows (node, head of the group) of a sequence and KV head are the columns of S^T = K Q^T.  A node's ancestors are the
// bits of one 64-bit word, which a wavefront finds with six exchanges (a node a lane) and a lane keeps for its columns: the
// mask of a tree costs a shift where a block holds rows of it, and nothing elsewhere.
// Cut: the keys of all sequences, laid end to end in blocks of 32, are cut into equal shares, a workgroup each for a KV head and a
// tile of query rows: so a batch of very unequal lengths keeps every CU busy, whatever the table's width.  A share is a
// piece of one sequence or of several; each piece leaves a partial (o, lse) a row at place share + sequence (both
// only grow along the keys, so a place is taken once), and tree_join_kernel joins a sequence's.  Where there is little for a
// sequence a workgroup takes a whole one, in one launch (pc_tree_plan).
// Bodies: up to 32 rows a wavefront takes a part of the keys, straight into registers; more rows share keys in LDS.
// Bound (4 D R flops against 4 D bytes a key for R query rows a KV head, 2 D + 8 in 8 bits): memory up to 64 rows, 32 sequences of
// 8300 rows on average, 4 query rows a KV head, 8 KV heads of 128 values 167 us = 6.5 TB/s; 16 sequences of 11500 rows, 64 query
// rows 138 us = 5.5 TB/s; with 128 rows, 8 sequences of 46000 rows in 8 bits some 330 us = 0.59 PFLOP/s, 0.89 with the products of the
// rotated queries' second parts: a block's chain of a barrier, scalar instructions, reads of LDS, products and softmax, of which
// two wavefronts a SIMD hide a part of each other's (what was taken off the chain gained, what was taken off the counts did not).
#include <type_traits>
#include "decode_core.h"
#include "paged.h"
#include "shared_core.h"
#include "serve.h"

#define TREE_WAVES 4
// Blocks that a piece costs beside its own (0 / 4 / 8: 16 trees of 16 nodes 147 / 142 / 142 us, 8 of 32 over 8 bits 482 / 456 / 458)
#define TREE_EXTRA 4
#define TREE_THREADS (TREE_WAVES * PC_WAVE)
#define TREE_GROUPS ((1LL << 32) / TREE_THREADS - 8)       // workgroups of a launch: below 2^32 threads
// the N newest loads of this wavefront may still be on their way
#define TREE_WAIT_LOADS(N) __builtin_amdgcn_s_waitcnt(0x0F70 | ((N) & 15) | (((N) >> 4) << 14))
// ... and a barrier, with LDS reads done.  (A fence would wait for every load that goes to LDS.)
#define TREE_TILE_BARRIER(N)                                                         \
  do {                                                                               \
    asm volatile("" ::: "memory");                                                   \
    __builtin_amdgcn_s_waitcnt(0x0070 | ((N) & 15) | (((N) >> 4) << 14));            \
    __builtin_amdgcn_s_barrier();                                                    \
    asm volatile("" ::: "memory");                                                   \
  } while (0)

struct TreeArgs {
  PcTreeCall c;
  PcRope rope;
  int group, n_tiles, n_shares, n_groups, per_xcd, extra;   // n_shares 0: sequences are not cut; n_groups: shares or sequences, times heads
  PcDiv group_div, tiles_div, heads_div;
  float scale_log2;
  float* part_o;           // [n_shares + B][H_kv][n group][D]
  float* part_lse;         // [n_shares + B][H_kv][n group]
  int2* span;              // [B] first and last share of a sequence
};

// The lane's number again, as a value of its own: what is computed from it is computed here, and not kept in registers from in front
// of a loop on
__device__ __forceinline__ int tree_own(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A sequence: its nodes, its rows with theirs (0: none; they may be more than there are places for)
struct TreeSeq { int rows, len; };
__device__ __forceinline__ TreeSeq tree_seq(const PcTreeCall& c, int b) {
  TreeSeq s;
  s.rows = c.n;
  if (c.n_rows) s.rows = min(max(c.n_rows[b], 0), c.n);
  s.len = max(c.len[b], 0);
  return s;
}
// Rows that are there, and blocks of 32 of them: none where it has no nodes
__device__ __forceinline__ int tree_there(const PcTreeCall& c, const TreeSeq& s) {
  return (int)min((long long)s.len, (long long)c.pages.max_pages << c.pages.shift);
}
__device__ __forceinline__ int tree_blocks(const PcTreeCall& c, const TreeSeq& s) { return s.rows > 0 ? (tree_there(c, s) + 31) / 32 : 0; }

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
  // blocks in front of this one hold 32 rows that are there, in front of the tree (it may begin behind all that there is room for)
  __device__ __forceinline__ int whole() const { return max(min(base, len), 0) / 32; }
};

// A 32-key block: its two halves of 16 keys, each inside a page
struct TreeBlock {
  int blk;
  long long row[2];        // of the pool
  int keys[2];             // that are there
};

// A wavefront's window of the table: where the rows of 64 pages from entry `first` on begin in the pool (negative: no page).  The
// next 64 are waited for where they are asked for: a copy of registers that are still on their way would have every block
// wait for all that the wavefront has asked for.
struct TreeTable {
  long long here;
  int first;
  __device__ __forceinline__ long long entries(const TreeArgs& a, const TreePiece& x, int at) const {
    const int i = min(at + (int)(threadIdx.x % PC_WAVE), a.c.pages.max_pages - 1);
    const int page = a.c.pages.table[(long long)x.b * a.c.pages.max_pages + i];
    const long long row = pc_pool_row(a.c.pages, page, 0, x.g, a.c.n_kv_heads);
    return row < 0 ? -(1LL << 40) : row;
  }
  __device__ __forceinline__ void begin(const TreeArgs& a, const TreePiece& x, int at) {
    first = at;
    here = entries(a, x, at);
  }
  // are all the pages of entries lo .. hi there?
  __device__ __forceinline__ bool all(const TreeArgs& a, const TreePiece& x, int lo, int hi) const {
    bool there = true;
    for (int at = lo; at <= hi; at += PC_WAVE) {
      const long long row = at == lo ? here : entries(a, x, at);
      there &= at + (int)(threadIdx.x % PC_WAVE) > hi || row >= 0;
    }
    return __all(there);
  }
  // the row of the pool where key `key` lies, negative if it is not there; keys are asked for in order
  __device__ __forceinline__ long long row(const TreeArgs& a, const TreePiece& x, int key) {
    const int at = key >> a.c.pages.shift;
    if (at >= first + PC_WAVE) {
      first += PC_WAVE;
      here = entries(a, x, first);
      asm volatile("" : "+v"(here));
    }
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)here, at - first);
    const int hi = __builtin_amdgcn_readlane((int)(here >> 32), at - first);
    return ((long long)hi << 32 | lo) + (key & ((1 << a.c.pages.shift) - 1));
  }
};

template <int D, int NC, bool Q8>
struct TreeWalk {
  static constexpr int KSTEPS = D / 32, VE = D / 16, ELEM = Q8 ? 1 : 2, ROW = D * ELEM;
  static constexpr int KP = Q8 ? D / 64 : KSTEPS;
  typedef uint32_t vpiece __attribute__((ext_vector_type(VE * ELEM / 4)));
  u32x4 kbuf[2][KP];
  vpiece vbuf[8];
  float sbuf;
  TreeBlock cur;
  int whole_end, end;                                        // of the blocks that every column sees whole, of the run
  TreeTable tab;

  __device__ __forceinline__ TreeBlock block(const TreeArgs& a, const TreePiece& x, int blk) {
    TreeBlock t;
    t.blk = blk;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int key = 32 * blk + 16 * h;
      t.row[h] = blk < end && key < x.len ? tab.row(a, x, key) : -1;
      t.keys[h] = t.row[h] < 0 ? 0 : min(16, x.len - key);
      t.row[h] = max(t.row[h], 0LL);
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
      for (int p = 0; p < KP; ++p) kbuf[h][p] = __builtin_amdgcn_raw_buffer_load_b128(r, c16 * ROW + 16 * kk, 64 * p, PC_BUF_NT);
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
        if constexpr (sizeof(vpiece) == 16) vbuf[4 * h + i] = __builtin_amdgcn_raw_buffer_load_b128(r, off, i * ROW, PC_BUF_NT);
        else if constexpr (sizeof(vpiece) == 8) vbuf[4 * h + i] = __builtin_amdgcn_raw_buffer_load_b64(r, off, i * ROW, PC_BUF_NT);
        else vbuf[4 * h + i] = __builtin_amdgcn_raw_buffer_load_b32(r, off, i * ROW, PC_BUF_NT);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // the wavefront's run of the piece's blocks
  __device__ __forceinline__ void begin(const TreeArgs& a, const TreePiece& x, int blk0, int n_blk, int wave) {
    const int first = blk0 + (int)((long long)n_blk * wave / TREE_WAVES);
    end = blk0 + (int)((long long)n_blk * (wave + 1) / TREE_WAVES);
    tab.begin(a, x, (32 * first) >> a.c.pages.shift);
    whole_end = first < end && tab.all(a, x, (32 * first) >> a.c.pages.shift, (min(32 * end, x.len) - 1) >> a.c.pages.shift)
                    ? min(end, x.whole()) : first;
    cur = block(a, x, first);
    keys(a, cur);
    values(a, cur);
  }
  // One block.  MASKED: some of its keys are not there, or rows of the tree; few blocks are, so that the query operands come from
  // LDS there and leave their registers to the masks (in registers throughout, 128 values a row and 32 columns, 89 to 126
  // registers spilled, and every block waited for its own: 16 sequences of 11000 rows, 64 query rows a KV head, 363 us)
  template <bool MASKED>
  __device__ __forceinline__ void step(const TreeArgs& a, const TreePiece& x, SharedColumns<D, NC>& c, const unsigned long long (&above)[NC], float (*scale)[32],
                                       const uint16_t (*hi)[D + 8], const uint16_t (*lo)[D + 8]) {
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
            if constexpr (MASKED) q = *(const bf16x8*)&(h ? lo : hi)[16 * nc + lane % 16][shared_query_at(Q8, ks, kk)];
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
    shared_softmax<NC, 1, VE, Q8, !MASKED>(s, sc, MASKED, hidden, a.scale_log2, c.ref, c.sub, c.l, c.o, p);
    shared_values<NC, 1, VE, MASKED>([&](int, int e) { return shared_value_operand<Q8>(vbuf, e); }, rel + 32 > 0, p, c.o);
    __builtin_amdgcn_sched_barrier(0);
    values(a, nx);
    cur = nx;
  }
  // above: the nodes that the lane's columns see, as bits.  The blocks that every column sees whole come first (none where one of
  // the run's pages is not there).
  __device__ __forceinline__ void run(const TreeArgs& a, const TreePiece& x, SharedColumns<D, NC>& c, const unsigned long long (&above)[NC], float (*scale)[32],
                                      const uint16_t (*hi)[D + 8], const uint16_t (*lo)[D + 8]) {
    while (cur.blk < whole_end) step<false>(a, x, c, above, scale, hi, lo);
    while (cur.blk < end) step<true>(a, x, c, above, scale, hi, lo);
  }
};

struct TreeScanLds { int sums[TREE_WAVES], begin[2]; TreeSeq seq[TREE_THREADS]; };      // of the lengths' scan
template <int D, int NC>
struct TreeLds {
  SharedFewLds<D, NC, 1, TREE_WAVES> few;
  TreeScanLds scan;
};
// The nodes that node t sees, from the lanes' own
__device__ __forceinline__ unsigned long long tree_above_of(unsigned long long mine, int t) {
  const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)mine, t), hi = (uint32_t)__shfl((int)(uint32_t)(mine >> 32), t);
  return (unsigned long long)hi << 32 | lo;
}
// Four pairs of a row turned by their angles, into two bf16 parts of each half
__device__ __forceinline__ void tree_turn(u32x4& u, u32x4& v, u32x4& ul, u32x4& vl, double at, const double (&theta)[8]) {
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
    uint32_t hi, lo;
    split_bf16x2(y1[0], y1[1], hi, lo);
    u[w] = hi; ul[w] = lo;
    split_bf16x2(y2[0], y2[1], hi, lo);
    v[w] = hi; vl[w] = lo;
  }
}

// Query rows -> LDS as two bf16 parts, rotated at their nodes' positions (rows behind the last one: zeros).  D / 16 threads a
// row, 8 values of each half.  mine: what the lane's node sees
template <int D, int N>
__device__ __forceinline__ void tree_query_rows(const TreeArgs& a, const TreePiece& x, unsigned long long mine, uint16_t (*hi)[D + 8],
                                                uint16_t (*lo)[D + 8]) {
  constexpr int HALF = D / 2, TPR = HALF / 8, PASS = TREE_THREADS / TPR, PASSES = (N + PASS - 1) / PASS;
  const int thread = tree_own(threadIdx.x), i0 = thread % TPR * 8;
  u32x4 lo_half[PASSES], hi_half[PASSES];
  int depth[PASSES];
#pragma unroll
  for (int n = 0; n < PASSES; ++n) {
    const int r = x.row0 + min(thread / TPR + n * PASS, x.n_here - 1);
    const int t = pc_div(r, a.group_div), h = r - t * a.group;
    const uint16_t* src = a.c.q + x.b * a.c.batch_stride + t * a.c.row_stride + (x.g * a.group + h) * D + i0;
    lo_half[n] = *(const u32x4*)src; hi_half[n] = *(const u32x4*)(src + HALF);
    depth[n] = __popcll(tree_above_of(mine, t)) - 1;
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
    const int r = thread / TPR + n * PASS;
    if (r >= N) break;
    u32x4 u = lo_half[n], v = hi_half[n], ul = {0, 0, 0, 0}, vl = {0, 0, 0, 0};
    if (r >= x.n_here) u = v = u32x4{0, 0, 0, 0};
    if (a.c.pos) tree_turn(u, v, ul, vl, first + depth[n], theta);
    *(u32x4*)&hi[r][i0] = u; *(u32x4*)&hi[r][i0 + HALF] = v;
    *(u32x4*)&lo[r][i0] = ul; *(u32x4*)&lo[r][i0 + HALF] = vl;
  }
}

// Place of a query row's result: [B, n, H_q]; and of its logsumexp: [B, H_q, n]
struct TreeOut { long long row, lse; };
__device__ __forceinline__ TreeOut tree_out(const TreeArgs& a, const TreePiece& x, int r) {
  const int t = pc_div(x.row0 + r, a.group_div), h = x.g * a.group + x.row0 + r - t * a.group;
  return {((long long)x.b * a.c.n + t) * a.c.n_q_heads + h, ((long long)x.b * a.c.n_q_heads + h) * a.c.n + t};
}
__device__ __forceinline__ long long tree_part_row(const TreeArgs& a, const TreePiece& x, int place, int r) {
  return ((long long)place * a.c.n_kv_heads + x.g) * (a.c.n * a.group) + x.row0 + r;
}

// Blocks blk0 .. of a sequence for its 16 NC query rows -> a partial at `place`; a wavefront has a part of the blocks
template <int D, int NC, bool Q8>
__device__ __forceinline__ void tree_piece(const TreeArgs& a, const TreePiece& x, int blk0, int n_blk, int place, TreeLds<D, NC>& sm) {
  const int lane = tree_own(threadIdx.x % PC_WAVE), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PC_WAVE);
  TreeWalk<D, NC, Q8> walk;
  walk.begin(a, x, blk0, n_blk, wave);
  const unsigned long long mine = pc_tree_above(a.c.parent, x.b, a.c.n, lane);
  PC_LDS_BARRIER();                                          // (the piece before this one is done with LDS)
  tree_query_rows<D, 16 * NC>(a, x, mine, sm.few.q[0], sm.few.q[1]);
  PC_LDS_BARRIER();
  SharedColumns<D, NC> c;
  c.clear();
  shared_query_operands<D, NC, Q8>(c, sm.few.q[0], sm.few.q[1], 0);
  unsigned long long above[NC];
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) above[nc] = tree_above_of(mine, pc_div(x.row0 + min(16 * nc + lane % 16, x.n_here - 1), a.group_div));
  walk.run(a, x, c, above, sm.few.scale[wave], sm.few.q[0], sm.few.q[1]);
  PC_LDS_BARRIER();                                          // (the query rows are written over)
  shared_columns_out<D, NC>(c, sm.few, wave, 0, x.n_here);
  PC_LDS_BARRIER();
  for (int idx = threadIdx.x; idx < x.n_here * (D / 4); idx += TREE_THREADS) {
    const int r = idx / (D / 4), d4 = idx % (D / 4) * 4;
    SharedRowSum sum;
    sum.clear();
#pragma unroll
    for (int w = 0; w < TREE_WAVES; ++w) sum.add(sm.few.m[w][r], sm.few.l[w][r], *(const floatx4*)&sm.few.o[w][r][d4]);
    if (a.n_shares == 0) {                                   // the whole sequence's
      const TreeOut to = tree_out(a, x, r);
      const floatx4 y = sum.mean();
      *(uint2*)(a.c.out + to.row * D + d4) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
      if (a.c.lse && d4 == 0) a.c.lse[to.lse] = sum.lse();
      continue;
    }
    const long long row = tree_part_row(a, x, place, r);
    *(floatx4*)(a.part_o + row * D + d4) = sum.mean();
    if (d4 == 0) a.part_lse[row] = sum.lse();
  }
}

// ------------------------------------------------------------------------------------------ many rows
// Blocks of 32 keys on their way from memory straight into LDS, 32 to 56 KB of them, each read there by all four wavefronts, which
// have 16 NC query rows each.  8 bits: the workgroup widens a block once, a block ahead of the products (each wavefront for itself,
// with 48 conversions and 16 permutations more a block: 128 rows 113 us instead of 110, rows of 64 values 104 instead of 102, 64 rows of
// 128 values 150 instead of 154).  A row of 16 bits is PPR
// pieces of 16 bytes, piece p of row r in place p ^ swizzle(r), and a load instruction brings whole rows.  With 128 values the operands of
// the keys (16 rows at once) come without bank conflicts, those of the values, transposed on the way (eight rows of 32 bytes at once), two
// to a bank; with 64 values the other way round.  Conflicts are a third of the LDS's busy cycles with 128 values.
// (Keys straight into registers, two wavefronts to a key, keep half as many bytes on their way: 16 sequences of 11000 rows, 64
// query rows a KV head, 188 us instead of 140.  32 rows a wavefront, two blocks at a time: 1 to 10 us slower.)
template <int D, bool Q8>
struct TreeTiles {
  static constexpr int RB = D * (Q8 ? 1 : 2), WB = D * 2, PPR = WB / 16;        // bytes of a row as it comes, as it is used; pieces
  static constexpr int STAGES = Q8 ? (D == 128 ? 5 : 8) : (D == 128 ? 4 : 8);
  static constexpr int LAG = Q8 ? STAGES : STAGES - 1;              // blocks issued ahead of the one at hand
  static constexpr int LOADS = RB / 64 + (Q8 ? 1 : 0);              // of a wavefront, a block
  struct Narrow {
    uint8_t rows[STAGES][2][32 * RB];                               // [keys, values]
    float scale[STAGES][2][32];
  };
  struct Wide {
    uint8_t rows[2][2][32 * WB];
    float scale[2][2][32];
  };
  struct Nothing {};
  struct Lds {
    Narrow in;
    typename std::conditional<Q8, Wide, Nothing>::type wide;
    unsigned long long above[PC_TREE_NODES];
    TreeScanLds scan;
  };
  __device__ __forceinline__ static int swizzle(int row) { return row & (PPR - 1); }
};

// PARTS: bf16 parts of a query (1: they arrive rotated)
template <int D, int NC, bool Q8, int PARTS>
__device__ __forceinline__ void tree_tile_piece(const TreeArgs& a, const TreePiece& x, int blk0, int n_blk, int place,
                                                typename TreeTiles<D, Q8>::Lds& sm) {
  typedef TreeTiles<D, Q8> Tiles;
  constexpr int KSTEPS = D / 32, VE = D / 16, RB = Tiles::RB, WB = Tiles::WB, STAGES = Tiles::STAGES, LAG = Tiles::LAG;
  typedef __attribute__((address_space(3))) void* lptr_t;
  const int lane = tree_own(threadIdx.x % PC_WAVE), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PC_WAVE);
  const int kk = lane / 16, c16 = lane % 16;
  const int end = blk0 + n_blk;

  TreeTable tab;
  tab.begin(a, x, (32 * blk0) >> a.c.pages.shift);
  const bool all_there = tab.all(a, x, (32 * blk0) >> a.c.pages.shift, (min(32 * end, x.len) - 1) >> a.c.pages.shift);

  // ---- the wavefront's query rows, as they lie in the operands: both values of a pair are the same lane's
  SharedColumns<D, NC> c;
  c.clear();
  auto node_of = [&](int nc, int c16) { return pc_div(x.row0 + min(16 * (NC * wave + nc) + c16, x.n_here - 1), a.group_div); };
  u32x4 q[NC][KSTEPS];
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    const int r = x.row0 + min(16 * (NC * wave + nc) + c16, x.n_here - 1), t = node_of(nc, c16);
    const uint16_t* src = a.c.q + x.b * a.c.batch_stride + t * a.c.row_stride + (x.g * a.group + r - t * a.group) * D + 8 * kk;
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) q[nc][ks] = *(const u32x4*)(src + 32 * ks);
  }
  const int first_pos = a.c.pos ? a.c.pos[x.b] : 0;
  const unsigned long long mine = pc_tree_above(a.c.parent, x.b, a.c.n, lane);
  // Waited for in front of the loads to LDS: behind those the compiler, which does not count them through the loop, waits for too many
  asm volatile("" : "+v"(tab.here));
#pragma unroll
  for (int nc = 0; nc < NC; ++nc)
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) asm volatile("" : "+v"(q[nc][ks]));

  // ---- the blocks' loads: wavefront w brings half w / 2 of a block, rows 8 w .. of keys and values, or, of rows shorter than 128 bytes, all 16
  // of the keys or values; and 16 scales of the keys or values.  Rows that are not there are out of the descriptor: zeros.
  const int my_half = wave / 2, row0 = RB >= 128 ? 8 * wave : 16 * my_half;      // (of the block)
  const int at_row = row0 % 16 + lane / (RB / 16);                   // of the half
  const int off = at_row * RB + 16 * (Q8 ? lane % (RB / 16) : lane % (RB / 16) ^ Tiles::swizzle(at_row));
  int to = 0, from = 0;                                              // the next block's stage; the one at hand's, 8 bits: that one's to widen
  uint32_t there = 0;                                                // two bits a block, where pages are missing: are the halves' there
  auto issue = [&](int blk, bool known) __attribute__((always_inline)) {          // known: that all pages are there
    const int key = 32 * blk + 16 * my_half;
    int keys = blk < end ? min(x.len - key, 16) : 0;
    long long at = 0;
    if (known || all_there) {                                        // (a wavefront needs to know of its half alone)
      if (keys > 0) at = tab.row(a, x, key);
    } else {
      long long row[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) row[h] = blk < end && 32 * blk + 16 * h < x.len ? tab.row(a, x, 32 * blk + 16 * h) : -1;
      there = there << 2 | (row[0] >= 0 ? 1u : 0u) | (row[1] >= 0 ? 2u : 0u);
      at = my_half ? row[1] : row[0];
      if (at < 0) at = keys = 0;
    }
    keys = max(keys, 0);
    const int stage = to;
    to = to + 1 == STAGES ? 0 : to + 1;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      if (RB < 128 && kv != wave % 2) continue;
      const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)(kv ? a.c.pages.v : a.c.pages.k) + at * RB), 0, keys * RB, 0x00020000);
#pragma unroll
      for (int i = 0; i < (RB == 256 ? 2 : 1); ++i)                  // (rows 4 further on: another bit of the swizzle)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lptr_t)(sm.in.rows[stage][kv] + (row0 + 4 * i) * RB), 16, off ^ (64 * i), 4 * i * RB, 0, NC == 1 ? PC_BUF_NT : 0);
    }
    if constexpr (Q8) {
      const float* scales = wave % 2 ? a.c.pages.v_scale : a.c.pages.k_scale;
      const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(scales + at), 0, keys * 4, 0x00020000);
      if (lane < 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lptr_t)(sm.in.scale[stage][wave % 2] + 16 * my_half), 4, lane * 4, 0, 0, 0);
    }
  };
  __builtin_amdgcn_sched_barrier(0);
  __syncthreads();                                                   // (the piece before this one is done with LDS)
  if (wave == 0) sm.above[lane] = mine;
#pragma unroll 1
  for (int i = 0; i < LAG; ++i) issue(blk0 + i, false);
  __builtin_amdgcn_sched_barrier(0);

  // ---- meanwhile the rotation
  {
    const double first = (double)a.c.pos0 + first_pos;
#pragma unroll
    for (int ks = 0; ks < KSTEPS / 2; ++ks) {
      double theta[8];
      if constexpr (PARTS == 2) {
#pragma unroll
        for (int e = 0; e < 8; ++e) theta[e] = pc_rope_theta(a.rope, 32 * ks + 8 * kk + e);
      }
#pragma unroll
      for (int nc = 0; nc < NC; ++nc) {
        u32x4 u = q[nc][ks], v = q[nc][ks + KSTEPS / 2];
        if constexpr (PARTS == 2) {
          u32x4 ul, vl;
          tree_turn(u, v, ul, vl, first + (__popcll(tree_above_of(mine, node_of(nc, c16))) - 1), theta);
          c.q[1][nc][ks] = *(bf16x8*)&ul; c.q[1][nc][ks + KSTEPS / 2] = *(bf16x8*)&vl;
        }
        c.q[0][nc][ks] = *(bf16x8*)&u; c.q[0][nc][ks + KSTEPS / 2] = *(bf16x8*)&v;
      }
    }
  }

  const int k_at = c16 * WB + 16 * (kk ^ Tiles::swizzle(c16));
  // reads that transpose: 16 lanes point at 4 rows of 16 values, 8 bytes a lane, and get a value's 4 rows: operand e is values 16 e + d
  const int v_at = (4 * kk + c16 / 4) * WB + 16 * (c16 % 4 / 2 ^ Tiles::swizzle(4 * kk + c16 / 4)) + 8 * (c16 % 2);
  // 8 bits: a thread's 16 codes of the keys, of the values (rows of 64 values: of either), which it widens
  constexpr int CODES = Q8 ? D / 64 : 1;
  const int w_row = threadIdx.x % (2 * D) / (D / 16), w_piece = threadIdx.x % (D / 16), w_side = D == 64 ? threadIdx.x / 128 : 0;
  const int w_at = w_row * WB + 16 * (2 * w_piece ^ Tiles::swizzle(w_row));
  u32x4 codes[CODES];
  float w_scale = 0.f;
  auto take = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < CODES; ++i) codes[i] = *(const u32x4*)(sm.in.rows[from][w_side + i] + w_row * RB + 16 * w_piece);
    w_scale = sm.in.scale[from][threadIdx.x / 32 % 2][threadIdx.x % 32];
    from = from + 1 == STAGES ? 0 : from + 1;
  };
  auto widen = [&](int to_half) __attribute__((always_inline)) {
    if constexpr (Q8) {
#pragma unroll
      for (int i = 0; i < CODES; ++i) {
        uint8_t* at = sm.wide.rows[to_half][w_side + i];
        *(u32x4*)(at + w_at) = u32x4{shared_widen(codes[i][0], false), shared_widen(codes[i][0], true), shared_widen(codes[i][1], false), shared_widen(codes[i][1], true)};
        *(u32x4*)(at + (w_at ^ 16)) = u32x4{shared_widen(codes[i][2], false), shared_widen(codes[i][2], true), shared_widen(codes[i][3], false), shared_widen(codes[i][3], true)};
      }
      if (threadIdx.x < 64) sm.wide.scale[to_half][threadIdx.x / 32][threadIdx.x % 32] = w_scale;
    }
  };
  int half = 0;                                                      // of the widened blocks, the one at hand
  // A wavefront without rows brings its part of the blocks alone (16 sequences of 8192 rows, 132 rows 155 -> 140 us, 72 rows 100 -> 92;
  // 8 bits, where it widens its part, too: 132 rows 175 -> 182)
  const bool idle = !Q8 && 16 * NC * wave >= x.n_here;
  auto block = [&](auto masked_tag, int blk, const bool (&in)[2]) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked_tag)::value;
    const uint8_t *ks_rows, *vs_rows;
    const float* scales = nullptr;
    if constexpr (Q8) {
      ks_rows = sm.wide.rows[half][0]; vs_rows = sm.wide.rows[half][1]; scales = sm.wide.scale[half][0] + 4 * kk;
      take();                                                        // (the next one's)
    } else {
      ks_rows = sm.in.rows[from][0]; vs_rows = sm.in.rows[from][1];
      from = from + 1 == STAGES ? 0 : from + 1;
    }
    if (idle) {
      issue(blk + LAG, !MASKED);
      return;
    }
    u32x4 ka[2][2];                                                  // a step's and the next one's operands, which are on their way
    auto key_operands = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) ka[ks % 2][bi] = *(const u32x4*)(ks_rows + (k_at ^ (64 * ks)) + 16 * bi * WB);
    };
    key_operands(0);
    SharedScales sc[1];                                              // on their way in front of the products that they wait behind
    if constexpr (Q8) {
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) sc[0].k[bi] = *(const floatx4*)(scales + 16 * bi);
    }
    issue(blk + LAG, !MASKED);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);                                   // the first product goes first (64 rows 144 -> 142 us, 128 over 8 bits 350 -> 342)
    floatx4 s[NC][1][2];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc)
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) s[nc][0][bi] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
      if (ks + 1 < KSTEPS) key_operands(ks + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int h = PARTS - 1; h >= 0; --h)
#pragma unroll
        for (int bi = 0; bi < 2; ++bi)
#pragma unroll
          for (int nc = 0; nc < NC; ++nc)
            s[nc][0][bi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(bf16x8*)&ka[ks % 2][bi], c.q[h][nc][ks], s[nc][0][bi], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (Q8) {
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) sc[0].v[bi] = *(const floatx4*)(scales + 32 + 16 * bi);
      widen(half ^ 1);
    }
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);                               // (every operand in flight at once has no registers)
    u32x4 va4[4];                                                    // four operands of V^T
    auto value_operands = [&](int e0) __attribute__((always_inline)) {
      // (the builtin would be taken to read what is on its way to LDS, and wait for all of it)
      const uint32_t at = (uint32_t)(uintptr_t)(lptr_t)(vs_rows + 0);
      const uint32_t a0 = at + (v_at ^ (32 * e0)), a1 = at + (v_at ^ (32 * (e0 + 1))), a2 = at + (v_at ^ (32 * (e0 + 2))), a3 = at + (v_at ^ (32 * (e0 + 3)));
      u32x2 r[8];
      asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
                   "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
                   "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
                   "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\ts_waitcnt lgkmcnt(0)"
                   : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
                   : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(16 * WB) : "memory");
#pragma unroll
      for (int e = 0; e < 4; ++e) va4[e] = u32x4{r[2 * e][0], r[2 * e][1], r[2 * e + 1][0], r[2 * e + 1][1]};
    };
    const int rel = 32 * blk - x.base;
    unsigned long long above[NC];
    int own_kk = 0;
    if constexpr (MASKED) {
      const int own = tree_own(lane);
      own_kk = own / 16;
#pragma unroll
      for (int nc = 0; nc < NC; ++nc) above[nc] = sm.above[node_of(nc, own % 16)];
    }
    const auto hidden = [&](int nc, int, int bi, int j) {
      const int keys = in[bi] ? x.len - 32 * blk - 16 * bi : 0;
      return !(tree_sight(above[nc], rel + 16 * bi + 4 * own_kk, min(keys, 16) - 4 * own_kk) >> j & 1);
    };
    u32x4 p[NC][1];
    shared_softmax<NC, 1, VE, Q8, !MASKED>(s, sc, MASKED, hidden, a.scale_log2, c.ref, c.sub, c.l, c.o, p);
    __builtin_amdgcn_sched_barrier(0);
    uint32_t not_finite = 0;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      if (e % 4 == 0) value_operands(e);
      u32x4 va = va4[e % 4];
      if constexpr (MASKED) {                                        // 0 times infinity or NaN is NaN: out of the operand
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t bad = ((va[i] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((va[i] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
          va[i] &= ~bad;
          not_finite |= bad;
        }
      }
#pragma unroll
      for (int nc = 0; nc < NC; ++nc)
        c.o[nc][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)&va, *(const bf16x8*)&p[nc][0], c.o[nc][e], 0, 0, 0);
    }
    if constexpr (MASKED) {
      if (__any(not_finite != 0)) {                                  // .. and added to the columns that see the key, value by value
        const int own_kk = tree_own(lane) / 16;
        uint32_t seen[NC];                                           // keys of probability above 0, of the lane's column
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
          uint32_t mine_seen = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            mine_seen |= ((p[nc][0][i] & 0x7fffu ? 1u : 0u) | (p[nc][0][i] & 0x7fff0000u ? 2u : 0u)) << (i < 2 ? 4 * own_kk + 2 * i : 12 + 4 * own_kk + 2 * i);
          mine_seen |= (uint32_t)__shfl_xor((int)mine_seen, 16);
          seen[nc] = mine_seen | (uint32_t)__shfl_xor((int)mine_seen, 32);
        }
#pragma unroll 1
        for (int key = 0; key < 32; ++key) {
#pragma unroll
          for (int e = 0; e < VE; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int byte = 2 * (16 * e + 4 * tree_own(own_kk) + i);
              const float v = bf16_bits_to_f32(*(const uint16_t*)(vs_rows + key * WB + 16 * (byte / 16 ^ Tiles::swizzle(key)) + byte % 16));
              const bool bad = !(fabsf(v) < INFINITY);
#pragma unroll
              for (int nc = 0; nc < NC; ++nc) c.o[nc][e][i] += bad && (seen[nc] >> key & 1) ? v : 0.f;
            }
        }
      }
    }
  };
  // A block has arrived when all but the wavefront's loads of those behind it have, and everybody says so; by then everybody has left
  // the block in front of it, whose place the next one takes.  8 bits: the block behind the one at hand has, to be widened, and the one
  // at hand is.  Blocks that every column sees whole come first, in a loop of their own (none where one of the piece's pages is not there).
  const int whole_end = all_there ? min(end, x.whole()) : blk0;
  auto arrive = [&]() __attribute__((always_inline)) {
    TREE_TILE_BARRIER((LAG - (Q8 ? 2 : 1)) * Tiles::LOADS);
    __builtin_amdgcn_sched_barrier(0);
  };
  if constexpr (Q8) {
    TREE_TILE_BARRIER((LAG - 1) * Tiles::LOADS);
    take();
    widen(half);
  }
  int blk = blk0;
  for (; blk < whole_end; ++blk, half ^= 1) {
    arrive();
    const bool in[2] = {true, true};
    block(std::integral_constant<bool, false>{}, blk, in);
  }
  for (; blk < end; ++blk, half ^= 1) {
    arrive();
    const bool in[2] = {all_there || (there >> (2 * LAG - 2) & 1) != 0, all_there || (there >> (2 * LAG - 2) & 2) != 0};
    block(std::integral_constant<bool, true>{}, blk, in);
  }
  TREE_WAIT_LOADS(0);                                                // (nothing is on its way to LDS when the workgroup ends)

  // ---- partials
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    const float l = pc_rows_sum(c.l[nc]);
    const int r = 16 * (NC * wave + nc) + c16;
    if (r >= x.n_here) continue;
    const bool whole = a.n_shares == 0;
    const TreeOut to = tree_out(a, x, r);
    const long long row = whole ? 0 : tree_part_row(a, x, place, r);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int u = 0; u < VE; ++u) {                                   // four values of the row at a time
      floatx4 y;
#pragma unroll
      for (int w = 0; w < 4; ++w) y[w] = l == 0.f ? 0.f : c.o[nc][u][w] * inv;
      const int d = 16 * u + 4 * kk;
      if (whole) *(uint2*)(a.c.out + to.row * D + d) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
      else *(floatx4*)(a.part_o + row * D + d) = y;
    }
    if (kk == 0) {
      const float lse = l == 0.f ? -INFINITY : (c.ref[nc] + log2f(l)) * SHARED_LN2;
      if (!whole) a.part_lse[row] = lse;
      else if (a.c.lse) a.c.lse[to.lse] = lse;
    }
  }
}

// A share's first place on the line of all sequences' blocks: of sequence begin[0], at its begin[1].  In front of a sequence's
// blocks are `extra` places without one, for what a piece costs beside its keys.  Every thread counts those of a run of sequences.
__device__ __forceinline__ int tree_scan(const TreeArgs& a, int share, TreeScanLds& sm) {
  const int lane = threadIdx.x % PC_WAVE, wave = threadIdx.x / PC_WAVE;
  const int per = (a.c.batch + TREE_THREADS - 1) / TREE_THREADS, b0 = min((int)threadIdx.x * per, a.c.batch), b1 = min(b0 + per, a.c.batch);
  auto places = [&](const TreeSeq& s) { const int nb = tree_blocks(a.c, s); return nb > 0 ? nb + a.extra : 0; };
  int mine = 0;
  for (int b = b0; b < b1; ++b) {
    const TreeSeq s = tree_seq(a.c, b);
    if (per == 1) sm.seq[b] = s;
    mine += places(s);
  }
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
  const int each = total / n_eff, rest = total - each * n_eff;
  const int lo = share * each + min(share, rest), n = each + (share < rest);
  if (n == 0) return 0;
  if (lo >= before && lo < before + mine) {
    int off = lo - before, b = b0;
    for (; b < b1; ++b) {
      const int p = places(tree_seq(a.c, b));
      if (off < p) break;
      off -= p;
    }
    sm.begin[0] = b; sm.begin[1] = off;
  }
  __syncthreads();
  return n;
}

// What a workgroup is: 16 or 32 query rows, each wavefront with a part of the keys; or 64 or 128, keys in LDS
template <int D, int ROWS, bool Q8>
struct TreeBody {
  static constexpr bool FEW = ROWS <= 32;
  static constexpr int NC = FEW ? ROWS / 16 : ROWS / 64;
  typedef typename std::conditional<FEW, TreeLds<D, FEW ? NC : 1>, typename TreeTiles<D, Q8>::Lds>::type Lds;
};
template <int D, int ROWS, bool Q8, int PARTS>
__global__ __launch_bounds__(TREE_THREADS, 2) void tree_rows_kernel(TreeArgs a) {
  typedef TreeBody<D, ROWS, Q8> Body;
  extern __shared__ __align__(16) unsigned char lds[];
  typename Body::Lds& sm = *(typename Body::Lds*)lds;
  // an XCD (number mod 8) has an eighth of (share, head, tile), the tiles behind each other: its L2 serves the keys to them
  const int at = (int)(blockIdx.x % 8) * a.per_xcd + (int)(blockIdx.x / 8);
  if (at >= a.n_groups * a.n_tiles) return;
  const int sg = pc_div(at, a.tiles_div), tile = at - sg * a.n_tiles;
  const int share = pc_div(sg, a.heads_div), g = sg - share * a.c.n_kv_heads;
  auto piece = [&](int b, const TreeSeq& s, int blk0, int n_blk, int place) __attribute__((always_inline)) {
    TreePiece x;
    x.b = b; x.g = g; x.row0 = tile * ROWS;
    x.n_here = min(ROWS, s.rows * a.group - x.row0);
    if (x.n_here <= 0) return;
    x.len = tree_there(a.c, s); x.base = s.len - s.rows;
    if constexpr (Body::FEW) tree_piece<D, Body::NC, Q8>(a, x, blk0, n_blk, place, sm);
    else tree_tile_piece<D, Body::NC, Q8, PARTS>(a, x, blk0, n_blk, place, sm);
  };
  // sequences are not cut: a workgroup has a whole one's, and its result; else a share of all of them
  const bool whole = a.n_shares == 0;
  int left = 1, b = share, off = 0;
  if (!whole) {
    left = tree_scan(a, share, sm.scan);
    if (left == 0) return;
    b = __builtin_amdgcn_readfirstlane(sm.scan.begin[0]); off = __builtin_amdgcn_readfirstlane(sm.scan.begin[1]);
  }
  for (; left > 0 && b < a.c.batch; ++b, off = 0) {
    TreeSeq s;
    if (!whole && a.c.batch <= TREE_THREADS) s = sm.scan.seq[b];
    else s = tree_seq(a.c, b);
    s.rows = __builtin_amdgcn_readfirstlane(s.rows); s.len = __builtin_amdgcn_readfirstlane(s.len);
    const int nb = tree_blocks(a.c, s);
    int blk0 = 0, n_blk = nb;
    if (whole) {
      left = 0;
    } else {
      if (nb == 0) continue;
      const int take = min(left, nb + a.extra - off);
      left -= take;
      blk0 = max(off - a.extra, 0); n_blk = max(off + take - a.extra, 0) - blk0;
      if (n_blk == 0) continue;
      if (g == 0 && tile == 0 && threadIdx.x == 0) {
        if (blk0 == 0) a.span[b].x = share;
        if (blk0 + n_blk == nb) a.span[b].y = share;
      }
    }
    piece(b, s, blk0, n_blk, share + b);
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
  const TreeSeq seq = tree_seq(a.c, b);
  if (t >= seq.rows) return;
  const int g = pc_div(h, a.group_div), r = t * a.group + h - g * a.group;
  float m = -INFINITY, den = 0.f;
  floatx4 num = {0.f, 0.f, 0.f, 0.f};
  if (tree_blocks(a.c, seq) > 0) {
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
  const long long cap = (long long)c.pages.max_pages << c.pages.shift, blocks = c.batch * ((cap + 31) / 32);
  // 17 to 32 rows: the body of 64 keeps more of the longest rows on their way, though it leaves half of its own empty.  us a call,
  // 32 query rows a KV head, 8 KV heads, sequences x places (and a page), body of 32 / of 64:
  //   bf16, 128 values    (2 x 512) 15 / 17   (2 x 8192) 37 / 27   (16 x 512) 18 / 17   (16 x 2048) 41 / 29   (16 x 4096) 58 / 44   (64 x 8192) 275 / 255
  //   bf16, 64 values     (2 x 512) 11 / 14   (2 x 8192) 25 / 23   (16 x 512) 12 / 14   (16 x 2048) 26 / 23   (16 x 4096) 32 / 30   (64 x 8192) 130 / 129
  //   8 bits, 128 values  (2 x 512) 15 / 20   (2 x 8192) 31 / 30   (16 x 512) 16 / 21   (16 x 2048) 36 / 33   (16 x 4096) 43 / 46   (64 x 8192) 167 / 239
  //   8 bits, 64 values   (2 x 512) 11 / 15   (2 x 8192) 24 / 24   (16 x 512) 12 / 15   (16 x 2048) 25 / 25   (16 x 4096) 29 / 34   (64 x 8192) 90 / 152
  // (Shorter rows than the longest take the body of 32 throughout: where that of 64 is ahead, it is by 10 % at most.)
  const bool longest = !c.pages.k_scale && c.head_dim == 128 && cap > 1024;
  p.rows = rows <= 16 ? 16 : (rows <= 32 && !longest ? 32 : (rows <= 64 ? 64 : 128));
  p.tiles = (rows + p.rows - 1) / p.rows;
  // One launch, a workgroup a sequence (and KV head and tile), where the pages hold little for each, or workgroups are many.  us a
  // call, cut / whole, lengths from a third of the pages' on, 8 KV heads of 128 values, sequences x query rows a KV head x places:
  //   bf16 (2 x 4 x 576) 15.5 / 10.5   (2 x 4 x 1024) 14.0 / 18.6   (16 x 4 x 1024) 21.4 / 19.7   (64 x 4 x 2048) 63.7 / 60.4   (16 x 4 x 2048) 26.0 / 33.6
  //   (2 x 64 x 512) 19.2 / 16.4   (16 x 64 x 1024) 29.0 / 26.9   (64 x 64 x 2048) 86.5 / 68.7   (64 x 128 x 2048) 125 / 96
  //   8 bits (2 x 4 x 1024) 13.0 / 13.8   (16 x 4 x 1024) 19.5 / 14.5   (16 x 4 x 2048) 21.7 / 21.7   (16 x 128 x 512) 35 / 27   (64 x 128 x 2048) 126 / 102
  // One rule for both formats and all numbers of sequences, by the pages alone: two sequences of 1024 places lose up to 5 us by it, sixteen gain 2 to 5;
  // sixteen of 1024 places and 64 rows a KV head would gain 2.  Lengths are not known here, so short sequences in wide tables are cut: up to
  // 512 rows in tables of 131072 places, 16 sequences x 4 rows, 19.2 us, whole 13.3; x 64 rows 28.3, whole 18.9.
  const long long groups = (long long)c.batch * c.n_kv_heads * p.tiles;
  if ((cap <= (rows <= 32 ? 1024 : 512) || (cap <= 2048 && groups >= 512)) && groups < TREE_GROUPS) {
    p.shares = 0;
    return p;
  }
  long long shares = 512 / ((long long)c.n_kv_heads * p.tiles);
  if (shares > blocks / 8) shares = blocks / 8;
  p.shares = shares < 1 ? 1 : (int)shares;
  return p;
}
static long long groups(const PcTreeCall& c, const PcTreePlan& p) { return (long long)(p.shares ? p.shares : c.batch) * c.n_kv_heads; }
bool pc_tree_fits(const PcTreeCall& c, const PcTreePlan& p) {
  const long long blocks = (((long long)c.pages.max_pages << c.pages.shift) + 31) / 32;
  return groups(c, p) * p.tiles < TREE_GROUPS && c.batch * (blocks + TREE_EXTRA) < (1LL << 31);
}
static size_t part_rows(const PcTreeCall& c, const PcTreePlan& p) { return p.shares ? (size_t)(p.shares + c.batch) * c.n * c.n_q_heads : 0; }
size_t pc_tree_ws_bytes(const PcTreeCall& c, const PcTreePlan& p) {
  const size_t rows = part_rows(c, p);
  return pc_align_up(rows * c.head_dim * 4, 256) + pc_align_up(rows * 4, 256) + pc_align_up((size_t)c.batch * sizeof(int2), 256);
}

template <int D, int ROWS, bool Q8, int PARTS>
static int launch_rows(const TreeArgs& a, hipStream_t st) {
  static std::atomic<uint64_t> raised{0};
  constexpr int LDS = sizeof(typename TreeBody<D, ROWS, Q8>::Lds);
  const int rc = pc_raise_dynamic_lds((const void*)tree_rows_kernel<D, ROWS, Q8, PARTS>, LDS, raised);
  if (rc != PC_OK) return rc;
  PcProfScope prof(PC_KERNEL_TREE_ATTN, st);
  hipLaunchKernelGGL((tree_rows_kernel<D, ROWS, Q8, PARTS>), dim3((unsigned)(8 * a.per_xcd)), dim3(TREE_THREADS), LDS, st, a);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
template <int D, bool Q8>
static int launch_body(const TreeArgs& a, const PcTreePlan& p, hipStream_t st) {
  if (p.rows == 16) return launch_rows<D, 16, Q8, 2>(a, st);
  if (p.rows == 32) return launch_rows<D, 32, Q8, 2>(a, st);
  if (p.rows == 64) return a.c.pos ? launch_rows<D, 64, Q8, 2>(a, st) : launch_rows<D, 64, Q8, 1>(a, st);
  return a.c.pos ? launch_rows<D, 128, Q8, 2>(a, st) : launch_rows<D, 128, Q8, 1>(a, st);
}
template <int D>
static int launch_all(const PcTreeCall& c, const PcTreePlan& p, void* ws, hipStream_t st) {
  TreeArgs a;
  a.c = c;
  a.rope = pc_rope_factors(c.pos ? c.rope_base : 2.0f, c.head_dim);
  a.group = c.n_q_heads / c.n_kv_heads; a.n_tiles = p.tiles; a.n_shares = p.shares;
  a.n_groups = (int)groups(c, p);
  a.per_xcd = (int)((groups(c, p) * p.tiles + 7) / 8); a.extra = TREE_EXTRA;
  a.group_div = pc_div_by(a.group); a.tiles_div = pc_div_by(p.tiles); a.heads_div = pc_div_by(c.n_kv_heads);
  a.scale_log2 = c.scale * SHARED_LOG2E;
  const size_t rows = part_rows(c, p);
  a.part_o = (float*)ws;
  a.part_lse = (float*)((char*)ws + pc_align_up(rows * D * 4, 256));
  a.span = (int2*)((char*)a.part_lse + pc_align_up(rows * 4, 256));
  const int rc = c.pages.k_scale ? launch_body<D, true>(a, p, st) : launch_body<D, false>(a, p, st);
  if (rc != PC_OK || p.shares == 0) return rc;
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
