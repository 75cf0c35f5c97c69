// Attention of a batch whose sequences share a prefix: the prefix's keys are read once for the query rows of all its
// sequences, each sequence's own tail once for its rows, under one softmax.
//
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q . k_j,  over the prefix's keys and the tail's.
//
// The rows (sequence, t, head of the group) of one KV head are the columns of S^T = K Q^T, so that a key that has been
// loaded serves them all.  A workgroup of eight wavefronts takes a CU and a run of keys, and leaves a partial (o, lse) a
// row, which shared_merge_kernel joins by logsumexp:
//   few rows   (16, 32 or 64): a wavefront has 16 or 32 of them and a part of the run, from memory straight into
//              registers, a key read by as many wavefronts as there are groups of 32 rows;
//   row tiles  (256 rows): a wavefront has 32 rows; tiles of 128 keys go through LDS as matrix operands, widened and
//              transposed once on the way in, so that every wavefront reads them with 16 consecutive bytes a lane;
//   tails      of up to 16 rows: one to eight wavefronts each, behind the prefix's workgroups in their launch; of more rows
//              the same bodies in a launch of their own, where 128 values spill 23 to 77 registers (32 columns' state beside
//              the path for values that are not finite).
// Where few keys are shared, one launch takes every (sequence, KV head) for itself, prefix and tail (shared_alone).
// Bound by memory up to some 170 rows (8-bit rows: 85), by the matrix cores and the softmax's vector instructions beyond.
// Measured (8 KV heads of 128 values): 64 rows, 8 x 2048 keys, 16 tails of 512: 26 us (the loop at 28 GB/s a CU, then starts and
// the merge); 64 rows, 32 x 2048 keys of 8 bits 48 us; 4096 rows, 8 x 2048 keys 430 us (0.65 PFLOP/s), 322 as they arrive; 4 rows,
// 128 keys 7.0 us.
// Rows of 8 bits: a code is a bf16 value exactly, the key's scale multiplies the logit in fp32, the value's scale the
// probability in front of its rounding.  Rotated query rows keep two bf16 parts (2^-17).  Probabilities are rounded to bf16 once
// (up to 2^-8 of each, 1.7e-3 of the result's norm on average, as much as the result's own rounding): a second part would
// double the second product.
#include "decode_core.h"
#include "shared_core.h"
#include "serve.h"

#define SHARED_WAVES 8
#define SHARED_THREADS (SHARED_WAVES * PC_WAVE)

struct SharedArgs {
  const uint16_t* q;
  const int32_t* q_pos;
  int pos0;
  PcRope rope;
  PcRows rows;             // the prefixes or the tails
  int fan, n_q, n_q_heads, n_kv_heads, group;   // sequences a cache (1: tails)
  int own;                 // the last n_q rows are the query rows' own
  int n_rows, n_tiles;     // fan n_q group, and in tiles
  int n_runs, n_parts, part0, per_xcd, tail_waves;
  PcDiv parts_div, heads_div, group_div, q_div, tiles_div, fan_div;      // fan_div: by the sequences of a prefix
  float scale_log2;
  float* part_o;           // [part][B n_q H_q][D]
  float* part_lse;         // [part][B n_q H_q]
  long long part_rows;     // B n_q H_q
  uint16_t* out;           // where the launch joins
  float* lse;
};

// The place of a workgroup: its cache, KV head, run of keys and rows
struct SharedPlace {
  int c, g, part, row0, n_here;
  long long tok0;          // the cache's first (sequence, t)
};
__device__ __forceinline__ SharedPlace shared_place(const SharedArgs& a, int run, int tile, int tile_rows) {
  SharedPlace x;
  const int cg = pc_div(run, a.parts_div);
  x.part = run - cg * a.n_parts;
  x.c = pc_div(cg, a.heads_div); x.g = cg - x.c * a.n_kv_heads;
  x.row0 = tile * tile_rows;
  x.n_here = min(tile_rows, a.n_rows - x.row0);
  x.tok0 = (long long)x.c * a.fan * a.n_q;
  return x;
}
__device__ __forceinline__ PcSegLens shared_lens(const SharedArgs& a, const SharedPlace& x) {
  PcSegLens l;
  l.seg_len = a.rows.len; l.per_head = a.rows.len_per_head; l.n_seg = a.rows.n_seg;
  l.n_kv_heads = a.n_kv_heads; l.k_t = a.rows.cap; l.b = x.c; l.g = x.g;
  return l;
}
// A 32-key block: where its rows start, how many are valid, how many of its segment's follow from its first one on
struct SharedBlock { PcBlockCursor at; long long row; int keys; };
__device__ __forceinline__ SharedBlock shared_block(const SharedArgs& a, const SharedPlace& x, const PcBlockCursor& at) {
  SharedBlock b; b.at = at; b.row = 0; b.keys = 0;           // behind the run's end: nothing is read
  if (at.left > 0) {
    b.row = (((long long)x.c * a.rows.n_seg + at.s) * a.n_kv_heads + x.g) * a.rows.cap + 32LL * at.blk;
    b.keys = min(32, at.len - 32 * at.blk);
  }
  return b;
}

// The tile's N query rows into LDS (rows behind the last one: zeros), rotated.  A rotated row is kept as two bf16 parts, whose
// sum is the row to 2^-17 (`lo` is nullptr only where rows arrive rotated).  D / 16 threads a row, 8 values of each half; every load
// is asked for in front of the arithmetic (`begin`), which has the first keys in flight behind it.
template <int D, int N, int WAVES>
struct SharedQueryRows {
  static constexpr int HALF = D / 2, TPR = HALF / 8, PASS = WAVES * PC_WAVE / TPR, PASSES = (N + PASS - 1) / PASS;
  u32x4 lo_half[PASSES], hi_half[PASSES];
  int pos[PASSES];
  __device__ __forceinline__ void begin(const SharedArgs& a, const SharedPlace& x, int thread) {
    const int i0 = thread % TPR * 8;
#pragma unroll
    for (int n = 0; n < PASSES; ++n) {
      const int r = min(x.row0 + min(thread / TPR + n * PASS, x.n_here - 1), a.n_rows - 1);
      const int ft = pc_div(r, a.group_div), h = r - ft * a.group;
      const uint16_t* src = a.q + ((x.tok0 + ft) * a.n_q_heads + x.g * a.group + h) * D + i0;
      lo_half[n] = *(const u32x4*)src; hi_half[n] = *(const u32x4*)(src + HALF);
      if (a.q_pos) {
        const int f = pc_div(ft, a.q_div);
        pos[n] = a.q_pos[(long long)x.c * a.fan + f] + (ft - f * a.n_q);
      }
    }
  }
  __device__ __forceinline__ void finish(const SharedArgs& a, const SharedPlace& x, uint16_t (*hi)[D + 8], uint16_t (*lo)[D + 8], int thread) {
    const int i0 = thread % TPR * 8;
    double theta[8];
    if (a.q_pos) {
#pragma unroll
      for (int e = 0; e < 8; ++e) theta[e] = pc_rope_theta(a.rope, i0 + e);
    }
#pragma unroll
    for (int n = 0; n < PASSES; ++n) {
      const int r = thread / TPR + n * PASS;
      if (r >= N) break;
      u32x4 u = lo_half[n], v = hi_half[n], ul = {0, 0, 0, 0}, vl = {0, 0, 0, 0};
      if (r >= x.n_here) u = v = u32x4{0, 0, 0, 0};
      if (a.q_pos) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float y1[2], y2[2];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const float x1 = b ? bf16_hi_to_f32(u[w]) : bf16_lo_to_f32(u[w]), x2 = b ? bf16_hi_to_f32(v[w]) : bf16_lo_to_f32(v[w]);
            float sn, cs;
            pc_sincos_f32(((double)a.pos0 + pos[n]) * theta[2 * w + b], sn, cs);
            y1[b] = x1 * cs - x2 * sn; y2[b] = x2 * cs + x1 * sn;
          }
          u[w] = pack_bf16x2(y1[0], y1[1]); v[w] = pack_bf16x2(y2[0], y2[1]);
          ul[w] = pack_bf16x2(y1[0] - bf16_lo_to_f32(u[w]), y1[1] - bf16_hi_to_f32(u[w]));
          vl[w] = pack_bf16x2(y2[0] - bf16_lo_to_f32(v[w]), y2[1] - bf16_hi_to_f32(v[w]));
        }
      }
      *(u32x4*)&hi[r][i0] = u; *(u32x4*)&hi[r][i0 + HALF] = v;
      if (lo) { *(u32x4*)&lo[r][i0] = ul; *(u32x4*)&lo[r][i0 + HALF] = vl; }
    }
  }
};
__device__ __forceinline__ long long shared_partial_row(const SharedArgs& a, const SharedPlace& x, int r) {
  const int ft = pc_div(x.row0 + r, a.group_div), h = x.row0 + r - ft * a.group;
  return (long long)(a.part0 + x.part) * a.part_rows + (x.tok0 + ft) * a.n_q_heads + x.g * a.group + h;
}
// the last rows of a cache that a column does not see
__device__ __forceinline__ int shared_unseen(const SharedArgs& a, int row) {
  return a.own ? a.n_q - 1 - pc_div(min(row, a.n_rows - 1), a.group_div) : 0;        // (own: fan = 1, so that is t)
}

// ------------------------------------------------------------------------------------------ few rows
// A wavefront's walk over its run of 32-key blocks, from memory into registers: `begin` asks for the first block, `run`
// takes all of them.  One buffer for the keys and one for the values: the next block's keys are asked for behind the
// first product, its values behind the second one, and the SIMD's other wavefronts work meanwhile.  Rows behind a
// block's last valid one are out of the descriptor and arrive as zeros.  V: key i of the lane is 4 kk + i (i < 4) or
// 16 + 4 kk + i - 4, the keys whose logits the lane holds.
template <int D, int NC, int WK, bool Q8, bool OWN, int HINT>
struct SharedWalk {
  static constexpr int KSTEPS = D / 32, VE = D / 16, ELEM = Q8 ? 1 : 2, ROW = D * ELEM;      // VE: values a lane takes of a V row
  static constexpr int KP = Q8 ? D / 64 : KSTEPS;           // 16-byte pieces of a key a lane takes: a k-step, or two in 8 bits
  typedef uint32_t vpiece __attribute__((ext_vector_type(VE * ELEM / 4)));
  u32x4 kbuf[2][KP];
  vpiece vbuf[8];
  float sbuf;                                               // scale of key `lane` (lanes 0 .. 31), of value lane - 32
  SharedBlock cur;
  PcSegLens lens;

  __device__ __forceinline__ void keys(const SharedArgs& a, const SharedBlock& b) {
    const int lane = threadIdx.x % PC_WAVE, kk = lane / 16, c16 = lane % 16;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)a.rows.k + b.row * ROW), 0, b.keys * ROW, 0x00020000);
    if constexpr (Q8)                                        // (every lane reads a row that is there)
      sbuf = (lane < 32 ? a.rows.k_scale : a.rows.v_scale)[b.row + max(min(lane % 32, b.keys - 1), 0)];
#pragma unroll
    for (int bi = 0; bi < 2; ++bi)
#pragma unroll
      for (int p = 0; p < KP; ++p) kbuf[bi][p] = __builtin_amdgcn_raw_buffer_load_b128(r, c16 * ROW + 16 * kk, 16 * bi * ROW + 64 * p, HINT);
    __builtin_amdgcn_sched_barrier(0);                       // not behind the arithmetic that follows
  }
  __device__ __forceinline__ void values(const SharedArgs& a, const SharedBlock& b) {
    const int lane = threadIdx.x % PC_WAVE, kk = lane / 16, c16 = lane % 16;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)a.rows.v + b.row * ROW), 0, b.keys * ROW, 0x00020000);
    const int off = (4 * kk * D + VE * c16) * ELEM;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(vpiece) == 16) vbuf[i] = __builtin_amdgcn_raw_buffer_load_b128(r, off, (i < 4 ? i : i + 12) * ROW, HINT);
      else if constexpr (sizeof(vpiece) == 8) vbuf[i] = __builtin_amdgcn_raw_buffer_load_b64(r, off, (i < 4 ? i : i + 12) * ROW, HINT);
      else vbuf[i] = __builtin_amdgcn_raw_buffer_load_b32(r, off, (i < 4 ? i : i + 12) * ROW, HINT);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ void begin(const SharedArgs& a, const SharedPlace& x, int wk, int first_lens, int waves = WK) {
    lens = shared_lens(a, x);
    cur = shared_block(a, x, pc_blocks_begin<WK>(lens, x.part, a.n_parts, a.parts_div, wk, threadIdx.x % PC_WAVE, first_lens, waves));
    keys(a, cur);
    values(a, cur);
  }
  // scale: the wavefront's room in LDS for a block's scales
  __device__ __forceinline__ void run(const SharedArgs& a, const SharedPlace& x, SharedColumns<D, NC>& c, const int (&unseen)[NC], float (*scale)[32]) {
    const int lane = threadIdx.x % PC_WAVE, kk = lane / 16;
    const int most_unseen = OWN && a.own ? a.n_q - 1 : 0;
    while (cur.at.left > 0) {
      const SharedBlock nx = shared_block(a, x, pc_blocks_next(lens, cur.at));
      if constexpr (Q8) scale[lane / 32][lane % 32] = sbuf;
      floatx4 s[NC][1][2];
#pragma unroll
      for (int nc = 0; nc < NC; ++nc)
#pragma unroll
        for (int bi = 0; bi < 2; ++bi) s[nc][0][bi] = floatx4{0.f, 0.f, 0.f, 0.f};
      __builtin_amdgcn_s_setprio(1);                         // the first product goes first (8-bit rows 1 to 2 % faster)
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
            for (int nc = 0; nc < NC; ++nc)
              s[nc][0][bi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(bf16x8*)&ka, c.q[h][nc][ks], s[nc][0][bi], 0, 0, 0);
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
      const int left[1] = {cur.at.len - 32 * cur.at.blk};
      const bool masked = left[0] - most_unseen < 32;
      const auto hidden = [&](int nc, int b, int bi, int j) { return 16 * bi + 4 * kk + j >= left[b] - unseen[nc]; };
      u32x4 p[NC][1];
      __builtin_amdgcn_s_setprio(0);
      shared_softmax<NC, 1, VE, Q8>(s, sc, masked, hidden, a.scale_log2, c.ref, c.sub, c.l, c.o, p);
      shared_values<NC, 1, VE, OWN>([&](int, int e) { return shared_value_operand<Q8>(vbuf, e); }, masked && most_unseen > 0, p, c.o);
      __builtin_amdgcn_sched_barrier(0);
      values(a, nx);
      cur = nx;
    }
  }
};

// Partials of a run of the prefix's (or, OWN, a tail's) keys
template <int D, int NC, int WR, int WAVES, bool Q8, bool OWN>
__device__ __forceinline__ void shared_few_rows(const SharedArgs& a, int run, int tile, SharedFewLds<D, NC, WR, WAVES>& sm) {
  constexpr int ROWS = 16 * NC * WR, WK = WAVES / WR;
  const int lane = threadIdx.x % PC_WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PC_WAVE);
  const int wk = wave / WR, col0 = 16 * NC * (wave % WR);
  const SharedPlace x = shared_place(a, run, tile, ROWS);
  const int first_lens = pc_first_lens(shared_lens(a, x), lane);
  SharedQueryRows<D, ROWS, WAVES> rows;
  rows.begin(a, x, threadIdx.x);                                         // (the older loads: waiting for them leaves the keys in flight)
  SharedWalk<D, NC, WK, Q8, OWN, WR == 1 ? PC_BUF_NT : 0> walk;      // (a block is read by WR wavefronts)
  walk.begin(a, x, wk, first_lens);
  rows.finish(a, x, sm.q[0], sm.q[1], threadIdx.x);
  PC_LDS_BARRIER();
  SharedColumns<D, NC> c;
  c.clear();
  shared_query_operands<D, NC, Q8>(c, sm.q[0], sm.q[1], col0);
  PC_LDS_BARRIER();
  int unseen[NC];
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) unseen[nc] = OWN ? shared_unseen(a, x.row0 + col0 + 16 * nc + lane % 16) : 0;
  walk.run(a, x, c, unseen, sm.scale[wave]);

  // ---- the wavefronts' totals -> the workgroup's partial
  shared_columns_out<D, NC>(c, sm, wk, col0, x.n_here);
  __syncthreads();
  for (int idx = threadIdx.x; idx < x.n_here * (D / 4); idx += WAVES * PC_WAVE) {
    const int r = idx / (D / 4), d4 = idx % (D / 4) * 4;
    SharedRowSum sum;
    sum.clear();
#pragma unroll
    for (int w = 0; w < WK; ++w) sum.add(sm.m[w][r], sm.l[w][r], *(const floatx4*)&sm.o[w][r][d4]);
    const long long row = shared_partial_row(a, x, r);
    *(floatx4*)(a.part_o + row * D + d4) = sum.mean();
    if (d4 == 0) a.part_lse[row] = sum.lse();
  }
}

// Partials of tails of up to 16 rows: `waves` wavefronts a run of a tail's keys, 8 / waves runs a workgroup.  A workgroup
// takes a CU, so with one tail a workgroup many short tails wait for each other's latencies.
template <int D>
struct SharedTailsLds {
  union {
    float o[SHARED_WAVES][16][D + 4];
    uint16_t q[SHARED_WAVES][2][16][D + 8];
  };
  float m[SHARED_WAVES][16], l[SHARED_WAVES][16];
  float scale[SHARED_WAVES][2][32];
};
template <int D, bool Q8>
__device__ __forceinline__ void shared_tail_rows(const SharedArgs& a, int wg, SharedTailsLds<D>& sm) {
  const int lane = threadIdx.x % PC_WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PC_WAVE);
  const int waves = a.tail_waves, per = SHARED_WAVES / waves;
  const int run = wg * per + wave / waves;
  const SharedPlace x = shared_place(a, min(run, a.n_runs - 1), 0, 16);
  const int first_lens = pc_first_lens(shared_lens(a, x), lane);
  SharedQueryRows<D, 16, 1> rows;
  rows.begin(a, x, lane);
  SharedWalk<D, 1, 1, Q8, true, PC_BUF_NT> walk;
  walk.begin(a, x, wave % waves, first_lens, waves);
  rows.finish(a, x, sm.q[wave][0], sm.q[wave][1], lane);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  SharedColumns<D, 1> c;
  c.clear();
  shared_query_operands<D, 1, Q8>(c, sm.q[wave][0], sm.q[wave][1], 0);
  const int unseen[1] = {shared_unseen(a, lane % 16)};
  walk.run(a, x, c, unseen, sm.scale[wave]);
  PC_LDS_BARRIER();                                          // (the query rows are written over)
  shared_columns_out<D, 1>(c, sm, wave, 0, x.n_here);
  __syncthreads();
  const int n_here = min(16, a.n_rows), runs = min(per, a.n_runs - wg * per);
  for (int idx = threadIdx.x; idx < runs * n_here * (D / 4); idx += SHARED_THREADS) {
    const int d4 = idx % (D / 4) * 4, rr = idx / (D / 4), which = rr / n_here, r = rr - which * n_here;
    SharedRowSum sum;
    sum.clear();
    for (int w = which * waves; w < (which + 1) * waves; ++w) sum.add(sm.m[w][r], sm.l[w][r], *(const floatx4*)&sm.o[w][r][d4]);
    const long long row = shared_partial_row(a, shared_place(a, wg * per + which, 0, 16), r);
    *(floatx4*)(a.part_o + row * D + d4) = sum.mean();
    if (d4 == 0) a.part_lse[row] = sum.lse();
  }
}

// The whole call in one launch, where few keys are shared: one workgroup a (sequence, KV head) of up to 16 query rows
// takes the prefix's keys (PREFIX: 1 16-bit, 2 8-bit rows, 0 none), then the tail's, and writes the result.
template <int D, int PREFIX, bool Q8, int WAVES>
__device__ __forceinline__ void shared_alone(const SharedArgs& p, const SharedArgs& a, int run, SharedFewLds<D, 1, 1, WAVES>& sm) {
  const int lane = threadIdx.x % PC_WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PC_WAVE);
  const SharedPlace x = shared_place(a, run, 0, 16);
  SharedPlace xp = x;                                        // the same rows over their prefix
  xp.c = pc_div(x.c, a.fan_div);
  const int first_lens = pc_first_lens(shared_lens(a, x), lane);
  int prefix_lens = 0;
  if (PREFIX) prefix_lens = pc_first_lens(shared_lens(p, xp), lane);
  SharedQueryRows<D, 16, WAVES> rows;
  rows.begin(a, x, threadIdx.x);
  SharedWalk<D, 1, WAVES, PREFIX == 2, false, 0> prefix;
  SharedWalk<D, 1, WAVES, Q8, true, PC_BUF_NT> tail;
  if constexpr (PREFIX) prefix.begin(p, xp, wave, prefix_lens);
  else tail.begin(a, x, wave, first_lens);
  rows.finish(a, x, sm.q[0], sm.q[1], threadIdx.x);
  PC_LDS_BARRIER();
  SharedColumns<D, 1> c;
  c.clear();
  shared_query_operands<D, 1, PREFIX ? PREFIX == 2 : Q8>(c, sm.q[0], sm.q[1], 0);
  const int unseen[1] = {shared_unseen(a, lane % 16)}, none[1] = {0};
  if constexpr (PREFIX) {
    prefix.run(p, xp, c, none, sm.scale[wave]);
    tail.begin(a, x, wave, first_lens);
    if constexpr ((PREFIX == 2) != Q8) shared_query_operands<D, 1, Q8>(c, sm.q[0], sm.q[1], 0);
  }
  tail.run(a, x, c, unseen, sm.scale[wave]);
  PC_LDS_BARRIER();                                          // (the query rows are written over)

  shared_columns_out<D, 1>(c, sm, wave, 0, x.n_here);
  __syncthreads();
  for (int idx = threadIdx.x; idx < x.n_here * (D / 4); idx += WAVES * PC_WAVE) {
    const int r = idx / (D / 4), i4 = idx % (D / 4) * 4;
    SharedRowSum sum;
    sum.clear();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum.add(sm.m[w][r], sm.l[w][r], *(const floatx4*)&sm.o[w][r][i4]);
    const floatx4 y = sum.mean();
    const int t = pc_div(r, a.group_div), h = x.g * a.group + r - t * a.group;
    *(uint2*)(a.out + ((x.tok0 + t) * a.n_q_heads + h) * D + i4) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
    if (a.lse && i4 == 0) a.lse[((long long)x.c * a.n_q_heads + h) * a.n_q + t] = sum.lse();
  }
}

// ------------------------------------------------------------------------------------------ row tiles
// A tile of keys in LDS: SHARED_BLOCKS 32-key blocks as matrix operands of 64 lanes x 16 bytes
#define SHARED_BLOCKS 4
template <int D>
struct SharedTile {
  u32x4 k[SHARED_BLOCKS][2][D / 32][PC_WAVE];       // [block][16 keys][k-step]
  u32x4 v[SHARED_BLOCKS][D / 16][PC_WAVE];          // [block][operand e of V^T]
  float scale[2][SHARED_BLOCKS][32];                // [keys, values][block]
};
#define SHARED_TILE_ROWS (SHARED_WAVES * 32)
template <int D, int PARTS>
struct SharedTilesLds {
  union {
    SharedTile<D> tile[2];
    uint16_t q[PARTS][SHARED_TILE_ROWS][D + 8];
  };
};

// PARTS: bf16 parts of a query row, two where it is rotated.  The second one's products and registers cost (4096 rows, 16384
// keys) 340 -> 433 us, with 8-bit rows 422 -> 474; without it the result's error is 2.9e-3 of its norm instead of 2.3e-3 where
// logits have a deviation of 1, and grows with that.  With 128 values a row, one block at a time then: two blocks' logits
// beside both parts spill (452 and 504 us).
template <int D, bool Q8, bool OWN, int PARTS>
__device__ __forceinline__ void shared_row_tiles(const SharedArgs& a, int run, int tile, SharedTilesLds<D, PARTS>& sm) {
  constexpr int KSTEPS = D / 32, VE = D / 16, ELEM = Q8 ? 1 : 2, ROW = D * ELEM, NC = 2, KB = PARTS == 2 && D == 128 ? 1 : 2;
  typedef uint32_t piece_t __attribute__((ext_vector_type(VE * ELEM / 4)));
  const int lane = threadIdx.x % PC_WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PC_WAVE);
  const int kk = lane / 16, c16 = lane % 16;
  const SharedPlace x = shared_place(a, run, tile, SHARED_TILE_ROWS);
  const PcSegLens lens = shared_lens(a, x);
  auto next = [&](const SharedBlock& b) { return shared_block(a, x, pc_blocks_next(lens, b.at)); };

  // Wavefronts 0 to 3 bring the keys of the tile's blocks, 4 to 7 the values, by eight loads of D / 16 values a lane:
  // a key operand's 8 values (32 ks + 8 kk ..) of 16 keys, D / 64 loads each, or whole rows, D / 16 values of the lane's
  // 8 keys.  The same instructions for both, at other offsets: under conditions the waits in front of a tile's use would
  // take the later tiles' loads for its own.  Rows behind a block's last valid one are out of the descriptor: zeros.
  const int my_block = wave % SHARED_BLOCKS;
  const bool my_values = wave >= SHARED_BLOCKS;
  // (by arithmetic: a choice between two fields of the arguments would send them through memory)
  const uint8_t* my_rows = (const uint8_t*)a.rows.k + my_values * ((intptr_t)a.rows.v - (intptr_t)a.rows.k);
  const float* my_scales = (const float*)((intptr_t)a.rows.k_scale + my_values * ((intptr_t)a.rows.v_scale - (intptr_t)a.rows.k_scale));
  const int my_off = my_values ? (4 * kk * D + VE * c16) * ELEM : (c16 * D + 8 * kk) * ELEM;
  int my_step[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    my_step[i] = (my_values ? (i < 4 ? i : i + 12) * D : 16 * (i / 4) * D + 32 * (i % 4 * VE / 8) + VE * (i % (8 / VE))) * ELEM;
  struct Pieces { piece_t at[8]; float scale; };
  Pieces pieces;
  struct Left { int b0, b1, b2, b3; };                      // keys of a block's segment from its first one on; 0: no block
  // Asks for a tile whose first block is `b`, leaves the last one there
  auto issue = [&](Pieces& to, SharedBlock& b) __attribute__((always_inline)) {
    Left l;
    auto left = [&]() { return b.at.left > 0 ? b.at.len - 32 * b.at.blk : 0; };
    long long row = b.row;
    int keys = b.keys;
    l.b0 = left();
    b = next(b); l.b1 = left();
    if (my_block == 1) { row = b.row; keys = b.keys; }
    b = next(b); l.b2 = left();
    if (my_block == 2) { row = b.row; keys = b.keys; }
    b = next(b); l.b3 = left();
    if (my_block == 3) { row = b.row; keys = b.keys; }
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(my_rows + row * ROW), 0, keys * ROW, 0x00020000);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(piece_t) == 16) to.at[i] = __builtin_amdgcn_raw_buffer_load_b128(r, my_off, my_step[i], 0);
      else if constexpr (sizeof(piece_t) == 8) to.at[i] = __builtin_amdgcn_raw_buffer_load_b64(r, my_off, my_step[i], 0);
      else to.at[i] = __builtin_amdgcn_raw_buffer_load_b32(r, my_off, my_step[i], 0);
    }
    if constexpr (Q8) to.scale = my_scales[row + max(min(lane % 32, keys - 1), 0)];      // (a row that is there, in every lane)
    __builtin_amdgcn_sched_barrier(0);
    return l;
  };
  auto commit = [&](int buf, const Pieces& from) __attribute__((always_inline)) {
    SharedTile<D>& t = sm.tile[buf];
    if (!my_values) {
#pragma unroll
      for (int op = 0; op < 2 * KSTEPS; ++op) {              // operand (16 keys op / KSTEPS, k-step op % KSTEPS): 8 / VE pieces
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          constexpr int PER = 8 / VE;                        // pieces an operand
          const piece_t x = from.at[op * PER + i * PER / 4];
          if constexpr (Q8) w[i] = shared_widen(x[i / 2 % (VE / 4)], i % 2);
          else w[i] = x[i % (VE / 2)];
        }
        t.k[my_block][op / KSTEPS][op % KSTEPS][lane] = w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) t.v[my_block][e][lane] = shared_value_operand<Q8>(from.at, e);
    }
    if constexpr (Q8) {
      if (lane < 32) t.scale[my_values][my_block][lane] = from.scale;
    }
  };

  // ---- the query rows; meanwhile the first tile is on its way
  const int first_lens = pc_first_lens(lens, lane);
  SharedQueryRows<D, SHARED_TILE_ROWS, SHARED_WAVES> rows;
  rows.begin(a, x, threadIdx.x);
  SharedBlock last = shared_block(a, x, pc_blocks_begin<1>(lens, x.part, a.n_parts, a.parts_div, 0, lane, first_lens));
  Left at = issue(pieces, last);                            // the tile at hand
  rows.finish(a, x, sm.q[0], PARTS == 2 ? sm.q[PARTS - 1] : nullptr, threadIdx.x);
  PC_LDS_BARRIER();
  bf16x8 bq[PARTS][NC][KSTEPS];
#pragma unroll
  for (int h = 0; h < PARTS; ++h)
#pragma unroll
    for (int nc = 0; nc < NC; ++nc)
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) bq[h][nc][ks] = *(const bf16x8*)&sm.q[h][16 * (wave * NC + nc) + c16][32 * ks + 8 * kk];
  PC_LDS_BARRIER();
  int unseen[NC];
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) unseen[nc] = !OWN ? 0 : shared_unseen(a, x.row0 + 16 * (wave * NC + nc) + c16);
  const int most_unseen = OWN && a.own ? a.n_q - 1 : 0;
  float ref[NC], sub[NC], l_run[NC];
  floatx4 o[NC][VE];
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    ref[nc] = -INFINITY; sub[nc] = 0.f; l_run[nc] = 0.f;
#pragma unroll
    for (int e = 0; e < VE; ++e) o[nc][e] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // KB blocks together, so that their chains overlap; a block behind the run's end has no keys.  The products go first where
  // both wavefronts of a SIMD can issue (4096 rows as they arrive, 16384 keys: 335 -> 322 us; rotated ones 429 -> 434, 8-bit rows 448
  // -> 442).
  auto consume = [&](const SharedTile<D>& t, int first, const int (&left)[KB]) __attribute__((always_inline)) {
    __builtin_amdgcn_s_setprio(1);
    floatx4 s[NC][KB][2];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc)
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int bi = 0; bi < 2; ++bi) s[nc][b][bi] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) {
      u32x4 ka[KB][2];
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int bi = 0; bi < 2; ++bi) ka[b][bi] = t.k[first + b][bi][ks][lane];
#pragma unroll
      for (int h = PARTS - 1; h >= 0; --h)                   // (a sum's two parts are four products apart)
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int bi = 0; bi < 2; ++bi)
#pragma unroll
            for (int nc = 0; nc < NC; ++nc)
              s[nc][b][bi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)&ka[b][bi], bq[h][nc][ks], s[nc][b][bi], 0, 0, 0);
    }
    SharedScales sc[KB];
    if constexpr (Q8) {
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int bi = 0; bi < 2; ++bi) {
          sc[b].k[bi] = *(const floatx4*)&t.scale[0][first + b][16 * bi + 4 * kk];
          sc[b].v[bi] = *(const floatx4*)&t.scale[1][first + b][16 * bi + 4 * kk];
        }
    }
    int least = left[0];
#pragma unroll
    for (int b = 1; b < KB; ++b) least = min(least, left[b]);
    const bool masked = least - most_unseen < 32;
    const auto hidden = [&](int nc, int b, int bi, int j) { return 16 * bi + 4 * kk + j >= left[b] - unseen[nc]; };
    u32x4 p[NC][KB];
    __builtin_amdgcn_s_setprio(0);
    shared_softmax<NC, KB, VE, Q8>(s, sc, masked, hidden, a.scale_log2, ref, sub, l_run, o, p);
    __builtin_amdgcn_s_setprio(1);
    shared_values<NC, KB, VE, OWN>([&](int b, int e) { return t.v[first + b][e][lane]; }, masked && most_unseen > 0, p, o);
    __builtin_amdgcn_s_setprio(0);
  };

  // Tile t is in LDS buffer t % 2 while tile t + 1 is on its way into registers: that is written to the other buffer,
  // which everybody left at the barrier in front, behind tile t's arithmetic.
  commit(0, pieces);
  last = next(last);
  Left ahead = issue(pieces, last);                         // the one on its way
  PC_LDS_BARRIER();
  for (int buf = 0; at.b0 > 0; buf ^= 1) {
    if constexpr (KB == 2) {
      consume(sm.tile[buf], 0, {at.b0, at.b1});
      if (at.b2 > 0) consume(sm.tile[buf], 2, {at.b2, at.b3});
    } else {
      consume(sm.tile[buf], 0, {at.b0});
      if (at.b1 > 0) consume(sm.tile[buf], 1, {at.b1});
      if (at.b2 > 0) consume(sm.tile[buf], 2, {at.b2});
      if (at.b3 > 0) consume(sm.tile[buf], 3, {at.b3});
    }
    commit(buf ^ 1, pieces);
    at = ahead;
    last = next(last);
    ahead = issue(pieces, last);
    PC_LDS_BARRIER();
  }

  // ---- partials
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    const float l = pc_rows_sum(l_run[nc]);
    const int r = 16 * (wave * NC + nc) + c16;
    if (r >= x.n_here) continue;
    const long long row = shared_partial_row(a, x, r);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < VE; e += 4) {
        floatx4 y;
#pragma unroll
        for (int u = 0; u < 4; ++u) y[u] = l == 0.f ? 0.f : o[nc][e + u][i] * inv;
        *(floatx4*)(a.part_o + row * D + VE * (4 * kk + i) + e) = y;
      }
    if (kk == 0) a.part_lse[row] = l == 0.f ? -INFINITY : (ref[nc] + log2f(l)) * SHARED_LN2;
  }
}

// ------------------------------------------------------------------------------------------ merge
// The partials of a row, joined: D / 4 threads take 4 values each of every SPLIT-th partial under a maximum of their own;
// with SPLIT > 1 the row's groups of threads are put together through LDS in a fixed order.
struct SharedMergeArgs {
  const float* part_o;
  const float* part_lse;
  uint16_t* out;
  float* lse;
  long long n_rows;
  int n_parts, n_q, n_q_heads;
};
template <int D, int SPLIT>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedMergeArgs a) {
  constexpr int TPR = D / 4, U = 4;
  __shared__ floatx4 num_lds[SPLIT > 1 ? 256 : 1];
  __shared__ float2 ml_lds[256 / TPR];
  const int grp = threadIdx.x / TPR, d4 = threadIdx.x % TPR * 4;
  const long long row = (long long)blockIdx.x * (256 / TPR / SPLIT) + grp / SPLIT;          // (b, t, h)
  const long long at_row = min(row, a.n_rows - 1);
  float m = -INFINITY, den = 0.f;
  floatx4 num = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = grp % SPLIT; p0 < a.n_parts; p0 += U * SPLIT) {
    float l[U];
    floatx4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long at = (long long)min(p0 + u * SPLIT, a.n_parts - 1) * a.n_rows + at_row;
      l[u] = a.part_lse[at];
      x[u] = *(const floatx4*)(a.part_o + at * D + d4);
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p0 + u * SPLIT >= a.n_parts) l[u] = -INFINITY;
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
      for (int e = 0; e < 4; ++e) num[e] += l[u] == -INFINITY ? 0.f : w * x[u][e];     // (the last one again may hold infinities)
    }
  }
  if constexpr (SPLIT > 1) {
    num_lds[threadIdx.x] = num;
    if (d4 == 0) ml_lds[grp] = make_float2(m, den);
    __syncthreads();
    if (grp % SPLIT != 0) return;
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < SPLIT; ++i) M = fmaxf(M, ml_lds[grp + i].x);
    const float ref = M == -INFINITY ? 0.f : M;
    den = 0.f;
    num = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < SPLIT; ++i) {
      const float w = expf(ml_lds[grp + i].x - ref);
      const floatx4 y = num_lds[threadIdx.x + i * TPR];
      den += w * ml_lds[grp + i].y;
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] += w * y[e];
    }
    m = M;
  }
  if (row >= a.n_rows) return;
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = den == 0.f ? 0.f : num[e] / den;
  *(uint2*)(a.out + row * D + d4) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
  if (a.lse && d4 == 0) {
    const long long bt = row / a.n_q_heads, b = bt / a.n_q;
    a.lse[(b * a.n_q_heads + row % a.n_q_heads) * a.n_q + bt % a.n_q] = den == 0.f ? -INFINITY : m + logf(den);
  }
}

// ------------------------------------------------------------------------------------------ launches
// What a launch's workgroups are: few rows (16, 32 or 64 of them), row tiles of 256 rows, those of rotated rows (the launch
// sees to it: a plan has SHARED_TILE); odd numbers: 8-bit rows
enum SharedBody { SHARED_FEW16 = 2, SHARED_FEW32 = 4, SHARED_FEW64 = 6, SHARED_TILE = 8, SHARED_TILE_ROTATED = 10 };
static constexpr int shared_body_rows(int body) { return body >= SHARED_TILE ? SHARED_TILE_ROWS : 8 << body / 2; }
template <int D, int BODY>
struct SharedBodyOf {
  static constexpr bool Q8 = BODY % 2, FEW = BODY < SHARED_TILE;
  static constexpr int ROWS = shared_body_rows(BODY), NC = ROWS < 32 ? 1 : 2, WR = FEW ? ROWS / (16 * NC) : 1;
  static constexpr int PARTS = BODY >= SHARED_TILE_ROTATED ? 2 : 1;
  typedef SharedFewLds<D, NC, WR, SHARED_WAVES> FewLds;
  static constexpr int LDS = FEW ? sizeof(FewLds) : sizeof(SharedTilesLds<D, PARTS>);
};
// Partials of `a`'s keys: OWN, of tails; else of prefixes, and behind their n_first workgroups those of the tails of up
// to 16 rows.  An XCD (number mod 8) has an eighth of (run, tile), the tiles of a run behind each other: its L2 serves
// the run's keys to them.
template <int D, int BODY, bool OWN>
__global__ __launch_bounds__(SHARED_THREADS, 2) void shared_rows_kernel(SharedArgs a, SharedArgs tail, int n_first) {
  typedef SharedBodyOf<D, BODY> B;
  extern __shared__ __align__(16) unsigned char lds[];
  if (!OWN && (int)blockIdx.x >= n_first) {
    if (tail.rows.k_scale) shared_tail_rows<D, true>(tail, (int)blockIdx.x - n_first, *(SharedTailsLds<D>*)lds);
    else shared_tail_rows<D, false>(tail, (int)blockIdx.x - n_first, *(SharedTailsLds<D>*)lds);
    return;
  }
  const int at = (int)(blockIdx.x % 8) * a.per_xcd + (int)(blockIdx.x / 8);
  if (at >= a.n_runs * a.n_tiles) return;
  const int run = pc_div(at, a.tiles_div), tile = at - run * a.n_tiles;
  if constexpr (B::FEW) shared_few_rows<D, B::NC, B::WR, SHARED_WAVES, B::Q8, OWN>(a, run, tile, *(typename B::FewLds*)lds);
  else shared_row_tiles<D, B::Q8, OWN, B::PARTS>(a, run, tile, *(SharedTilesLds<D, B::PARTS>*)lds);
}
// Four wavefronts: with eight (128 keys, tails of 64) 8.7 us instead of 7.6 at 8 workgroups, 15.1 instead of 9.5 at 512
#define SHARED_ALONE 4
template <int D, int PREFIX, bool Q8>
__global__ __launch_bounds__(SHARED_ALONE * PC_WAVE, 2) void shared_alone_kernel(SharedArgs prefix, SharedArgs tail) {
  __shared__ SharedFewLds<D, 1, 1, SHARED_ALONE> sm;
  shared_alone<D, PREFIX, Q8, SHARED_ALONE>(prefix, tail, (int)blockIdx.x, sm);
}

// ---- host
struct SharedCost { double start, block, bytes, blocks; int most; };      // us of a workgroup, of a 32-key block in it; a block's bytes
static double block_bytes(const PcRows& r, int D) { return 32.0 * (r.k_scale ? 2.0 * D + 8 : 4.0 * D); }
static double blocks_of(const PcRows& r, double share) { return share * r.n_seg * (double)((r.cap + 31) / 32); }
static PcSharedSide side_of(long long n_caches, long long rows, int n_kv_heads, int body) {
  PcSharedSide s = {};
  s.body = body; s.parts = 1; s.waves = SHARED_WAVES;
  s.tiles = (rows + shared_body_rows(s.body) - 1) / shared_body_rows(s.body);
  s.caches_heads = n_caches * n_kv_heads;
  s.runs = s.caches_heads;
  return s;
}
// Measured, one workgroup a CU: 27 GB/s of keys a CU; or the arithmetic, rows x keys of a block at 1.8 to 3.0 TFLOP/s a CU,
// or a block's latencies (64 values a row: half); queries, partials and latencies 5.5 to 12 us a workgroup (0.6 of that).
// Tails in a launch of their own are priced as prefixes are
static SharedCost cost_of(const PcSharedSide& s, const PcRows& r, int D, double share) {
  static const struct { double start, bf16, row8, least; } of[] = {      // us, TFLOP/s, TFLOP/s, us
      {5.5, 2.6, 2.0, 0.0}, {6.5, 1.8, 3.0, 0.0}, {7.5, 2.5, 2.3, 0.35}, {12.0, 2.7, 1.9, 1.7}};
  const auto& m = of[s.body / 2 - 1];
  SharedCost c = {};
  c.bytes = block_bytes(r, D);
  const double memory = c.bytes / 27e3, arithmetic = 4.0 * 32 * shared_body_rows(s.body) * D / ((r.k_scale ? m.row8 : m.bf16) * 1e6);
  c.start = m.start * (D == 64 ? 0.6 : 1.0);
  c.block = fmax(fmax(memory, arithmetic), m.least * (D == 64 ? 0.5 : 1.0));
  c.blocks = blocks_of(r, share) + 1.0;
  c.most = c.blocks < 8.0 ? 1 : (c.blocks > 256.0 ? 64 : (int)(c.blocks / 4.0));
  return c;
}
// One launch, a workgroup of four wavefronts a (sequence, KV head), as many a CU as the fullest one has: prefix keys at 55 GB/s
// a CU (they are in its L2), the tail's at 31, or a block's latency.  380 such calls: 8 % off (root mean square)
static double alone_us(const PcSharedCall& c) {
  const double a_cu = (double)c.batch * c.n_kv_heads / 256.0, at_once = ceil(a_cu);
  const double p = blocks_of(c.prefix, 1.0), t = blocks_of(c.tail, 0.75) + 1.0;
  return 5.7 + 0.7 * a_cu + fmax(at_once * p * block_bytes(c.prefix, c.head_dim) / 55e3, 0.13 * p) +
         fmax(at_once * t * block_bytes(c.tail, c.head_dim) / 31e3, 0.2 * t);
}
// A workgroup of 8 / waves tails' runs: the CU's reads, or a wavefront's blocks one after the other
static double tails_us(const SharedCost& c, int waves, int tp) {
  const double reads = SHARED_WAVES / waves * c.blocks / tp * c.bytes / 33e3, chain = c.blocks / (waves * tp) * 0.9;
  return c.start + (reads > chain ? reads : chain);
}
// The call's time: the prefix's np workgroups of one_p us first, then the tails' nt of one_t
static double time_of(double one_p, int np, double one_t, int nt) {
  const int rest = np & 255, room = 256 - rest;
  const double us = (np >> 8) * one_p, last = rest ? one_p : 0.0;
  if (nt == 0) return us + last;
  const double beside = rest ? floor(one_p / (1.4 * one_t)) * room : 0.0;      // tails that are surely done next to the last prefix ones
  if (nt > beside && nt > room) return us + last + ((nt - (int)beside + 255) >> 8) * one_t;
  const double t_us = ((nt + room - 1) / room) * one_t;
  return us + (t_us > last ? t_us : last);
}
static bool tails_behind(const PcSharedPlan& p) { return p.prefix.body && p.tail.body && p.tail.body <= SHARED_FEW16 + 1; }
// The cuts of least time for p's bodies; returns that time without the launches'
static double cut_of(const PcSharedCall& c, PcSharedPlan& p) {
  SharedCost pc = {0, 0, 0, 0, 1}, tc = {0, 0, 0, 0, 1};
  if (p.prefix.body) pc = cost_of(p.prefix, c.prefix, c.head_dim, 1.0);
  if (p.tail.body) tc = cost_of(p.tail, c.tail, c.head_dim, 0.75);
  const double row_us = (double)c.batch * c.n_q * c.n_q_heads * c.head_dim * 8.0 / 5e6;
  // a few cuts: the tails' coarse ones, and for each those of the prefix that fill one to three rounds of the CUs by
  // themselves, with the tails, or with a half of them
  const long long pg = p.prefix.body ? p.prefix.caches_heads * p.prefix.tiles : 0, tg = p.tail.body ? p.tail.caches_heads * p.tail.tiles : 0;
  const bool behind = tails_behind(p);
  static const int cuts[][2] = {{8, 1}, {4, 1}, {2, 1}, {1, 1}, {8, 2}, {8, 4}, {8, 8}, {8, 16}};      // wavefronts a run, parts
  double least = -1.0;
  for (const auto& cut : cuts) {
    const int waves = cut[0], tp = cut[1];
    if (tp > 1 && tp > tc.most) break;
    if (waves < SHARED_WAVES && !behind) continue;
    const long long tails = (tg * tp * waves + SHARED_WAVES - 1) / SHARED_WAVES;
    const int nt = (int)(tails < (1 << 24) ? tails : 1 << 24);
    const double one_t = tg ? (behind ? tails_us(tc, waves, tp) : tc.start + tc.block * tc.blocks / tp) : 0.0;
    long long weighed = 0;
    auto weigh = [&](long long pp) {
      pp = pp < 1 ? 1 : (pp > pc.most ? pc.most : pp);
      if (pp == weighed) return;
      weighed = pp;
      const int np = (int)(pg * pp < (1 << 24) ? pg * pp : 1 << 24);
      const double us = time_of(pc.start + pc.block * pc.blocks / (double)pp, np, one_t, nt) + row_us * (double)((pg ? pp : 0) + (tg ? tp : 0));
      if (least < 0.0 || us < least) {
        least = us;
        if (pg) p.prefix.parts = (int)pp;
        if (tg) { p.tail.parts = tp; p.tail.waves = waves; }
      }
    };
    weigh(1);
    if (!pg) continue;
    weigh(pc.most);
    for (int fill = 256; fill <= 768; fill += 256)
      for (int part : {0, nt, nt / 2}) weigh((fill - part) / pg);
  }
  return least;
}
// Of the bodies that fit, and of one launch for all (up to 16 rows), the one of least estimated time, rows taken as rotated (the
// plan does not know).  600 calls with tails of up to 16 rows (2 to 4096 rows a KV head, 60 to 32768 keys, both formats, 64 and
// 128 values) and 200 with tails of more were timed with each body.  The choice costs 2 % and 4 % over the best in the mean, 9 and
// 17 % at the 90th percentile, 33 and 65 % at most; one launch throughout 61 % more than it, 32 rows 9 and 3 %, 64 rows 8 and
// 3 %, tiles 33 and 14 %.  us with 32 rows / 64 rows / tiles, bf16: (64 rows x 1024 keys) 13.2 / 15.2 / -, (512 x 1024) 22.8 / 22.7 /
// 32.4, (512 x 16384) 110 / 94 / 87, (4096 x 16384) 840 / 605 / 407; 8 bits: (64 x 1024) 13.4 / 15.1 / -, (512 x 16384) 74 / 71 / 90,
// (4096 x 16384) 478 / 438 / 451.  One launch / two: (16 sequences, 128 keys, tails of 64) 7.6 / 11.2, (16, 1024, 64) 14.6 / 12.9,
// (4, 1024, 512) 20.1 / 13.9.  Tails, 8 x 2048 keys in front: (16 sequences, 64 rows, 512) 151 / 152 / -, (16, 256, 512) 493 / 461 /
// 430, (4, 1200, 600) 673 / 644 / 586.
PcSharedPlan pc_shared_plan(const PcSharedCall& c) {
  const long long own_rows = (long long)c.n_q * (c.n_q_heads / c.n_kv_heads), rows = c.batch / c.n_prefix * own_rows;
  auto bodies = [](long long n, int (&of)[3]) {
    if (n <= 16) { of[0] = SHARED_FEW16; return 1; }
    of[0] = SHARED_FEW32; of[1] = SHARED_FEW64; of[2] = SHARED_TILE;
    return n <= 32 ? 1 : (n <= 64 ? 2 : 3);
  };
  int of_prefix[3] = {0}, of_tail[3] = {0};
  const int n_of_prefix = c.prefix.n_seg > 0 ? bodies(rows, of_prefix) : 1, n_of_tail = c.tail.n_seg > 0 ? bodies(own_rows, of_tail) : 1;
  PcSharedPlan best = {}, alone = {};
  alone.alone = true;
  const double one = own_rows <= 16 ? alone_us(c) : 1e30, launch = 6.0;  // (a second launch)
  if (one < launch + 3.0) return alone;                      // (less than any cut)
  double least = -1.0;
  for (int i = 0; i < n_of_prefix; ++i)
    for (int j = 0; j < n_of_tail; ++j) {
      PcSharedPlan p = {};
      if (c.prefix.n_seg > 0) p.prefix = side_of(c.n_prefix, rows, c.n_kv_heads, of_prefix[i] + (c.prefix.k_scale != nullptr));
      if (c.tail.n_seg > 0) p.tail = side_of(c.batch, own_rows, c.n_kv_heads, of_tail[j] + (c.tail.k_scale != nullptr));
      const double us = cut_of(c, p);
      if (least < 0.0 || us < least) { least = us; best = p; }
    }
  if (one < least + launch) return alone;
  best.prefix.runs = best.prefix.caches_heads * best.prefix.parts;
  best.tail.runs = best.tail.caches_heads * best.tail.parts;
  return best;
}
static long long workgroups(const PcSharedSide& s) { return s.body ? (s.runs * s.tiles + 7) / 8 * 8 : 0; }
static int partials(const PcSharedPlan& p) { return p.prefix.parts + p.tail.parts; }

// The one-launch kernel's bodies: 0 no keys, 1 16-bit, 2 8-bit rows (it has no body without a tail: an empty 16-bit one)
struct AloneFormats { int prefix, tail; };
static AloneFormats alone_formats(const PcSharedCall& c) {
  return {c.prefix.n_seg == 0 ? 0 : (c.prefix.k_scale ? 2 : 1), c.tail.k_scale ? 2 : 1};
}
void pc_shared_plan_info(const PcSharedCall& c, const PcSharedPlan& p, pc_shared_attn_plan_info& info) {
  info = {};
  info.alone = p.alone;
  if (p.alone) {
    const auto f = alone_formats(c);
    info.prefix_format = f.prefix; info.tail_format = f.tail;
    info.prefix_rows = f.prefix ? 16 : 0; info.tail_rows = 16;
    info.prefix_parts = f.prefix ? 1 : 0; info.tail_parts = 1; info.tail_waves = SHARED_ALONE;
    return;
  }
  if (p.prefix.body) { info.prefix_format = 1 + p.prefix.body % 2; info.prefix_rows = shared_body_rows(p.prefix.body); info.prefix_parts = p.prefix.parts; }
  if (p.tail.body) {
    info.tail_format = 1 + p.tail.body % 2; info.tail_rows = shared_body_rows(p.tail.body); info.tail_parts = p.tail.parts;
    info.tail_waves = p.tail.waves; info.tails_behind = tails_behind(p);
  }
}
bool pc_shared_fits(const PcSharedCall& c, const PcSharedPlan& p) {
  return workgroups(p.prefix) + workgroups(p.tail) < (1LL << 32) / SHARED_THREADS &&
         (long long)c.batch * c.n_kv_heads < (1LL << 32) / SHARED_THREADS;
}
size_t pc_shared_ws_bytes(const PcSharedCall& c, const PcSharedPlan& p) {
  const size_t rows = (size_t)c.batch * c.n_q * c.n_q_heads * partials(p);
  return pc_align_up(rows * c.head_dim * 4, 256) + pc_align_up(rows * 4, 256) + 256;
}

static SharedArgs side_args(const PcSharedCall& c, const PcRows& rows, const PcSharedSide& s, int n_caches, int own, int part0,
                            float* part_o, float* part_lse) {
  SharedArgs a;
  a.q = (const uint16_t*)c.q; a.q_pos = c.q_pos; a.pos0 = c.pos0; a.rope = pc_rope_factors(c.q_pos ? c.rope_base : 2.0f, c.head_dim);
  a.rows = rows; a.fan = c.batch / n_caches; a.own = own;
  a.n_q = c.n_q; a.n_q_heads = c.n_q_heads; a.n_kv_heads = c.n_kv_heads; a.group = c.n_q_heads / c.n_kv_heads;
  a.n_rows = a.fan * a.n_q * a.group;
  a.n_tiles = (int)s.tiles; a.n_runs = (int)s.runs; a.per_xcd = (int)((s.runs * s.tiles + 7) / 8); a.n_parts = s.parts; a.part0 = part0; a.tail_waves = s.waves;
  a.parts_div = pc_div_by(s.parts); a.heads_div = pc_div_by(a.n_kv_heads); a.group_div = pc_div_by(a.group);
  a.q_div = pc_div_by(a.n_q); a.tiles_div = pc_div_by(a.n_tiles); a.fan_div = pc_div_by(c.batch / c.n_prefix);
  a.scale_log2 = c.scale * SHARED_LOG2E;
  a.part_o = part_o; a.part_lse = part_lse; a.part_rows = (long long)c.batch * c.n_q * c.n_q_heads;
  a.out = (uint16_t*)c.out; a.lse = c.lse;
  return a;
}

template <int D, int BODY, bool OWN>
static int launch(const SharedArgs& a, const SharedArgs& tail, long long n, long long n_tail, hipStream_t st) {
  static std::atomic<uint64_t> raised{0};
  constexpr int A = SharedBodyOf<D, BODY>::LDS, B = sizeof(SharedTailsLds<D>), LDS = OWN || A > B ? A : B;
  const int rc = pc_raise_dynamic_lds((const void*)shared_rows_kernel<D, BODY, OWN>, LDS, raised);
  if (rc != PC_OK) return rc;
  PcProfScope prof(OWN ? PC_KERNEL_SHARED_TAIL : PC_KERNEL_SHARED_PREFIX, st);
  hipLaunchKernelGGL((shared_rows_kernel<D, BODY, OWN>), dim3((unsigned)(n + n_tail)), dim3(SHARED_THREADS), LDS, st, a, tail, (int)n);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
template <int D, bool OWN>
static int launch_rows(const PcSharedSide& s, const SharedArgs& a, const SharedArgs& tail, long long n_tail, hipStream_t st) {
  const long long n = workgroups(s);
  switch (s.body >= SHARED_TILE && a.q_pos ? s.body + SHARED_TILE_ROTATED - SHARED_TILE : s.body) {
    case SHARED_FEW16: return launch<D, SHARED_FEW16, OWN>(a, tail, n, n_tail, st);
    case SHARED_FEW16 + 1: return launch<D, SHARED_FEW16 + 1, OWN>(a, tail, n, n_tail, st);
    case SHARED_FEW32: return launch<D, SHARED_FEW32, OWN>(a, tail, n, n_tail, st);
    case SHARED_FEW32 + 1: return launch<D, SHARED_FEW32 + 1, OWN>(a, tail, n, n_tail, st);
    case SHARED_FEW64: return launch<D, SHARED_FEW64, OWN>(a, tail, n, n_tail, st);
    case SHARED_FEW64 + 1: return launch<D, SHARED_FEW64 + 1, OWN>(a, tail, n, n_tail, st);
    case SHARED_TILE: return launch<D, SHARED_TILE, OWN>(a, tail, n, n_tail, st);
    case SHARED_TILE + 1: return launch<D, SHARED_TILE + 1, OWN>(a, tail, n, n_tail, st);
    case SHARED_TILE_ROTATED: return launch<D, SHARED_TILE_ROTATED, OWN>(a, tail, n, n_tail, st);
    case SHARED_TILE_ROTATED + 1: return launch<D, SHARED_TILE_ROTATED + 1, OWN>(a, tail, n, n_tail, st);
    default: return PC_OK;                                   // no such rows
  }
}
template <int D, int PREFIX>
static int launch_alone(const PcSharedCall& c, const SharedArgs& p, const SharedArgs& t, long long n, hipStream_t st) {
  const dim3 grid((unsigned)n), block(SHARED_ALONE * PC_WAVE);
  if (alone_formats(c).tail == 2) hipLaunchKernelGGL((shared_alone_kernel<D, PREFIX, true>), grid, block, 0, st, p, t);
  else hipLaunchKernelGGL((shared_alone_kernel<D, PREFIX, false>), grid, block, 0, st, p, t);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
template <int D>
static int launch_alone_of(const PcSharedCall& c, const SharedArgs& p, const SharedArgs& t, hipStream_t st) {
  PcProfScope prof(PC_KERNEL_SHARED_ALONE, st);
  const long long n = (long long)c.batch * c.n_kv_heads;
  const int prefix = alone_formats(c).prefix;
  return prefix == 0 ? launch_alone<D, 0>(c, p, t, n, st) : (prefix == 1 ? launch_alone<D, 1>(c, p, t, n, st) : launch_alone<D, 2>(c, p, t, n, st));
}

template <int D>
static int launch_merge(const SharedMergeArgs& m, hipStream_t st) {
  constexpr int GROUPS = 256 / (D / 4);
  PcProfScope prof(PC_KERNEL_SHARED_MERGE, st);
  // A workgroup's groups of threads share a row where rows are few and each group has more than one partial of it.  us a call, a
  // row a group / a workgroup (128 values): 32 rows of 8 partials 23.6 / 23.5, of 25 16.8 / 13.8; 512 of 25 23.8 / 21.2;
  // 2048 of 25 47.6 / 47.8; 8192 of 7 77.9 / 81.8; 512 of 16 and of 25 with 64 values 16.8 / 16.8, 17.6 / 15.5
  const bool wide = m.n_parts > GROUPS && m.n_rows <= 1024;
  if (wide) hipLaunchKernelGGL((shared_merge_kernel<D, GROUPS>), dim3((unsigned)m.n_rows), dim3(256), 0, st, m);
  else hipLaunchKernelGGL((shared_merge_kernel<D, 1>), dim3((unsigned)((m.n_rows + GROUPS - 1) / GROUPS)), dim3(256), 0, st, m);
  PC_LAUNCH_CHECK();
  return PC_OK;
}

template <int D>
static int launch_all(const PcSharedCall& c, const PcSharedPlan& pl, void* ws, hipStream_t st) {
  const size_t rows = (size_t)c.batch * c.n_q * c.n_q_heads;
  const int parts = partials(pl);
  float* part_o = (float*)ws;
  float* part_lse = (float*)((char*)ws + pc_align_up(rows * parts * D * 4, 256));
  if (pl.alone) {
    const PcSharedSide one = {0, 1, SHARED_WAVES, 1, (long long)c.batch * c.n_kv_heads, (long long)c.batch * c.n_kv_heads};
    return launch_alone_of<D>(c, side_args(c, c.prefix, one, c.batch, 0, 0, part_o, part_lse),
                              side_args(c, c.tail, one, c.batch, c.tail_own, 0, part_o, part_lse), st);
  }
  SharedArgs t = {};
  if (pl.tail.body) t = side_args(c, c.tail, pl.tail, c.batch, c.tail_own, pl.prefix.parts, part_o, part_lse);
  const bool behind = tails_behind(pl);
  if (pl.prefix.body) {
    const SharedArgs p = side_args(c, c.prefix, pl.prefix, c.n_prefix, 0, 0, part_o, part_lse);
    const int rc = launch_rows<D, false>(pl.prefix, p, behind ? t : p, behind ? (pl.tail.runs * pl.tail.waves + SHARED_WAVES - 1) / SHARED_WAVES : 0, st);
    if (rc != PC_OK) return rc;
  }
  if (pl.tail.body && !behind) {
    const int rc = launch_rows<D, true>(pl.tail, t, t, 0, st);
    if (rc != PC_OK) return rc;
  }
  SharedMergeArgs m;
  m.part_o = part_o; m.part_lse = part_lse; m.out = (uint16_t*)c.out; m.lse = c.lse;
  m.n_rows = (long long)rows; m.n_parts = parts; m.n_q = c.n_q; m.n_q_heads = c.n_q_heads;
  return launch_merge<D>(m, st);
}
int pc_launch_shared_attn(const PcSharedCall& c, const PcSharedPlan& pl, void* ws, hipStream_t st) {
  return c.head_dim == 128 ? launch_all<128>(c, pl, ws, st) : launch_all<64>(c, pl, ws, st);
}
