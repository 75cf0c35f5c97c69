// Attention of a batch whose sequences share a prefix: the prefix's keys are read once for the query rows of all its
// sequences, each sequence's own tail once for its rows, under one softmax.
//
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = scale q . k_j,  over the prefix's keys and the tail's.
//
// The rows (sequence, t, head of the group) of one KV head are the columns of S^T = K Q^T, so a key that has been
// loaded serves them all: a column block is 16 of them, a workgroup takes NC blocks (up to 64 rows), its four
// wavefronts a quarter of a run of 32-key blocks each.  Runs leave partials (o, lse), which shared_merge_kernel joins
// by logsumexp.  Rows of 8 bits are widened in registers: a code is a bf16 value exactly, the key's scale multiplies
// the logit in fp32, the value's scale the probability in front of its rounding.
#include "serve.h"

#define SHARED_WAVES 4
#define SHARED_THREADS (SHARED_WAVES * PC_WAVE)
#define SHARED_LOG2E 1.4426950408889634f
#define SHARED_LN2 0.6931471805599453f

struct SharedArgs {
  const uint16_t* q;
  const int32_t* q_pos;
  int pos0;
  PcRope rope;
  PcRows rows;             // the prefixes or the tails
  int fan, n_q, n_q_heads, n_kv_heads, group;   // sequences a cache (1: tails)
  int own;                 // the last n_q rows are the query rows' own
  int n_rows, n_tiles;     // fan n_q group, and in tiles of 16 NC
  int n_caches, n_parts, part0;
  PcDiv parts_div, heads_div, group_div, q_div, tiles_div;
  float scale_log2;
  float* part_o;           // [part][B n_q H_q][D]
  float* part_lse;         // [part][B n_q H_q]
  long long part_rows;     // B n_q H_q
};

// four E4M3 codes of a word -> two packed bf16 pairs, exactly
typedef __bf16 shared_bf2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t shared_widen(uint32_t w, bool high) {
  const shared_bf2 a = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
  return *(const uint32_t*)&a;
}

template <int D, int NC>
struct SharedLds {
  float o[SHARED_WAVES][16 * NC][D];
  float m[SHARED_WAVES][16 * NC], l[SHARED_WAVES][16 * NC];
  float scale[SHARED_WAVES][2][32];     // the 8-bit rows' scales of a wavefront's block: keys, values
};

// Two bf16 of a word that are infinite or NaN -> 1.0 in their places, 0 elsewhere
__device__ __forceinline__ uint32_t shared_bad(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0x3f80u : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0x3f800000u : 0u);
}

template <int D, int NC, bool Q8>
__device__ __forceinline__ void shared_workgroup(const SharedArgs& a, int run, int tile, unsigned char* lds) {
  constexpr int KSTEPS = D / 32, VE = D / 16;               // VE: values a lane takes of a V row
  constexpr int KP = Q8 ? D / 64 : KSTEPS;                  // 16-byte pieces of a key a lane takes
  constexpr int ROW = Q8 ? D : 2 * D;                       // bytes of a row
  typedef uint32_t vpiece __attribute__((ext_vector_type(Q8 ? VE / 4 : VE / 2)));
  SharedLds<D, NC>& sm = *(SharedLds<D, NC>*)lds;
  uint16_t(*sq)[D + 8] = (uint16_t(*)[D + 8])lds;           // the query rows, in front of the loop only

  const int lane = threadIdx.x % PC_WAVE, wave = threadIdx.x / PC_WAVE;
  const int kk = lane / 16, c16 = lane % 16, G = a.group;
  const int cg = pc_div(run, a.parts_div), part = run - cg * a.n_parts;
  const int c = pc_div(cg, a.heads_div), g = cg - c * a.n_kv_heads;
  const int row0 = tile * 16 * NC;
  const int n_here = min(16 * NC, a.n_rows - row0);
  const long long tok0 = (long long)c * a.fan * a.n_q;      // the cache's first (sequence, t)

  PcSegLens lens;
  lens.seg_len = a.rows.len; lens.per_head = a.rows.len_per_head; lens.n_seg = a.rows.n_seg;
  lens.n_kv_heads = a.n_kv_heads; lens.k_t = a.rows.cap; lens.b = c; lens.g = g;
  struct Cursor { PcBlockCursor at; long long row; int keys; };
  auto place = [&](const PcBlockCursor& at) {
    Cursor x; x.at = at; x.row = 0; x.keys = 0;             // behind the run's end: nothing is read
    if (at.left > 0) {
      x.row = (((long long)c * a.rows.n_seg + at.s) * a.n_kv_heads + g) * a.rows.cap + 32LL * at.blk;
      x.keys = min(32, at.len - 32 * at.blk);
    }
    return x;
  };
  auto next = [&](const Cursor& x) { return place(pc_blocks_next(lens, x.at)); };

  // Rows behind the last valid one are out of the descriptor and arrive as zeros.  V: key i of the lane is 4 kk + i
  // (i < 4) or 16 + 4 kk + i - 4, the keys whose logits the lane holds.
  u32x4 kbuf[2][2][KP];
  vpiece vbuf[2][8];
  float sbuf[2];                                            // key scale of key lane (lanes 0 .. 31), value scale of lane - 32
  const int k_off = Q8 ? c16 * D + 16 * kk : 2 * (c16 * D + 8 * kk);
  const int v_off = Q8 ? 4 * kk * D + VE * c16 : 2 * (4 * kk * D + VE * c16);
  auto issue_loads = [&](int buf, const Cursor& x) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)a.rows.k + x.row * ROW), 0, x.keys * ROW, 0x00020000);
    const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)a.rows.v + x.row * ROW), 0, x.keys * ROW, 0x00020000);
#pragma unroll
    for (int bi = 0; bi < 2; ++bi)
#pragma unroll
      for (int p = 0; p < KP; ++p)
        kbuf[buf][bi][p] = __builtin_amdgcn_raw_buffer_load_b128(kr, k_off, 16 * bi * ROW + 64 * p, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(vpiece) == 16) vbuf[buf][i] = __builtin_amdgcn_raw_buffer_load_b128(vr, v_off, (i < 4 ? i : i + 12) * ROW, 0);
      else if constexpr (sizeof(vpiece) == 8) vbuf[buf][i] = __builtin_amdgcn_raw_buffer_load_b64(vr, v_off, (i < 4 ? i : i + 12) * ROW, 0);
      else vbuf[buf][i] = __builtin_amdgcn_raw_buffer_load_b32(vr, v_off, (i < 4 ? i : i + 12) * ROW, 0);
    }
    if constexpr (Q8)                                        // (every lane reads a row that is there)
      sbuf[buf] = (lane < 32 ? a.rows.k_scale : a.rows.v_scale)[x.row + max(min(lane % 32, x.keys - 1), 0)];
    __builtin_amdgcn_sched_barrier(0);                       // not behind the arithmetic that follows
  };

  const int first_lens = pc_first_lens(lens, lane);
  Cursor cur = place(pc_blocks_begin(lens, part, a.n_parts, a.parts_div, __builtin_amdgcn_readfirstlane(wave), lane, first_lens));
  issue_loads(0, cur);

  // ---- the query rows into LDS, rotated
  {
    constexpr int HALF = D / 2;
    const int i = threadIdx.x % HALF;
    const double theta = a.q_pos ? pc_rope_theta(a.rope, i) : 0.0;
    int at = -1;
    float sn = 0.f, cs = 1.f;
    for (int r = threadIdx.x / HALF; r < 16 * NC; r += SHARED_THREADS / HALF) {
      uint32_t x = 0, y = 0;                                 // rows behind the last one: zeros
      if (r < n_here) {
        const int ft = pc_div(row0 + r, a.group_div), h = row0 + r - ft * G;
        const uint16_t* src = a.q + ((tok0 + ft) * a.n_q_heads + g * G + h) * D + i;
        x = src[0]; y = src[HALF];
        if (a.q_pos) {
          if (ft != at) {
            const int f = pc_div(ft, a.q_div);
            pc_sincos_f32(((double)a.pos0 + a.q_pos[(long long)c * a.fan + f] + (ft - f * a.n_q)) * theta, sn, cs);
            at = ft;
          }
          const float x1 = bf16_bits_to_f32((uint16_t)x), x2 = bf16_bits_to_f32((uint16_t)y);
          x = f32_to_bf16_bits(x1 * cs - x2 * sn);
          y = f32_to_bf16_bits(x2 * cs + x1 * sn);
        }
      }
      sq[r][i] = (uint16_t)x; sq[r][i + HALF] = (uint16_t)y;
    }
  }
  __syncthreads();
  // B operands: column c16; 16-bit rows: k-step ks holds d = 32 ks + 8 kk ..; 8-bit rows: 64 (ks / 2) + 16 kk + 8 (ks % 2) ..
  bf16x8 bq[NC][KSTEPS];
#pragma unroll
  for (int nc = 0; nc < NC; ++nc)
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks)
      bq[nc][ks] = *(const bf16x8*)&sq[16 * nc + c16][Q8 ? 64 * (ks / 2) + 16 * kk + 8 * (ks % 2) : 32 * ks + 8 * kk];
  __syncthreads();

  // the row's last keys that it does not see, of its cache's (own rows)
  int unseen[NC];
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    const int ft = pc_div(min(row0 + 16 * nc + c16, a.n_rows - 1), a.group_div);
    unseen[nc] = a.own ? a.n_q - 1 - ft : 0;                 // (fan = 1: ft = t)
  }
  const int most_unseen = a.own ? a.n_q - 1 : 0;

  float m_run[NC], l_run[NC];
  floatx4 o_acc[NC][VE];                                     // register i of [e]: value VE (4 kk + i) + e of column c16
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    m_run[nc] = -INFINITY; l_run[nc] = 0.f;
#pragma unroll
    for (int e = 0; e < VE; ++e) o_acc[nc][e] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  auto consume = [&](int buf, const Cursor& x) __attribute__((always_inline)) {
    if constexpr (Q8) sm.scale[wave][lane / 32][lane % 32] = sbuf[buf];
    floatx4 acc[NC][2];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc)
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) acc[nc][bi] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int bi = 0; bi < 2; ++bi)
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
        u32x4 ka;
        if constexpr (Q8) {
#pragma unroll
          for (int w = 0; w < 4; ++w) ka[w] = shared_widen(kbuf[buf][bi][ks / 2][2 * (ks % 2) + w / 2], w % 2);
        } else {
          ka = kbuf[buf][bi][ks];
        }
#pragma unroll
        for (int nc = 0; nc < NC; ++nc)
          acc[nc][bi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(bf16x8*)&ka, bq[nc][ks], acc[nc][bi], 0, 0, 0);
      }
    // keys of the block that every row sees; the others are masked column by column
    const int left = x.at.len - 32 * x.at.blk;               // keys from the block's first one on
    const bool masked = left - most_unseen < 32;
    floatx4 ksc[2], vsc[2];
    if constexpr (Q8) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) {
        ksc[bi] = *(const floatx4*)&sm.scale[wave][0][16 * bi + 4 * kk];
        vsc[bi] = *(const floatx4*)&sm.scale[wave][1][16 * bi + 4 * kk];
      }
    }
    u32x4 p[NC];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      float pr[2][4];
#pragma unroll
      for (int bi = 0; bi < 2; ++bi)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          pr[bi][j] = acc[nc][bi][j] * a.scale_log2;
          if constexpr (Q8) pr[bi][j] *= ksc[bi][j];
        }
      if (masked) {
#pragma unroll
        for (int bi = 0; bi < 2; ++bi)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (16 * bi + 4 * kk + j >= left - unseen[nc]) pr[bi][j] = -INFINITY;
      }
      float top = fmaxf(fmaxf(fmaxf(pr[0][0], pr[0][1]), fmaxf(pr[0][2], pr[0][3])),
                        fmaxf(fmaxf(pr[1][0], pr[1][1]), fmaxf(pr[1][2], pr[1][3])));
      const float m_new = fmaxf(m_run[nc], pc_rows_max(top));
      const float ref = m_new == -INFINITY ? 0.f : m_new;    // no key seen yet
      const float alpha = __builtin_amdgcn_exp2f(m_run[nc] - ref);
      m_run[nc] = m_new;
      float sum = 0.f;
#pragma unroll
      for (int bi = 0; bi < 2; ++bi)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          pr[bi][j] = __builtin_amdgcn_exp2f(pr[bi][j] - ref);
          sum += pr[bi][j];
          if constexpr (Q8) pr[bi][j] = pr[bi][j] == 0.f ? 0.f : pr[bi][j] * vsc[bi][j];
        }
      l_run[nc] = l_run[nc] * alpha + sum;
#pragma unroll
      for (int bi = 0; bi < 2; ++bi)
#pragma unroll
        for (int j = 0; j < 4; j += 2) p[nc][2 * bi + j / 2] = pack_bf16x2(pr[bi][j], pr[bi][j + 1]);
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int e = 0; e < VE; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) o_acc[nc][e][i] *= alpha;
      }
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      u32x4 va;                                              // value VE c16 + e of the lane's 8 keys
      if constexpr (Q8) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          va[i] = shared_widen(__builtin_amdgcn_perm(vbuf[buf][2 * i + 1][e / 4], vbuf[buf][2 * i][e / 4],
                                                     e % 4 < 2 ? 0x05010400u : 0x07030602u), e % 2);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          va[i] = __builtin_amdgcn_perm(vbuf[buf][2 * i + 1][e / 2], vbuf[buf][2 * i][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
      }
      // A key that some rows see and others do not may hold infinities or NaN, and 0 times those is NaN: such values
      // count where the probability is not 0, by a product of its own.
      if (masked && most_unseen > 0) {
        u32x4 bad;
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) { bad[i] = shared_bad(va[i]); any |= bad[i]; }
        if (__any(any != 0)) {
          const u32x4 all = va;
#pragma unroll
          for (int sign = 0; sign < 3; ++sign) {             // NaN, +inf, -inf
            u32x4 is;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t lo = all[i] & 0xffffu, hi = all[i] >> 16;
              auto one = [&](uint32_t v) { return sign == 0 ? (v & 0x7fffu) > 0x7f80u : v == (sign == 1 ? 0x7f80u : 0xff80u); };
              is[i] = (one(lo) ? 0x3f80u : 0u) | (one(hi) ? 0x3f800000u : 0u);
            }
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) {
              u32x4 seen;
#pragma unroll
              for (int i = 0; i < 4; ++i) seen[i] = ((p[nc][i] & 0x7fffu) ? 0x3f80u : 0u) | ((p[nc][i] & 0x7fff0000u) ? 0x3f800000u : 0u);
              const floatx4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(bf16x8*)&is, *(bf16x8*)&seen, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (n[i] > 0.f) o_acc[nc][e][i] += sign == 0 ? NAN : (sign == 1 ? INFINITY : -INFINITY);
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) va[i] = all[i] & ~(((bad[i] & 0xffffu) ? 0xffffu : 0u) | ((bad[i] >> 16) ? 0xffff0000u : 0u));
        }
      }
#pragma unroll
      for (int nc = 0; nc < NC; ++nc)
        o_acc[nc][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(bf16x8*)&va, *(bf16x8*)&p[nc], o_acc[nc][e], 0, 0, 0);
    }
  };

  while (cur.at.left > 0) {
    const Cursor nx = next(cur);
    issue_loads(1, nx);
    consume(0, cur);
    cur = next(nx);
    issue_loads(0, cur);
    if (nx.at.left > 0) consume(1, nx);
  }

  // ---- the wavefronts' totals -> the workgroup's partial
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    const float l = pc_rows_sum(l_run[nc]);
    const int col = 16 * nc + c16;
    if (kk == 0) { sm.m[wave][col] = m_run[nc]; sm.l[wave][col] = l; }
    if (col < n_here) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < VE; e += 4)
          *(floatx4*)&sm.o[wave][col][VE * (4 * kk + i) + e] = floatx4{o_acc[nc][e][i], o_acc[nc][e + 1][i], o_acc[nc][e + 2][i], o_acc[nc][e + 3][i]};
    }
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < n_here * (D / 4); idx += SHARED_THREADS) {
    const int r = idx / (D / 4), d4 = idx % (D / 4) * 4;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < SHARED_WAVES; ++w) M = fmaxf(M, sm.m[w][r]);
    floatx4 num = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
#pragma unroll
    for (int w = 0; w < SHARED_WAVES; ++w) {
      if (sm.l[w][r] == 0.f) continue;                       // no key
      const float sc = exp2f(sm.m[w][r] - M);
      const floatx4 y = *(const floatx4*)&sm.o[w][r][d4];
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] += sc * y[e];
      den += sc * sm.l[w][r];
    }
    const int ft = pc_div(row0 + r, a.group_div), h = row0 + r - ft * G;
    const long long row = (long long)(a.part0 + part) * a.part_rows + (tok0 + ft) * a.n_q_heads + g * G + h;
    floatx4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = den == 0.f ? 0.f : num[e] / den;      // (a NaN stays one)
    *(floatx4*)(a.part_o + row * D + d4) = y;
    if (d4 == 0) a.part_lse[row] = den == 0.f ? -INFINITY : (M + log2f(den)) * SHARED_LN2;
  }
}

template <int D, int NC, bool Q8>
__global__ __launch_bounds__(SHARED_THREADS) void shared_rows_kernel(SharedArgs a) {
  extern __shared__ __align__(16) unsigned char lds[];
  // the tiles of a run follow each other on one XCD (number mod 8), whose L2 serves the run's keys to all of them
  const int id = blockIdx.x, oct = pc_div(id / 8, a.tiles_div);
  const int run = oct * 8 + id % 8, tile = id / 8 - oct * a.n_tiles;
  if (run >= a.n_caches * a.n_kv_heads * a.n_parts) return;
  shared_workgroup<D, NC, Q8>(a, run, tile, lds);
}

// ---- the partials of a row, joined: D / 4 threads a row, 4 values each
struct SharedMergeArgs {
  const float* part_o;
  const float* part_lse;
  uint16_t* out;
  float* lse;
  long long n_rows;
  int n_parts, n_q, n_q_heads;
};
template <int D>
__global__ __launch_bounds__(256) void shared_merge_kernel(SharedMergeArgs a) {
  constexpr int TPR = D / 4, U = 8;
  const long long row = ((long long)blockIdx.x * 256 + threadIdx.x) / TPR;      // (b, t, h)
  const int d4 = threadIdx.x % TPR * 4;
  if (row >= a.n_rows) return;
  float m = -INFINITY, den = 0.f;
  floatx4 num = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < a.n_parts; p0 += U) {
    float l[U];
    floatx4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long at = (long long)min(p0 + u, a.n_parts - 1) * a.n_rows + row;
      l[u] = a.part_lse[at];
      x[u] = __builtin_nontemporal_load((const floatx4*)(a.part_o + at * D + d4));
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p0 + u >= a.n_parts) l[u] = -INFINITY;
      top = fmaxf(top, l[u]);
    }
    const float ref = top == -INFINITY ? 0.f : top;
    const float w0 = expf(m - ref);
    m = top; den *= w0;
#pragma unroll
    for (int e = 0; e < 4; ++e) num[e] *= w0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (l[u] == -INFINITY) continue;                       // no key: its values do not count
      const float w = expf(l[u] - ref);
      den += w;
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] += w * x[u][e];
    }
  }
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = den == 0.f ? 0.f : num[e] / den;
  *(uint2*)(a.out + row * D + d4) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
  if (a.lse && d4 == 0) {
    const long long bt = row / a.n_q_heads, b = bt / a.n_q;
    a.lse[(b * a.n_q_heads + row % a.n_q_heads) * a.n_q + bt % a.n_q] = den == 0.f ? -INFINITY : m + logf(den);
  }
}

// ---- host
static int shared_blocks_of(int rows) { return rows <= 16 ? 1 : (rows <= 32 ? 2 : 4); }       // NC
static long long shared_tiles(long long rows, int nc) { return (rows + 16 * nc - 1) / (16 * nc); }

static int shared_parts(long long groups, const PcRows& r) {
  const long long blocks = (long long)r.n_seg * ((r.cap + 31) / 32);
  long long most = blocks / SHARED_WAVES;
  most = most < 1 ? 1 : (most > 64 ? 64 : most);
  int best = 1;
  double least = 0.0;
  for (int p = 1; p <= most; ++p) {
    const long long rounds = (groups * p + 255) / 256;
    const double cost = (double)rounds * ((double)blocks / p + 8.0);
    if (p == 1 || cost < least * 0.98) { least = cost; best = p; }
  }
  return best;
}
PcSharedSplit pc_shared_split(const PcSharedCall& c) {
  const int G = c.n_q_heads / c.n_kv_heads, fan = c.batch / c.n_prefix;
  PcSharedSplit s = {};
  if (c.prefix.n_seg > 0) {
    const long long rows = (long long)fan * c.n_q * G;
    const int nc = shared_blocks_of((int)(rows > 64 ? 64 : rows));
    s.prefix_parts = shared_parts((long long)c.n_prefix * c.n_kv_heads * shared_tiles(rows, nc), c.prefix);
  }
  if (c.tail.n_seg > 0) {
    const long long rows = (long long)c.n_q * G;
    const int nc = shared_blocks_of((int)(rows > 64 ? 64 : rows));
    s.tail_parts = shared_parts((long long)c.batch * c.n_kv_heads * shared_tiles(rows, nc), c.tail);
  }
  return s;
}
// Workgroups of either launch: fewer than a grid dimension's 2^32 threads
bool pc_shared_fits(const PcSharedCall& c) {
  const PcSharedSplit s = pc_shared_split(c);
  const int G = c.n_q_heads / c.n_kv_heads;
  auto fits = [&](long long n_caches, long long rows, int parts) {
    const long long runs = n_caches * c.n_kv_heads * parts + 7;
    return runs * shared_tiles(rows, shared_blocks_of((int)(rows > 64 ? 64 : rows))) < (1LL << 32) / SHARED_THREADS;
  };
  return fits(c.n_prefix, (long long)(c.batch / c.n_prefix) * c.n_q * G, s.prefix_parts) &&
         fits(c.batch, (long long)c.n_q * G, s.tail_parts);
}
size_t pc_shared_ws_bytes(const PcSharedCall& c) {
  const PcSharedSplit s = pc_shared_split(c);
  const size_t rows = (size_t)c.batch * c.n_q * c.n_q_heads * (s.prefix_parts + s.tail_parts);
  return pc_align_up(rows * c.head_dim * 4, 256) + pc_align_up(rows * 4, 256);
}

template <int D, int NC, bool Q8>
static int launch_rows(const SharedArgs& a, hipStream_t st) {
  static std::atomic<uint64_t> raised{0};
  const int lds = (int)sizeof(SharedLds<D, NC>);
  const int rc = pc_raise_dynamic_lds((const void*)shared_rows_kernel<D, NC, Q8>, lds, raised);
  if (rc != PC_OK) return rc;
  const long long runs = ((long long)a.n_caches * a.n_kv_heads * a.n_parts + 7) / 8 * 8;
  hipLaunchKernelGGL((shared_rows_kernel<D, NC, Q8>), dim3((unsigned)(runs * a.n_tiles)), dim3(SHARED_THREADS), lds, st, a);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
template <int D>
static int launch_rows_of(SharedArgs& a, int nc, hipStream_t st) {
  const bool q8 = a.rows.k_scale != nullptr;
  switch (nc) {
    case 1: return q8 ? launch_rows<D, 1, true>(a, st) : launch_rows<D, 1, false>(a, st);
    case 2: return q8 ? launch_rows<D, 2, true>(a, st) : launch_rows<D, 2, false>(a, st);
    default: return q8 ? launch_rows<D, 4, true>(a, st) : launch_rows<D, 4, false>(a, st);
  }
}
static int launch_part(const PcSharedCall& c, const PcRows& rows, int n_caches, int own, int n_parts, int part0, float* part_o,
                       float* part_lse, hipStream_t st) {
  SharedArgs a;
  a.q = (const uint16_t*)c.q; a.q_pos = c.q_pos; a.pos0 = c.pos0; a.rope = pc_rope_factors(c.q_pos ? c.rope_base : 2.0f, c.head_dim);
  a.rows = rows; a.n_caches = n_caches; a.fan = c.batch / n_caches; a.own = own;
  a.n_q = c.n_q; a.n_q_heads = c.n_q_heads; a.n_kv_heads = c.n_kv_heads; a.group = c.n_q_heads / c.n_kv_heads;
  a.n_rows = a.fan * a.n_q * a.group;
  const int nc = shared_blocks_of(a.n_rows);
  a.n_tiles = (int)shared_tiles(a.n_rows, nc);
  a.n_parts = n_parts; a.part0 = part0;
  a.parts_div = pc_div_by(n_parts); a.heads_div = pc_div_by(a.n_kv_heads); a.group_div = pc_div_by(a.group);
  a.q_div = pc_div_by(a.n_q); a.tiles_div = pc_div_by(a.n_tiles);
  a.scale_log2 = c.scale * SHARED_LOG2E;
  a.part_o = part_o; a.part_lse = part_lse; a.part_rows = (long long)c.batch * c.n_q * c.n_q_heads;
  return c.head_dim == 128 ? launch_rows_of<128>(a, nc, st) : launch_rows_of<64>(a, nc, st);
}

int pc_launch_shared_attn(const PcSharedCall& c, void* ws, hipStream_t st) {
  const PcSharedSplit s = pc_shared_split(c);
  const size_t rows = (size_t)c.batch * c.n_q * c.n_q_heads;
  const int parts = s.prefix_parts + s.tail_parts;
  float* part_o = (float*)ws;
  float* part_lse = (float*)((char*)ws + pc_align_up(rows * parts * c.head_dim * 4, 256));
  if (s.prefix_parts > 0) {
    PcProfScope prof(PC_KERNEL_SHARED_PREFIX, st);
    const int rc = launch_part(c, c.prefix, c.n_prefix, 0, s.prefix_parts, 0, part_o, part_lse, st);
    if (rc != PC_OK) return rc;
  }
  if (s.tail_parts > 0) {
    PcProfScope prof(PC_KERNEL_SHARED_TAIL, st);
    const int rc = launch_part(c, c.tail, c.batch, c.tail_own, s.tail_parts, s.prefix_parts, part_o, part_lse, st);
    if (rc != PC_OK) return rc;
  }
  SharedMergeArgs m;
  m.part_o = part_o; m.part_lse = part_lse; m.out = (uint16_t*)c.out; m.lse = c.lse;
  m.n_rows = (long long)rows; m.n_parts = parts; m.n_q = c.n_q; m.n_q_heads = c.n_q_heads;
  const long long blocks = (m.n_rows * (c.head_dim / 4) + 255) / 256;
  PcProfScope prof(PC_KERNEL_SHARED_MERGE, st);
  if (c.head_dim == 128) hipLaunchKernelGGL(shared_merge_kernel<128>, dim3((unsigned)blocks), dim3(256), 0, st, m);
  else hipLaunchKernelGGL(shared_merge_kernel<64>, dim3((unsigned)blocks), dim3(256), 0, st, m);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
