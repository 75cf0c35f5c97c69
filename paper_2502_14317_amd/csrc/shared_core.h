// What the attentions over many query rows a KV head share (shared_attn.hip: a prefix and tails; tree_attn.hip: pages):
// the products' operands, the softmax of a wavefront's columns, the join of the wavefronts.  The rows of a KV head are the
// columns of S^T = K Q^T, keys 16 bi + 4 kk + j of a 32-key block in lane 16 kk + c16 of column c16.
#pragma once
#include "pc_common.h"

#define SHARED_LOG2E 1.4426950408889634f
#define SHARED_LN2 0.6931471805599453f
#define SHARED_WINDOW 8.0f   // log2 units above a row's largest logit that its reference moves to, when a logit exceeds it

// two of a word's four E4M3 codes -> a packed bf16 pair, exactly
typedef __bf16 shared_bf2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t shared_widen(uint32_t w, bool high) {
  const shared_bf2 a = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
  return *(const uint32_t*)&a;
}
// Operand e of V^T for the lane's 8 keys from their pieces of a row (D / 16 values each)
template <bool Q8, typename Piece>
__device__ __forceinline__ u32x4 shared_value_operand(const Piece (&v)[8], int e) {
  u32x4 a;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (Q8)
      a[i] = shared_widen(__builtin_amdgcn_perm(v[2 * i + 1][e / 4], v[2 * i][e / 4], e % 4 < 2 ? 0x05010400u : 0x07030602u), e % 2);
    else
      a[i] = __builtin_amdgcn_perm(v[2 * i + 1][e / 2], v[2 * i][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
  }
  return a;
}

// KB blocks of 32 keys for NC blocks of columns: logits (lane: column c16, keys 16 bi + 4 kk + j of a block) ->
// probabilities as the B operand of the second product, relative to the column's reference, which moves only when a
// logit exceeds it, and then to the window above that logit: everything before is worth exp2(the move) of what it was.  So a
// probability is never above 1, and sums of values times probabilities stay inside fp32 wherever those relative to the row's
// maximum do.
// hidden(nc, b, bi, j): is key 16 bi + 4 kk + j of block b out of column nc's sight?  Asked only where `masked`, and without a
// branch of its own: the compiler has lost the assignment behind one with several outcomes.
// ALL: no probability is 0 because its key is not there (0 times a scale that is not finite stays out then).
struct SharedScales { floatx4 k[2], v[2]; };
template <int NC, int KB, int VE, bool Q8, bool ALL = false, typename Scales, typename Hidden>
__device__ __forceinline__ void shared_softmax(floatx4 (&s)[NC][KB][2], const Scales (&sc)[KB], bool masked, const Hidden& hidden,
                                               float scale_log2, float (&ref)[NC], float (&sub)[NC],
                                               float (&l)[NC], floatx4 (&o)[NC][VE], u32x4 (&p)[NC][KB]) {
  if constexpr (Q8) {
#pragma unroll
    for (int nc = 0; nc < NC; ++nc)
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int bi = 0; bi < 2; ++bi)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[nc][b][bi][j] *= sc[b].k[bi][j];
  }
  if (masked) {
    asm volatile("");                                        // (a branch: as selects the masks would be everybody's)
#pragma unroll
    for (int nc = 0; nc < NC; ++nc)
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int bi = 0; bi < 2; ++bi)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (hidden(nc, b, bi, j)) s[nc][b][bi][j] = -INFINITY;
  }
  float top[NC];
  bool beyond = false;
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    top[nc] = -INFINITY;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int bi = 0; bi < 2; ++bi)
        top[nc] = fmaxf(fmaxf(top[nc], fmaxf(s[nc][b][bi][0], s[nc][b][bi][1])), fmaxf(s[nc][b][bi][2], s[nc][b][bi][3]));
    beyond |= top[nc] * scale_log2 > ref[nc];
  }
  if (__any(beyond)) {
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      const float most = pc_rows_max(top[nc]) * scale_log2;
      const float m = most > ref[nc] ? most + SHARED_WINDOW : ref[nc];      // (a column's results do not hang on the others')
      sub[nc] = m == -INFINITY ? 0.f : m;                    // no key seen yet
      const float alpha = __builtin_amdgcn_exp2f(ref[nc] - sub[nc]);
      ref[nc] = m;
      l[nc] *= alpha;
#pragma unroll
      for (int e = 0; e < VE; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[nc][e][i] *= alpha;
    }
  }
#pragma unroll
  for (int nc = 0; nc < NC; ++nc)
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int bi = 0; bi < 2; ++bi) {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j] = __builtin_amdgcn_exp2f(fmaf(s[nc][b][bi][j], scale_log2, -sub[nc]));
          l[nc] += x[j];
        }
        if constexpr (Q8) {
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = !ALL && x[j] == 0.f ? 0.f : x[j] * sc[b].v[bi][j];
        }
        p[nc][b][2 * bi] = pack_bf16x2(x[0], x[1]);
        p[nc][b][2 * bi + 1] = pack_bf16x2(x[2], x[3]);
      }
}

// A key that some rows see and others do not may hold values that are infinite or NaN, and 0 times those is NaN: they
// are taken out of the operand and count where the probability is not 0, by products of their own.
template <int NC, int KB, int VE>
__device__ __forceinline__ void shared_values_not_finite(u32x4& va, const u32x4 (&p)[NC][KB], int b, floatx4 (&o)[NC][VE], int e) {
  u32x4 bad;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bad[i] = ((va[i] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((va[i] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
    any |= bad[i];
  }
  if (!__any(any != 0)) return;
#pragma unroll
  for (int kind = 0; kind < 3; ++kind) {                     // NaN, +inf, -inf
    u32x4 is;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      auto one = [&](uint32_t v) { return kind == 0 ? (v & 0x7fffu) > 0x7f80u : v == (kind == 1 ? 0x7f80u : 0xff80u); };
      is[i] = (one(va[i] & 0xffffu) ? 0x3f80u : 0u) | (one(va[i] >> 16) ? 0x3f800000u : 0u);
    }
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      u32x4 seen;
#pragma unroll
      for (int i = 0; i < 4; ++i) seen[i] = ((p[nc][b][i] & 0x7fffu) ? 0x3f80u : 0u) | ((p[nc][b][i] & 0x7fff0000u) ? 0x3f800000u : 0u);
      const floatx4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(bf16x8*)&is, *(bf16x8*)&seen, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n[i] > 0.f) o[nc][e][i] += kind == 0 ? NAN : (kind == 1 ? INFINITY : -INFINITY);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) va[i] &= ~bad[i];
}

// O^T += V^T P^T, operand e of V^T of block b from `operand`
template <int NC, int KB, int VE, bool OWN, typename Operand>
__device__ __forceinline__ void shared_values(const Operand& operand, bool own_rows, const u32x4 (&p)[NC][KB], floatx4 (&o)[NC][VE]) {
  if constexpr (OWN) {
    if (own_rows) {                                          // (a path of its own: the loop below stays free of conditions)
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          u32x4 va = operand(b, e);
          shared_values_not_finite<NC, KB, VE>(va, p, b, o, e);
#pragma unroll
          for (int nc = 0; nc < NC; ++nc)
            o[nc][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)&va, *(const bf16x8*)&p[nc][b], o[nc][e], 0, 0, 0);
        }
      return;
    }
  }
#pragma unroll
  for (int b = 0; b < KB; ++b)
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const u32x4 va = operand(b, e);
#pragma unroll
      for (int nc = 0; nc < NC; ++nc)
        o[nc][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)&va, *(const bf16x8*)&p[nc][b], o[nc][e], 0, 0, 0);
    }
}

// A wavefront's state of 16 NC columns: register i of o[][e] is value VE (4 kk + i) + e of the lane's column c16
template <int D, int NC>
struct SharedColumns {
  static constexpr int KSTEPS = D / 32, VE = D / 16;
  bf16x8 q[2][NC][KSTEPS];              // B operands, values shared_query_at ..; [1]: second parts of rotated rows
  float ref[NC], sub[NC], l[NC];
  floatx4 o[NC][VE];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
      ref[nc] = -INFINITY; sub[nc] = 0.f; l[nc] = 0.f;
#pragma unroll
      for (int e = 0; e < VE; ++e) o[nc][e] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  }
};

// ROWS query rows of a workgroup of WAVES wavefronts: wavefront w has columns 16 NC (w % WR) .. and run w / WR of the
// workgroup's WK = WAVES / WR runs of keys.
template <int D, int NC, int WR, int WAVES>
struct SharedFewLds {
  static constexpr int ROWS = 16 * NC * WR, WK = WAVES / WR;
  union {
    float o[WK][ROWS][D + 4];           // (a row's stride is 4 banks on: 16 lanes write 16 rows at a time)
    uint16_t q[2][ROWS][D + 8];         // the rows, and the second parts of rotated ones
  };
  float m[WK][ROWS], l[WK][ROWS];
  float scale[WAVES][2][32];            // the 8-bit rows' scales of a wavefront's block: keys, values
};
// Where a lane's B operand of a k-step starts in a query row, as the walk's keys arrive
__device__ __forceinline__ int shared_query_at(bool q8, int ks, int kk) { return q8 ? 64 * (ks / 2) + 16 * kk + 8 * (ks % 2) : 32 * ks + 8 * kk; }
// Query rows -> the operands of a wavefront's columns
template <int D, int NC, bool Q8>
__device__ __forceinline__ void shared_query_operands(SharedColumns<D, NC>& c, const uint16_t (*hi)[D + 8], const uint16_t (*lo)[D + 8], int col0) {
  const int lane = threadIdx.x % PC_WAVE, kk = lane / 16, c16 = lane % 16;
#pragma unroll
  for (int nc = 0; nc < NC; ++nc)
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      c.q[0][nc][ks] = *(const bf16x8*)&hi[col0 + 16 * nc + c16][shared_query_at(Q8, ks, kk)];
      c.q[1][nc][ks] = *(const bf16x8*)&lo[col0 + 16 * nc + c16][shared_query_at(Q8, ks, kk)];
    }
}
template <int D, int NC, typename Lds>
__device__ __forceinline__ void shared_columns_out(const SharedColumns<D, NC>& c, Lds& sm, int wk, int col0, int n_here) {
  constexpr int VE = D / 16;
  const int lane = threadIdx.x % PC_WAVE, kk = lane / 16, c16 = lane % 16;
#pragma unroll
  for (int nc = 0; nc < NC; ++nc) {
    const float l = pc_rows_sum(c.l[nc]);
    const int col = col0 + 16 * nc + c16;
    if (kk == 0) { sm.m[wk][col] = c.ref[nc]; sm.l[wk][col] = l; }
    if (col < n_here) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < VE; e += 4)
          *(floatx4*)&sm.o[wk][col][VE * (4 * kk + i) + e] = floatx4{c.o[nc][e][i], c.o[nc][e + 1][i], c.o[nc][e + 2][i], c.o[nc][e + 3][i]};
    }
  }
}
// Four values of a row under a maximum in log2 units, joined piece by piece
struct SharedRowSum {
  float m, den;
  floatx4 num;
  __device__ __forceinline__ void clear() { m = -INFINITY; den = 0.f; num = floatx4{0.f, 0.f, 0.f, 0.f}; }
  // a piece that holds `weight` exp2(m2) of the sum and its values times that; none where weight is 0
  __device__ __forceinline__ void add(float m2, float weight, const floatx4& y) {
    if (weight == 0.f) return;
    const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top;
    const float before = __builtin_amdgcn_exp2f(m - base), w = __builtin_amdgcn_exp2f(m2 - base);
    m = top;
    den = den * before + w * weight;
#pragma unroll
    for (int e = 0; e < 4; ++e) num[e] = num[e] * before + w * y[e];
  }
  __device__ __forceinline__ floatx4 mean() const {
    floatx4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = den == 0.f ? 0.f : num[e] / den;      // (a NaN stays one)
    return y;
  }
  __device__ __forceinline__ float lse() const { return den == 0.f ? -INFINITY : (m + log2f(den)) * SHARED_LN2; }
};
