// Serving many answers over one compressed document: internal declarations of the shared-prefix attention
// (shared_attn.hip), the 8-bit rows (row8.hip) and the draft verification (verify.hip).
#pragma once
#include "pc_common.h"

// sine and cosine of x, 0 <= x < 2^31, in 32 bits: the reduction by multiples of pi / 2 in 64 bits (Cody and Waite: two
// parts, each product exact in the fused multiply-add), then the Taylor polynomials on [-pi / 4, pi / 4], whose first
// omitted terms are below 3e-8 (sine) and 3e-9 (cosine).  For values that are rounded to bf16 or 8 bits next.
__host__ __device__ __forceinline__ void pc_sincos_f32(double x, float& sn, float& cs) {
  const double n = rint(x * 0.63661977236758134308);               // 2 / pi
  const float r = (float)fma(-n, 6.123233995736766e-17, fma(-n, 1.5707963267948966, x));
  const int quadrant = (int)(unsigned)n;
  const float z = r * r;
  float s = 1.0f / 362880.0f;                                      // 1 / 9!
  s = fmaf(s, z, -1.0f / 5040.0f);
  s = fmaf(s, z, 1.0f / 120.0f);
  s = fmaf(s, z, -1.0f / 6.0f);
  s = fmaf(s * z, r, r);
  float c = -1.0f / 3628800.0f;                                    // 1 / 10!
  c = fmaf(c, z, 1.0f / 40320.0f);
  c = fmaf(c, z, -1.0f / 720.0f);
  c = fmaf(c, z, 1.0f / 24.0f);
  c = fmaf(c, z, -0.5f);
  c = fmaf(c, z, 1.0f);
  const float a = quadrant & 1 ? c : s, b = quadrant & 1 ? s : c;
  sn = quadrant & 2 ? -a : a;
  cs = (quadrant + 1) & 2 ? -b : b;
}

// ---- shared-prefix attention
// Rows of keys and values: [n, n_seg, H_kv, cap, D], bf16 or (scales given) E4M3 codes with a scale a row
struct PcRows {
  const void* k;
  const void* v;
  const float* k_scale;    // [n, n_seg, H_kv, cap] or nullptr
  const float* v_scale;
  const int32_t* len;      // [n, n_seg] ([n, n_seg, H_kv] if len_per_head) or nullptr (= cap)
  int len_per_head, n_seg, cap;
};
struct PcSharedCall {
  const void* q;           // [B, n_q, H_q, D]
  const int32_t* q_pos;    // [B] or nullptr
  int pos0;
  float rope_base, scale;
  PcRows prefix, tail;     // n_seg = 0: none
  int tail_own;
  int batch, n_prefix, n_q, n_q_heads, n_kv_heads, head_dim;
  void* out;               // [B, n_q, H_q, D]
  float* lse;              // [B, H_q, n_q] or nullptr
};
// How a call is done: alone, one launch; else the sides' partials (the tails' of up to 16 rows behind the prefix's, in
// their launch) and the merge.  A side: groups (caches x KV heads x tiles) of workgroups, `parts` runs of keys each.
struct PcSharedSide { int body, parts, waves; long long tiles, caches_heads, runs; };      // body 0: no such side; waves: of a run behind the prefix's
struct PcSharedPlan { PcSharedSide prefix, tail; bool alone; };
PcSharedPlan pc_shared_plan(const PcSharedCall& c);
void pc_shared_plan_info(const PcSharedCall& c, const PcSharedPlan& p, pc_shared_attn_plan_info& info);
bool pc_shared_fits(const PcSharedCall& c, const PcSharedPlan& p);
size_t pc_shared_ws_bytes(const PcSharedCall& c, const PcSharedPlan& p);
int pc_launch_shared_attn(const PcSharedCall& c, const PcSharedPlan& p, void* ws, hipStream_t st);

// ---- 8-bit rows
int pc_launch_append_row8(const void* k_new, const void* v_new, const int32_t* pos, int pos0, float base, int batch, int n_new,
                          int cap, int n_kv_heads, int head_dim, void* k8, void* v8, float* k_scale, float* v_scale,
                          const int32_t* len_in, int32_t* len_out, hipStream_t st);
int pc_launch_read_row8(const void* k8, const void* v8, const float* k_scale, const float* v_scale, const int32_t* len,
                        int batch, int cap, int n_kv_heads, int head_dim, void* k, void* v, hipStream_t st);

// ---- draft verification
struct PcVerifyCall {
  const int32_t* draft;    // [B, n_draft]
  const float* draft_prob; // [B, n_draft, V] or nullptr (a point mass on each drafted token)
  const float* target_prob;// [B, n_draft + 1, V]
  const float* u;          // [B, n_draft]
  const float* noise;      // [B, V]
  const int32_t* draft_len;// [B] or nullptr (= n_draft)
  int batch, n_draft, vocab;
  int32_t* tokens;         // [B, n_draft + 1]
  int32_t* count;          // [B]
  const int32_t* len_in;   // [B] or nullptr
  int32_t* len_out;
};
size_t pc_verify_ws_bytes(int batch, int vocab);
int pc_launch_verify(const PcVerifyCall& c, void* ws, hipStream_t st);
