// Keys and values kept in 8 bits a value with one fp32 scale a row, rounded as they are written:
//   scale = max_d |x_d| / 448 (1 where that is 0; never below 2^-126, so that the quotient stays a normal one),
//   code  = E4M3(x / scale), round to nearest, ties to the even code;
// a row that holds an infinity or a NaN gets the code of NaN throughout (scale 1), so it shows and stays a row's matter.
// Both directions are bound by memory: 3 bytes a value and 4 a row move, nothing is read twice.
#include "serve.h"
#include "fp8_quotient.h"

#define ROW8_THREADS 256
#define ROW8_MAX 448.0f

// maximum over 16 neighbouring lanes, in all of them
__device__ __forceinline__ float row8_max16(float x) {
  for (int off = 8; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}

// VE values of a row in a lane, 16 lanes a row -> VE code bytes; the row's scale in every lane
template <int VE>
__device__ __forceinline__ void row8_encode(const float (&x)[VE], uint32_t (&code)[VE / 4], float& scale) {
  float top = 0.f;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    top = fmaxf(top, fabsf(x[e]));
    bad |= !(fabsf(x[e]) < INFINITY);
  }
  top = row8_max16(bad ? INFINITY : top);
  const bool nan = top == INFINITY;
  scale = top > 0.f && !nan ? fmaxf(top / ROW8_MAX, 0x1p-126f) : 1.0f;
  const float inv = 1.0f / scale;
  const bool fast = scale > 0x1p-60f && scale < 0x1p60f;     // the quotient by one reciprocal a row, exact there
  float y[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    y[e] = fast ? pc_quotient_by_reciprocal(x[e], scale, inv) : x[e] / scale;
    y[e] = __builtin_amdgcn_fmed3f(y[e], -ROW8_MAX, ROW8_MAX);
  }
#pragma unroll
  for (int e = 0; e < VE; e += 4) {
    uint32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(y[e], y[e + 1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[e + 2], y[e + 3], w, true);
    code[e / 4] = nan ? 0x7f7f7f7fu : w;
  }
}

struct Row8AppendArgs {
  const uint16_t* k_new;   // [B, n_new, H_kv, D]
  const uint16_t* v_new;
  const int32_t* pos;      // [B] or nullptr
  PcRope rope;
  int pos0, batch, n_new, cap, n_kv_heads;
  long long n_rows;        // B n_new H_kv
  uint8_t* k8;             // [B, H_kv, cap, D]
  uint8_t* v8;
  float* k_scale;          // [B, H_kv, cap]
  float* v_scale;
  const int32_t* len_in;   // [B] or nullptr (= 0)
  int32_t* len_out;        // [B] or nullptr
};

// 16 lanes a row: lane m holds values VE / 2 m .. of both halves, so that a rotation pair (i, i + D / 2) is a lane's own
template <int D>
__global__ __launch_bounds__(ROW8_THREADS) void append_row8_kernel(Row8AppendArgs a) {
  constexpr int HALF = D / 2, VH = HALF / 16;               // values a lane takes of each half
  typedef uint32_t piece __attribute__((ext_vector_type(VH / 2)));
  const int m = threadIdx.x % 16;
  const long long bid = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  const long long it = bid * (ROW8_THREADS / 16) + threadIdx.x / 16;
  if (bid == 0 && a.len_out)
    for (int b = threadIdx.x; b < a.batch; b += ROW8_THREADS) {
      const int len = a.len_in ? min(max(a.len_in[b], 0), a.cap) : 0;
      a.len_out[b] = len + min(a.n_new, a.cap - len);
    }
  if (it >= a.n_rows) return;
  const int g = (int)(it % a.n_kv_heads);
  const long long bt = it / a.n_kv_heads;
  const int t = (int)(bt % a.n_new), b = (int)(bt / a.n_new);
  const int len = a.len_in ? min(max(a.len_in[b], 0), a.cap) : 0;
  if (len + (long long)t >= a.cap) return;                  // no room left
  const long long row = ((long long)b * a.n_kv_heads + g) * a.cap + len + t;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const uint16_t* src = (which ? a.v_new : a.k_new) + it * D + VH * m;
    const piece lo = *(const piece*)src, hi = *(const piece*)(src + HALF);
    float x[2 * VH];
#pragma unroll
    for (int e = 0; e < VH; e += 2) {
      x[e] = bf16_lo_to_f32(lo[e / 2]); x[e + 1] = bf16_hi_to_f32(lo[e / 2]);
      x[VH + e] = bf16_lo_to_f32(hi[e / 2]); x[VH + e + 1] = bf16_hi_to_f32(hi[e / 2]);
    }
    if (which == 0 && a.pos) {                              // rounded once, to the code: the rotation stays in 32 bits
      const double at = (double)a.pos0 + a.pos[b] + t;
#pragma unroll
      for (int e = 0; e < VH; ++e) {
        float sn, cs;
        pc_sincos_f32(at * pc_rope_theta(a.rope, VH * m + e), sn, cs);
        const float p = x[e], q = x[VH + e];
        x[e] = p * cs - q * sn;
        x[VH + e] = q * cs + p * sn;
      }
    }
    uint32_t code[VH / 2];
    float scale;
    row8_encode<2 * VH>(x, code, scale);
    uint8_t* dst = (which ? a.v8 : a.k8) + row * D + VH * m;
    if constexpr (VH == 4) {
      *(uint32_t*)dst = code[0];
      *(uint32_t*)(dst + HALF) = code[1];
    } else {                                                // D = 64: two values of each half
      *(uint16_t*)dst = (uint16_t)code[0];
      *(uint16_t*)(dst + HALF) = (uint16_t)(code[0] >> 16);
    }
    if (m == 0) (which ? a.v_scale : a.k_scale)[row] = scale;
  }
}

int pc_launch_append_row8(const void* k_new, const void* v_new, const int32_t* pos, int pos0, float base, int batch, int n_new,
                          int cap, int n_kv_heads, int head_dim, void* k8, void* v8, float* k_scale, float* v_scale,
                          const int32_t* len_in, int32_t* len_out, hipStream_t st) {
  Row8AppendArgs a;
  a.k_new = (const uint16_t*)k_new; a.v_new = (const uint16_t*)v_new; a.pos = pos; a.pos0 = pos0;
  a.rope = pc_rope_factors(pos ? base : 2.0f, head_dim);
  a.batch = batch; a.n_new = n_new; a.cap = cap; a.n_kv_heads = n_kv_heads;
  a.n_rows = (long long)batch * n_new * n_kv_heads;
  a.k8 = (uint8_t*)k8; a.v8 = (uint8_t*)v8; a.k_scale = k_scale; a.v_scale = v_scale;
  a.len_in = len_in; a.len_out = len_out;
  const long long rows = a.n_rows > 0 ? a.n_rows : 1;       // (no rows: the lengths alone)
  const long long blocks = (rows + ROW8_THREADS / 16 - 1) / (ROW8_THREADS / 16);
  PcProfScope prof(PC_KERNEL_ROW8_APPEND, st);
  const dim3 grid = pc_grid_2d(blocks), block(ROW8_THREADS);
  if (head_dim == 128) hipLaunchKernelGGL(append_row8_kernel<128>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(append_row8_kernel<64>, grid, block, 0, st, a);
  PC_LAUNCH_CHECK();
  return PC_OK;
}

struct Row8ReadArgs {
  const uint8_t* k8;       // [B, H_kv, cap, D]
  const uint8_t* v8;
  const float* k_scale;    // [B, H_kv, cap]
  const float* v_scale;
  const int32_t* len;      // [B] or nullptr
  int cap, n_kv_heads;
  long long n_rows;        // B H_kv cap
  uint16_t* k;             // [B, H_kv, cap, D]
  uint16_t* v;
};

// D / 8 lanes a row, 8 codes a lane; value = code * scale in fp32, rounded to bf16 once
template <int D>
__global__ __launch_bounds__(ROW8_THREADS) void read_row8_kernel(Row8ReadArgs a) {
  constexpr int TPR = D / 8;
  const long long bid = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  const long long row = bid * (ROW8_THREADS / TPR) + threadIdx.x / TPR;
  if (row >= a.n_rows) return;
  const int d0 = threadIdx.x % TPR * 8;
  const long long bg = row / a.cap;
  const int j = (int)(row - bg * a.cap);
  if (a.len && j >= a.len[bg / a.n_kv_heads]) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const u32x2 c = *(const u32x2*)((which ? a.v8 : a.k8) + row * D + d0);
    const float s = (which ? a.v_scale : a.k_scale)[row];
    u32x4 y;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const pc_f32x2 p = __builtin_amdgcn_cvt_pk_f32_fp8(c[w], false), q = __builtin_amdgcn_cvt_pk_f32_fp8(c[w], true);
      y[2 * w] = pack_bf16x2(p[0] * s, p[1] * s);
      y[2 * w + 1] = pack_bf16x2(q[0] * s, q[1] * s);
    }
    *(u32x4*)((which ? a.v : a.k) + row * D + d0) = y;
  }
}

int pc_launch_read_row8(const void* k8, const void* v8, const float* k_scale, const float* v_scale, const int32_t* len,
                        int batch, int cap, int n_kv_heads, int head_dim, void* k, void* v, hipStream_t st) {
  Row8ReadArgs a;
  a.k8 = (const uint8_t*)k8; a.v8 = (const uint8_t*)v8; a.k_scale = k_scale; a.v_scale = v_scale; a.len = len;
  a.cap = cap; a.n_kv_heads = n_kv_heads; a.n_rows = (long long)batch * n_kv_heads * cap;
  a.k = (uint16_t*)k; a.v = (uint16_t*)v;
  const int rows = ROW8_THREADS / (head_dim / 8);
  PcProfScope prof(PC_KERNEL_ROW8_READ, st);
  const dim3 grid = pc_grid_2d((a.n_rows + rows - 1) / rows), block(ROW8_THREADS);
  if (head_dim == 128) hipLaunchKernelGGL(read_row8_kernel<128>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(read_row8_kernel<64>, grid, block, 0, st, a);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
