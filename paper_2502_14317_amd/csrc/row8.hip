// Keys and values kept in 8 bits a value with one fp32 scale a row, rounded as they are written:
//   scale = max_d |x_d| / 448 (1 where that is 0; never below 2^-126, so that the quotient stays a normal one),
//   code  = E4M3(x / scale), round to nearest, ties to the even code;
// a row that holds an infinity or a NaN gets the code of NaN throughout (scale 1), so it shows and stays a row's matter.
// Both directions are bound by memory: 3 bytes a value and 4 a row move, nothing is read twice.  Measured: 256 x 2048 rows of
// 128 values written in 68 us (5.9 TB/s; 16 lanes a row with 8 values each, 82 us with 4-byte stores of 32 lanes), read in 68 us;
// 16 rows of 8 heads in 7.5 us, a launch's.
#include "serve.h"
#include "fp8_quotient.h"

#define ROW8_THREADS 256
#define ROW8_MAX 448.0f

// A row is 16 lanes' of D / 16 consecutive values each.  Maximum over them, in all of them: exchanges within quads, then
// of quads and of halves mirrored.
template <int CTRL>
__device__ __forceinline__ uint32_t row8_from(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t row8_max16(uint32_t x) {
  x = max(x, row8_from<0xb1>(x));        // quad_perm: 1 0 3 2
  x = max(x, row8_from<0x4e>(x));        // quad_perm: 2 3 0 1
  x = max(x, row8_from<0x141>(x));       // row_half_mirror
  return max(x, row8_from<0x140>(x));    // row_mirror
}

// VE values of a row in a lane -> VE code bytes; the row's scale in every lane
template <int VE>
__device__ __forceinline__ void row8_encode(const float (&x)[VE], uint32_t (&code)[VE / 4], float& scale) {
  uint32_t bits = 0;                     // of the largest magnitude: infinities and NaN are above every number
#pragma unroll
  for (int e = 0; e < VE; ++e) bits = max(bits, __float_as_uint(x[e]) & 0x7fffffffu);
  bits = row8_max16(bits);
  const bool nan = bits >= 0x7f800000u;
  const float top = __uint_as_float(bits);
  scale = bits > 0 && !nan ? fmaxf(top / ROW8_MAX, 0x1p-126f) : 1.0f;
  const float inv = 1.0f / scale;
  const bool fast = scale > 0x1p-60f && scale < 0x1p60f;     // the quotient by one reciprocal a row, exact there
  float y[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) y[e] = pc_quotient_by_reciprocal(x[e], scale, inv);
  if (!fast) {
#pragma unroll
    for (int e = 0; e < VE; ++e) y[e] = x[e] / scale;
  }
#pragma unroll
  for (int e = 0; e < VE; e += 4) {
    uint32_t w = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(y[e], -ROW8_MAX, ROW8_MAX),
                                                 __builtin_amdgcn_fmed3f(y[e + 1], -ROW8_MAX, ROW8_MAX), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(y[e + 2], -ROW8_MAX, ROW8_MAX),
                                        __builtin_amdgcn_fmed3f(y[e + 3], -ROW8_MAX, ROW8_MAX), w, true);
    code[e / 4] = nan ? 0x7f7f7f7fu : w;
  }
}

struct Row8AppendArgs {
  const uint16_t* k_new;   // [B, n_new, H_kv, D]
  const uint16_t* v_new;
  const int32_t* pos;      // [B] or nullptr
  PcRope rope;
  int pos0, batch, n_new, cap, n_kv_heads;
  int n_rows;              // B n_new H_kv
  PcDiv heads_div, new_div;
  uint8_t* k8;             // [B, H_kv, cap, D]
  uint8_t* v8;
  float* k_scale;          // [B, H_kv, cap]
  float* v_scale;
  const int32_t* len_in;   // [B] or nullptr (= 0)
  int32_t* len_out;        // [B] or nullptr
};

template <int D>
__global__ __launch_bounds__(ROW8_THREADS) void append_row8_kernel(Row8AppendArgs a) {
  constexpr int VE = D / 16;
  typedef uint32_t in_t __attribute__((ext_vector_type(VE / 2)));
  typedef uint32_t out_t __attribute__((ext_vector_type(VE / 4)));
  const int m = threadIdx.x % 16;
  const uint32_t bid = blockIdx.y * gridDim.x + blockIdx.x;
  const long long it = (long long)bid * (ROW8_THREADS / 16) + threadIdx.x / 16;
  if (bid == 0 && a.len_out)
    for (int b = threadIdx.x; b < a.batch; b += ROW8_THREADS) {
      const int len = a.len_in ? min(max(a.len_in[b], 0), a.cap) : 0;
      a.len_out[b] = len + min(a.n_new, a.cap - len);
    }
  if (it >= a.n_rows) return;
  const in_t kx = __builtin_nontemporal_load((const in_t*)(a.k_new + it * D + VE * m));
  const in_t vx = __builtin_nontemporal_load((const in_t*)(a.v_new + it * D + VE * m));
  const int bt = pc_div((int)it, a.heads_div), g = (int)it - bt * a.n_kv_heads;
  const int b = pc_div(bt, a.new_div), t = bt - b * a.n_new;
  const int len = a.len_in ? min(max(a.len_in[b], 0), a.cap) : 0;
  if (t >= a.cap - len) return;                             // no room left
  const long long row = ((long long)b * a.n_kv_heads + g) * a.cap + len + t;
  float x[VE], scale;
  uint32_t code[VE / 4];
#pragma unroll
  for (int e = 0; e < VE; e += 2) { x[e] = bf16_lo_to_f32(kx[e / 2]); x[e + 1] = bf16_hi_to_f32(kx[e / 2]); }
  if (a.pos) {                                              // rounded once, to the code: the rotation stays in 32 bits
    // lane m turns its values with lane m ^ 8's; each computes half of their common angles
    const double at = (double)a.pos0 + a.pos[b] + t;
    float sn[VE], cs[VE];
    const bool upper = m >= 8;
#pragma unroll
    for (int e = 0; e < VE / 2; ++e) {
      float s, c;
      pc_sincos_f32(at * pc_rope_theta(a.rope, VE * (m % 8) + e + (upper ? VE / 2 : 0)), s, c);
      const float s2 = __uint_as_float(row8_from<0x128>(__float_as_uint(s)));        // row_ror:8
      const float c2 = __uint_as_float(row8_from<0x128>(__float_as_uint(c)));
      sn[e] = upper ? s2 : s; cs[e] = upper ? c2 : c;
      sn[e + VE / 2] = upper ? s : s2; cs[e + VE / 2] = upper ? c : c2;
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float y = __uint_as_float(row8_from<0x128>(__float_as_uint(x[e])));
      sn[e] = upper ? sn[e] : -sn[e];
      x[e] = x[e] * cs[e] + y * sn[e];
    }
  }
  row8_encode<VE>(x, code, scale);
  out_t w;
#pragma unroll
  for (int e = 0; e < VE / 4; ++e) w[e] = code[e];
  __builtin_nontemporal_store(w, (out_t*)(a.k8 + row * D + VE * m));
  if (m == 0) a.k_scale[row] = scale;
#pragma unroll
  for (int e = 0; e < VE; e += 2) { x[e] = bf16_lo_to_f32(vx[e / 2]); x[e + 1] = bf16_hi_to_f32(vx[e / 2]); }
  row8_encode<VE>(x, code, scale);
#pragma unroll
  for (int e = 0; e < VE / 4; ++e) w[e] = code[e];
  __builtin_nontemporal_store(w, (out_t*)(a.v8 + row * D + VE * m));
  if (m == 0) a.v_scale[row] = scale;
}

int pc_launch_append_row8(const void* k_new, const void* v_new, const int32_t* pos, int pos0, float base, int batch, int n_new,
                          int cap, int n_kv_heads, int head_dim, void* k8, void* v8, float* k_scale, float* v_scale,
                          const int32_t* len_in, int32_t* len_out, hipStream_t st) {
  Row8AppendArgs a;
  a.k_new = (const uint16_t*)k_new; a.v_new = (const uint16_t*)v_new; a.pos = pos; a.pos0 = pos0;
  a.rope = pc_rope_factors(pos ? base : 2.0f, head_dim);
  a.batch = batch; a.n_new = n_new; a.cap = cap; a.n_kv_heads = n_kv_heads;
  a.n_rows = batch * n_new * n_kv_heads;                    // (fewer than 2^31)
  a.heads_div = pc_div_by(n_kv_heads); a.new_div = pc_div_by(n_new);
  a.k8 = (uint8_t*)k8; a.v8 = (uint8_t*)v8; a.k_scale = k_scale; a.v_scale = v_scale;
  a.len_in = len_in; a.len_out = len_out;
  const int rows = a.n_rows > 0 ? a.n_rows : 1;       // (no rows: the lengths alone)
  const long long blocks = ((long long)rows + ROW8_THREADS / 16 - 1) / (ROW8_THREADS / 16);
  PcProfScope prof(PC_KERNEL_ROW8_APPEND, st);
  const dim3 grid = pc_grid_2d(blocks), block(ROW8_THREADS);
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a); };
  head_dim == 128 ? run(append_row8_kernel<128>) : run(append_row8_kernel<64>);
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
  int n_rows;              // B H_kv cap
  PcDiv cap_div, heads_div;
  uint16_t* k;             // [B, H_kv, cap, D]
  uint16_t* v;
};

// Beyond half of the last-level cache (256 MB) the rows go past it; smaller ones stay there for whoever reads them next.  us,
// through the cache / past it, rows of 128 values: 48 MB moved 10.0 / 10.5, 144 MB 30.9 / 27.5, 384 MB 70.9 / 65.5; with a
// third of the rows beyond the lengths (sizes as if full): 96 MB 12.9 / 14.3, 192 MB 28.4 / 26.0.
static bool row8_stream(long long rows, int head_dim) { return rows * head_dim * 6 > (128LL << 20); }
template <bool STREAM, class T>
__device__ __forceinline__ T row8_load(const T* p) { return STREAM ? __builtin_nontemporal_load(p) : *p; }
template <bool STREAM, class T>
__device__ __forceinline__ void row8_store(T* p, T x) {
  if (STREAM) __builtin_nontemporal_store(x, p);
  else *p = x;
}

// D / 8 lanes a row, 8 codes a lane; value = code * scale in fp32, rounded to bf16 once
__device__ __forceinline__ u32x4 row8_values(u32x2 c, float s) {
  u32x4 y;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const pc_f32x2 p = __builtin_amdgcn_cvt_pk_f32_fp8(c[w], false), q = __builtin_amdgcn_cvt_pk_f32_fp8(c[w], true);
    y[2 * w] = pack_bf16x2(p[0] * s, p[1] * s);
    y[2 * w + 1] = pack_bf16x2(q[0] * s, q[1] * s);
  }
  return y;
}
template <int D, bool STREAM>
__global__ __launch_bounds__(ROW8_THREADS) void read_row8_kernel(Row8ReadArgs a) {
  constexpr int TPR = D / 8;
  const uint32_t bid = blockIdx.y * gridDim.x + blockIdx.x;
  const long long row = (long long)bid * (ROW8_THREADS / TPR) + threadIdx.x / TPR;
  if (row >= a.n_rows) return;
  if (a.len) {
    const int bg = pc_div((int)row, a.cap_div);
    if ((int)row - bg * a.cap >= a.len[pc_div(bg, a.heads_div)]) return;
  }
  const long long at = row * D + threadIdx.x % TPR * 8;
  const u32x2 k = row8_load<STREAM>((const u32x2*)(a.k8 + at)), v = row8_load<STREAM>((const u32x2*)(a.v8 + at));
  const float ks = a.k_scale[row], vs = a.v_scale[row];
  row8_store<STREAM>((u32x4*)(a.k + at), row8_values(k, ks));
  row8_store<STREAM>((u32x4*)(a.v + at), row8_values(v, vs));
}

int pc_launch_read_row8(const void* k8, const void* v8, const float* k_scale, const float* v_scale, const int32_t* len,
                        int batch, int cap, int n_kv_heads, int head_dim, void* k, void* v, hipStream_t st) {
  Row8ReadArgs a;
  a.k8 = (const uint8_t*)k8; a.v8 = (const uint8_t*)v8; a.k_scale = k_scale; a.v_scale = v_scale; a.len = len;
  a.cap = cap; a.n_kv_heads = n_kv_heads; a.n_rows = batch * n_kv_heads * cap;      // (fewer than 2^31)
  a.cap_div = pc_div_by(cap); a.heads_div = pc_div_by(n_kv_heads);
  a.k = (uint16_t*)k; a.v = (uint16_t*)v;
  const int rows = ROW8_THREADS / (head_dim / 8);
  PcProfScope prof(PC_KERNEL_ROW8_READ, st);
  const dim3 grid = pc_grid_2d(((long long)a.n_rows + rows - 1) / rows), block(ROW8_THREADS);
  const bool stream = row8_stream(a.n_rows, head_dim);
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a); };
  if (head_dim == 128) stream ? run(read_row8_kernel<128, true>) : run(read_row8_kernel<128, false>);
  else stream ? run(read_row8_kernel<64, true>) : run(read_row8_kernel<64, false>);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
