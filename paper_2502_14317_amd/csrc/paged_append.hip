// Keys and values into the pages of their sequences: keys rotated on the way at their node's depth, both rounded once as they
// are written (bf16, or E4M3 with a scale a row).  A row is 16 lanes' of D / 16 consecutive values each; lane m turns its
// values with lane m ^ 8's, and each computes half of their common angles.
// Bound by memory for prompts, by a launch's latency for a step.
#include "paged.h"
#include "row8.h"
#include "serve.h"

#define APPEND_THREADS 256
#define APPEND_ROWS (APPEND_THREADS / 16)

struct AppendArgs {
  PcPagedAppend c;
  PcRope rope;
  int chunks;              // workgroups a sequence
  PcDiv chunks_div, heads_div;
};

template <int D, bool Q8>
__global__ __launch_bounds__(APPEND_THREADS) void append_paged_kernel(AppendArgs x) {
  constexpr int VE = D / 16;
  typedef uint32_t in_t __attribute__((ext_vector_type(VE / 2)));
  typedef uint32_t code_t __attribute__((ext_vector_type(VE / 4)));
  const PcPagedAppend& c = x.c;
  const int lane = threadIdx.x % PC_WAVE, m = threadIdx.x % 16;
  const uint32_t bid = blockIdx.y * gridDim.x + blockIdx.x;
  const int b = pc_div((int)bid, x.chunks_div), chunk = (int)bid - b * x.chunks;
  if (b >= c.batch) return;                                 // (uniform: the grid's last row holds more than there are)
  const int n_rows = pc_tree_rows(c.n_rows, b, c.n_new), len = c.len_in ? max(c.len_in[b], 0) : 0;
  if (chunk == 0 && threadIdx.x == 0 && c.len_out) c.len_out[b] = len + n_rows;
  const int it = chunk * APPEND_ROWS + threadIdx.x / 16;
  const int t = pc_div(it, x.heads_div), g = it - t * c.n_kv_heads;
  int depth = t;
  if (c.parent) {                                           // (every lane: the exchange needs all)
    const int mine = __popcll(pc_tree_above(c.parent, b, c.n_new, lane)) - 1;
    depth = __shfl(mine, min(t, PC_TREE_NODES - 1));
  }
  if (t >= n_rows) return;
  const long long src = b * c.batch_stride + t * c.row_stride + g * c.head_stride + VE * m;
  const in_t kx = __builtin_nontemporal_load((const in_t*)(c.k_new + src));
  const in_t vx = __builtin_nontemporal_load((const in_t*)(c.v_new + src));
  const long long row = pc_page_row(c.pages, b, (long long)len + t, g, c.n_kv_heads);
  if (row < 0) return;                                      // (16 lanes as one)
  float y[VE];
#pragma unroll
  for (int e = 0; e < VE; e += 2) { y[e] = bf16_lo_to_f32(kx[e / 2]); y[e + 1] = bf16_hi_to_f32(kx[e / 2]); }
  if (c.pos) {
    const double at = (double)c.pos0 + c.pos[b] + depth;
    float sn[VE], cs[VE];
    const bool upper = m >= 8;
#pragma unroll
    for (int e = 0; e < VE / 2; ++e) {
      float s, o;
      pc_sincos_f32(at * pc_rope_theta(x.rope, VE * (m % 8) + e + (upper ? VE / 2 : 0)), s, o);
      const float s2 = __uint_as_float(row8_from<0x128>(__float_as_uint(s)));        // row_ror:8
      const float o2 = __uint_as_float(row8_from<0x128>(__float_as_uint(o)));
      sn[e] = upper ? s2 : s; cs[e] = upper ? o2 : o;
      sn[e + VE / 2] = upper ? s : s2; cs[e + VE / 2] = upper ? o : o2;
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float z = __uint_as_float(row8_from<0x128>(__float_as_uint(y[e])));
      sn[e] = upper ? sn[e] : -sn[e];
      y[e] = y[e] * cs[e] + z * sn[e];
    }
  }
  if constexpr (!Q8) {
    in_t w;
#pragma unroll
    for (int e = 0; e < VE; e += 2) w[e / 2] = pack_bf16x2(y[e], y[e + 1]);
    if (!c.pos) w = kx;                                     // (a NaN keeps its bits)
    *(in_t*)((uint16_t*)c.pages.k + row * D + VE * m) = w;
    *(in_t*)((uint16_t*)c.pages.v + row * D + VE * m) = vx;
  } else {
    float scale;
    uint32_t code[VE / 4];
    code_t w;
    row8_encode<VE>(y, code, scale);
#pragma unroll
    for (int e = 0; e < VE / 4; ++e) w[e] = code[e];
    *(code_t*)((uint8_t*)c.pages.k + row * D + VE * m) = w;
    if (m == 0) c.pages.k_scale[row] = scale;
#pragma unroll
    for (int e = 0; e < VE; e += 2) { y[e] = bf16_lo_to_f32(vx[e / 2]); y[e + 1] = bf16_hi_to_f32(vx[e / 2]); }
    row8_encode<VE>(y, code, scale);
#pragma unroll
    for (int e = 0; e < VE / 4; ++e) w[e] = code[e];
    *(code_t*)((uint8_t*)c.pages.v + row * D + VE * m) = w;
    if (m == 0) c.pages.v_scale[row] = scale;
  }
}

int pc_launch_append_paged(const PcPagedAppend& c, hipStream_t st) {
  AppendArgs x;
  x.c = c;
  x.rope = pc_rope_factors(c.pos ? c.rope_base : 2.0f, c.head_dim);
  const long long rows = (long long)c.n_new * c.n_kv_heads;
  x.chunks = rows > 0 ? (int)((rows + APPEND_ROWS - 1) / APPEND_ROWS) : 1;            // (no rows: the lengths alone)
  x.chunks_div = pc_div_by(x.chunks); x.heads_div = pc_div_by(c.n_kv_heads);
  PcProfScope prof(PC_KERNEL_PAGED_APPEND, st);
  const dim3 grid = pc_grid_2d((long long)c.batch * x.chunks), block(APPEND_THREADS);
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, x); };
  const bool q8 = c.pages.k_scale != nullptr;
  if (c.head_dim == 128) q8 ? run(append_paged_kernel<128, true>) : run(append_paged_kernel<128, false>);
  else q8 ? run(append_paged_kernel<64, true>) : run(append_paged_kernel<64, false>);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
