// Keys and values into the pages of their sequences: keys rotated on the way at their node's depth, both rounded once as they
// are written (bf16, or E4M3 with a scale a row).  A row is 16 lanes' of D / 16 consecutive values each; lane m turns its
// values with lane m ^ 8's, and each computes half of their common angles.
// A token's angles are its KV heads' alike: with many rows 16 lanes take up to 8 heads of a token one after the other (each head with
// its own angles, whose 64-bit arithmetic was the bound); four tokens of a wavefront lie behind each other in a page.  us for 8 x 8192
// tokens of 8 heads, 1 / 2 / 4 / 8 heads one after the other:
//   128 values to 8 bits  106 / 88 / 88 / 88, the same input again and again 102 / 79 / 72 / 73      64 values to 8 bits  72 / 53 / 46 / 44
//   128 values to 16 bits 112 / 108 / 109 / 110 (95 / 81 / 81 / 81)
// Bound by memory for prompts (inputs that change: 87 us = 4.7 TB/s, to 16 bits 110 us = 4.9, a large copy 5.1), by a launch's latency for
// a step.  Stores past the caches: 81 us instead of 88 and 106 instead of 111, but with inputs from the caches 80 instead of 73 and 105
// instead of 81, and 45 instead of 43 with 64 values.
#include "paged.h"
#include "row8.h"
#include "serve.h"

#define APPEND_THREADS 256
#define APPEND_ROWS (APPEND_THREADS / 16)

struct AppendArgs {
  PcPagedAppend c;
  PcRope rope;
  int chunks, heads;       // workgroups a sequence, KV heads of a token that 16 lanes take one after the other
  PcDiv chunks_div, new_div;
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
  const int part = pc_div(it, x.new_div), t = it - part * c.n_new, g0 = part * x.heads, g1 = min(g0 + x.heads, c.n_kv_heads);
  const bool mine = g0 < c.n_kv_heads && t < n_rows;
  const long long src = b * c.batch_stride + t * c.row_stride + VE * m;
  const auto load = [&](const uint16_t* from, int g) { return __builtin_nontemporal_load((const in_t*)(from + src + g * c.head_stride)); };
  in_t kx = {}, vx = {};
  if (mine) { kx = load(c.k_new, g0); vx = load(c.v_new, g0); }
  int depth = t;
  if (c.parent) {                                           // (every lane: the exchange needs all)
    const int own = __popcll(pc_tree_above(c.parent, b, c.n_new, lane)) - 1;
    depth = __shfl(own, min(t, PC_TREE_NODES - 1));
  }
  const long long row0 = mine ? pc_page_row(c.pages, b, (long long)len + t, 0, c.n_kv_heads) : -1;
  if (row0 < 0) return;                                     // (16 lanes as one)
  float sn[VE], cs[VE];
  if (c.pos) {
    const double at = (double)c.pos0 + c.pos[b] + depth;
    const bool upper = m >= 8;
#pragma unroll
    for (int e = 0; e < VE / 2; ++e) {
      float s, o;
      pc_sincos_f32(at * pc_rope_theta(x.rope, VE * (m % 8) + e + (upper ? VE / 2 : 0)), s, o);
      const float s2 = __uint_as_float(row8_from<0x128>(__float_as_uint(s)));        // row_ror:8
      const float o2 = __uint_as_float(row8_from<0x128>(__float_as_uint(o)));
      sn[e] = upper ? s2 : -s; cs[e] = upper ? o2 : o;
      sn[e + VE / 2] = upper ? s : -s2; cs[e + VE / 2] = upper ? o : o2;
    }
  }
  for (int g = g0; g < g1; ++g) {
    const in_t k0 = kx, v0 = vx;
    if (g + 1 < g1) { kx = load(c.k_new, g + 1); vx = load(c.v_new, g + 1); }
    const long long row = row0 + ((long long)g << c.pages.shift);
    float y[VE];
#pragma unroll
    for (int e = 0; e < VE; e += 2) { y[e] = bf16_lo_to_f32(k0[e / 2]); y[e + 1] = bf16_hi_to_f32(k0[e / 2]); }
    if (c.pos) {
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float z = __uint_as_float(row8_from<0x128>(__float_as_uint(y[e])));
        y[e] = y[e] * cs[e] + z * sn[e];
      }
    }
    if constexpr (!Q8) {
      in_t w;
#pragma unroll
      for (int e = 0; e < VE; e += 2) w[e / 2] = pack_bf16x2(y[e], y[e + 1]);
      if (!c.pos) w = k0;                                   // (a NaN keeps its bits)
      *(in_t*)((uint16_t*)c.pages.k + row * D + VE * m) = w;
      *(in_t*)((uint16_t*)c.pages.v + row * D + VE * m) = v0;
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
      for (int e = 0; e < VE; e += 2) { y[e] = bf16_lo_to_f32(v0[e / 2]); y[e + 1] = bf16_hi_to_f32(v0[e / 2]); }
      row8_encode<VE>(y, code, scale);
#pragma unroll
      for (int e = 0; e < VE / 4; ++e) w[e] = code[e];
      *(code_t*)((uint8_t*)c.pages.v + row * D + VE * m) = w;
      if (m == 0) c.pages.v_scale[row] = scale;
    }
  }
}

// As many heads as leave some 16384 of 16 lanes
static int append_heads(const PcPagedAppend& c) {
  int heads = 1;
  while (heads < 8 && heads < c.n_kv_heads && (long long)c.batch * c.n_new * ((c.n_kv_heads + 2 * heads - 1) / (2 * heads)) >= 16384) heads *= 2;
  return heads;
}
int pc_launch_append_paged(const PcPagedAppend& c, hipStream_t st) {
  AppendArgs x;
  x.c = c;
  x.rope = pc_rope_factors(c.pos ? c.rope_base : 2.0f, c.head_dim);
  x.heads = append_heads(c);
  const long long items = (long long)c.n_new * ((c.n_kv_heads + x.heads - 1) / x.heads);
  x.chunks = items > 0 ? (int)((items + APPEND_ROWS - 1) / APPEND_ROWS) : 1;          // (no rows: the lengths alone)
  x.chunks_div = pc_div_by(x.chunks); x.new_div = pc_div_by(c.n_new);
  PcProfScope prof(PC_KERNEL_PAGED_APPEND, st);
  const dim3 grid = pc_grid_2d((long long)c.batch * x.chunks), block(APPEND_THREADS);
  const bool q8 = c.pages.k_scale != nullptr;
  const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, x); };
  if (c.head_dim == 128) q8 ? run(append_paged_kernel<128, true>) : run(append_paged_kernel<128, false>);
  else q8 ? run(append_paged_kernel<64, true>) : run(append_paged_kernel<64, false>);
  PC_LAUNCH_CHECK();
  return PC_OK;
}
