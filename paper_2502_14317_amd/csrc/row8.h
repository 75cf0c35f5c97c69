// A row of keys or values -> E4M3 codes with one fp32 scale (row8.hip has the format).
#pragma once
#include "pc_common.h"
#include "fp8_quotient.h"

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
