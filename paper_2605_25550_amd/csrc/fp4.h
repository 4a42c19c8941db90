// MXFP4 blocks (ditmi.h: dit_quantize_fp4): e2m1 codes and the power of two that 32 of them share.
#pragma once
#include "common.h"

namespace ditmi {

// Bits of the largest magnitude: NaN and infinities compare above every finite value.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Stored scale of a block whose largest magnitude has these bits: the least e >= -127 with
// amax / 2^e < 7, plus 127.  amax = 1.f * 2^(E - 127) is below 7 * 2^e = 1.75 * 2^(e + 2) for e = E - 129,
// or, from 1.75 on, for the next e: the sum carries into the exponent exactly then.
__device__ __forceinline__ uint32_t f4_scale(uint32_t amax) {
  const int e = (int)((amax + 0x200000u) >> 23) - 2;
  return amax >= 0x7F800000u ? 255u : (uint32_t)max(e, 0);
}
// The power of two of a stored scale (255: not a number).
__device__ __forceinline__ float f4_scale_value(uint32_t s) {
  return __uint_as_float(s == 255u ? 0x7FC00000u : s == 0u ? 0x00400000u : s << 23);
}

// Eight values over 2^(s - 127) as codes, the first in the lowest four bits: to nearest, ties to the
// even code; a block that is not a number has codes 0.
__device__ __forceinline__ uint32_t pack_f4x8(const float (&v)[8], uint32_t s) {
  const float sc = f4_scale_value(s);
  uint32_t w = 0u;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], sc, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], sc, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], sc, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], sc, 3);
  return s == 255u ? 0u : w;
}

// The values of eight codes times sc.
__device__ __forceinline__ void unpack_f4x8(uint32_t w, float sc, float (&v)[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 3);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
}
// max over the four lanes of a quad
__device__ __forceinline__ uint32_t max_quad(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, false));
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, false));
}

// Scales lie in panels of 256 columns, [ceil(cols / 256)][rows][8]: what a tile of a product needs of
// a panel is contiguous.
__host__ __device__ __forceinline__ long f4_scale_at(long rows, long row, int block) {
  return ((block >> 3) * rows + row) * 8 + (block & 7);
}

}  // namespace ditmi
