// e4m3 codes and block scales (ditmi.h: dit_quantize_fp8), and 8-element loads.
#pragma once
#include "common.h"

namespace ditmi {

constexpr float F8_MAX = 448.f, F8_TINY = 1.17549435e-38f;  // 2^-126: the least scale

__device__ __forceinline__ float f8_scale(float amax) { return fmaxf(amax * (1.0f / F8_MAX), F8_TINY); }
// Four values to e4m3 codes.  The conversion makes NaN of values from 464 on;
// x / scale exceeds 448 by a rounding at most.
__device__ __forceinline__ uint32_t pack_f8x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Eight values that are read once: streamed past the caches.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    const f32x4 a = __builtin_nontemporal_load((const f32x4*)p), b = __builtin_nontemporal_load((const f32x4*)(p + 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  } else {
    const u32x4 w = __builtin_nontemporal_load((const u32x4*)p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ float amax8(const float (&v)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
  return m;
}
// max over the 16 lanes of a row group
__device__ __forceinline__ float max16(float m) {
  m = fmaxf(m, dpp_move<0xB1>(m));
  m = fmaxf(m, dpp_move<0x4E>(m));
  m = fmaxf(m, dpp_move<0x141>(m));
  return fmaxf(m, dpp_move<0x140>(m));
}
__device__ __forceinline__ u32x2 pack_f8x8(const float (&v)[8], float inv) {
  return u32x2{pack_f8x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
               pack_f8x4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
}

}  // namespace ditmi
