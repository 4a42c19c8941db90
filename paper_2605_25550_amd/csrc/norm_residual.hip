// The norms around a sub-layer with its gate and residual, in one pass
// (ditmi.h: dit_norm_residual): a row of x and y is read once and held in
// registers while its statistics are taken (mean, then deviations from it, in
// fp32), the residual is updated, and the new row is normalised in turn.
//
// Bound by memory: 17550 x 3072 (bf16 y, e4m3 h) 121 us, 4.9 TB/s, where a plain
// copy of 1 to 4 GiB reaches 5.0 to 5.2; 77 x 1152 4.8 us, a launch and a chain of
// loads.  A wave owns a row (no barriers; its sums go through DPP), 4 columns per lane
// and chunk of 256, so that every fp32 access is 16 contiguous bytes per lane; where
// there are too few rows to fill the card with waves, or a row is too wide for one
// wave's registers, a workgroup of four waves owns it.  Absent vectors are read from
// x's row and replaced (a branch around every load would take the loads apart).
#include "common.h"
#include "fp8.h"
#include "kernels.h"

namespace ditmi {

// Sum over the row's waves; every lane gets it.
template <int NW>
__device__ __forceinline__ float row_sum(float v, float* s) {
  v = wave_sum(v);
  if (NW == 1) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) t += s[w];
  return t;
}

// max over the 32 lanes of a half-wave
__device__ __forceinline__ float max32(float m) {
  m = max16(m);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ f32x4 load4(const float* p) { return *(const f32x4*)p; }
// x and y are read once, and x_out is not read by this launch: streamed past
// the caches, which the modulation vectors need (131 -> 125 us at 17550 x 3072).
__device__ __forceinline__ f32x4 stream4(const float* p) { return __builtin_nontemporal_load((const f32x4*)p); }
__device__ __forceinline__ f32x4 stream4(const bf16_t* p) {
  const u32x2 w = __builtin_nontemporal_load((const u32x2*)p);
  return f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16),
               __uint_as_float(w[1] & 0xFFFF0000u)};
}

// NW waves own a row (NW = 1: four rows per workgroup); a lane holds NC chunks
// of 4 columns, chunk i at 4 (lane of the row + 64 NW i).  Y: y's dtype, -1: no y.
template <int NW, int NC, int Y, int H>
__global__ __launch_bounds__(256) void norm_residual_kernel(NormResArgs a) {
  __shared__ float red[4];
  const int tid = threadIdx.x, lr = NW == 1 ? tid & 63 : tid;
  const long row = NW == 1 ? (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(tid >> 6) : (long)blockIdx.x;
  if (row >= a.rows) return;
  const int D = a.D;
  auto col = [&](int i) { return 4 * (lr + 64 * NW * i); };
  auto at = [&](int i) { return min(col(i), D - 4); };

  const float* xr = a.x + row * D;
  f32x4 x[NC], y[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) x[i] = stream4(xr + at(i));
  if (Y == 0)
#pragma unroll
    for (int i = 0; i < NC; ++i) y[i] = stream4((const float*)a.y + row * D + at(i));
  if (Y == 1)
#pragma unroll
    for (int i = 0; i < NC; ++i) y[i] = stream4((const bf16_t*)a.y + row * D + at(i));

  int b = a.row_batch ? a.row_batch[row] : (int)(row / a.per_batch);
  const long mod = min(max(b, 0), a.batch - 1) * a.mod_stride;
  const float rD = 1.0f / (float)D;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  // (mean, 1 / deviation) of the row held in v
  auto stats = [&](const f32x4 (&v)[NC], int kind, float* mean, float* rstd) {
    float mu = 0.f;
    if (kind == 1) {
      f32x4 s = zero;
#pragma unroll
      for (int i = 0; i < NC; ++i) s += col(i) < D ? v[i] : zero;
      mu = row_sum<NW>((s[0] + s[1]) + (s[2] + s[3]), red) * rD;
    }
    f32x4 q = zero;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const f32x4 t = col(i) < D ? v[i] - mu : zero;
      q += t * t;
    }
    *mean = mu;
    *rstd = 1.0f / sqrtf(row_sum<NW>((q[0] + q[1]) + (q[2] + q[3]), red) * rD + a.eps);
  };
  const f32x4 one = {1.f, 1.f, 1.f, 1.f};
  if (Y >= 0) {
    float mean = 0.f, rstd = 1.f;
    if (a.post) stats(y, a.post, &mean, &rstd);
    const float* wp = a.w_post ? a.w_post : xr;
    const float* gp = a.gate ? a.gate + mod : xr;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const f32x4 w = load4(wp + at(i)), g = load4(gp + at(i));
      f32x4 t = (y[i] - mean) * rstd * (a.w_post ? w : one);
      t *= a.gate ? g : one;
      x[i] = x[i] * a.res_scale + t;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NC; ++i) x[i] *= a.res_scale;
  }
  if (a.x_out)
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (col(i) < D) __builtin_nontemporal_store(x[i], (f32x4*)(a.x_out + row * D + col(i)));
  if (H < 0) return;

  float mean, rstd;
  stats(x, a.pre, &mean, &rstd);
  const float* wp = a.w_pre ? a.w_pre : (const float*)a.x + row * D;
  const float* sp = a.scale ? a.scale + mod : a.x + row * D;
  const float* hp = a.shift ? a.shift + mod : a.x + row * D;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = col(i);
    const f32x4 w = load4(wp + at(i)), s = load4(sp + at(i)), f = load4(hp + at(i));
    f32x4 t = (x[i] - mean) * rstd * (a.w_pre ? w : one);
    if (a.scale) t = t * (s + 1.0f) + f;
    if (H == 2) {
      if (c >= D) t = zero;
      // 32 lanes hold a block of 128 columns
      const float sc = f8_scale(max32(fmaxf(fmaxf(fabsf(t[0]), fabsf(t[1])), fmaxf(fabsf(t[2]), fabsf(t[3]))))), inv = 1.0f / sc;
      if (c < D) *(uint32_t*)((uint8_t*)a.h + row * D + c) = pack_f8x4(t[0] * inv, t[1] * inv, t[2] * inv, t[3] * inv);
      if (c < D && c % 128 == 0) a.h_scale[row * ((D + 127) / 128) + c / 128] = sc;
    } else if (c < D) {
      if (H == 1) *(u32x2*)((bf16_t*)a.h + row * D + c) = u32x2{pack_bf16x2(t[0], t[1]), pack_bf16x2(t[2], t[3])};
      else *(f32x4*)((float*)a.h + row * D + c) = t;
    }
  }
}

template <int Y, int H>
static void launch_yh(const NormResArgs& a, hipStream_t st) {
  const dim3 four((a.rows + 3) / 4), each(a.rows), block(256);
#define NORM_RES(NW, NC) hipLaunchKernelGGL((norm_residual_kernel<NW, NC, Y, H>), NW == 1 ? four : each, block, 0, st, a)
  // A wave per row from 2048 rows (two waves per SIMD) on: 8192 x 1152 22.8 us
  // against 28.7 with four, 17550 x 3072 127 against 132, 2048 x 1152 7.9
  // against 7.6, 1024 x 1152 6.4 against 5.1.
  if (a.rows >= 2048 && a.D <= 4096) {
    if (a.D <= 1024) NORM_RES(1, 4);
    else if (a.D <= 1536) NORM_RES(1, 6);
    else if (a.D <= 2048) NORM_RES(1, 8);
    else if (a.D <= 3072) NORM_RES(1, 12);
    else NORM_RES(1, 16);
  } else {
    if (a.D <= 1024) NORM_RES(4, 1);
    else if (a.D <= 2048) NORM_RES(4, 2);
    else if (a.D <= 3072) NORM_RES(4, 3);
    else if (a.D <= 4096) NORM_RES(4, 4);
    else NORM_RES(4, 8);
  }
#undef NORM_RES
}

template <int Y>
static void launch_y(const NormResArgs& a, hipStream_t st) {
  if (!a.h) launch_yh<Y, -1>(a, st);
  else if (a.h_dtype == 0) launch_yh<Y, 0>(a, st);
  else if (a.h_dtype == 1) launch_yh<Y, 1>(a, st);
  else launch_yh<Y, 2>(a, st);
}

hipError_t launch_norm_residual(const NormResArgs& a, hipStream_t st) {
  if (!a.y) launch_y<-1>(a, st);
  else if (a.y_dtype == 0) launch_y<0>(a, st);
  else launch_y<1>(a, st);
  return hipGetLastError();
}

}  // namespace ditmi
