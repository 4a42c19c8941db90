// The norms around a sub-layer with its gate and residual, in one pass
// (ditmi.h: dit_norm_residual).  A workgroup owns one row, held in registers
// between its passes: the statistics of y, the residual, the statistics of the
// new row, the modulated output.  Bound by memory.
#include "common.h"
#include "fp8.h"
#include "kernels.h"

namespace ditmi {

// Sums over a workgroup of NW waves, two values at a time; every lane gets them.
template <int NW>
__device__ __forceinline__ float wg_sum(float v, float* s) {
  v = wave_sum(v);
  if (NW == 1) return v;
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[wave] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) t += s[w];
  return t;
}

// NW waves, each lane NC chunks of 8 columns, chunk i at 8 * (tid + i * NW * 64).
template <int NW, int NC>
__global__ __launch_bounds__(NW * 64) void norm_residual_kernel(NormResArgs a) {
  __shared__ float red[NW];
  const int tid = threadIdx.x;
  const long row = blockIdx.x;
  const int D = a.D;
  int b = a.row_batch ? a.row_batch[row] : (int)(row / a.per_batch);
  b = min(max(b, 0), a.batch - 1);
  const float* gate = a.gate ? a.gate + b * a.mod_stride : nullptr;
  const float* shift = a.shift ? a.shift + b * a.mod_stride : nullptr;
  const float* scale = a.scale ? a.scale + b * a.mod_stride : nullptr;
  const float rD = 1.0f / (float)D;

  float x[NC][8], y[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = 8 * (tid + i * NW * 64);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = y[i][e] = 0.f;
    if (c < D) {
      load8(a.x + row * D + c, x[i]);
      if (a.y) {
        if (a.y_dtype == 0) load8((const float*)a.y + row * D + c, y[i]);
        else load8((const bf16_t*)a.y + row * D + c, y[i]);
      }
    }
  }
  // (mean, 1 / deviation) of a row held as v
  auto stats = [&](const float (&v)[NC][8], int kind, float* mean, float* rstd) {
    float mu = 0.f;
    if (kind == 1) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[i][e];
      mu = wg_sum<NW>(s, red) * rD;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (8 * (tid + i * NW * 64) < D)
#pragma unroll
        for (int e = 0; e < 8; ++e) q += (v[i][e] - mu) * (v[i][e] - mu);
    *mean = mu;
    *rstd = 1.0f / sqrtf(wg_sum<NW>(q, red) * rD + a.eps);
  };
  float mean = 0.f, rstd = 1.f;
  if (a.y && a.post) stats(y, a.post, &mean, &rstd);
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = 8 * (tid + i * NW * 64);
    if (c >= D) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float t = (y[i][e] - mean) * rstd;
      if (a.y) {
        if (a.w_post) t *= a.w_post[c + e];
        if (gate) t *= gate[c + e];
        x[i][e] = fmaf(a.res_scale, x[i][e], t);
      } else {
        x[i][e] *= a.res_scale;
      }
    }
    if (a.x_out) {
      *(f32x4*)(a.x_out + row * D + c) = f32x4{x[i][0], x[i][1], x[i][2], x[i][3]};
      *(f32x4*)(a.x_out + row * D + c + 4) = f32x4{x[i][4], x[i][5], x[i][6], x[i][7]};
    }
  }
  if (!a.h) return;
  stats(x, a.pre, &mean, &rstd);
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = 8 * (tid + i * NW * 64);
    const bool in = c < D;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float t = (x[i][e] - mean) * rstd;
      if (in) {
        if (a.w_pre) t *= a.w_pre[c + e];
        if (scale) t = fmaf(t, 1.0f + scale[c + e], shift[c + e]);
      }
      x[i][e] = in ? t : 0.f;
    }
    if (a.h_dtype == 2) {
      // 16 lanes hold a block of 128 columns
      const float sc = f8_scale(max16(amax8(x[i]))), inv = 1.0f / sc;
      if (!in) continue;
      *(u32x2*)((uint8_t*)a.h + row * D + c) = pack_f8x8(x[i], inv);
      if (c % 128 == 0) a.h_scale[row * ((D + 127) / 128) + c / 128] = sc;
    } else if (in && a.h_dtype == 1) {
      *(u32x4*)((bf16_t*)a.h + row * D + c) = u32x4{pack_bf16x2(x[i][0], x[i][1]), pack_bf16x2(x[i][2], x[i][3]),
                                                    pack_bf16x2(x[i][4], x[i][5]), pack_bf16x2(x[i][6], x[i][7])};
    } else if (in) {
      *(f32x4*)((float*)a.h + row * D + c) = f32x4{x[i][0], x[i][1], x[i][2], x[i][3]};
      *(f32x4*)((float*)a.h + row * D + c + 4) = f32x4{x[i][4], x[i][5], x[i][6], x[i][7]};
    }
  }
}

hipError_t launch_norm_residual(const NormResArgs& a, hipStream_t st) {
  const dim3 grid(a.rows);
  if (a.D <= 2048) hipLaunchKernelGGL((norm_residual_kernel<4, 1>), grid, dim3(256), 0, st, a);
  else if (a.D <= 4096) hipLaunchKernelGGL((norm_residual_kernel<4, 2>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((norm_residual_kernel<4, 4>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace ditmi
