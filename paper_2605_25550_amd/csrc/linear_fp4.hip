// Linear layer on MXFP4 operands (ditmi.h: dit_linear_fp4), and the quantisation into such blocks
// and back.
#include <algorithm>

#include "common.h"
#include "fp4.h"
#include "fp8.h"
#include "kernels.h"

namespace ditmi {

typedef int i32x8 __attribute__((ext_vector_type(8)));

template <int OUT>
__device__ __forceinline__ float bias_at(const LinF4Args& a, int n) {
  return OUT == 0 ? ((const float*)a.bias)[n] : bf2f(((const bf16_t*)a.bias)[n]);
}

__device__ __forceinline__ i32x8 operand(u32x4 c) { return i32x8{(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0}; }

// A workgroup owns 16 outputs of up to 16 TM rows; its waves divide the blocks of 128 k, load fragments
// from global memory and add their sums through LDS in order.
template <int TM, int NW, int OUT>
__global__ __launch_bounds__(NW * 64) void linear_f4_rows_kernel(LinF4Args a) {
  constexpr int U = TM == 1 ? 4 : 2;  // blocks of k in flight per wave
  __shared__ f32x4 sum[NW][TM][64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16 * TM;
  const int KB = (a.K + 127) / 128;
  const long half = a.K / 2;
  const int wn = min(n0 + r16, a.N - 1);
  const uint8_t* wrow = a.w + (long)wn * half;
  const uint8_t* arow[TM];
  int am[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    am[i] = min(m0 + i * 16 + r16, a.M - 1);
    arow[i] = a.a + (long)am[i] * half;
  }
  f32x4 acc[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 wf[U], af[U][TM];
  int sw[U], sa[U][TM];
  auto load = [&](int u, int kb) {
    if (kb >= KB) return;
    const int blk = kb * 4 + kq;
    const bool in = blk * 32 < a.K;  // past the end: zeros, and a scale that is a number
    const u32x4 z = {0u, 0u, 0u, 0u};
    wf[u] = in ? *(const u32x4*)(wrow + blk * 16) : z;
    sw[u] = in ? (int)a.w_scale[f4_scale_at(a.N, wn, blk)] : 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      af[u][i] = in ? *(const u32x4*)(arow[i] + blk * 16) : z;
      sa[u][i] = in ? (int)a.a_scale[f4_scale_at(a.M, am[i], blk)] : 0;
    }
  };
#pragma unroll
  for (int u = 0; u < U; ++u) load(u, wave + u * NW);
  for (int kb = wave; kb < KB; kb += U * NW)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (kb + u * NW >= KB) break;
#pragma unroll
      for (int i = 0; i < TM; ++i)
        acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(wf[u]), operand(af[u][i]), acc[i], 4, 4, 0, sw[u],
                                                                  0, sa[u][i]);
      load(u, kb + (u + U) * NW);
    }
#pragma unroll
  for (int i = 0; i < TM; ++i) sum[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < TM; i += NW) {
    f32x4 y = sum[0][i][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) y += sum[w][i][lane];
    const int m = m0 + i * 16 + r16, n = n0 + kq * 4;
    if (m >= a.M || n >= a.N) continue;
    if (OUT == 3) {
      *(f32x4*)(a.part + (long)m * a.N + n) = y;
      continue;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.N) {
        if (a.bias) y[e] += bias_at<OUT>(a, n + e);
        if (a.act) y[e] = gelu_tanh(y[e]);
        if (OUT == 0) ((float*)a.out)[(long)m * a.N + n + e] = y[e];
        else ((bf16_t*)a.out)[(long)m * a.N + n + e] = f2bf(y[e]);
      }
  }
}

// Bias, activation and quantisation of fp32 sums [M][N]: a lane takes 8 columns.
__global__ __launch_bounds__(256) void linear_f4_finish_kernel(LinF4Args a) {
  const long groups = (long)a.M * (a.N / 8), i = (long)blockIdx.x * 256 + threadIdx.x;
  const long at = min(i, groups - 1);
  const int m = (int)(at / (a.N / 8)), n = (int)(at - (long)m * (a.N / 8)) * 8;
  float y[8];
  const float* p = a.part + (long)m * a.N + n;
  uint32_t mx = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = p[e];
    if (a.bias) y[e] += bias_at<3>(a, n + e);
    if (a.act) y[e] = gelu_tanh(y[e]);
    mx = max(mx, abs_bits(y[e]));
  }
  const uint32_t s = f4_scale(max_quad(mx));
  if (i >= groups) return;
  *(uint32_t*)((uint8_t*)a.out + ((long)m * a.N + n) / 2) = pack_f4x8(y, s);
  if ((n & 31) == 0) a.out_scale[f4_scale_at(a.M, m, n / 32)] = (uint8_t)s;
  // the scales behind the last column
  if (n + 8 == a.N)
    for (int b = a.N / 32; b & 7; ++b) a.out_scale[f4_scale_at(a.M, m, b)] = 0;
}

static constexpr long MAX_THREADS = 1L << 32;  // a grid has fewer

LinF4Plan linear_fp4_plan(int M, int N, int K, int dtype) {
  LinF4Plan p{};
  const long wgs = (long)((N + 15) / 16) * ((M + 63) / 64);
  if ((M + 63) / 64 > 65535 || wgs * 512 >= MAX_THREADS) p.tile = -1;
  p.bytes = dtype == 3 ? (size_t)M * N * 4 : 0;
  return p;
}

template <int OUT>
static void launch_out(const LinF4Args& a, hipStream_t st) {
  const dim3 block(512);
  if (a.M <= 16) hipLaunchKernelGGL((linear_f4_rows_kernel<1, 8, OUT>), dim3((a.N + 15) / 16), block, 0, st, a);
  else if (a.M <= 32) hipLaunchKernelGGL((linear_f4_rows_kernel<2, 8, OUT>), dim3((a.N + 15) / 16), block, 0, st, a);
  else hipLaunchKernelGGL((linear_f4_rows_kernel<4, 8, OUT>), dim3((a.N + 15) / 16, (a.M + 63) / 64), block, 0, st, a);
  if (OUT == 3)
    hipLaunchKernelGGL(linear_f4_finish_kernel, dim3((unsigned)(((long)a.M * (a.N / 8) + 255) / 256)), dim3(256), 0, st, a);
}

hipError_t launch_linear_fp4(const LinF4Args& a, const LinF4Plan& p, hipStream_t st) {
  if (a.dtype == 0) launch_out<0>(a, st);
  else if (a.dtype == 1) launch_out<1>(a, st);
  else launch_out<3>(a, st);
  return hipGetLastError();
}

// ------------------------------------------------------------------ quantisation
// 32 lanes take the 256 columns of one panel of one row, 8 columns each; a workgroup 8 rows.
__device__ __forceinline__ void panel_at(int cols, int* panel, long* row0) {
  const unsigned np = (unsigned)(cols + 255) / 256u, grp = blockIdx.x / np;
  *panel = (int)(blockIdx.x - grp * np);
  *row0 = (long)grp * 8;
}

template <typename T>
__global__ __launch_bounds__(256) void quant_f4_kernel(int rows, int cols, const T* x, long x_row, uint8_t* q, uint8_t* scale) {
  int panel;
  long r;
  panel_at(cols, &panel, &r);
  const int c = panel * 256 + (threadIdx.x & 31) * 8;
  r += threadIdx.x >> 5;
  const bool row_in = r < rows, in = row_in && c < cols;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (in) load8(x + r * x_row + c, v);
  uint32_t mx = 0u;
#pragma unroll
  for (int e = 0; e < 8; ++e) mx = max(mx, abs_bits(v[e]));
  const uint32_t s = f4_scale(max_quad(mx));
  if (in) *(uint32_t*)(q + (r * cols + c) / 2) = pack_f4x8(v, s);
  if (row_in && (threadIdx.x & 3) == 0) scale[f4_scale_at(rows, r, c / 32)] = (uint8_t)s;  // (0 behind the last column)
}

template <typename T>
__global__ __launch_bounds__(256) void dequant_f4_kernel(int rows, int cols, const uint8_t* q, const uint8_t* scale, T* x, long x_row) {
  int panel;
  long r;
  panel_at(cols, &panel, &r);
  const int c = panel * 256 + (threadIdx.x & 31) * 8;
  r += threadIdx.x >> 5;
  if (r >= rows || c >= cols) return;
  const uint32_t w = *(const uint32_t*)(q + (r * cols + c) / 2);
  const uint32_t s = scale[f4_scale_at(rows, r, c / 32)];
  const float sc = f4_scale_value(s);
  float v[8];
  unpack_f4x8(w, sc, v);
  if (s == 255u)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = sc;
  T* o = x + r * x_row + c;
  if constexpr (sizeof(T) == 4) {
    *(f32x4*)o = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)(o + 4) = f32x4{v[4], v[5], v[6], v[7]};
  } else {
    *(u32x4*)o = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  }
}

static dim3 panels(int rows, int cols) { return dim3((unsigned)(((long)cols + 255) / 256 * (((long)rows + 7) / 8))); }

template <typename T>
static void quantize_t(int rows, int cols, const void* x, long x_row, void* codes, void* scale, hipStream_t st) {
  hipLaunchKernelGGL((quant_f4_kernel<T>), panels(rows, cols), dim3(256), 0, st, rows, cols, (const T*)x, x_row, (uint8_t*)codes,
                     (uint8_t*)scale);
}
hipError_t launch_quantize_fp4(int rows, int cols, int dtype, const void* x, long x_row, void* codes, void* scale, hipStream_t st) {
  if (dtype == 0) quantize_t<float>(rows, cols, x, x_row, codes, scale, st);
  else quantize_t<bf16_t>(rows, cols, x, x_row, codes, scale, st);
  return hipGetLastError();
}

template <typename T>
static void dequantize_t(int rows, int cols, const void* codes, const void* scale, void* x, long x_row, hipStream_t st) {
  hipLaunchKernelGGL((dequant_f4_kernel<T>), panels(rows, cols), dim3(256), 0, st, rows, cols, (const uint8_t*)codes,
                     (const uint8_t*)scale, (T*)x, x_row);
}
hipError_t launch_dequantize_fp4(int rows, int cols, int dtype, const void* codes, const void* scale, void* x, long x_row,
                                 hipStream_t st) {
  if (dtype == 0) dequantize_t<float>(rows, cols, codes, scale, x, x_row, st);
  else dequantize_t<bf16_t>(rows, cols, codes, scale, x, x_row, st);
  return hipGetLastError();
}

}  // namespace ditmi
