// Linear layer on e4m3 operands with an fp32 scale for every block of 128
// (ditmi.h: dit_linear_fp8), and the quantisation into such blocks.
//
// v_mfma_f32_16x16x128_f8f6f4 takes a whole block of k at once: its result is
// the block's sum of products, which one FMA per element scales and adds to
// the fp32 accumulator.  The weights are the A operand and the activations the
// B operand, so that a lane (m = lane % 16, n = 4 (lane / 16) + e) belongs to
// one activation row: its block scale is one value, and its four outputs are
// consecutive.
#include <algorithm>

#include "common.h"
#include "fp8.h"
#include "kernels.h"

namespace ditmi {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// Codes 8h .. 8h+7 of a lane's 32 as bf16.
__device__ __forceinline__ bf16x8 widen(i32x8 v, int h) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * h + i], 1.0f, false));
    w[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * h + i], 1.0f, true));
  }
  return __builtin_bit_cast(bf16x8, w);
}

// Product of two 16 x 128 operands, a block of k, in fp32.  The 8-bit pipe adds
// the products of every 8 consecutive k aligned to the largest of them, with a
// last place of 2^-13 of its binade (measured with pairs of powers of two; the
// groups are added in fp32): 1.3e-5 of the result's norm on normal data, far
// below a bf16 or e4m3 rounding, but not fp32.  WIDE widens the codes to bf16
// (exact, as their products are in fp32) and takes the bf16 pipe, which keeps
// 24 bits at half the rate: that is what fp32 outputs are computed with.
template <bool WIDE>
__device__ __forceinline__ f32x4 mfma_block(i32x8 a, i32x8 b) {
  f32x4 c = {0.f, 0.f, 0.f, 0.f};
  if constexpr (!WIDE) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
  } else {
#pragma unroll
    for (int h = 0; h < 4; ++h) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(a, h), widen(b, h), c, 0, 0, 0);
    return c;
  }
}

// A workgroup of four waves owns 128 x 128 outputs, a wave 64 x 64; fragments
// come straight from global memory.
template <bool WIDE>
__global__ __launch_bounds__(256) void linear_f8_kernel(LinF8Args a) {
  __shared__ float amax_s[2][128];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int tiles_n = (a.N + 127) / 128;
  const int tile = xcd_remap(blockIdx.x, gridDim.x);
  const int tn = tile % tiles_n, tm = tile / tiles_n;
  const int wm = wave >> 1, wn = wave & 1;
  const int m0 = tm * 128 + wm * 64, n0 = tn * 128 + wn * 64;
  const int KB = (a.K + 127) / 128;

  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto frag = [&](const uint8_t* base, long row, int kb) {
    const int k = kb * 128 + kq * 32;
    const u32x4 z = {0u, 0u, 0u, 0u};
    const uint8_t* p = base + row * a.K + k;
    const u32x4 lo = k < a.K ? *(const u32x4*)p : z, hi = k + 16 < a.K ? *(const u32x4*)(p + 16) : z;
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };
  const float* ws = a.w_scale + (long)tn * KB;
  for (int kb = 0; kb < KB; ++kb) {
    i32x8 wf[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) wf[j] = frag(a.w, min(n0 + j * 16 + r16, a.N - 1), kb);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = min(m0 + i * 16 + r16, a.M - 1);
      const i32x8 af = frag(a.a, m, kb);
      const float s = a.a_scale[(long)m * KB + kb] * ws[kb];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] += s * mfma_block<WIDE>(wf[j], af);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = n0 + j * 16 + kq * 4 + e;
        float y = acc[i][j][e];
        if (a.bias && n < a.N) y += a.dtype == 0 ? ((const float*)a.bias)[n] : bf2f(((const bf16_t*)a.bias)[n]);
        if (a.act) y = gelu_tanh(y);
        acc[i][j][e] = n < a.N ? y : 0.f;
      }
  if (a.dtype == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float mx = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, fabsf(acc[i][j][e]));
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      if (kq == 0) amax_s[wn][wm * 64 + i * 16 + r16] = mx;
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + i * 16 + r16;
    if (m >= a.M) continue;
    float inv = 0.f;
    if (a.dtype == 2) {
      const int r = wm * 64 + i * 16 + r16;
      const float sc = f8_scale(fmaxf(amax_s[0][r], amax_s[1][r]));
      inv = 1.0f / sc;
      if (wn == 0 && kq == 0) a.out_scale[(long)m * tiles_n + tn] = sc;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 y = acc[i][j];
      const int n = n0 + j * 16 + kq * 4;
      const long o = (long)m * a.N + n;
      if (a.dtype == 2) {
        if (n < a.N) *(uint32_t*)((uint8_t*)a.out + o) = pack_f8x4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < a.N) {
            if (a.dtype == 0) ((float*)a.out)[o + e] = y[e];
            else ((bf16_t*)a.out)[o + e] = f2bf(y[e]);
          }
      }
    }
  }
}

int linear_fp8_split(int M, int N, int K) { return 1; }

hipError_t launch_linear_fp8(const LinF8Args& a, hipStream_t st) {
  const long tiles = (long)((a.M + 127) / 128) * ((a.N + 127) / 128);
  if (a.dtype == 0) hipLaunchKernelGGL(linear_f8_kernel<true>, dim3((unsigned)tiles), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(linear_f8_kernel<false>, dim3((unsigned)tiles), dim3(256), 0, st, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------ quantisation
// Rows: 16 lanes take the 128 columns of one block.
template <typename T>
__global__ __launch_bounds__(256) void quant_rows_kernel(int rows, int cols, const T* x, long x_row, uint8_t* q, float* scale) {
  const int nb = (cols + 127) / 128;
  const long blk = (long)blockIdx.x * 16 + (threadIdx.x >> 4);
  const long n = (long)rows * nb;
  const long bc = min(blk, n - 1);  // every lane stays for the exchange
  const long r = bc / nb;
  const int cb = (int)(bc - r * nb), c = cb * 128 + (threadIdx.x & 15) * 8;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (c < cols) load8(x + r * x_row + c, v);
  const float sc = f8_scale(max16(amax8(v))), inv = 1.0f / sc;
  if (blk >= n) return;
  if (c < cols)
    *(u32x2*)(q + r * cols + c) = pack_f8x8(v, inv);
  if ((threadIdx.x & 15) == 0) scale[blk] = sc;
}

// 128 x 128 blocks: a workgroup holds one in registers.
template <typename T>
__global__ __launch_bounds__(256) void quant_block_kernel(int rows, int cols, const T* x, long x_row, uint8_t* q, float* scale) {
  __shared__ float part[4];
  const int cb = blockIdx.x, rb = blockIdx.y, nb = gridDim.x;
  const int c = cb * 128 + (threadIdx.x & 15) * 8, r0 = rb * 128 + (threadIdx.x >> 4);
  float v[8][8], mx = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
    if (c < cols && r0 + 16 * i < rows) load8(x + (long)(r0 + 16 * i) * x_row + c, v[i]);
    mx = fmaxf(mx, amax8(v[i]));
  }
  mx = max16(mx);
  mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
  mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mx;
  __syncthreads();
  const float sc = f8_scale(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]))), inv = 1.0f / sc;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c < cols && r0 + 16 * i < rows)
      *(u32x2*)(q + (long)(r0 + 16 * i) * cols + c) = pack_f8x8(v[i], inv);
  if (threadIdx.x == 0) scale[(long)rb * nb + cb] = sc;
}

template <typename T>
static void quantize_t(int rows, int cols, int block_rows, const void* x, long x_row, void* codes, float* scale, hipStream_t st) {
  const int nb = (cols + 127) / 128;
  if (block_rows == 1)
    hipLaunchKernelGGL((quant_rows_kernel<T>), dim3((unsigned)(((long)rows * nb + 15) / 16)), dim3(256), 0, st, rows, cols,
                       (const T*)x, x_row, (uint8_t*)codes, scale);
  else
    hipLaunchKernelGGL((quant_block_kernel<T>), dim3(nb, (rows + 127) / 128), dim3(256), 0, st, rows, cols, (const T*)x,
                       x_row, (uint8_t*)codes, scale);
}
hipError_t launch_quantize_fp8(int rows, int cols, int block_rows, int dtype, const void* x, long x_row, void* codes,
                               float* scale, hipStream_t st) {
  if (dtype == 0) quantize_t<float>(rows, cols, block_rows, x, x_row, codes, scale, st);
  else quantize_t<bf16_t>(rows, cols, block_rows, x, x_row, codes, scale, st);
  return hipGetLastError();
}

}  // namespace ditmi
