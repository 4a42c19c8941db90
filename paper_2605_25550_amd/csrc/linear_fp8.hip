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

// 4 bytes per lane from gsrc into LDS at (wave-uniform) lds_base + 4 * lane.
__device__ __forceinline__ void dma_4(const void* gsrc, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds_base), "v"(gsrc) : "memory", "m0");
}

template <int OUT>
__device__ __forceinline__ float bias_at(const LinF8Args& a, int n) {
  return OUT == 0 ? ((const float*)a.bias)[n] : bf2f(((const bf16_t*)a.bias)[n]);
}
// Stores four consecutive outputs of row m from column n on (n < N); whole:
// N is a multiple of four, so groups are whole and aligned.  inv: of the new
// block's scale (e4m3).
template <int OUT>
__device__ __forceinline__ void store_y4(const LinF8Args& a, bool whole, int m, int n, f32x4 y, float inv) {
  const long o = (long)m * a.N + n;
  const uint32_t codes = OUT == 2 ? pack_f8x4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv) : 0u;
  if (whole) {
    if (OUT == 2) *(uint32_t*)((uint8_t*)a.out + o) = codes;
    else if (OUT == 0) *(f32x4*)((float*)a.out + o) = y;
    else *(u32x2*)((bf16_t*)a.out + o) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.N) {
        if (OUT == 2) ((uint8_t*)a.out)[o + e] = (uint8_t)(codes >> (8 * e));
        else if (OUT == 0) ((float*)a.out)[o + e] = y[e];
        else ((bf16_t*)a.out)[o + e] = f2bf(y[e]);
      }
  }
}

// Order of the tiles: groups of eight row tiles x all column tiles, rows
// fastest, so that what runs at once on an XCD shares operands in its L2.
__device__ __forceinline__ void tile_at(int tile, int tiles_m, int tiles_n, int* tm, int* tn) {
  const int per = 8 * tiles_n, grp = tile / per, gm = min(8, tiles_m - grp * 8), in_grp = tile - grp * per;
  *tm = grp * 8 + in_grp % gm;
  *tn = in_grp / gm;
}

__device__ const u32x4 zero_chunk = {0u, 0u, 0u, 0u};

// Many rows: a workgroup of WM x WN waves owns BM rows x BN outputs, a wave
// BM / WM x BN / WN of them.  Both operands' blocks of k (128 bytes per row) go
// HBM -> LDS by DMA, one block ahead of the math, with the activation scales
// of the block; 16-byte chunk c of row r lies at c ^ f(r), so that the 16 rows
// of a fragment read come from distinct banks.
//
// Bound by the LDS (fragment reads beside the DMA's writes) and, in long runs, by
// power: 17550 x 12288 x 3072 640 us, 2.07 PFLOP/s of the 3.6 that a bare loop of
// these products and scalings reaches, MFMA busy 51% at 1.85 GHz; 1997 x 1152 x
// 4608 with GELU 23.3 us, of which nine blocks of k take about 12.
template <int BM, int BN, int WM, int WN, int OUT>  // OUT: the output's dtype
__global__ __launch_bounds__(WM * WN * 64) void linear_f8_tile_kernel(LinF8Args a) {
  constexpr bool WIDE = OUT == 0;
  constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr int IPW = (BM + BN) / (8 * NW);  // 1 KB DMA instructions per wave and block of k
  constexpr int STAGE = (BM + BN) * 128;  // W rows, then A rows
  constexpr int SC = BM * 32;             // scales of BM rows x 8 blocks
  constexpr int PAIRS = (IPW + 1) / 2;
  static_assert(TN % 2 == 0 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && BM % 64 == 0 && BM / 64 <= NW && 128 % (BN / WN) == 0, "tile split");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * STAGE + 2 * SC];
  float(*amax_s)[BM] = (float(*)[BM])smem;  // [WN][BM], after the last block

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int tiles_n = (a.N + BN - 1) / BN, tiles_m = (a.M + BM - 1) / BM;
  // the first n_full tiles whole, then the units of the others: range by range
  int tile, part = 0, split = 1;
  if ((int)blockIdx.x < a.n_full) {
    tile = xcd_remap(blockIdx.x, a.n_full);
  } else {
    const int n_tail = tiles_m * tiles_n - a.n_full, unit = xcd_remap(blockIdx.x - a.n_full, n_tail * a.split);
    part = unit / n_tail;
    tile = a.n_full + unit - part * n_tail;
    split = a.split;
  }
  int tm, tn;
  tile_at(tile, tiles_m, tiles_n, &tm, &tn);
  const int wm = wave % WM, wn = wave / WM;
  const int KB = (a.K + 127) / 128;
  const int kb0 = (int)((long)KB * part / split), kb1 = (int)((long)KB * (part + 1) / split);
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));

  // DMA: instruction t of this wave covers rows 8 q .. 8 q + 7, q = wave + NW t, of
  // the stage's W rows then A rows; the lane's chunk is the same in all of them.
  // Past a row's end W has zeros, and A the row's last chunk again: its values
  // meet the zeros (and a NaN among them is in the row's sums anyway).
  unsigned off[IPW];
#pragma unroll
  for (int t = 0; t < IPW; ++t) {
    const int R = (wave + NW * t) * 8 + (lane >> 3);
    off[t] = (unsigned)(R < BN ? min(R, a.N - 1 - tn * BN) : min(R - BN, a.M - 1 - tm * BM)) * (unsigned)a.K;
  }
  const int chunk = (lane & 7) ^ (lane >> 3) ^ (wave & 1);
  static_assert(NW % 2 == 0, "the chunk of a lane does not depend on the instruction");
  const uint8_t* wb = a.w + (long)tn * BN * a.K;
  const uint8_t* ab = a.a + (long)tm * BM * a.K;
  auto issue_one = [&](int kb, int sl, int t) {
    const unsigned k = (unsigned)(kb * 128 + chunk * 16), dst = lds0 + (unsigned)(sl * STAGE + (wave + NW * t) * 1024);
    if (t * NW * 8 < BN)
      dma_16((int)k < a.K ? (const void*)(wb + (off[t] + k)) : (const void*)&zero_chunk, dst);
    else
      dma_16s(ab, off[t] + min(k, (unsigned)a.K - 16u), dst);
  };
  // Activation scales, eight blocks of k at a time (a scale of each row alone
  // would fetch as many cache lines as the rows themselves): instruction u of
  // a chunk copies 8 rows x 8 blocks, block x of row r to 8 r + (x ^ (r & 7)).
  const float* sab = a.a_scale + (long)tm * BM * KB;
  auto issue_scales = [&](int c, int u) {
    const int r = u * 8 + (lane >> 3), x = (lane & 7) ^ (r & 7);
    dma_4(sab + (long)min(r, a.M - 1 - tm * BM) * KB + min(kb0 + c * 8 + x, KB - 1),
          lds0 + (unsigned)(2 * STAGE + (c & 1) * SC + u * 256));
  };
  const int swz = (r16 & 7) ^ ((r16 >> 3) & 1);
  auto frag = [&](const unsigned char* rows, int r) {
    const unsigned char* p = rows + r * 128;
    const u32x4 lo = *(const u32x4*)(p + (((2 * kq) ^ swz) << 4)), hi = *(const u32x4*)(p + (((2 * kq + 1) ^ swz) << 4));
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };

  f32x4 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int n0 = tn * BN + wn * (BN / WN), m0 = tm * BM + wm * (BM / WM);
  const float* ws = a.w_scale + (long)__builtin_amdgcn_readfirstlane(min(n0 / 128, (a.N - 1) / 128)) * KB;

  i32x8 af[TM], wf[2];
  float s[TM];
  auto wrow = [&](int i) { return smem + (i & 1) * STAGE + wn * (BN / WN) * 128; };
  auto arow = [&](int i) { return smem + (i & 1) * STAGE + (BN + wm * (BM / WM)) * 128; };
  auto srow = [&](int i) {
    return (const float*)(smem + 2 * STAGE + ((i >> 3) & 1) * SC) + (wm * (BM / WM) + r16) * 8 + ((i & 7) ^ (r16 & 7));
  };
  if (kb0 < kb1) {
    for (int u = wave; u < BM / 8; u += NW) issue_scales(0, u);
#pragma unroll
    for (int t = 0; t < IPW; ++t) issue_one(kb0, 0, t);
    wait_vmcnt<0>();
    __syncthreads();
    wf[0] = frag(wrow(0), r16);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      af[i] = frag(arow(0), i * 16 + r16);
      s[i] = srow(0)[i * 128];
    }
  }
  float sw = kb0 < kb1 ? ws[kb0] : 0.f;  // a scalar load, one block ahead
  for (int kb = kb0; kb < kb1; ++kb) {
    const int b = kb - kb0;
    const float sw_next = ws[min(kb + 1, KB - 1)];
    if (wave < BM / 64) issue_scales((b >> 3) + 1, (b & 7) * (BM / 64) + wave);  // an eighth of the next chunk
#pragma unroll
    for (int i = 0; i < TM; ++i) s[i] *= sw;
    float s_next[TM];
    // Products in the order of the weights' fragments, each read one group of
    // TM ahead; the scaled sum of a product follows three products behind, when
    // it is ready.  Before the last group, whose operands are in registers, the
    // waves meet: the next block has landed, and this one's slot may be
    // refilled.  The next block's first operands are then read behind the last
    // products, so that the matrix pipe has work across the barrier.
    f32x4 d[4];
#pragma unroll
    for (int x = 0; x < TN * TM + 3; ++x) {
      const int j = x / TM, i = x % TM;
      if (x < TN * TM) {
        if (i == 0 && j + 1 < TN) wf[(j + 1) & 1] = frag(wrow(b), (j + 1) * 16 + r16);
        if (x == (TN - 1) * TM) {
          wait_vmcnt<0>();
          __syncthreads();
          wf[TN & 1] = frag(wrow(b + 1), r16);
        }
        d[x % 4] = mfma_block<WIDE>(wf[j & 1], af[i]);
        if (j == TN - 1) {
          af[i] = frag(arow(b + 1), i * 16 + r16);
          s_next[i] = srow(b + 1)[i * 128];
        }
      }
      if (x >= 3) {
        const int jp = (x - 3) / TM, ip = (x - 3) % TM;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[jp][ip][e] = fmaf(s[ip], d[(x - 3) % 4][e], acc[jp][ip][e]);
      }
      // the next block's DMA, two instructions behind each of the first
      // products: spread further they arrive late (up to 6% slower), right
      // behind the barrier they hold up the reads there (16% slower).  After the
      // last block: not read
      if (x < PAIRS) {
        issue_one(kb + 1, ~b & 1, 2 * x);
        if (2 * x + 1 < IPW) issue_one(kb + 1, ~b & 1, 2 * x + 1);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) s[i] = s_next[i];
    sw = sw_next;
  }

  wait_vmcnt<0>();
  __syncthreads();
  if (split > 1) {  // to the range's own copy of the tile, [BM][BN]
    const int n_tail = tiles_m * tiles_n - a.n_full;
    float* pp = a.part + ((long)part * n_tail + (tile - a.n_full)) * (BM * BN);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        *(f32x4*)(pp + (wm * (BM / WM) + i * 16 + r16) * BN + wn * (BN / WN) + j * 16 + kq * 4) = acc[j][i];
    return;
  }
  if (a.bias) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float b = bias_at<OUT>(a, min(n0 + j * 16 + kq * 4 + e, a.N - 1));
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i][e] += b;
      }
  }
  if (a.act) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][i][e] = gelu_tanh(acc[j][i][e]);
  }
  float inv[TM] = {};
  if (OUT == 2) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      float mx = 0.f;
#pragma unroll
      for (int j = 0; j < TN; ++j)
        // (columns past N repeat column N - 1, of the same block)
        if (n0 + j * 16 + kq * 4 < a.N)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx = fmaxf(mx, fabsf(acc[j][i][e]));
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      inv[i] = mx;
    }
    constexpr int SH = 128 / (BN / WN);  // waves that share a block of 128 outputs
    if (SH > 1) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
        if (kq == 0) amax_s[wn][wm * (BM / WM) + i * 16 + r16] = inv[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int w = 0; w < SH; ++w) inv[i] = fmaxf(inv[i], amax_s[wn / SH * SH + w][wm * (BM / WM) + i * 16 + r16]);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const float sc = f8_scale(inv[i]);
      const int m = m0 + i * 16 + r16;
      if (wn % SH == 0 && kq == 0 && m < a.M && n0 < a.N) a.out_scale[(long)m * ((a.N + 127) / 128) + n0 / 128] = sc;
      inv[i] = 1.0f / sc;
    }
  }
  auto store_all = [&](bool whole) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = m0 + i * 16 + r16;
      if (m < a.M)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const int n = n0 + j * 16 + kq * 4;
          if (n < a.N) store_y4<OUT>(a, whole, m, n, acc[j][i], inv[i]);
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (a.N % 4 == 0) store_all(true);
  else store_all(false);
}

// Adds the k-ranges of the divided tiles, in order, and applies the epilogue.
// 32 lanes take the 128 columns of one block of one row of a tile.
template <int BM, int BN, int OUT>
__global__ __launch_bounds__(256) void linear_f8_reduce_kernel(LinF8Args a) {
  const int tiles_n = (a.N + BN - 1) / BN, tiles_m = (a.M + BM - 1) / BM, n_tail = tiles_m * tiles_n - a.n_full;
  const int blk = blockIdx.x * 8 + (threadIdx.x >> 5);  // (tile, row, block), blocks fastest
  const int t = blk / (BM * (BN / 128)), in_t = blk - t * (BM * (BN / 128));
  const int r = in_t / (BN / 128), col = in_t % (BN / 128) * 128 + (threadIdx.x & 31) * 4;
  int tm, tn;
  tile_at(a.n_full + t, tiles_m, tiles_n, &tm, &tn);
  const int m = tm * BM + r, n = tn * BN + col;
  const bool in = m < a.M && n < a.N;
  const float* p = a.part + (long)t * (BM * BN) + r * BN + col;
  const long stride = (long)n_tail * (BM * BN);
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  if (in) {
    y = sum_parts<8>(p, a.split, stride);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (a.bias && n + e < a.N) y[e] += bias_at<OUT>(a, n + e);
      if (a.act) y[e] = gelu_tanh(y[e]);
      if (OUT == 2 && n + e >= a.N) y[e] = 0.f;  // (no part of the block's maximum)
    }
  }
  if (OUT != 2) {
    if (in) store_y4<OUT>(a, a.N % 4 == 0, m, n, y, 0.f);
    return;
  }
  float mx = fmaxf(fmaxf(fabsf(y[0]), fabsf(y[1])), fmaxf(fabsf(y[2]), fabsf(y[3])));
  mx = max16(mx);
  mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
  const float sc = f8_scale(mx), inv = 1.0f / sc;
  if (!in) return;
  store_y4<OUT>(a, a.N % 4 == 0, m, n, y, inv);
  if ((threadIdx.x & 31) == 0) a.out_scale[(long)m * ((a.N + 127) / 128) + n / 128] = sc;
}

// Few rows (at most 16 TM): bound by the weights' bytes, and when those are few
// by the launch and a chain of loads (8 x 1152 x 6912: 8 MB, 6.8 us, 1.2 TB/s).
// A workgroup owns 16 outputs of every row; its waves divide the blocks of k, with
// the fragments of the next blocks loading from global memory while one is
// multiplied, and add their sums through LDS in order.  e4m3, whose scales span
// 128 outputs: fp32 sums go to part[M][part_row(N)], and the finish kernel quantises them.
__host__ __device__ __forceinline__ int part_row(int N) { return (N + 3) & ~3; }  // of part: whole groups of four
template <int TM, int NW, int OUT>
__global__ __launch_bounds__(NW * 64) void linear_f8_rows_kernel(LinF8Args a) {
  constexpr bool WIDE = OUT == 0;
  constexpr int U = TM == 1 ? 4 : 2;  // blocks of k in flight per wave
  __shared__ f32x4 sum[NW][TM][64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int n0 = blockIdx.x * 16, KB = (a.K + 127) / 128;
  const uint8_t* wrow = a.w + (long)min(n0 + r16, a.N - 1) * a.K;
  const float* ws = a.w_scale + (long)(n0 / 128) * KB;
  const uint8_t* arow[TM];
  const float* srow[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const long m = min(i * 16 + r16, a.M - 1);
    arow[i] = a.a + m * a.K;
    srow[i] = a.a_scale + m * KB;
  }
  auto frag = [&](const uint8_t* row, int kb) {
    const int k = kb * 128 + kq * 32;
    const u32x4 z = {0u, 0u, 0u, 0u};
    const u32x4 lo = k < a.K ? *(const u32x4*)(row + k) : z, hi = k + 16 < a.K ? *(const u32x4*)(row + k + 16) : z;
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };
  f32x4 acc[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  i32x8 wf[U], af[U][TM];
  float sw[U], sa[U][TM];
  auto load = [&](int u, int kb) {
    if (kb >= KB) return;
    wf[u] = frag(wrow, kb);
    sw[u] = ws[kb];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      af[u][i] = frag(arow[i], kb);
      sa[u][i] = srow[i][kb];
    }
  };
#pragma unroll
  for (int u = 0; u < U; ++u) load(u, wave + u * NW);
  for (int kb = wave; kb < KB; kb += U * NW)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (kb + u * NW >= KB) break;
#pragma unroll
      for (int i = 0; i < TM; ++i) acc[i] += sa[u][i] * sw[u] * mfma_block<WIDE>(wf[u], af[u][i]);
      load(u, kb + (u + U) * NW);
    }
#pragma unroll
  for (int i = 0; i < TM; ++i) sum[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < TM; i += NW) {
    f32x4 y = sum[0][i][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) y += sum[w][i][lane];
    const int m = i * 16 + r16, n = n0 + kq * 4;
    if (m >= a.M || n >= a.N) continue;
    if (OUT == 2) {
      *(f32x4*)(a.part + (long)m * part_row(a.N) + n) = y;
      continue;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (a.bias && n + e < a.N) y[e] += bias_at<OUT>(a, n + e);
      if (a.act) y[e] = gelu_tanh(y[e]);
    }
    store_y4<OUT>(a, a.N % 4 == 0, m, n, y, 0.f);
  }
}

// Bias, activation and quantisation of few rows' fp32 sums.  32 lanes take the
// 128 columns of one block of one row.
__global__ __launch_bounds__(256) void linear_f8_finish_kernel(LinF8Args a) {
  const int nb = (a.N + 127) / 128, blk = blockIdx.x * 8 + (threadIdx.x >> 5), bc = min(blk, a.M * nb - 1);
  const int m = bc / nb, n = (bc - m * nb) * 128 + (threadIdx.x & 31) * 4;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  if (n < a.N) {
    y = *(const f32x4*)(a.part + (long)m * part_row(a.N) + n);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (a.bias && n + e < a.N) y[e] += bias_at<2>(a, n + e);
      if (a.act) y[e] = gelu_tanh(y[e]);
      if (n + e >= a.N) y[e] = 0.f;
    }
  }
  float mx = fmaxf(fmaxf(fabsf(y[0]), fabsf(y[1])), fmaxf(fabsf(y[2]), fabsf(y[3])));
  mx = max16(mx);
  mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
  const float sc = f8_scale(mx);
  if (blk >= a.M * nb) return;
  if (n < a.N) store_y4<2>(a, a.N % 4 == 0, m, n, y, 1.0f / sc);
  if ((threadIdx.x & 31) == 0) a.out_scale[blk] = sc;
}

// The plan of a product: at most 64 rows go to the kernel of few rows; else
// tiles of 256 x 256 or 192 x 256 (one workgroup per CU; not for fp32 outputs,
// whose widened operands need the registers) or 128 x 128 (two per CU), the last
// round's tiles divided over k into up to eight ranges, by the least estimate of
//   `round` us for a round of up to `slots` tiles + `block` us for each of its
//   blocks of k (`half` where it leaves half of the slots empty),
//   `join` us for adding ranges up.
// Measured at 1024 .. 17550 rows, in tiles of 128, 192 and 256:
//   2048 x 1152 x 4608   27.7, 22.8, 27.9 us     8192 x 4608 x 1152  68, 54, 61
//   6000 x 4096 x 4096   124, 101, 117           4352 x 3072 x 3072  63, 60, 49
//   17550 x 12288 x 3072 904, 768, 724           1024 x 1152 x 4608  16, 19, 25
// Ranges of two blocks did not pay: 1024 x 1152 x 1152 23 us in four ranges, 10.1
// us whole; 1024 x 4608 x 1152 25 against 32.
static constexpr long MAX_THREADS = 1L << 32;  // a grid has fewer
// Waves of a workgroup of the kernel of few rows: at least two blocks of k for each;
// sixteen have the registers of up to 32 rows.
static int rows_waves(int M, int KB) { return KB < 16 ? 4 : KB < 32 || M > 32 ? 8 : 16; }

LinF8Plan linear_fp8_plan(int M, int N, int K, int dtype) {
  LinF8Plan p{};
  p.split = 1;
  const int KB = (K + 127) / 128;
  if (M <= 64) {
    if ((long)((N + 15) / 16) * rows_waves(M, KB) * 64 >= MAX_THREADS) p.tile = -1;
    p.bytes = dtype == 2 ? (size_t)M * part_row(N) * 4 : 0;
    return p;
  }
  p.tile = -1;
  double best = 0;
  struct Tile {
    int bm, bn, slots;
    double round, block, half, join;
  };
  static const Tile tiles[3] = {{128, 128, 512, 4, 1.3, 0.7, 6}, {192, 256, 256, 9, 1.4, 1.4, 10}, {256, 256, 256, 11, 1.85, 1.85, 10}};
  for (const Tile& c : tiles) {
    if (dtype == 0 && c.bm != 128) break;
    const long t = (long)((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn), full = t / c.slots, rem = t % c.slots;
    for (int s = 1; s <= 8 && (s == 1 || (KB >= 4 * s && rem * s <= c.slots && rem > 0)); ++s) {
      const double part = rem * s <= 256 ? c.half : c.block;
      const double us = full * (c.round + KB * c.block) + (rem ? c.round + KB * part / s + (s == 1 ? 0 : c.join) : 0);
      if ((t + c.slots) * 512 >= MAX_THREADS || (p.tile > 0 && us >= best)) continue;
      best = us;
      p.tile = c.bm;
      p.split = s;
      p.n_full = (int)(s > 1 ? t - rem : t);
      p.bytes = s > 1 ? (size_t)s * rem * c.bm * c.bn * 4 : 0;
    }
  }
  return p;
}

template <int BM, int BN, int WM, int WN, int OUT>
static void launch_tile(const LinF8Args& a, hipStream_t st) {
  const int t = ((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN), tail = t - a.n_full;
  hipLaunchKernelGGL((linear_f8_tile_kernel<BM, BN, WM, WN, OUT>), dim3(a.n_full + tail * a.split), dim3(WM * WN * 64), 0, st, a);
  if (tail)
    hipLaunchKernelGGL((linear_f8_reduce_kernel<BM, BN, OUT>), dim3(tail * BM * (BN / 128) / 8), dim3(256), 0, st, a);
}

template <int TM, int OUT>
static void launch_rows(const LinF8Args& a, hipStream_t st) {
  const dim3 grid((a.N + 15) / 16);
  const int nw = rows_waves(a.M, (a.K + 127) / 128);
  if (nw == 4) hipLaunchKernelGGL((linear_f8_rows_kernel<TM, 4, OUT>), grid, dim3(256), 0, st, a);
  else if (nw == 8) hipLaunchKernelGGL((linear_f8_rows_kernel<TM, 8, OUT>), grid, dim3(512), 0, st, a);
  else hipLaunchKernelGGL((linear_f8_rows_kernel<TM == 4 ? 2 : TM, 16, OUT>), grid, dim3(1024), 0, st, a);
  if (OUT == 2)
    hipLaunchKernelGGL(linear_f8_finish_kernel, dim3((a.M * ((a.N + 127) / 128) + 7) / 8), dim3(256), 0, st, a);
}

template <int OUT>
static void launch_out(const LinF8Args& a, int tile, hipStream_t st) {
  if (tile == 0) {
    if (a.M <= 16) launch_rows<1, OUT>(a, st);
    else if (a.M <= 32) launch_rows<2, OUT>(a, st);
    else launch_rows<4, OUT>(a, st);
    return;
  }
  if constexpr (OUT != 0) {
    if (tile == 256) return launch_tile<256, 256, 4, 2, OUT>(a, st);
    if (tile == 192) return launch_tile<192, 256, 4, 2, OUT>(a, st);
  }
  launch_tile<128, 128, 4, 2, OUT>(a, st);
}

hipError_t launch_linear_fp8(const LinF8Args& a, int tile, hipStream_t st) {
  if (a.dtype == 0) launch_out<0>(a, tile, st);
  else if (a.dtype == 1) launch_out<1>(a, tile, st);
  else launch_out<2>(a, tile, st);
  return hipGetLastError();
}

// ------------------------------------------------------------------ quantisation
// Bound by memory: 12288 x 3072 bf16 weights 22 us, 5.1 TB/s, the rate of a large
// copy; small activations by the launch (256 x 1152: the kernel 2.3 us).
// Rows: 16 lanes take the 128 columns of one block, 16 bytes of bf16 (32 of fp32)
// each.
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
