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

// Stores eight consecutive outputs of row m from column n on, as far as there are such.  MXFP4: the four
// lanes of a quad hold a block of 32 (out is a multiple of 32: a block is whole or not there).
template <int OUT>
__device__ __forceinline__ void store_y8(const LinF4Args& a, int m, int n, const float (&y)[8]) {
  const long o = (long)m * a.N + n;
  if (OUT == 3) {
    uint32_t mx = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) mx = max(mx, abs_bits(y[e]));
    const uint32_t s = f4_scale(max_quad(mx));
    if (m >= a.M || n >= a.N) return;
    *(uint32_t*)((uint8_t*)a.out + o / 2) = pack_f4x8(y, s);
    if (n % 32 == 0) {
      uint8_t* p = a.out_scale + f4_scale_at(a.M, m, n / 32);
      *p = (uint8_t)s;
      if (n + 32 == a.N)  // the scales behind the last column
        for (int b = a.N / 32; b & 7; ++b) *++p = 0;
    }
    return;
  }
  if (m >= a.M || n >= a.N) return;
  if (a.N % 8 == 0) {
    if (OUT == 1) {
      *(u32x4*)((bf16_t*)a.out + o) = u32x4{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
    } else {
      *(f32x4*)((float*)a.out + o) = f32x4{y[0], y[1], y[2], y[3]};
      *(f32x4*)((float*)a.out + o + 4) = f32x4{y[4], y[5], y[6], y[7]};
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (n + e < a.N) {
        if (OUT == 1) ((bf16_t*)a.out)[o + e] = f2bf(y[e]);
        else ((float*)a.out)[o + e] = y[e];
      }
  }
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
  const int n0 = blockIdx.x * 16;
  const int KB = (a.K + 127) / 128;
  const long half = a.K / 2;
  const int wn = min(n0 + r16, a.N - 1);
  const uint8_t* wrow = a.w + (long)wn * half;
  const uint8_t* arow[TM];
  int am[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    am[i] = min(i * 16 + r16, a.M - 1);
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
    const int m = i * 16 + r16, n = n0 + kq * 4;
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
  const long at = min(i, groups - 1);  // (whole quads)
  const int m = (int)(at / (a.N / 8)), n = (int)(at - (long)m * (a.N / 8)) * 8;
  float y[8];
  const float* p = a.part + (long)m * a.N + n;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = p[e];
    if (a.bias) y[e] += bias_at<3>(a, n + e);
    if (a.act) y[e] = gelu_tanh(y[e]);
  }
  store_y8<3>(a, i < groups ? m : a.M, n, y);
}

// Order of the tiles: groups of eight row tiles x all column tiles, rows fastest, so that what runs at
// once on an XCD shares operands in its L2.
__device__ __forceinline__ void tile_at(int tile, int tiles_m, int tiles_n, int* tm, int* tn) {
  const int per = 8 * tiles_n, grp = tile / per, gm = min(8, tiles_m - grp * 8), in_grp = tile - grp * per;
  *tm = grp * 8 + in_grp % gm;
  *tn = in_grp / gm;
}

// 4 bytes per lane from sbase + voff (sbase wave-uniform) into LDS at (wave-uniform) lds_base + 4 * lane.
__device__ __forceinline__ void dma_4s(const void* sbase, unsigned voff, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(lds_base), "v"(voff), "s"(sbase)
               : "memory", "m0");
}

// Many rows: a workgroup of WM x WN waves owns BM rows x BN outputs.  Stages of 128 k (64 bytes and four
// scales per row of both operands) go HBM -> LDS by DMA into a ring of S slots; 16-byte chunk c of row r
// lies at c ^ (r / 4 & 3), so that 16 rows of a fragment read come from distinct banks.  The weights are
// the A operand of v_mfma_scale_f32_32x32x64_f8f6f4 and the activations the B operand: a lane holds 16
// outputs of one activation row, block scales of both operands go in with the product.
template <int BM, int BN, int WM, int WN, int S, int OUT>
__global__ __launch_bounds__(WM * WN * 64) void linear_f4_tile_kernel(LinF4Args a) {
  constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr int IPW = (BM + BN) / (16 * NW);           // 1 KB DMA instructions per wave and stage
  constexpr int SU = (BM + BN) / 64, SPW = (SU + NW - 1) / NW;  // 256-byte ones of scales
  constexpr int PER = IPW + SPW;
  constexpr int SCALES = (BM + BN) * 64, STAGE = (BM + BN) * 68;  // W rows, A rows; their scales
  static_assert(BM % (16 * NW) == 0 && BN % (16 * NW) == 0 && BN % 64 == 0 && BM % 64 == 0 && S >= 3, "tile split");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S * STAGE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, kq = lane >> 5;
  const int tiles_n = (a.N + BN - 1) / BN, tiles_m = (a.M + BM - 1) / BM;
  int tm, tn;
  tile_at(xcd_remap(blockIdx.x, tiles_m * tiles_n), tiles_m, tiles_n, &tm, &tn);
  const int wm = wave % WM, wn = wave / WM;
  const int KB = (a.K + 127) / 128, half = a.K / 2;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));

  // DMA: instruction t of this wave covers rows 16 q .. 16 q + 15, q = wave + NW t, of the stage's W rows
  // then A rows.  Past K a row's last chunk comes again: its scales there are made 0 (2^-127) below.
  unsigned off[IPW], soff[SPW];
#pragma unroll
  for (int t = 0; t < IPW; ++t) {
    const int R = (wave + NW * t) * 16 + (lane >> 2);
    off[t] = (unsigned)(t * NW * 16 < BN ? min(R, a.N - 1 - tn * BN) : min(R - BN, a.M - 1 - tm * BM)) * (unsigned)half;
  }
  int su[SPW];
#pragma unroll
  for (int t = 0; t < SPW; ++t) {
    su[t] = min(wave + NW * t, SU - 1);
    const int R = su[t] * 64 + lane;
    soff[t] = (unsigned)(su[t] * 64 < BN ? min(R, a.N - 1 - tn * BN) : min(R - BN, a.M - 1 - tm * BM)) * 8u;
  }
  const unsigned chunk = (unsigned)((lane & 3) ^ (lane >> 4)) * 16u;
  const uint8_t* wb = a.w + (long)tn * BN * half;
  const uint8_t* ab = a.a + (long)tm * BM * half;
  auto issue_one = [&](int kb, int slot, int t) {
    const unsigned dst = lds0 + (unsigned)(slot * STAGE);
    if (t < IPW) {
      const unsigned k = min((unsigned)kb * 64u + chunk, (unsigned)half - 16u);
      dma_16s(t * NW * 16 < BN ? wb : ab, off[t] + k, dst + (unsigned)((wave + NW * t) * 1024));
    } else {
      const int u = su[t - IPW];
      const uint8_t* sb = u * 64 < BN ? a.w_scale + ((long)(kb >> 1) * a.N + tn * BN) * 8 : a.a_scale + ((long)(kb >> 1) * a.M + tm * BM) * 8;
      dma_4s(sb, soff[t - IPW] + (unsigned)(kb & 1) * 4u, dst + (unsigned)(SCALES + u * 256));
    }
  };

  f32x16 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.f;

  // fragment f < TN: of W, else of A; k step s of the stage's two
  const int wrow = wn * (BN / WN) + r32, arow = BN + wm * (BM / WM) + r32;
  const int ch0 = (kq ^ ((lane >> 2) & 3)) << 4;
  auto frag = [&](int slot, int f, int s) {
    const int row = f < TN ? wrow + f * 32 : arow + (f - TN) * 32;
    return *(const u32x4*)(smem + slot * STAGE + row * 64 + (ch0 ^ (s << 5)));
  };
  auto scale = [&](int slot, int f) {
    const int row = f < TN ? wrow + f * 32 : arow + (f - TN) * 32;
    return *(const uint32_t*)(smem + slot * STAGE + SCALES + row * 4);
  };
  constexpr int F = TN + TM;
  u32x4 f0[F], f1[F];
  uint32_t raw[F], sc[F];

#pragma unroll
  for (int p = 0; p < S - 1; ++p)
    if (p < KB)
#pragma unroll
      for (int t = 0; t < PER; ++t) issue_one(p, p, t);
  if (KB >= S - 1) wait_vmcnt<(S - 2) * PER>();
  else wait_vmcnt<0>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int f = 0; f < F; ++f) f0[f] = frag(0, f, 0), raw[f] = scale(0, f);

  int slot = 0, fill = S - 1;
  // MORE: there is a stage S - 1 ahead to load
  auto step = [&](int kb, auto MORE) {
    constexpr bool more = decltype(MORE)::value;
    const int next = slot + 1 == S ? 0 : slot + 1;
    const int left = a.K / 32 - kb * 4;
    const uint32_t mask = more || left >= 4 ? ~0u : (1u << (8 * left)) - 1u;
#pragma unroll
    for (int f = 0; f < F; ++f) sc[f] = (raw[f] & mask) >> (8 * kq);
    // the first k step, beside it the second one's fragments and the DMA of the stage S - 1 ahead
#pragma unroll
    for (int x = 0; x < TN * TM; ++x) {
      const int j = x / TM, i = x % TM;
      constexpr int RP = (F + TN * TM - 1) / (TN * TM), DP = (PER + TN * TM - 1) / (TN * TM);
#pragma unroll
      for (int y = 0; y < RP; ++y)
        if (x * RP + y < F) f1[x * RP + y] = frag(slot, x * RP + y, 1);
      acc[j][i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(f0[j]), operand(f0[TN + i]), acc[j][i], 4, 4, 0, sc[j],
                                                                  0, sc[TN + i]);
      if (more)
#pragma unroll
        for (int y = 0; y < DP; ++y)
          if (x * DP + y < PER) issue_one(kb + S - 1, fill, x * DP + y);
      __builtin_amdgcn_sched_barrier(0);
    }
    // the second, in whose middle the waves meet: the next stage has landed, and nobody reads the last
#pragma unroll
    for (int x = 0; x < TN * TM; ++x) {
      const int j = x / TM, i = x % TM;
      constexpr int H = TN * TM / 2, RP = (F + H - 1) / H;
      if (x == H) {
        if (more) wait_vmcnt<(S - 2) * PER>();
        else wait_vmcnt<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      if (x >= H)
#pragma unroll
        for (int y = 0; y < RP; ++y) {
          const int u = (x - H) * RP + y, both = 2 * (TN < TM ? TN : TM);  // of W and of A in turn
          const int f = u < both ? u % 2 * TN + u / 2 : TN < TM ? u : u - TM;
          if (u < F) f0[f] = frag(next, f, 0), raw[f] = scale(next, f);
        }
      acc[j][i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(f1[j]), operand(f1[TN + i]), acc[j][i], 4, 4, 2, sc[j],
                                                                  2, sc[TN + i]);
      __builtin_amdgcn_sched_barrier(0);
    }
    slot = next;
    fill = fill + 1 == S ? 0 : fill + 1;
  };
  int kb = 0;
  for (; kb + S - 1 < KB; ++kb) step(kb, std::true_type());
  for (; kb < KB; ++kb) step(kb, std::false_type());

  // Epilogue, 32 rows of the wave at a time through LDS, so that its code is short (it runs once, and
  // every line of it is fetched) and its stores are whole: element e of a lane is output 8 (e / 4) + 4 kq +
  // e % 4 of its row; read back, a lane has eight outputs in a row, the same ones of every row it takes.
  constexpr int WC = BN / WN, PITCH = WC + 4, LPR = WC / 8, RPI = 64 / LPR;
  static_assert(NW * 32 * PITCH * 4 <= S * STAGE, "the ring holds the rows");
  float* rows = (float*)smem + wave * 32 * PITCH;
  const int c8 = (lane % LPR) * 8, n = tn * BN + wn * WC + c8;
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = a.bias ? bias_at<OUT>(a, min(n + e, a.N - 1)) : 0.f;
#pragma unroll 1
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int ii = 0; ii < TM; ++ii)
      if (i == ii)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *(f32x4*)(rows + r32 * PITCH + j * 32 + 8 * g + 4 * kq) =
                f32x4{acc[j][ii][4 * g], acc[j][ii][4 * g + 1], acc[j][ii][4 * g + 2], acc[j][ii][4 * g + 3]};
    wave_lds_fence();
#pragma unroll 1
    for (int r0 = lane / LPR; r0 < 32; r0 += 4 * RPI) {  // four rows at once: one alone waits for its reads
      f32x4 v[4][2];
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int h = 0; h < 2; ++h) v[q][h] = *(const f32x4*)(rows + (r0 + q * RPI) * PITCH + c8 + 4 * h);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = v[q][e / 4][e % 4] + bias[e];
        if (a.act)
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = gelu_tanh(y[e]);
        store_y8<OUT>(a, tm * BM + wm * (BM / WM) + i * 32 + r0 + q * RPI, n, y);
      }
    }
    wave_lds_fence();
  }
}

static constexpr long MAX_THREADS = 1L << 32;  // a grid has fewer

static long tiles_of(int M, int N, int bm, int bn) { return (long)((M + bm - 1) / bm) * ((N + bn - 1) / bn); }

LinF4Plan linear_fp4_plan(int M, int N, int K, int dtype) {
  LinF4Plan p{};
  if (M <= 64) {
    if ((long)((N + 15) / 16) * 512 >= MAX_THREADS) p.tile = -1;
    p.bytes = dtype == 3 ? (size_t)M * N * 4 : 0;
    return p;
  }
  if (tiles_of(M, N, 128, 128) * 256 >= MAX_THREADS) {
    p.tile = -1;
    return p;
  }
  p.tile = tiles_of(M, N, 256, 256) >= 256 ? 256 : 128;
  if (const char* f = getenv("F4_TILE")) p.tile = atoi(f);
  return p;
}

template <int OUT>
static void launch_rows(const LinF4Args& a, hipStream_t st) {
  const dim3 grid((a.N + 15) / 16), block(512);
  if (a.M <= 16) hipLaunchKernelGGL((linear_f4_rows_kernel<1, 8, OUT>), grid, block, 0, st, a);
  else if (a.M <= 32) hipLaunchKernelGGL((linear_f4_rows_kernel<2, 8, OUT>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((linear_f4_rows_kernel<4, 8, OUT>), grid, block, 0, st, a);
  if (OUT == 3)
    hipLaunchKernelGGL(linear_f4_finish_kernel, dim3((unsigned)(((long)a.M * (a.N / 8) + 255) / 256)), dim3(256), 0, st, a);
}

template <int BM, int BN, int WM, int WN, int S, int OUT>
static void launch_tile(const LinF4Args& a, hipStream_t st) {
  hipLaunchKernelGGL((linear_f4_tile_kernel<BM, BN, WM, WN, S, OUT>), dim3((unsigned)tiles_of(a.M, a.N, BM, BN)), dim3(WM * WN * 64),
                     0, st, a);
}

template <int OUT>
static void launch_out(const LinF4Args& a, int tile, hipStream_t st) {
  if (tile == 0) launch_rows<OUT>(a, st);
  else if (tile == 256) launch_tile<256, 256, 2, 2, 4, OUT>(a, st);
  else if (tile == 255) launch_tile<256, 128, 2, 2, 4, OUT>(a, st);
  else launch_tile<128, 128, 2, 2, 4, OUT>(a, st);
}

hipError_t launch_linear_fp4(const LinF4Args& a, const LinF4Plan& p, hipStream_t st) {
  if (a.dtype == 0) launch_out<0>(a, p.tile, st);
  else if (a.dtype == 1) launch_out<1>(a, p.tile, st);
  else launch_out<3>(a, p.tile, st);
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
