// Linear layer on MXFP4 operands (ditmi.h: dit_linear_fp4), and the quantisation into such blocks
// and back.
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

// Stores the scale of the block from column n on, and those behind the last column.
__device__ __forceinline__ void store_scale(const LinF4Args& a, int m, int n, uint32_t s) {
  uint8_t* p = a.out_scale + f4_scale_at(a.M, m, n / 32);
  *p = (uint8_t)s;
  if (n + 32 == a.N)
    for (int b = a.N / 32; b & 7; ++b) *++p = 0;
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
    if (n % 32 == 0) store_scale(a, m, n, s);
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

// 4 bytes per lane from gsrc into LDS at (wave-uniform) lds_base + 4 * lane.
__device__ __forceinline__ void dma_4(const void* gsrc, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds_base), "v"(gsrc) : "memory", "m0");
}

// 4 bytes per lane from sbase + voff (sbase wave-uniform) into LDS at (wave-uniform) lds_base + 4 * lane.
__device__ __forceinline__ void dma_4s(const void* sbase, unsigned voff, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(lds_base), "v"(voff), "s"(sbase)
               : "memory", "m0");
}

// Scales of the eight blocks of a panel as a lane needs them: those of its quarter of 128 k (or half of
// 64) in the low byte of each word; behind the last of `left` blocks 0, 2^-127, beside which codes are nothing.
__device__ __forceinline__ u32x2 panel_mask(int left) {
  return u32x2{left >= 4 ? ~0u : (1u << (8 * left)) - 1u, left >= 8 ? ~0u : left <= 4 ? 0u : (1u << (8 * left - 32)) - 1u};
}

// Few rows: bound by the weights' bytes (16 x 18432 x 4608 11 us, 4.1 TB/s), and when those are few by the
// launch and a chain of loads (8 x 1152 x 6912 3.4 us, 77 x 4608 x 1152 4.5).  A workgroup owns 16 outputs (32 where they are quantised: a block) of 16 TM rows; its waves divide the
// panels of 256 k, each with a ring of two of its own that DMA fills, so that no wave waits for another,
// and add their sums through LDS in order.  DMA brings whole lines of eight rows an instruction, laid out as
// the tiles' (loads of fragments, 16 rows at once, take four times as long: 16 x 18432 x 4608 21.6 us,
// against 10.9).  Past K a row's last bytes come again.
template <int TM, int TN, int NW, int OUT>
__global__ __launch_bounds__(NW * 64) void linear_f4_rows_kernel(LinF4Args a) {
  constexpr int U = 2, F = TN + TM, R = 16 * F, PANEL = R * 136, DATA = R / 8, SC = (R + 31) / 32, PER = DATA + SC;
  static_assert(OUT != 3 || TN == 2, "a block of 32");
  __shared__ __attribute__((aligned(1024))) unsigned char ring[NW * U * PANEL];  // rows of W, rows of A; their scales
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int n0 = blockIdx.x * 16 * TN, m0 = blockIdx.y * 16 * TM, panels = (a.K + 255) / 256;
  const long half = a.K / 2;
  unsigned char* mine = ring + wave * U * PANEL;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(mine));

  // instruction t: rows 8 t .. 8 t + 7 of W, then of A; of the scales: rows 32 t .. 32 t + 31
  auto w_row = [&](int r) { return (long)min(n0 + r, a.N - 1); };
  auto a_row = [&](int r) { return (long)min(m0 + r - 16 * TN, a.M - 1); };
  const uint8_t *src[DATA], *sc_src[SC];
  long sc_step[SC];
#pragma unroll
  for (int t = 0; t < DATA; ++t)
    src[t] = t < 2 * TN ? a.w + w_row(8 * t + (lane >> 3)) * half : a.a + a_row(8 * t + (lane >> 3)) * half;
#pragma unroll
  for (int t = 0; t < SC; ++t) {
    const int r = min(32 * t + (lane >> 1), R - 1);
    sc_src[t] = (r < 16 * TN ? a.w_scale + w_row(r) * 8 : a.a_scale + a_row(r) * 8) + (lane & 1) * 4;
    sc_step[t] = (r < 16 * TN ? a.N : a.M) * 8L;
  }
  auto issue = [&](int p, int u) {
    const unsigned dst = lds0 + (unsigned)(u * PANEL);
#pragma unroll
    for (int t = 0; t < DATA; ++t) {
      const int chunk = (lane & 7) ^ ((4 * t + (lane >> 4)) & 7);
      dma_16(src[t] + min(p * 128L + chunk * 16, half - 16), dst + (unsigned)(t * 1024));
    }
#pragma unroll
    for (int t = 0; t < SC; ++t)
      if (32 * t + (lane >> 1) < R) dma_4(sc_src[t] + p * sc_step[t], dst + (unsigned)(R * 128 + t * 256));
  };
  f32x4 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int count = (panels - wave + NW - 1) / NW;  // panels wave, wave + NW, ...
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (u < count) issue(wave + u * NW, u);
  for (int i0 = 0; i0 < count; i0 += U)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int n = i0 + u, p = wave + n * NW;
      if (n >= count) break;
      if (n + U <= count) wait_vmcnt<(U - 1) * PER>();  // (the later ones may be on their way)
      else wait_vmcnt<0>();
      const unsigned char* at = mine + u * PANEL;
      const u32x2 mask = panel_mask(a.K / 32 - p * 8);
      u32x4 fr[F][2];
      uint32_t sc[F][2];
#pragma unroll
      for (int f = 0; f < F; ++f) {
        const u32x2 raw = *(const u32x2*)(at + R * 128 + (f * 16 + r16) * 8);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          fr[f][h] = *(const u32x4*)(at + (f * 16 + r16) * 128 + (((h * 4 + kq) ^ ((r16 >> 1) & 7)) << 4));
          sc[f][h] = (raw[h] & mask[h]) >> (8 * kq);
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int i = 0; i < TM; ++i)
            acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(fr[j][h]), operand(fr[TN + i][h]), acc[j][i], 4,
                                                                         4, 0, sc[j][h], 0, sc[TN + i][h]);
      if (n + U < count) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot has been read
        issue(p + U * NW, u);
      }
    }
  __syncthreads();
  f32x4(*sum)[TN][TM][64] = (f32x4(*)[TN][TM][64])ring;
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i) sum[wave][j][i][lane] = acc[j][i];
  __syncthreads();
  // a lane: outputs 4 kq .. 4 kq + 3 of each 16, of row r16 of each 16
  for (int i = wave; i < TM; i += NW) {
    const int m = m0 + i * 16 + r16, n = n0 + kq * 4;
    float y[TN][4];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      f32x4 t = sum[0][j][i][lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) t += sum[w][j][i][lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[j][e] = t[e];
        if (a.bias) y[j][e] += bias_at<OUT>(a, min(n + j * 16 + e, a.N - 1));
        if (a.act) y[j][e] = gelu_tanh(y[j][e]);
      }
    }
    if constexpr (OUT == 3) {
      uint32_t mx = 0u;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = max(mx, abs_bits(y[j][e]));
      const auto p16 = __builtin_amdgcn_permlane16_swap(mx, mx, false, false);
      mx = max(p16[0], p16[1]);
      const auto p32 = __builtin_amdgcn_permlane32_swap(mx, mx, false, false);
      const uint32_t s = f4_scale(max(p32[0], p32[1]));
      if (m >= a.M) continue;
      const float v[8] = {y[0][0], y[0][1], y[0][2], y[0][3], y[1][0], y[1][1], y[1][2], y[1][3]};
      const uint32_t c = pack_f4x8(v, s);
      uint8_t* o = (uint8_t*)a.out + ((long)m * a.N + n) / 2;
      *(uint16_t*)o = (uint16_t)c;
      *(uint16_t*)(o + 8) = (uint16_t)(c >> 16);
      if (kq == 0) store_scale(a, m, n0, s);
    } else {
      if (m >= a.M) continue;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int nj = n + j * 16;
        const long o = (long)m * a.N + nj;
        if (nj < a.N && a.N % 4 == 0) {
          if (OUT == 0) *(f32x4*)((float*)a.out + o) = f32x4{y[j][0], y[j][1], y[j][2], y[j][3]};
          else *(u32x2*)((bf16_t*)a.out + o) = u32x2{pack_bf16x2(y[j][0], y[j][1]), pack_bf16x2(y[j][2], y[j][3])};
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (nj + e < a.N) {
              if (OUT == 0) ((float*)a.out)[o + e] = y[j][e];
              else ((bf16_t*)a.out)[o + e] = f2bf(y[j][e]);
            }
        }
      }
    }
  }
}

__host__ __device__ __forceinline__ int part_row(int N) { return (N + 7) & ~7; }  // of part: whole groups of eight

// Order of the tiles: groups of eight row tiles x all column tiles, rows fastest, so that what runs at
// once on an XCD shares operands in its L2.
__device__ __forceinline__ void tile_at(int tile, int tiles_m, int tiles_n, int* tm, int* tn) {
  const int per = 8 * tiles_n, grp = tile / per, gm = min(8, tiles_m - grp * 8), in_grp = tile - grp * per;
  *tm = grp * 8 + in_grp % gm;
  *tn = in_grp / gm;
}

// Many rows: a workgroup of WM x WN waves owns BM rows x BN outputs.  Stages of 256 k (128 bytes, whole
// cache lines, and eight scales per row of both operands) go HBM -> LDS by DMA into a ring of S slots;
// 16-byte chunk c of row r lies at c ^ (r / 2 & 7), so that 16 rows of a fragment read come from distinct
// banks.  The weights are the A operand of v_mfma_scale_f32_32x32x64_f8f6f4 and the activations the B
// operand: a lane holds 16 outputs of one activation row, block scales of both operands go in with the
// product (of 32 x 32 x 64: a loop of these alone reaches 6.5 PFLOP/s on random codes, of 16 x 16 x 128 5.4).
//
// Bound by power when it runs long: 17550 x 18432 x 4608 654 us, 4.6 PFLOP/s, and 489 us on codes of zero.
// Beside that a 256 x 256 tile's panel takes 2048 cycles of products, 1300 of the CU's address unit for its
// DMA, and some 2100 for its 68 KB from the L2.  Short ones: 4096 x 4608 x 1152 18 us, of which 11 are 18
// panels and the rest the launch, the first loads and the epilogue.  Many rows over short k by what every round
// of workgroups costs beside its panels, for one workgroup fills a CU's LDS and nothing runs beside its first
// loads and its epilogue: 17550 x 1152 x 4608 93 us, 2.0 PFLOP/s (89 and, with GELU, 109 into 4 bits, 120 into
// fp32), 17550 x 3072 x 9216 281 us, 3.5 PFLOP/s.
template <int BM, int BN, int WM, int WN, int S, int OUT>
__global__ __launch_bounds__(WM * WN * 64) void linear_f4_tile_kernel(LinF4Args a) {
  constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, T = TM * TN, F = TN + TM;
  constexpr int IPW = (BM + BN) / (8 * NW);   // 1 KB DMA instructions per wave and stage
  constexpr int SU = (BM + BN) / 32, SPW = (SU + NW - 1) / NW;  // 256-byte ones of scales
  constexpr int PER = IPW + SPW;
  constexpr int SCALES = (BM + BN) * 128, STAGE = (BM + BN) * 136;  // W rows, A rows; their scales
  static_assert(NW % 2 == 0 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && BM % 32 == 0 && BN % 32 == 0 && S >= 2, "tile split");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S * STAGE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, kq = lane >> 5;
  const int tiles_n = (a.N + BN - 1) / BN, tiles_m = (a.M + BM - 1) / BM;
  const int unit = xcd_remap(blockIdx.x, tiles_m * tiles_n * a.split), part = unit / (tiles_m * tiles_n);
  int tm, tn;
  tile_at(unit - part * (tiles_m * tiles_n), tiles_m, tiles_n, &tm, &tn);
  const int wm = wave % WM, wn = wave / WM;
  const int panels = (a.K + 255) / 256, half = a.K / 2;
  const int kb0 = (int)((long)panels * part / a.split), KB = (int)((long)panels * (part + 1) / a.split);
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));

  // DMA: instruction t of this wave covers rows 8 q .. 8 q + 7, q = wave + NW t, of the stage's W rows then
  // A rows (of the scales: rows 32 q .. 32 q + 31).  Past K a row's last chunk comes again: its scales there
  // are made 0 (2^-127) below.
  unsigned off[IPW], soff[SPW];
#pragma unroll
  for (int t = 0; t < IPW; ++t) {
    const int R = (wave + NW * t) * 8 + (lane >> 3);
    off[t] = (unsigned)(t * NW * 8 < BN ? min(R, a.N - 1 - tn * BN) : min(R - BN, a.M - 1 - tm * BM)) * (unsigned)half;
  }
#pragma unroll
  for (int t = 0; t < SPW; ++t) {
    const int u = min(wave + NW * t, SU - 1), R = u * 32 + (lane >> 1);  // (the last one more than once)
    soff[t] = (unsigned)(u * 32 < BN ? min(R, a.N - 1 - tn * BN) : min(R - BN, a.M - 1 - tm * BM)) * 8u + (lane & 1) * 4u;
  }
  const unsigned chunk = (unsigned)((lane & 7) ^ ((wave & 1) * 4 + (lane >> 4))) * 16u;
  const uint8_t* wb = a.w + (long)tn * BN * half;
  const uint8_t* ab = a.a + (long)tm * BM * half;
  auto issue_one = [&](int kb, int slot, int t) {
    const unsigned dst = lds0 + (unsigned)(slot * STAGE);
    if (t < IPW) {
      const unsigned k = min((unsigned)kb * 128u + chunk, (unsigned)half - 16u);
      dma_16s(t * NW * 8 < BN ? wb : ab, off[t] + k, dst + (unsigned)((wave + NW * t) * 1024));
    } else {
      const int u = min(wave + NW * (t - IPW), SU - 1);
      const uint8_t* sb = u * 32 < BN ? a.w_scale + ((long)kb * a.N + tn * BN) * 8 : a.a_scale + ((long)kb * a.M + tm * BM) * 8;
      dma_4s(sb, soff[t - IPW], dst + (unsigned)(SCALES + u * 256));
    }
  };

  f32x16 acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.f;

  // fragment f < TN: of W, else of A; k step s of the stage's four
  const int wrow = wn * (BN / WN) + r32, arow = BN + wm * (BM / WM) + r32;
  const int ch0 = (kq ^ ((lane >> 1) & 7)) << 4;
  auto row_of = [&](int f) { return f < TN ? wrow + f * 32 : arow + (f - TN) * 32; };
  auto frag = [&](int slot, int f, int s) { return *(const u32x4*)(smem + slot * STAGE + row_of(f) * 128 + (ch0 ^ (s << 5))); };
  auto scale = [&](int slot, int f) { return *(const u32x2*)(smem + slot * STAGE + SCALES + row_of(f) * 8); };
  // the order in which fragments are read: of W and of A in turn
  auto nth = [](int u) { return u < 2 * (TN < TM ? TN : TM) ? u % 2 * TN + u / 2 : TN < TM ? u : u - TM; };
  if constexpr (T == 1) {
    // One product a step: too few to read the next step's operands beside them, so all of the next panel's
    // are read beside those of one (77 x 18432 x 4608 in tiles of 32 x 64 19.8 us against 22.5; with two
    // products a step the other order is the faster one, 9.7 us against 10.3 at 77 x 4608 x 1152).
    u32x4 fr[2][4][F];
    u32x2 raw[2][F];
    auto read = [&](int slot, int b) {
#pragma unroll
      for (int f = 0; f < F; ++f) {
        raw[b][f] = scale(slot, f);
#pragma unroll
        for (int s = 0; s < 4; ++s) fr[b][s][f] = frag(slot, f, s);
      }
    };
#pragma unroll
    for (int p = 0; p < S; ++p)
      if (kb0 + p < KB)
#pragma unroll
        for (int t = 0; t < PER; ++t) issue_one(kb0 + p, p, t);
    if (kb0 + S <= KB) wait_vmcnt<(S - 1) * PER>();
    else wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read(0, 0);
    int slot = 0;
    auto panel = [&](int kb, auto CUR, auto MORE) {  // MORE: there is a panel S ahead to load
      constexpr int b = decltype(CUR)::value;
      constexpr bool more = decltype(MORE)::value;
      const int next = slot + 1 == S ? 0 : slot + 1;
      // the waves meet: the next panel has landed, and this one, in registers, leaves its slot
      if (more) wait_vmcnt<(S - 2) * PER>();
      else wait_vmcnt<0>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      read(next, 1 - b);
      if (more)
#pragma unroll
        for (int t = 0; t < PER; ++t) issue_one(kb + S, slot, t);
      const u32x2 mask = more ? u32x2{~0u, ~0u} : panel_mask(a.K / 32 - kb * 8);
      uint32_t sc[2][F];
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int h = 0; h < 2; ++h) sc[h][f] = (raw[b][f][h] & mask[h]) >> (8 * kq);
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int x = 0; x < T; ++x) {
          const int j = x / TM, i = x % TM;
          const uint32_t sw = sc[s >> 1][j], sa = sc[s >> 1][TN + i];
          const i32x8 wf = operand(fr[b][s][j]), af = operand(fr[b][s][TN + i]);
          acc[j][i] = s & 1 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf, af, acc[j][i], 4, 4, 2, sw, 2, sa)
                            : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf, af, acc[j][i], 4, 4, 0, sw, 0, sa);
        }
      slot = next;
    };
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    int kb = kb0;
    for (; kb + 1 + S < KB; kb += 2) panel(kb, even, std::true_type()), panel(kb + 1, odd, std::true_type());
    if (kb + S < KB) {
      panel(kb++, even, std::true_type());
      for (; kb < KB; kb += 2) {
        panel(kb, odd, std::false_type());
        if (kb + 1 < KB) panel(kb + 1, even, std::false_type());
      }
    } else {
      for (; kb < KB; kb += 2) {
        panel(kb, even, std::false_type());
        if (kb + 1 < KB) panel(kb + 1, odd, std::false_type());
      }
    }
  } else {
    u32x4 fr[2][F];
    u32x2 raw[F];
    uint32_t sc[2][F];

    // The DMA of a stage is spread over three of its four steps: a CU takes 16 cycles for an instruction, and a
    // wave that issues them faster waits with its products.  Instruction t follows product issue_at(t) behind
    // the barrier that frees the slot; the first EARLY thus the stage's last step, the others the next one's.
    constexpr auto issue_at = [](int t) { return t * 3 * T / PER; };
    constexpr int EARLY = (PER + 2) / 3;  // issue_at(t) < T
    static_assert(issue_at(EARLY - 1) < T && issue_at(EARLY) >= T && issue_at(PER - 1) < 3 * T, "a third follows the last step");
#pragma unroll
    for (int p = 0; p < S; ++p)
      if (kb0 + p < KB)
#pragma unroll
        for (int t = 0; t < (p < S - 1 ? PER : EARLY); ++t) issue_one(kb0 + p, p, t);
    if (kb0 + S <= KB) wait_vmcnt<(S - 2) * PER + EARLY>();
    else wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int u = 0; u < F; ++u) {
      const int f = nth(u);
      fr[0][f] = frag(0, f, 0), raw[f] = scale(0, f);
    }

    int slot = 0;
    // MORE: 2, there is a stage S ahead to load; 1, one S - 1 ahead; 0, none
    auto stage = [&](int kb, auto MORE) {
      constexpr int more = decltype(MORE)::value;
      const int prev = slot == 0 ? S - 1 : slot - 1;
      const int next = slot + 1 == S ? 0 : slot + 1;
      const int left = a.K / 32 - kb * 8;  // blocks of 32
      const u32x2 mask = more == 2 ? u32x2{~0u, ~0u} : panel_mask(left);
#pragma unroll
      for (int f = 0; f < F; ++f) sc[0][f] = (raw[f][0] & mask[0]) >> (8 * kq), sc[1][f] = (raw[f][1] & mask[1]) >> (8 * kq);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        // before the last step, whose operands are in registers, the waves meet: the next stage has landed,
        // and this one's slot may be filled again
        if (s == 3) {
          if (more == 2) wait_vmcnt<(S - 2) * PER>();
          else wait_vmcnt<0>();
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
        }
#pragma unroll
        for (int x = 0; x < T; ++x) {
          const int j = x / TM, i = x % TM;
          constexpr int RP = (F + T - 1) / T;
#pragma unroll
          for (int y = 0; y < RP; ++y)
            if (x * RP + y < F) {
              const int f = nth(x * RP + y);
              fr[(s + 1) & 1][f] = s < 3 ? frag(slot, f, s + 1) : frag(next, f, 0);
              if (s == 3) raw[f] = scale(next, f);
            }
          const uint32_t sw = sc[s >> 1][j], sa = sc[s >> 1][TN + i];
          const i32x8 wf = operand(fr[s & 1][j]), af = operand(fr[s & 1][TN + i]);
          acc[j][i] = s & 1 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf, af, acc[j][i], 4, 4, 2, sw, 2, sa)
                            : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf, af, acc[j][i], 4, 4, 0, sw, 0, sa);
          const int at = ((s + 1) & 3) * T + x;  // products behind the barrier
          if (s == 3 ? more == 2 : more >= 1)
#pragma unroll
            for (int t = 0; t < PER; ++t)
              if (issue_at(t) == at) issue_one(s == 3 ? kb + S : kb + S - 1, s == 3 ? slot : prev, t);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      slot = next;
    };
    int kb = kb0;
    for (; kb + S < KB; ++kb) stage(kb, std::integral_constant<int, 2>());
    if (kb + S == KB) stage(kb++, std::integral_constant<int, 1>());
    for (; kb < KB; ++kb) stage(kb, std::integral_constant<int, 0>());
  }

  // Epilogue, 32 rows of the wave at a time through LDS, so that its code is short (it runs once, and
  // every line of it is fetched) and its stores are whole: element e of a lane is output 8 (e / 4) + 4 kq +
  // e % 4 of its row; read back, a lane has eight outputs in a row, the same ones of every row it takes.
  constexpr int WC = BN / WN, PITCH = WC + 4, LPR = WC / 8, RPI = 64 / LPR, RB = RPI > 8 ? 32 / RPI : 4;
  static_assert(NW * 32 * PITCH * 4 <= S * STAGE && 32 % (RB * RPI) == 0, "the ring holds the rows");
  float* rows = (float*)smem + wave * 32 * PITCH;
  const int c8 = (lane % LPR) * 8, n = tn * BN + wn * WC + c8;
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = a.bias && a.split == 1 ? bias_at<OUT>(a, min(n + e, a.N - 1)) : 0.f;
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
    for (int r0 = lane / LPR; r0 < 32; r0 += RB * RPI) {  // some rows at once: one alone waits for its reads
      f32x4 v[RB][2];
#pragma unroll
      for (int q = 0; q < RB; ++q)
#pragma unroll
        for (int h = 0; h < 2; ++h) v[q][h] = *(const f32x4*)(rows + (r0 + q * RPI) * PITCH + c8 + 4 * h);
#pragma unroll
      for (int q = 0; q < RB; ++q) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = v[q][e / 4][e % 4] + bias[e];
        const int m = tm * BM + wm * (BM / WM) + i * 32 + r0 + q * RPI;
        if (a.split > 1) {  // the range's own sums
          if (m < a.M && n < a.N) {
            float* o = a.part + ((long)part * a.M + m) * part_row(a.N) + n;
            *(f32x4*)o = v[q][0], *(f32x4*)(o + 4) = v[q][1];
          }
          continue;
        }
        if (a.act)
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = gelu_tanh(y[e]);
        store_y8<OUT>(a, m, n, y);
      }
    }
    wave_lds_fence();
  }
}

// Adds the ranges of k in order and applies the epilogue: a lane takes eight outputs of a row.
template <int OUT>
__global__ __launch_bounds__(256) void linear_f4_join_kernel(LinF4Args a) {
  const int per = part_row(a.N) / 8;
  const long i = (long)blockIdx.x * 256 + threadIdx.x, groups = (long)a.M * per;
  const int m = (int)(i / per), n = (int)(i - (long)m * per) * 8;
  const long at = min(i, groups - 1) * 8, stride = (long)a.M * part_row(a.N);
  const f32x4 lo = sum_parts<8>(a.part + at, a.split, stride), hi = sum_parts<8>(a.part + at + 4, a.split, stride);
  float y[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (a.bias) y[e] += bias_at<OUT>(a, min(n + e, a.N - 1));
    if (a.act) y[e] = gelu_tanh(y[e]);
  }
  store_y8<OUT>(a, i < groups ? m : a.M, n, y);
}

// The plan of a product: the kernel of few rows (16 or 32 of them a workgroup) or the tile with the least
// estimate of
//   `first` us for every round of workgroups (`tail` for a last one with few) and `stage` us for each of its
//   panels of k (`light` where there are few workgroups),
// fitted to 1000 timings (1 .. 17550 rows, K of 384 .. 18432, N of 384 .. 12288); what it picks takes 0.8%
// more than the best of all in the mean, 12% at most.  Measured, us:
//                        256x256 192x256 192x128 128x128 64x128 64x64 32x64 32 rows 16 rows
//   17550 x 4608 x 4608     190     208     242     230    282
//   4096 x 4608 x 1152       31      27      20      21     25    28
//   1997 x 1152 x 4608       17      14      19      18     19    25
//   600 x 1152 x 4608        13      11     9.8     8.9    9.2    11    12      20
//   77 x 1152 x 4608                                7.8    6.4   5.5   5.3     6.1     6.0
//   77 x 4608 x 1152                                 13     10   8.0   7.9     5.0     4.8
//   16 x 8192 x 6144                                 20     15    11    11     7.8     6.6
// Ranges of k that are added in a second launch pay where there are few tiles and k is long: 1000 x 18432 x
// 384 16 us in two, 19 in one.
// `slots` went into the fit as workgroups of a round and are what LDS admits but for three kernels, of which it
// admits fewer: 32 x 64 (768 workgroups), and those of few rows that quantise (768 of 16 rows, 512 of 32).  The
// other constants are fitted to the slots as they stand.
struct Tile {
  int id, bm, bn, slots;
  double first, stage, tail, light;
};
static const Tile tiles[] = {{256, 256, 256, 256, 8.4, 1.68, 5.8, 0.90}, {193, 192, 256, 256, 6.5, 1.40, 4.2, 0.74},
                             {192, 192, 128, 256, 5.4, 0.74, 4.3, 0.43}, {128, 128, 128, 512, 5.1, 1.06, 3.0, 0.41},
                             {65, 64, 128, 512, 3.8, 0.64, 2.7, 0.25},   {64, 64, 64, 512, 3.2, 0.41, 2.3, 0.16},
                             {32, 32, 64, 1024, 3.7, 0.50, 2.0, 0.17},   {2, 32, 16, 768, 1.56, 0.24, 1.52, 0.05},
                             {1, 16, 16, 1024, 1.37, 0.20, 1.35, 0.04}};
static constexpr long MAX_THREADS = 1L << 32;  // a grid has fewer

static long tiles_of(int M, int N, int bm, int bn) { return (long)((M + bm - 1) / bm) * ((N + bn - 1) / bn); }

LinF4Plan linear_fp4_plan(int M, int N, int K, int dtype) {
  LinF4Plan p{};
  p.split = 1;
  p.tile = -1;
  double best = 0;
  const int panels = (K + 255) / 256;
  for (const Tile& c : tiles) {
    const bool rows = c.id <= 2;
    if (rows && M > 4096) continue;  // (their grid's second dimension)
    const long t = tiles_of(M, N, c.bm, rows && dtype == 3 ? 32 : c.bn);
    for (int s = 1; s <= 8 && (s == 1 || (!rows && t * s <= c.slots && panels >= 4 * s)); ++s) {
      const long wg = t * s, full = wg / c.slots, rem = wg % c.slots;
      // (workgroups of few rows take 1.6 times as long for the 32 outputs that they quantise)
      const double u = (double)rem / c.slots, n = (double)panels / s * (rows && dtype == 3 ? 1.6 : 1.0);
      double us = full * (c.first + n * c.stage);
      if (rem) us += c.tail + (c.first - c.tail) * u + n * (c.light + (c.stage - c.light) * u);
      if (s > 1) us += 3.0 + 2.5e-6 * s * M * N;
      if (wg * 512 >= MAX_THREADS || (p.tile > 0 && us >= best)) continue;
      best = us;
      p.tile = c.id;
      p.split = s;
      p.bytes = s > 1 ? (size_t)s * M * part_row(N) * 4 : 0;
    }
  }
  return p;
}

template <int TM, int OUT>
static void launch_rows(const LinF4Args& a, hipStream_t st) {
  constexpr int TN = OUT == 3 ? 2 : 1;
  const dim3 grid((a.N + 16 * TN - 1) / (16 * TN), (a.M + 16 * TM - 1) / (16 * TM));
  hipLaunchKernelGGL((linear_f4_rows_kernel<TM, TN, 4, OUT>), grid, dim3(256), 0, st, a);
}

template <int BM, int BN, int WM, int WN, int S, int OUT>
static void launch_tile(const LinF4Args& a, hipStream_t st) {
  hipLaunchKernelGGL((linear_f4_tile_kernel<BM, BN, WM, WN, S, OUT>), dim3((unsigned)tiles_of(a.M, a.N, BM, BN) * a.split),
                     dim3(WM * WN * 64), 0, st, a);
  if (a.split > 1)
    hipLaunchKernelGGL((linear_f4_join_kernel<OUT>), dim3((unsigned)(((long)a.M * (part_row(a.N) / 8) + 255) / 256)), dim3(256), 0,
                       st, a);
}

template <int OUT>
static void launch_out(const LinF4Args& a, int tile, hipStream_t st) {
  if (tile == 1) launch_rows<1, OUT>(a, st);
  else if (tile == 2) launch_rows<2, OUT>(a, st);
  else if (tile == 256) launch_tile<256, 256, 4, 2, 2, OUT>(a, st);
  else if (tile == 193) launch_tile<192, 256, 2, 4, 2, OUT>(a, st);
  else if (tile == 192) launch_tile<192, 128, 2, 2, 3, OUT>(a, st);
  else if (tile == 128) launch_tile<128, 128, 2, 2, 2, OUT>(a, st);
  else if (tile == 65) launch_tile<64, 128, 2, 2, 3, OUT>(a, st);
  else if (tile == 64) launch_tile<64, 64, 2, 2, 4, OUT>(a, st);
  else launch_tile<32, 64, 1, 2, 4, OUT>(a, st);
}

hipError_t launch_linear_fp4(const LinF4Args& a, const LinF4Plan& p, hipStream_t st) {
  if (a.dtype == 0) launch_out<0>(a, p.tile, st);
  else if (a.dtype == 1) launch_out<1>(a, p.tile, st);
  else launch_out<3>(a, p.tile, st);
  return hipGetLastError();
}

// ------------------------------------------------------------------ quantisation
// Bound by memory: 17550 x 12288 fp32 177 us there (5.5 TB/s) and 172 back (5.7), a copy reaches 5.1; small
// ones by the launch (256 x 1152 2.2 us each).
// 32 lanes take the 256 columns of one panel of one row, 8 columns each, and the four of a block share its
// maximum; a workgroup takes 8 rows, whose scales of the panel lie together.
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
