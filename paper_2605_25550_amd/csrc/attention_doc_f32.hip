// Masked attention over documents, fp32 (ditmi.h: dit_attention): fp32 products
// on the matrix cores (v_mfma_f32_16x16x4_f32), fp32 exponentials (the hardware's
// 2^x, within an ulp), tanh and sums.
//
// A workgroup of four waves owns 16 QT rows (query, head of the group that
// shares keys) of one document.  The waves divide the keys of the workgroup's
// range: wave w takes the 32-key groups w, w + 4, ... with a softmax state of
// its own, and the four are merged through LDS at the end: no two waves of a
// workgroup read the same key, and none waits for another.  The layout of the
// products is that of the block's fp32 attention: S^T = K Q^T leaves a lane
// (r16 = lane % 16, kq = lane / 16) keys 4 kq + e of row r16, which is the B
// operand of O^T = V^T P^T as it is.
//
// The fp32 products and the vector instructions share their pipe (no cycle has
// both: 0 of SQ_VALU_MFMA_COEXEC_CYCLES), so that running the softmax between the
// products gains nothing; what counts is that neither waits.  K fragments, loaded
// as they lie, cost a cache access for every 16 bytes (16 lanes, 16 rows): for
// head_dim 64 and 72 whole rows come by DMA into a ring of the wave's own in LDS,
// a group ahead, which also leaves registers for two waves per SIMD.  V, whose
// rows 16 lanes read together, comes straight from global memory.
// 2048 queries and keys, 16 heads of 72: 213 us, 91 TFLOP/s (245 us with K straight
// into registers); 2 x 333: 26.7 us (34.7).  Head_dim 128, whose ring and
// registers leave room for one wave per SIMD either way: 181 us straight, 189 through LDS
// (1500 queries and keys, causal, 24 heads).
#include <algorithm>
#include <utility>

#include "common.h"
#include "doc.h"
#include "kernels.h"

namespace ditmi {

// f(0), f(1) .. with constant arguments: the unroller gives up on bodies this long
template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}

// max over the four lanes of a row (lane % 16 the same)
__device__ __forceinline__ float max_kq(float m) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

template <int DH, int QT, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, DH < 128 ? 2 : 1) void doc_attn_f32_kernel(DocAttnArgs a) {
  constexpr int KS = (DH + 15) / 16;      // 16-wide steps of QK^T; the last of head_dim 72 is half empty
  constexpr int VB = DH / 64;             // 64-column blocks of V (16-byte loads) ...
  constexpr int VX = DH % 64 ? 1 : 0;     // ... and a tile of the last DH % 64 columns (head_dim 72)
  constexpr int TV = 4 * VB + VX;         // O^T tiles
  constexpr int OS = DH + 4;              // row stride of a wave's O in LDS
  constexpr int BM = 16 * QT;
  constexpr bool KLDS = DH < 128;         // K through LDS
  constexpr int CPR = DH / 4;             // 16-byte chunks of a K row
  constexpr int KT = 32 * DH * 4;         // bytes of a group's K
  static_assert(KT % 1024 == 0 && 2 * KT >= BM * OS * 4, "whole DMA blocks; a wave's O takes the place of its ring");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4][KLDS ? 2 * KT : BM * OS * 4];  // a ring of two groups for each wave
  __shared__ float ml[4][2][BM];
  __shared__ int bad[3][DH];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const Doc doc = load_doc(a, blockIdx.y);
  const int rows = doc.nq * a.G;
  const int nqb = (rows + BM - 1) / BM, items = nqb * a.Hk;
  if ((int)blockIdx.x >= items) return;
  const int item = xcd_remap(blockIdx.x, items);
  const int hk = item / nqb;
  const int qb = a.mask ? nqb - 1 - item % nqb : item % nqb;
  const int lim_lo = __builtin_amdgcn_readfirstlane(row_limit(a, doc, min(qb * BM, rows - 1) / a.G));
  const int lim_hi = __builtin_amdgcn_readfirstlane(row_limit(a, doc, min(qb * BM + BM - 1, rows - 1) / a.G));
  const int ng_all = (lim_hi + 31) / 32, part = blockIdx.z;
  const int g0 = (int)((long)ng_all * part / a.split), g1 = (int)((long)ng_all * (part + 1) / a.split);
  const float* __restrict__ kp = (const float*)a.k + (long)doc.k0 * a.k_row + hk * a.k_head;
  const float* __restrict__ vp = (const float*)a.v + (long)doc.k0 * a.v_row + hk * a.v_head;

  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const bool dlast = 16 * (KS - 1) + 4 * kq < DH;  // the lane's columns of the last step exist
  f32x4 qf[QT][KS], o[QT][TV];
  float m_run[QT], l_run[QT], slope[QT];
  int lim[QT], here[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int row = min(qb * BM + 16 * t + r16, rows - 1), qi = row / a.G, h = hk * a.G + row % a.G;
    lim[t] = row_limit(a, doc, qi);
    here[t] = qi + doc.nk - doc.nq;
    slope[t] = BIAS ? a.slopes[h] * LOG2E : 0.f;
    const float* qr = (const float*)a.q + (long)(doc.q0 + qi) * a.q_row + h * a.q_head + 4 * kq;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[t][s] = s < KS - 1 || dlast ? *(const f32x4*)(qr + 16 * s) : zero;
#pragma unroll
    for (int v = 0; v < TV; ++v) o[t][v] = zero;
    m_run[t] = -INFINITY;
    l_run[t] = 0.f;
  }

  for (int e = tid; e < 3 * DH; e += 256) bad[0][e] = NO_KEY;
  __syncthreads();

  // K of a group (past the end the last row again: masked).  KLDS: by DMA into half
  // n of the wave's ring, chunk c of row R at c ^ swz(R), so that the 16 rows of a
  // fragment read come from different banks; else straight into registers.
  f32x4 kf[KLDS ? 2 : KS][2];
  auto swz = [](int R) { return DH == 72 ? (R >> 3) & 1 : R & 15; };
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem[wave]));
  auto issue_k = [&](int gr, int n) __attribute__((always_inline)) {
    const int last = doc.nk - 1 - gr * 32;
    const float* base = kp + (long)(gr * 32) * a.k_row;
#pragma unroll
    for (int i = 0; i < KT / 1024; ++i) {
      const int x = i * 64 + lane, R = x / CPR, c = (x - R * CPR) ^ swz(R);
      dma_16s(base, (unsigned)min(R, last) * (unsigned)(a.k_row * 4) + c * 16, lds0 + n * KT + i * 1024);
    }
  };
  auto read_k = [&](int n, int d) __attribute__((always_inline)) {
    const unsigned char* p = smem[wave] + n * KT + r16 * (DH * 4) + (((4 * d + kq) ^ swz(r16)) << 4);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      kf[d & 1][c] = *(const f32x4*)(p + 16 * c * (DH * 4));
      if (DH % 16 && d == KS - 1 && !dlast) kf[d & 1][c] = zero;  // (another row's: it may be anything)
    }
  };
  auto load_k = [&](int gr) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float* kr = kp + (long)min(gr * 32 + 16 * c + r16, doc.nk - 1) * a.k_row + 4 * kq;
#pragma unroll
      for (int d = 0; d < (KLDS ? 0 : KS); ++d) kf[d][c] = *(const f32x4*)(kr + 16 * d);
    }
  };
  static_assert(KLDS || DH % 16 == 0, "whole steps of K in registers");
  // product i of QK^T: accumulators t, c fastest; the next step's K is read behind a step's first
  constexpr int NQ = KS * 4 * QT * 2;
  auto qk = [&](f32x4 (&s)[QT][2], int n, int i) __attribute__((always_inline)) {
    const int c = i % 2, t = i / 2 % QT, e = i / (2 * QT) % 4, d = i / (8 * QT);
    s[t][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[KLDS ? d & 1 : d][c][e], qf[t][d][e], i < 2 * QT ? zero : s[t][c], 0, 0, 0);
    if (KLDS && i % (8 * QT) == 0 && d + 1 < KS) read_k(n, d + 1);
  };
  if (g0 + wave < g1) {
    if (KLDS) issue_k(g0 + wave, 0);
    else load_k(g0 + wave);
  }
  for (int gr = g0 + wave, n = 0; gr < g1; gr += 4, n ^= 1) {
    const int kv0 = gr * 32;
    if (KLDS) {
      // this group's K is here; the next one's is requested before V, so that
      // waiting for V does not wait for more
      wait_vmcnt<0>();
      read_k(n, 0);
      issue_k(min(gr + 4, g1 - 1), n ^ 1);
    }
    const bool masked = kv0 + 32 > lim_lo;
    // V rows 4 kq + e of both 16-key halves, requested before the scores
    f32x4 vf[2][4][VB];
    float vx[2][4];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float* vr = vp + (long)min(kv0 + 16 * c + 4 * kq + e, doc.nk - 1) * a.v_row;
#pragma unroll
        for (int v = 0; v < VB; ++v) vf[c][e][v] = *(const f32x4*)(vr + 64 * v + 4 * r16);
        vx[c][e] = VX && r16 < DH % 64 ? vr[64 * VB + r16] : 0.f;
      }
    f32x4 s[QT][2];
    each<NQ>([&](auto i) __attribute__((always_inline)) { qk(s, n, i); });
    if (!KLDS) load_k(min(gr + 4, g1 - 1));
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float mt = -INFINITY;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = kv0 + 16 * c + 4 * kq + e;
          // the exponent in the exp2 domain
          float z = CAP ? a.cap * LOG2E * tanhf(s[t][c][e] * (a.scale / a.cap)) : s[t][c][e] * (a.scale * LOG2E);
          if (BIAS) z -= slope[t] * fabsf((float)(here[t] - key));
          s[t][c][e] = masked && key >= lim[t] ? -INFINITY : z;
          mt = fmaxf(mt, s[t][c][e]);
        }
      const float m_new = fmaxf(m_run[t], max_kq(mt));
      // nothing visible so far: 2^(-inf - 0) instead of -inf - (-inf)
      const float m_ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m_run[t] - m_ref);
      m_run[t] = m_new;
      l_run[t] *= alpha;
#pragma unroll
      for (int v = 0; v < TV; ++v) o[t][v] *= alpha;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[t][c][e] = __builtin_amdgcn_exp2f(s[t][c][e] - m_ref);
          l_run[t] += s[t][c][e];
        }
    }
    if (masked) {
      // values that are not finite, in a group that some row does not see
      // whole: taken out, and brought at the end to the rows that see their key
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int v = 0; v < TV; ++v) {
            float& x = v < 4 * VB ? ((float*)&vf[c][e][v >> 2])[v & 3] : vx[c][e];
            if (!(fabsf(x) < INFINITY)) {
              const int d = v < 4 * VB ? 64 * (v >> 2) + 4 * r16 + (v & 3) : 64 * VB + r16;
              note_bad(bad, x != x ? 0 : x > 0.f ? 1 : 2, d, kv0 + 16 * c + 4 * kq + e);
              x = 0.f;
            }
          }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int v = 0; v < TV; ++v)
            o[t][v] = __builtin_amdgcn_mfma_f32_16x16x4f32(v < 4 * VB ? vf[c][e][v >> 2][v & 3] : vx[c][e], s[t][c][e],
                                                           o[t][v], 0, 0, 0);
  }

  wait_vmcnt<0>();  // the ring is the wave's O from here on
  float* os = (float*)smem[wave];
  // Merge of the four waves: with m = max_w m_w and f_w = 2^(m_w - m),
  // O = sum_w f_w O_w, l = sum_w f_w l_w (a wave without keys has m = -inf
  // and zeros).
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l_run[t] += __shfl_xor(l_run[t], 16, 64);
    l_run[t] += __shfl_xor(l_run[t], 32, 64);
    const int qr = 16 * t + r16;
    if (kq == 0) {
      ml[wave][0][qr] = m_run[t];
      ml[wave][1][qr] = l_run[t];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int v = 0; v < VB; ++v)
        *(f32x4*)&os[qr * OS + 64 * v + 16 * kq + 4 * e] =
            f32x4{o[t][4 * v][e], o[t][4 * v + 1][e], o[t][4 * v + 2][e], o[t][4 * v + 3][e]};
      if (VX && 4 * kq + e < DH % 64) os[qr * OS + 64 * VB + 4 * kq + e] = o[t][TV - 1][e];
    }
  }
  __syncthreads();
  constexpr int G4 = DH / 4;  // 4-column groups per row
  for (int i = tid; i < BM * G4; i += 256) {
    const int qr = i / G4, d = (i - qr * G4) * 4, row = qb * BM + qr;
    if (row >= rows) continue;
    const int qi = row / a.G, h = hk * a.G + row % a.G;
    float m = ml[0][0][qr];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, ml[w][0][qr]);
    const float mr = m == -INFINITY ? 0.f : m;
    float den = 0.f;
    f32x4 num = zero;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w][0][qr] - mr);
      den += f * ml[w][1][qr];
      num += f * *(const f32x4*)&((const float*)smem[w])[qr * OS + d];
    }
    if (lim_lo < ng_all * 32) {
      const int lim_row = row_limit(a, doc, qi);
#pragma unroll
      for (int x = 0; x < 4; ++x) num[x] = add_bad(num[x], bad, d + x, lim_row);
    }
    if (a.split > 1) {
      float* pr = a.part + ((long)part * a.q_rows * a.H + (long)(doc.q0 + qi) * a.H + h) * (DH + 4);
      *(f32x4*)(pr + d) = num;
      if (d == 0) *(f32x2*)(pr + DH) = f32x2{m, den};
    } else {
      *(f32x4*)((float*)a.o + (long)(doc.q0 + qi) * a.o_row + h * a.o_head + d) = num * (den == 0.f ? 0.f : 1.0f / den);
    }
  }
}

template <int DH, int QT>
static void launch_qt(const DocAttnArgs& a, hipStream_t st) {
  const long nqb = ((long)a.max_q * a.G + 16 * QT - 1) / (16 * QT);
  const dim3 grid((unsigned)(nqb * a.Hk), a.docs, a.split), block(256);
  const bool cap = a.cap > 0.f, bias = a.slopes != nullptr;
  if (cap && bias) hipLaunchKernelGGL((doc_attn_f32_kernel<DH, QT, true, true>), grid, block, 0, st, a);
  else if (cap) hipLaunchKernelGGL((doc_attn_f32_kernel<DH, QT, true, false>), grid, block, 0, st, a);
  else if (bias) hipLaunchKernelGGL((doc_attn_f32_kernel<DH, QT, false, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((doc_attn_f32_kernel<DH, QT, false, false>), grid, block, 0, st, a);
}

template <int DH>
static void launch_dh(const DocAttnArgs& a, hipStream_t st) {
  const long rows = std::min((long)a.docs * a.max_q, (long)a.q_rows) * a.G;
  if (rows / 32 * a.Hk >= 512) launch_qt<DH, 2>(a, st);
  else launch_qt<DH, 1>(a, st);
}

hipError_t launch_doc_attn_f32(const DocAttnArgs& a, const DocAttnPlan& p, int head_dim, hipStream_t st) {
  switch (head_dim) {
    case 64: launch_dh<64>(a, st); break;
    case 72: launch_dh<72>(a, st); break;
    case 128: launch_dh<128>(a, st); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace ditmi
