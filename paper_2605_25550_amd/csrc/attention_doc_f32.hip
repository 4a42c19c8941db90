// Masked attention over documents, fp32 (ditmi.h: dit_attention): fp32 products
// on the matrix cores (v_mfma_f32_16x16x4_f32), fp32 exponentials (the hardware's
// 2^x, within an ulp), tanh and sums.
//
// A workgroup of four waves owns 16 QT rows (query, head of the group that
// shares keys) of one document.  The waves divide the keys of the workgroup's
// range: wave w takes the 32-key groups w, w + 4, ... with a softmax state of
// its own, and the four are merged through LDS at the end.  K and V fragments
// come straight from global memory (L2) as 16-byte loads: no two waves of a
// workgroup read the same key.  The layout of the products is that of the
// block's fp32 attention: S^T = K Q^T leaves a lane (r16 = lane % 16,
// kq = lane / 16) keys 4 kq + e of row r16, which is the B operand of
// O^T = V^T P^T as it is.
#include <algorithm>

#include "common.h"
#include "doc.h"
#include "kernels.h"

namespace ditmi {

template <int DH, int QT, bool CAP, bool BIAS>
__global__ __launch_bounds__(256) void doc_attn_f32_kernel(DocAttnArgs a) {
  constexpr int KS = (DH + 15) / 16;      // 16-wide steps of QK^T; the last of head_dim 72 is half empty
  constexpr int VB = DH / 64;             // 64-column blocks of V (16-byte loads) ...
  constexpr int VX = DH % 64 ? 1 : 0;     // ... and a tile of the last DH % 64 columns (head_dim 72)
  constexpr int TV = 4 * VB + VX;         // O^T tiles
  constexpr int OS = DH + 4;              // row stride of a wave's O in LDS
  constexpr int BM = 16 * QT;
  __shared__ __attribute__((aligned(16))) float os[4][BM][OS];
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
  const int lim_lo = row_limit(a, doc, min(qb * BM, rows - 1) / a.G);
  const int lim_hi = row_limit(a, doc, min(qb * BM + BM - 1, rows - 1) / a.G);
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

  f32x4 kf[2][KS];
  auto load_k = [&](int gr) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float* kr = kp + (long)min(gr * 32 + 16 * c + r16, doc.nk - 1) * a.k_row + 4 * kq;  // past the end: masked
#pragma unroll
      for (int s = 0; s < KS; ++s) kf[c][s] = s < KS - 1 || dlast ? *(const f32x4*)(kr + 16 * s) : zero;
    }
  };
  if (g0 + wave < g1) load_k(g0 + wave);
  for (int gr = g0 + wave; gr < g1; gr += 4) {
    const int kv0 = gr * 32;
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
#pragma unroll
    for (int t = 0; t < QT; ++t) s[t][0] = s[t][1] = zero;
#pragma unroll
    for (int d = 0; d < KS; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int c = 0; c < 2; ++c)
            s[t][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[c][d][e], qf[t][d][e], s[t][c], 0, 0, 0);
    if (gr + 4 < g1) load_k(gr + 4);
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
      mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
      mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
      const float m_new = fmaxf(m_run[t], mt);
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
        *(f32x4*)&os[wave][qr][64 * v + 16 * kq + 4 * e] =
            f32x4{o[t][4 * v][e], o[t][4 * v + 1][e], o[t][4 * v + 2][e], o[t][4 * v + 3][e]};
      if (VX && 4 * kq + e < DH % 64) os[wave][qr][64 * VB + 4 * kq + e] = o[t][TV - 1][e];
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
      num += f * *(const f32x4*)&os[w][qr][d];
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
