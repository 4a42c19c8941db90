// Queries and keys normed for each head and turned by the row's positions, in one pass (ditmi.h:
// dit_qk_norm_rope).
#include "common.h"
#include "kernels.h"

namespace ditmi {

// Sum over aligned groups of N lanes; every lane gets it.
template <int N>
__device__ __forceinline__ float group_sum(float v) {
  if (N > 1) v += dpp_move<0xB1>(v);
  if (N > 2) v += dpp_move<0x4E>(v);
  if (N > 4) v += dpp_move<0x141>(v);
  if (N > 8) v += dpp_move<0x140>(v);
  if (N > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// Eight values of a head as they lie in memory: a piece of four at p, another at p + gap.
template <typename T>
struct Raw;
template <>
struct Raw<bf16_t> {
  u32x2 lo, hi;
  __device__ void load(const bf16_t* p, int gap) { lo = *(const u32x2*)p, hi = *(const u32x2*)(p + gap); }
  __device__ void store(bf16_t* p, int gap) const { *(u32x2*)p = lo, *(u32x2*)(p + gap) = hi; }
  __device__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[2 * i] = __uint_as_float(lo[i] << 16), x[2 * i + 1] = __uint_as_float(lo[i] & 0xFFFF0000u);
      x[4 + 2 * i] = __uint_as_float(hi[i] << 16), x[5 + 2 * i] = __uint_as_float(hi[i] & 0xFFFF0000u);
    }
  }
  __device__ void set(const float (&x)[8]) {
    lo = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    hi = u32x2{pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
  }
};
template <>
struct Raw<float> {
  f32x4 lo, hi;
  __device__ void load(const float* p, int gap) { lo = *(const f32x4*)p, hi = *(const f32x4*)(p + gap); }
  __device__ void store(float* p, int gap) const { *(f32x4*)p = lo, *(f32x4*)(p + gap) = hi; }
  __device__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = lo[i], x[4 + i] = hi[i];
  }
  __device__ void set(const float (&x)[8]) { lo = f32x4{x[0], x[1], x[2], x[3]}, hi = f32x4{x[4], x[5], x[6], x[7]}; }
};

// A wave takes `seg` of a row's segments: heads chunk * (64 / LP) + lane / LP for chunk = segment,
// segment + segments, ...; the heads of q, k and v count through.  LP lanes (a power of two, dh / 8 of
// them at work) hold a head, lane l its pairs 4 l .. 4 l + 3: eight neighbours, or, where a head's
// halves are paired, four of each.
template <typename T, int LP, bool HALVES>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkArgs a) {
  constexpr int HPW = 64 / LP;
  const int lane = threadIdx.x & 63, l = lane & (LP - 1);
  const long unit = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= (long)a.rows * a.segments) return;
  const int row = (int)(unit / a.segments), seg = (int)(unit - (long)row * a.segments);
  const bool work = l < a.dh / 8;
  const int lc = work ? l : 0;
  const bool turned = lc * 4 < a.P;  // (where halves are paired P is a multiple of four)
  const int at = HALVES ? (turned ? lc * 4 : 8 * lc) : 8 * lc;
  const int gap = HALVES ? (turned ? a.P : 4) : 4;

  // cos and sin of the lane's four pairs: the angle in turns, in 64 bits, less its whole turns
  float c[4], s[4];
  bool rot[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int p = lc * 4 + j;
    rot[j] = p < a.P;
    if (rot[j]) {
      int axis = 0;
#pragma unroll
      for (int i = 0; i < 3; ++i) axis += p >= a.axis_end[i] ? 1 : 0;
      double t = (double)a.pos[(long)row * a.axes + axis] * (a.freqs[p] * 0.15915494309189533577);
      t -= rint(t);
      if (sizeof(T) == 2) {
        c[j] = __builtin_amdgcn_cosf((float)t), s[j] = __builtin_amdgcn_sinf((float)t);
      } else {
        sincospif((float)(2 * t), &s[j], &c[j]);
      }
    } else {
      c[j] = 1.f, s[j] = 0.f;
    }
  }
  const int heads = a.H + a.Hk + a.Hv, chunks = (heads + HPW - 1) / HPW;
  const long qd = a.q_dst ? a.q_dst[row] : row, kd = a.k_dst ? a.k_dst[row] : row;
  const bool q_in = qd >= 0 && qd < a.q_out_rows, k_in = kd >= 0 && kd < a.k_out_rows;
  const float rdh = 1.f / (float)a.dh;
  float wq[8], wk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = at + (i < 4 ? i : gap + i - 4);
    wq[i] = a.w_q ? a.w_q[e] : 1.f;
    wk[i] = a.w_k ? a.w_k[e] : 1.f;
  }
  for (int chunk = seg; chunk < chunks; chunk += a.segments) {
    const int h = chunk * HPW + lane / LP, hc = min(h, heads - 1);
    const int kind = hc < a.H ? 0 : hc < a.H + a.Hk ? 1 : 2;
    const int hh = kind == 0 ? hc : kind == 1 ? hc - a.H : hc - a.H - a.Hk;
    const T* src = (const T*)(kind == 0 ? a.q : kind == 1 ? a.k : a.v);
    T* dst = (T*)(kind == 0 ? a.q_out : kind == 1 ? a.k_out : a.v_out);
    src += row * (kind == 0 ? a.q_row : kind == 1 ? a.k_row : a.v_row) + hh * (kind == 0 ? a.q_head : kind == 1 ? a.k_head : a.v_head) + at;
    dst += (kind == 0 ? qd : kd) * (kind == 0 ? a.qo_row : kind == 1 ? a.ko_row : a.vo_row) +
           hh * (kind == 0 ? a.qo_head : kind == 1 ? a.ko_head : a.vo_head) + at;
    Raw<T> raw;
    raw.load(src, gap);
    float x[8];
    raw.get(x);
    if (a.norm) {
      float mu = 0.f;
      if (a.norm == 1) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += x[i];
        mu = group_sum<LP>(work ? t : 0.f) * rdh;
      }
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] -= mu;
        t = fmaf(x[i], x[i], t);
      }
      const float r = 1.f / sqrtf(group_sum<LP>(work ? t : 0.f) * rdh + a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= r * (kind == 0 ? wq[i] : wk[i]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i0 = HALVES ? j : 2 * j, i1 = HALVES ? 4 + j : 2 * j + 1;
      const float u = x[i0], v = x[i1];
      x[i0] = rot[j] ? u * c[j] - v * s[j] : u;
      x[i1] = rot[j] ? u * s[j] + v * c[j] : v;
    }
    Raw<T> out = raw;
    if (kind != 2) out.set(x);
    if (work && h < heads && (kind == 0 ? q_in : k_in)) out.store(dst, gap);
  }
}

template <typename T, bool HALVES>
static void launch_qk(const QkArgs& a, hipStream_t st) {
  const int lanes = a.dh / 8, lp = lanes <= 1 ? 1 : lanes <= 2 ? 2 : lanes <= 4 ? 4 : lanes <= 8 ? 8 : lanes <= 16 ? 16 : 32;
  const dim3 grid((unsigned)(((long)a.rows * a.segments + 3) / 4)), block(256);
#define QK(LP) hipLaunchKernelGGL((qk_norm_rope_kernel<T, LP, HALVES>), grid, block, 0, st, a)
  if (lp == 1) QK(1);
  else if (lp == 2) QK(2);
  else if (lp == 4) QK(4);
  else if (lp == 8) QK(8);
  else if (lp == 16) QK(16);
  else QK(32);
#undef QK
}

hipError_t launch_qk_norm_rope(QkArgs a, int dtype, hipStream_t st) {
  const int lanes = a.dh / 8;
  int lp = 1;
  while (lp < lanes) lp *= 2;
  const int hpw = 64 / lp, chunks = (a.H + a.Hk + a.Hv + hpw - 1) / hpw;
  // enough waves to fill the card
  const long want = (16384 + a.rows - 1) / a.rows;
  a.segments = (int)(want < chunks ? want : chunks);
  if (dtype == 0) a.halves ? launch_qk<float, true>(a, st) : launch_qk<float, false>(a, st);
  else a.halves ? launch_qk<bf16_t, true>(a, st) : launch_qk<bf16_t, false>(a, st);
  return hipGetLastError();
}

}  // namespace ditmi
