// Queries and keys normed for each head and turned by the row's positions, in one pass (ditmi.h:
// dit_qk_norm_rope): a head is read once and held in registers between its statistics, the rotation and
// the store.  The angle of a pair is the same for every head of a row: a wave makes the cosines and sines
// of its lanes' pairs once and keeps them for all the heads that it takes.
//
// Bound by memory: 17550 rows of 24 + 24 heads of 128 bf16 83 us, 5.2 TB/s (a copy 5.1), of 16 + 16 heads of
// 72 34 us, 4.7 TB/s (41 with nine lanes of sixteen at work instead of seven heads in a wave).  Smaller calls
// by a wave's chain of loads: 4 rows 3.6 us, 3431 rows of 16 + 16 heads of 72 with layer norms 11 (2.9 TB/s).
#include "common.h"
#include "kernels.h"

namespace ditmi {

// Sum over groups of N lanes, every lane gets it: 9, or a power of two.
template <int N>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (N == 9) {  // sums of 2, 4 and 8 neighbours round the group, and the ninth
    const int lane = threadIdx.x & 63, base = lane / 9 * 9, l = lane - base;
    auto from = [&](float x, int k) {
      const int src = base + (l + k >= 9 ? l + k - 9 : l + k);
      return __int_as_float(__builtin_amdgcn_ds_bpermute(src * 4, __float_as_int(x)));
    };
    const float ninth = from(v, 8);
    v += from(v, 1);
    v += from(v, 2);
    return v + from(v, 4) + ninth;
  }
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

// Eight values of a head as they lie in memory: neighbours, or (HALVES) a piece of four at p and another
// at p + gap.
template <typename T, bool HALVES>
struct Raw {
  static constexpr int N = sizeof(T) == 2 ? 2 : 4;  // dwords of a piece
  u32x4 w[N / 2];

  __device__ void load(const T* p, int gap) {
    if constexpr (N == 4) w[0] = *(const u32x4*)p, w[1] = *(const u32x4*)(p + (HALVES ? gap : 4));
    else if constexpr (!HALVES) w[0] = *(const u32x4*)p;
    else {
      const u32x2 lo = *(const u32x2*)p, hi = *(const u32x2*)(p + gap);
      w[0] = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  }
  __device__ void store(T* p, int gap) const {
    if constexpr (N == 4) *(u32x4*)p = w[0], *(u32x4*)(p + (HALVES ? gap : 4)) = w[1];
    else if constexpr (!HALVES) *(u32x4*)p = w[0];
    else *(u32x2*)p = u32x2{w[0][0], w[0][1]}, *(u32x2*)(p + gap) = u32x2{w[0][2], w[0][3]};
  }
  __device__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (N == 4) x[i] = __uint_as_float(w[0][i]), x[4 + i] = __uint_as_float(w[1][i]);
      else x[2 * i] = __uint_as_float(w[0][i] << 16), x[2 * i + 1] = __uint_as_float(w[0][i] & 0xFFFF0000u);
    }
  }
  __device__ void set(const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (N == 4) w[0][i] = __float_as_uint(x[i]), w[1][i] = __float_as_uint(x[4 + i]);
      else w[0][i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    }
  }
};

// A wave takes one of a row's segments: chunks seg, seg + segments, ... of 64 / LP heads of one tensor,
// those of q before those of k and of v.  LP lanes (dh / 8 of them at work) hold a head,
// lane l its pairs 4 l .. 4 l + 3: eight neighbours, or, where a head's halves are paired, four of each.
// The first chunk's values are on their way while the angles are made, the next chunk's while one is
// computed.
template <typename T, int LP, bool HALVES>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkArgs a) {
  constexpr int HPW = 64 / LP;
  // one of each 64 bytes of the arguments, so that their cache lines come together (1700 rows of 9 + 9 heads
  // of 128 7.57 us against 7.73, 6862 of 16 + 16 of 72 16.9 against 17.1)
  asm volatile("" ::"s"(a.w_q), "s"(a.rows), "s"(a.P), "s"(a.k_head), "s"(a.vo_head));
  const int lane = threadIdx.x & 63, g = lane / LP, l = lane - g * LP;
  const long unit = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= (long)a.rows * a.segments) return;
  const int row = (int)((unsigned)unit / (unsigned)a.segments), seg = (int)unit - row * a.segments;
  const bool work = l < a.dh / 8 && g < HPW;
  const int lc = work ? l : 0;
  const bool turned = lc * 4 < a.P;  // (where halves are paired P is a multiple of four)
  const int at = HALVES && turned ? lc * 4 : 8 * lc;
  const int gap = HALVES && turned ? a.P : 4;

  const int cq = (a.H + HPW - 1) / HPW, ck = (a.Hk + HPW - 1) / HPW, chunks = cq + ck + (a.Hv + HPW - 1) / HPW;
  const long qd = a.q_dst ? a.q_dst[row] : row, kd = a.k_dst ? a.k_dst[row] : row;
  const bool q_in = qd >= 0 && qd < a.q_out_rows, k_in = kd >= 0 && kd < a.k_out_rows;
  Raw<T, HALVES> raw;
  auto load = [&](int chunk) {
    const bool is_q = chunk < cq, is_k = chunk < cq + ck;  // (the same for the whole wave, as all of this but g and at)
    const int h0 = (is_q ? chunk : is_k ? chunk - cq : chunk - cq - ck) * HPW, last = (is_q ? a.H : a.Hk) - 1;
    const T* p = (const T*)(is_q ? a.q : is_k ? a.k : a.v) + row * (is_q ? a.q_row : is_k ? a.k_row : a.v_row);
    raw.load(p + min(h0 + g, last) * (is_q ? a.q_head : is_k ? a.k_head : a.v_head) + at, gap);
  };
  load(seg);

  const f32x4 one = {1.f, 1.f, 1.f, 1.f};
  f32x4 wq[2] = {one, one}, wk[2] = {one, one};
  if (a.w_q) wq[0] = *(const f32x4*)(a.w_q + at), wq[1] = *(const f32x4*)(a.w_q + at + gap);
  if (a.w_k) wk[0] = *(const f32x4*)(a.w_k + at), wk[1] = *(const f32x4*)(a.w_k + at + gap);

  // cos and sin of the lane's four pairs: the angle in turns, in 64 bits, less its whole turns.  In bf16 by the
  // hardware's functions, off by 2^-18 at most against half a step of 2^-8: as exact ones, of 4 million outputs 254
  // instead of 236 are rounded otherwise than those of an fp32 form, and 1000 rows of 16 + 16 heads of 72 take 7.1
  // us instead of 7.5, 17550 rows of 12 + 12 of 64 23.4 instead of 24.7
  float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
  if (a.P) {
    int pos[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) pos[i] = a.pos[(long)row * a.axes + min(i, a.axes - 1)];
    double f[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = a.freqs[min(lc * 4 + j, a.P - 1)];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = lc * 4 + j;
      const int at_axis = p < a.axis_end[0] ? pos[0] : p < a.axis_end[1] ? pos[1] : p < a.axis_end[2] ? pos[2] : pos[3];
      double t = (double)at_axis * (f[j] * 0.15915494309189533577);
      t -= rint(t);
      if (sizeof(T) == 2) c[j] = __builtin_amdgcn_cosf((float)t), s[j] = __builtin_amdgcn_sinf((float)t);
      else sincospif((float)(2 * t), &s[j], &c[j]);
    }
  }
  const bool whole = 2 * a.P == a.dh;
  const float rdh = 1.f / (float)a.dh;
  for (int chunk = seg; chunk < chunks; chunk += a.segments) {
    const bool is_q = chunk < cq, is_k = chunk < cq + ck;
    const int h = (is_q ? chunk : is_k ? chunk - cq : chunk - cq - ck) * HPW + g;
    Raw<T, HALVES> out = raw;
    if (chunk + a.segments < chunks) load(chunk + a.segments);
    if (is_k) {  // (not v)
      float x[8];
      out.get(x);
      if (a.norm) {
        float mu = 0.f;
        if (a.norm == 1) {
          const float t = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
          mu = group_sum<LP>(work ? t : 0.f) * rdh;
        }
        // (not inside the branch: hipcc of ROCm 7.2.0, clang 22.0.0git 7b800a19, leaves fp32 heads undefined on the
        // other path then, as every test of RMS norms in fp32 shows)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] -= mu;
        float t = x[0] * x[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) t = fmaf(x[i], x[i], t);
        // (eps is a normal number: so is what the root is taken of)
        const float r = __builtin_amdgcn_rsqf(group_sum<LP>(work ? t : 0.f) * rdh + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= r * (is_q ? wq[i / 4][i % 4] : wk[i / 4][i % 4]);
      }
      if (a.P)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i0 = HALVES ? j : 2 * j, i1 = HALVES ? 4 + j : 2 * j + 1;
          const float u = x[i0], v = x[i1];
          x[i0] = u * c[j] - v * s[j];
          x[i1] = u * s[j] + v * c[j];
          if (!whole && lc * 4 + j >= a.P) x[i0] = u, x[i1] = v;  // (what is not turned may be infinite)
        }
      out.set(x);
    }
    const bool in = is_q ? q_in : k_in;
    if (in && work && h < (is_q ? a.H : a.Hk)) {
      T* p = (T*)(is_q ? a.q_out : is_k ? a.k_out : a.v_out) + (is_q ? qd * a.qo_row : kd * (is_k ? a.ko_row : a.vo_row));
      out.store(p + h * (is_q ? a.qo_head : is_k ? a.ko_head : a.vo_head) + at, gap);
    }
  }
}

static int lanes_per_head(int dh) {
  const int lanes = dh / 8;  // (nine: DiT-XL/2's head_dim of 72)
  int lp = 1;
  while (lp < lanes) lp *= 2;
  return lanes == 9 ? 9 : lp;
}

template <typename T, bool HALVES>
static void launch_qk(const QkArgs& a, hipStream_t st) {
  const int lp = lanes_per_head(a.dh);
  const dim3 grid((unsigned)(((long)a.rows * a.segments + 3) / 4)), block(256);
#define QK(LP) hipLaunchKernelGGL((qk_norm_rope_kernel<T, LP, HALVES>), grid, block, 0, st, a)
  if (lp == 1) QK(1);
  else if (lp == 2) QK(2);
  else if (lp == 4) QK(4);
  else if (lp == 8) QK(8);
  else if (lp == 9) QK(9);
  else if (lp == 16) QK(16);
  else QK(32);
#undef QK
}

int qk_segments(int rows, int dh, int H, int Hk, int Hv) {
  const int hpw = 64 / lanes_per_head(dh), chunks = (H + hpw - 1) / hpw + (Hk + hpw - 1) / hpw + (Hv + hpw - 1) / hpw;
  // four waves per SIMD, and no wave with more than six chunks.  Measured, us in one, two, three, six segments:
  // 17550 rows of 24 + 24 heads of 128 89, 84, 81, 86 (twelve: 114), 3431 rows 19.8, 16.7, 17.2, 18.1; 17550 rows
  // of 16 + 16 of 72 34, 35, 39, 51, 3431 rows 13.3, 12.1, 12.6, 14.2
  const int fill = (4096 + rows - 1) / rows, most = (chunks + 5) / 6;
  const int want = fill > chunks ? chunks : fill > most ? fill : most;
  // (a grid has fewer than 2^32 threads, 64 for a segment in workgroups of four: 2^24 rows leave three)
  const int room = ((1 << 26) - 4) / rows;
  return want < room ? want : room;
}

hipError_t launch_qk_norm_rope(QkArgs a, int dtype, hipStream_t st) {
  a.segments = qk_segments(a.rows, a.dh, a.H, a.Hk, a.Hv);
  if (dtype == 0) a.halves ? launch_qk<float, true>(a, st) : launch_qk<float, false>(a, st);
  else a.halves ? launch_qk<bf16_t, true>(a, st) : launch_qk<bf16_t, false>(a, st);
  return hipGetLastError();
}

}  // namespace ditmi
