// Masked attention over documents, bf16: packed or padded documents, key
// lengths, causal and prefix masks, scores capped by a tanh or biased by the
// distance, heads that share keys (ditmi.h: dit_attention).
#include <algorithm>

#include "common.h"
#include "doc.h"
#include "kernels.h"

namespace ditmi {

typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int DH>
struct DocCfg {
  static constexpr int DHP = (DH + 15) / 16 * 16;
  static constexpr int BKV = 64;
  static constexpr int ROW = DHP * 2;            // bytes per K or V row in LDS
  static constexpr int CPR = ROW / 16;           // 16-byte chunks per row ...
  static constexpr int RC = DH / 8;              // ... of which hold data
  static constexpr int TILE = BKV * ROW;         // bytes of a K or V tile
  static constexpr int SLOT = 2 * TILE;
  static constexpr int DT = (DH + 31) / 32;      // 32-row tiles of O^T
  static constexpr int KS = DHP / 16;
  static constexpr int DMA = TILE / 1024;        // DMA instructions of a K or V tile
  static constexpr int STAGES = 3;
  // stored position of 16-byte chunk c of K row r / V row r
  static __device__ __forceinline__ int pos_k(int r, int c) {
    return c ^ (DHP == 128 ? (r & 15) : (DHP == 64 ? ((r >> 1) & 7) : ((r >> 3) & 1)));
  }
  // A transposed read takes 64 bytes of each of four consecutive rows: they
  // go to different quarters of the 64 banks.
  static __device__ __forceinline__ int pos_v(int r, int c) {
    return c ^ (DHP == 128 ? (r & 3) << 2 : (DHP == 64 ? ((r >> 1) & 1) << 2 : 0));
  }
  static_assert(TILE % 1024 == 0, "tiles are whole 1 KB DMA blocks");
};

template <int DH, int NW, bool CAP, bool BIAS>
__global__ __launch_bounds__(NW * 64) void doc_attn_bf16_kernel(DocAttnArgs a) {
  using C = DocCfg<DH>;
  constexpr int BM = NW * 32;
  constexpr int IPW = (2 * C::DMA + NW - 1) / NW;
  // ring of slots, then a line that absorbs spare DMAs (and what transposed
  // reads of head_dim 72 touch past the last V row)
  __shared__ __attribute__((aligned(1024))) unsigned char smem[C::STAGES * C::SLOT + 1024];

  __shared__ int bad[3][DH];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r32 = lane & 31;
  const Doc doc = load_doc(a, blockIdx.y);
  const int rows = doc.nq * a.G;
  const int nqb = (rows + BM - 1) / BM;
  const int items = nqb * a.Hk;
  if ((int)blockIdx.x >= items) return;
  const int item = xcd_remap(blockIdx.x, items);
  const int hk = item / nqb;
  // heaviest query blocks first where later queries see more keys
  const int qb = a.mask ? nqb - 1 - item % nqb : item % nqb;
  const int r0 = qb * BM + wave * 32;                     // first row of this wave
  const int row = min(r0 + r32, rows - 1);                // lanes past the end repeat the last row
  const int qi = row / a.G, h = hk * a.G + row % a.G;
  const int lim = row_limit(a, doc, qi);
  const int lim_lo = __builtin_amdgcn_readfirstlane(row_limit(a, doc, min(qb * BM, rows - 1) / a.G));
  const int lim_hi = __builtin_amdgcn_readfirstlane(row_limit(a, doc, min(qb * BM + BM - 1, rows - 1) / a.G));

  const int nkv_all = (lim_hi + C::BKV - 1) / C::BKV;
  const int part = blockIdx.z;
  const int t0 = (int)((long)nkv_all * part / a.split), t1 = (int)((long)nkv_all * (part + 1) / a.split);

  const bf16_t* __restrict__ kp = (const bf16_t*)a.k + (long)doc.k0 * a.k_row + hk * a.k_head;
  const bf16_t* __restrict__ vp = (const bf16_t*)a.v + (long)doc.k0 * a.v_row + hk * a.v_head;
  const bf16_t* __restrict__ qp = (const bf16_t*)a.q + (long)(doc.q0 + qi) * a.q_row + h * a.q_head;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));

  bf16x8 qf[C::KS];
#pragma unroll
  for (int s = 0; s < C::KS; ++s)
    qf[s] = s * 16 + g * 8 < DH ? *(const bf16x8*)(qp + s * 16 + g * 8) : bf16x8{};

  // DMA of one tile into its slot: instruction i < DMA covers K bytes
  // [1024 i, +1024), the next DMA the V bytes.  The pad chunk of head_dim 72's
  // rows is no lane's: it keeps the zeros written below.
  auto issue = [&](int tile) {
    const unsigned base = lds0 + (unsigned)((tile % C::STAGES) * C::SLOT);
    const int kv0 = min(tile, t1 - 1) * C::BKV;
#pragma unroll
    for (int t = 0; t < IPW; ++t) {
      const int qi_ = wave + NW * t;
      if (qi_ < 2 * C::DMA) {
        const bool isv = qi_ >= C::DMA;
        const int byte = (isv ? qi_ - C::DMA : qi_) * 1024 + lane * 16;
        const int R = byte / C::ROW, pos = (byte % C::ROW) >> 4;
        const int c = isv ? C::pos_v(R, pos) : C::pos_k(R, pos);
        const long key = min(kv0 + R, doc.nk - 1);
        const bf16_t* src = isv ? vp + key * a.v_row + c * 8 : kp + key * a.k_row + c * 8;
        if (c < C::RC) dma_16(src, base + (unsigned)(qi_ * 1024));
      }
    }
  };
  for (int e = tid; e < 3 * DH; e += NW * 64) bad[0][e] = NO_KEY;
  if (C::CPR > C::RC) {
    for (int e = tid; e < 256; e += NW * 64) ((uint32_t*)(smem + C::STAGES * C::SLOT))[e] = 0;
    for (int e = tid; e < C::STAGES * 2 * C::BKV * 4; e += NW * 64) {
      const int R = (e >> 2) & (C::BKV - 1), half = e >> 2 >> 6;  // K or V tile of a slot
      const int pos = half & 1 ? C::pos_v(R, C::RC) : C::pos_k(R, C::RC);
      ((uint32_t*)(smem + half * C::TILE + R * C::ROW + pos * 16))[e & 3] = 0;
    }
  }

  int k_off[C::KS];
#pragma unroll
  for (int s = 0; s < C::KS; ++s) k_off[s] = r32 * C::ROW + (C::pos_k(r32, 2 * s + g) << 4);
  // transposed reads: of each 16-lane group lane l addresses 8 bytes of row
  // l / 4 and receives column l of the four rows (keys 4 g .. 4 g + 3)
  int v_off[C::DT];
  {
    const int R = 4 * g + ((lane & 15) >> 2), half = (lane >> 4) & 1;
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
      v_off[t] = C::TILE + R * C::ROW + (C::pos_v(R, t * 4 + half * 2 + ((lane & 3) >> 1)) << 4) + (lane & 1) * 8;
  }

  const float sc = a.scale * LOG2E;
  const float cap_in = CAP ? 2.0f * sc / a.cap : 0.f, cap_out = CAP ? a.cap * LOG2E : 0.f;
  const float slope = BIAS ? a.slopes[h] * LOG2E : 0.f;
  const int here = qi + doc.nk - doc.nq;
  const float TAU = 64.0f;
  // V values that are not finite, in tiles that some row does not see whole:
  // a product would bring them to the other rows too (0 * inf).  They are
  // taken out of LDS, and bad[class][column] keeps the first key of each
  // class (NaN, +inf, -inf); the rows whose limit lies behind it get theirs
  // at the end.
  auto clean_v = [&](int tile) {
    unsigned char* vt = smem + (tile % C::STAGES) * C::SLOT + C::TILE;
    for (int e = tid; e < C::BKV * C::RC; e += NW * 64) {
      const int R = e / C::RC, c = e - R * C::RC;
      bf16_t* p = (bf16_t*)(vt + R * C::ROW + C::pos_v(R, c) * 16);
      const u32x4 w = *(const u32x4*)p;
      uint32_t any = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        any |= ((w[x] & 0x7F80u) == 0x7F80u) | ((w[x] & 0x7F800000u) == 0x7F800000u);
      if (any) keep_bad(bad, p, 8, c * 8, tile * C::BKV + R);
    }
  };
  float m_run = -INFINITY, l_run = 0.f;
  f32x16 oacc[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t) oacc[t] = f32x16{};

  if (t0 < t1)
#pragma unroll
    for (int s = 0; s < C::STAGES - 1; ++s) issue(t0 + s);

  for (int it = t0; it < t1; ++it) {
    const int kv0 = it * C::BKV;
    wait_vmcnt<0>();
    __syncthreads();
    issue(it + C::STAGES - 1);
    const unsigned char* slot = smem + (it % C::STAGES) * C::SLOT;
    const bool masked = kv0 + C::BKV > lim_lo;  // some row of the workgroup does not see the whole tile

    if (masked) clean_v(it);
    f32x16 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      s[kt] = f32x16{};
#pragma unroll
      for (int st = 0; st < C::KS; ++st) {
        const bf16x8 kf = *(const bf16x8*)(slot + kt * 32 * C::ROW + k_off[st]);
        s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[st], s[kt], 0, 0, 0);
      }
    }
    // scores in the exp2 domain (lane: key kv0 + kt*32 + 8*(e/4) + 4*g + e%4 of its own row)
    float m = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = kv0 + kt * 32 + (e >> 2) * 8 + g * 4 + (e & 3);
        float z = s[kt][e];
        if (CAP) {
          z = cap_out - 2.0f * cap_out * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z * cap_in) + 1.0f);
        } else {
          z *= sc;
        }
        if (BIAS) z -= slope * fabsf((float)(here - key));
        if (masked && key >= lim) z = -INFINITY;
        s[kt][e] = z;
        m = fmaxf(m, z);
      }
    m = max_halves(m);
    if (__builtin_amdgcn_ballot_w64(m > m_run + TAU) != 0) {
      const float m_new = fmaxf(m_run, m);
      // nothing seen so far: O and l are zero, any finite factor will do
      const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int t = 0; t < C::DT; ++t) oacc[t] *= alpha;
      m_run = m_new;
    }
    const float mneg = m_run == -INFINITY ? 0.f : -m_run;
    u32x4 pw[4];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kt][e] = __builtin_amdgcn_exp2f(s[kt][e] + mneg);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        pw[c][w] = pack_bf16x2(s[c >> 1][(c & 1) * 8 + 2 * w], s[c >> 1][(c & 1) * 8 + 2 * w + 1]);
        l_run += __uint_as_float(pw[c][w] << 16) + __uint_as_float(pw[c][w] & 0xFFFF0000u);
      }
    auto vread = [&](int c, int t) {
      typedef __attribute__((address_space(3))) s16x4* lds_p;
      const unsigned ad = lds0 + (unsigned)((it % C::STAGES) * C::SLOT + v_off[t] + c * 16 * C::ROW);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(size_t)ad);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(size_t)(ad + 8 * C::ROW));
      const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
      return u32x4{l2[0], l2[1], h2[0], h2[1]};
    };
    if (masked) __syncthreads();  // the tile's V has been cleaned
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int t = 0; t < C::DT; ++t)
        oacc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vread(c, t)),
                                                          __builtin_bit_cast(bf16x8, pw[c]), oacc[t], 0, 0, 0);
  }
  wait_vmcnt<0>();
  __syncthreads();
  if (lim_lo < nkv_all * C::BKV)
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int d = t * 32 + (e >> 2) * 8 + g * 4 + (e & 3);
        if (d < DH) oacc[t][e] = add_bad(oacc[t][e], bad, d, lim);
      }

  const float l_tot = sum_halves(l_run);
  const bool live = r0 + r32 < rows;
  if (a.split > 1) {
    if (!live) return;
    float* pr = a.part + ((long)part * a.q_rows * a.H + (long)(doc.q0 + qi) * a.H + h) * (DH + 4);
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const int d = t * 32 + jj * 8 + g * 4;
        if (d < DH)
          *(f32x4*)(pr + d) = f32x4{oacc[t][jj * 4 + 0], oacc[t][jj * 4 + 1], oacc[t][jj * 4 + 2], oacc[t][jj * 4 + 3]};
      }
    if (g == 0) *(f32x2*)(pr + DH) = f32x2{m_run, l_tot};
    return;
  }
  const float inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;  // no visible key: zeros
  bf16_t* op = (bf16_t*)a.o + (long)(doc.q0 + qi) * a.o_row + h * a.o_head;
  // lane half g holds columns 8 jj + 4 g .. +3: a swap between the halves
  // gives each lane 16 contiguous bytes
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int jp = 0; jp < 2; ++jp) {
      const int d0 = t * 32 + jp * 16;
      auto word = [&](int jj, int k) {
        return pack_bf16x2(oacc[t][jj * 4 + 2 * k] * inv, oacc[t][jj * 4 + 2 * k + 1] * inv);
      };
      u32x4 w;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const auto r = __builtin_amdgcn_permlane32_swap(word(2 * jp, k), word(2 * jp + 1, k), false, false);
        w[k] = r[0];
        w[2 + k] = r[1];
      }
      if (live && d0 + g * 8 < DH) *(u32x4*)(op + d0 + g * 8) = w;
    }
}

// Joins the key ranges of a split call: with m = max_s m_s and f_s = 2^(m_s - m),
// O = sum_s f_s O_s / sum_s f_s l_s, ranges in order.  One thread takes four
// columns of one (query, head).
template <int DH, typename T>
__global__ __launch_bounds__(256) void doc_attn_merge_kernel(DocAttnArgs a) {
  constexpr int G4 = DH / 4;
  const Doc doc = load_doc(a, blockIdx.y);
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  const long rh = i / G4;
  if (rh >= (long)doc.nq * a.H) return;
  const int d = (int)(i - rh * G4) * 4, qi = (int)(rh / a.H), h = (int)(rh - (long)qi * a.H);
  const float* p = a.part + ((long)(doc.q0 + qi) * a.H + h) * (DH + 4);
  const long stride = (long)a.q_rows * a.H * (DH + 4);
  float m = -INFINITY;
  for (int s = 0; s < a.split; ++s) m = fmaxf(m, p[s * stride + DH]);
  const float mr = m == -INFINITY ? 0.f : m;
  float den = 0.f;
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.split; ++s) {
    const f32x2 ml = *(const f32x2*)(p + s * stride + DH);
    const float f = __builtin_amdgcn_exp2f(ml[0] - mr);
    // an empty range has m = -inf and zeros
    den += f * ml[1];
    num += f * *(const f32x4*)(p + s * stride + d);
  }
  const float inv = den == 0.f ? 0.f : 1.0f / den;
  T* op = (T*)a.o + (long)(doc.q0 + qi) * a.o_row + h * a.o_head + d;
  if constexpr (sizeof(T) == 2)
    *(u32x2*)op = u32x2{pack_bf16x2(num[0] * inv, num[1] * inv), pack_bf16x2(num[2] * inv, num[3] * inv)};
  else
    *(f32x4*)op = num * inv;
}

template <int DH>
static hipError_t launch_dh(const DocAttnArgs& a, hipStream_t st) {
  constexpr int NW = 4;
  const long nqb = ((long)a.max_q * a.G + NW * 32 - 1) / (NW * 32);
  const dim3 grid((unsigned)(nqb * a.Hk), a.docs, a.split), block(NW * 64);
  const bool cap = a.cap > 0.f, bias = a.slopes != nullptr;
  if (cap && bias) hipLaunchKernelGGL((doc_attn_bf16_kernel<DH, NW, true, true>), grid, block, 0, st, a);
  else if (cap) hipLaunchKernelGGL((doc_attn_bf16_kernel<DH, NW, true, false>), grid, block, 0, st, a);
  else if (bias) hipLaunchKernelGGL((doc_attn_bf16_kernel<DH, NW, false, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((doc_attn_bf16_kernel<DH, NW, false, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_doc_attn_bf16(const DocAttnArgs& a, const DocAttnPlan& p, int head_dim, hipStream_t st) {
  switch (head_dim) {
    case 64: return launch_dh<64>(a, st);
    case 72: return launch_dh<72>(a, st);
    case 128: return launch_dh<128>(a, st);
    default: return hipErrorInvalidValue;
  }
}

template <int DH>
static void merge_dh(const DocAttnArgs& a, int dtype, hipStream_t st) {
  const long n = (long)a.max_q * a.H * (DH / 4);
  const dim3 grid((unsigned)((n + 255) / 256), a.docs);
  if (dtype == 1) hipLaunchKernelGGL((doc_attn_merge_kernel<DH, bf16_t>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((doc_attn_merge_kernel<DH, float>), grid, dim3(256), 0, st, a);
}
hipError_t launch_doc_attn_merge(const DocAttnArgs& a, int head_dim, int dtype, hipStream_t st) {
  switch (head_dim) {
    case 64: merge_dh<64>(a, dtype, st); break;
    case 72: merge_dh<72>(a, dtype, st); break;
    case 128: merge_dh<128>(a, dtype, st); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

// A grid of fewer than 256 workgroups leaves compute units idle: the keys are
// divided until there are about two workgroups for each, with at least four
// tiles per range.
DocAttnPlan doc_attn_plan(const DocAttnArgs& a, int head_dim, int dtype) {
  DocAttnPlan p{DOC_ROWS, 1};
  const long bm = 128;
  const long per_doc = ((long)a.max_q * a.G + bm - 1) / bm;
  const long items = a.Hk * std::max(1L, std::min(a.docs * per_doc, (long)a.q_rows * a.G / bm + a.docs));
  const long tiles = ((long)a.max_k + 63) / 64;
  if (items < 256) p.split = (int)std::max(1L, std::min({512 / items, tiles / 4, 32L}));
  return p;
}

}  // namespace ditmi
