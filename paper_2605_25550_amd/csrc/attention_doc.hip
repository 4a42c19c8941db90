// Masked attention over documents, bf16: packed or padded documents, key
// lengths, causal and prefix masks, scores capped by a tanh or biased by the
// distance, heads that share keys (ditmi.h: dit_attention).
//
// Orientation and schedule are those of the block's attention: a wave owns 32
// rows (query, head of the group that shares keys) and computes S^T = K Q^T with
// v_mfma_f32_32x32x16_bf16, so that a lane holds scores of one row, then
// O^T += V^T P^T with the probabilities as they lie; K and V tiles of 64 keys go
// HBM -> LDS by DMA into a ring of four slots, two to three tiles ahead.  What
// differs: the tensors are the caller's (token-major, strided), so V^T comes from
// V's rows by the transposing LDS read (ds_read_b64_tr_b16: of each 16 lanes,
// lane l addresses 8 bytes of row l / 4 and receives column l of the four rows),
// and the scale is applied in fp32 to the scores.
//
// Every mask is a limit per row, keys j < lim.  Tiles that every row of the
// workgroup sees whole run software-pipelined: the QK^T MFMAs of tile j + 1 are
// issued between the exponentials of tile j, its PV MFMAs between the row maxima
// of tile j + 1.  The few others (the last of a document, those on the diagonal)
// run one after the other, with the limits applied.
//
// The running max moves only when a tile exceeds it by more than 2^16, which keeps
// the rescale rare; probabilities are taken relative to 2^16 times it, so that none
// exceeds 1 and a sum over keys stays below their number times the largest value
// (values of v below 2^-110 lose digits instead).  A lead of 2^64 is reached less
// often where a distance bias lifts every tile over the last: 4352 queries and keys, 24
// heads, 273 us against 280.
// They are rounded to bf16 for the PV product (half a step, 2^-8 of each) and summed
// as rounded, so that a common error cancels.
//
// Bound by the matrix pipe and the vector instructions beside it (32 exponentials,
// scalings, maxima and packs per lane and tile), which overlap in part: MFMA busy
// 56% of the cycles at head_dim 128 (4352 queries and keys, 24 heads: 228 us, 1.02
// PFLOP/s; clips of 12870 and 4680: 1910 us, 1.21), 28% at head_dim 72, whose
// products pad to 80 and 96 columns (4 x 1024, 16 heads: 31.6 us, 0.61 PFLOP/s; a
// slope of 1.5 us per tile and 8 us besides).  256 rows per workgroup, because
// each row's share of the LDS reads of K and V falls with them; four waves a
// workgroup were slower, and key ranges pay in few grids only (doc_attn_plan).
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
  static constexpr int ROW = DHP * 2;            // bytes per K row in LDS ...
  // ... and per V row: a transposed read takes 64 bytes of each of four
  // consecutive rows, which 192 bytes (unlike 160) send to different banks
  static constexpr int VROW = DHP == 80 ? 192 : ROW;
  static constexpr int RC = DH / 8;              // 16-byte chunks of a row that hold data
  static constexpr int TILE = BKV * ROW, VTILE = BKV * VROW;  // bytes of a K, a V tile
  static constexpr int DT = (DH + 31) / 32;      // 32-row tiles of O^T
  static constexpr int KS = DHP / 16;
  static constexpr int KDMA = TILE / 1024, VDMA = VTILE / 1024;  // DMA instructions of a K, a V tile
  static constexpr int ST = 4;                   // ring slots: the K tiles of all, then the V tiles
  // head_dim 72: V's pad column 72 holds ones, so that O^T row 72 is the row sum
  static constexpr bool FOLD = DHP > DH;
  static constexpr int LT = DH / 32, LG = (DH % 32) % 8 / 4, LE = (DH % 32) / 8 * 4 + DH % 4;
  // stored position of 16-byte chunk c of K row r / V row r
  static __device__ __forceinline__ int pos_k(int r, int c) {
    return c ^ (DHP == 128 ? (r & 15) : (DHP == 64 ? ((r >> 1) & 7) : ((r >> 3) & 1)));
  }
  // (a transposed read's four rows in different quarters of the 64 banks)
  static __device__ __forceinline__ int pos_v(int r, int c) {
    return c ^ (DHP == 128 ? (r & 3) << 2 : (DHP == 64 ? ((r >> 1) & 1) << 2 : 0));
  }
  static_assert(TILE % 1024 == 0 && VTILE % 1024 == 0 && ST * VTILE <= 65536, "whole DMA blocks; slot offsets fit the LDS immediate");
  static_assert(DT * 64 <= VROW, "transposed reads stay in their rows");
};

// Holds a value's computation where it is written: the compiler orders pure
// arithmetic by its uses, past the scheduling barriers between matrix products.
__device__ __forceinline__ void pin(float& x) { asm volatile("" : "+v"(x)); }

typedef __attribute__((address_space(3))) unsigned char lds_byte;
__device__ __forceinline__ s16x4 read_tr(const lds_byte* p) {
  typedef __attribute__((address_space(3))) s16x4* lds_p;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)p);
}

// The pad chunk (columns 72 .. 79) of head_dim 72's K rows, and of its V rows.
__device__ const uint32_t doc_pads[8] = {0u, 0u, 0u, 0u, 0x3F80u, 0u, 0u, 0u};

// A row's scores, raw -> z (the exponent in the exp2 domain) -> probability.  The
// scale and the cap keep the order of scores, so that they can wait for the
// exponential, after the row max; the bias cannot.
template <bool CAP, bool BIAS>
struct DocScore {
  float sc, cap_in, cap_out, slope;
  int here;
  __device__ __forceinline__ DocScore(const DocAttnArgs& a, int h, int place) {
    sc = a.scale * LOG2E;
    cap_in = CAP ? 2.0f * sc / a.cap : 0.f;
    cap_out = CAP ? a.cap * LOG2E : 0.f;
    slope = BIAS ? a.slopes[h] * LOG2E : 0.f;
    here = place;  // the key at the row's own place: distances to it are taken as integers
  }
  // cap tanh(s scale / cap) = cap - 2 cap / (exp(2 s scale / cap) + 1), plus `more`, in the exp2 domain
  __device__ __forceinline__ float capped(float s, float more) const {
    return fmaf(-2.0f * cap_out, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s * cap_in) + 1.0f), cap_out + more);
  }
  // before the max; the key is `first - off` places before the row's own
  __device__ __forceinline__ float pre(float s, float first, int off) const {
    if (!BIAS) return s;
    return fmaf(-slope, fabsf(first - (float)off), CAP ? capped(s, 0.f) : s * sc);
  }
  __device__ __forceinline__ float z_of_max(float m) const { return BIAS ? m : CAP ? capped(m, 0.f) : m * sc; }
  __device__ __forceinline__ float prob(float s, float mneg) const {
    return __builtin_amdgcn_exp2f(BIAS ? s + mneg : CAP ? capped(s, mneg) : fmaf(s, sc, mneg));
  }
};

// Values of a V tile (in LDS from vt, key kv0 on) that are not finite are noted
// in bad and become 0; NT threads share the work, all their reads in flight.
template <int DH, int NT>
__device__ __forceinline__ void clean_v(int (&bad)[3][DH], unsigned char* vt, int kv0, int t) {
  using C = DocCfg<DH>;
  constexpr int N = C::BKV * C::RC, PER = (N + NT - 1) / NT;
  auto at = [&](int i) {
    const int e = min(t + i * NT, N - 1), R = e / C::RC, c = e - R * C::RC;
    return (bf16_t*)(vt + R * C::VROW + C::pos_v(R, c) * 16);
  };
  uint32_t odd = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const u32x4 w = *(const u32x4*)at(i);
    uint32_t any = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) any |= ((w[x] & 0x7F80u) == 0x7F80u) | ((w[x] & 0x7F800000u) == 0x7F800000u);
    odd |= any << i;
  }
  for (; odd; odd &= odd - 1) {
    const int i = __builtin_ctz(odd), e = min(t + i * NT, N - 1), R = e / C::RC;
    keep_bad(bad, at(i), 8, (e - R * C::RC) * 8, kv0 + R);
  }
}

template <int DH, int NW, bool CAP, bool BIAS>
__global__ __launch_bounds__(NW * 64, 1) void doc_attn_bf16_kernel(DocAttnArgs a) {
  using C = DocCfg<DH>;
  constexpr int ST = C::ST, BM = NW * 32;
  constexpr int NDMA = C::KDMA + C::VDMA, IPW = (NDMA + NW - 1) / NW;  // DMA instructions per wave and tile (uniform)
  constexpr bool SPARE = IPW * NW > NDMA;
  constexpr int VBASE = ST * C::TILE, SPARE_AT = VBASE + ST * C::VTILE;
  // the ring, then a line that absorbs spare DMAs
  __shared__ __attribute__((aligned(1024))) unsigned char smem[ST * (C::TILE + C::VTILE) + 1024];
  __shared__ int bad[3][DH];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r32 = lane & 31;
  const Doc doc = load_doc(a, blockIdx.y);
  const int rows = doc.nq * a.G;
  const int nqb = (rows + BM - 1) / BM;
  const int items = nqb * a.Hk;
  if ((int)blockIdx.x >= items) return;
  // query blocks of a head in contiguous ranges per XCD: they share its K and V
  // in that XCD's L2; heaviest first where later queries see more keys
  const int item = xcd_remap(blockIdx.x, items);
  const int hk = item / nqb;
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
  const int tf = max(t0, min(t1, lim_lo / C::BKV));       // tiles [t0, tf) are seen whole

  const bf16_t* __restrict__ kp = (const bf16_t*)a.k + (long)doc.k0 * a.k_row + hk * a.k_head;
  const bf16_t* __restrict__ vp = (const bf16_t*)a.v + (long)doc.k0 * a.v_row + hk * a.v_head;
  const bf16_t* __restrict__ qp = (const bf16_t*)a.q + (long)(doc.q0 + qi) * a.q_row + h * a.q_head;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));

  bf16x8 qf[C::KS];
#pragma unroll
  for (int s = 0; s < C::KS; ++s)
    qf[s] = s * 16 + g * 8 < DH ? *(const bf16x8*)(qp + s * 16 + g * 8) : bf16x8{};

  // DMA of one tile into its slot: instruction i < KDMA covers K bytes
  // [1024 i, +1024), the next VDMA the V bytes; wave w issues i = w + NW t.  The
  // source is a scalar base (the tile's first row) plus a 32-bit lane offset;
  // the last tile's rows past the document's end repeat its last row.  Head_dim
  // 72's pad chunks come from doc_pads: a select, because a branch around the copy
  // (lanes switched off) would end the basic block, and the compiler would sink
  // the exponentials out of the products they are meant to run beside.
  // Past the last tile, and for spare instructions, the copy goes to the spare
  // line, so that every wave counts the same.
  const int kv_last = (t1 - 1) * C::BKV;  // (some of its rows may lie past the end)
  unsigned off[IPW], off_last[IPW];
  bool copies[IPW];
#pragma unroll
  for (int t = 0; t < IPW; ++t) {
    const int i = wave + NW * t;  // wave-uniform
    const bool real = !SPARE || i < NDMA, isv = real && i >= C::KDMA;
    const int byte = (isv ? i - C::KDMA : real ? i : 0) * 1024 + lane * 16, pitch = isv ? C::VROW : C::ROW;
    const int R = byte / pitch, pos = (byte - R * pitch) >> 4, c = isv ? C::pos_v(R, pos) : C::pos_k(R, pos);
    const unsigned rs = (unsigned)(isv ? a.v_row : a.k_row) * 2;
    off[t] = R * rs + c * 16;
    off_last[t] = min(R, doc.nk - 1 - kv_last) * rs + c * 16;
    copies[t] = !C::FOLD || c < C::RC;
  }
  auto issue_one = [&](int tile, int slot, int t) {
    const int i = wave + NW * t;
    const bool real = !SPARE || i < NDMA, isv = real && i >= C::KDMA;
    const int tl = min(tile, t1 - 1);
    const bf16_t* base = isv ? vp + (long)(tl * C::BKV) * a.v_row : kp + (long)(tl * C::BKV) * a.k_row;
    const unsigned dst = real && tile < t1 ? lds0 + (isv ? VBASE + slot * C::VTILE + (i - C::KDMA) * 1024 : slot * C::TILE + i * 1024)
                                           : lds0 + SPARE_AT;
    const unsigned o = tl == t1 - 1 ? off_last[t] : off[t];
    if (C::FOLD)
      dma_16(copies[t] ? (const void*)((const char*)base + o) : (const void*)(doc_pads + (isv ? 4 : 0)), dst);
    else
      dma_16s(base, o, dst);
  };
  for (int e = tid; e < 3 * DH; e += NW * 64) bad[0][e] = NO_KEY;

  const lds_byte* k_at[C::KS];
#pragma unroll
  for (int s = 0; s < C::KS; ++s) k_at[s] = (const lds_byte*)smem + r32 * C::ROW + (C::pos_k(r32, 2 * s + g) << 4);
  const lds_byte* v_at[C::DT];
  {
    const int R = 4 * g + ((lane & 15) >> 2), half = (lane >> 4) & 1;
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
      v_at[t] = (const lds_byte*)smem + VBASE + R * C::VROW +
                (C::pos_v(R, t * 4 + half * 2 + ((lane & 3) >> 1)) << 4) + (lane & 1) * 8;
  }
  auto kread = [&](int slot, int kt, int s) {
    return *(const __attribute__((address_space(3))) bf16x8*)(k_at[s] + slot * C::TILE + kt * 32 * C::ROW);
  };
  // keys 16 c + 4 g + 0..3 and 16 c + 8 + 4 g + 0..3 of column 32 t + r32: the
  // keys of the lane's probabilities
  auto vread = [&](int slot, int c, int t) {
    const lds_byte* p = v_at[t] + slot * C::VTILE + c * 16 * C::VROW;
    const u32x2 lo = __builtin_bit_cast(u32x2, read_tr(p)), hi = __builtin_bit_cast(u32x2, read_tr(p + 8 * C::VROW));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
  };

  const DocScore<CAP, BIAS> score(a, h, qi + doc.nk - doc.nq);
  auto pre = [&](float x, float first, int kt, int e) { return score.pre(x, first, kt * 32 + (e >> 2) * 8 + (e & 3)); };
  const float TAU = 16.0f;
  float m_run = -INFINITY, mneg = 0.f;  // mneg = -(m_run + TAU), 0 while nothing has been seen
  auto prob = [&](float x) { return score.prob(x, mneg); };
  // Row sums of the bf16 probabilities (the values the PV product multiplies) on
  // the matrix pipe: a 4x4x4 MFMA with ones adds the four of a lane's operand.
  f32x4 lacc = f32x4{};
  typedef short i16x4 __attribute__((ext_vector_type(4)));
  const i16x4 ones4 = {0x3F80, 0x3F80, 0x3F80, 0x3F80};
  auto add_sum = [&](uint32_t w0, uint32_t w1) {
    if (!C::FOLD) lacc = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones4, __builtin_bit_cast(i16x4, u32x2{w0, w1}), lacc, 0, 0, 0);
  };
  f32x16 oacc[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t) oacc[t] = f32x16{};
  auto pv = [&](const u32x4& v, const u32x4& p, int t) {
    oacc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p), oacc[t], 0, 0, 0);
  };
  // moves the running max to that of a tile (z domain, whole row) where it leads by more than 2^TAU
  auto lead = [&](float z) {
    if (__builtin_amdgcn_ballot_w64(z > m_run + TAU) == 0) return;
    const float m_new = fmaxf(m_run, z);
    // nothing seen so far: O and l are zero, any finite factor will do
    const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
    lacc *= alpha;
#pragma unroll
    for (int t = 0; t < C::DT; ++t) oacc[t] *= alpha;
    m_run = m_new;
    mneg = m_new == -INFINITY ? 0.f : -m_new - TAU;
  };

  if (t0 < t1)
#pragma unroll
    for (int d = 0; d < ST - 1; ++d)
#pragma unroll
      for (int t = 0; t < IPW; ++t) issue_one(t0 + d, d, t);

  if (t0 < tf) {
    wait_vmcnt<(ST - 3) * IPW>();
    __syncthreads();
    f32x16 sa[2], sb[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      sa[kt] = f32x16{};
#pragma unroll
      for (int s = 0; s < C::KS; ++s) sa[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kread(0, kt, s), qf[s], sa[kt], 0, 0, 0);
    }
    float mcur = -INFINITY;  // row max of the current tile (what pre() gives), both halves
    {
      const float first = (float)(score.here - (t0 * C::BKV + 4 * g));
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          sa[kt][e] = pre(sa[kt][e], first, kt, e);
          mcur = fmaxf(mcur, sa[kt][e]);
        }
      mcur = max_halves(mcur);
    }
    // One key tile: the exponentials of scur (tile j, slot sj) beside the QK^T
    // MFMAs of tile j + 1 into snext, then the PV MFMAs of tile j beside the row
    // max of tile j + 1 and the DMA of tile j + 3.  (The last tile's QK^T reads
    // the slot behind it: computed, and not used.)
    auto tile_step = [&](const int j, const int sj, f32x16 (&scur)[2], f32x16 (&snext)[2]) __attribute__((always_inline)) {
      lead(score.z_of_max(mcur));
      constexpr int EX = C::FOLD || CAP ? 16 : 24;  // exponentials beside QK^T; the rest beside the first PV MFMAs
      constexpr int NP = 4 * C::DT, NPRE = EX / 8 * C::DT, ND = 3, NQ = 2 * C::KS;
      u32x4 pw[4], vf[3];
      auto pack = [&](int p) { pw[p >> 2][p & 3] = pack_bf16x2(scur[p >> 3][(2 * p) & 15], scur[p >> 3][(2 * p + 1) & 15]); };
      {
        const int sl = (sj + 1) % ST;
        bf16x8 kf[3];
        kf[0] = kread(sl, 0, 0);
        kf[1] = kread(sl, 1, 0);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          if (i + 2 < NQ) kf[(i + 2) % 3] = kread(sl, (i + 2) & 1, (i + 2) >> 1);
          snext[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % 3], qf[i >> 1], i < 2 ? f32x16{} : snext[i & 1], 0, 0, 0);
          if (i == NQ - 2) vf[0] = vread(sj, 0, 0);
          if (i == NQ - 1) vf[1] = vread(sj, 1 / C::DT, 1 % C::DT);
#pragma unroll
          for (int e = i * EX / NQ; e < (i + 1) * EX / NQ; ++e) {
            float x = prob(scur[e >> 4][e & 15]);
            pin(x);
            scur[e >> 4][e & 15] = x;
          }
#pragma unroll
          for (int p = 0; p < EX / 2; ++p)
            if (2 * p + 1 >= i * EX / NQ && 2 * p + 1 < (i + 1) * EX / NQ) pack(p);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      {
        const float first = (float)(score.here - ((j + 1) * C::BKV + 4 * g));
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          if (i + 2 < NP) vf[(i + 2) % 3] = vread(sj, (i + 2) / C::DT, (i + 2) % C::DT);
#pragma unroll
          for (int t = 0; t < IPW; ++t)
            if (i == t * (NP - ND) / IPW) issue_one(j + ST - 1, (sj + ST - 1) % ST, t);
          if (i < NP - ND) pv(vf[i % 3], pw[i / C::DT], i % C::DT);
#pragma unroll
          for (int e = i * 32 / NP; e < (i + 1) * 32 / NP; ++e) {
            snext[e >> 4][e & 15] = pre(snext[e >> 4][e & 15], first, e >> 4, e & 15);
            m = fmaxf(m, snext[e >> 4][e & 15]);
          }
          if (i % 4 == 3) pin(m);
          if (i < NPRE) {
#pragma unroll
            for (int e = EX + i * (32 - EX) / NPRE; e < EX + (i + 1) * (32 - EX) / NPRE; ++e)
            {
              float x = prob(scur[e >> 4][e & 15]);
              pin(x);
              scur[e >> 4][e & 15] = x;
            }
#pragma unroll
            for (int p = EX / 2; p < 16; ++p)
              if (2 * p + 1 >= EX + i * (32 - EX) / NPRE && 2 * p + 1 < EX + (i + 1) * (32 - EX) / NPRE) pack(p);
          }
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (i == (k * NP + NP - 1) / 8) add_sum(pw[k >> 1][(k & 1) * 2], pw[k >> 1][(k & 1) * 2 + 1]);
          __builtin_amdgcn_sched_barrier(0);
        }
        mcur = max_halves(m);
      }
      // tile j + 2 must have landed for every wave before the next QK^T, and
      // every wave must be done with tile j's slot before it is refilled; the
      // last PV MFMAs, on fragments in registers, run behind the barrier
      wait_vmcnt<(ST - 3) * IPW>();
      __syncthreads();
#pragma unroll
      for (int i = NP - ND; i < NP; ++i) pv(vf[i % 3], pw[i / C::DT], i % C::DT);
    };
    int j = t0;
    for (; j + 3 < tf; j += 4) {
      tile_step(j, 0, sa, sb);
      tile_step(j + 1, 1, sb, sa);
      tile_step(j + 2, 2, sa, sb);
      tile_step(j + 3, 3, sb, sa);
    }
    if (j < tf) tile_step(j, 0, sa, sb);
    if (j + 1 < tf) tile_step(j + 1, 1, sb, sa);
    if (j + 2 < tf) tile_step(j + 2, 2, sa, sb);
  }

  // Tiles that some row of the workgroup does not see whole.  Their V values that
  // are not finite would reach the other rows too (0 * inf): they are taken out
  // of LDS, bad[class][column] keeps the first key of each class (NaN, +inf,
  // -inf), and the rows whose limit lies behind it get theirs at the end.
  for (int it = tf; it < t1; ++it) {
    const int kv0 = it * C::BKV, slot = (it - t0) % ST;
    wait_vmcnt<0>();
    __syncthreads();
    for (int t = 0; t < IPW; ++t) issue_one(it + ST - 1, (slot + ST - 1) % ST, t);
    clean_v<DH, NW * 64>(bad, smem + VBASE + slot * C::VTILE, kv0, tid);
    f32x16 s[2];
    float m = -INFINITY;
    const float first = (float)(score.here - (kv0 + 4 * g));
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      s[kt] = f32x16{};
#pragma unroll
      for (int st = 0; st < C::KS; ++st) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kread(slot, kt, st), qf[st], s[kt], 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[kt][e] = kv0 + kt * 32 + (e >> 2) * 8 + g * 4 + (e & 3) < lim ? pre(s[kt][e], first, kt, e) : -INFINITY;
        m = fmaxf(m, s[kt][e]);
      }
    }
    m = max_halves(m);
    // The limit says what is visible, never the value: a raw score of -inf may be
    // visible, and -cap.  (Of a row without a visible key here the max stays -inf;
    // without a raw score to be capped, 2^-inf is the 0 of what is not visible.)
    lead(kv0 < lim ? score.z_of_max(m) : -INFINITY);
    const int seen = lim - kv0 - g * 4;
    auto seen_prob = [&](float x, int off) { return !CAP || BIAS || off < seen ? prob(x) : 0.f; };
    u32x4 pw[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int e = (c & 1) * 8 + 2 * w, off = (c >> 1) * 32 + (e >> 2) * 8 + (e & 3);
        pw[c][w] = pack_bf16x2(seen_prob(s[c >> 1][e], off), seen_prob(s[c >> 1][e + 1], off + 1));
        if (w & 1) add_sum(pw[c][w - 1], pw[c][w]);
      }
    __syncthreads();  // V has been cleaned
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int t = 0; t < C::DT; ++t) pv(vread(slot, c, t), pw[c], t);
  }
  wait_vmcnt<0>();
  __syncthreads();
  const float l_tot = sum_halves(C::FOLD ? (g == C::LG ? oacc[C::LT][C::LE] : 0.f) : lacc[0]);
  if (tf < t1)
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int d = t * 32 + (e >> 2) * 8 + g * 4 + (e & 3);
        if (d < DH) oacc[t][e] = add_bad(oacc[t][e], bad, d, lim);
      }

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

// Few rows (single tokens over a cache, bound by the keys' and values' bytes, and
// small grids, bound by the chain of tiles): a workgroup owns 32 rows, and its four
// waves take the 64-key tiles of its range in turn, each with a ring of its own
// (one K and one V tile, refilled as soon as it is used up) and a softmax state of
// its own, and no barrier until the four states are merged through LDS.  4 single
// tokens over caches of 77 to 4096 keys, 24 heads on 8 of 128: 17 us with the merge,
// 35 MB at 2.1 TB/s, a launch, a chain of loads per tile and the second launch (6 us
// at the rate of a large read); 256 queries and keys, 16 heads of 72: 8.4 us.
template <int DH, bool CAP, bool BIAS>
__global__ __launch_bounds__(256) void doc_attn_few_kernel(DocAttnArgs a) {
  using C = DocCfg<DH>;
  constexpr int NW = 4, OS = DH + 4;
  constexpr int RING = C::TILE + C::VTILE;  // of one wave
  static_assert(NW * RING >= NW * 32 * OS * 4, "the states are merged where the rings were");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[NW * RING];
  __shared__ float ml[NW][2][32];
  __shared__ int bad[3][DH];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, r32 = lane & 31;
  const Doc doc = load_doc(a, blockIdx.y);
  const int all_rows = doc.nq * a.G, nrb = (all_rows + 31) / 32, items = nrb * a.Hk, part = blockIdx.z;
  if ((int)blockIdx.x >= items) return;
  const int item = xcd_remap(blockIdx.x, items), hk = item / nrb, rb0 = item % nrb * 32;
  const int rows = min(32, all_rows - rb0);  // of this workgroup, from rb0 on
  const int row = rb0 + min(r32, rows - 1);
  const int qi = row / a.G, h = hk * a.G + row % a.G;
  const int lim = row_limit(a, doc, qi), lim_lo = row_limit(a, doc, rb0 / a.G), lim_hi = row_limit(a, doc, (rb0 + rows - 1) / a.G);
  const int nkv_all = (lim_hi + C::BKV - 1) / C::BKV;
  const int t0 = (int)((long)nkv_all * part / a.split), t1 = (int)((long)nkv_all * (part + 1) / a.split);

  const bf16_t* __restrict__ kp = (const bf16_t*)a.k + (long)doc.k0 * a.k_row + hk * a.k_head;
  const bf16_t* __restrict__ vp = (const bf16_t*)a.v + (long)doc.k0 * a.v_row + hk * a.v_head;
  const bf16_t* __restrict__ qp = (const bf16_t*)a.q + (long)(doc.q0 + qi) * a.q_row + h * a.q_head;
  unsigned char* ring = smem + wave * RING;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(ring));

  auto issue = [&](int tile, bool isv) {
    const int kv0 = tile * C::BKV;
    const long rs = isv ? a.v_row : a.k_row;
    const bf16_t* base = (isv ? vp : kp) + (long)kv0 * rs;
#pragma unroll
    for (int i = 0; i < (C::VDMA > C::KDMA ? C::VDMA : C::KDMA); ++i) {
      if (i >= (isv ? C::VDMA : C::KDMA)) break;
      const int byte = i * 1024 + lane * 16, pitch = isv ? C::VROW : C::ROW, R = byte / pitch, pos = (byte - R * pitch) >> 4;
      const int c = isv ? C::pos_v(R, pos) : C::pos_k(R, pos);
      const unsigned off = (unsigned)min(R, doc.nk - 1 - kv0) * (unsigned)(rs * 2) + c * 16;
      if (!C::FOLD || c < C::RC) dma_16s(base, off, lds0 + (isv ? C::TILE : 0) + i * 1024);
    }
  };
  if (t0 + wave < t1) {
    issue(t0 + wave, false);
    issue(t0 + wave, true);
  }
  bf16x8 qf[C::KS];
#pragma unroll
  for (int s = 0; s < C::KS; ++s)
    qf[s] = s * 16 + g * 8 < DH ? *(const bf16x8*)(qp + s * 16 + g * 8) : bf16x8{};
  for (int e = tid; e < 3 * DH; e += NW * 64) bad[0][e] = NO_KEY;
  if (C::FOLD)  // the pad chunks are no lane's: K's must be zero (what V's give is discarded)
    for (int e = lane; e < C::BKV * 4; e += 64)
      ((uint32_t*)(ring + (e >> 2) * C::ROW + C::pos_k(e >> 2, C::RC) * 16))[e & 3] = 0;
  __syncthreads();

  const lds_byte* k_at[C::KS];
#pragma unroll
  for (int s = 0; s < C::KS; ++s) k_at[s] = (const lds_byte*)ring + r32 * C::ROW + (C::pos_k(r32, 2 * s + g) << 4);
  const lds_byte* v_at[C::DT];
  {
    const int R = 4 * g + ((lane & 15) >> 2), half = (lane >> 4) & 1;
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
      v_at[t] = (const lds_byte*)ring + C::TILE + R * C::VROW +
                (C::pos_v(R, t * 4 + half * 2 + ((lane & 3) >> 1)) << 4) + (lane & 1) * 8;
  }
  const DocScore<CAP, BIAS> score(a, h, qi + doc.nk - doc.nq);
  float m_run = -INFINITY, l_run = 0.f;
  f32x16 oacc[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t) oacc[t] = f32x16{};
  // Q and the slope are here before the loop, whose waits count DMA alone
#pragma unroll
  for (int s = 0; s < C::KS; ++s) asm volatile("" : "+v"(qf[s]));
  if (BIAS) asm volatile("" : : "v"(score.slope));
  wait_vmcnt<0>();

  for (int it = t0 + wave; it < t1; it += NW) {
    const int kv0 = it * C::BKV;
    const bool more = it + NW < t1, masked = kv0 + C::BKV > lim_lo;
    if (it > t0 + wave) wait_vmcnt<C::VDMA>();  // this tile's K (its V, issued behind it, may still be under way)
    f32x16 s[2];
    float m = -INFINITY;
    const float first = (float)(score.here - (kv0 + 4 * g));
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      s[kt] = f32x16{};
#pragma unroll
      for (int st = 0; st < C::KS; ++st)
        s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            *(const __attribute__((address_space(3))) bf16x8*)(k_at[st] + kt * 32 * C::ROW), qf[st], s[kt], 0, 0, 0);
    }
    // the products have read K: its slot takes the next tile's
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) issue(it + NW, false);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int off = kt * 32 + (e >> 2) * 8 + (e & 3);
        s[kt][e] = kv0 + off + g * 4 < lim ? score.pre(s[kt][e], first, off) : -INFINITY;
        m = fmaxf(m, s[kt][e]);
      }
    m = max_halves(m);
    m = kv0 < lim ? score.z_of_max(m) : -INFINITY;
    const float m_new = fmaxf(m_run, m), mneg = m_new == -INFINITY ? 0.f : -m_new;
    const int seen = lim - kv0 - g * 4;  // (the limit says what is visible, as above)
    auto seen_prob = [&](float x, int off) { return !CAP || BIAS || off < seen ? score.prob(x, mneg) : 0.f; };
    const float alpha = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
    l_run *= alpha;
#pragma unroll
    for (int t = 0; t < C::DT; ++t) oacc[t] *= alpha;
    m_run = m_new;
    u32x4 pw[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int e = (c & 1) * 8 + 2 * w, off = (c >> 1) * 32 + (e >> 2) * 8 + (e & 3);
        pw[c][w] = pack_bf16x2(seen_prob(s[c >> 1][e], off), seen_prob(s[c >> 1][e + 1], off + 1));
        l_run += __uint_as_float(pw[c][w] << 16) + __uint_as_float(pw[c][w] & 0xFFFF0000u);
      }
    if (more) wait_vmcnt<C::KDMA>();  // this tile's V (the next K may be under way)
    else wait_vmcnt<0>();
    if (masked) {
      clean_v<DH, 64>(bad, ring + C::TILE, kv0, lane);
      wave_lds_fence();
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int t = 0; t < C::DT; ++t) {
        const lds_byte* p = v_at[t] + c * 16 * C::VROW;
        const u32x2 lo = __builtin_bit_cast(u32x2, read_tr(p)), hi = __builtin_bit_cast(u32x2, read_tr(p + 8 * C::VROW));
        oacc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]}),
                                                          __builtin_bit_cast(bf16x8, pw[c]), oacc[t], 0, 0, 0);
      }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) issue(it + NW, true);
  }

  __syncthreads();  // every ring has been read
  float* os = (float*)smem + wave * 32 * OS;
  l_run = sum_halves(l_run);
  if (r32 < rows) {
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const int d = t * 32 + jj * 8 + g * 4;
        if (d < DH)
          *(f32x4*)(os + r32 * OS + d) = f32x4{oacc[t][jj * 4 + 0], oacc[t][jj * 4 + 1], oacc[t][jj * 4 + 2], oacc[t][jj * 4 + 3]};
      }
    if (g == 0) ml[wave][0][r32] = m_run, ml[wave][1][r32] = l_run;
  }
  __syncthreads();
  constexpr int G4 = DH / 4;
  for (int i = tid; i < rows * G4; i += NW * 64) {
    const int r = i / G4, d = (i - r * G4) * 4, qr = (rb0 + r) / a.G, hr = hk * a.G + (rb0 + r) % a.G;
    float mx = ml[0][0][r];
#pragma unroll
    for (int w = 1; w < NW; ++w) mx = fmaxf(mx, ml[w][0][r]);
    const float mr = mx == -INFINITY ? 0.f : mx;
    float den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w][0][r] - mr);
      den += f * ml[w][1][r];
      num += f * *(const f32x4*)((const float*)smem + (w * 32 + r) * OS + d);
    }
    const int lim_r = row_limit(a, doc, qr);
#pragma unroll
    for (int x = 0; x < 4; ++x) num[x] = add_bad(num[x], bad, d + x, lim_r);
    if (a.split > 1) {
      float* pr = a.part + ((long)part * a.q_rows * a.H + (long)(doc.q0 + qr) * a.H + hr) * (DH + 4);
      *(f32x4*)(pr + d) = num;
      if (d == 0) *(f32x2*)(pr + DH) = f32x2{mx, den};
    } else {
      const float inv = den == 0.f ? 0.f : 1.0f / den;
      bf16_t* op = (bf16_t*)a.o + (long)(doc.q0 + qr) * a.o_row + hr * a.o_head + d;
      *(u32x2*)op = u32x2{pack_bf16x2(num[0] * inv, num[1] * inv), pack_bf16x2(num[2] * inv, num[3] * inv)};
    }
  }
}

// Joins the key ranges of a split call: with m = max_s m_s and f_s = 2^(m_s - m),
// O = sum_s f_s O_s / sum_s f_s l_s, ranges in order, eight loading at a time.
// One thread takes four columns of one (query, head).  Bound by its launch (about
// 3 us; the partial results are a few hundred KB in L2).
template <int DH, typename T>
__global__ __launch_bounds__(256) void doc_attn_merge_kernel(DocAttnArgs a) {
  constexpr int G4 = DH / 4, U = 8;
  const Doc doc = load_doc(a, blockIdx.y);
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  const long rh = i / G4;
  if (rh >= (long)doc.nq * a.H) return;
  const int d = (int)(i - rh * G4) * 4, qi = (int)(rh / a.H), h = (int)(rh - (long)qi * a.H);
  const float* p = a.part + ((long)(doc.q0 + qi) * a.H + h) * (DH + 4);
  const long stride = (long)a.q_rows * a.H * (DH + 4);
  float m = -INFINITY, den = 0.f;
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.split; s0 += U) {
    f32x2 ml[U];
    f32x4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* ps = p + min(s0 + u, a.split - 1) * stride;
      ml[u] = *(const f32x2*)(ps + DH);
      o[u] = *(const f32x4*)(ps + d);
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, ml[u][0]);
    const float mr = top == -INFINITY ? 0.f : top;  // an empty range has m = -inf and zeros
    const float keep = __builtin_amdgcn_exp2f(m - mr);
    den *= keep;
    num *= keep;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s0 + u < a.split) {
        const float f = __builtin_amdgcn_exp2f(ml[u][0] - mr);
        den += f * ml[u][1];
        num += f * o[u];
      }
    m = top;
  }
  const float inv = den == 0.f ? 0.f : 1.0f / den;
  T* op = (T*)a.o + (long)(doc.q0 + qi) * a.o_row + h * a.o_head + d;
  if constexpr (sizeof(T) == 2)
    *(u32x2*)op = u32x2{pack_bf16x2(num[0] * inv, num[1] * inv), pack_bf16x2(num[2] * inv, num[3] * inv)};
  else
    *(f32x4*)op = num * inv;
}

template <int DH, bool CAP, bool BIAS>
static void launch_score(const DocAttnArgs& a, const DocAttnPlan& p, hipStream_t st) {
  if (p.kernel == DOC_FEW) {
    hipLaunchKernelGGL((doc_attn_few_kernel<DH, CAP, BIAS>), dim3((unsigned)(((long)a.max_q * a.G + 31) / 32 * a.Hk), a.docs, a.split), dim3(256), 0, st, a);
  } else {
    const long nqb = ((long)a.max_q * a.G + 255) / 256;
    hipLaunchKernelGGL((doc_attn_bf16_kernel<DH, 8, CAP, BIAS>), dim3((unsigned)(nqb * a.Hk), a.docs, a.split), dim3(512), 0, st, a);
  }
}

template <int DH>
static hipError_t launch_dh(const DocAttnArgs& a, const DocAttnPlan& p, hipStream_t st) {
  const bool cap = a.cap > 0.f, bias = a.slopes != nullptr;
  if (cap && bias) launch_score<DH, true, true>(a, p, st);
  else if (cap) launch_score<DH, true, false>(a, p, st);
  else if (bias) launch_score<DH, false, true>(a, p, st);
  else launch_score<DH, false, false>(a, p, st);
  return hipGetLastError();
}

hipError_t launch_doc_attn_bf16(const DocAttnArgs& a, const DocAttnPlan& p, int head_dim, hipStream_t st) {
  switch (head_dim) {
    case 64: return launch_dh<64>(a, p, st);
    case 72: return launch_dh<72>(a, p, st);
    case 128: return launch_dh<128>(a, p, st);
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

// bf16: up to 32 rows of a document and key head, and grids that its 32-row
// workgroups do not fill (one for each CU; two of head_dim 64), go to the kernel
// of few rows (one document of 256 tokens, 16 heads of 72: 8.5 us against 10.6).
// Of few rows, and in fp32, a grid that leaves compute units idle divides the keys
// of its items into ranges, of four tiles (256 keys; fp32: 128) at least, until
// there is a workgroup for each unit (fp32, and few rows of 64: two).  More ranges
// cost more in the merge than they gain (single tokens over 4 caches 17.8 us, 22 with
// twice as many).
// 256-row workgroups divide where the least estimate says so: rounds of 256
// workgroups (of a causal or prefix mask half the work, heaviest first, behind which
// half an item ends) of 1.2 us a tile for head_dim 64, 1.5 for 72 and 128, and 10
// us + 0.6 us per MB for partial results (7151 queries and keys, 12 heads on 4 of
// 72: 280 us whole, 254 and 251 in two and three ranges; 881, 24 of 128: 30 and 37;
// 3000, 16 of 64: 50 and 70; 4000 causal, 12 of 128: 86 and 110).
DocAttnPlan doc_attn_plan(const DocAttnArgs& a, int head_dim, int dtype) {
  DocAttnPlan p{DOC_ROWS, 1};
  const long rows = (long)a.max_q * a.G;
  auto items = [&](long bm) {
    return a.Hk * std::max(1L, std::min(a.docs * ((rows + bm - 1) / bm), (long)a.q_rows * a.G / bm + a.docs));
  };
  const long fill = dtype == 1 && head_dim != 64 ? 256 : 512;
  if (dtype == 1 && (rows <= 32 || items(32) <= fill)) p.kernel = DOC_FEW;
  if (dtype != 1 || p.kernel == DOC_FEW) {
    const long n = items(p.kernel == DOC_FEW ? 32 : 16);
    if (n * 2 <= fill) p.split = (int)std::max(1L, std::min({fill / n, (long)a.max_k / (dtype == 1 ? 256 : 128), 32L}));
    return p;
  }
  const long n = items(256);
  const double T = (a.max_k + 63) / 64 * (head_dim == 64 ? 1.2 : 1.5);
  const double mb = (double)std::min((long)a.docs * a.max_q, (long)a.q_rows) * a.H * (head_dim + 4) * 4e-6;
  double best = 0;
  // (the merge pass takes a thread for four columns of a query and head, of fewer than 2^32 in a grid)
  const bool merges = (long)a.max_q * a.H * (head_dim / 4) < (1L << 32) - 256;
  for (int s = 1; s <= 8 && (s == 1 || (merges && a.max_k >= 256 * s)); ++s) {
    const double run = a.mask ? std::max(T / s, (n * T / 256 + T / s) / 2) : (double)((n * s + 255) / 256) / s * T;
    const double us = run + (s > 1 ? 10 + 0.6 * mb * s : 0);
    if (s > 1 && us >= best) continue;
    best = us;
    p.split = s;
  }
  return p;
}

}  // namespace ditmi
