// Device-side view of one document of the masked attention.
#pragma once
#include "common.h"
#include "kernels.h"

namespace ditmi {

constexpr float LOG2E = 1.4426950408889634f;

// One document as a workgroup sees it, every bound clamped into the tensors.
struct Doc {
  int q0, nq, k0, nk, prefix;
};
// The arrays' entries are requested at once (an absent array's from q, and not
// used): one after the other they would cost a memory round trip each.
__device__ __forceinline__ Doc load_doc(const DocAttnArgs& a, int d) {
  const int32_t* none = (const int32_t*)a.q;
  const int32_t *qs = a.q_start ? a.q_start + d : none, *ks = a.k_start ? a.k_start + d : none;
  const int32_t *kl = a.k_len ? a.k_len + d : none, *px = a.prefix ? a.prefix + d : none;
  const int q_lo = qs[0], q_hi = qs[1], k_lo = ks[0], k_hi = ks[1], len = kl[0], pre = px[0];
  Doc o;
  o.q0 = a.q_start ? min(max(q_lo, 0), a.q_rows) : (int)min((long)d * a.room_q, (long)a.q_rows);
  o.nq = min((a.q_start ? min(max(q_hi, o.q0), a.q_rows) : a.q_rows) - o.q0, a.max_q);
  o.k0 = a.k_start ? min(max(k_lo, 0), a.k_rows) : (int)min((long)d * a.room_k, (long)a.k_rows);
  o.nk = min((a.k_start ? min(max(k_hi, o.k0), a.k_rows) : a.k_rows) - o.k0, a.max_k);
  if (a.k_len) o.nk = min(o.nk, max(len, 0));
  o.prefix = a.prefix ? min(max(pre, 0), o.nk) : 0;
  return o;
}
// Keys visible to query i: j < row_limit.  It never falls as i grows.
__device__ __forceinline__ int row_limit(const DocAttnArgs& a, const Doc& d, int i) {
  if (a.mask == 0) return d.nk;
  return max(min(max(i + d.nk - d.nq + 1, 0), d.nk), d.prefix);
}

// First keys of V values that are not finite, per class and column.
constexpr int NO_KEY = 0x7FFFFFFF;
template <int DH>
__device__ __forceinline__ void note_bad(int (&bad)[3][DH], int cls, int d, int key) {
  __hip_atomic_fetch_min(&bad[cls][d], key, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
// n values of one V row at column d: those that are not finite become 0.
template <int DH>
__device__ __noinline__ void keep_bad(int (&bad)[3][DH], bf16_t* p, int n, int d, int key) {
  for (int x = 0; x < n; ++x) {
    const uint32_t u = p[x];
    if ((u & 0x7F80u) != 0x7F80u) continue;
    p[x] = 0;
    note_bad(bad, u & 0x7Fu ? 0 : 1 + (u >> 15), d + x, key);
  }
}
template <int DH>
__device__ __forceinline__ float add_bad(float o, const int (&bad)[3][DH], int d, int lim) {
  if (bad[0][d] < lim) o = NAN;
  if (bad[1][d] < lim) o += INFINITY;
  if (bad[2][d] < lim) o -= INFINITY;
  return o;
}

}  // namespace ditmi
