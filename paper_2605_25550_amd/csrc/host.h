// Host-side helpers shared by the C entry points (ditmi.cpp, operators.cpp).
#pragma once
#include <hip/hip_runtime.h>

#include "ditmi.h"

namespace ditmi {

// Records the calling thread's error text and returns st.
dit_status fail(dit_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// Timing hook around one launch: timed_begin returns the slot of the launch
// (-1: not recorded), timed_end records its stop event.
hipError_t timed_begin(int kclass, double flops, double bytes, hipStream_t st, int* slot);
hipError_t timed_end(int slot, hipStream_t st);

template <typename Fn>
hipError_t timed(int kclass, double flops, double bytes, hipStream_t st, Fn&& launch) {
  int slot = -1;
  hipError_t e = timed_begin(kclass, flops, bytes, st, &slot);
  if (e != hipSuccess) return e;
  e = launch();
  if (e != hipSuccess) return e;
  return slot >= 0 ? timed_end(slot, st) : hipSuccess;
}

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

}  // namespace ditmi

#define HIP_TRY(expr)                                                                     \
  do {                                                                                    \
    hipError_t e_ = (expr);                                                               \
    if (e_ != hipSuccess) return fail(DIT_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)
