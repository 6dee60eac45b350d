// The tables of a paged cache's batch as the kernels read them (device code only).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_ops.h"

namespace axe {

__device__ __forceinline__ uint32_t quotient(uint32_t n, Divisor d) { return d.d == 1 ? n : div31(n, d.by); }

// The sequence that row t belongs to, found by the whole wave: the number of sequences that end at or before t; -1 if there is none behind them.  A step looks at 64 evenly spaced ends.
__device__ __forceinline__ int sequence_of(const int32_t* seq_rows, int S, int64_t t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = S;                                               // the answer is in lo .. lo + n
  while (n > 0) {
    const int step = (n + 63) >> 6, i = lane * step + step - 1;
    const bool ends = i < n && seq_rows[lo + (i < n ? i : n - 1) + 1] <= t;
    const int c = __popcll(__ballot(ends)) * step;
    lo += c, n = step - 1 < n - c ? step - 1 : n - c;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  return lo < S ? lo : -1;
}

}  // namespace axe
