// The tables of a paged cache's batch as the kernels read them (device code only).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_ops.h"

namespace axe {

__device__ __forceinline__ uint32_t quotient(uint32_t n, Divisor d) { return d.d == 1 ? n : div31(n, d.by); }

// The number of sequences that end at or before a place, found by the whole wave: ends(s), of sequence s, true up to some s and false from there on.  A step looks at 64 evenly spaced sequences.
template <class ENDS>
__device__ __forceinline__ int ended(int S, ENDS ends) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = S;                                               // the answer is in lo .. lo + n
  while (n > 0) {
    const int step = (n + 63) >> 6, i = lane * step + step - 1;
    const bool e = i < n && ends(lo + (i < n ? i : n - 1));
    const int c = __popcll(__ballot(e)) * step;
    lo += c, n = step - 1 < n - c ? step - 1 : n - c;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}
// What seq_rows says, as it is taken: from 0 to T.
__device__ __forceinline__ int border(const CacheArgs& a, int row) { return row < 0 ? 0 : row < a.T ? row : (int)a.T; }
// The sequence that row t belongs to; -1: it is behind them all.
__device__ __forceinline__ int sequence_of(const int32_t* seq_rows, int S, int64_t t) {
  const int s = ended(S, [&](int i) __attribute__((always_inline)) { return seq_rows[i + 1] <= t; });
  return s < S ? s : -1;
}

}  // namespace axe
