// What the entry points share in planning a call: the pitched matrices among layouts, kept plans, error helpers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include "../../include/axe.h"

namespace axe {

// The error of a HIP call that failed (AXE_EHIP; the message names it).
int hip_fail(hipError_t e, const char* what);

// A matrix of shape (d0, d1) whose layout is a pitched one with unit stride along the inner dimension, inside `elems` elements:
// pitch and offset; else an error.
int strided_2d(const axe_layout_t* L, int mem_axis, int64_t d0, int64_t d1, bool inner_is_dim1, int64_t elems, const char* what,
               int64_t* pitch, int64_t* offset);

// The contents of a descriptor as a flat run of words: what a plan depends on, device pointers aside (of those
// only whether they are given and their alignment matter).  False when the descriptor is malformed in a way
// that makes its arrays unreadable: the planner then reports the error.
constexpr int kKeyWords = 24 + 6 * (12 + 3 * (AXE_MAX_D + AXE_MAX_R) + AXE_MAX_AXES);   // (six layouts at most)
struct PlanKey {
  int64_t w[kKeyWords];
  int n = 0;
  void put(int64_t v) { w[n++] = v; }
};
inline bool key_of_layout(const axe_layout_t& L, PlanKey& k) {
  if (L.n_axes < 1 || L.n_axes > AXE_MAX_AXES || L.n_d < 1 || L.n_d > AXE_MAX_D || L.n_r < 0 || L.n_r > AXE_MAX_R || !L.d ||
      (L.n_r && !L.r))
    return false;
  k.put(L.n_axes), k.put(L.n_d), k.put(L.n_r);
  for (int i = 0; i < L.n_d; ++i) k.put(L.d[i].extent), k.put(L.d[i].stride), k.put(L.d[i].axis);
  for (int i = 0; i < L.n_r; ++i) k.put(L.r[i].extent), k.put(L.r[i].stride), k.put(L.r[i].axis);
  for (int a = 0; a < L.n_axes; ++a) k.put(L.offset ? L.offset[a] : 0);
  k.put(L.swz_axis), k.put(L.swz_bits), k.put(L.swz_base), k.put(L.swz_shift);
  return true;
}

// The plan of the last call of one kind that this thread made: a caller that moves or evaluates the same layouts again
// (compared word by word; other buffers of the same alignment are fine) skips the layout analysis, 1 - 1.5 us of a
// call whose launch takes 2.5.
template <class Plan>
struct LastPlan {
  PlanKey key;
  Plan plan;
  bool have = false;
  bool holds(const PlanKey& k) const { return have && k.n == key.n && memcmp(k.w, key.w, sizeof(int64_t) * k.n) == 0; }
  void keep(const PlanKey& k, const Plan& p) { key = k, plan = p, have = true; }
};

}  // namespace axe
