// What the entry points of a layer's parts (api_layer.cpp, api_cache.cpp) share: error helpers, checks of buffers, matrices among layouts, the body that does not throw.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>
#include <new>
#include <type_traits>

#include "../../include/axe.h"
#include "host_layout.h"
#include "plans.h"

namespace axe {

inline bool real_type(int t) { return t == AXE_BF16 || t == AXE_F16 || t == AXE_F32; }

inline int invalid(const char* fn, const char* what) {
  set_error("%s: %s", fn, what);
  return AXE_EINVAL;
}
inline int unsupported(const char* fn, const char* what) {
  set_error("%s: %s", fn, what);
  return AXE_EUNSUPPORTED;
}

// A buffer of a call: where, how many bytes, what it has to be aligned to, and whether the call may not do without it.
struct Buf {
  const void* p;
  int64_t bytes;
  int align;
  bool needed;
};
inline bool meet(const Buf& a, const Buf& b) {
  return a.p && b.p && (const char*)a.p < (const char*)b.p + b.bytes && (const char*)b.p < (const char*)a.p + a.bytes;
}
inline int check_buffers(const char* fn, std::initializer_list<Buf> in, std::initializer_list<Buf> out) {
  for (const auto& list : {in, out})
    for (const Buf& b : list) {
      if (b.needed && !b.p) return invalid(fn, "NULL device pointer");
      if (b.p && (uintptr_t)b.p % (uintptr_t)b.align) return invalid(fn, "a buffer is not aligned to its elements");
    }
  for (const Buf& o : out) {
    for (const Buf& i : in)
      if (meet(i, o)) return invalid(fn, "an output overlaps an input");
    for (const Buf& p : out)
      if (&p != &o && meet(p, o)) return invalid(fn, "two outputs overlap");
  }
  return AXE_OK;
}

// One matrix of a call: its layout on the memory axis, planned once per descriptor.  Bytes of its buffer are computed of a matrix that was planned (or is not there) only: 64 bits hold them.
struct Mat {
  int64_t ld = 0, off = 0;
};
constexpr int64_t kMostElems = int64_t(1) << 58;
inline int plan_matrix(const axe_layout_t& L, int mem_axis, int64_t rows, int64_t cols, int64_t elems, const char* fn, Mat& m) {
  if (elems > kMostElems) return invalid(fn, "a buffer of more than 2^58 elements");
  return strided_2d(&L, mem_axis, rows, cols, true, elems, fn, &m.ld, &m.off);
}
inline int64_t bytes_of(const void* p, int64_t elems, int eb) { return p ? elems * eb : 0; }

// The body of an entry point; planning allocates, and an entry point neither throws nor aborts.
template <class F>
auto guarded(const char* fn, F&& f) -> decltype(f()) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    set_error("%s: out of host memory", fn);
    return AXE_EINVAL;
  }
}

inline int finish(hipError_t e, const char* fn) { return e == hipSuccess ? AXE_OK : hip_fail(e, fn); }

template <class V>
V* at(V* p, int64_t off, int eb) {
  using C = std::conditional_t<std::is_const<V>::value, const char, char>;
  return p ? (V*)((C*)p + off * eb) : nullptr;
}

}  // namespace axe
