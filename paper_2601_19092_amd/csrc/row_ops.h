// Pieces shared by the kernels around the experts' products (device code only): elements of a row as fp32, sums over a wave,
// the quantisation of 128 columns.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "layer_ops.h"

namespace axe {

// Eight neighbouring elements of a row, as bits: 16 bytes in 16-bit types, 32 in fp32, 8 in e4m3.  The kernels give every thread such runs.  They may start at any
// element: the hardware takes 16-byte accesses at any address, so rows of odd pitches need no path of their own, they only touch more lines.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <class V>
struct AnywhereOf {
  typedef V T __attribute__((aligned(1)));
};
// NT: data that this kernel touches once and leaves to the last-level cache's other tenants (see where it is asked for).
template <class V, bool NT = false>
__device__ __forceinline__ V load_bits(const void* p) {
  using A = typename AnywhereOf<V>::T;
  return NT ? __builtin_nontemporal_load((const A*)p) : *(const A*)p;
}
template <bool NT = false, class V>
__device__ __forceinline__ void store_bits(void* p, V v) {
  using A = typename AnywhereOf<V>::T;
  if (NT) __builtin_nontemporal_store(v, (A*)p);
  else *(A*)p = v;
}

template <int TYPE>
struct Run8;
template <>
struct Run8<kBf16> {
  using Elem = uint16_t;
  u32x4 b;
  __device__ __forceinline__ void clear() { b = u32x4{}; }
  __device__ __forceinline__ void keep(bool on) { b = on ? b : u32x4{}; }
  template <bool NT>
  __device__ __forceinline__ void load(const void* p) { b = load_bits<u32x4, NT>(p); }
  template <bool NT>
  __device__ __forceinline__ void store(void* p) const { store_bits<NT>(p, b); }
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? b[i >> 1] & 0xffff0000u : b[i >> 1] << 16); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
      b[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]});    // round to nearest even
    }
  }
  // the run moved down by n elements, zeros behind (0 <= n <= 8)
  __device__ __forceinline__ void down(int n) {
    const uint32_t h = (n & 1) * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = (uint32_t)(((uint64_t)(i < 3 ? b[i + 1] : 0) << 32 | b[i]) >> h);
    b = n & 2 ? u32x4{b[1], b[2], b[3], 0} : b;
    b = n & 4 ? u32x4{b[2], b[3], 0, 0} : b;
    b = n & 8 ? u32x4{} : b;
  }
  __device__ __forceinline__ void load_part(const Elem* p, int n) {
    clear();
    if (n & 4) {
      const u32x2 v = load_bits<u32x2>(p);
      b[0] = v[0], b[1] = v[1];
    }
    if (n & 2) b[n & 4 ? 2 : 0] = load_bits<uint32_t>(p + (n & 4));
    if (n & 1) b[n >> 1] = p[n & 6];
  }
  __device__ __forceinline__ void store_part(Elem* p, int n) const {
    Run8 r = *this;
    if (n & 4) store_bits(p, u32x2{r.b[0], r.b[1]}), p += 4, r.down(4);
    if (n & 2) store_bits(p, r.b[0]), p += 2, r.down(2);
    if (n & 1) *p = (Elem)r.b[0];
  }
};
template <>
struct Run8<kF16> {
  using Elem = uint16_t;
  u32x4 b;
  __device__ __forceinline__ void clear() { b = u32x4{}; }
  __device__ __forceinline__ void keep(bool on) { b = on ? b : u32x4{}; }
  template <bool NT>
  __device__ __forceinline__ void load(const void* p) { b = load_bits<u32x4, NT>(p); }
  template <bool NT>
  __device__ __forceinline__ void store(void* p) const { store_bits<NT>(p, b); }
  __device__ __forceinline__ float get(int i) const { return (float)__builtin_bit_cast(_Float16, (uint16_t)(b[i >> 1] >> (i & 1) * 16)); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
      b[i] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)v[2 * i], (_Float16)v[2 * i + 1]});
    }
  }
  // the run moved down by n elements, zeros behind (0 <= n <= 8)
  __device__ __forceinline__ void down(int n) {
    const uint32_t h = (n & 1) * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = (uint32_t)(((uint64_t)(i < 3 ? b[i + 1] : 0) << 32 | b[i]) >> h);
    b = n & 2 ? u32x4{b[1], b[2], b[3], 0} : b;
    b = n & 4 ? u32x4{b[2], b[3], 0, 0} : b;
    b = n & 8 ? u32x4{} : b;
  }
  __device__ __forceinline__ void load_part(const Elem* p, int n) {
    clear();
    if (n & 4) {
      const u32x2 v = load_bits<u32x2>(p);
      b[0] = v[0], b[1] = v[1];
    }
    if (n & 2) b[n & 4 ? 2 : 0] = load_bits<uint32_t>(p + (n & 4));
    if (n & 1) b[n >> 1] = p[n & 6];
  }
  __device__ __forceinline__ void store_part(Elem* p, int n) const {
    Run8 r = *this;
    if (n & 4) store_bits(p, u32x2{r.b[0], r.b[1]}), p += 4, r.down(4);
    if (n & 2) store_bits(p, r.b[0]), p += 2, r.down(2);
    if (n & 1) *p = (Elem)r.b[0];
  }
};
template <>
struct Run8<kF32> {
  using Elem = uint32_t;
  u32x4 b[2];
  __device__ __forceinline__ void clear() { b[0] = b[1] = u32x4{}; }
  __device__ __forceinline__ void keep(bool on) { b[0] = on ? b[0] : u32x4{}, b[1] = on ? b[1] : u32x4{}; }
  template <bool NT>
  __device__ __forceinline__ void load(const void* p) { b[0] = load_bits<u32x4, NT>(p), b[1] = load_bits<u32x4, NT>((const char*)p + 16); }
  template <bool NT>
  __device__ __forceinline__ void store(void* p) const { store_bits<NT>(p, b[0]), store_bits<NT>((char*)p + 16, b[1]); }
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(b[i >> 2][i & 3]); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i >> 2][i & 3] = __float_as_uint(v[i]);
  }
  __device__ __forceinline__ void down(int n) {
#pragma unroll
    for (int d = 1; d < 8; d *= 2)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t up = i + d < 8 ? b[(i + d) >> 2][(i + d) & 3] : 0;
        b[i >> 2][i & 3] = n & d ? up : b[i >> 2][i & 3];
      }
    if (n & 8) clear();
  }
  __device__ __forceinline__ void load_part(const Elem* p, int n) {
    clear();
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) b[i >> 2][i & 3] = p[i];
  }
  __device__ __forceinline__ void store_part(Elem* p, int n) const {
    Run8 r = *this;
    if (n & 4) store_bits(p, r.b[0]), p += 4, r.down(4);
    if (n & 2) store_bits(p, u32x2{r.b[0][0], r.b[0][1]}), p += 2, r.down(2);
    if (n & 1) *p = r.b[0][0];
  }
};
template <>
struct Run8<kFp8> {
  using Elem = uint8_t;
  u32x2 b;
  __device__ __forceinline__ void clear() { b = u32x2{}; }
  template <bool NT>
  __device__ __forceinline__ void load(const void* p) { b = load_bits<u32x2, NT>(p); }
  template <bool NT>
  __device__ __forceinline__ void store(void* p) const { store_bits<NT>(p, b); }
  __device__ __forceinline__ void set(const float (&v)[8]);
  __device__ __forceinline__ void down(int n) {
    const uint64_t v = n < 8 ? ((uint64_t)b[1] << 32 | b[0]) >> n * 8 : 0;
    b = u32x2{(uint32_t)v, (uint32_t)(v >> 32)};
  }
  __device__ __forceinline__ void load_part(const Elem* p, int n) {
    uint64_t v = 0;
    for (int i = 0; i < n; ++i) v |= (uint64_t)p[i] << i * 8;
    b = u32x2{(uint32_t)v, (uint32_t)(v >> 32)};
  }
  __device__ __forceinline__ void store_part(Elem* p, int n) const {
    Run8 r = *this;
    if (n & 4) store_bits(p, r.b[0]), p += 4, r.down(4);
    if (n & 2) store_bits(p, (uint16_t)r.b[0]), p += 2, r.down(2);
    if (n & 1) *p = (Elem)r.b[0];
  }
};

// The run at element i of a row of H elements, in two steps; what lies past the row's end comes out as zero.  A run that would reach past the end (or lies behind
// it) is read as the row's last eight elements and moved down in the second step: the loads of all threads are then single instructions with no branch
// around them, and all of a thread's can be in flight.  Rows of fewer than eight elements (SHORT) are put together from what they have.
template <bool SHORT, bool NT = false, int TYPE>
__device__ __forceinline__ void load_run(Run8<TYPE>& r, const void* row, int i, int H) {
  using E = typename Run8<TYPE>::Elem;
  if (SHORT) r.load_part((const E*)row, i == 0 ? H : 0);
  else r.template load<NT>((const E*)row + (i + 8 <= H ? i : H - 8));
}
template <bool SHORT, int TYPE>
__device__ __forceinline__ void end_run(Run8<TYPE>& r, int i, int H) {
  if (!SHORT && i + 8 > H) r.down(i < H ? i + 8 - H : 8);
}
template <bool NT = false, int TYPE>
__device__ __forceinline__ void store_run(const Run8<TYPE>& r, void* row, int i, int H) {
  using E = typename Run8<TYPE>::Elem;
  if (i + 8 <= H) r.template store<NT>((E*)row + i);
  else if (i < H) r.store_part((E*)row + i, H - i);
}
template <class E>
__host__ __device__ __forceinline__ E* elem_at(E* p, int64_t i, int bytes) { return (E*)((std::conditional_t<std::is_const<E>::value, const char, char>*)p + i * bytes); }

// RUNS runs of weights, TPR * 8 columns apart, of a type known at run time; null: ones (past the end: anything, it meets zeros).
template <bool SHORT, int TPR, int RUNS, int TYPE>
__device__ __forceinline__ void weights_of(float (&w)[RUNS][8], const void* p, int c, int H) {
  Run8<TYPE> r[RUNS];
#pragma unroll
  for (int i = 0; i < RUNS; ++i) load_run<SHORT>(r[i], p, c + i * TPR * 8, H);
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    end_run<SHORT>(r[i], c + i * TPR * 8, H);
#pragma unroll
    for (int k = 0; k < 8; ++k) w[i][k] = r[i].get(k);
  }
}
template <bool SHORT, int TPR, int RUNS>
__device__ __forceinline__ void load_weights(float (&w)[RUNS][8], const void* p, int type, int c, int H) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < RUNS; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) w[i][k] = 1.0f;
  } else if (type == kF32) weights_of<SHORT, TPR, RUNS, kF32>(w, p, c, H);
  else if (type == kBf16) weights_of<SHORT, TPR, RUNS, kBf16>(w, p, c, H);
  else weights_of<SHORT, TPR, RUNS, kF16>(w, p, c, H);
}

// The arguments of a kernel lie in lines of 64 bytes that no cache holds yet, and the compiler fetches a field where it is used first: a kernel that comes to a line late waits
// for memory once more.  One field of every line, named at the start, brings them all in together.
template <class T>
__device__ __forceinline__ void fetch_arguments(T of_a_line) { asm volatile("" ::"s"(of_a_line)); }
template <class T, class... U>
__device__ __forceinline__ void fetch_arguments(T first, U... others) {
  fetch_arguments(first);
  fetch_arguments(others...);
}

// A barrier of the workgroup that publishes what is in LDS, and nothing else: __syncthreads() also waits until the loads and stores of global memory under way are done, a
// microsecond that no one here needs.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Exchanges inside a row of 16 lanes are operands of the instruction that uses them (DPP); between rows gfx950 swaps whole rows.
template <int CTRL>
__device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_mov_dpp(v, CTRL, 0xf, 0xf, true); }
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
struct Add {
  __device__ __forceinline__ static float of(float a, float b) { return a + b; }
};
struct Max {
  __device__ __forceinline__ static float of(float a, float b) { return fmaxf(a, b); }
};
// v of all 16 lanes of a row, or of 32, or of all 64, joined, in every lane.  (Each step joins lanes that hold the same number of values: the
// two sides of a step are the same in both lanes, so the results are the same bits.)
template <class OP>
__device__ __forceinline__ float row8_all(float v) {               // eight lanes
  v = OP::of(v, __int_as_float(dpp<kXor1>(__float_as_int(v))));
  v = OP::of(v, __int_as_float(dpp<kXor2>(__float_as_int(v))));
  return OP::of(v, __int_as_float(dpp<kHalfMirror>(__float_as_int(v))));
}
template <class OP>
__device__ __forceinline__ float row16_all(float v) {
  v = row8_all<OP>(v);
  return OP::of(v, __int_as_float(dpp<kMirror>(__float_as_int(v))));
}
template <class OP>
__device__ __forceinline__ float half_all(float v) {               // 32 lanes
  v = row16_all<OP>(v);
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
  return OP::of(__int_as_float(a[0]), __int_as_float(a[1]));
}
template <class OP>
__device__ __forceinline__ float wave_all(float v) {
  v = half_all<OP>(v);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return OP::of(__int_as_float(b[0]), __int_as_float(b[1]));
}
__device__ __forceinline__ float wave_sum(float v) { return wave_all<Add>(v); }
// The sums of N values over the threads of a row that WAVES waves hold, in every thread; wave: which of them this is.  lds: N x WAVES floats of the row, which
// the caller does not reuse before another barrier.
template <int N, int WAVES>
__device__ __forceinline__ void row_sums(float (&v)[N], float* lds, int wave) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  if (WAVES == 1) return;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) lds[i * WAVES + wave] = v[i];
  lds_barrier();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float t = 0;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) t += lds[i * WAVES + k];
    v[i] = t;
  }
}

// The scale s of 128 columns whose largest magnitude is `most` (NaNs left out).  fp32: most / 448, not below 2^-126.  E8M0: the smallest power of two with
// most <= 448 2^n: most = 1.f 2^e, 448 = 1.75 2^8, so n = e - 8, one more where 1.f > 1.75; from the bits, hence exact.
struct Scale {
  float s;
  float inv, rest;                                                 // 1 / s and what that rounding left out
  float top;                                                       // what is larger is an infinity, or becomes 448
  bool divide;
  int code;                                                        // E8M0
};
__device__ __forceinline__ Scale scale_of(float most, bool e8m0) {
  const float largest = 3.4028234663852886e38f, big = fminf(most, largest);
  Scale r;
  if (e8m0) {
    const uint32_t bits = __float_as_uint(big);
    int code = (int)(bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000);
    code = code < 1 ? 1 : code;
    if (big == 0) code = 127;
    r.code = code;
    r.s = __uint_as_float((uint32_t)code << 23);
    r.inv = __uint_as_float((uint32_t)(254 - code) << 23), r.rest = 0;   // (code <= 247: 448 is 2^8 and more)
    r.divide = false;
  } else {
    r.code = 0;
    r.s = big == 0 ? 1.0f : fmaxf(big / 448.0f, 1.1754943508222875e-38f);
    r.inv = 1.0f / r.s;
    r.rest = fmaf(-r.inv, r.s, 1.0f) * r.inv;
    const uint32_t low = __float_as_uint(r.s) & 0xfffff;
    r.divide = (low != 0 && ((low + 16) & 0xfffff) <= 32) || r.s > 0x1p100f;
  }
  r.top = fminf(440.0f * r.s, largest);
  return r;
}
// What of y becomes e4m3: the codes of y / s in fp32, correctly rounded, though most of it is a product with 1 / s = inv + rest.  (With inv alone one code in 2000 of bf16 rows comes out as its
// neighbour: y and the largest of the 128, 448 s, have few bits there, so that y / s is a midpoint m of two codes often.)  The sum is fl(y / s (1 + d)), |d| < 2^-46.  That has another code than
// fl(y / s) only where a number h half way between two neighbours in fp32, one of them an m, is nearer to y / s than 2^-46.  h = (mu 2^20 +- 1) 2^b, mu whole, so with s = S 2^c, S of 24
// bits, and y = Y 2^f: |Y 2^a - S (mu 2^20 +- 1)| <= 8, a at least 23; hence S is within 8 of a multiple of 2^20, and not one itself (then the difference is one of 2^20, and not 0 as Y has
// no bit for it).  Such scales, and those above 2^100, whose rest is subnormal, divide (`divide`).
// us, times inv alone / this / divisions throughout: 32768 rows of 768 15.2 / 16.3 / 24, 1024 tokens to 8 rows of 2048 5.9 / 6.0 / 6.6, norm of 4096 x 2048 fp32 9.2 / 9.8 / 10.9.
template <int N>
__device__ __forceinline__ void over_scale(float (&y)[N], const Scale& s) {
  float q[N];
#pragma unroll
  for (int k = 0; k < N; ++k) q[k] = fmaf(y[k], s.inv, y[k] * s.rest);
  if (__builtin_expect(s.divide, 0)) {
#pragma unroll
    for (int k = 0; k < N; ++k) q[k] = y[k] / s.s;
  }
#pragma unroll
  for (int k = 0; k < N; ++k) y[k] = fabsf(y[k]) > s.top ? copysignf(448.0f, y[k]) : q[k];   // (432 and more round to 448; NaN stays)
}
// To e4m3, round to nearest even, of numbers of at most 448.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

__device__ __forceinline__ void Run8<kFp8>::set(const float (&v)[8]) { b = u32x2{pack_e4m3(v[0], v[1], v[2], v[3]), pack_e4m3(v[4], v[5], v[6], v[7])}; }
__device__ __forceinline__ void store_scale(void* scales, int64_t i, const Scale& s, bool e8m0) {
  if (e8m0) ((uint8_t*)scales)[i] = (uint8_t)s.code;
  else ((float*)scales)[i] = s.s;
}

}  // namespace axe
