// Pieces shared by the kernels around the experts' products (device code only): elements of a row as fp32, sums over a wave,
// the quantisation of 128 columns.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "layer_ops.h"

namespace axe {

template <int TYPE>
struct ElemOf;
template <>
struct ElemOf<kBf16> { using T = __bf16; };
template <>
struct ElemOf<kF16> { using T = _Float16; };
template <>
struct ElemOf<kF32> { using T = float; };
template <>
struct ElemOf<kFp8> { using T = uint8_t; };

__device__ __forceinline__ float load_elem(const void* p, int64_t i, int type) {
  return type == kBf16 ? (float)((const __bf16*)p)[i] : type == kF16 ? (float)((const _Float16*)p)[i] : ((const float*)p)[i];
}
__device__ __forceinline__ void store_elem(void* p, int64_t i, int type, float v) {
  if (type == kBf16) ((__bf16*)p)[i] = (__bf16)v;
  else if (type == kF16) ((_Float16*)p)[i] = (_Float16)v;
  else ((float*)p)[i] = v;
}

// The sum over a wave, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
// The sum over a workgroup of WAVES waves, in every thread; lds: WAVES floats, free again after the caller's next barrier.
template <int WAVES>
__device__ __forceinline__ float group_sum(float v, float* lds) {
  v = wave_sum(v);
  if (WAVES == 1) return v;
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) t += lds[i];
  __syncthreads();
  return t;
}

// The scale of 128 columns whose largest magnitude is `most` (NaNs left out): s, and 1 / s, which the columns are multiplied by.  fp32: most / 448, not below
// 2^-126, where the reciprocal is still finite.  E8M0: the smallest power of two with most <= 448 2^n: most = 1.f 2^e, 448 = 1.75 2^8, so
// n = e - 8, one more where 1.f > 1.75; from the bits, hence exact.
struct Scale {
  float s, inv;
  int code;                                                        // E8M0
};
__device__ __forceinline__ Scale scale_of(float most, bool e8m0) {
  const float big = fminf(most, 3.4028234663852886e38f);
  Scale r;
  if (e8m0) {
    const uint32_t bits = __float_as_uint(big);
    int code = (int)(bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000);
    code = code < 1 ? 1 : code;
    if (big == 0) code = 127;
    r.code = code;
    r.s = __uint_as_float((uint32_t)code << 23);
    r.inv = __uint_as_float((uint32_t)(254 - code) << 23);         // (code <= 247: 448 is 2^8 and more)
  } else {
    r.code = 0;
    r.s = big == 0 ? 1.0f : fmaxf(big / 448.0f, 1.1754943508222875e-38f);
    r.inv = 1.0f / r.s;
  }
  return r;
}
// To e4m3, round to nearest even; what is beyond 448 becomes 448, NaN stays.
__device__ __forceinline__ float clamp_e4m3(float v) { return fabsf(v) > 448.0f ? copysignf(448.0f, v) : v; }
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(a), clamp_e4m3(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(c), clamp_e4m3(d), w, true);
}

}  // namespace axe
