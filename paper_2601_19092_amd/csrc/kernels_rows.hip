// The tokens' rows in the experts' order and back (axe_rows_dispatch, axe_rows_combine, axe_rows_combine_backward).  gfx950 only.
#include <hip/hip_runtime.h>

#include "layer_ops.h"
#include "row_ops.h"

namespace axe {

// The row of a token's j-th choice, or -1.
__device__ __forceinline__ int64_t row_at(const RowsArgs& a, int64_t t, int j) {
  if (!a.row_of) return t;
  const int64_t r = a.row_of[t * a.k + j];
  return r >= 0 && r < a.M ? r : -1;
}

// One workgroup per token.
__global__ __launch_bounds__(256) void rows_dispatch_kernel(RowsArgs a) {
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, blocks = (a.H + 127) / 128;
  if (a.t_type == a.r_type) {
    const int eb = elem_bytes(a.t_type);
    for (int j = 0; j < a.k; ++j) {
      const int64_t r = row_at(a, t, j);
      if (r < 0) continue;
      for (int64_t c = tid; c < a.H; c += 256) {
        if (eb == 1) ((uint8_t*)a.to_rows)[r * a.ldr + c] = ((const uint8_t*)a.tokens)[t * a.ldt + c];
        else if (eb == 2) ((uint16_t*)a.to_rows)[r * a.ldr + c] = ((const uint16_t*)a.tokens)[t * a.ldt + c];
        else ((uint32_t*)a.to_rows)[r * a.ldr + c] = ((const uint32_t*)a.tokens)[t * a.ldt + c];
      }
      if (eb == 1)
        for (int b = tid; b < blocks; b += 256) {
          if (a.e8m0) ((uint8_t*)a.scales)[r * blocks + b] = ((const uint8_t*)a.token_scales)[t * blocks + b];
          else ((uint32_t*)a.scales)[r * blocks + b] = ((const uint32_t*)a.token_scales)[t * blocks + b];
        }
    }
    return;
  }
  for (int b = tid >> 6; b < blocks; b += 4) {                     // a wave per 128 columns
    const int64_t c0 = b * 128 + lane, c1 = c0 + 64;
    const float y0 = c0 < a.H ? load_elem(a.tokens, t * a.ldt + c0, a.t_type) : 0.0f, y1 = c1 < a.H ? load_elem(a.tokens, t * a.ldt + c1, a.t_type) : 0.0f;
    float most = fmaxf(fabsf(y0), fabsf(y1));
    for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    const Scale s = scale_of(fmaxf(most, 0.0f), a.e8m0);
    const uint32_t q = pack_e4m3(y0 * s.inv, y1 * s.inv, 0, 0);
    for (int j = 0; j < a.k; ++j) {
      const int64_t r = row_at(a, t, j);
      if (r < 0) continue;
      if (c0 < a.H) ((uint8_t*)a.to_rows)[r * a.ldr + c0] = (uint8_t)q;
      if (c1 < a.H) ((uint8_t*)a.to_rows)[r * a.ldr + c1] = (uint8_t)(q >> 8);
      if (lane) continue;
      if (a.e8m0) ((uint8_t*)a.scales)[r * blocks + b] = (uint8_t)s.code;
      else ((float*)a.scales)[r * blocks + b] = s.s;
    }
  }
}

__global__ __launch_bounds__(256) void rows_combine_kernel(RowsArgs a) {
  const int64_t t = blockIdx.x;
  for (int64_t c = threadIdx.x; c < a.H; c += 256) {
    float v = a.add ? load_elem(a.add, t * a.ldt + c, a.t_type) : 0.0f;
    for (int j = 0; j < a.k; ++j) {
      const int64_t r = row_at(a, t, j);
      if (r >= 0) v += (a.weights ? a.weights[t * a.k + j] : 1.0f) * load_elem(a.rows, r * a.ldr + c, a.r_type);
    }
    store_elem(a.to_tokens, t * a.ldt + c, a.t_type, v);
  }
}

// One workgroup per pair.
__global__ __launch_bounds__(256) void rows_combine_backward_kernel(RowsArgs a) {
  __shared__ float lds[4];
  const int64_t pair = blockIdx.x, t = pair / a.k;
  const int64_t r = row_at(a, t, (int)(pair - t * a.k));
  float dot = 0;
  if (r >= 0) {
    const float w = a.weights ? a.weights[pair] : 1.0f;
    for (int64_t c = threadIdx.x; c < a.H; c += 256) {
      const float d = load_elem(a.tokens, t * a.ldt + c, a.t_type);
      if (a.rows) dot += d * load_elem(a.rows, r * a.ldr + c, a.r_type);
      if (a.to_rows) store_elem(a.to_rows, r * a.ldr + c, a.r_type, w * d);
    }
  }
  dot = group_sum<4>(dot, lds);
  if (a.dweights && threadIdx.x == 0) a.dweights[pair] = dot;
}

hipError_t launch_rows_dispatch(const RowsArgs& a, hipStream_t s) {
  rows_dispatch_kernel<<<(uint32_t)a.T, 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_rows_combine(const RowsArgs& a, hipStream_t s) {
  rows_combine_kernel<<<(uint32_t)a.T, 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_rows_combine_backward(const RowsArgs& a, hipStream_t s) {
  rows_combine_backward_kernel<<<(uint32_t)(a.T * a.k), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace axe
