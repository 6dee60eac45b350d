// Root-mean-square norm of a residual stream, and its gradient (axe_rmsnorm, axe_rmsnorm_backward).  gfx950 only.
#include <hip/hip_runtime.h>

#include "layer_ops.h"
#include "row_ops.h"

namespace axe {

// One workgroup per row, in two passes over it.
__global__ __launch_bounds__(256) void rmsnorm_kernel(NormArgs a) {
  __shared__ float lds[4];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  auto h = [&](int c) { return load_elem(a.x, t * a.ldx + c, a.x_type) + (a.r ? load_elem(a.r, t * a.ldr + c, a.x_type) : 0.0f); };
  float sq = 0;
  for (int c = tid; c < a.H; c += 256) {
    const float v = h(c);
    sq += v * v;
  }
  const float rho = 1.0f / sqrtf(group_sum<4>(sq, lds) / (float)a.H + a.eps);
  auto y = [&](int c, float v) { return v * rho * (a.w ? load_elem(a.w, c, a.w_type) : 1.0f); };
  if (a.y_type != kFp8) {
    for (int c = tid; c < a.H; c += 256) {
      const float v = h(c);
      if (a.sum) store_elem(a.sum, t * a.lds + c, a.x_type, v);
      store_elem(a.y, t * a.ldy + c, a.y_type, y(c, v));
    }
    return;
  }
  const int blocks = (a.H + 127) / 128, lane = tid & 63;
  for (int b = tid >> 6; b < blocks; b += 4) {                     // a wave per 128 columns
    const int c0 = b * 128 + lane, c1 = c0 + 64;
    const float h0 = c0 < a.H ? h(c0) : 0.0f, h1 = c1 < a.H ? h(c1) : 0.0f;
    const float y0 = c0 < a.H ? y(c0, h0) : 0.0f, y1 = c1 < a.H ? y(c1, h1) : 0.0f;
    float most = fmaxf(fabsf(y0), fabsf(y1));
    for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    const Scale s = scale_of(fmaxf(most, 0.0f), a.e8m0);
    const uint32_t q = pack_e4m3(y0 * s.inv, y1 * s.inv, 0, 0);
    if (c0 < a.H) ((uint8_t*)a.y)[t * a.ldy + c0] = (uint8_t)q;
    if (c1 < a.H) ((uint8_t*)a.y)[t * a.ldy + c1] = (uint8_t)(q >> 8);
    if (a.sum && c0 < a.H) store_elem(a.sum, t * a.lds + c0, a.x_type, h0);
    if (a.sum && c1 < a.H) store_elem(a.sum, t * a.lds + c1, a.x_type, h1);
    if (lane == 0) {
      if (a.e8m0) ((uint8_t*)a.scales)[t * blocks + b] = (uint8_t)s.code;
      else ((float*)a.scales)[t * blocks + b] = s.s;
    }
  }
}

// Gradient of the rows; rho of every row to the workspace.
__global__ __launch_bounds__(256) void rmsnorm_backward_kernel(NormArgs a) {
  __shared__ float lds[4];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  auto u = [&](int c) { return load_elem(a.x, t * a.ldx + c, a.y_type) * (a.w ? load_elem(a.w, c, a.w_type) : 1.0f); };
  float sq = 0, uh = 0;
  for (int c = tid; c < a.H; c += 256) {
    const float v = load_elem(a.h, t * a.lds + c, a.x_type);
    sq += v * v, uh += v * u(c);
  }
  const float rho = 1.0f / sqrtf(group_sum<4>(sq, lds) / (float)a.H + a.eps);
  const float along = group_sum<4>(uh, lds) / (float)a.H * rho * rho;
  for (int c = tid; c < a.H; c += 256) {
    float v = rho * (u(c) - load_elem(a.h, t * a.lds + c, a.x_type) * along);
    if (a.r) v += load_elem(a.r, t * a.ldr + c, a.x_type);
    store_elem(a.y, t * a.ldy + c, a.x_type, v);
  }
}
// dw, a column a thread.
__global__ __launch_bounds__(256) void rmsnorm_dweight_kernel(NormArgs a) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  __shared__ float lds[4];
  float dw = 0;
  for (int64_t t = 0; t < a.T; ++t) {
    float sq = 0;
    for (int i = threadIdx.x; i < a.H; i += 256) {
      const float v = load_elem(a.h, t * a.lds + i, a.x_type);
      sq += v * v;
    }
    const float rho = 1.0f / sqrtf(group_sum<4>(sq, lds) / (float)a.H + a.eps);
    if (c < a.H) dw += load_elem(a.x, t * a.ldx + c, a.y_type) * load_elem(a.h, t * a.lds + c, a.x_type) * rho;
  }
  if (c < a.H) a.dw[c] = dw;
}

int64_t rmsnorm_workspace_words(int64_t, int64_t) { return 0; }

hipError_t launch_rmsnorm(const NormArgs& a, hipStream_t s) {
  rmsnorm_kernel<<<(uint32_t)a.T, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_rmsnorm_backward(const NormArgs& a, hipStream_t s) {
  // (dx may be dy: the weights' gradient first)
  if (a.dw) rmsnorm_dweight_kernel<<<(a.H + 255) / 256, 256, 0, s>>>(a);
  if (a.T) rmsnorm_backward_kernel<<<(uint32_t)a.T, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace axe
