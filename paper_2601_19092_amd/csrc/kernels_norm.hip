// Root-mean-square norm of a residual stream, and its gradient (axe_rmsnorm, axe_rmsnorm_backward).  gfx950 only.
//
// Both are bound by memory: a row is read once and held in registers as fp32, in runs of 8 columns a thread (thread i of the TPR threads of a row holds the runs
// i, i + TPR, ...: neighbouring lanes read neighbouring 16 bytes), its sum of squares is joined over the wave by DPP and over the waves of a row through LDS, and what is
// written comes from the registers.  A run of 128 columns that shares a scale is 16 neighbouring lanes: its maximum never leaves a DPP row.
#include <hip/hip_runtime.h>

#include "layer_ops.h"
#include "row_ops.h"

namespace axe {

// Threads of a workgroup whose rows have TPR threads each: rows of one wave go four to a workgroup.
constexpr int norm_threads(int tpr) { return tpr < 256 ? 256 : tpr; }

// XT: x, residual and sum; YT: y.  A row of up to TPR * 8 * RUNS columns.
template <int XT, int YT, int TPR, int RUNS>
__global__ __launch_bounds__(norm_threads(TPR)) void rmsnorm_kernel(NormArgs a) {
  constexpr int WAVES = TPR / 64;
  __shared__ float lds[WAVES];
  const int tid = threadIdx.x % TPR;
  const int64_t t = (int64_t)blockIdx.x * (norm_threads(TPR) / TPR) + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  if (t >= a.T) return;                                            // (whole waves of rows of one wave, or none)
  Run8<XT> x[RUNS], r[RUNS];
  float w[RUNS][8];
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    const int c = (i * TPR + tid) * 8, left = a.H - c;
    load_run(x[i], a.x, t * a.ldx + c, left);
    if (a.r) load_run(r[i], a.r, t * a.ldr + c, left);
  }
#pragma unroll
  for (int i = 0; i < RUNS; ++i) load_weights(w[i], a.w, a.w_type, (i * TPR + tid) * 8, a.H - (i * TPR + tid) * 8);
  float h[RUNS][8], sq[1] = {0};
#pragma unroll
  for (int i = 0; i < RUNS; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      h[i][k] = a.r ? x[i].get(k) + r[i].get(k) : x[i].get(k);
      sq[0] += h[i][k] * h[i][k];
    }
  if (a.sum) {
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      const int c = (i * TPR + tid) * 8;
      x[i].set(h[i]);
      store_run(x[i], a.sum, t * a.lds + c, a.H - c);
    }
  }
  row_sums<1, WAVES>(sq, lds);
  const float rho = 1.0f / sqrtf(sq[0] / (float)a.H + a.eps);
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    const int c = (i * TPR + tid) * 8, left = a.H - c;
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = h[i][k] * rho * w[i][k];
    if constexpr (YT == kFp8) {
      float most = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) most = fmaxf(most, fabsf(y[k]));  // (NaN: the other operand)
      const Scale s = scale_of(row16_all<Max>(most), a.e8m0);
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] *= s.inv;
      Run8<kFp8> q;
      q.set(y);
      store_run(q, a.y, t * a.ldy + c, left);
      if ((tid & 15) == 0 && left > 0) store_scale(a.scales, t * ((a.H + 127) >> 7) + (c >> 7), s, a.e8m0);
    } else {
      Run8<YT> q;
      q.set(y);
      store_run(q, a.y, t * a.ldy + c, left);
    }
  }
}

// Gradients.  XT: h, dsum and dx; YT: dy.  A workgroup takes every gridDim-th row (rows of one wave: four at a time) and keeps its threads' columns of dw in
// registers; what a workgroup has of dw goes to its row of the workspace, and a second kernel adds these rows up.
template <int XT, int YT, int TPR, int RUNS>
__global__ __launch_bounds__(norm_threads(TPR)) void rmsnorm_backward_kernel(NormArgs a) {
  constexpr int WAVES = TPR / 64, ROWS = norm_threads(TPR) / TPR;
  __shared__ float lds[2][2 * WAVES];
  extern __shared__ float part[];
  const int tid = threadIdx.x % TPR, sub = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  float dw[RUNS][8] = {};
  int turn = 0;
  for (int64_t t = (int64_t)blockIdx.x * ROWS + sub; t < a.T; t += (int64_t)gridDim.x * ROWS, turn ^= 1) {
    Run8<YT> dy[RUNS];
    Run8<XT> h[RUNS], ds[RUNS];
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      const int c = (i * TPR + tid) * 8, left = a.H - c;
      load_run(dy[i], a.x, t * a.ldx + c, left);
      load_run(h[i], a.h, t * a.lds + c, left);
      if (a.r) load_run(ds[i], a.r, t * a.ldr + c, left);
    }
    float s[2] = {0, 0};
    float u[RUNS][8];
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      const int c = (i * TPR + tid) * 8;
      load_weights(u[i], a.w, a.w_type, c, a.H - c);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        u[i][k] *= dy[i].get(k);
        s[0] += h[i].get(k) * h[i].get(k), s[1] += u[i][k] * h[i].get(k);
      }
    }
    row_sums<2, WAVES>(s, lds[turn]);                              // (two arrays: no thread is two rows ahead of another)
    const float rho = 1.0f / sqrtf(s[0] / (float)a.H + a.eps);
    const float along = s[1] / (float)a.H * rho * rho;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      const int c = (i * TPR + tid) * 8;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[k] = rho * (u[i][k] - h[i].get(k) * along);
        if (a.r) v[k] += ds[i].get(k);
        dw[i][k] += dy[i].get(k) * (h[i].get(k) * rho);
      }
      Run8<XT> out;
      out.set(v);
      store_run(out, a.y, t * a.ldy + c, a.H - c);
    }
  }
  if (!a.dw) return;
  if constexpr (ROWS > 1) {                                        // the workgroup's rows together: waves 1 .. to LDS, wave 0 adds them in order
    constexpr int W = TPR * RUNS * 8;
    if (sub > 0)
#pragma unroll
      for (int i = 0; i < RUNS; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) part[(sub - 1) * W + (i * 8 + k) * TPR + tid] = dw[i][k];
    __syncthreads();
    if (sub > 0) return;
    for (int o = 0; o < ROWS - 1; ++o)
#pragma unroll
      for (int i = 0; i < RUNS; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) dw[i][k] += part[o * W + (i * 8 + k) * TPR + tid];
  }
  float* to = gridDim.x > 1 ? a.ws + (int64_t)blockIdx.x * a.H : a.dw;
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    const int c = (i * TPR + tid) * 8;
    Run8<kF32> out;
    out.set(dw[i]);
    store_run(out, to, c, a.H - c);
  }
}

// dw: the sum of n rows of the workspace.  A wave adds 16 lanes x 4 columns of four rows at a time, a workgroup 64 rows; what its waves have is joined in LDS.
__global__ __launch_bounds__(1024) void rmsnorm_dweight_kernel(const float* ws, float* dw, int n, int H) {
  __shared__ float lds[64][65];
  const int lane = threadIdx.x & 15, row = threadIdx.x >> 4, c = blockIdx.x * 64 + lane * 4;
  float v[4] = {};
#pragma unroll 4
  for (int r = row; r < n; r += 64) {
    const float* p = ws + (int64_t)r * H + c;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += c + k < H ? p[k] : 0.0f;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) lds[lane * 4 + k][row] = v[k];
  __syncthreads();
  // column threadIdx.x / 16: its 64 numbers on 16 lanes
  const int col = threadIdx.x >> 4;
  float s = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) s += lds[col][lane + 16 * k];
  s = row16_all<Add>(s);
  if (lane == 0 && blockIdx.x * 64 + col < H) dw[blockIdx.x * 64 + col] = s;
}
__global__ __launch_bounds__(256) void rmsnorm_no_rows_kernel(float* dw, int H) {
  if (blockIdx.x * 256 + threadIdx.x < (uint32_t)H) dw[blockIdx.x * 256 + threadIdx.x] = 0;
}

// Threads and runs of a row.
template <int TPR_, int RUNS_>
struct RowShape {
  static constexpr int TPR = TPR_, RUNS = RUNS_, ROWS = norm_threads(TPR) / TPR;
};
template <class F>
void by_row_shape(int H, F&& f) {
  if (H <= 64 * 8) f(RowShape<64, 1>());
  else if (H <= 128 * 8) f(RowShape<64, 2>());
  else if (H <= 256 * 8) f(RowShape<256, 1>());
  else if (H <= 512 * 8) f(RowShape<256, 2>());
  else if (H <= 1024 * 8) f(RowShape<256, 4>());
  else if (H <= 2048 * 8) f(RowShape<1024, 2>());
  else f(RowShape<1024, 4>());
}

template <int XT, int YT>
void launch_forward(const NormArgs& a, hipStream_t s) {
  by_row_shape(a.H, [&](auto shape) {
    using S = decltype(shape);
    rmsnorm_kernel<XT, YT, S::TPR, S::RUNS><<<(uint32_t)((a.T + S::ROWS - 1) / S::ROWS), norm_threads(S::TPR), 0, s>>>(a);
  });
}

hipError_t launch_rmsnorm(const NormArgs& a, hipStream_t s) {
  const bool fp8 = a.y_type == kFp8;
  if (a.x_type == kBf16) fp8 ? launch_forward<kBf16, kFp8>(a, s) : launch_forward<kBf16, kBf16>(a, s);
  else if (a.x_type == kF16) fp8 ? launch_forward<kF16, kFp8>(a, s) : launch_forward<kF16, kF16>(a, s);
  else if (fp8) launch_forward<kF32, kFp8>(a, s);
  else if (a.y_type == kBf16) launch_forward<kF32, kBf16>(a, s);
  else if (a.y_type == kF16) launch_forward<kF32, kF16>(a, s);
  else launch_forward<kF32, kF32>(a, s);
  return hipGetLastError();
}

// Workgroups of the backward kernel.
static int64_t backward_groups(int64_t T, int64_t H) {
  const int rows = H <= 1024 ? 4 : 1;
  const int64_t most = H <= 8192 ? 512 : 256, n = (T + rows - 1) / rows;
  return n < most ? n : most;
}
int64_t rmsnorm_workspace_words(int64_t T, int64_t H) {
  const int64_t n = backward_groups(T, H);
  return n > 1 ? n * H : 0;
}

template <int XT, int YT>
void launch_backward(const NormArgs& a, uint32_t groups, hipStream_t s) {
  by_row_shape(a.H, [&](auto shape) {
    using S = decltype(shape);
    rmsnorm_backward_kernel<XT, YT, S::TPR, S::RUNS><<<groups, norm_threads(S::TPR), (S::ROWS - 1) * S::TPR * S::RUNS * 8 * 4, s>>>(a);
  });
}

hipError_t launch_rmsnorm_backward(const NormArgs& a, hipStream_t s) {
  const uint32_t groups = (uint32_t)backward_groups(a.T, a.H);
  if (!groups) {
    rmsnorm_no_rows_kernel<<<(a.H + 255) / 256, 256, 0, s>>>(a.dw, a.H);
    return hipGetLastError();
  }
  if (a.x_type == kBf16) launch_backward<kBf16, kBf16>(a, groups, s);
  else if (a.x_type == kF16) launch_backward<kF16, kF16>(a, groups, s);
  else if (a.y_type == kBf16) launch_backward<kF32, kBf16>(a, groups, s);
  else if (a.y_type == kF16) launch_backward<kF32, kF16>(a, groups, s);
  else launch_backward<kF32, kF32>(a, groups, s);
  if (a.dw && groups > 1) rmsnorm_dweight_kernel<<<(a.H + 63) / 64, 1024, 0, s>>>(a.ws, a.dw, (int)groups, a.H);
  return hipGetLastError();
}

}  // namespace axe
