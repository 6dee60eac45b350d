// Root-mean-square norm of a residual stream, and its gradient (axe_rmsnorm, axe_rmsnorm_backward).  gfx950 only.
//
// Both are bound by memory: a row is read once and held in registers as fp32, in runs of 8 columns a thread (thread i of the TPR threads of a row holds the runs
// i, i + TPR, ...: neighbouring lanes read neighbouring 16 bytes), its sum of squares is joined over the wave by DPP and over the waves of a row through LDS, and what is
// written comes from the registers.  A run of 128 columns that shares a scale is 16 neighbouring lanes: its maximum never leaves a DPP row.
#include <hip/hip_runtime.h>

#include "layer_ops.h"
#include "layer_shapes.h"
#include "row_ops.h"

namespace axe {

// XT: x, residual and sum; YT: y.  A row of up to TPR * 8 * RUNS columns; SHORT: of fewer than 8.
template <int XT, int YT, int TPR, int RUNS, bool SHORT>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void rmsnorm_kernel(NormArgs a) {
  constexpr int WAVES = TPR / 64, ROWS = TPR == 64 ? 4 : 1;
  __shared__ float lds[WAVES];
  fetch_arguments(a.x, a.T, a.eps);
  const int c = threadIdx.x % TPR * 8;                             // column of the thread's first run
  const int64_t t = (int64_t)blockIdx.x * ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  if (t >= a.T) return;                                            // (whole waves of rows of one wave, or none)
  Run8<XT> x[RUNS], r[RUNS];
  const void *rx = elem_at(a.x, t * a.ldx, elem_bytes(XT)), *rr = elem_at(a.r, t * a.ldr, elem_bytes(XT));
#pragma unroll
  for (int i = 0; i < RUNS; ++i) load_run<SHORT>(x[i], rx, c + i * TPR * 8, a.H);
  if (a.r) {
#pragma unroll
    for (int i = 0; i < RUNS; ++i) load_run<SHORT>(r[i], rr, c + i * TPR * 8, a.H);
  } else {
#pragma unroll
    for (int i = 0; i < RUNS; ++i) r[i].clear();
  }
  float w[RUNS][8];
  load_weights<SHORT, TPR>(w, a.w, a.w_type, c, a.H);
  float h[RUNS][8], sq[1] = {0};
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    end_run<SHORT>(x[i], c + i * TPR * 8, a.H);
    end_run<SHORT>(r[i], c + i * TPR * 8, a.H);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      h[i][k] = x[i].get(k) + r[i].get(k);
      sq[0] += h[i][k] * h[i][k];
    }
  }
  if (a.sum) {
    void* rs = elem_at(a.sum, t * a.lds, elem_bytes(XT));
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      x[i].set(h[i]);
      store_run<true>(x[i], rs, c + i * TPR * 8, a.H);             // (past the caches: read again behind the experts' products at the soonest; us, past / cached: 4096 x 2048 11.1 / 11.5, 1000 x 8192 11.6 / 11.9, 64 x 2048 2.7 / 2.6, a whole layer the same)
    }
  }
  row_sums<1, WAVES>(sq, lds, threadIdx.x % TPR >> 6);
  const float rho = 1.0f / sqrtf(sq[0] / (float)a.H + a.eps);
  void* ry = elem_at(a.y, t * a.ldy, elem_bytes(YT));
#pragma unroll
  for (int i = 0; i < RUNS; ++i) {
    const int ci = c + i * TPR * 8;
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = h[i][k] * rho * w[i][k];
    Run8<YT> q;
    if constexpr (YT == kFp8) {
      float most = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) most = fmaxf(most, fabsf(y[k]));  // (NaN: the other operand)
      const Scale s = scale_of(row16_all<Max>(most), a.e8m0);
      over_scale(y, s);
      if ((threadIdx.x & 15) == 0 && ci < a.H) store_scale(a.scales, t * ((a.H + 127) >> 7) + (ci >> 7), s, a.e8m0);
    }
    q.set(y);
    store_run(q, ry, ci, a.H);
  }
}

// Gradients.  XT: h, dsum and dx; YT: dy.  A workgroup takes every gridDim-th row (rows of one wave: four at a time) and keeps its threads' columns of dw in
// registers; what a workgroup has of dw goes to its row of the workspace, and a second kernel adds these rows up.  ONCE: loads past the caches.
template <int XT, int YT, int TPR, int RUNS, int ROWS, bool ONCE, bool SHORT>
__global__ __launch_bounds__(TPR * ROWS) void rmsnorm_backward_kernel(NormArgs a) {
  constexpr int WAVES = TPR / 64;
  __shared__ float lds[2][ROWS][2 * WAVES];
  extern __shared__ float part[];
  fetch_arguments(a.x, a.T, a.eps);
  const int tid = threadIdx.x % TPR, c = tid * 8, sub = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  float dw[RUNS][8] = {};
  int turn = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * ROWS; t0 < a.T; t0 += (int64_t)gridDim.x * ROWS, turn ^= 1) {
    const bool there = t0 + sub < a.T;
    const int64_t t = there ? t0 + sub : a.T - 1;                  // (all rows of a workgroup take part in its barriers)
    Run8<YT> dy[RUNS];
    Run8<XT> h[RUNS], ds[RUNS];
    const void *rd = elem_at(a.x, t * a.ldx, elem_bytes(YT)), *rh = elem_at(a.h, t * a.lds, elem_bytes(XT)), *rs = elem_at(a.r, t * a.ldr, elem_bytes(XT));
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      load_run<SHORT, ONCE>(dy[i], rd, c + i * TPR * 8, a.H);
      load_run<SHORT, ONCE>(h[i], rh, c + i * TPR * 8, a.H);
    }
    if (a.r) {
#pragma unroll
      for (int i = 0; i < RUNS; ++i) load_run<SHORT, ONCE>(ds[i], rs, c + i * TPR * 8, a.H);
    } else {
#pragma unroll
      for (int i = 0; i < RUNS; ++i) ds[i].clear();
    }
    float u[RUNS][8], s[2] = {0, 0};
    load_weights<SHORT, TPR>(u, a.w, a.w_type, c, a.H);
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      end_run<SHORT>(dy[i], c + i * TPR * 8, a.H);
      if (!there) dy[i].clear();
      end_run<SHORT>(h[i], c + i * TPR * 8, a.H);
      end_run<SHORT>(ds[i], c + i * TPR * 8, a.H);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        u[i][k] *= dy[i].get(k);
        s[0] += h[i].get(k) * h[i].get(k), s[1] += u[i][k] * h[i].get(k);
      }
    }
    row_sums<2, WAVES>(s, lds[turn][sub], tid >> 6);                            // (two arrays: no thread is two rows ahead of another)
    const float rho = 1.0f / sqrtf(s[0] / (float)a.H + a.eps);
    const float along = s[1] / (float)a.H * rho * rho;
    void* ro = elem_at(a.y, t * a.ldy, elem_bytes(XT));
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[k] = rho * (u[i][k] - h[i].get(k) * along) + ds[i].get(k);
        dw[i][k] += dy[i].get(k) * (h[i].get(k) * rho);
      }
      Run8<XT> out;
      out.set(v);
      if (there) store_run(out, ro, c + i * TPR * 8, a.H);
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
    lds_barrier();
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
    Run8<kF32> out;
    out.set(dw[i]);
    store_run(out, to, c + i * TPR * 8, a.H);
  }
}

// dw: the sum of n rows of the workspace, 64 columns a workgroup: wave i adds the rows i, i + 16, ... -- loads without an order, eight in flight -- and the sums of the
// sixteen waves are joined through LDS.  us, 512 rows of 2048 / 8192: 3.8 / 4.9; 16 columns a workgroup 3.9 / 7.0.
__global__ __launch_bounds__(1024) void rmsnorm_dweight_kernel(const float* ws, float* dw, int n, int H) {
  __shared__ float lds[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane, at = c < H ? c : H - 1;
  float v[8] = {};
  int r = wave;
  for (; r + 7 * 16 < n; r += 8 * 16)
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += ws[(int64_t)(r + 16 * k) * H + at];
#pragma unroll
  for (int k = 0; k < 7; ++k)
    if (r + 16 * k < n) v[k] += ws[(int64_t)(r + 16 * k) * H + at];
  lds[wave][lane] = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  lds_barrier();
  if (wave) return;
  float s = 0;
#pragma unroll
  for (int k = 0; k < 16; ++k) s += lds[k][lane];
  if (c < H) dw[c] = s;
}
__global__ __launch_bounds__(256) void rmsnorm_no_rows_kernel(float* dw, int H) {
  if (blockIdx.x * 256 + threadIdx.x < (uint32_t)H) dw[blockIdx.x * 256 + threadIdx.x] = 0;
}

template <int XT, int YT>
void launch_forward(const NormArgs& all, hipStream_t s) {
  // (a launch holds fewer than 2^32 threads)
  constexpr int64_t kPiece = int64_t(1) << 21;
  for (int64_t t0 = 0; t0 < all.T; t0 += kPiece) {
    NormArgs a = all;
    a.T = all.T - t0 < kPiece ? all.T - t0 : kPiece;
    a.x = elem_at(all.x, t0 * all.ldx, elem_bytes(XT));
    if (all.r) a.r = elem_at(all.r, t0 * all.ldr, elem_bytes(XT));
    if (all.sum) a.sum = elem_at(all.sum, t0 * all.lds, elem_bytes(XT));
    a.y = elem_at(all.y, t0 * all.ldy, elem_bytes(YT));
    a.scales = elem_at(all.scales, t0 * ((all.H + 127) / 128), all.e8m0 ? 1 : 4);
    by_row_shape(a.H, [&](auto shape) {
      using S = decltype(shape);
      if (S::TPR == 64) rmsnorm_kernel<XT, YT, S::TPR, S::RUNS, S::SHORT><<<(uint32_t)((a.T + 3) / 4), 256, 0, s>>>(a);
      else rmsnorm_kernel<XT, YT, S::TPR, S::RUNS, S::SHORT><<<(uint32_t)a.T, S::TPR, 0, s>>>(a);
    });
  }
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

template <int XT, int YT>
void launch_backward(const NormArgs& a, uint32_t groups, hipStream_t s) {
  const bool once = a.T * a.H * (elem_bytes(YT) + elem_bytes(XT) * (a.r ? 3 : 2)) >= kReadsPastCaches;
  by_row_shape(a.H, [&](auto shape) {
    using S = decltype(shape);
    constexpr int lds = (S::ROWS - 1) * S::TPR * S::RUNS * 8 * 4;
    if (once && !S::SHORT) rmsnorm_backward_kernel<XT, YT, S::TPR, S::RUNS, S::ROWS, !S::SHORT, S::SHORT><<<groups, S::TPR * S::ROWS, lds, s>>>(a);
    else rmsnorm_backward_kernel<XT, YT, S::TPR, S::RUNS, S::ROWS, false, S::SHORT><<<groups, S::TPR * S::ROWS, lds, s>>>(a);
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
