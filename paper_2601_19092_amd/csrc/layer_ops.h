// Arguments of the kernels around the experts' products (norm, routing, rows), by value, and their launches.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace axe {

// Element types by the codes of axe.h.
constexpr int kBf16 = 1, kFp8 = 2, kF32 = 3, kF16 = 4;
constexpr int elem_bytes(int type) { return type == kF32 ? 4 : type == kFp8 ? 1 : 2; }

// (Every field of a line of 64 bytes comes with the others: the kernels name one of each, fetch_arguments.)
struct NormArgs {
  const void *x, *r, *w;       // rows, residual (or null), weights (or null: ones); backward: dy, dsum, weights
  const void* h;               // backward: the normed rows
  void *sum, *y;               // h out (or null), y; backward: y = dx
  void* scales;                // of an 8-bit y
  float* dw;                   // backward
  float* ws;
  int64_t T, ldx, ldr, lds, ldy;
  int32_t H;
  int32_t x_type, y_type, w_type, e8m0;
  float eps;
};
constexpr int64_t kNormMaxH = 32768;
hipError_t launch_rmsnorm(const NormArgs& a, hipStream_t s);
hipError_t launch_rmsnorm_backward(const NormArgs& a, hipStream_t s);

struct RouteArgs {
  const void* logits;
  const float* bias;
  int32_t *ids, *group_rows, *row_of, *ws;
  float* weights;
  const int32_t* ids_in;       // backward
  const float* dweights;
  void* dlogits;
  int64_t T, ld;
  int32_t E, k, type, sigmoid, renorm, groups, kept, top2;
  int32_t per;                 // experts of a group
  float scale;
};
constexpr int kRouteMaxE = 1024, kRouteMaxK = 64, kRouteMaxGroups = 64;
hipError_t launch_route(const RouteArgs& a, hipStream_t s);
hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s);

// Bytes of a call from which its large operands go past the caches (non-temporal): they do not stay until they are touched again, and evicting for them costs time.  us, three sets of
// buffers in turn.  Loads of combine's rows, cached / past: 2048 tokens of 8 rows of 2048 bf16 (72 MiB in all) 12.8 / 14.4, 3000 (105 MiB) 22.8 / 19.8, 4096 30.9 / 27.1.
// Its gradient's stores: 1024 (68 MiB) 12.8 / 12.8, 1500 (100 MiB) 20.6 / 17.6, 2048 30.4 / 23.4; its loads as well: 2048 (136 MiB) 23.4 / 27.7, 4096 (272 MiB) 56.2 / 52.4.  The norm's gradient's loads:
// 4096 x 2048 (64 MiB) 13.4 / 15.8, 3000 x 8192 (188 MiB) 42.4 / 39.2, 4096 x 8192 55.9 / 53.0.  dispatch keeps its stores in the caches: past them 4096 tokens to e4m3 take
// 14.7 for 15.4, but with the next kernel, which reads them, 45.4 for 41.4.  (The other lines are those of this loop: between the layer's products combine takes the same either way, and its gradient with a
// reader of its rows behind it, one set of buffers, 2048 / 4096 / 8000 tokens, 33.7 / 81 / 157, all cached 31.5 / 66 / 172.)
constexpr int64_t kPastCaches = int64_t(96) << 20, kReadsPastCaches = int64_t(128) << 20, kAllPastCaches = int64_t(256) << 20;

struct RowsArgs {
  const void *tokens, *rows;   // what is read of the two matrices
  void *to_tokens, *to_rows;   // what is written
  const void *add, *token_scales;
  void* scales;
  const int32_t* row_of;
  const float* weights;
  float* dweights;
  int64_t T, M, ldt, ldr;
  int32_t H, k, t_type, r_type, e8m0;
};
constexpr int kRowsMaxK = 64;
hipError_t launch_rows_dispatch(const RowsArgs& a, hipStream_t s);
hipError_t launch_rows_combine(const RowsArgs& a, hipStream_t s);
hipError_t launch_rows_combine_backward(const RowsArgs& a, hipStream_t s);

}  // namespace axe
