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
int64_t rmsnorm_workspace_words(int64_t T, int64_t H);

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
  float scale;
};
constexpr int kRouteMaxE = 1024, kRouteMaxK = 64, kRouteMaxGroups = 64;
hipError_t launch_route(const RouteArgs& a, hipStream_t s);
hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s);
int64_t route_workspace_words(int64_t T, int E, int k);

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
