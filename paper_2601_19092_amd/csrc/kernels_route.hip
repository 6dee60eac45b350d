// Routing of tokens to experts, the experts' order of the pairs, and the gradient of the logits (axe_route, axe_route_backward).  gfx950 only.
#include <hip/hip_runtime.h>

#include "layer_ops.h"
#include "row_ops.h"

namespace axe {

// A logit as the formulas take it: NaN is a masked expert (-inf), +inf the largest number.
__device__ __forceinline__ float logit_at(const RouteArgs& a, int64_t t, int e) {
  const float l = load_elem(a.logits, t * a.ld + e, a.type);
  return l != l ? -__builtin_inff() : fminf(l, 3.4028234663852886e38f);
}
__device__ __forceinline__ float sigmoid(float l) { return 1.0f / (1.0f + expf(-l)); }
__device__ __forceinline__ float wave_max(float v) {
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ int wave_min(int v) {
  for (int d = 32; d; d >>= 1) v = min(v, __shfl_xor(v, d));
  return v;
}

// One wave per token: scores and choices in LDS, k times the largest choice.
__global__ __launch_bounds__(64) void route_kernel(RouteArgs a) {
  __shared__ float score[kRouteMaxE], choice[kRouteMaxE], gscore[kRouteMaxGroups];
  const int64_t t = blockIdx.x;
  const int lane = threadIdx.x;
  const float none = -__builtin_inff();
  float m = none, total = 0;
  if (!a.sigmoid) {
    for (int e = lane; e < a.E; e += 64) m = fmaxf(m, logit_at(a, t, e));
    m = wave_max(m);
    if (m == none) m = 0;
    for (int e = lane; e < a.E; e += 64) total += expf(logit_at(a, t, e) - m);
    total = wave_sum(total);
  }
  for (int e = lane; e < a.E; e += 64) {
    const float l = logit_at(a, t, e);
    const float s = a.sigmoid ? sigmoid(l) : total > 0 ? expf(l - m) / total : 0.0f;
    float c = a.bias ? s + a.bias[e] : a.sigmoid ? s : l;
    score[e] = s;
    choice[e] = l == none || c != c ? none : c;
  }
  __syncthreads();
  if (a.groups > 1) {
    const int per = a.E / a.groups;
    if (lane < a.groups) {
      float first = none, second = none;
      for (int i = 0; i < per; ++i) {
        float c = choice[lane * per + i];
        if (!a.bias && !a.sigmoid && c != none) c = score[lane * per + i];
        if (c > first) second = first, first = c;
        else if (c > second) second = c;
      }
      gscore[lane] = a.top2 && second != none ? first + second : first;
    }
    __syncthreads();
    for (int e = lane; e < a.E; e += 64) {
      const int g = e / per;
      int better = 0;
      for (int o = 0; o < a.groups; ++o) better += gscore[o] > gscore[g] || (gscore[o] == gscore[g] && o < g);
      if (better >= a.kept) choice[e] = none;
    }
    __syncthreads();
  }
  float mine = 0, sum = 0;
  int id = -1;
  for (int j = 0; j < a.k; ++j) {
    float best = none;
    int at = 1 << 30;
    for (int e = lane; e < a.E; e += 64)
      if (choice[e] > best) best = choice[e], at = e;
    const float top = wave_max(best);
    if (top == none) break;
    at = wave_min(best == top ? at : 1 << 30);
    if (lane == j) id = at, mine = score[at];
    sum += score[at];
    __syncthreads();
    if (lane == 0) choice[at] = none;
    __syncthreads();
  }
  if (lane < a.k) {
    a.ids[t * a.k + lane] = id;
    a.weights[t * a.k + lane] = id < 0 || (a.renorm && !(sum > 0)) ? 0.0f : a.renorm ? a.scale * (mine / sum) : a.scale * mine;
  }
}

// One workgroup: a thread per expert counts, then places its pairs.
__global__ __launch_bounds__(kRouteMaxE) void route_order_kernel(RouteArgs a) {
  __shared__ int count[kRouteMaxE + 1];
  const int e = threadIdx.x;
  const int64_t pairs = a.T * a.k;
  int n = 0;
  for (int64_t p = 0; p < pairs; ++p) n += a.ids[p] == e;
  count[e] = n;
  __syncthreads();
  int at = 0;
  for (int o = 0; o < e; ++o) at += count[o];
  if (e < a.E) a.group_rows[e] = at;
  if (e == a.E - 1) a.group_rows[a.E] = at + n;
  for (int64_t p = 0; p < pairs; ++p) {
    if (a.ids[p] == e && e < a.E) a.row_of[p] = at++;
    if (a.ids[p] < 0 && e == 0) a.row_of[p] = -1;
  }
}

__global__ __launch_bounds__(64) void route_backward_kernel(RouteArgs a) {
  __shared__ float ds[kRouteMaxE];
  const int64_t t = blockIdx.x;
  const int lane = threadIdx.x;
  const float none = -__builtin_inff();
  float m = none, total = 0;
  if (!a.sigmoid) {
    for (int e = lane; e < a.E; e += 64) m = fmaxf(m, logit_at(a, t, e));
    m = wave_max(m);
    if (m == none) m = 0;
    for (int e = lane; e < a.E; e += 64) total += expf(logit_at(a, t, e) - m);
    total = wave_sum(total);
  }
  auto score = [&](float l) { return a.sigmoid ? sigmoid(l) : total > 0 ? expf(l - m) / total : 0.0f; };
  for (int e = lane; e < a.E; e += 64) ds[e] = 0;
  __syncthreads();
  const int id = lane < a.k ? a.ids_in[t * a.k + lane] : -1;
  const bool there = id >= 0 && id < a.E;
  const float s = there ? score(logit_at(a, t, id)) : 0.0f;
  float g = there ? a.dweights[t * a.k + lane] * a.scale : 0.0f;
  if (a.renorm) {
    const float sum = wave_sum(s);
    const float mean = wave_sum(sum > 0 ? g * (s / sum) : 0.0f);
    g = there && sum > 0 ? (g - mean) / sum : 0.0f;
  }
  if (there) ds[id] = g;
  __syncthreads();
  const float along = a.sigmoid || a.renorm ? 0.0f : wave_sum(g * s);
  for (int e = lane; e < a.E; e += 64) {
    const float l = logit_at(a, t, e), p = score(l);
    store_elem(a.dlogits, t * a.ld + e, a.type, l == none ? 0.0f : a.sigmoid ? p * (1.0f - p) * ds[e] : p * (ds[e] - along));
  }
}

int64_t route_workspace_words(int64_t, int, int) { return 0; }

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
  if (a.T) route_kernel<<<(uint32_t)a.T, 64, 0, s>>>(a);
  if (a.group_rows) route_order_kernel<<<1, kRouteMaxE, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s) {
  route_backward_kernel<<<(uint32_t)a.T, 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace axe
