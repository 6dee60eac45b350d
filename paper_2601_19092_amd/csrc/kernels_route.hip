// Routing of tokens to experts, the experts' order of the pairs, and the gradient of the logits (axe_route, axe_route_backward).  gfx950 only.
//
// A token's logits are a few hundred bytes, so what these calls cost is the launches and the chain of dependent steps behind each token, not memory.  A
// token has 16 lanes (64 beyond 256 experts or 16 choices), each with 8 or 16 neighbouring experts in registers; k times its lanes agree on the largest choice (a maximum by DPP,
// then the lowest index that has it) and its owner strikes it out.  Choices are compared as integers of the same order as the numbers.
//
// The experts' order is a stable counting sort.  A workgroup has a block of consecutive tokens, 64 at a time, as bits of one 64-bit mask per expert in LDS: whatever the order
// in which the bits arrive, the number of set bits below a token's is its place among the expert's pairs.  Up to 64 tokens are one workgroup, which goes on to add up the
// experts.  More leave places inside the block and the block's count per expert (16 bits) behind; a second kernel, a workgroup per block, adds up the counts of
// all blocks (its own share of that work is small, and there is nothing to wait for) and moves the places to where expert and block begin.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "layer_ops.h"
#include "row_ops.h"

namespace axe {

constexpr int kMaskTokens = 64;                                    // tokens of a mask
constexpr int kNone = INT32_MIN;                                   // below every choice

// A logit as the formulas take it: NaN is a masked expert (-inf), +inf the largest number; -0 is 0.
__device__ __forceinline__ float as_logit(float l) { return l != l ? -__builtin_inff() : fminf(l, 3.4028234663852886e38f) + 0.0f; }
__device__ __forceinline__ float sigmoid(float l) { return 1.0f / (1.0f + expf(-l)); }
// Integers in the order of numbers above -inf; -inf and NaN: none.
__device__ __forceinline__ int key_of(float v) {
  const int b = __float_as_int(v);
  return v > -__builtin_inff() ? b ^ ((b >> 31) & 0x7fffffff) : kNone;
}
// Over the LPT lanes of a token, in each of them.
struct IMax {
  __device__ __forceinline__ static int of(int a, int b) { return max(a, b); }
};
struct IMin {
  __device__ __forceinline__ static int of(int a, int b) { return min(a, b); }
};
template <int LPT, class OP>
__device__ __forceinline__ int all_int(int v) {
  v = OP::of(v, dpp<kXor1>(v));
  v = OP::of(v, dpp<kXor2>(v));
  v = OP::of(v, dpp<kHalfMirror>(v));
  v = OP::of(v, dpp<kMirror>(v));
  if (LPT == 16) return v;
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = OP::of((int)a[0], (int)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return OP::of((int)b[0], (int)b[1]);
}
template <int LPT, class OP>
__device__ __forceinline__ float all_float(float v) { return LPT == 16 ? row16_all<OP>(v) : wave_all<OP>(v); }

// What a lane has of a token's logits: experts e0 .. e0 + V - 1, -inf beyond the last.
template <int XT, int LPT, int V, bool SHORT>
struct Logits {
  float l[V];
  int e0;
  __device__ __forceinline__ Logits(const RouteArgs& a, const void* row, int lane) {
    e0 = lane * V;
    Run8<XT> r[V / 8];
#pragma unroll
    for (int i = 0; i < V / 8; ++i) load_run<SHORT>(r[i], row, e0 + 8 * i, a.E);
#pragma unroll
    for (int i = 0; i < V / 8; ++i) {
      end_run<SHORT>(r[i], e0 + 8 * i, a.E);
#pragma unroll
      for (int k = 0; k < 8; ++k) l[8 * i + k] = e0 + 8 * i + k < a.E ? as_logit(r[i].get(k)) : -__builtin_inff();
    }
  }
  __device__ __forceinline__ float top() const {                   // the row's largest, 0 if there is none
    float m = l[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, l[v]);
    m = all_float<LPT, Max>(m);
    return m > -__builtin_inff() ? m : 0.0f;
  }
};

// Exclusive sums of n <= 1024 numbers in LDS, by one wave; the last lane's return value is the sum of all.
__device__ __forceinline__ int scan_in_place(int* x, int n) {
  const int lane = threadIdx.x & 63, per = (n + 63) / 64, first = lane * per;
  int s = 0;
  for (int i = first; i < first + per && i < n; ++i) s += x[i];
  int before = s;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(before, d);
    if (lane >= d) before += o;
  }
  const int all = before;
  before -= s;
  for (int i = first; i < first + per && i < n; ++i) {
    const int c = x[i];
    x[i] = before;
    before += c;
  }
  return all;
}

// LDS of a workgroup of `threads` threads.
template <int LPT, bool GROUPS>
size_t route_lds(const RouteArgs& a, int threads) {
  return (size_t)a.E * 12 + kMaskTokens * a.k * 2 + 16 + (GROUPS ? (size_t)(threads / LPT) * (a.E + 2 * a.groups) * 4 : 0);
}

// Strikes out the experts of the groups that do not stay.  by: what the lane's experts' groups are judged by (-inf: masked).
template <int LPT, int V>
__device__ __forceinline__ void keep_groups(const RouteArgs& a, int lane, int e0, const float (&by)[V], int (&key)[V], float* mine) {
  const int per = a.E / a.groups;
  float* score = mine + a.E;
  int* keep = (int*)(score + a.groups);
  auto wave_sync = [] {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  wave_sync();                                                     // (the token before has been read)
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (e0 + v < a.E) mine[e0 + v] = by[v];
  wave_sync();
  const float none = -__builtin_inff();
  for (int g = lane; g < a.groups; g += LPT) {
    float first = none, second = none;
    for (int n = 0, i = g % per; n < per; ++n, i = i + 1 == per ? 0 : i + 1) {     // (started apart: neighbouring lanes on neighbouring banks)
      const float c = mine[g * per + i];
      second = fmaxf(second, fminf(first, c));
      first = fmaxf(first, c);
    }
    score[g] = a.top2 && second > none ? first + second : first;
  }
  wave_sync();
  for (int g = lane; g < a.groups; g += LPT) {
    const float s = score[g];
    int better = 0;
    for (int o = 0; o < a.groups; ++o) better += score[o] > s || (score[o] == s && o < g);
    keep[g] = better < a.kept;
  }
  wave_sync();
  int g = e0 / per, left = (g + 1) * per - e0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (e0 + v < a.E && !keep[g]) key[v] = kNone;
    if (--left == 0) ++g, left = per;
  }
}

// tokens: of a workgroup.  With the order: places inside the block to row_of and the block's counts to the workspace, or, alone, the whole order.
template <int XT, int LPT, int V, bool GROUPS, bool SHORT>
__global__ __launch_bounds__(GROUPS ? 512 : 1024) void route_kernel(RouteArgs a, int tokens, bool alone, int counts_pitch) {
  extern __shared__ char mem[];
  uint64_t* mask = (uint64_t*)mem;
  int* run = (int*)(mask + a.E);                                   // the expert's pairs in the block's tokens before these
  uint16_t* chosen = (uint16_t*)(run + a.E);
  float* by_group = (float*)(((uintptr_t)(chosen + kMaskTokens * a.k) + 15) & ~(uintptr_t)15) + (GROUPS ? threadIdx.x / LPT * (a.E + 2 * a.groups) : 0);
  const int tid = threadIdx.x, threads = blockDim.x, lane = tid % LPT;
  const int64_t b0 = (int64_t)blockIdx.x * tokens, b1 = b0 + tokens < a.T ? b0 + tokens : a.T;
  const bool order = a.row_of != nullptr;
  if (order)
    for (int e = tid; e < a.E; e += threads) run[e] = 0;
  for (int64_t s0 = b0; s0 < b1; s0 += kMaskTokens) {
    const int n = (int)(b1 - s0 < kMaskTokens ? b1 - s0 : kMaskTokens);
    if (order) {
      for (int e = tid; e < a.E; e += threads) mask[e] = 0;
      __syncthreads();
    }
    for (int i = tid / LPT; i < n; i += threads / LPT) {
      const int64_t t = s0 + i;
      const void* row = elem_at(a.logits, t * a.ld, elem_bytes(XT));
      const Logits<XT, LPT, V, SHORT> x(a, row, lane);
      const float none = -__builtin_inff();
      const float m = a.sigmoid ? 0.0f : x.top();
      float total = 1.0f;
      int key[V];
      if (!a.sigmoid && !a.bias) {                                 // by the logits themselves
        if (!a.renorm) {
          total = 0;
#pragma unroll
          for (int v = 0; v < V; ++v) total += expf(x.l[v] - m);
          total = all_float<LPT, Add>(total);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = key_of(x.l[v]);
        if (GROUPS) {
          float by[V];                                             // (scores up to a common factor)
#pragma unroll
          for (int v = 0; v < V; ++v) by[v] = key[v] == kNone ? none : a.top2 ? expf(x.l[v] - m) : x.l[v];
          keep_groups<LPT, V>(a, lane, x.e0, by, key, by_group);
        }
      } else {
        float s[V];
        if (a.sigmoid) {
#pragma unroll
          for (int v = 0; v < V; ++v) s[v] = sigmoid(x.l[v]);
        } else {
          total = 0;
#pragma unroll
          for (int v = 0; v < V; ++v) total += s[v] = expf(x.l[v] - m);
          total = all_float<LPT, Add>(total);
          const float inv = total > 0 ? 1.0f / total : 0.0f;
#pragma unroll
          for (int v = 0; v < V; ++v) s[v] *= inv;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (a.bias && x.e0 + v < a.E) s[v] += a.bias[x.e0 + v];
          s[v] = x.l[v] > none && s[v] > none ? s[v] + 0.0f : none;  // (NaN compares false)
          key[v] = key_of(s[v]);
        }
        if (GROUPS) keep_groups<LPT, V>(a, lane, x.e0, s, key, by_group);
      }
      int id = -1;
      for (int j = 0; j < a.k; ++j) {
        int best = key[0];
#pragma unroll
        for (int v = 1; v < V; ++v) best = max(best, key[v]);
        best = all_int<LPT, IMax>(best);
        int at = INT32_MAX;
#pragma unroll
        for (int v = V - 1; v >= 0; --v) at = key[v] == best ? x.e0 + v : at;
        at = all_int<LPT, IMin>(at);
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = x.e0 + v == at ? kNone : key[v];
        if (lane == j && best != kNone) id = at;
      }
      // lane j: the weight of choice j
      float w = 0;
      if (id >= 0) {
        float l[1];
        Run8<XT> one;
        one.load_part((const typename Run8<XT>::Elem*)row + id, 1);
        l[0] = as_logit(one.get(0));
        w = a.sigmoid ? sigmoid(l[0]) : expf(l[0] - m);
      }
      if (a.renorm) total = all_float<LPT, Add>(w);
      w = total > 0 ? a.scale * (w / total) : 0.0f;
      if (lane < a.k) {
        a.ids[t * a.k + lane] = id;
        a.weights[t * a.k + lane] = w;
        if (order) {
          chosen[i * a.k + lane] = (uint16_t)id;
          if (id >= 0) atomicOr((unsigned long long*)&mask[id], 1ull << i);
        }
      }
    }
    if (!order) continue;
    __syncthreads();
    if (alone) {                                                   // (one mask: run becomes where the expert's rows begin)
      for (int e = tid; e < a.E; e += threads) run[e] = __popcll(mask[e]);
      __syncthreads();
      if (tid < 64) {
        const int all = scan_in_place(run, a.E);
        if (tid == 63) a.group_rows[a.E] = all;
      }
      __syncthreads();
      for (int e = tid; e < a.E; e += threads) a.group_rows[e] = run[e];
    }
    for (int p = tid; p < n * a.k; p += threads) {
      const uint16_t e = chosen[p];
      const int i = p / a.k;
      a.row_of[s0 * a.k + p] = e == 0xffff ? -1 : run[e] + __popcll(mask[e] & ((1ull << i) - 1));
    }
    if (alone) return;
    __syncthreads();
    for (int e = tid; e < a.E; e += threads) run[e] += __popcll(mask[e]);
  }
  if (!order) return;
  uint16_t* counts = (uint16_t*)a.ws + (int64_t)blockIdx.x * counts_pitch;
  for (int e = tid; e < counts_pitch; e += threads) counts[e] = e < a.E ? (uint16_t)run[e] : 0;
}

// Places inside the blocks to places of all.  counts: blocks x pitch, pitch a power of two from 8 on.
__global__ __launch_bounds__(1024) void route_order_kernel(RouteArgs a, int tokens, int blocks, int pitch) {
  __shared__ int total[kRouteMaxE], before[kRouteMaxE];
  const int tid = threadIdx.x, lane = tid & 63, runs = pitch / 8;
  for (int e = tid; e < pitch; e += 1024) total[e] = before[e] = 0;
  __syncthreads();
  int all[8] = {}, upto[8] = {};
  const int c = tid & (runs - 1);                                  // a thread: eight experts of every (1024 / runs)-th block
#pragma unroll 4
  for (int b = tid / runs; b < blocks; b += 1024 / runs) {
    const u32x4 v = load_bits<u32x4>((const uint16_t*)a.ws + (int64_t)b * pitch + c * 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int lo = v[i] & 0xffff, hi = v[i] >> 16;
      all[2 * i] += lo, all[2 * i + 1] += hi;
      if (b < (int)blockIdx.x) upto[2 * i] += lo, upto[2 * i + 1] += hi;
    }
  }
  for (int d = runs; d < 64; d <<= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i) all[i] += __shfl_xor(all[i], d), upto[i] += __shfl_xor(upto[i], d);
  if (lane < runs)
#pragma unroll
    for (int i = 0; i < 8; ++i) atomicAdd(&total[c * 8 + i], all[i]), atomicAdd(&before[c * 8 + i], upto[i]);   // (integers: any order, one sum)
  __syncthreads();
  if (tid < 64) {
    const int n = scan_in_place(total, a.E);
    if (tid == 63 && blockIdx.x == 0) a.group_rows[a.E] = n;
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int e = tid; e < a.E; e += 1024) a.group_rows[e] = total[e];
  const int64_t p0 = (int64_t)blockIdx.x * tokens * a.k, p1 = p0 + (int64_t)tokens * a.k, end = a.T * a.k;
  for (int64_t p = p0 + tid; p < p1 && p < end; p += 1024) {
    const int e = a.ids[p];
    if (e >= 0) a.row_of[p] += total[e] + before[e];
  }
}
__global__ __launch_bounds__(1024) void route_no_tokens_kernel(int32_t* group_rows, int E) {
  for (int e = threadIdx.x; e <= E; e += 1024) group_rows[e] = 0;
}

// Gradient of the logits; lanes as above.
template <int XT, int LPT, int V, bool SHORT>
__global__ __launch_bounds__(256) void route_backward_kernel(RouteArgs a) {
  const int lane = threadIdx.x % LPT;
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPT;
  if (t >= a.T) return;                                            // (all lanes of a token)
  const void* row = elem_at(a.logits, t * a.ld, elem_bytes(XT));
  const Logits<XT, LPT, V, SHORT> x(a, row, lane);
  int id = lane < a.k ? a.ids_in[t * a.k + lane] : -1;
  if (id >= a.E) id = -1;
  float g = id >= 0 ? a.dweights[t * a.k + lane] * a.scale : 0.0f, own = 0;
  const float m = a.sigmoid ? 0.0f : x.top();
  float s[V], total = 1.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) s[v] = a.sigmoid ? sigmoid(x.l[v]) : expf(x.l[v] - m);
  if (!a.sigmoid) {
    total = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) total += s[v];
    total = all_float<LPT, Add>(total);
  }
  const float inv = total > 0 ? 1.0f / total : 0.0f;
  if (id >= 0) {
    Run8<XT> one;
    one.load_part((const typename Run8<XT>::Elem*)row + id, 1);
    const float l = as_logit(one.get(0));
    own = a.sigmoid ? sigmoid(l) : expf(l - m) * inv;
  }
  float along = 0;
  if (a.renorm) {                                                  // (then the sum of s ds is 0)
    const float sum = all_float<LPT, Add>(own);
    const float share = sum > 0 ? 1.0f / sum : 0.0f;
    const float mean = all_float<LPT, Add>(g * (own * share));
    g = id >= 0 ? (g - mean) * share : 0.0f;
  } else if (!a.sigmoid) {
    along = all_float<LPT, Add>(g * own);
  }
  float ds[V] = {};
  for (int j = 0; j < a.k; ++j) {
    const int e = __shfl(id, j, LPT) - x.e0;
    const float gj = __shfl(g, j, LPT);
#pragma unroll
    for (int v = 0; v < V; ++v) ds[v] += v == e ? gj : 0.0f;
  }
  void* out = elem_at(a.dlogits, t * a.ld, elem_bytes(XT));
#pragma unroll
  for (int i = 0; i < V / 8; ++i) {
    float d[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int v = 8 * i + k;
      const float p = s[v] * inv;
      d[k] = x.l[v] == -__builtin_inff() ? 0.0f : a.sigmoid ? s[v] * (1.0f - s[v]) * ds[v] : p * (ds[v] - along);
    }
    Run8<XT> r;
    r.set(d);
    store_run(r, out, x.e0 + 8 * i, a.E);
  }
}

// Lanes and experts a lane.
template <int LPT_, int V_, bool SHORT_ = false>
struct RouteShape {
  static constexpr int LPT = LPT_, V = V_;
  static constexpr bool SHORT = SHORT_;
};
template <class F>
void by_route_shape(int E, int k, F&& f) {
  if (E < 8) f(RouteShape<16, 8, true>());
  else if (E <= 128 && k <= 16) f(RouteShape<16, 8>());
  else if (E <= 256 && k <= 16) f(RouteShape<16, 16>());
  else if (E <= 512) f(RouteShape<64, 8>());
  else f(RouteShape<64, 16>());
}

// Blocks of tokens: 16 a block, more once that makes more than 256 of them; a block's counts have 16 bits.
static int block_tokens(int64_t T) {
  if (T <= kMaskTokens) return kMaskTokens;
  const int64_t n = (T + 255) / 256;
  return n <= 16 ? 16 : n <= 32 ? 32 : (int)std::min<int64_t>((n + kMaskTokens - 1) / kMaskTokens * kMaskTokens, 65536 - kMaskTokens);
}
static int counts_pitch(int E) {
  int p = 8;
  while (p < E) p *= 2;
  return p;
}
int64_t route_workspace_words(int64_t T, int E, int) {
  if (T <= kMaskTokens) return 0;
  const int tokens = block_tokens(T);
  return (T + tokens - 1) / tokens * counts_pitch(E) / 2;
}

template <int XT>
void launch_route_of(const RouteArgs& a, hipStream_t s) {
  by_route_shape(a.E, a.k, [&](auto shape) {
    using S = decltype(shape);
    const int tokens = block_tokens(a.T), pitch = counts_pitch(a.E), blocks = (int)((a.T + tokens - 1) / tokens);
    const bool alone = blocks == 1;
    const int here = (int)(a.T < tokens ? a.T : tokens);           // tokens at once: all of a mask's, as far as threads and LDS go
    auto threads = [&](int most) { return std::min(most, (std::min(here, kMaskTokens) * S::LPT + 63) / 64 * 64); };
    if (a.groups > 1) {
      const int n = threads(512);
      route_kernel<XT, S::LPT, S::V, true, S::SHORT><<<blocks, n, route_lds<S::LPT, true>(a, n), s>>>(a, tokens, alone, pitch);
    } else {
      const int n = threads(1024);
      route_kernel<XT, S::LPT, S::V, false, S::SHORT><<<blocks, n, route_lds<S::LPT, false>(a, n), s>>>(a, tokens, alone, pitch);
    }
    if (a.row_of && !alone) route_order_kernel<<<blocks, 1024, 0, s>>>(a, tokens, blocks, pitch);
  });
}
hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
  if (a.T == 0) route_no_tokens_kernel<<<1, 1024, 0, s>>>(a.group_rows, a.E);
  else if (a.type == kBf16) launch_route_of<kBf16>(a, s);
  else if (a.type == kF16) launch_route_of<kF16>(a, s);
  else launch_route_of<kF32>(a, s);
  return hipGetLastError();
}

template <int XT>
void launch_route_backward_of(const RouteArgs& all, hipStream_t s) {
  by_route_shape(all.E, all.k, [&](auto shape) {
    using S = decltype(shape);
    constexpr int64_t kPiece = int64_t(1) << 24;                   // (a launch holds fewer than 2^32 threads)
    for (int64_t t0 = 0; t0 < all.T; t0 += kPiece) {
      RouteArgs a = all;
      a.T = std::min(all.T - t0, kPiece);
      a.logits = elem_at(all.logits, t0 * all.ld, elem_bytes(XT)), a.dlogits = elem_at(all.dlogits, t0 * all.ld, elem_bytes(XT));
      a.ids_in += t0 * a.k, a.dweights += t0 * a.k;
      route_backward_kernel<XT, S::LPT, S::V, S::SHORT><<<(uint32_t)((a.T * S::LPT + 255) / 256), 256, 0, s>>>(a);
    }
  });
}
hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s) {
  if (a.type == kBf16) launch_route_backward_of<kBf16>(a, s);
  else if (a.type == kF16) launch_route_backward_of<kF16>(a, s);
  else launch_route_backward_of<kF32>(a, s);
  return hipGetLastError();
}

}  // namespace axe
