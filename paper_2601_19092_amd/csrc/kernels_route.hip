// Routing of tokens to experts, the experts' order of the pairs, and the gradient of the logits (axe_route, axe_route_backward).  gfx950 only.
//
// A token's logits are a few hundred bytes, so what these calls cost is the launches and the chain of dependent steps behind each token, not memory.  A
// token has 16 to 64 lanes, each with up to 16 neighbouring experts, sorted, in registers; k times its lanes agree on the largest choice (a maximum of their first ones by DPP,
// then the first lane that has it), whose owner notes it down and moves its list up: some 170 ns each.  Choices are compared as integers of the same order as the numbers.
//
// The experts' order is a stable counting sort.  A workgroup has a block of consecutive tokens, 64 at a time, as bits of one 64-bit mask per expert in LDS: whatever the order
// in which the bits arrive, the number of set bits below a token's is its place among the expert's pairs.  Few tokens (one_workgroup) are one workgroup, which goes on to add up the
// experts.  More leave places inside the block and the block's count per expert (16 bits) behind; a second kernel, a workgroup per block, adds up the counts of
// all blocks (its own share of that work is small, and there is nothing to wait for) and moves the places to where expert and block begin.
#include <hip/hip_runtime.h>

#include "layer_ops.h"
#include "layer_shapes.h"
#include "row_ops.h"

namespace axe {

constexpr int kNone = INT32_MIN;                                   // below every choice

// A logit as the formulas take it: NaN is a masked expert (-inf), +inf the largest number; -0 is 0.
__device__ __forceinline__ float as_logit(float l) { return l != l ? -__builtin_inff() : fminf(l, 3.4028234663852886e38f) + 0.0f; }
// exp(x) = 2^t (1 + d), t = x / ln 2 in fp32 and d ln 2's share of what that rounding left out: the hardware's 2^t is good to its last bit, and so is this.  (Infinities and what is
// beyond fp32 either way end at 200, whose exp is infinite or 0.)
__device__ __forceinline__ float exp_of(float x) {
  x = __builtin_amdgcn_fmed3f(x, -200.0f, 200.0f);
  const float t = x * 1.4426950216293335f;                         // 1 / ln 2 = 1.44269502163 + 1.92596299e-8
  const float d = fmaf(x, 1.925962991126617e-8f, fmaf(x, 1.4426950216293335f, -t));
  const float p = __builtin_amdgcn_exp2f(t);
  return t < 128.0f ? fmaf(p, d * 0.6931471805599453f, p) : p;
}
__device__ __forceinline__ float sigmoid(float l) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-l)); }   // (the reciprocal, too)
// The same down to the smallest subnormal number (the hardware's 2^t ends at the smallest normal one): e^-64 = 1.60381089e-28.
__device__ __forceinline__ float exp_below(float x) {
  const bool far = x < -64.0f;
  return exp_of(far ? x + 64.0f : x) * (far ? 1.60381089e-28f : 1.0f);
}
// The score that a weight is made of.  softmax: exp of how far the logit l is below `largest`.  sigmoid: where `largest` is below 0, that much larger than it is.  With the chosen experts' largest
// logit the largest score of a token is at least 1/2, however small it is itself, and so is the sum that the weights are divided by; without that division `largest` is the row's, or 0.  A sigmoid
// below e^-700 counts as 0: a row whose logits are all the lowest finite value gets no weights.
constexpr float kLowestLogit = -700.0f;
__device__ __forceinline__ float score_of(float l, float largest, bool sigmoid) {
  if (!sigmoid) return exp_below(l - largest);
  const float s = exp_below(fminf(l, 0.0f) - fminf(largest, 0.0f)) * __builtin_amdgcn_rcpf(1.0f + exp_of(-fabsf(l)));
  return l < kLowestLogit ? 0.0f : s;
}
// Integers in the order of numbers above -inf, and back; -inf and NaN: none.
__device__ __forceinline__ int key_of(float v) {
  const int b = __float_as_int(v);
  return v > -__builtin_inff() ? b ^ ((b >> 31) & 0x7fffffff) : kNone;
}
__device__ __forceinline__ float value_of(int key) { return __int_as_float(key ^ ((key >> 31) & 0x7fffffff)); }
// Over the LPT lanes of a token, in each of them.
struct IMax {
  __device__ __forceinline__ static int of(int a, int b) { return max(a, b); }
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
  if (LPT == 32) return v;
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return OP::of((int)b[0], (int)b[1]);
}
template <int LPT, class OP>
__device__ __forceinline__ float all_float(float v) { return LPT == 16 ? row16_all<OP>(v) : LPT == 32 ? half_all<OP>(v) : wave_all<OP>(v); }

// What a lane has of a token's logits: experts e0 .. e0 + V - 1, -inf beyond the last.
template <int XT, int LPT, int V, bool SHORT>
struct Logits {
  float l[V];
  int e0;
  __device__ __forceinline__ Logits(const RouteArgs& a, const void* row, int lane) {
    e0 = lane * V;
    if constexpr (V < 8) {
      Run8<XT> r[V];
#pragma unroll
      for (int v = 0; v < V; ++v) r[v].load_part((const typename Run8<XT>::Elem*)row + min(e0 + v, a.E - 1), 1);
#pragma unroll
      for (int v = 0; v < V; ++v) l[v] = e0 + v < a.E ? as_logit(r[v].get(0)) : -__builtin_inff();
    } else {
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
  }
  __device__ __forceinline__ float top() const {                   // the row's largest, 0 if there is none
    float m = l[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, l[v]);
    m = all_float<LPT, Max>(m);
    return m > -__builtin_inff() ? m : 0.0f;
  }
};

// Sums over lanes. The shifts are operands of the additions (DPP): within a row of 16 lanes, then from the last lane of a row to the next one, of the first two rows to the others.
template <int CTRL, int ROWS>
__device__ __forceinline__ int plus_from(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int sums_up_to(int v) {                 // of this lane and those before it
  v = plus_from<0x111, 0xf>(v);                                    // row_shr 1, 2, 4, 8
  v = plus_from<0x112, 0xf>(v);
  v = plus_from<0x114, 0xf>(v);
  v = plus_from<0x118, 0xf>(v);
  v = plus_from<0x142, 0xa>(v);                                    // row_bcast 15 to rows 1 and 3
  return plus_from<0x143, 0xc>(v);                                 // row_bcast 31 to rows 2 and 3
}
// of the lanes that are the same mod N (1, 2, 4, ...), in each of them
template <int N>
__device__ __forceinline__ int sums_mod(int v) {
  if (N <= 1) v += dpp<0x121>(v);                                  // row_ror 1, 2, 4, 8
  if (N <= 2) v += dpp<0x122>(v);
  if (N <= 4) v += dpp<0x124>(v);
  if (N <= 8) v += dpp<0x128>(v);
  if (N <= 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = (int)a[0] + (int)a[1];
  }
  if (N <= 32) {
    const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = (int)a[0] + (int)a[1];
  }
  return v;
}
// Exclusive sums of n <= 1024 numbers in LDS, by one wave; the last lane's return value is the sum of all.
__device__ __forceinline__ int scan_in_place(int* x, int n) {
  const int lane = threadIdx.x & 63, per = (n + 63) / 64, first = lane * per;
  int s = 0;
  for (int i = first; i < first + per && i < n; ++i) s += x[i];
  const int all = sums_up_to(s);
  int before = all - s;
  for (int i = first; i < first + per && i < n; ++i) {
    const int c = x[i];
    x[i] = before;
    before += c;
  }
  return all;
}

// LDS: masks and running counts, the choices of 64 tokens with what they were chosen by, and for each token at work its logits (with a bias) and what its groups need.
struct RouteLds {
  int run, chosen, tokens, token_words;                            // byte offsets; words of a token
  __host__ __device__ RouteLds(const RouteArgs& a, int lanes_experts, bool logits, bool groups) {
    run = a.E * 8;
    chosen = (run + a.E * 4 + 7) / 8 * 8;
    tokens = (chosen + kMaskTokens * a.k * 8 + 15) / 16 * 16;
    token_words = (logits ? 0 : lanes_experts) + (groups ? lanes_experts + 2 * a.groups : 0);
    token_words = (token_words + 3) / 4 * 4;
  }
};
// Lanes of a token see each other's LDS: they are of one wave.
__device__ __forceinline__ void token_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The two largest of what lanes D apart have (first >= second).
template <int D>
__device__ __forceinline__ void join_two(float& first, float& second) {
  float f, s;
  if constexpr (D >= 16) {
    const auto a = D == 16 ? __builtin_amdgcn_permlane16_swap(__float_as_int(first), __float_as_int(first), false, false)
                           : __builtin_amdgcn_permlane32_swap(__float_as_int(first), __float_as_int(first), false, false);
    const auto b = D == 16 ? __builtin_amdgcn_permlane16_swap(__float_as_int(second), __float_as_int(second), false, false)
                           : __builtin_amdgcn_permlane32_swap(__float_as_int(second), __float_as_int(second), false, false);
    first = __int_as_float(a[0]), f = __int_as_float(a[1]), second = __int_as_float(b[0]), s = __int_as_float(b[1]);
  } else {
    constexpr int CTRL = D == 1 ? kXor1 : D == 2 ? kXor2 : D == 4 ? kHalfMirror : kMirror;
    f = __int_as_float(dpp<CTRL>(__float_as_int(first))), s = __int_as_float(dpp<CTRL>(__float_as_int(second)));
  }
  second = fmaxf(fminf(first, f), fmaxf(second, s));
  first = fmaxf(first, f);
}

// Strikes out the experts of the groups that do not stay.  by: what the lane's experts' groups are judged by (-inf: masked).  Groups of 1, 2, 4, ... whole lanes are judged in
// registers (kWholeLanes), others through LDS.  (Kernels of their own: what the compiler prepares for the one costs the other registers and a microsecond.)
constexpr int kNoGroups = 0, kWholeLanes = 1, kAnyGroups = 2;
template <int LPT, int V, int GROUPS>
__device__ __forceinline__ void keep_groups(const RouteArgs& a, int lane, int e0, const float (&by)[V], int (&key)[V], float* mine) {
  const int per = a.per;
  const float none = -__builtin_inff();
  if constexpr (GROUPS == kWholeLanes) {
    const int lanes = per / V;                                     // of a group
    float first = none, second = none;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      second = fmaxf(second, fminf(first, by[v]));
      first = fmaxf(first, by[v]);
    }
    if (lanes > 1) join_two<1>(first, second);
    if (lanes > 2) join_two<2>(first, second);
    if (lanes > 4) join_two<4>(first, second);
    if (lanes > 8) join_two<8>(first, second);
    if (LPT > 16 && lanes > 16) join_two<16>(first, second);
    const float score = a.top2 && second > none ? first + second : first;
    const int g = lane >> (31 - __builtin_clz(lanes));
    int better = 0;
    for (int o = 0; o < a.groups; o += 4)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // (beyond the last group: not counted)
        const float s = LPT == 64 ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(score), (o + i) * lanes & 63)) : __shfl(score, (o + i) * lanes, LPT);
        better += o + i < a.groups && (s > score || (s == score && o + i < g));
      }
    if (better >= a.kept)
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = kNone;
    return;
  }
  float* score = mine + LPT * V;
  int* keep = (int*)(score + a.groups);
  token_sync();                                                    // (the token before has been read)
#pragma unroll
  for (int v = 0; v < V; ++v) mine[e0 + v] = by[v];                // (room for all lanes' experts, those that are none too)
  token_sync();
  for (int g = lane; g < a.groups; g += LPT) {
    float first = none, second = none;
    int i = g % per;                                               // (started apart: neighbouring lanes on neighbouring banks)
#pragma unroll 8
    for (int n = 0; n < per; ++n, i = i + 1 == per ? 0 : i + 1) {
      const float c = mine[g * per + i];
      second = fmaxf(second, fminf(first, c));
      first = fmaxf(first, c);
    }
    score[g] = a.top2 && second > none ? first + second : first;
  }
  token_sync();
  for (int g = lane; g < a.groups; g += LPT) {
    const float s = score[g];
    int better = 0;
#pragma unroll 8
    for (int o = 0; o < a.groups; ++o) better += score[o] > s || (score[o] == s && o < g);
    keep[g] = better < a.kept;
  }
  token_sync();
  int g = min(e0, a.E - 1) / per, left = (g + 1) * per - e0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (e0 + v < a.E && !keep[g]) key[v] = kNone;
    if (--left == 0) ++g, left = per;
  }
}

// A lane's experts by descending key, equal ones by index, as lists of up to eight: neighbours change places only where the right one is larger, which keeps
// the order of equals.  place: four bits for each, where it came from.
template <int V>
struct Lists {
  static constexpr int W = V < 8 ? V : 8, N = V / W;
  int key[N][W];
  uint32_t place[N];
  __device__ __forceinline__ explicit Lists(const int (&k)[V]) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      int at[W];
#pragma unroll
      for (int v = 0; v < W; ++v) at[v] = v, key[n][v] = k[n * W + v];
#pragma unroll
      for (int round = 0; round < W; ++round)
#pragma unroll
        for (int v = round & 1; v + 1 < W; v += 2) {
          const int swap = key[n][v + 1] > key[n][v] ? at[v] ^ at[v + 1] : 0;     // (a choice between at[v] and at[v + 1] becomes one between all of them)
          const int hi = max(key[n][v], key[n][v + 1]), lo = min(key[n][v], key[n][v + 1]);
          key[n][v] = hi, key[n][v + 1] = lo, at[v] ^= swap, at[v + 1] ^= swap;
        }
      place[n] = 0;
#pragma unroll
      for (int v = 0; v < W; ++v) place[n] |= (uint32_t)at[v] << 4 * v;
    }
  }
  __device__ __forceinline__ int first() const { return N == 1 ? key[0][0] : max(key[0][0], key[N - 1][0]); }
  // which of the lane's experts the first one is (a key of the lane's largest), and the lists without it
  __device__ __forceinline__ int index() const {
    return N == 1 || key[0][0] >= key[N - 1][0] ? (int)(place[0] & 15) : W + (int)(place[N - 1] & 15);
  }
  __device__ __forceinline__ void drop(bool mine) {
    const bool right = N > 1 && key[N - 1][0] > key[0][0];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const bool up = mine && right == (n > 0);
#pragma unroll
      for (int v = 0; v + 1 < W; ++v) key[n][v] = up ? key[n][v + 1] : key[n][v];
      key[n][W - 1] = up ? kNone : key[n][W - 1];
      place[n] = up ? place[n] >> 4 : place[n];
    }
  }
};

// Which lane of a token has the first of its experts with this property (64: none).
template <int LPT>
__device__ __forceinline__ int first_lane(bool mine) {
  const uint64_t all = __ballot(mine);
  if (LPT == 64) return all ? __builtin_ctzll(all) : 64;
  const uint32_t half = threadIdx.x & 32 ? (uint32_t)(all >> 32) : (uint32_t)all;
  if (LPT == 32) return half ? __builtin_ctz(half) : 64;
  const uint32_t row = threadIdx.x & 16 ? half >> 16 : half & 0xffff;
  return row ? __builtin_ctz(row) : 64;
}

// LOGITS: without a bias, chosen by the logits themselves (both scores grow with them, but in fp32 not all of them: sigmoids of 18 and 19 are one number).  tokens: of a workgroup.  With the order: places inside the block to row_of and the block's counts to the
// workspace, or, alone, the whole order.
template <int XT, int LPT, int V, bool LOGITS, int GROUPS, bool SHORT>
__global__ __launch_bounds__(1024) void route_kernel(RouteArgs a, int tokens, bool alone, int counts_pitch) {
  fetch_arguments(a.logits, a.T, a.scale);
  extern __shared__ __align__(16) char mem[];
  const RouteLds at(a, LPT * V, LOGITS, GROUPS == kAnyGroups);
  uint64_t* mask = (uint64_t*)mem;
  int* run = (int*)(mem + at.run);                                 // the expert's pairs in the block's tokens before these
  int2* chosen = (int2*)(mem + at.chosen);                         // expert (-1: none) and what it was chosen by
  float* own_logits = (float*)(mem + at.tokens) + threadIdx.x / LPT * at.token_words;
  float* by_group = own_logits + (LOGITS ? 0 : LPT * V);
  const int tid = threadIdx.x, threads = blockDim.x, lane = tid % LPT;
  const int64_t b0 = (int64_t)blockIdx.x * tokens, b1 = b0 + tokens < a.T ? b0 + tokens : a.T;
  const bool order = a.row_of != nullptr;
  const float none = -__builtin_inff();
  if (order)
    for (int e = tid; e < a.E; e += threads) run[e] = 0;
  for (int64_t s0 = b0; s0 < b1; s0 += kMaskTokens) {
    const int n = (int)(b1 - s0 < kMaskTokens ? b1 - s0 : kMaskTokens);
    if (order)
      for (int e = tid; e < a.E; e += threads) mask[e] = 0;
    for (int i = tid / LPT; i < n; i += threads / LPT) {
      const int64_t t = s0 + i;
      float bias[LOGITS ? 1 : V];
      if constexpr (!LOGITS) {
#pragma unroll
        for (int v = 0; v < V; ++v) bias[v] = a.bias[min(lane * V + v, a.E - 1)];
      }
      const Logits<XT, LPT, V, SHORT> x(a, elem_at(a.logits, t * a.ld, elem_bytes(XT)), lane);
      // softmax: the row's largest, and the sum of exp behind it, where more than the chosen ones' own matter
      float m = 0, total = 1.0f;
      if (!a.sigmoid && (!LOGITS || !a.renorm || (GROUPS && a.top2))) m = x.top();
      int key[V];
      if constexpr (LOGITS) {
        if (!a.sigmoid && !a.renorm) {
          total = 0;
#pragma unroll
          for (int v = 0; v < V; ++v) total += exp_of(x.l[v] - m);
          total = all_float<LPT, Add>(total);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = key_of(x.l[v]);
        if (GROUPS) {
          float by[V];                                             // (sums of scores up to a common factor)
#pragma unroll
          for (int v = 0; v < V; ++v) by[v] = key[v] == kNone ? none : !a.top2 ? x.l[v] : a.sigmoid ? sigmoid(x.l[v]) : exp_of(x.l[v] - m);
          keep_groups<LPT, V, GROUPS>(a, lane, x.e0, by, key, by_group);
        }
      } else {
        float s[V];
        if (a.sigmoid) {
#pragma unroll
          for (int v = 0; v < V; ++v) s[v] = sigmoid(x.l[v]);
        } else {
          total = 0;
#pragma unroll
          for (int v = 0; v < V; ++v) total += s[v] = exp_of(x.l[v] - m);
          total = all_float<LPT, Add>(total);
          const float inv = total > 0 ? 1.0f / total : 0.0f;
#pragma unroll
          for (int v = 0; v < V; ++v) s[v] *= inv;
        }
        token_sync();                                              // (the token before has read its own)
#pragma unroll
        for (int v = 0; v < V; ++v) own_logits[x.e0 + v] = x.l[v]; // (the chosen ones' are read back there)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          s[v] += bias[v];
          s[v] = x.l[v] > none && s[v] > none ? s[v] + 0.0f : none;  // (NaN compares false)
          key[v] = key_of(s[v]);
        }
        if (GROUPS) keep_groups<LPT, V, GROUPS>(a, lane, x.e0, s, key, by_group);
      }
      // k times the largest of the lanes' first ones; of lanes that have it, the first; that lane notes the choice down
      Lists<V> list(key);
      for (int j = 0; j < a.k; ++j) {
        const int first = list.first(), best = all_int<LPT, IMax>(first);
        const bool mine = lane == first_lane<LPT>(first == best);
        if (mine) chosen[i * a.k + j] = int2{best == kNone ? -1 : x.e0 + list.index(), best};
        list.drop(mine);
      }
      token_sync();
      // lane j: choice j and its weight (without a bias the key is its logit)
      const int2 mine = lane < a.k ? chosen[i * a.k + lane] : int2{-1, kNone};
      const int id = mine.x, by = mine.y;
      const float l = LOGITS ? value_of(by) : id >= 0 ? own_logits[id] : none;
      if (a.renorm) m = LOGITS ? value_of(all_int<LPT, IMax>(by)) : all_float<LPT, Max>(l);         // (no choice: not a number, or none, and not used)
      float w = id >= 0 ? score_of(l, m, a.sigmoid) : 0.0f;
      if (a.renorm) total = all_float<LPT, Add>(w);
      w = total > 0 ? a.scale * (w / total) : 0.0f;
      if (lane < a.k) {
        a.ids[t * a.k + lane] = id;
        a.weights[t * a.k + lane] = w;
      }
    }
    if (!order) continue;
    lds_barrier();
    for (int p = tid; p < n * a.k; p += threads) {
      const int e = chosen[p].x;
      if (e >= 0) atomicOr((unsigned long long*)&mask[e], 1ull << (p / a.k));
    }
    lds_barrier();
    if (alone) {                                                   // (one mask: run becomes where the expert's rows begin)
      for (int e = tid; e < a.E; e += threads) run[e] = __popcll(mask[e]);
      lds_barrier();
      if (tid < 64) {
        const int all = scan_in_place(run, a.E);
        if (tid == 63) a.group_rows[a.E] = all;
      }
      lds_barrier();
      for (int e = tid; e < a.E; e += threads) a.group_rows[e] = run[e];
    }
    for (int p = tid; p < n * a.k; p += threads) {
      const int e = chosen[p].x;
      const int i = p / a.k;
      a.row_of[s0 * a.k + p] = e < 0 ? -1 : run[e] + __popcll(mask[e] & ((1ull << i) - 1));
    }
    if (alone) return;
    lds_barrier();
    for (int e = tid; e < a.E; e += threads) run[e] += __popcll(mask[e]);   // (its own mask and count: the next tokens' mask may be cleared at once)
  }
  if (!order) return;
  uint16_t* counts = (uint16_t*)a.ws + (int64_t)blockIdx.x * counts_pitch;
  for (int e = tid; e < counts_pitch; e += threads) counts[e] = e < a.E ? (uint16_t)run[e] : 0;
}

// Places inside the blocks to places of all.  The workspace: for each block the counts of RUNS runs of eight experts.
template <int RUNS>
__global__ __launch_bounds__(1024) void route_order_kernel(RouteArgs a, int tokens, int blocks) {
  constexpr int pitch = 8 * RUNS;
  __shared__ int sum[2][pitch], total[pitch], before[pitch];
  fetch_arguments(a.logits, a.T, a.scale);
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t p0 = (int64_t)blockIdx.x * tokens * a.k, end = a.T * a.k, p1 = p0 + (int64_t)tokens * a.k < end ? p0 + (int64_t)tokens * a.k : end;
  int first_id = -1, first_row = 0;                                // (on their way while the counts are added up)
  if (p0 + tid < p1) first_id = a.ids[p0 + tid], first_row = a.row_of[p0 + tid];
  for (int e = tid; e < pitch; e += 1024) sum[0][e] = sum[1][e] = 0;
  lds_barrier();
  int all[8] = {}, upto[8] = {};
  const int c = tid & (RUNS - 1);                                  // a thread: eight experts of every (1024 / RUNS)-th block
#pragma unroll 4
  for (int b = tid / RUNS; b < blocks; b += 1024 / RUNS) {
    const u32x4 v = load_bits<u32x4>((const uint16_t*)a.ws + (int64_t)b * pitch + c * 8);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int lo = v[i] & 0xffff, hi = v[i] >> 16;
      all[2 * i] += lo, all[2 * i + 1] += hi;
      if (b < (int)blockIdx.x) upto[2 * i] += lo, upto[2 * i + 1] += hi;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) all[i] = sums_mod<RUNS>(all[i]), upto[i] = sums_mod<RUNS>(upto[i]);
  if (lane < RUNS)                                                 // (integers: any order, one sum; lanes side by side in LDS: expert 8 c + i at i * RUNS + c)
#pragma unroll
    for (int i = 0; i < 8; ++i) atomicAdd(&sum[0][i * RUNS + c], all[i]), atomicAdd(&sum[1][i * RUNS + c], upto[i]);
  lds_barrier();
  for (int e = tid; e < pitch; e += 1024) total[e] = sum[0][(e & 7) * RUNS + (e >> 3)], before[e] = sum[1][(e & 7) * RUNS + (e >> 3)];
  lds_barrier();
  if (tid < 64) {
    const int n = scan_in_place(total, a.E);
    if (tid == 63 && blockIdx.x == 0) a.group_rows[a.E] = n;
  }
  lds_barrier();
  if (blockIdx.x == 0)
    for (int e = tid; e < a.E; e += 1024) a.group_rows[e] = total[e];
  for (int64_t p = p0 + tid; p < p1; p += 1024) {
    const int e = p == p0 + tid ? first_id : a.ids[p];
    if (e >= 0) a.row_of[p] = (p == p0 + tid ? first_row : a.row_of[p]) + total[e] + before[e];
  }
}
__global__ __launch_bounds__(1024) void route_no_tokens_kernel(int32_t* group_rows, int E) {
  for (int e = threadIdx.x; e <= E; e += 1024) group_rows[e] = 0;
}

// Gradient of the logits; lanes as above.
template <int XT, int LPT, int V, bool SHORT>
__global__ __launch_bounds__(256) void route_backward_kernel(RouteArgs a) {
  fetch_arguments(a.logits, a.T, a.scale);
  const int lane = threadIdx.x % LPT;
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPT;
  if (t >= a.T) return;                                            // (all lanes of a token)
  const void* row = elem_at(a.logits, t * a.ld, elem_bytes(XT));
  const Logits<XT, LPT, V, SHORT> x(a, row, lane);
  int id = lane < a.k ? a.ids_in[t * a.k + lane] : -1;
  if (id >= a.E) id = -1;
  float g = id >= 0 ? a.dweights[t * a.k + lane] * a.scale : 0.0f;
  float l = -__builtin_inff();                                     // of choice `lane`
  if (id >= 0) {
    Run8<XT> one;
    one.load_part((const typename Run8<XT>::Elem*)row + id, 1);
    l = as_logit(one.get(0));
  }
  // The gradient is f_e (ds_e - along); ds: what the choices bring to their experts.
  float f[V], along = 0;
  if (a.renorm) {
    // w_e (g_e - sum w g), for a sigmoid times 1 - s_e: of the weights, which are ordinary numbers however small the scores and their sum are
    const float largest = all_float<LPT, Max>(l);
    const float sc = l > -__builtin_inff() ? score_of(l, largest, a.sigmoid) : 0.0f;
    const float total = all_float<LPT, Add>(sc), w = total > 0 ? sc / total : 0.0f;
    g = w * (g - all_float<LPT, Add>(g * w));
    if (a.sigmoid) g *= sigmoid(-l);
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = 1.0f;
  } else if (a.sigmoid) {
    // s (1 - s) = e / (1 + e)^2, e = exp(-|l|): without the difference, of which nothing is left from 17 on
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float e = exp_of(-fabsf(x.l[v])), r = __builtin_amdgcn_rcpf(1.0f + e);
      f[v] = e * r * r;
    }
  } else {
    const float m = x.top();
    float total = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) total += f[v] = exp_of(x.l[v] - m);
    total = all_float<LPT, Add>(total);
    const float inv = total > 0 ? 1.0f / total : 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] *= inv;
    along = all_float<LPT, Add>(id >= 0 ? g * (exp_of(l - m) * inv) : 0.0f);
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
  for (int i = 0; i < (V + 7) / 8; ++i) {
    float d[8] = {};
#pragma unroll
    for (int k = 0; k < 8 && k < V; ++k) {
      const int v = 8 * i + k;
      d[k] = x.l[v] == -__builtin_inff() ? 0.0f : f[v] * (ds[v] - along);
    }
    Run8<XT> r;
    r.set(d);
    if (V < 8) {
      if (x.e0 < a.E) r.store_part((typename Run8<XT>::Elem*)out + x.e0, min(V, a.E - x.e0));
    } else {
      store_run(r, out, x.e0 + 8 * i, a.E);
    }
  }
}

template <int RUNS>
void launch_order(const RouteArgs& a, int tokens, int blocks, int pitch, hipStream_t s) {
  if (pitch == 8 * RUNS) route_order_kernel<RUNS><<<blocks, 1024, 0, s>>>(a, tokens, blocks);
  else if constexpr (8 * RUNS < kRouteMaxE) launch_order<2 * RUNS>(a, tokens, blocks, pitch, s);
}

template <int XT>
void launch_route_of(const RouteArgs& a, hipStream_t s) {
  by_route_shape(few_tokens(a.T), a.E, a.k, [&](auto shape) {
    using S = decltype(shape);
    const bool alone = one_workgroup(a.T, a.E, a.k);
    const int tokens = alone ? kMaskTokens : block_tokens(a.T), pitch = counts_pitch(a.E), blocks = (int)((a.T + tokens - 1) / tokens);
    const int here = (int)(a.T < tokens ? a.T : tokens);
    auto launch = [&](auto logits, auto groups) {
      constexpr bool L = decltype(logits)::value;
      constexpr int G = decltype(groups)::value;
      const RouteLds lds(a, S::LPT * S::V, L, G == kAnyGroups);
      // tokens at once: all of a mask's, as far as threads and LDS go
      int n = std::min(1024, (std::min(here, kMaskTokens) * S::LPT + 63) / 64 * 64);
      while (n > 64 && lds.tokens + n / S::LPT * lds.token_words * 4 > 65536) n = (n / 2 + 63) / 64 * 64;
      route_kernel<XT, S::LPT, S::V, L, G, S::SHORT><<<blocks, n, lds.tokens + n / S::LPT * lds.token_words * 4, s>>>(a, tokens, alone, pitch);
    };
    auto by_groups = [&](auto logits) {
      const int lanes = a.per / S::V;
      if (a.groups == 1) launch(logits, std::integral_constant<int, kNoGroups>());
      else if (!S::SHORT && a.per == lanes * S::V && (lanes & (lanes - 1)) == 0) launch(logits, std::integral_constant<int, S::SHORT ? kAnyGroups : kWholeLanes>());
      else launch(logits, std::integral_constant<int, kAnyGroups>());
    };
    if (!a.bias) by_groups(std::true_type());
    else by_groups(std::false_type());
    if (a.row_of && !alone) launch_order<1>(a, tokens, blocks, pitch, s);
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
  by_route_shape(all.T <= 8192, all.E, all.k, [&](auto shape) {
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
