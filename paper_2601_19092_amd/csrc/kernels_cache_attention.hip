// Attention over a paged cache: launches, wide tiles, and the kernel that joins partial results (cache_attention.h).
#include <hip/hip_runtime.h>

#include "cache_attention.h"

namespace axe {

// Partial results of one tile: those of the workgroup that began it, then of the workgroups behind it up to the one that ended it.  A wave joins RB rows at once; LANES lanes
// have four columns each of a part's row and take every 64 / LANES-th part, DEPTH of them with their maxima and sums under way together.
template <int TYPE, int DP>
struct Join {
  static constexpr int LANES = DP / 4, AT_ONCE = 64 / LANES;
  const CacheArgs& a;
  int group, n, token, kv_head, rows;                              // n parts
  const int lane = threadIdx.x & 63;

  template <int RB, int DEPTH>
  __device__ __forceinline__ void run(int first, int step) const {
    const int c = lane % LANES * 4;
    for (int r0 = first; r0 < rows; r0 += RB * step) {
      float top[RB], l[RB];
      f32x4 o[RB];
      int row[RB];
#pragma unroll
      for (int i = 0; i < RB; ++i) top[i] = -INFINITY, l[i] = 0, o[i] = f32x4{}, row[i] = r0 + i * step < rows ? r0 + i * step : rows - 1;
      for (int j0 = lane / LANES; j0 < n; j0 += AT_ONCE * DEPTH) {
        float pm[RB][DEPTH], pl[RB][DEPTH];
        f32x4 v[RB][DEPTH];
#pragma unroll
        for (int k = 0; k < DEPTH; ++k) {
          const int j = j0 + k * AT_ONCE, at = j < n ? j : n - 1;
          const float* p = a.ws + part_at(a, group + at, at == 0, DP) + 4;
#pragma unroll
          for (int i = 0; i < RB; ++i) {
            pm[i][k] = j < n ? p[row[i]] : -INFINITY, pl[i][k] = p[a.ws_rows + row[i]];
            v[i][k] = *(const f32x4*)(p + 2 * a.ws_rows + (int64_t)row[i] * DP + c);
          }
        }
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int k = 0; k < DEPTH; ++k) {
            const bool there = j0 + k * AT_ONCE < n;
            add(top[i], l[i], o[i], pm[i][k], there ? pl[i][k] : 0.0f, there ? v[i][k] : f32x4{});
          }
      }
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        if constexpr (AT_ONCE >= 4) other<16>(top[i], l[i], o[i]);
        if constexpr (AT_ONCE >= 2) other<32>(top[i], l[i], o[i]);
        const float by = l[i] == 0 ? 0.0f : 1.0f / l[i];
        const int t = (int)quotient(row[i], a.group), g = row[i] - t * (int)a.group.d;
        uint16_t* to = (uint16_t*)a.out + (int64_t)(token + t) * a.os.token + (int64_t)(kv_head * (int)a.group.d + g) * a.os.head + c;
        if (lane < LANES && c < a.D && r0 + i * step < rows) store_bits(to, u32x2{pack2<TYPE>(o[i][0] * by, o[i][1] * by), pack2<TYPE>(o[i][2] * by, o[i][3] * by)});
      }
    }
  }
  // Two results of one row.  (A maximum of -inf: no key was seen, and the rest is 0, or none of the scores was a number, and it is NaN, which stays.)
  static __device__ __forceinline__ void add(float& top, float& l, f32x4& o, float pm, float pl, f32x4 v) {
    const float t = fmaxf(top, pm), base = t == -INFINITY ? 0.0f : t, old = exp2_fast(top - base), by = exp2_fast(pm - base);
    top = t, l = l * old + pl * by, o = o * old + v * by;
  }
  template <int FAR>
  static __device__ __forceinline__ void other(float& top, float& l, f32x4& o) {
    auto far = [&](float x) __attribute__((always_inline)) { return __shfl_xor(x, FAR); };
    const float pm = far(top), pl = far(l);
    const f32x4 v = {far(o[0]), far(o[1]), far(o[2]), far(o[3])};
    add(top, l, o, pm, pl, v);
  }
};

template <int TYPE, int DP>
__global__ __launch_bounds__(256) void cache_attention_join_kernel(CacheArgs a) {
  const int group = blockIdx.x, lane = threadIdx.x & 63;
  const uint32_t* head = (const uint32_t*)(a.ws + part_at(a, group, 1, DP));
  const uint32_t begun = head[0];
  int n = 1;
  for (int g = group + 1;; g += 64) {                              // parts behind the first: up to the one that ends the tile
    const uint32_t flags = g + lane < a.groups ? *(const uint32_t*)(a.ws + part_at(a, g + lane, 0, DP)) : 0;
    const uint64_t none = __ballot(flags == 0), end = __ballot((flags & 2) != 0);
    const int until = none ? __ffsll((unsigned long long)none) - 1 : 64, last = end ? __ffsll((unsigned long long)end) : 64;
    n += until < last ? until : last;
    if (none || end) break;
  }
  if (!begun) return;
  const Join<TYPE, DP> join{a, group, n, (int)head[1], (int)head[2], (int)head[3]};
  const int first = blockIdx.y * 4 + (int)(threadIdx.x >> 6), step = gridDim.y * 4;
  constexpr int AT_ONCE = Join<TYPE, DP>::AT_ONCE;
  if (join.rows <= 16) join.template run<1, 8>(first, step);
  else if (n <= AT_ONCE) join.template run<4, 1>(first, step);
  else if (n <= 2 * AT_ONCE) join.template run<4, 2>(first, step);
  else join.template run<4, 4>(first, step);
}

template <int TYPE>
void launch_join(const CacheArgs& a, hipStream_t s) {
  const int dp = attn_columns(a.D);
  const dim3 grid(a.groups, a.ws_rows <= 32 ? 4 : 8);
  if (dp == 64) cache_attention_join_kernel<TYPE, 64><<<grid, 256, 0, s>>>(a);
  else if (dp == 128) cache_attention_join_kernel<TYPE, 128><<<grid, 256, 0, s>>>(a);
  else cache_attention_join_kernel<TYPE, 256><<<grid, 256, 0, s>>>(a);
}

hipError_t launch_cache_attention(const CacheArgs& a, hipStream_t s) {
  if (a.groups) {
    if (a.tile_rows == 16) launch_attention_narrow<1>(a, a.groups, s);
    else if (a.tile_rows == 32) launch_attention_narrow<2>(a, a.groups, s);
    else launch_attention<0, true>(a, a.groups, s);
    a.type == kBf16 ? launch_join<kBf16>(a, s) : launch_join<kF16>(a, s);
    return hipGetLastError();
  }
  const int tokens = a.tile_rows / (int)a.group.d;
  const int64_t tiles = (a.T / tokens + (a.S < a.T || a.S > 64 ? a.S : a.T)) * a.kv_heads;   // as many as there can be; places, where there are more than 64 sequences
  constexpr int64_t kPiece = int64_t(1) << 23;                     // (a launch holds fewer than 2^32 threads)
  CacheArgs piece = a;
  for (piece.t0 = 0; piece.t0 < tiles; piece.t0 += kPiece) {
    const uint32_t n = (uint32_t)(tiles - piece.t0 < kPiece ? tiles - piece.t0 : kPiece);
    if (a.tile_rows == 16) launch_attention_narrow<1>(piece, n, s);
    else if (a.tile_rows == 32) launch_attention_narrow<2>(piece, n, s);
    else launch_attention<0, false>(piece, n, s);
  }
  return hipGetLastError();
}

}  // namespace axe
