// Attention over a paged cache: launches, wide tiles, and the kernel that joins partial results (cache_attention.h).
#include <hip/hip_runtime.h>

#include "cache_attention.h"

namespace axe {

// Partial results of one tile: the workgroup that began it, then the workgroups behind it up to the one that ended it.  A wave joins a row: a lane a part for the maxima and sums, then
// LANES lanes a part for the row itself, the parts' weights on the way, so that as many loads as possible are under way at once.
template <int TYPE, int DP>
__global__ __launch_bounds__(256) void cache_attention_join_kernel(CacheArgs a) {
  constexpr int LANES = DP / 4, AT_ONCE = 64 / LANES, DEPTH = 8;   // a lane has four columns
  const int group = blockIdx.x, lane = threadIdx.x & 63;
  const uint32_t* head = (const uint32_t*)(a.ws + part_at(a, group, 1, DP));
  const uint32_t valid = head[0];
  const int token = (int)head[1], kv_head = (int)head[2], rows = (int)head[3];
  int parts = 0;                                                   // behind the first
  for (int g = group + 1; parts == g - group - 1; g += 64) {
    const uint32_t flags = g + lane < a.groups ? *(const uint32_t*)(a.ws + part_at(a, g + lane, 0, DP)) : 0;
    const uint64_t none = __ballot(flags == 0), end = __ballot((flags & 2) != 0);
    const int until = none ? __ffsll((unsigned long long)none) - 1 : 64, last = end ? __ffsll((unsigned long long)end) : 64;
    parts += until < last ? until : last;
    if (until < 64 || last <= 64 && end) break;
  }
  if (!valid) return;
  const int n = parts + 1;
  auto part = [&](int i) __attribute__((always_inline)) { return a.ws + part_at(a, group + i, i == 0, DP); };
  for (int r = blockIdx.y * 4 + (int)(threadIdx.x >> 6); r < rows; r += gridDim.y * 4) {
    float top = -INFINITY;
    for (int i = lane; i < n; i += 64) top = fmaxf(top, part(i)[4 + r]);
    top = wave_all<Max>(top);
    const float base = top == -INFINITY ? 0.0f : top;
    float l = 0;
    f32x4 o = {0, 0, 0, 0};
    for (int i0 = 0; i0 < n; i0 += 64) {
      const int mine = i0 + lane;
      float by = 0;
      if (mine < n) {
        by = exp2_fast(part(mine)[4 + r] - base);
        l += part(mine)[4 + a.ws_rows + r] * by;
      }
      const int many = n - i0 < 64 ? n - i0 : 64;
      for (int j0 = 0; j0 < many; j0 += AT_ONCE * DEPTH) {
        f32x4 v[DEPTH];
#pragma unroll
        for (int k = 0; k < DEPTH; ++k) {
          const int j = j0 + k * AT_ONCE + lane / LANES;
          v[k] = *(const f32x4*)(part(i0 + (j < many ? j : many - 1)) + 4 + 2 * a.ws_rows + (int64_t)r * DP + lane % LANES * 4);
        }
#pragma unroll
        for (int k = 0; k < DEPTH; ++k) {
          const int j = j0 + k * AT_ONCE + lane / LANES;
          const float w = __shfl(by, j & 63);
          if (j < many) o += v[k] * w;
        }
      }
    }
    l = wave_sum(l);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if constexpr (AT_ONCE >= 2) o[c] += other_half(o[c]);
      if constexpr (AT_ONCE >= 4) {
        const auto x = __builtin_amdgcn_permlane16_swap(__float_as_int(o[c]), __float_as_int(o[c]), false, false);
        o[c] = __int_as_float(x[0]) + __int_as_float(x[1]);
      }
    }
    const float by = l == 0 ? 0.0f : 1.0f / l;
    const int i = (int)quotient(r, a.group), g = r - i * (int)a.group.d, c = lane % LANES * 4;
    uint16_t* to = (uint16_t*)a.out + (int64_t)(token + i) * a.os.token + (int64_t)(kv_head * (int)a.group.d + g) * a.os.head + c;
    if (lane < LANES && c < a.D) store_bits(to, u32x2{pack2<TYPE>(o[0] * by, o[1] * by), pack2<TYPE>(o[2] * by, o[3] * by)});
  }
}

template <int TYPE>
void launch_join(const CacheArgs& a, hipStream_t s) {
  const int dp = attn_columns(a.D);
  const dim3 grid(a.groups, a.ws_rows <= 32 ? 4 : 16);
  if (dp == 64) cache_attention_join_kernel<TYPE, 64><<<grid, 256, 0, s>>>(a);
  else if (dp == 128) cache_attention_join_kernel<TYPE, 128><<<grid, 256, 0, s>>>(a);
  else cache_attention_join_kernel<TYPE, 256><<<grid, 256, 0, s>>>(a);
}

hipError_t launch_cache_attention(const CacheArgs& a, hipStream_t s) {
  if (a.groups) {
    if (a.tile_rows == 16) launch_attention_narrow<1>(a, s);
    else if (a.tile_rows == 32) launch_attention_narrow<2>(a, s);
    else launch_attention<0, true>(a, a.groups, s);
    a.type == kBf16 ? launch_join<kBf16>(a, s) : launch_join<kF16>(a, s);
    return hipGetLastError();
  }
  const int tokens = kAttnRows / (int)a.group.d;
  const int64_t tiles = (a.T / tokens + (a.S < a.T ? a.S : a.T)) * a.kv_heads;   // as many as there can be
  constexpr int64_t kPiece = int64_t(1) << 23;                     // (a launch holds fewer than 2^32 threads)
  CacheArgs piece = a;
  for (piece.t0 = 0; piece.t0 < tiles; piece.t0 += kPiece) launch_attention<0, false>(piece, (uint32_t)(tiles - piece.t0 < kPiece ? tiles - piece.t0 : kPiece), s);
  return hipGetLastError();
}

}  // namespace axe
