// Appending keys and values to a paged cache, with the rotation by position (axe_cache_append).  gfx950 only.
//
// Bound by memory: every element is read once and written once.  A row (one head of one token) is held by LPR lanes, a run of eight columns each, in fp32; the columns that a run
// is turned with are read a second time, from the line that the neighbouring lanes have just brought in, and the largest magnitude of a row that becomes e4m3 stays inside
// the row's lanes.
#include <hip/hip_runtime.h>

#include "cache_ops.h"
#include "cache_tables.h"
#include "row_ops.h"

namespace axe {

template <int LPR>
__device__ __forceinline__ float row_max(float v) {
  if constexpr (LPR == 8) return row8_all<Max>(v);
  else if constexpr (LPR == 16) return row16_all<Max>(v);
  else return half_all<Max>(v);
}

// TYPE: of q, k, v; CACHE: of the caches.  LPR lanes hold a row of up to 8 LPR columns.
template <int TYPE, int CACHE, int LPR>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheArgs a) {
  constexpr int ROWS = 256 / LPR;
  fetch_arguments(a.q, a.v_scales, a.qs.token, a.vp.page, a.S, a.rotary);
  const uint32_t chunks = (a.rows.d + ROWS - 1) / ROWS, chunk = blockIdx.x % chunks;
  const int64_t t = a.t0 + blockIdx.x / chunks;
  const int s = sequence_of(a.seq_rows, a.S, t);
  if (s < 0) return;
  const int64_t first = a.seq_rows[s], last = a.seq_rows[s + 1], p = a.lengths[s] - last + t;
  if (t < first || p < 0 || p >= a.capacity) return;               // no token, or one without a place
  const int pos = (int)p;
  const uint32_t in_table = quotient(pos, a.page);
  const int page = a.table[(int64_t)s * a.max_pages + in_table], slot = pos - (int)(in_table * a.page.d);
  const uint32_t row = chunk * ROWS + threadIdx.x / LPR;
  const int c = threadIdx.x % LPR * 8;
  if (row >= a.rows.d) return;
  const uint32_t n_q = a.rows.d - 2 * a.kv_heads;
  const int what = row < n_q ? 0 : row < n_q + a.kv_heads ? 1 : 2;
  const int head = (int)(what == 0 ? row : what == 1 ? row - n_q : row - n_q - a.kv_heads);
  if (what && (uint32_t)page >= (uint64_t)a.pages) return;
  const bool there = c < a.D;
  const HeadRows& in = what == 0 ? a.qs : what == 1 ? a.ks : a.vs;
  const void* x = elem_at(what == 0 ? a.q : what == 1 ? a.k : a.v, t * in.token + head * in.head, 2);
  Run8<TYPE> run;
  run.clear();
  if (there) run.template load<false>((const uint16_t*)x + c);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = run.get(i);
  if (what < 2 && there && c < a.rotary) {
    const float* angles = a.rotation + (int64_t)pos * a.rotary;
    const int half = a.rotary >> 1;
    if (a.pairs) {
#pragma unroll
      for (int i = 0; i < 8; i += 2)
        if (c + i < a.rotary) {
          const float cs = angles[(c + i) >> 1], sn = angles[half + ((c + i) >> 1)], u = v[i], w = v[i + 1];
          v[i] = u * cs - w * sn, v[i + 1] = w * cs + u * sn;
        }
    } else if ((half & 7) == 0) {                                  // a run's partners are a run
      const bool low = c < half;
      Run8<TYPE> other;
      Run8<kF32> cs, sn;
      other.template load<false>((const uint16_t*)x + (low ? c + half : c - half));
      cs.template load<false>(angles + (low ? c : c - half)), sn.template load<false>(angles + half + (low ? c : c - half));
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = v[i] * cs.get(i) + (low ? -other.get(i) : other.get(i)) * sn.get(i);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < a.rotary) {
          const bool low = c + i < half;
          const int j = low ? c + i : c + i - half;
          Run8<TYPE> other;
          other.b[0] = ((const uint16_t*)x)[low ? j + half : j];
          v[i] = v[i] * angles[j] + (low ? -other.get(0) : other.get(0)) * angles[half + j];
        }
    }
  }
  if (what == 0) {
    run.set(v);
    if (there) run.template store<false>((uint16_t*)a.out + t * a.os.token + head * a.os.head + c);
    return;
  }
  const CachePlaces& to = what == 1 ? a.kp : a.vp;
  void* dst = elem_at(what == 1 ? a.k_cache : a.v_cache, page * to.page + slot * to.slot + head * to.head + c, elem_bytes(CACHE));
  Run8<CACHE> q;
  if constexpr (CACHE == kFp8) {
    float most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[i]));   // (NaN: the other operand)
    const Scale sc = scale_of(row_max<LPR>(most), false);
    over_scale(v, sc);
    if (c == 0) (what == 1 ? a.k_scales : a.v_scales)[((int64_t)page * a.page.d + slot) * a.kv_heads + head] = sc.s;
  }
  q.set(v);
  if (there) q.template store<false>(dst);
}

template <int TYPE, int CACHE>
void launch(const CacheArgs& all, hipStream_t s) {
  const int lpr = all.D <= 64 ? 8 : all.D <= 128 ? 16 : 32, rows = 256 / lpr;
  const int64_t chunks = (all.rows.d + rows - 1) / rows;
  // (a launch holds fewer than 2^32 threads)
  const int64_t piece = ((int64_t(1) << 23) + chunks - 1) / chunks;
  CacheArgs a = all;
  for (a.t0 = 0; a.t0 < all.T; a.t0 += piece) {
    const uint32_t groups = (uint32_t)((all.T - a.t0 < piece ? all.T - a.t0 : piece) * chunks);
    if (lpr == 8) cache_append_kernel<TYPE, CACHE, 8><<<groups, 256, 0, s>>>(a);
    else if (lpr == 16) cache_append_kernel<TYPE, CACHE, 16><<<groups, 256, 0, s>>>(a);
    else cache_append_kernel<TYPE, CACHE, 32><<<groups, 256, 0, s>>>(a);
  }
}

hipError_t launch_cache_append(const CacheArgs& a, hipStream_t s) {
  if (a.type == kBf16) a.fp8 ? launch<kBf16, kFp8>(a, s) : launch<kBf16, kBf16>(a, s);
  else a.fp8 ? launch<kF16, kFp8>(a, s) : launch<kF16, kF16>(a, s);
  return hipGetLastError();
}

}  // namespace axe
