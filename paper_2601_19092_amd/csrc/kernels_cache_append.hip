// Appending keys and values to a paged cache, with the rotation by position (axe_cache_append).  gfx950 only.
//
// Bound by memory: every element is read once and written once.  A row (one head of one token) is held by LPR lanes, a run of eight columns each, in fp32; the columns that a run
// is turned with are read a second time, from the line that the neighbouring lanes have just brought in, and the largest magnitude of a row that becomes e4m3 stays inside
// the row's lanes.  4000 tokens of 32 + 2 x 4 heads of 128 columns, fp16, 83 MB of rows: 19 - 22 us (an earlier form, one row a lane, loads behind the look-up: 26); one token 5.8, of which the kernel has 3.
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

// TYPE: of q, k, v; CACHE: of the caches.  LPR lanes hold a row of up to 8 LPR columns; a workgroup has P times 256 / LPR rows of one token.  What is read of the rows does not depend on where the
// token is, and is on its way before that is looked up; the angles are those of a lane's columns in all its rows.
template <int TYPE, int CACHE, int LPR, int P>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheArgs a) {
  constexpr int ROWS = 256 / LPR;
  fetch_arguments(a.q, a.v_scales, a.qs.token, a.vp.page, a.S, a.rotary);
  const uint32_t chunks = (a.rows.d + P * ROWS - 1) / (P * ROWS), chunk = blockIdx.x % chunks;
  const int64_t t = a.t0 + blockIdx.x / chunks;
  const int c = threadIdx.x % LPR * 8, half = a.rotary >> 1;
  const uint32_t n_q = a.rows.d - 2 * a.kv_heads;
  const bool there = c < a.D, runs = !a.pairs && (half & 7) == 0, low = c < half;   // runs: a run is turned with another run
  Run8<TYPE> run[P], other[P];
  int what[P], head[P];                                            // 0, 1, 2: a row of q, k, v; 3: none
  const uint16_t* x[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const uint32_t row = chunk * (P * ROWS) + i * ROWS + threadIdx.x / LPR;
    what[i] = row < n_q ? 0 : row < n_q + a.kv_heads ? 1 : row < a.rows.d ? 2 : 3;
    head[i] = (int)(what[i] == 0 ? row : what[i] == 1 ? row - n_q : row - n_q - a.kv_heads);
    const HeadRows& in = what[i] == 0 ? a.qs : what[i] == 1 ? a.ks : a.vs;
    x[i] = (const uint16_t*)(what[i] == 0 ? a.q : what[i] == 1 ? a.k : a.v) + t * in.token + head[i] * in.head;
    run[i].clear(), other[i].clear();
    if (there && what[i] < 3) {
      run[i].template load<false>(x[i] + c);
      if (what[i] < 2 && runs && c < a.rotary) other[i].template load<false>(x[i] + (low ? c + half : c - half));
    }
  }
  const int s = sequence_of(a.seq_rows, a.S, t);
  if (s < 0) return;
  const int64_t first = border(a, a.seq_rows[s]), last = border(a, a.seq_rows[s + 1]), p = a.lengths[s] - last + t;
  if (t < first || p < 0 || p >= a.capacity) return;               // no token, or one without a place
  const int pos = (int)p;
  const uint32_t in_table = quotient(pos, a.page);
  const int page = a.table[(int64_t)s * a.max_pages + in_table], slot = pos - (int)(in_table * a.page.d);
  const float* angles = a.rotation + (int64_t)pos * a.rotary;
  // of the lane's columns; pairs: four of either
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = 1, sn[i] = 0;
  if (there && c < a.rotary) {
    if (runs) {
      Run8<kF32> u, w;
      u.template load<false>(angles + (low ? c : c - half)), w.template load<false>(angles + half + (low ? c : c - half));
#pragma unroll
      for (int i = 0; i < 8; ++i) cs[i] = u.get(i), sn[i] = low ? -w.get(i) : w.get(i);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < a.rotary) {
          const int j = a.pairs ? (c + i) >> 1 : c + i < half ? c + i : c + i - half;
          const bool minus = a.pairs ? !(i & 1) : c + i < half;
          cs[i] = angles[j], sn[i] = minus ? -angles[half + j] : angles[half + j];
        }
    }
  }
  const bool stored = (uint32_t)page < (uint64_t)a.pages;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (what[i] == 3 || (what[i] && !stored)) continue;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = run[i].get(k);
    if (what[i] < 2 && there && c < a.rotary) {
      if (a.pairs) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c + k < a.rotary) v[k] = run[i].get(k) * cs[k] + run[i].get(k ^ 1) * sn[k];
      } else if (runs) {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = v[k] * cs[k] + other[i].get(k) * sn[k];
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (c + k < a.rotary) {
            Run8<TYPE> o;
            o.b[0] = x[i][c + k < half ? c + k + half : c + k - half];
            v[k] = v[k] * cs[k] + o.get(0) * sn[k];
          }
      }
    }
    if (what[i] == 0) {
      run[i].set(v);
      if (there) run[i].template store<false>((uint16_t*)a.out + t * a.os.token + head[i] * a.os.head + c);
      continue;
    }
    const CachePlaces& to = what[i] == 1 ? a.kp : a.vp;
    void* dst = elem_at(what[i] == 1 ? a.k_cache : a.v_cache, page * to.page + slot * to.slot + head[i] * to.head + c, elem_bytes(CACHE));
    Run8<CACHE> q;
    if constexpr (CACHE == kFp8) {
      float most = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) most = fmaxf(most, fabsf(v[k])); // (NaN: the other operand)
      const Scale sc = scale_of(row_max<LPR>(most), false);
      over_scale(v, sc);
      if (c == 0) (what[i] == 1 ? a.k_scales : a.v_scales)[((int64_t)page * a.page.d + slot) * a.kv_heads + head[i]] = sc.s;
    }
    q.set(v);
    if (there) q.template store<false>(dst);
  }
}

template <int TYPE, int CACHE, int LPR, int P>
void launch_rows(const CacheArgs& all, hipStream_t s) {
  constexpr int rows = P * 256 / LPR;
  const int64_t chunks = (all.rows.d + rows - 1) / rows;
  // (a launch holds fewer than 2^32 threads)
  const int64_t piece = ((int64_t(1) << 23) + chunks - 1) / chunks;
  CacheArgs a = all;
  for (a.t0 = 0; a.t0 < all.T; a.t0 += piece) cache_append_kernel<TYPE, CACHE, LPR, P><<<(uint32_t)((all.T - a.t0 < piece ? all.T - a.t0 : piece) * chunks), 256, 0, s>>>(a);
}
template <int TYPE, int CACHE, int LPR>
void launch_lanes(const CacheArgs& a, hipStream_t s) {
  // Rows of a lane: one as long as the workgroups do not fill the chip, else up to three.
  constexpr int rows = 256 / LPR;
  const int64_t groups = (a.rows.d + rows - 1) / rows;
  if (groups == 1 || a.T * groups <= 2048) launch_rows<TYPE, CACHE, LPR, 1>(a, s);
  else if (groups == 2) launch_rows<TYPE, CACHE, LPR, 2>(a, s);
  else launch_rows<TYPE, CACHE, LPR, 3>(a, s);
}
template <int TYPE, int CACHE>
void launch(const CacheArgs& a, hipStream_t s) {
  if (a.D <= 64) launch_lanes<TYPE, CACHE, 8>(a, s);
  else if (a.D <= 128) launch_lanes<TYPE, CACHE, 16>(a, s);
  else launch_lanes<TYPE, CACHE, 32>(a, s);
}

hipError_t launch_cache_append(const CacheArgs& a, hipStream_t s) {
  if (a.type == kBf16) a.fp8 ? launch<kBf16, kFp8>(a, s) : launch<kBf16, kBf16>(a, s);
  else a.fp8 ? launch<kF16, kFp8>(a, s) : launch<kF16, kF16>(a, s);
  return hipGetLastError();
}

}  // namespace axe
