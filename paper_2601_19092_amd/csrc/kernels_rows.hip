// The tokens' rows in the experts' order and back (axe_rows_dispatch, axe_rows_combine, axe_rows_combine_backward).  gfx950 only.
//
// All three are bound by memory.  A wave takes 512 columns of a token, eight a lane, or 1024 where it quantises (of a pair in the gradient, whose dot product wants the whole
// row): columns are independent, so there is nothing to wait for but the memory, and a run of 128 columns that shares a scale is eight neighbouring lanes.  dispatch
// reads a token once and stores its k copies from registers; combine has the loads of eight rows in flight.
#include <hip/hip_runtime.h>

#include "layer_ops.h"
#include "row_ops.h"

namespace axe {

constexpr int kSlab = 512;                                         // columns of a wave

// A token's rows: lane j holds the row of choice j (-1: none).
struct RowsOf {
  int mine;
  __device__ __forceinline__ RowsOf(const RowsArgs& a, int64_t t, int lane) {
    mine = -1;
    if (!a.row_of) mine = (int)t;
    else if (lane < a.k) mine = a.row_of[t * a.k + lane];
    if (mine < 0 || mine >= a.M) mine = -1;
  }
  __device__ __forceinline__ int row(int j) const { return __builtin_amdgcn_readlane(mine, j); }
};
// Which token and which columns a wave has, RUNS runs of eight a lane.
template <int RUNS = 1>
struct WaveAt {
  int lane, c;
  int64_t t;
  bool there;
  __device__ __forceinline__ WaveAt(int64_t T, int H) {
    const int slabs = (H + kSlab * RUNS - 1) / (kSlab * RUNS);
    const uint32_t w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lane = threadIdx.x & 63;
    t = w / (uint32_t)slabs;
    c = ((int)(w - (uint32_t)t * slabs) * kSlab + lane * 8) * RUNS;
    there = t < T;
  }
};

// Copies of elements of TYPE's size (fp32 as pairs of 16 bits).
template <int TYPE, bool SHORT>
__global__ __launch_bounds__(256) void rows_copy_kernel(RowsArgs a, int H, int64_t ldt, int64_t ldr) {
  fetch_arguments(a.tokens, a.row_of, a.H);
  const WaveAt<> w(a.T, H);
  if (!w.there) return;
  constexpr int EB = elem_bytes(TYPE);
  Run8<TYPE> v;
  load_run<SHORT>(v, elem_at(a.tokens, w.t * ldt, EB), w.c, H);
  const RowsOf rows(a, w.t, w.lane);
  end_run<SHORT>(v, w.c, H);
  for (int j = 0; j < a.k; ++j) {
    const int64_t r = rows.row(j);
    if (r >= 0) store_run(v, elem_at(a.to_rows, r * ldr, EB), w.c, H);
  }
}
// The scales of e4m3 tokens to their rows: a thread per pair and scale.
template <class S>
__global__ __launch_bounds__(256) void rows_copy_scales_kernel(RowsArgs a, int blocks) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, pair = i / blocks;
  if (pair >= a.T * a.k) return;
  const int b = (int)(i - pair * blocks);
  const int64_t t = pair / a.k, r = a.row_of ? a.row_of[pair] : t;
  if (r >= 0 && r < a.M) ((S*)a.scales)[r * blocks + b] = ((const S*)a.token_scales)[t * blocks + b];
}

// Sixteen columns a lane: its store is 16 bytes (us, with eight and 8 / sixteen and 16: 1024 tokens to 8 rows of 2048 6.7 / 5.9, 32768 rows of 768 in order 18.8 / 15.7; with the codes of the quotient 6.1 and 16.3).
template <int TYPE, bool SHORT>
__global__ __launch_bounds__(256) void rows_quantise_kernel(RowsArgs a) {
  fetch_arguments(a.tokens, a.row_of, a.H);
  const WaveAt<2> w(a.T, a.H);
  if (!w.there) return;
  Run8<TYPE> v[2];
  const void* row = elem_at(a.tokens, w.t * a.ldt, elem_bytes(TYPE));
#pragma unroll
  for (int i = 0; i < 2; ++i) load_run<SHORT>(v[i], row, w.c + 8 * i, a.H);
  const RowsOf rows(a, w.t, w.lane);
  float y[2][8], most = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    end_run<SHORT>(v[i], w.c + 8 * i, a.H);
#pragma unroll
    for (int k = 0; k < 8; ++k) y[i][k] = v[i].get(k), most = fmaxf(most, fabsf(y[i][k]));
  }
  const Scale s = scale_of(row8_all<Max>(most), a.e8m0);
  Run8<kFp8> q[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    over_scale(y[i], s);
    q[i].set(y[i]);
  }
  const int blocks = (a.H + 127) >> 7;
  for (int j = 0; j < a.k; ++j) {
    const int64_t r = rows.row(j);
    if (r < 0) continue;
    uint8_t* to = (uint8_t*)a.to_rows + r * a.ldr;
    if (w.c + 16 <= a.H) store_bits(to + w.c, u32x4{q[0].b[0], q[0].b[1], q[1].b[0], q[1].b[1]});
    else store_run(q[0], to, w.c, a.H), store_run(q[1], to, w.c + 8, a.H);
    if ((w.lane & 7) == 0 && w.c < a.H) store_scale(a.scales, r * blocks + (w.c >> 7), s, a.e8m0);
  }
}

// ROWS: rows whose loads are in flight together; ONCE: they go past the caches.
template <int TYPE, int ROWS, bool ONCE, bool SHORT>
__global__ __launch_bounds__(256) void rows_combine_kernel(RowsArgs a) {
  fetch_arguments(a.tokens, a.row_of, a.H);
  const WaveAt<> w(a.T, a.H);
  if (!w.there) return;
  constexpr int EB = elem_bytes(TYPE);
  const RowsOf rows(a, w.t, w.lane);
  const float weight = a.weights && w.lane < a.k ? a.weights[w.t * a.k + w.lane] : 1.0f;
  float sum[8];
  Run8<TYPE> v;
  v.clear();
  if (a.add) load_run<SHORT>(v, elem_at(a.add, w.t * a.ldt, EB), w.c, a.H), end_run<SHORT>(v, w.c, a.H);
#pragma unroll
  for (int k = 0; k < 8; ++k) sum[k] = v.get(k);
  for (int j0 = 0; j0 < a.k; j0 += ROWS) {
    Run8<TYPE> c[ROWS];
    int r[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {                               // (a row that is none: the first one, whose bits are then dropped -- a branch would put each load behind the one before)
      r[j] = j0 + j < a.k ? rows.row(j0 + j) : -1;
      load_run<SHORT, ONCE>(c[j], elem_at(a.rows, max(r[j], 0) * a.ldr, EB), w.c, a.H);
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
      c[j].keep(r[j] >= 0);
      end_run<SHORT>(c[j], w.c, a.H);
      const float wj = r[j] >= 0 ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(weight), (j0 + j) & 63)) : 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) sum[k] += wj * c[j].get(k);
    }
  }
  v.set(sum);
  store_run(v, elem_at(a.to_tokens, w.t * a.ldt, EB), w.c, a.H);
}

// A wave per pair, eight to a workgroup (the pairs of a token read its row together: with four, and two workgroups on different XCDs, 4096 tokens of 8 rows fetched 170 MB for 151),
// RUNS runs of a lane at a time.  DOT: the rows are read, for dweights.  PAST: what goes past the caches, 1: stores, 2: loads of the rows, too.
template <int TYPE, int RUNS, bool DOT, int PAST, bool SHORT>
__global__ __launch_bounds__(512) void rows_combine_backward_kernel(RowsArgs a) {
  fetch_arguments(a.tokens, a.row_of, a.H);
  constexpr int EB = elem_bytes(TYPE);
  const int lane = threadIdx.x & 63;
  const int64_t pair = (int64_t)blockIdx.x * 8 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (pair >= a.T * a.k) return;
  const int64_t t = pair / a.k;
  const int64_t r = a.row_of[pair];
  float dot = 0;
  if (r >= 0 && r < a.M) {
    const float w = a.weights ? a.weights[pair] : 1.0f;
    const void *rd = elem_at(a.tokens, t * a.ldt, EB), *rc = elem_at(a.rows, r * a.ldr, EB);
    void* ro = elem_at(a.to_rows, r * a.ldr, EB);
    for (int c0 = lane * 8; c0 - lane * 8 < a.H; c0 += kSlab * RUNS) {
      Run8<TYPE> d[RUNS], c[RUNS];
#pragma unroll
      for (int i = 0; i < RUNS; ++i) {                             // (runs behind the row's end: its last one, and zeros in the end)
        if (DOT) load_run<SHORT, PAST == 2>(c[i], rc, c0 + i * kSlab, a.H);
        load_run<SHORT>(d[i], rd, c0 + i * kSlab, a.H);
      }
#pragma unroll
      for (int i = 0; i < RUNS; ++i) {
        end_run<SHORT>(d[i], c0 + i * kSlab, a.H);
        if (DOT) {
          end_run<SHORT>(c[i], c0 + i * kSlab, a.H);
#pragma unroll
          for (int k = 0; k < 8; ++k) dot += d[i].get(k) * c[i].get(k);
        }
      }
      if (a.to_rows) {
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
          float v[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = w * d[i].get(k);
          d[i].set(v);
          store_run<PAST != 0>(d[i], ro, c0 + i * kSlab, a.H);
        }
      }
    }
    if (DOT) dot = wave_sum(dot);
  }
  if (DOT && lane == 0) a.dweights[pair] = dot;
}

// A launch holds fewer than 2^32 threads: calls of more waves go in pieces of whole tokens.
template <class F>
hipError_t in_pieces(const RowsArgs& a, int64_t waves_per_token, F&& f) {
  const int64_t most = ((int64_t)1 << 25) / waves_per_token, piece = most ? most : 1;
  for (int64_t t0 = 0; t0 < a.T; t0 += piece) {
    RowsArgs p = a;
    p.T = a.T - t0 < piece ? a.T - t0 : piece;
    const int64_t blocks = (a.H + 127) / 128;
    p.tokens = elem_at(a.tokens, t0 * a.ldt, elem_bytes(a.t_type)), p.to_tokens = elem_at(a.to_tokens, t0 * a.ldt, elem_bytes(a.t_type));
    p.token_scales = elem_at(a.token_scales, t0 * blocks, a.e8m0 ? 1 : 4);
    if (a.add) p.add = elem_at(a.add, t0 * a.ldt, elem_bytes(a.t_type));
    if (a.row_of) p.row_of = a.row_of + t0 * a.k;
    else p.to_rows = elem_at(a.to_rows, t0 * a.ldr, elem_bytes(a.r_type)), p.scales = elem_at(a.scales, t0 * blocks, a.e8m0 ? 1 : 4), p.M = p.T;
    if (a.weights) p.weights = a.weights + t0 * a.k;
    if (a.dweights) p.dweights = a.dweights + t0 * a.k;
    f(p, (uint32_t)((p.T * waves_per_token + 3) / 4));
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}
static int64_t slabs_of(int64_t columns) { return (columns + kSlab - 1) / kSlab; }

template <int TYPE>
void launch_quantise(const RowsArgs& p, uint32_t groups, hipStream_t s) {
  if (p.H < 8) rows_quantise_kernel<TYPE, true><<<groups, 256, 0, s>>>(p);
  else rows_quantise_kernel<TYPE, false><<<groups, 256, 0, s>>>(p);
}
hipError_t launch_rows_dispatch(const RowsArgs& a, hipStream_t s) {
  if (a.t_type != a.r_type)
    return in_pieces(a, (a.H + 2 * kSlab - 1) / (2 * kSlab), [&](const RowsArgs& p, uint32_t groups) {
      if (a.t_type == kBf16) launch_quantise<kBf16>(p, groups, s);
      else if (a.t_type == kF16) launch_quantise<kF16>(p, groups, s);
      else launch_quantise<kF32>(p, groups, s);
    });
  // as 16-bit elements, but e4m3 whose rows are odd or start anywhere
  const int eb = elem_bytes(a.t_type);
  const bool bytes = eb == 1 && ((a.H | a.ldt | a.ldr | (int64_t)(uintptr_t)a.tokens | (int64_t)(uintptr_t)a.to_rows) & 1);
  const int n = bytes ? a.H : a.H * eb / 2;
  const int64_t scale_waves = a.t_type == kFp8 ? (int64_t)a.k * ((a.H + 127) / 128) / 64 + 1 : 0, slabs = slabs_of(n);
  return in_pieces(a, slabs > scale_waves ? slabs : scale_waves, [&](const RowsArgs& p, uint32_t) {
    const uint32_t groups = (uint32_t)((p.T * slabs + 3) / 4);
    const int64_t ldt = bytes ? p.ldt : p.ldt * eb / 2, ldr = bytes ? p.ldr : p.ldr * eb / 2;
    if (bytes && n < 8) rows_copy_kernel<kFp8, true><<<groups, 256, 0, s>>>(p, n, ldt, ldr);
    else if (bytes) rows_copy_kernel<kFp8, false><<<groups, 256, 0, s>>>(p, n, ldt, ldr);
    else if (n < 8) rows_copy_kernel<kBf16, true><<<groups, 256, 0, s>>>(p, n, ldt, ldr);
    else rows_copy_kernel<kBf16, false><<<groups, 256, 0, s>>>(p, n, ldt, ldr);
    if (a.t_type == kFp8) {
      const int blocks = (a.H + 127) / 128;
      const uint32_t sg = (uint32_t)((p.T * p.k * blocks + 255) / 256);
      if (a.e8m0) rows_copy_scales_kernel<uint8_t><<<sg, 256, 0, s>>>(p, blocks);
      else rows_copy_scales_kernel<uint32_t><<<sg, 256, 0, s>>>(p, blocks);
    }
  });
}

// What a call of all its pairs moves.
static int64_t rows_bytes(const RowsArgs& a, int rows_times, int tokens_times) { return ((int64_t)a.k * rows_times + tokens_times) * a.T * a.H * elem_bytes(a.r_type); }

template <int TYPE, bool ONCE>
hipError_t launch_combine(const RowsArgs& a, hipStream_t s) {
  return in_pieces(a, slabs_of(a.H), [&](const RowsArgs& p, uint32_t groups) {
    if (a.H < 8) rows_combine_kernel<TYPE, 8, false, true><<<groups, 256, 0, s>>>(p);
    else if (a.k == 1) rows_combine_kernel<TYPE, 1, ONCE, false><<<groups, 256, 0, s>>>(p);
    else if (a.k == 2) rows_combine_kernel<TYPE, 2, ONCE, false><<<groups, 256, 0, s>>>(p);
    else if (a.k <= 4) rows_combine_kernel<TYPE, 4, ONCE, false><<<groups, 256, 0, s>>>(p);
    else rows_combine_kernel<TYPE, 8, ONCE, false><<<groups, 256, 0, s>>>(p);
  });
}
template <bool ONCE>
hipError_t launch_combine_of(const RowsArgs& a, hipStream_t s) {
  return a.r_type == kBf16 ? launch_combine<kBf16, ONCE>(a, s) : a.r_type == kF16 ? launch_combine<kF16, ONCE>(a, s) : launch_combine<kF32, ONCE>(a, s);
}
hipError_t launch_rows_combine(const RowsArgs& a, hipStream_t s) {
  return rows_bytes(a, 1, a.add ? 2 : 1) >= kPastCaches ? launch_combine_of<true>(a, s) : launch_combine_of<false>(a, s);
}

template <int TYPE, bool DOT, int PAST>
hipError_t launch_combine_backward(const RowsArgs& a, hipStream_t s) {
  return in_pieces(a, a.k, [&](const RowsArgs& p, uint32_t) {
    const uint32_t groups = (uint32_t)((p.T * p.k + 7) / 8);
    if (a.H < 8) rows_combine_backward_kernel<TYPE, 1, DOT, 0, true><<<groups, 512, 0, s>>>(p);
    else if (a.H <= kSlab) rows_combine_backward_kernel<TYPE, 1, DOT, PAST, false><<<groups, 512, 0, s>>>(p);
    else if (a.H <= 2 * kSlab) rows_combine_backward_kernel<TYPE, 2, DOT, PAST, false><<<groups, 512, 0, s>>>(p);
    else rows_combine_backward_kernel<TYPE, 4, DOT, PAST, false><<<groups, 512, 0, s>>>(p);
  });
}
template <bool DOT, int PAST>
hipError_t launch_combine_backward_of(const RowsArgs& a, hipStream_t s) {
  return a.r_type == kBf16 ? launch_combine_backward<kBf16, DOT, PAST>(a, s)
                           : a.r_type == kF16 ? launch_combine_backward<kF16, DOT, PAST>(a, s) : launch_combine_backward<kF32, DOT, PAST>(a, s);
}
hipError_t launch_rows_combine_backward(const RowsArgs& a, hipStream_t s) {
  const int64_t bytes = rows_bytes(a, (a.dweights ? 1 : 0) + (a.to_rows ? 1 : 0), 1);
  if (!a.dweights) return bytes >= kPastCaches ? launch_combine_backward_of<false, 1>(a, s) : launch_combine_backward_of<false, 0>(a, s);
  return bytes >= kAllPastCaches ? launch_combine_backward_of<true, 2>(a, s)
                                 : bytes >= kPastCaches ? launch_combine_backward_of<true, 1>(a, s) : launch_combine_backward_of<true, 0>(a, s);
}

}  // namespace axe
