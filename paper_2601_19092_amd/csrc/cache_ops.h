// Arguments of the kernels around the paged cache (append, attention), by value, and their launches; what follows from sizes alone.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_types.h"
#include "layer_ops.h"

namespace axe {

// Division of 31-bit numbers by a fixed d >= 1.
struct Divisor {
  uint32_t d;
  Div31 by;
};
inline Divisor divisor(int64_t d) { return Divisor{(uint32_t)d, div31_by(d)}; }

// Strides in elements.
struct HeadRows {
  int64_t token, head;
};
struct CachePlaces {
  int64_t page, slot, head;
};

struct CacheArgs {
  const void *q, *k, *v;
  void *out, *k_cache, *v_cache;   // (attention reads the caches and their scales)
  float *k_scales, *v_scales;
  const float* rotation;
  const int32_t *seq_rows, *lengths, *table;
  float* ws;
  HeadRows qs, ks, vs, os;
  CachePlaces kp, vp;
  int64_t T, pages;
  int64_t t0;                      // the launch's first row (append), or tile
  int32_t S, q_heads, kv_heads, D;
  int32_t max_pages, capacity;     // capacity: max_pages times the tokens of a page
  Divisor page, group, rows;       // tokens of a page; query heads of a head of the cache; append: rows (heads) of a token
  int32_t rotary, pairs;
  int32_t causal, window;
  float scale_log2;                // scale / ln 2
  int32_t type, fp8;               // kBf16 or kF16; e4m3 cache
  int32_t groups;                  // attention, split form: workgroups
  int32_t ws_rows;                 // rows of a partial result
};
hipError_t launch_cache_append(const CacheArgs& a, hipStream_t s);
hipError_t launch_cache_attention(const CacheArgs& a, hipStream_t s);

// ---- attention: the shape of a call

constexpr int kAttnRows = 128;     // rows (tokens x query heads of one head of the cache) of a tile
constexpr int kAttnKeys = 64;      // keys of a block
constexpr int kAttnMaxGroup = 128; // query heads of a head of the cache
constexpr int kAttnSplitSeqs = 4096;

inline int attn_columns(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }
inline int attn_tile_tokens(int group) { return kAttnRows / group; }
// Workgroups that the chip holds at once.
inline int attn_slots(int D) { return attn_columns(D) <= 128 ? 512 : 256; }
// Whether the keys of a tile are split among workgroups: not where there are tiles enough to fill the chip some times over, each a workgroup's.
inline bool attn_split(int64_t T, int S, int kv_heads, int group, int D) {
  const int64_t tokens = attn_tile_tokens(group), tiles = (T + tokens - 1) / tokens * kv_heads;
  return S <= kAttnSplitSeqs && tiles < 2 * (int64_t)attn_slots(D);
}
inline int attn_ws_rows(int64_t T, int group) {
  const int64_t rows = T < attn_tile_tokens(group) ? T * group : kAttnRows;
  return (int)((rows + 31) / 32 * 32);
}
// A partial result: a head of four words, the maxima and sums of its rows, the rows themselves.
inline int64_t attn_part_words(int rows, int D) { return 4 + 2 * (int64_t)rows + (int64_t)rows * attn_columns(D); }
inline int64_t attn_workspace_words(int64_t T, int S, int kv_heads, int group, int D) {
  if (T == 0 || !attn_split(T, S, kv_heads, group, D)) return 0;
  return 2 * attn_slots(D) * attn_part_words(attn_ws_rows(T, group), D);
}

}  // namespace axe
