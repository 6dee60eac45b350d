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
  int32_t sixteens;                // attention: 16 keys from a multiple of 16 on lie in one page, within 2^31 bytes of each other
  int32_t reach31;                 // attention: both caches' elements lie within 2^31 bytes
  int32_t groups;                  // attention, split form: workgroups
  int32_t tile_rows;               // 16, 32 or kAttnRows
  int32_t ws_rows;                 // rows of a partial result
};
hipError_t launch_cache_append(const CacheArgs& a, hipStream_t s);
hipError_t launch_cache_attention(const CacheArgs& a, hipStream_t s);

template <int RT>
void launch_attention_narrow(const CacheArgs& a, uint32_t groups, hipStream_t s);   // groups: workgroups (a.groups in the split form)
template <>
void launch_attention_narrow<1>(const CacheArgs& a, uint32_t groups, hipStream_t s);
template <>
void launch_attention_narrow<2>(const CacheArgs& a, uint32_t groups, hipStream_t s);

// ---- attention: the shape of a call

constexpr int kAttnRows = 128;     // rows (tokens x query heads of one head of the cache) of a wide tile
constexpr int kAttnKeys = 64;      // keys of a block
constexpr int kAttnMaxGroup = 128; // query heads of a head of the cache
constexpr int kAttnSplitSeqs = 4096;
constexpr int kAttnFewKeys = 768;

inline int attn_columns(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }
// Workgroups that the chip holds at once.
inline int attn_slots(int D) { return attn_columns(D) <= 128 ? 512 : 256; }

// groups: workgroups of the split form, 0: every tile a workgroup's.  Splitting a tile's keys among workgroups costs partial results and a second launch, some 20 us of wide tiles, for which ten blocks
// of keys are done.  It is not done where there are tiles enough to fill the chip some times over, nor where all workgroups are through with their tiles by the time: 24 blocks at most, and 16
// on average that a place on the chip is idle.  us, split / whole: 512 new tokens, 32 heads over 4, 39 / 18; 1024, 32 over 8, 51 / 29; 24 x 100 over 1100 keys, 16 heads of 64 columns, 56 / 32;
// 256 over 2048 keys 42 / 75.  Narrow tiles, by the same: up to 768 keys, twice that where 64 tiles or more share the chip's bandwidth; one token, 32 heads over 4, of 512 keys 12.4 / 11.0, of 1024
// 14.4 / 16.3; 16 tokens, 32 over 8, of 1536 27.3 / 25.2; 64 tokens of 1024 51.8 / 46.5.
// The keys counted are those that the table has room for, not the lengths: these are the device's to know, and launches and the workspace follow from the descriptor alone.  So the same call is split under a table
// of a server's longest sequence.  us, a table as wide as the longest sequence / one of 8192 pages: 512 new tokens, 32 heads over 4, 19.3 / 39.7; 1024, 32 over 8, 32.1 / 49.9; 24 x 100 over 1100 keys 36.5 / 52.8; one
// token of 500 keys 12.2 / 13.5; 16 of 1000 19.4 / 22.0.
// Rows of a tile: 128 where those alone fill the chip twice, or above 4096 sequences (one token of each of 512 sequences of 100 keys, 128 heads over 16 of 256 columns: 394 us, of 496, in tiles of 16, 404).  Else as many
// as the sequences have on average, up to 32; from there on 128, or 32 where 128 would leave most of the chip without a tile.  us, 128 / 32 rows: 38 wide tiles, 600 new
// tokens over 700 keys of 256 columns, 39 / 30; 32, 128 tokens over 8192, 77 / 69; 16, 64 over 2048, 36 / 34; 64, 256 over 2048, 42 / 49; 128, 100 of each of 8 over 2200, 54 / 79.
struct AttnShape {
  int tile_rows, groups, ws_rows;
};
// window: keys that a token sees at most, 0: all.
inline AttnShape attn_shape(int64_t T, int S, int kv_heads, int group, int D, int64_t capacity, int window) {
  AttnShape r = {kAttnRows, 0, 0};
  if (T == 0 || S == 0) return r;
  const int64_t wide = kAttnRows / group, tiles = (T + wide - 1) / wide * kv_heads;
  if (S > kAttnSplitSeqs || tiles >= 2 * (int64_t)attn_slots(D)) return r;
  const int64_t rows = (T + S - 1) / S * group;
  const int64_t whole = T < S ? T : S, wides = (T + wide - 1) / wide > whole ? tiles : whole * kv_heads;   // (as all sequences have new tokens)
  if (rows <= 32 || (group <= 32 && wides < 48)) r.tile_rows = rows <= 16 ? 16 : 32;
  const int64_t reach = window && window + wide < capacity ? window + wide : capacity, blocks = (reach + kAttnKeys - 1) / kAttnKeys, slots = attn_slots(D);
  const int64_t idle = (slots - tiles % slots) % slots;
  const int64_t tokens = r.tile_rows / group, cut = (T + tokens - 1) / tokens, narrows = (cut > whole ? cut : whole) * kv_heads;
  if (r.tile_rows <= 32 ? reach <= (narrows < 64 ? kAttnFewKeys : 2 * kAttnFewKeys) : blocks <= 24 && blocks * idle <= 16 * slots) return r;
  r.groups = attn_slots(D);
  const int64_t most = T < tokens ? T * group : r.tile_rows;
  r.ws_rows = (int)((most + 15) / 16 * 16);
  return r;
}
// A partial result: a head of four words, the maxima and sums of its rows, the rows themselves.
inline int64_t attn_part_words(int rows, int D) { return 4 + 2 * (int64_t)rows + (int64_t)rows * attn_columns(D); }
inline int64_t attn_workspace_words(const AttnShape& s, int D) { return 2 * s.groups * attn_part_words(s.ws_rows, D); }

}  // namespace axe
