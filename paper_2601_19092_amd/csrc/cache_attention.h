// Attention of new tokens over a paged cache (axe_cache_attention): the kernels.  Device code, gfx950 only.
//
//   o[t, h] = sum_j softmax_j(scale q[t, h] . K[j]) V[j]
//
// A tile is 128 rows: the query heads of one head of the cache, of consecutive new tokens of one sequence (row r: token r / G, head r mod G), so that one pass over the keys
// serves all of them.  A workgroup of four waves takes a tile's keys 64 at a time: K and V of the 64 go straight from their pages to LDS (two blocks of LDS, one filled while the
// other is read), and every wave has 32 rows for itself:
//   S^T = K Q^T      a lane holds 32 of the 64 scores of one row, lane + 32 the others: maximum and sum of a row are a chain in the lane and one exchange;
//   O^T += V^T P^T   the scores' registers, in 16 bits, are the product's operand as they are: its contraction runs over the keys in the order in which the registers hold them, and V comes out of LDS in
//                    that order by transposing reads.
// The maximum is a running one: when it grows, sums and O are multiplied down.  Everything but the products' operands is fp32.  The terms are one of them: matrix instructions take 16-bit operands at 16 times the rate
// of fp32 ones, and a term's rounding, 2^-8 or 2^-11 of it at most, is no larger than the result's own (relative error against 64 bits 2.0e-3 in bf16, 2.6e-4 in fp16; with terms in fp32 1.6e-3, 2.1e-4).
//
// Where a batch has few tiles, the list of all (tile, block of keys) is cut into as many equal runs as there are workgroups, wherever that falls; a tile that is cut leaves partial
// results (maximum, sum, O) in the workspace, and a second kernel joins them, in the order of the keys.  Which run a workgroup has follows from the lengths alone: results repeat
// their bits.
//
// Tiles of 16 and 32 rows, for sequences with few new tokens, are bound by memory: every wave has keys and LDS for itself, two turns of loads under way.  One token of each of 64 sequences up to 8192
// tokens, 32 heads over 4 of 128 columns: 606 MB in 111 us, 5.5 TB/s; one of 131072, fp16: 537 MB in 97 us.  Wide tiles are bound by the matrix and the vector unit, which overlap in part: a prompt of 4096 tokens, 32 heads
// over 8, 137 GFLOP in 148 - 157 us; matrix instructions and LDS reads alone 113, the terms and maxima alone 71, without the loads 146; one workgroup a compute unit in place of two 234.  4 x 512 over 8192 keys: 266
// GFLOP in 270 - 288 us.
#pragma once
#include <hip/hip_runtime.h>

#include "cache_ops.h"
#include "cache_tables.h"
#include "gemm_common.h"
#include "row_ops.h"

namespace axe {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((address_space(3))) s16x4* tr_ptr;
typedef __attribute__((address_space(3))) i32x2* tr8_ptr;

template <int TYPE>
__device__ __forceinline__ f32x16 mfma32(s16x8 a, s16x8 b, f32x16 c) {
  if constexpr (TYPE == kBf16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if constexpr (TYPE == kBf16) return pack_bf16(lo, hi);
  else {
    typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
    return __builtin_bit_cast(uint32_t, f16x2{(_Float16)lo, (_Float16)hi});
  }
}
template <int TYPE>
__device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (TYPE == kBf16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int TYPE>
__device__ __forceinline__ f32x4 mfma16_short(s16x4 a, s16x4 b, f32x4 c) {
  typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
  if constexpr (TYPE == kBf16) return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4, a), __builtin_bit_cast(f16x4, b), c, 0, 0, 0);
}
// Eight e4m3 numbers in 16 bits, which hold them all.
template <int TYPE>
__device__ __forceinline__ s16x8 widen(u32x2 v) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (TYPE == kBf16) {
      r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], 1.0f, false));
      r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], 1.0f, true));
    } else {
      r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[i], 1.0f, false));
      r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[i], 1.0f, true));
    }
  }
  return __builtin_bit_cast(s16x8, r);
}
template <int TYPE>
__device__ __forceinline__ float half(uint32_t two, int which) {
  if constexpr (TYPE == kBf16) return __uint_as_float(which ? two & 0xffff0000u : two << 16);
  else return (float)__builtin_bit_cast(_Float16, (uint16_t)(two >> which * 16));
}
// Their sum, and c.
template <int TYPE>
__device__ __forceinline__ float add2(uint32_t two, float c) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
  if constexpr (TYPE == kBf16) return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, 0x3f803f80u), c, false);
  else return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, two), f16x2{(_Float16)1.0f, (_Float16)1.0f}, c, false);
}
// What a term p counts in the sum when the product with V has t = p v / lift, v the scale of V's row, as `rounded`: rounded lift / v.  A key that has nearly all the weight then has V's row for its result, not
// that times the error of one rounding.  Where t is below the type's smallest steps, or near them, `rounded` says nothing of p, which then counts as it is: what a key weighs is not for the size of its value to say.
template <int TYPE>
__device__ __forceinline__ float weight(float p, float t, float v, float rounded, float lift) {
  constexpr float LEAST = TYPE == kBf16 ? 0x1p-100f : 0x1p-14f;       // (p is at most 2^15: 1 / v is in range)
  const float by = __builtin_amdgcn_rcpf(v);
  return fabsf(t) >= LEAST && fabsf(v) <= 1e30f ? fmaf((rounded - t) * lift, by, p) : p;
}
// e4m3 values in fp16: terms times scales stay inside fp16's range, and above its smallest steps, by being divided by `lift`, a power of two (2^-90 to 2^126): for every row the one above the largest scale that
// it has seen, however small or large that is.  (A scale that is no number has no say in it; a row that sees an infinite one is not finite, whatever it is divided by.  By the row
// and not by the tile: 7 - 9 % of the time in tiles of 32 rows, 0 - 3 elsewhere.)
constexpr float kLeastLift = 0x1p-90f;
__device__ __forceinline__ float lift_above(float most) {
  const uint32_t up = (__float_as_uint(most) & 0x7f800000u) + 0x800000u;
  return __uint_as_float(up < 0x7e800000u ? up : 0x7e800000u);
}
__device__ __forceinline__ float over_lift(float lift) { return __uint_as_float(0x7f000000u - __float_as_uint(lift)); }   // 1 / lift
// v of the four lanes of a column (lane mod 16) joined.
template <class OP>
__device__ __forceinline__ float quarters(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
  v = OP::of(__int_as_float(a[0]), __int_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return OP::of(__int_as_float(b[0]), __int_as_float(b[1]));
}
__device__ __forceinline__ float other_half(float v) {              // of lane ^ 32
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float((threadIdx.x & 32) ? s[0] : s[1]);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// The terms are exp2(s by + less), by = scale / ln 2 and less = LIFT - m, m the row's maximum: one instruction, which does not round the product s by as m was rounded.  What that leaves between the largest score and
// m is nothing beside LIFT as long as m is small (2^-4 at this size), and out of the terms' range when it is not (fp16 from 2^28 on).  There the scores become s by, rounded, less m first.
constexpr float kLargeScore = 0x1p20f;
__device__ __forceinline__ float less_maximum(float s, float by, float m) {
  float x = s * by;
  asm volatile("" : "+v"(x));                                       // (rounded here)
  return x - m;
}

// 16 bytes that are zero: what a lane brings to LDS for a key that is not there.
__device__ const u32x4 kNothing = {0, 0, 0, 0};

// Loads into LDS, 16 bytes a lane: the wave's 1024 bytes from `lds` on.  (Written as asm: the compiler would wait for them before it reads any of LDS.  M0 holds the address;
// the wait states are for registers that a vector instruction may just have written.)
template <bool ONCE>
__device__ __forceinline__ void load_lds(const void* from, uint32_t lds) {
  if constexpr (ONCE) asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(from), "s"(lds) : "memory");
  else asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(lds) : "memory");
}
template <bool ONCE>
__device__ __forceinline__ void load_lds(uint32_t offset, const void* base, uint32_t lds) {
  if constexpr (ONCE) asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(offset), "s"(base), "s"(lds) : "memory");
  else asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(lds) : "memory");
}
// Two of them, the second's 1024 bytes behind the first's.
template <bool ONCE>
__device__ __forceinline__ void load_lds(uint32_t offset, uint32_t offset2, const void* base, uint32_t lds) {
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %2 nt\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"v"(offset), "v"(offset2),
                 "s"(base), "s"(lds)
                 : "memory", "scc");
  else
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %2\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"v"(offset), "v"(offset2), "s"(base),
                 "s"(lds)
                 : "memory", "scc");
}
// The same, 4 bytes a lane.
__device__ __forceinline__ void load_lds4(const void* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(lds) : "memory");
}

// ---- the batch

struct Seq {
  int row0, n;                     // its rows
  int first;                       // position of its first new token
  int len;                         // keys
};
__device__ __forceinline__ Seq sequence(const CacheArgs& a, int s) {
  const int end = border(a, a.seq_rows[s + 1]), l = a.lengths[s];
  Seq q;
  q.row0 = border(a, a.seq_rows[s]);
  q.n = end > q.row0 ? end - q.row0 : 0;
  const int length = l < 0 ? 0 : l;
  q.len = length < a.capacity ? length : a.capacity;
  q.first = length - q.n;
  return q;
}
// Keys that tokens i0 .. i1 of a sequence see between them, [lo, hi).
struct Range {
  int lo, hi;
};
__device__ __forceinline__ Range seen(const CacheArgs& a, const Seq& q, int i0, int i1) {
  Range r = {0, q.len};
  if (a.causal) {
    const int end = q.first + i1 + 1;
    r.hi = end < r.hi ? (end > 0 ? end : 0) : r.hi;
    if (a.window) {
      const int at = q.first + i0 + 1 - a.window;
      r.lo = at < 0 ? 0 : at < a.capacity ? at : a.capacity;
    }
  }
  return r;
}
struct Blocks {
  int first, count;                // a tile without keys has one block, without keys
};
__device__ __forceinline__ Blocks blocks_of(const Range& r) {
  const int first = r.lo / kAttnKeys, end = (r.hi + kAttnKeys - 1) / kAttnKeys;
  return Blocks{first, end > first ? end - first : 1};
}
__device__ __forceinline__ int tiles_of(const CacheArgs& a, const Seq& q, int tokens) { return (q.n + tokens - 1) / tokens; }
__device__ __forceinline__ Blocks tile_blocks(const CacheArgs& a, const Seq& q, int tokens, int tile) {
  const int i0 = tile * tokens, i1 = (i0 + tokens < q.n ? i0 + tokens : q.n) - 1;
  return blocks_of(seen(a, q, i0, i1));
}
// The split form takes a sequence's tiles in pairs, the first with the last: they have about the same number of blocks together, at most `cell`, which is what a pair counts.
struct Cost {
  int pairs, cell;
};
__device__ __forceinline__ Cost cost_of(const CacheArgs& a, const Seq& q, int tokens) {
  const int tiles = tiles_of(a, q, tokens);
  if (tiles <= 1) return Cost{tiles, tiles ? tile_blocks(a, q, tokens, 0).count : 0};
  int64_t cell = 2 * (int64_t)((q.len + kAttnKeys - 1) / kAttnKeys);
  if (a.causal) {
    const int64_t up = (2 * (int64_t)(q.first > 0 ? q.first : 0) + (int64_t)(tiles + 1) * tokens + 2 * (kAttnKeys - 1)) / kAttnKeys;
    cell = up < cell ? up : cell;
    if (a.window) {
      const int64_t w = 2 * (((int64_t)a.window + tokens) / kAttnKeys + 2);
      cell = w < cell ? w : cell;
    }
  }
  return Cost{(tiles + 1) / 2, (int)(cell > 2 ? cell : 2)};
}

// What a workgroup works on: a tile, or a run of its blocks.
struct Item {
  Seq q;
  int s, head;                     // sequence, head of the cache
  int i0, tokens;                  // its tokens
  Range keys;
  int b0, b1;                      // blocks of keys
};

// Offset of a partial result in the workspace, words.
__device__ __forceinline__ int64_t part_at(const CacheArgs& a, int group, int which, int DP) { return ((int64_t)group * 2 + which) * (4 + 2 * (int64_t)a.ws_rows + (int64_t)a.ws_rows * DP); }

// ---- the kernel

// RT 0: wide tiles of 128 rows; 1, 2: narrow ones of 16 RT rows.
template <int TYPE, bool FP8, int DP, int RT>
struct Attention {
  static constexpr int ROWS = RT ? 16 * RT : kAttnRows;
  static constexpr int ROW = DP * 2;                               // bytes of a key in LDS, in 16 bits
  static constexpr int BLOCK = kAttnKeys * ROW;                    // of K, or V, of a block
  static constexpr int STEPS = DP / 16, DT = DP / 32;
  // exp2 of this is a factor of the softmax's terms: fp16 has few numbers below 1
  static constexpr float LIFT = TYPE == kBf16 ? 0.0f : 9.0f;
  // The running maximum is left alone until a score is this much (in powers of two) above it: terms are up to 2^LAG, and hardly ever is all that has been summed multiplied down.
  static constexpr float LAG = 6.0f;

  // Sixteen keys as loads of 16 bytes a lane bring them to LDS: CH chunks a key, RPI keys a load, NI loads.  Chunks change places by the key's number, so that what is read
  // together lies in different banks.
  template <int EB>
  struct Sixteen {
    static constexpr int CH = DP * EB / 16, RPI = 64 / CH, NI = 16 / RPI;
    static constexpr int LINE = CH >= 16 ? 1 : 16 / CH;            // keys that lie in 256 bytes, the width of LDS
    // What a key's chunks are moved by (XOR).  K is read by 16 lanes at a time, the same chunk of 16 keys.
    static __device__ __forceinline__ int k(int row) { return row / LINE & (CH < 16 ? CH - 1 : 15); }
    // V, wide: by 32 lanes, 64 bytes of 4 keys; narrow: 32 bytes of 8 keys; narrow in e4m3: 16 bytes of 16 keys, those of 16 .. with those of 0 ..
    static __device__ __forceinline__ int v(int row) {
      if constexpr (EB == 1) return (row % 8 / LINE | (row >> 4 & 1) * (8 / LINE)) & (CH < 16 ? CH - 1 : 15);
      else if constexpr (RT == 0) return (row % 4 / LINE << 2) & (CH - 1);
      else return (row % 8 / LINE << 1) & (CH - 1);
    }
    static __device__ __forceinline__ int place(bool of_v, int row) { return of_v ? v(row) : k(row); }
  };
  using S2 = Sixteen<2>;
  using SN = Sixteen<FP8 ? 1 : 2>;

  // Narrow tiles: a wave has keys for itself, KT at a time, and LDS of its own for two such turns.
  static constexpr int KT = FP8 ? 32 : 16, NROW = FP8 ? DP : ROW, TURN = KT * NROW;

  struct Shared {
    union {
      __attribute__((aligned(16))) uint8_t kv[2][2][BLOCK];        // wide: [stage][K, V]
      __attribute__((aligned(16))) uint8_t own[4][2][2][TURN];     // narrow: [wave][turn][K, V]
    };
    float scales[2][2][2 * kAttnKeys];                             // wide: [stage][K, V] of 64 keys; narrow: [wave][turn] of 32 keys, K then V
    float top[4][32], sum[4][32];                                  // narrow: the waves' maxima and sums
    uint16_t there[2][4];                                          // wide: of a wave's 16 keys: which there are
    int flags[4];
    uint8_t marks[kAttnRows];                                      // of a tile's tokens, see survey
    int64_t sums[8];
    int64_t found[4];
  };
  static_assert(4 * 2 * 2 * TURN <= 2 * 2 * BLOCK && sizeof(Shared::scales) == 4 * 2 * 64 * 4, "a turn of all waves is no more than a stage");

  // Operands in LDS are read AHEAD of the product that takes them, which the compiler would not do: it reads, waits, multiplies.  Hence steps that stay in the order written.
  static constexpr int AHEAD = 4;
  static __device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

  const CacheArgs& a;
  Shared& sh;
  const int lane, wave, h;
  Item it;

  // 64 entries of the sequence's page table, a lane each, from page `page0` on
  int entries, page0;

  __device__ __forceinline__ Attention(const CacheArgs& a_, Shared& s_) : a(a_), sh(s_), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), h((threadIdx.x >> 5) & 1) {}

  static __device__ __forceinline__ uint32_t lds_at(const void* p) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)p); }

  // ---- keys from their pages

  __device__ __forceinline__ void need_pages(int first, int count) {   // of keys first .. first + count - 1, at most 32
    const int from = first > it.keys.lo ? first : it.keys.lo, end = first + count < it.keys.hi ? first + count : it.keys.hi;
    if (from >= end) return;
    const int p0 = (int)quotient(from, a.page), p1 = (int)quotient(end - 1, a.page);
    if (p1 - page0 < 64 && p0 >= page0) return;
    page0 = p0;
    entries = p0 + lane < a.max_pages ? a.table[(int64_t)it.s * a.max_pages + p0 + lane] : -1;
    asm volatile("" : "+v"(entries));                              // (waited for here, where it is rare: the loads into LDS would be waited for too)
  }
  // The same before an item's first keys, not waited for: the queries come with them.
  __device__ __forceinline__ void first_pages(int first) {
    const int from = first > it.keys.lo ? first : it.keys.lo;
    page0 = -1000, entries = -1;
    if (from >= it.keys.hi) return;
    page0 = (int)quotient(from, a.page);
    if (page0 + lane < a.max_pages) entries = a.table[(int64_t)it.s * a.max_pages + page0 + lane];
  }
  // Whether sixteen keys from `first`, a multiple of 16, on all are there, side by side in one page; then where they begin.
  __device__ __forceinline__ bool together(int first, int& page, int& slot) {
    if (!a.sixteens || first < it.keys.lo || first + 16 > it.keys.hi) return false;
    const int p = (int)quotient(first, a.page);
    page = __builtin_amdgcn_readlane(entries, p - page0);
    slot = first - p * (int)a.page.d;
    return (uint32_t)page < (uint64_t)a.pages;
  }
  // Where a lane's key lies; false: it is not there.  (All lanes take part.)
  __device__ __forceinline__ bool where(int key, int& page, int& slot) {
    const bool in = key >= it.keys.lo && key < it.keys.hi;
    const int p = in ? (int)quotient(key, a.page) : page0;
    page = __shfl(entries, (p - page0) & 63);
    slot = in ? key - p * (int)a.page.d : 0;
    return in && (uint32_t)page < (uint64_t)a.pages;
  }
  // Where sixteen keys lie.
  struct Found {
    int first, page, slot;
    bool side_by_side;
  };
  __device__ __forceinline__ Found find(int first) {
    Found f = {first, 0, 0, false};
    f.side_by_side = together(first, f.page, f.slot);
    return f;
  }
  // Sixteen keys (K or V) to LDS, as keys row0 .. there.
  template <int EB>
  __device__ __forceinline__ void bring(bool v, const Found& f, int row0, uint32_t lds) {
    using S = Sixteen<EB>;
    constexpr bool ONCE = RT > 0;
    const CachePlaces& pl = v ? a.vp : a.kp;
    const uint8_t* cache = (const uint8_t*)(v ? a.v_cache : a.k_cache) + (int64_t)it.head * pl.head * EB;
    auto column = [&](int i) __attribute__((always_inline)) { return (lane % S::CH ^ S::place(v, row0 + i * S::RPI + lane / S::CH)) * 16; };
    if (f.side_by_side) {
      const uint8_t* base = cache + (f.page * pl.page + f.slot * pl.slot) * EB;
      auto offset = [&](int i) __attribute__((always_inline)) { return (uint32_t)((i * S::RPI + lane / S::CH) * (int)pl.slot * EB + column(i)); };
      if (a.D == DP) {
        if constexpr (S::NI == 1) load_lds<ONCE>(offset(0), base, lds);
        else
#pragma unroll
          for (int i = 0; i < S::NI; i += 2) load_lds<ONCE>(offset(i), offset(i + 1), base, lds + i * 1024);
      } else {
#pragma unroll
        for (int i = 0; i < S::NI; ++i)                            // (the other lanes' places hold zeros, see clear_lds)
          if (column(i) < a.D * EB) load_lds<ONCE>(offset(i), base, lds + i * 1024);
      }
      return;
    }
    int ln = lane, page, slot;
    if (RT > 0 && a.reach31 && f.first >= it.keys.lo && f.first + 16 <= it.keys.hi) {   // all there, in pages of their own, and 32 bits hold the way to each: a lane works it out for each key (wide: bring_apart)
      asm volatile("" : "+v"(ln));
      const bool on = where(f.first + (ln & 15), page, slot);
      if (__all(on)) {
        const uint32_t at = (uint32_t)page * (uint32_t)(pl.page * EB) + (uint32_t)slot * (uint32_t)(pl.slot * EB);
#pragma unroll
        for (int i = 0; i < S::NI; ++i) {
          const int row = i * S::RPI + ln / S::CH, c = (ln % S::CH ^ S::place(v, row0 + row)) * 16;
          const uint32_t off = (uint32_t)__shfl((int)at, row) + c;
          if (c < a.D * EB) load_lds<ONCE>(off, cache, lds + i * 1024);
        }
        return;
      }
    }
    const bool any = f.first < it.keys.hi && f.first + 16 > it.keys.lo;
    asm volatile("" : "+v"(ln));                                   // (nothing of this is made ahead of the loop: it is rare, and the registers are needed)
#pragma unroll 1
    for (int i = 0; i < S::NI; ++i) {
      const int row = i * S::RPI + ln / S::CH, c = (ln % S::CH ^ S::place(v, row0 + row)) * 16;
      const void* from = &kNothing;
      if (any && where(f.first + row, page, slot) && c < a.D * EB) from = cache + (page * pl.page + slot * pl.slot) * EB + c;
      load_lds<false>(from, lds + i * 1024);
    }
  }
  // Sixteen keys, K and V, that are all there, in pages of their own, where 32 bits hold the way to each: where they lie is worked out once.
  // (Pages of 24, us, before / now: prompts and single tokens of 24 sequences, 16 heads of 64 columns, window 1000, 48 / 43; 4 x 512 over 8192 keys 343 / 314.  Worked out a block ahead: no faster.)
  __device__ __forceinline__ bool bring_apart(int first, uint32_t k_lds, uint32_t v_lds) {
    if (!a.reach31 || first < it.keys.lo || first + 16 > it.keys.hi) return false;
    int ln = lane, page, slot;
    asm volatile("" : "+v"(ln));
    const bool on = where(first + (ln & 15), page, slot);
    if (!__all(on)) return false;
    const uint32_t k_at = (uint32_t)page * (uint32_t)(a.kp.page * 2) + (uint32_t)slot * (uint32_t)(a.kp.slot * 2);
    const uint32_t v_at = (uint32_t)page * (uint32_t)(a.vp.page * 2) + (uint32_t)slot * (uint32_t)(a.vp.slot * 2);
    const uint8_t *kb = (const uint8_t*)a.k_cache + (int64_t)it.head * a.kp.head * 2, *vb = (const uint8_t*)a.v_cache + (int64_t)it.head * a.vp.head * 2;
    const bool alike = a.kp.page == a.vp.page && a.kp.slot == a.vp.slot;
#pragma unroll
    for (int i = 0; i < S2::NI; ++i) {
      const int row = i * S2::RPI + ln / S2::CH, kc = (ln % S2::CH ^ S2::k(row)) * 16, vc = (ln % S2::CH ^ S2::v(row)) * 16;
      const uint32_t k = (uint32_t)__shfl((int)k_at, row);
      uint32_t v = k;
      if (!alike) v = (uint32_t)__shfl((int)v_at, row);
      if (kc < a.D * 2) load_lds<false>(k + kc, kb, k_lds + i * 1024);
      if (vc < a.D * 2) load_lds<false>(v + vc, vb, v_lds + i * 1024);
    }
    return true;
  }
  // Which of KEYS keys there are.
  template <int KEYS>
  __device__ __forceinline__ uint32_t which(int first) {
    if (first >= it.keys.hi || first + KEYS <= it.keys.lo) return 0;
    int ln = lane, page, slot;
    asm volatile("" : "+v"(ln));
    return (uint32_t)__ballot(where(first + ln, page, slot) && ln < KEYS);
  }
  // Columns from D to DP stay zero: nothing is loaded there.
  __device__ __forceinline__ void clear_lds() {
    if (a.D == DP) return;
    for (int i = threadIdx.x; i < (int)sizeof(sh.kv) / 16; i += 256) ((u32x4*)&sh.kv[0][0][0])[i] = u32x4{};
    lds_barrier();
  }

  // ---- wide tiles

  s16x8 q[RT ? 1 : STEPS];
  f32x16 o[RT ? 1 : DT];
  float m, l;                                                      // running maximum (scaled) and this lane's part of the sum
  int lo, hi;                                                      // keys that this lane's row sees
  int w_lo, w_hi;                                                  // that all of the wave's rows see
  bool rows_here;
  float lift_v;                                                    // e4m3 values in fp16: what their scales are divided by (lift_above)
  u32x2 kreg[FP8 ? S2::NI : 1], vreg[FP8 ? S2::NI : 1];            // e4m3: a block on its way
  float sreg[2];

  // Starts the loads of a wave's keys of a block into a stage (e4m3: into registers).
  __device__ __forceinline__ void issue(int block, int stage) {
    const int first = block * kAttnKeys + wave * 16;
    need_pages(first, 16);
    const Found f = find(first);
    uint32_t there = 0xffff;
    if constexpr (!FP8) {
      const uint32_t k_lds = lds_at(&sh.kv[stage][0][wave * 16 * ROW]), v_lds = lds_at(&sh.kv[stage][1][wave * 16 * ROW]);
      if (f.side_by_side) {
        bring<2>(false, f, 0, k_lds);
        bring<2>(true, f, 0, v_lds);
      } else if (!bring_apart(first, k_lds, v_lds)) {
        there = which<16>(first);
        bring<2>(false, f, 0, k_lds);
        bring<2>(true, f, 0, v_lds);
      }
    } else {
      const uint8_t *kb = (const uint8_t*)a.k_cache + it.head * a.kp.head, *vb = (const uint8_t*)a.v_cache + it.head * a.vp.head;
      int64_t at = 0;                                              // of the scales: lane i brings those of key i
      bool on = true;
      if (f.side_by_side) {
        kb += f.page * a.kp.page + f.slot * a.kp.slot, vb += f.page * a.vp.page + f.slot * a.vp.slot;
#pragma unroll
        for (int i = 0; i < S2::NI; ++i) {
          const int row = i * S2::RPI + lane / S2::CH, kc = (lane % S2::CH ^ S2::k(row)) * 8, vc = (lane % S2::CH ^ S2::v(row)) * 8;
          kreg[i] = vreg[i] = u32x2{};
          if (kc < a.D) kreg[i] = *(const u32x2*)(kb + (uint32_t)(row * (int)a.kp.slot + kc));
          if (vc < a.D) vreg[i] = *(const u32x2*)(vb + (uint32_t)(row * (int)a.vp.slot + vc));
        }
        at = (int64_t)f.page * a.page.d + f.slot + (lane & 15);
      } else {
        int ln = lane, page, slot;
        asm volatile("" : "+v"(ln));
        on = where(first + (ln & 15), page, slot);
        there = (uint32_t)__ballot(on) & 0xffff;
        at = (int64_t)page * a.page.d + slot;
        if (a.reach31 && there == 0xffff) {                        // (as bring_apart; a prompt of 1300 tokens, 20 heads over 5 of 80 columns, pages of 7, 67 -> 56 us; 8 x 1100, 24 over 3 of 192, pages of 100, 667 -> 524)
          const uint32_t k_at = (uint32_t)page * (uint32_t)a.kp.page + (uint32_t)slot * (uint32_t)a.kp.slot, v_at = (uint32_t)page * (uint32_t)a.vp.page + (uint32_t)slot * (uint32_t)a.vp.slot;
#pragma unroll
          for (int i = 0; i < S2::NI; ++i) {
            const int row = i * S2::RPI + ln / S2::CH, kc = (ln % S2::CH ^ S2::k(row)) * 8, vc = (ln % S2::CH ^ S2::v(row)) * 8;
            const uint32_t k = (uint32_t)__shfl((int)k_at, row), v = (uint32_t)__shfl((int)v_at, row);
            kreg[i] = vreg[i] = u32x2{};
            if (kc < a.D) kreg[i] = *(const u32x2*)(kb + (k + kc));
            if (vc < a.D) vreg[i] = *(const u32x2*)(vb + (v + vc));
          }
        } else {
#pragma unroll
          for (int i = 0; i < S2::NI; ++i) {
            const int row = i * S2::RPI + ln / S2::CH, kc = (ln % S2::CH ^ S2::k(row)) * 8, vc = (ln % S2::CH ^ S2::v(row)) * 8;
            int p2, s2;
            const bool is = where(first + row, p2, s2);
            kreg[i] = vreg[i] = u32x2{};
            if (is && kc < a.D) kreg[i] = *(const u32x2*)(kb + p2 * a.kp.page + s2 * a.kp.slot + kc);
            if (is && vc < a.D) vreg[i] = *(const u32x2*)(vb + p2 * a.vp.page + s2 * a.vp.slot + vc);
          }
        }
      }
      sreg[0] = sreg[1] = 0;
      if (on) sreg[0] = a.k_scales[at * a.kv_heads + it.head], sreg[1] = a.v_scales[at * a.kv_heads + it.head];
    }
    if (lane == 0) sh.there[stage][wave] = (uint16_t)there;
  }
  // e4m3: the block in registers becomes 16 bits in LDS.
  __device__ __forceinline__ void settle(int stage) {
    if constexpr (FP8) {
#pragma unroll
      for (int i = 0; i < S2::NI; ++i) {
        const uint32_t at = (wave * 16 + i * S2::RPI) * ROW + lane * 16;
        *(s16x8*)&sh.kv[stage][0][at] = widen<TYPE>(kreg[i]);
        *(s16x8*)&sh.kv[stage][1][at] = widen<TYPE>(vreg[i]);
      }
      if (lane < 16) sh.scales[stage][0][wave * 16 + lane] = sreg[0], sh.scales[stage][1][wave * 16 + lane] = sreg[1];
    }
  }

  __device__ __forceinline__ void begin() {
    const int G = a.group.d;
    const int r = wave * 32 + (lane & 31), rows = it.tokens * G;
    const bool on = r < rows;
    rows_here = wave * 32 < rows;
    const int rr = on ? r : rows - 1, i = (int)quotient(rr, a.group), g = rr - i * G;
    const uint16_t* from = (const uint16_t*)a.q + (int64_t)(it.q.row0 + it.i0 + i) * a.qs.token + (int64_t)(it.head * G + g) * a.qs.head;
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int c = k * 16 + h * 8;
      q[k] = s16x8{};
      if (on && c < a.D) q[k] = __builtin_bit_cast(s16x8, load_bits<u32x4>(from + c));
    }
    asm volatile("" : "+v"(entries));
#pragma unroll
    for (int k = 0; k < STEPS; ++k) asm volatile("" : "+v"(q[k])); // (waited for here: where they are used a wait would be one for the keys on their way)
    const Range mine = seen(a, it.q, it.i0 + i, it.i0 + i);
    lo = mine.lo, hi = mine.hi;
    const int last = rows - 1 < wave * 32 + 31 ? rows - 1 : wave * 32 + 31;
    w_lo = seen(a, it.q, it.i0 + (int)quotient(last, a.group), it.i0 + (int)quotient(last, a.group)).lo;   // (both ends grow with the token)
    w_hi = seen(a, it.q, it.i0 + (int)quotient(rows_here ? wave * 32 : 0, a.group), it.i0 + (int)quotient(rows_here ? wave * 32 : 0, a.group)).hi;
    m = -INFINITY, l = 0, lift_v = kLeastLift;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = f32x16{};
  }

  // A block's share of the wave's rows, from a stage.
  __device__ __forceinline__ void compute(int block, int stage) {
    const int k0 = block * kAttnKeys;
    const uint64_t there = *(const uint64_t*)&sh.there[stage][0];
    const uint32_t t0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)there), t1 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(there >> 32));
    const bool masked = (t0 & t1) != 0xffffffffu || k0 < w_lo || k0 + kAttnKeys > w_hi;
    const uint8_t *K = sh.kv[stage][0], *V = sh.kv[stage][1];
    f32x16 s[2] = {f32x16{}, f32x16{}};
    {
      const uint32_t at = (lane & 31) * ROW + (h ^ S2::k(lane & 31)) * 16;
      auto read = [&](int i) __attribute__((always_inline)) { return *(const s16x8*)(K + ((at ^ ((i >> 1) * 32)) + (i & 1) * 32 * ROW)); };
      s16x8 k[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) k[i] = read(i);
#pragma unroll
      for (int i = 0; i < STEPS * 2; ++i) {
        const s16x8 now = k[i % AHEAD];
        in_order();
        if (i + AHEAD < STEPS * 2) k[i % AHEAD] = read(i + AHEAD);
        s[i & 1] = mfma32<TYPE>(now, q[i >> 1], s[i & 1]);
      }
    }
    if constexpr (FP8) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const f32x4 sc = *(const f32x4*)&sh.scales[stage][0][t * 32 + r * 8 + h * 4];
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t][r * 4 + e] *= sc[e];
        }
    }
    if (masked) {
      const uint32_t mine[2] = {t0 >> (h * 4), t1 >> (h * 4)};
      const int low = lo - k0 - h * 4;
      const uint32_t many = hi > lo ? hi - lo : 0;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int k = (r >> 2) * 8 + (r & 3);
          s[t][r] = (uint32_t)(t * 32 + k - low) < many && (mine[t] & 1u << k) ? s[t][r] : -INFINITY;
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int r = 1; r < 32; ++r) top = fmaxf(top, s[r >> 4][r & 15]);
    top = fmaxf(top, other_half(top)) * a.scale_log2;
    if (__any(top > m + LAG)) {
      const float grown = fmaxf(m, top), by = grown > m ? exp2_fast(m - grown) : 1.0f;   // (the first time: m is -inf, the sums are 0)
      m = grown, l *= by;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= by;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    float less = LIFT - base, by_s = a.scale_log2;
    if (__builtin_expect(__any(fabsf(base) > kLargeScore), 0)) {
#pragma unroll
      for (int r = 0; r < 32; ++r) s[r >> 4][r & 15] = less_maximum(s[r >> 4][r & 15], by_s, base);
      less = LIFT, by_s = 1;
    }
    float by_v = 1;
    if constexpr (FP8 && TYPE == kF16) {
      float most = 0;
      if (masked) {                                                // (of the keys that the row sees)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const f32x4 sv = *(const f32x4*)&sh.scales[stage][1][t * 32 + r * 8 + h * 4];
#pragma unroll
            for (int e = 0; e < 4; ++e) most = fmaxf(most, s[t][r * 4 + e] > -INFINITY ? fabsf(sv[e]) : 0.0f);
          }
        most = fmaxf(most, other_half(most));
      } else most = wave_all<Max>(fabsf(sh.scales[stage][1][lane]));
      if (__any(most >= lift_v)) {
        const float to = fmaxf(lift_v, lift_above(most)), down = lift_v / to;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[t][r] *= down;
        lift_v = to;
      }
      by_v = over_lift(lift_v);
    }
    // lane i of 16 points at 4 columns of key i / 4 and receives 4 keys of column i
    const int i = lane & 15, row = h * 4 + (i >> 2);
    const uint32_t at = row * ROW + ((((lane >> 4) & 1) * 2 + ((i & 3) >> 1)) ^ S2::v(row)) * 16 + (i & 1) * 8;
    auto read = [&](int i) __attribute__((always_inline)) {        // of keys 16 (i / DT) .., columns 32 (i mod DT) ..
      const uint8_t* v0 = V + ((at ^ (i % DT * 64)) + i / DT * 16 * ROW);
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)v0), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(v0 + 8 * ROW));
      return s16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    };
    // Two terms of 16 keys k: p[k], pair e of four.
    u32x4 p[4];
    auto two = [&](int k, int e) __attribute__((always_inline)) {
      const int r = (k & 1) * 8 + 2 * e;
      const float x = exp2_fast(fmaf(s[k >> 1][r], by_s, less)), y = exp2_fast(fmaf(s[k >> 1][r + 1], by_s, less));
      if constexpr (FP8) {
        const float* sc = &sh.scales[stage][1][k * 16 + (e >> 1) * 8 + h * 4 + (e & 1) * 2];
        const float v0 = sc[0] * by_v, v1 = sc[1] * by_v, t0 = x * v0, t1 = y * v1;
        p[k][e] = pack2<TYPE>(t0, t1);
        l += x + y;                                                // (not as they are rounded, as in run_narrow: here the vector unit is what bounds)
      } else {
        p[k][e] = pack2<TYPE>(x, y);
        l = add2<TYPE>(p[k][e], l);
      }
    };
    // The terms of 16 keys, and their product with V: the next 16 keys' terms keep the vector unit while this product keeps the matrix unit.
    s16x8 v[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) v[i] = read(i);
#pragma unroll
    for (int e = 0; e < 4; ++e) two(0, e);
#pragma unroll
    for (int i = 0; i < DT * 4; ++i) {
      const s16x8 now = v[i % AHEAD];
      in_order();
      if (i + AHEAD < DT * 4) v[i % AHEAD] = read(i + AHEAD);
      o[i % DT] = mfma32<TYPE>(now, __builtin_bit_cast(s16x8, p[i / DT]), o[i % DT]);
      if (i / DT < 3) {
#pragma unroll
        for (int e = 4 * (i % DT) / DT; e < 4 * (i % DT + 1) / DT; ++e) two(i / DT + 1, e);
      }
    }
    in_order();
  }

  // All blocks of the item, for the rows of all waves.
  __device__ __forceinline__ void run_wide() {
    first_pages(it.b0 * kAttnKeys + wave * 16);
    begin();
    clear_lds();
    issue(it.b0, 0);
    auto blocks = [&](auto rows) __attribute__((always_inline)) {
      for (int b = it.b0; b < it.b1; ++b) {
        const int stage = (b - it.b0) & 1;
        settle(stage);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        if (b + 1 < it.b1) issue(b + 1, stage ^ 1);
        if constexpr (decltype(rows)::value) compute(b, stage);
      }
    };
    if (rows_here) blocks(std::true_type());
    else blocks(std::false_type());                                // (a wave without rows brings its keys)
    l += other_half(l);
    if constexpr (FP8 && TYPE == kF16) {
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= lift_v;
    }
  }
  // Whether x, 0 as long as all results are finite, is anything else in a thread of the workgroup.
  __device__ __forceinline__ bool not_finite(float x) {
    const bool any = __any(!(x == 0.0f));
    if (lane == 0) sh.flags[wave] = any;
    lds_barrier();
    return (sh.flags[0] | sh.flags[1] | sh.flags[2] | sh.flags[3]) != 0;
  }
  __device__ __forceinline__ float check_wide() {
    float x = 0;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) x = fmaf(o[t][r], 0.0f, x);
    return x;
  }

  // The item's result: part < 0: to out; else a partial result, of all of the tile's tokens or of some (see work).
  __device__ __forceinline__ void finish_wide(int group, int part, int ends, uint32_t once_more) {
    const int skip = once_more & 255, of = once_more ? once_more >> 8 : it.tokens;
    const int G = a.group.d, r = wave * 32 + (lane & 31), rows = it.tokens * G;
    const bool on = r < rows;
    if (part < 0) {
      const float by = l == 0 ? 0.0f : 1.0f / l;
      const int i = (int)quotient(on ? r : 0, a.group), g = (on ? r : 0) - i * G;
      uint16_t* to = (uint16_t*)a.out + (int64_t)(it.q.row0 + it.i0 + i) * a.os.token + (int64_t)(it.head * G + g) * a.os.head;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int c = 0; c < 4; c += 2) {                           // the two halves of a lane pair hold columns 4 h .. of chunks c and c + 1: they swap, and each has a chunk
          const f32x16& v = o[t];
          const auto x = __builtin_amdgcn_permlane32_swap(pack2<TYPE>(v[c * 4] * by, v[c * 4 + 1] * by), pack2<TYPE>(v[c * 4 + 4] * by, v[c * 4 + 5] * by), false, false);
          const auto y = __builtin_amdgcn_permlane32_swap(pack2<TYPE>(v[c * 4 + 2] * by, v[c * 4 + 3] * by), pack2<TYPE>(v[c * 4 + 6] * by, v[c * 4 + 7] * by), false, false);
          const int col = t * 32 + (c + h) * 8;
          if (on && col < a.D) store_bits(to + col, u32x4{(uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]});
        }
      return;
    }
    float* p = a.ws + part_at(a, group, part, DP);
    if (threadIdx.x == 0) *(u32x4*)p = u32x4{(uint32_t)(1 | ends << 1), (uint32_t)(it.q.row0 + it.i0 - skip), (uint32_t)it.head, (uint32_t)(of * G)};
    if (on) {
      const int at = skip * G + r;
      if (h == 0) p[4 + at] = m, p[4 + a.ws_rows + at] = l;
      float* to = p + 4 + 2 * a.ws_rows + (int64_t)at * DP;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c) *(f32x4*)(to + t * 32 + c * 8 + h * 4) = f32x4{o[t][c * 4], o[t][c * 4 + 1], o[t][c * 4 + 2], o[t][c * 4 + 3]};
    }
  }

  // ---- narrow tiles: up to 16 RT rows

  // Every wave has all rows, and keys of its own: KT of every 4 KT.  They come into its own LDS, K and V each two turns ahead, waited for by count: no barrier, and as soon as a
  // turn's K is read the next but one is on its way.  What the waves have is joined at the end.  (Where keys are read for few rows, memory is what bounds; the loads under way are what counts.)
  __device__ __forceinline__ void run_narrow(int group, int part, int ends, uint32_t once_more, bool& again) {
    constexpr int N = KT / 16, DN = DP / 16, SN32 = DP / 32;
    constexpr int LK = N * SN::NI + (FP8 ? 1 : 0), LV = N * SN::NI;  // loads of a turn
    const int G = a.group.d, col = lane & 15, kg = lane >> 4, rows = it.tokens * G;
    const int k_begin = it.b0 * kAttnKeys, k_end = it.b1 * kAttnKeys;
    Range keys = it.keys;                                          // (this item's share of them)
    keys.lo = keys.lo > k_begin ? keys.lo : k_begin, keys.hi = keys.hi < k_end ? keys.hi : k_end;
    const Range all = it.keys;
    it.keys = keys;
    first_pages(k_begin + wave * KT);
    s16x8 qn[RT][SN32];
    int rlo[RT], rhi[RT];
    float mx[RT], ls[RT];
    f32x4 on[RT][DN];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      const int r = x * 16 + col, rr = r < rows ? r : rows - 1, i = (int)quotient(rr, a.group), g = rr - i * G;
      const uint16_t* from = (const uint16_t*)a.q + (int64_t)(it.q.row0 + it.i0 + i) * a.qs.token + (int64_t)(it.head * G + g) * a.qs.head;
#pragma unroll
      for (int k = 0; k < SN32; ++k) {
        const int c = k * 32 + kg * 8;
        qn[x][k] = s16x8{};
        if (r < rows && c < a.D) qn[x][k] = __builtin_bit_cast(s16x8, load_bits<u32x4>(from + c));
      }
      if (x == RT - 1) {
        asm volatile("" : "+v"(entries));
#pragma unroll
        for (int y = 0; y < RT; ++y)
#pragma unroll
          for (int k = 0; k < SN32; ++k) asm volatile("" : "+v"(qn[y][k]));   // (as in begin)
      }
      const Range mine = seen(a, it.q, it.i0 + i, it.i0 + i);
      rlo[x] = mine.lo, rhi[x] = mine.hi;
      mx[x] = -INFINITY, ls[x] = 0;
#pragma unroll
      for (int t = 0; t < DN; ++t) on[x][t] = f32x4{};
    }
    // keys that all rows see
    const int all_lo = seen(a, it.q, it.i0 + it.tokens - 1, it.i0 + it.tokens - 1).lo, all_hi = seen(a, it.q, it.i0, it.i0).hi;
    float lift[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) lift[x] = kLeastLift;
    clear_lds();
    uint32_t there[2];
    Found place[2][N];
    auto issue_k = [&](int first, int turn) __attribute__((always_inline)) {
      need_pages(first, KT);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        place[turn][n] = find(first + n * 16);
        bring<FP8 ? 1 : 2>(false, place[turn][n], n * 16, lds_at(&sh.own[wave][turn][0][n * 16 * NROW]));
      }
      there[turn] = N == 1 && place[turn][0].side_by_side ? 0xffffu : N == 2 && place[turn][0].side_by_side && place[turn][N - 1].side_by_side ? 0xffffffffu : which<KT>(first);
      if constexpr (FP8) {                                         // lanes 0 .. 31: scales of K, the others: of V
        int page, slot;
        const bool is = where(first + (lane & 31), page, slot);
        const float* from = (lane < 32 ? a.k_scales : a.v_scales) + ((int64_t)page * a.page.d + slot) * a.kv_heads + it.head;
        load_lds4(is ? (const void*)from : (const void*)&kNothing, lds_at(&sh.scales[0][0][0]) + (wave * 2 + turn) * 256);
      }
    };
    auto issue_v = [&](int turn) __attribute__((always_inline)) {   // (of the keys whose K was issued last: their pages' entries are there)
#pragma unroll
      for (int n = 0; n < N; ++n) bring<FP8 ? 1 : 2>(true, place[turn][n], n * 16, lds_at(&sh.own[wave][turn][1][n * 16 * NROW]));
    };
    auto body = [&](int first, int turn, int ahead) __attribute__((always_inline)) {
      const uint8_t *K = sh.own[wave][turn][0], *V = sh.own[wave][turn][1];
      const float* sc = &sh.scales[0][0][0] + (wave * 2 + turn) * 64;
      const uint32_t is = there[turn];
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LV + LK) : "memory");
      f32x4 s[RT][N];
#pragma unroll
      for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int n = 0; n < N; ++n) s[x][n] = f32x4{};
      {
        using Raw = std::conditional_t<FP8, u32x2, u32x4>;
        auto read = [&](int i) __attribute__((always_inline)) {
          const int row = i / SN32 * 16 + col;
          if constexpr (FP8) return *(const u32x2*)(K + ((row * NROW + ((kg >> 1) ^ SN::k(row)) * 16 + (kg & 1) * 8) ^ (i % SN32 * 32)));
          else return *(const u32x4*)(K + ((row * NROW + (kg ^ SN::k(row)) * 16) ^ (i % SN32 * 64)));
        };
        Raw k[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD && i < N * SN32; ++i) k[i] = read(i);
#pragma unroll
        for (int i = 0; i < N * SN32; ++i) {
          s16x8 now;
          if constexpr (FP8) now = widen<TYPE>(k[i % AHEAD]);
          else now = __builtin_bit_cast(s16x8, k[i % AHEAD]);
          in_order();
          if (i + AHEAD < N * SN32) k[i % AHEAD] = read(i + AHEAD);
#pragma unroll
          for (int x = 0; x < RT; ++x) s[x][i / SN32] = mfma16<TYPE>(now, qn[x][i % SN32], s[x][i / SN32]);
        }
      }
      f32x4 vs[N];
      if constexpr (FP8) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const f32x4 ks = *(const f32x4*)(sc + n * 16 + kg * 4);
          vs[n] = *(const f32x4*)(sc + 32 + n * 16 + kg * 4);
#pragma unroll
          for (int x = 0; x < RT; ++x) s[x][n] *= ks;
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // K is read: its place is free
      issue_k(ahead, turn);
      const bool masked = is != (N == 2 ? 0xffffffffu : 0xffffu) || first < all_lo || first + KT > all_hi;
      s16x8 pk[RT];
      float of_all = 0;
      if constexpr (FP8 && TYPE == kF16) {
        if (!masked) {
#pragma unroll
          for (int e = 0; e < 8; ++e) of_all = fmaxf(of_all, fabsf(vs[e >> 2][e & 3]));
          of_all = quarters<Max>(of_all);
        }
      }
#pragma unroll
      for (int x = 0; x < RT; ++x) {
        if (masked) {
#pragma unroll
          for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int k = n * 16 + kg * 4 + e;
              s[x][n][e] = first + k >= rlo[x] && first + k < rhi[x] && (is >> k & 1) ? s[x][n][e] : -INFINITY;
            }
        }
        float top = fmaxf(fmaxf(s[x][0][0], s[x][0][1]), fmaxf(s[x][0][2], s[x][0][3]));
        if constexpr (N == 2) top = fmaxf(top, fmaxf(fmaxf(s[x][N - 1][0], s[x][N - 1][1]), fmaxf(s[x][N - 1][2], s[x][N - 1][3])));
        top = quarters<Max>(top) * a.scale_log2;
        if (__any(top > mx[x] + LAG)) {
          const float grown = fmaxf(mx[x], top), by = grown > mx[x] ? exp2_fast(mx[x] - grown) : 1.0f;
          mx[x] = grown, ls[x] *= by;
#pragma unroll
          for (int t = 0; t < DN; ++t) on[x][t] *= by;
        }
        const float base = mx[x] == -INFINITY ? 0.0f : mx[x];
        float less = LIFT - base, by_s = a.scale_log2;
        if (__builtin_expect(__any(fabsf(base) > kLargeScore), 0)) {
#pragma unroll
          for (int e = 0; e < 4 * N; ++e) s[x][e >> 2][e & 3] = less_maximum(s[x][e >> 2][e & 3], by_s, base);
          less = LIFT, by_s = 1;
        }
        float p[4 * N];
#pragma unroll
        for (int e = 0; e < 4 * N; ++e) p[e] = exp2_fast(fmaf(s[x][e >> 2][e & 3], by_s, less));
        u32x4 w = {};
        if constexpr (FP8) {
          float by = 1, over = 1;
          if constexpr (TYPE == kF16) {
            float most = of_all;
            if (masked) {                                          // (of the keys that the row sees)
              most = 0;
#pragma unroll
              for (int e = 0; e < 8; ++e) most = fmaxf(most, s[x][e >> 2][e & 3] > -INFINITY ? fabsf(vs[e >> 2][e & 3]) : 0.0f);
              most = quarters<Max>(most);
            }
            if (__any(most >= lift[x])) {
              const float to = fmaxf(lift[x], lift_above(most)), down = lift[x] / to;
#pragma unroll
              for (int t = 0; t < DN; ++t) on[x][t] *= down;
              lift[x] = to;
            }
            over = lift[x], by = over_lift(over);
          }
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const float v0 = vs[e >> 2][e & 3], v1 = vs[e >> 2][e & 3 | 1], t0 = p[e] * by * v0, t1 = p[e + 1] * by * v1;
            w[e >> 1] = pack2<TYPE>(t0, t1);
            ls[x] += weight<TYPE>(p[e], t0, v0, half<TYPE>(w[e >> 1], 0), over) + weight<TYPE>(p[e + 1], t1, v1, half<TYPE>(w[e >> 1], 1), over);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            w[e >> 1] = pack2<TYPE>(p[e], p[e + 1]);
            ls[x] = add2<TYPE>(w[e >> 1], ls[x]);
          }
        }
        pk[x] = __builtin_bit_cast(s16x8, w);
      }
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LK + LV) : "memory");
      {
        using Raw = std::conditional_t<FP8, i32x2, s16x4>;
        auto read = [&](int t) __attribute__((always_inline)) {
          if constexpr (FP8) {
            const int j = col >> 1, row = 16 * (j >> 2) + 4 * kg + (j & 3);
            return __builtin_amdgcn_ds_read_tr8_b64_v2i32((tr8_ptr)(V + ((row * NROW + SN::v(row) * 16 + (col & 1) * 8) ^ (t * 16))));
          } else {
            const int row = 4 * kg + (col >> 2);
            return __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(V + ((row * NROW + (((col & 3) >> 1) ^ SN::v(row)) * 16 + (col & 1) * 8) ^ (t * 32))));
          }
        };
        Raw v[AHEAD];
#pragma unroll
        for (int t = 0; t < AHEAD; ++t) v[t] = read(t);
#pragma unroll
        for (int t = 0; t < DN; ++t) {
          const Raw raw = v[t % AHEAD];
          in_order();
          if (t + AHEAD < DN) v[t % AHEAD] = read(t + AHEAD);
          if constexpr (FP8) {
            const s16x8 now = widen<TYPE>(u32x2{(uint32_t)raw[0], (uint32_t)raw[1]});
#pragma unroll
            for (int x = 0; x < RT; ++x) on[x][t] = mfma16<TYPE>(now, pk[x], on[x][t]);
          } else {
#pragma unroll
            for (int x = 0; x < RT; ++x) on[x][t] = mfma16_short<TYPE>(raw, s16x4{pk[x][0], pk[x][1], pk[x][2], pk[x][3]}, on[x][t]);
          }
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      issue_v(turn);
    };
    const int step = 4 * KT, first = k_begin + wave * KT;
    issue_k(first, 0), issue_v(0), issue_k(first + step, 1), issue_v(1);
    for (int at = k_begin; at < k_end; at += 2 * step) {
      body(at + wave * KT, 0, at + wave * KT + 2 * step);
      if (at + step < k_end) body(at + step + wave * KT, 1, at + wave * KT + 3 * step);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    it.keys = all;
    float bad = 0;
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      ls[x] = quarters<Add>(ls[x]);
#pragma unroll
      for (int t = 0; t < DN; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) bad = fmaf(on[x][t][e], 0.0f, bad);
    }
    again = checked(once_more) && not_finite(bad);
    const int skip = once_more & 255, of = once_more ? once_more >> 8 : it.tokens;
    lds_barrier();                                                 // (the turns are free)
    // the waves' results, 16 bytes changing places by the row
    float* mine = (float*)&sh.kv[0][0][0] + wave * (RT * 16 * DP);
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      const int r = x * 16 + col;
      if (kg == 0) sh.top[wave][r] = mx[x], sh.sum[wave][r] = ls[x];
#pragma unroll
      for (int t = 0; t < DN; ++t) *(f32x4*)(mine + r * DP + ((t * 4 + kg) ^ (r & 7)) * 4) = FP8 && TYPE == kF16 ? on[x][t] * lift[x] : on[x][t];
    }
    lds_barrier();
    constexpr int PER = DP / 64;                                   // f32x4 of a thread: 16 threads a row
    float* p = part < 0 ? nullptr : a.ws + part_at(a, group, part, DP);
    if (p && threadIdx.x == 0) *(u32x4*)p = u32x4{(uint32_t)(1 | ends << 1), (uint32_t)(it.q.row0 + it.i0 - skip), (uint32_t)it.head, (uint32_t)(of * G)};
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      const int r = x * 16 + (int)(threadIdx.x >> 4), c = threadIdx.x & 15;
      if (r >= rows) break;
      const float top = fmaxf(fmaxf(sh.top[0][r], sh.top[1][r]), fmaxf(sh.top[2][r], sh.top[3][r])), base = top == -INFINITY ? 0.0f : top;
      float sum = 0;
      f32x4 v[PER];
#pragma unroll
      for (int k = 0; k < PER; ++k) v[k] = f32x4{};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float by = exp2_fast(sh.top[w][r] - base);
        sum += sh.sum[w][r] * by;
#pragma unroll
        for (int k = 0; k < PER; ++k) v[k] += *(const f32x4*)((float*)&sh.kv[0][0][0] + (w * RT * 16 + r) * DP + ((c * PER + k) ^ (r & 7)) * 4) * by;
      }
      if (p) {
        const int at = skip * G + r;
        if (c == 0) p[4 + at] = top, p[4 + a.ws_rows + at] = sum;
#pragma unroll
        for (int k = 0; k < PER; ++k) *(f32x4*)(p + 4 + 2 * a.ws_rows + (int64_t)at * DP + (c * PER + k) * 4) = v[k];
      } else {
        const float by = sum == 0 ? 0.0f : 1.0f / sum;
        const int i = (int)quotient(r, a.group), g = r - i * G;
        uint16_t* to = (uint16_t*)a.out + (int64_t)(it.q.row0 + it.i0 + i) * a.os.token + (int64_t)(it.head * G + g) * a.os.head;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
          const int at = (c * PER + k) * 4;
          if (at < a.D) store_bits(to + at, u32x2{pack2<TYPE>(v[k][0] * by, v[k][1] * by), pack2<TYPE>(v[k][2] * by, v[k][3] * by)});
        }
      }
    }
    lds_barrier();
  }

  // Values of keys that some rows of a tile see and others do not: the product has them in all rows, times 0, which is not 0 if they are not finite.  So where something that is not finite has come
  // out, such keys are looked at: at token i of the tile one may come into sight (its own) and, with a window, one go out of sight.  marks[i]: kEnters, kLeaves: that one's value is not finite; kEntersNaN,
  // kLeavesNaN: and nothing but NaN, so that the tokens which see it need no second pass.  (12000 keys under 128 tokens, 48 heads, us: 84; one value not finite 148, a query 150, all new values NaN 169.  All tokens
  // one by one, as it was: 2100 - 4600.)
  static constexpr uint32_t kEnters = 1, kLeaves = 2, kEntersNaN = 4, kLeavesNaN = 8;
  __device__ __forceinline__ void survey() {
    const int first = it.q.first + it.i0;                          // position of the first token
    const int from = it.keys.lo > it.b0 * kAttnKeys ? it.keys.lo : it.b0 * kAttnKeys, end = it.keys.hi < it.b1 * kAttnKeys ? it.keys.hi : it.b1 * kAttnKeys;
#pragma unroll 1
    for (int i = wave; i < it.tokens; i += 4) {
      uint32_t mark = 0;
#pragma unroll 1
      for (int leaves = 0; leaves < (a.window ? 2 : 1); ++leaves) {
        const int key = leaves ? first + i - a.window : first + i;
        if (key < from || key >= end) continue;
        const int p = (int)quotient(key, a.page), page = a.table[(int64_t)it.s * a.max_pages + p], slot = key - p * (int)a.page.d;
        if ((uint32_t)page >= (uint64_t)a.pages) continue;
        constexpr int EB = FP8 ? 1 : 2;
        const bool in = lane * 16 < a.D * EB;
        u32x4 v = {};
        if (in) v = load_bits<u32x4>((const uint8_t*)a.v_cache + (page * a.vp.page + slot * a.vp.slot + it.head * a.vp.head) * EB + lane * 16);
        bool any = false, all = true;                              // not finite; NaN
#pragma unroll
        for (int k = 0; k < 16 / EB; ++k) {
          const uint32_t x = v[k * EB / 4] >> (k * EB % 4 * 8) & (FP8 ? 0x7f : 0x7fff), top = FP8 ? 0x7f : TYPE == kBf16 ? 0x7f80 : 0x7c00;   // (e4m3: 0x7f is NaN, the rest is finite)
          any |= x >= top, all &= FP8 ? x == top : x > top;
        }
        any = __any(any), all = __all(all || !in);
        if constexpr (FP8) {
          const float sc = a.v_scales[((int64_t)page * a.page.d + slot) * a.kv_heads + it.head];
          any |= !(fabsf(sc) <= (TYPE == kF16 ? 0x1p30f : 3.4028234663852886e38f));   // (fp16: large enough, relative to others, to be an infinity on the way)
          all |= sc != sc;
        }
        if (any) mark |= (kEnters | (all ? kEntersNaN : 0)) << leaves;
      }
      if (lane == 0) sh.marks[i] = (uint8_t)mark;
    }
    lds_barrier();
  }
  // Whether a bit from `from` up to `end` is set.
  static __device__ __forceinline__ bool any_of(const uint64_t (&b)[2], int from, int end) {
    auto below = [](int n) __attribute__((always_inline)) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; };
    return (b[0] & below(end) & ~below(from)) | (b[1] & below(end - 64) & ~below(from - 64));
  }
  // The next of a tile's `tokens` from token `from` on, as many as see the same of the marked keys, that do not see one of them, unless they see one that is NaN all through: `first`, and how many; 0: no more.
  __device__ __forceinline__ int spoilt(int tokens, int from, int& first) {
    const uint32_t m0 = lane < tokens ? sh.marks[lane] : 0, m1 = 64 + lane < tokens ? sh.marks[64 + lane] : 0;
    auto bits = [&](uint32_t kind, uint64_t (&b)[2]) __attribute__((always_inline)) { b[0] = __ballot((m0 & kind) != 0), b[1] = __ballot((m1 & kind) != 0); };
    uint64_t enters[2], leaves[2], enters_nan[2], leaves_nan[2], changes[2];
    bits(kEnters, enters), bits(kLeaves, leaves), bits(kEntersNaN, enters_nan), bits(kLeavesNaN, leaves_nan), bits(kEnters | kLeaves, changes);
    const int window = a.window && a.window < tokens ? a.window : tokens;
    int next;
    for (first = from; first < tokens; first = next) {
      for (next = first + 1; next < tokens && !any_of(changes, next, next + 1);) ++next;
      const bool unseen = any_of(leaves, 0, first + 1) || any_of(enters, first + 1, tokens);
      const bool lost = any_of(enters_nan, first - window + 1, first + 1) || any_of(leaves_nan, first + 1, first + window + 1);
      if (unseen && !lost) return next - first;
    }
    return 0;
  }
  __device__ __forceinline__ void work(int group, int part, int ends) {
    // 0: all of the tile's tokens; else some of them once more: how many the tile has, and the first of these.  (One register for the loop over the keys, which has none to spare.)
    uint32_t once_more = 0;
    for (bool again = false;;) {
      if constexpr (RT > 0) run_narrow(group, part, ends, once_more, again);
      else {
        run_wide();
        again = checked(once_more) && not_finite(check_wide());
        lds_barrier();                                             // (the stages are free)
        finish_wide(group, part, ends, once_more);
      }
      if (__builtin_expect(!once_more && !again, 1)) return;
      int skip = once_more & 255, n = it.tokens, first;
      const int tokens = once_more ? once_more >> 8 : n;
      if (!once_more) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (what is done again is written again, by other waves)
        survey();
        n = 0;
      }
      it.i0 -= skip;
      n = __builtin_amdgcn_readfirstlane(spoilt(tokens, skip + n, first)), skip = __builtin_amdgcn_readfirstlane(first);
      if (n == 0) return;
      once_more = tokens << 8 | skip, it.i0 += skip, it.tokens = n, it.keys = seen(a, it.q, it.i0, it.i0 + n - 1);
    }
  }
  // Whether the tokens see different keys, and it has not been looked at yet what those hold.
  __device__ __forceinline__ bool checked(uint32_t once_more) const { return !once_more && a.causal && it.tokens > 1; }

  __device__ __forceinline__ void tile(int tile, int tokens) {
    it.i0 = tile * tokens;
    it.tokens = it.i0 + tokens < it.q.n ? tokens : it.q.n - it.i0;
    it.keys = seen(a, it.q, it.i0, it.i0 + it.tokens - 1);
  }

  // Sum of v over the workgroup's threads before this one, and of all.
  __device__ __forceinline__ int64_t scan(int64_t v, int64_t& total) {
    int64_t x = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    lds_barrier();
    if (lane == 63) sh.sums[wave] = x;
    lds_barrier();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) before += sh.sums[w];
      total += sh.sums[w];
    }
    return before + x - v;
  }

  // Every workgroup a tile, the last of a sequence first (they see the most keys); a head's tiles go to workgroups that share an XCD where 8 divides the heads.
  __device__ __forceinline__ void whole_tiles() {
    const int tokens = ROWS / a.group.d;
    const int64_t number = a.t0 + blockIdx.x, want = number / a.kv_heads;
    it.head = (int)(number - want * a.kv_heads);
    int t;
    if (a.S <= 64) {                                               // a lane each, in every wave
      Seq mine = {0, 0, 0, 0};
      if (lane < a.S) mine = sequence(a, lane);
      const int n = tiles_of(a, mine, tokens);
      int upto = n;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
      }
      const int64_t at = __builtin_amdgcn_readlane(upto, 63) - 1 - want;
      if (at < 0) return;
      upto -= n;
      it.s = __popcll(__ballot(lane < a.S && upto <= at)) - 1;     // (the last that begins there or before: it has tiles)
      it.q = {__builtin_amdgcn_readlane(mine.row0, it.s), __builtin_amdgcn_readlane(mine.n, it.s), __builtin_amdgcn_readlane(mine.first, it.s), __builtin_amdgcn_readlane(mine.len, it.s)};
      t = (int)at - __builtin_amdgcn_readlane(upto, it.s);
    } else {
      // Places are counted so that a sequence's first follows from its first row alone: rows / tokens + the sequences before.  One place of a sequence may have no tile.
      const int64_t at = a.T / tokens + a.S - 1 - want;
      auto first_place = [&](int s) __attribute__((always_inline)) {
        return (int64_t)((uint32_t)border(a, a.seq_rows[s]) / (uint32_t)tokens) + s;
      };
      const int s = at < 0 ? a.S : ended(a.S, [&](int i) __attribute__((always_inline)) { return first_place(i + 1) <= at; });
      if (s >= a.S) return;
      it.s = s, it.q = sequence(a, s);
      const int64_t place = at - first_place(s);
      if (place < 0 || place >= tiles_of(a, it.q, tokens)) return;
      t = __builtin_amdgcn_readfirstlane((int)place);
    }
    tile(t, tokens);
    const Blocks b = blocks_of(it.keys);
    it.b0 = b.first, it.b1 = b.first + b.count;
    work(0, -1, 0);
  }

  static __device__ __forceinline__ int64_t over(int64_t x, int64_t y) { return (x | y) >> 31 ? x / y : (int64_t)((uint32_t)x / (uint32_t)y); }   // (not negative)

  // A place in the list of all blocks.
  struct Spot {
    Seq q;
    Cost c;
    int s, head, pair, at;                                         // block of the pair
  };
  __device__ __forceinline__ Spot spot(int64_t u, int s, const Seq& q, int64_t before, int tokens) {
    Spot p;
    p.s = __builtin_amdgcn_readfirstlane(s);
    p.q = q;
    p.c = cost_of(a, p.q, tokens);
    const int64_t of_head = (int64_t)p.c.pairs * p.c.cell;
    int64_t rest = u - before;
    p.head = __builtin_amdgcn_readfirstlane((int)over(rest, of_head));
    rest -= p.head * of_head;
    p.pair = __builtin_amdgcn_readfirstlane((int)over(rest, p.c.cell));
    p.at = __builtin_amdgcn_readfirstlane((int)(rest - (int64_t)p.pair * p.c.cell));
    return p;
  }
  // By how much a border there is moved.
  __device__ __forceinline__ int64_t moved(const Spot& p, int tokens, int64_t near) {
    const int tiles = tiles_of(a, p.q, tokens), last = tiles - 1 - p.pair;
    const int n0 = tile_blocks(a, p.q, tokens, p.pair).count, n1 = last > p.pair ? tile_blocks(a, p.q, tokens, last).count : 0;
    if (p.at <= near) return -p.at;
    if (p.at - n0 <= near && n0 - p.at <= near) return n0 - p.at;
    if (n0 + n1 - p.at <= near) return p.c.cell - p.at;
    return 0;
  }

  // A run of the list of all blocks.
  __device__ __forceinline__ void split() {
    const int tokens = ROWS / a.group.d, groups = a.groups;
    // neighbours in the list share keys: they go to one XCD
    const int group = (int)(blockIdx.x & 7) * (groups >> 3) + (int)(blockIdx.x >> 3);
    int64_t* before = (int64_t*)&sh.kv[0][0][0];                   // of the sequences, in blocks of one head
    int64_t carry = 0;
    // Up to 64 sequences: a lane each, in every wave.
    Seq mine = {0, 0, 0, 0};
    int upto = 0;
    bool few = a.S <= 64;
    if (few) {
      Cost c = {0, 0};
      if (lane < a.S) mine = sequence(a, lane), c = cost_of(a, mine, tokens);
      const int64_t v = (int64_t)c.pairs * c.cell;
      few = !__any(v >> 24);
      upto = (int)v;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
      }
      carry = few ? __builtin_amdgcn_readlane(upto, 63) : 0;
      upto -= (int)v;                                              // before this lane's
    }
    if (!few) {
      for (int base = 0; base < a.S; base += 256) {
        const int s = base + (int)threadIdx.x;
        Cost c = {0, 0};
        if (s < a.S) c = cost_of(a, sequence(a, s), tokens);
        int64_t total;
        const int64_t at = scan((int64_t)c.pairs * c.cell, total);
        if (s < a.S) before[s] = carry + at;
        carry += total;
      }
      lds_barrier();
    }
    const int64_t all = carry * a.kv_heads;
    // Each of them has a block at least (parts of a tile lie in neighbouring workgroups' places); of wide tiles four, where that makes 128 of them: a partial result takes as long as a block or two.
    int64_t busy = RT || all < 512 ? all : all / 4;
    busy = RT == 0 && all < 512 && busy > 128 ? 128 : busy < groups ? busy : groups;
    int wrote = 0;                                                 // parts
    auto done = [&]() __attribute__((always_inline)) {
      if (threadIdx.x < 2 && !(wrote >> threadIdx.x & 1)) *(uint32_t*)(a.ws + part_at(a, group, threadIdx.x, DP)) = 0;
    };
    if (group >= busy) return done();
    int64_t u = over(all * group, busy), end = over(all * (group + 1), busy);
    // Wide tiles: a border near a tile's is moved there, and the tile is not cut.  (Both sides of a border come to the same.)
    const int64_t share = over(all, busy), near = share / 32 + 1 + (share >= 16);
    const bool snap = RT == 0 && share >= 8;
    Spot at, e;
    if (few) {
      auto find = [&](int64_t where) __attribute__((always_inline)) {
        const int s = __popcll(__ballot(lane < a.S && (int64_t)upto * a.kv_heads <= where)) - 1;   // (the last that begins there or before: it has blocks, or `where` is the end)
        const Seq q = {__builtin_amdgcn_readlane(mine.row0, s), __builtin_amdgcn_readlane(mine.n, s), __builtin_amdgcn_readlane(mine.first, s), __builtin_amdgcn_readlane(mine.len, s)};
        return spot(where, s, q, (int64_t)__builtin_amdgcn_readlane(upto, s) * a.kv_heads, tokens);
      };
      at = find(u);
      if (snap && end < all) e = find(end);
    } else {
      for (int s = threadIdx.x; s < a.S; s += 256) {
        const int64_t from = before[s] * a.kv_heads, to = (s + 1 < a.S ? before[s + 1] : carry) * a.kv_heads;
        if (from <= u && u < to) sh.found[0] = s, sh.found[1] = from;
        if (from <= end && end < to) sh.found[2] = s, sh.found[3] = from;
      }
      lds_barrier();
      auto find = [&](int64_t where, int k) __attribute__((always_inline)) {
        const int s = __builtin_amdgcn_readfirstlane((int)sh.found[k]);
        return spot(where, s, sequence(a, s), sh.found[k + 1], tokens);
      };
      at = find(u, 0);
      if (snap && end < all) e = find(end, 2);
      lds_barrier();
    }
    if (snap && end < all) end += moved(e, tokens, near);
    if (snap && u > 0) {
      const int64_t by = moved(at, tokens, near);
      u += by, at.at += (int)by;
    }
    it.s = at.s, it.q = at.q, it.head = at.head;
    Cost c = at.c;
    int pair = at.pair, in_pair = at.at;
    while (u < end) {
      const int tiles = tiles_of(a, it.q, tokens), lastt = tiles - 1 - pair;
      const int n0 = tile_blocks(a, it.q, tokens, pair).count, n1 = lastt > pair ? tile_blocks(a, it.q, tokens, lastt).count : 0;
      if (in_pair < n0 + n1) {
        const bool second = in_pair >= n0;
        tile(second ? lastt : pair, tokens);
        const Blocks b = blocks_of(it.keys);
        const int from = second ? in_pair - n0 : in_pair;
        const int64_t left = end - u;
        const int to = b.count - from <= left ? b.count : from + (int)left;
        it.b0 = b.first + from, it.b1 = b.first + to;
        const bool starts = from == 0, ends = to == b.count;
        work(group, starts && ends ? -1 : starts ? 1 : 0, ends);
        if (!(starts && ends)) wrote |= starts ? 2 : 1;
        u += to - from, in_pair += to - from;
      }
      if (in_pair >= n0 + n1) {                                         // the next pair, head, sequence
        u += c.cell - in_pair, in_pair = 0;
        if (u >= end) break;
        if (++pair == c.pairs) {
          pair = 0;
          if (++it.head == a.kv_heads) {
            it.head = 0;
            do {
              if (++it.s >= a.S) return done();
              it.q = sequence(a, it.s);
              c = cost_of(a, it.q, tokens);
            } while (c.pairs == 0);
          }
        }
      }
    }
    done();
  }
};

template <int TYPE, bool FP8, int DP, int RT, bool SPLIT>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void cache_attention_kernel(CacheArgs a) {
  using A = Attention<TYPE, FP8, DP, RT>;
  __shared__ typename A::Shared sh;
  fetch_arguments(a.q, a.k_scales, a.qs.token, a.kp.page, a.T, a.S, a.page.by.mul, a.type);
  A w(a, sh);
  if constexpr (SPLIT) w.split();
  else w.whole_tiles();
}

// By types and columns.
template <int RT, bool SPLIT, int TYPE, bool FP8>
void launch_attention_columns(const CacheArgs& a, uint32_t groups, hipStream_t s) {
  const int dp = attn_columns(a.D);
  if (dp == 64) cache_attention_kernel<TYPE, FP8, 64, RT, SPLIT><<<groups, 256, 0, s>>>(a);
  else if (dp == 128) cache_attention_kernel<TYPE, FP8, 128, RT, SPLIT><<<groups, 256, 0, s>>>(a);
  else cache_attention_kernel<TYPE, FP8, 256, RT, SPLIT><<<groups, 256, 0, s>>>(a);
}
template <int RT, bool SPLIT>
void launch_attention(const CacheArgs& a, uint32_t groups, hipStream_t s) {
  if (a.type == kBf16) a.fp8 ? launch_attention_columns<RT, SPLIT, kBf16, true>(a, groups, s) : launch_attention_columns<RT, SPLIT, kBf16, false>(a, groups, s);
  else a.fp8 ? launch_attention_columns<RT, SPLIT, kF16, true>(a, groups, s) : launch_attention_columns<RT, SPLIT, kF16, false>(a, groups, s);
}

}  // namespace axe
