// Attention of new tokens over a paged cache (axe_cache_attention).  gfx950 only.
//
//   o[t, h] = sum_j softmax_j(scale q[t, h] . K[j]) V[j]
//
// A tile is 128 rows: the query heads of one head of the cache, of consecutive new tokens of one sequence (row r: token r / G, head r mod G), so that one pass over the keys
// serves all of them.  A workgroup of four waves takes a tile's keys 64 at a time: K and V of the 64 go straight from their pages to LDS (two blocks of LDS, one filled while the
// other is read), and every wave has 32 rows for itself:
//   S^T = K Q^T      a lane holds 32 of the 64 scores of one row, lane + 32 the others: maximum and sum of a row are a chain in the lane and one exchange;
//   O^T += V^T P^T   the scores' registers, in 16 bits, are the product's operand as they are: its contraction runs over the keys in the order in which the registers hold them, and V comes out of LDS in
//                    that order by transposing reads.
// The maximum is a running one: when it grows, sums and O are multiplied down.  Everything but the products' operands is fp32.
//
// Where a batch has few tiles, the list of all (tile, block of keys) is cut into as many equal runs as there are workgroups, wherever that falls; a tile that is cut leaves partial
// results (maximum, sum, O) in the workspace, and a second kernel joins them, in the order of the keys.  Which run a workgroup has follows from the lengths alone: results repeat
// their bits.
#include <hip/hip_runtime.h>

#include "cache_ops.h"
#include "cache_tables.h"
#include "gemm_common.h"
#include "row_ops.h"

namespace axe {

namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((address_space(3))) s16x4* tr_ptr;

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
__device__ __forceinline__ float other_half(float v) {              // of lane ^ 32
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float((threadIdx.x & 32) ? s[0] : s[1]);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// 16 bytes that are zero: what a lane brings to LDS for a key that is not there.
__device__ const u32x4 kNothing = {0, 0, 0, 0};

// Loads into LDS, 16 bytes a lane: the wave's 1024 bytes from `lds` on.  (Written as asm: the compiler would wait for them before it reads any of LDS.  M0 holds the address;
// the wait states are for registers that a vector instruction may just have written.)
__device__ __forceinline__ void load_lds(const void* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(lds) : "memory");
}
__device__ __forceinline__ void load_lds(uint32_t offset, const void* base, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(lds) : "memory");
}

// ---- the batch

struct Seq {
  int row0, n;                     // its rows
  int first;                       // position of its first new token
  int len;                         // keys
};
__device__ __forceinline__ Seq sequence(const CacheArgs& a, int s) {
  const int T = (int)a.T, b0 = a.seq_rows[s], b1 = a.seq_rows[s + 1], l = a.lengths[s];
  Seq q;
  q.row0 = b0 < 0 ? 0 : b0 > T ? T : b0;
  const int end = b1 > T ? T : b1;
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

}  // namespace

// ---- the kernel

template <int TYPE, bool FP8, int DP>
struct Attention {
  static constexpr int ROW = DP * 2;                               // bytes of a key in LDS
  static constexpr int BLOCK = kAttnKeys * ROW;                    // of K, or V, of a block
  static constexpr int CH = DP / 8;                                // 16-byte chunks of a row
  static constexpr int NI = 16 * ROW / 1024;                       // loads of a wave for its 16 keys of K, or V
  static constexpr int RPI = 64 / CH;                              // keys of a load
  static constexpr int STEPS = DP / 16, DT = DP / 32;
  // exp2 of this is added to the softmax's terms: fp16 has few of them below 1
  static constexpr float LIFT = TYPE == kBf16 ? 0.0f : FP8 ? 8.0f : 15.0f;

  struct Shared {
    __attribute__((aligned(16))) uint8_t kv[2][2][BLOCK];          // [stage][K, V]
    float scales[2][2][kAttnKeys];
    uint16_t there[2][4];                                          // of a wave's 16 keys: which there are
    int flags[4];
    int64_t sums[8];
    int64_t found[4];
  };

  const CacheArgs& a;
  Shared& sh;
  const int lane, wave, h;
  Item it;

  s16x8 q[STEPS];
  f32x16 o[DT];
  float m, l;                                                      // running maximum (scaled) and this lane's part of the sum
  int lo, hi;                                                      // keys that this lane's row sees
  int w_lo, w_hi_all, w_lo_all, w_hi;                              // of the wave's rows: seen by any, by all
  bool rows_here;
  float lift_v;                                                    // e4m3 values in fp16: what their scales are divided by, a power of two

  // keys on their way
  int entry[NI];
  u32x2 kreg[FP8 ? NI : 1], vreg[FP8 ? NI : 1];
  float sreg[2];

  __device__ __forceinline__ Attention(const CacheArgs& a_, Shared& s_) : a(a_), sh(s_), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), h((threadIdx.x >> 5) & 1) {}

  static __device__ __forceinline__ uint32_t k_slot(int row, int chunk) { return (uint32_t)(chunk ^ (row & 7)); }
  static __device__ __forceinline__ uint32_t v_slot(int row, int chunk) { return (uint32_t)(chunk ^ ((row & 3) << 1)); }
  __device__ __forceinline__ uint32_t lds_of(int stage, int which) const { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&sh.kv[stage][which][0]; }

  __device__ __forceinline__ int key_of(int block, int i) const { return block * kAttnKeys + wave * 16 + i * RPI + lane / CH; }

  // Page entries of a block's keys.
  __device__ __forceinline__ void fetch_entries(int block) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int key = key_of(block, i);
      entry[i] = -1;
      if (key >= it.keys.lo && key < it.keys.hi) entry[i] = a.table[(int64_t)it.s * a.max_pages + quotient(key, a.page)];
    }
  }
  // Starts the loads of a block into a stage (e4m3: into registers).
  __device__ __forceinline__ void issue(int block, int stage) {
    uint32_t there = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int key = key_of(block, i), row = wave * 16 + i * RPI + lane / CH, slot = lane % CH;
      const bool on = (uint32_t)entry[i] < (uint64_t)a.pages;
      there |= on ? 1u << (i * RPI + lane / CH) : 0u;
      const int place = on ? key - (int)(quotient(key, a.page) * a.page.d) : 0;
      const int64_t kat = entry[i] * a.kp.page + place * a.kp.slot + it.head * a.kp.head, vat = entry[i] * a.vp.page + place * a.vp.slot + it.head * a.vp.head;
      const int kc = (int)k_slot(row, slot) * 8, vc = (int)v_slot(row, slot) * 8;
      if constexpr (!FP8) {
        const void* kp = on && kc < a.D ? (const void*)((const uint16_t*)a.k_cache + kat + kc) : (const void*)&kNothing;
        const void* vp = on && vc < a.D ? (const void*)((const uint16_t*)a.v_cache + vat + vc) : (const void*)&kNothing;
        load_lds(kp, lds_of(stage, 0) + (wave * 16 + i * RPI) * ROW);
        load_lds(vp, lds_of(stage, 1) + (wave * 16 + i * RPI) * ROW);
      } else {
        kreg[i] = vreg[i] = u32x2{};
        if (on && kc < a.D) kreg[i] = *(const u32x2*)((const uint8_t*)a.k_cache + kat + kc);
        if (on && vc < a.D) vreg[i] = *(const u32x2*)((const uint8_t*)a.v_cache + vat + vc);
      }
    }
    if constexpr (FP8) {                                           // the scales: lane i of a wave has key i of its sixteen
      const int key = block * kAttnKeys + wave * 16 + (lane & 15);
      sreg[0] = sreg[1] = 0;
      if (lane < 16 && key >= it.keys.lo && key < it.keys.hi) {
        const uint32_t pi = quotient(key, a.page);
        const int pg = a.table[(int64_t)it.s * a.max_pages + pi];
        if ((uint32_t)pg < (uint64_t)a.pages) {
          const int64_t at = ((int64_t)pg * a.page.d + (key - (int)(pi * a.page.d))) * a.kv_heads + it.head;
          sreg[0] = a.k_scales[at], sreg[1] = a.v_scales[at];
        }
      }
    }
    there = (uint32_t)__builtin_amdgcn_readfirstlane((int)wave_or(there));
    if (lane == 0) sh.there[stage][wave] = (uint16_t)there;
  }
  static __device__ __forceinline__ uint32_t wave_or(uint32_t v) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v |= (uint32_t)__shfl_xor((int)v, d);
    return v;
  }
  // e4m3: the block in registers becomes 16 bits in LDS.
  __device__ __forceinline__ void settle(int stage) {
    if constexpr (FP8) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const uint32_t at = (wave * 16 + i * RPI) * ROW + lane * 16;
        *(u32x4*)&sh.kv[stage][0][at] = widen(kreg[i]);
        *(u32x4*)&sh.kv[stage][1][at] = widen(vreg[i]);
      }
      if (lane < 16) sh.scales[stage][0][wave * 16 + lane] = sreg[0], sh.scales[stage][1][wave * 16 + lane] = sreg[1];
    }
  }
  static __device__ __forceinline__ u32x4 widen(u32x2 v) {         // (e4m3 has fewer bits than either type: exact)
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const auto x = __builtin_amdgcn_cvt_pk_f32_fp8(v[i], false), y = __builtin_amdgcn_cvt_pk_f32_fp8(v[i], true);
      r[2 * i] = pack2<TYPE>(x[0], x[1]), r[2 * i + 1] = pack2<TYPE>(y[0], y[1]);
    }
    return r;
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
    const Range mine = seen(a, it.q, it.i0 + i, it.i0 + i);
    lo = mine.lo, hi = mine.hi;
    const int last = rows - 1 < wave * 32 + 31 ? rows - 1 : wave * 32 + 31;
    const Range f = seen(a, it.q, it.i0 + (int)quotient(rows_here ? wave * 32 : 0, a.group), it.i0 + (int)quotient(rows_here ? wave * 32 : 0, a.group));
    const Range b = seen(a, it.q, it.i0 + (int)quotient(last, a.group), it.i0 + (int)quotient(last, a.group));
    w_lo = f.lo, w_lo_all = b.lo, w_hi_all = f.hi, w_hi = b.hi;    // (both ends grow with the token)
    m = -INFINITY, l = 0, lift_v = 1;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = f32x16{};
  }

  // A block's share of the wave's rows, from a stage.
  __device__ __forceinline__ void compute(int block, int stage) {
    const int k0 = block * kAttnKeys;
    if (!rows_here || k0 >= w_hi || k0 + kAttnKeys <= w_lo) return;
    const uint64_t there = *(const uint64_t*)&sh.there[stage][0];
    const uint32_t t0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)there), t1 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(there >> 32));
    const bool masked = (t0 & t1) != 0xffffffffu || k0 < w_lo_all || k0 + kAttnKeys > w_hi_all;
    const uint8_t *K = sh.kv[stage][0], *V = sh.kv[stage][1];
    f32x16 s[2] = {f32x16{}, f32x16{}};
    {
      const uint32_t at = (lane & 31) * ROW + k_slot(lane & 31, h) * 16;
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
#pragma unroll
        for (int t = 0; t < 2; ++t) s[t] = mfma32<TYPE>(*(const s16x8*)(K + ((at ^ (k * 32)) + t * 32 * ROW)), q[k], s[t]);
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
    const float grown = fmaxf(m, top);
    if (__any(grown > m)) {
      const float by = grown > m ? exp2_fast(m - grown) : 1.0f;    // (the first time: m is -inf, the sums are 0)
      m = grown, l *= by;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= by;
    }
    const float less = LIFT - (m == -INFINITY ? 0.0f : m);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[t][r] = exp2_fast(fmaf(s[t][r], a.scale_log2, less));
        l += s[t][r];
      }
    if constexpr (FP8) {
      float sv = sh.scales[stage][1][lane];
      float by = 1;
      if constexpr (TYPE == kF16) {                                // terms times scales stay in fp16's range: the scales relative to a power of two that the largest so far is below
        float most = wave_all<Max>(fabsf(sv) <= 3.0e38f ? fabsf(sv) : 0.0f);
        if (most > lift_v) {
          const float to = __uint_as_float((__float_as_uint(most) & 0x7f800000u) + 0x800000u);
          const float down = lift_v / to;
#pragma unroll
          for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[t][r] *= down;
          lift_v = to;
        }
        by = 1.0f / lift_v;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const f32x4 sc = *(const f32x4*)&sh.scales[stage][1][t * 32 + r * 8 + h * 4];
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t][r * 4 + e] *= sc[e] * by;
        }
    }
    s16x8 p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack2<TYPE>(s[k >> 1][(k & 1) * 8 + 2 * e], s[k >> 1][(k & 1) * 8 + 2 * e + 1]);
      p[k] = __builtin_bit_cast(s16x8, w);
    }
    // lane i of 16 points at 4 columns of key i / 4 and receives 4 keys of column i
    const int i = lane & 15, row = h * 4 + (i >> 2);
    const uint32_t at = row * ROW + v_slot(row, ((lane >> 4) & 1) * 2 + ((i & 3) >> 1)) * 16 + (i & 1) * 8;
    auto values = [&](int t, int k) __attribute__((always_inline)) {
      const uint8_t* v0 = V + ((at ^ (t * 64)) + k * 16 * ROW);
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)v0), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(v0 + 8 * ROW));
      return s16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    };
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[t] = mfma32<TYPE>(values(t, k), p[k], o[t]);
  }

  // All blocks of the item, for the rows of all waves.
  __device__ __forceinline__ void run() {
    begin();
    fetch_entries(it.b0);
    issue(it.b0, 0);
    if (it.b0 + 1 < it.b1) fetch_entries(it.b0 + 1);
    for (int b = it.b0; b < it.b1; ++b) {
      const int stage = (b - it.b0) & 1;
      settle(stage);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      lds_barrier();
      if (b + 1 < it.b1) {
        issue(b + 1, stage ^ 1);
        if (b + 2 < it.b1) fetch_entries(b + 2);
      }
      compute(b, stage);
    }
    l += other_half(l);
    if constexpr (FP8 && TYPE == kF16) {
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= lift_v;
    }
  }
  // Whether a value that is not finite came out, in any row of the workgroup.
  __device__ __forceinline__ bool not_finite() {
    float x = 0;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) x = fmaf(o[t][r], 0.0f, x);
    const bool any = __any(!(x == 0.0f));
    if (lane == 0) sh.flags[wave] = any;
    lds_barrier();
    const bool all = (sh.flags[0] | sh.flags[1] | sh.flags[2] | sh.flags[3]) != 0;
    return all;
  }

  // The item's result: part < 0: to out; else a partial result, of which these are the tokens from `skip` on.
  __device__ __forceinline__ void finish(int group, int part, int ends, int skip, int of) {
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

  // Values of keys that some rows of a tile see and others do not: the product has them in all rows, times 0, which is not 0 if they are not finite.  So where something that is not finite has come
  // out, the tokens are done one by one: a token's rows see the same keys, and the others are zeros in LDS.
  __device__ __forceinline__ void work(int group, int part, int ends) {
    const int i0 = it.i0, tokens = it.tokens;
    for (int i = -1; i < tokens; ++i) {
      if (i >= 0) it.i0 = i0 + i, it.tokens = 1, it.keys = seen(a, it.q, it.i0, it.i0);
      run();
      const bool again = i < 0 && a.causal && tokens > 1 && not_finite();
      lds_barrier();                                               // (the stages are free)
      if (again) continue;
      finish(group, part, ends, i < 0 ? 0 : i, tokens);
      if (i < 0) break;
    }
  }

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
    __syncthreads();
    if (lane == 63) sh.sums[wave] = x;
    __syncthreads();
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
    const int tokens = kAttnRows / a.group.d;
    const int64_t number = a.t0 + blockIdx.x, want = number / a.kv_heads;
    it.head = (int)(number - want * a.kv_heads);
    int64_t carry = 0;
    if (threadIdx.x == 0) sh.found[0] = -1;
    for (int base = 0; base < a.S; base += 256) {                  // sequences from the last on
      const int s = a.S - 1 - base - (int)threadIdx.x;
      const int n = s >= 0 ? tiles_of(a, sequence(a, s), tokens) : 0;
      int64_t total;
      const int64_t before = carry + scan(n, total);
      if (want >= before && want < before + n) sh.found[0] = s, sh.found[1] = n - 1 - (want - before);
      carry += total;
      __syncthreads();
      if (want < carry) break;
    }
    const int s = __builtin_amdgcn_readfirstlane((int)sh.found[0]), t = __builtin_amdgcn_readfirstlane((int)sh.found[1]);
    if (s < 0) return;
    it.s = s;
    it.q = sequence(a, s);
    tile(t, tokens);
    const Blocks b = blocks_of(it.keys);
    it.b0 = b.first, it.b1 = b.first + b.count;
    work(0, -1, 0);
  }

  // A run of the list of all blocks.
  __device__ __forceinline__ void split() {
    const int tokens = kAttnRows / a.group.d, groups = a.groups;
    // neighbours in the list share keys: they go to one XCD
    const int group = (int)(blockIdx.x & 7) * (groups >> 3) + (int)(blockIdx.x >> 3);
    int64_t* before = (int64_t*)&sh.kv[0][0][0];                   // of the sequences, in blocks of one head
    int64_t carry = 0;
    for (int base = 0; base < a.S; base += 256) {
      const int s = base + (int)threadIdx.x;
      Cost c = {0, 0};
      if (s < a.S) c = cost_of(a, sequence(a, s), tokens);
      int64_t total;
      const int64_t at = scan((int64_t)c.pairs * c.cell, total);
      if (s < a.S) before[s] = carry + at;
      carry += total;
    }
    if (threadIdx.x < 2) *(u32x4*)(a.ws + part_at(a, group, threadIdx.x, DP)) = u32x4{};
    __syncthreads();
    const int64_t all = carry * a.kv_heads;
    const int64_t busy = all < groups ? all : groups;              // (each of them has a block at least: parts of a tile lie in neighbouring workgroups' places)
    if (group >= busy) return;
    int64_t u = all * group / busy;
    const int64_t end = all * (group + 1) / busy;
    for (int s = threadIdx.x; s < a.S; s += 256) {
      const int64_t to = s + 1 < a.S ? before[s + 1] : carry;
      if (before[s] * a.kv_heads <= u && u < to * a.kv_heads) sh.found[0] = s, sh.found[1] = before[s];
    }
    __syncthreads();
    int s = __builtin_amdgcn_readfirstlane((int)sh.found[0]);
    int64_t rest = u - sh.found[1] * a.kv_heads;
    __syncthreads();
    it.s = s, it.q = sequence(a, s);
    Cost c = cost_of(a, it.q, tokens);
    int64_t of_head = (int64_t)c.pairs * c.cell;
    it.head = __builtin_amdgcn_readfirstlane((int)(rest / of_head));
    rest -= it.head * of_head;
    int pair = __builtin_amdgcn_readfirstlane((int)(rest / c.cell)), at = __builtin_amdgcn_readfirstlane((int)(rest - (int64_t)pair * c.cell));
    while (u < end) {
      const int tiles = tiles_of(a, it.q, tokens), lastt = tiles - 1 - pair;
      const int n0 = tile_blocks(a, it.q, tokens, pair).count, n1 = lastt > pair ? tile_blocks(a, it.q, tokens, lastt).count : 0;
      if (at < n0 + n1) {
        const bool second = at >= n0;
        tile(second ? lastt : pair, tokens);
        const Blocks b = blocks_of(it.keys);
        const int from = second ? at - n0 : at;
        const int64_t left = end - u;
        const int to = b.count - from <= left ? b.count : from + (int)left;
        it.b0 = b.first + from, it.b1 = b.first + to;
        const bool starts = from == 0, ends = to == b.count;
        work(group, starts && ends ? -1 : starts ? 1 : 0, ends);
        u += to - from, at += to - from;
      }
      if (at >= n0 + n1) {                                         // the next pair, head, sequence
        u += c.cell - at, at = 0;
        if (u >= end) break;
        if (++pair == c.pairs) {
          pair = 0;
          if (++it.head == a.kv_heads) {
            it.head = 0;
            do {
              if (++it.s >= a.S) return;
              it.q = sequence(a, it.s);
              c = cost_of(a, it.q, tokens);
            } while (c.pairs == 0);
          }
        }
      }
    }
  }
};

template <int TYPE, bool FP8, int DP, bool SPLIT>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void cache_attention_kernel(CacheArgs a) {
  using A = Attention<TYPE, FP8, DP>;
  __shared__ typename A::Shared sh;
  A w(a, sh);
  if constexpr (SPLIT) w.split();
  else w.whole_tiles();
}

// Partial results of one tile: the workgroup that began it, then the workgroups behind it up to the one that ended it.  A wave joins a row.
template <int TYPE, int DP>
__global__ __launch_bounds__(256) void cache_attention_join_kernel(CacheArgs a) {
  constexpr int PER = DP / 64;
  const int group = blockIdx.x, lane = threadIdx.x & 63;
  const uint32_t* head = (const uint32_t*)(a.ws + part_at(a, group, 1, DP));
  if (!head[0]) return;
  const int token = (int)head[1], kv_head = (int)head[2], rows = (int)head[3];
  for (int r = blockIdx.y * 4 + (int)(threadIdx.x >> 6); r < rows; r += gridDim.y * 4) {
    float m = -INFINITY, l = 0, o[PER] = {};
    for (int g = group, which = 1;; ++g, which = 0) {
      if (g >= a.groups) break;
      const float* p = a.ws + part_at(a, g, which, DP);
      const uint32_t flags = ((const uint32_t*)p)[0];
      if (!flags) break;
      const float pm = p[4 + r], pl = p[4 + a.ws_rows + r];
      const float* po = p + 4 + 2 * a.ws_rows + (int64_t)r * DP + lane * PER;
      const float top = fmaxf(m, pm), base = top == -INFINITY ? 0.0f : top;
      const float old = exp2_fast(m - base), add = exp2_fast(pm - base);
      m = top, l = l * old + pl * add;
#pragma unroll
      for (int i = 0; i < PER; ++i) o[i] = o[i] * old + po[i] * add;
      if (flags & 2) break;
    }
    const float by = l == 0 ? 0.0f : 1.0f / l;
    const int i = (int)quotient(r, a.group), g = r - i * (int)a.group.d;
    uint16_t* to = (uint16_t*)a.out + (int64_t)(token + i) * a.os.token + (int64_t)(kv_head * (int)a.group.d + g) * a.os.head;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int c = lane * PER + k;
      if (c < a.D) to[c] = (uint16_t)pack2<TYPE>(o[k] * by, 0.0f);
    }
  }
}

template <int TYPE, bool FP8, int DP>
hipError_t launch_columns(const CacheArgs& a, hipStream_t s) {
  if (a.groups) {
    cache_attention_kernel<TYPE, FP8, DP, true><<<a.groups, 256, 0, s>>>(a);
    cache_attention_join_kernel<TYPE, DP><<<dim3(a.groups, 4), 256, 0, s>>>(a);
    return hipGetLastError();
  }
  const int tokens = kAttnRows / (int)a.group.d;
  const int64_t tiles = (a.T / tokens + (a.S < a.T ? a.S : a.T)) * a.kv_heads;   // as many as there can be
  constexpr int64_t kPiece = int64_t(1) << 23;                     // (a launch holds fewer than 2^32 threads)
  CacheArgs piece = a;
  for (piece.t0 = 0; piece.t0 < tiles; piece.t0 += kPiece)
    cache_attention_kernel<TYPE, FP8, DP, false><<<(uint32_t)(tiles - piece.t0 < kPiece ? tiles - piece.t0 : kPiece), 256, 0, s>>>(piece);
  return hipGetLastError();
}
template <int TYPE, bool FP8>
hipError_t launch_types(const CacheArgs& a, hipStream_t s) {
  const int dp = attn_columns(a.D);
  return dp == 64 ? launch_columns<TYPE, FP8, 64>(a, s) : dp == 128 ? launch_columns<TYPE, FP8, 128>(a, s) : launch_columns<TYPE, FP8, 256>(a, s);
}
hipError_t launch_cache_attention(const CacheArgs& a, hipStream_t s) {
  if (a.type == kBf16) return a.fp8 ? launch_types<kBf16, true>(a, s) : launch_types<kBf16, false>(a, s);
  return a.fp8 ? launch_types<kF16, true>(a, s) : launch_types<kF16, false>(a, s);
}

}  // namespace axe
