// Which shape of a kernel around the experts' products a call takes, and the workspace that follows from it: host arithmetic on sizes alone, the same with and without a GPU.
#pragma once
#include <stdint.h>

#include <algorithm>

namespace axe {

// ---- norm

// Threads and runs of a row: as many threads as a run each needs, up to 512, then two and four runs.  Measured, us: 1000 x 8192 bf16 to e4m3 with 256 x 4 / 512 x 2 / 1024 x 1
// 13.2 / 11.9 / 12.7, one row of 2048 with 64 x 4 / 256 x 1 3.4 / 2.3, fp16 2000 x 1999 6.0 / 5.8.  Backward, rows of a workgroup (of 512 or 1024 threads): it has
// one row of the workspace to write for all of them; 4096 x 2048 bf16, 512 workgroups of 1 / 2 / 4 rows 16.1 / 14.6 / 13.6, 256 of 4 15.0, 1024 of 1 14.8.
template <int TPR_, int RUNS_, bool SHORT_ = false>
struct RowShape {
  static constexpr int TPR = TPR_, RUNS = RUNS_, ROWS = TPR == 64 ? 8 : 1024 / TPR;
  static constexpr bool SHORT = SHORT_;
};
template <class F>
void by_row_shape(int H, F&& f) {
  if (H < 8) f(RowShape<64, 1, true>());
  else if (H <= 64 * 8) f(RowShape<64, 1>());
  else if (H <= 128 * 8) f(RowShape<128, 1>());
  else if (H <= 256 * 8) f(RowShape<256, 1>());
  else if (H <= 512 * 8) f(RowShape<512, 1>());
  else if (H <= 1024 * 8) f(RowShape<512, 2>());
  else if (H <= 2048 * 8) f(RowShape<1024, 2>());
  else f(RowShape<1024, 4>());
}

// Workgroups of the backward kernel: two for every compute unit, and one where it has at most two turns to make (a second launch costs more than they do).
inline int64_t backward_groups(int64_t T, int64_t H) {
  int rows = 1;
  by_row_shape((int)H, [&](auto shape) { rows = decltype(shape)::ROWS; });
  const int64_t n = (T + rows - 1) / rows;
  return n <= 2 ? (n ? 1 : 0) : n < 512 ? n : 512;
}
inline int64_t rmsnorm_workspace_words(int64_t T, int64_t H) {
  const int64_t n = backward_groups(T, H);
  return n > 1 ? n * H : 0;
}

// ---- routing

constexpr int kMaskTokens = 64;                                    // tokens of a mask

// Lanes of a token and experts of a lane: as many lanes as the experts fill while the tokens do not fill the chip (`few`: that many tokens), else fewer, whose lists are longer.  us,
// 4096 tokens of 128 experts, 64 lanes x 2 / 16 x 8: 6.0 / 5.2, their gradient 4.2 / 4.5; one token 3.8 / 4.2; 1000 tokens of 256 experts with groups, 64 x 4 / 32 x 8: 7.8 / 8.2.  A
// workgroup that has all tokens to itself holds 16 of 64 lanes or 64 of 16 at once (whole calls, 128 experts: 16 tokens 5.6 / 5.8, 32 tokens 7.5 / 5.7, 64 tokens 11.9 / 7.0).
template <int LPT_, int V_, bool SHORT_ = false>
struct RouteShape {
  static constexpr int LPT = LPT_, V = V_;
  static constexpr bool SHORT = SHORT_;
};
template <class F>
void by_route_shape(bool few, int E, int k, F&& f) {
  if (E < 8) f(RouteShape<16, 8, true>());
  else if (E <= 128 && (few || k > 16)) f(RouteShape<64, 2>());
  else if (E <= 128) f(RouteShape<16, 8>());
  else if (E <= 256 && (few || k > 32)) f(RouteShape<64, 4>());
  else if (E <= 256) f(RouteShape<32, 8>());
  else if (E <= 512) f(RouteShape<64, 8>());
  else f(RouteShape<64, 16>());
}

inline bool few_tokens(int64_t T) { return T <= 16 || (T > kMaskTokens && T <= 2048); }
// Whether one workgroup takes all tokens, in one launch: as many as it holds at once, or in two turns where it saves the second launch all the same (whole calls, us, 32 lanes a
// token: 48 tokens 8.5, 64 tokens 11.0; 64 lanes: 32 tokens 8.6, 48 tokens 11.3; two launches 8.7 - 9.1).
inline bool one_workgroup(int64_t T, int E, int k) {
  int lanes = 0;
  by_route_shape(few_tokens(T), E, k, [&](auto shape) { lanes = decltype(shape)::LPT; });
  return T <= (lanes == 16 ? kMaskTokens : lanes == 32 ? 48 : 32);
}
// Blocks of tokens: 8 a block, more once that makes more than 256 of them; a block's counts have 16 bits.  (33333 tokens of 256
// experts in whole masks of 64, 174 blocks, 31.6 us, in multiples of 16, 232 blocks, 26.1.)  us, 1000 tokens in blocks of 4 / 8 / 16: 7.2 + 6.2 / 7.8 + 5.2 /
// 9.7 + 5.0 for the two kernels, 4096 tokens in blocks of 16 / 32 / 64: 5.2 + 5.6 / 8.5 + 5.2 / 13.0 + 4.6 (with the second kernel a microsecond slower than it is now).
inline int block_tokens(int64_t T) {
  const int64_t n = (T + 255) / 256;
  if (n <= 32) return n <= 8 ? 8 : n <= 16 ? 16 : 32;
  return (int)std::min<int64_t>((n + 15) / 16 * 16, 65536 - kMaskTokens);
}
inline int counts_pitch(int E) {
  int p = 8;
  while (p < E) p *= 2;
  return p;
}
inline int64_t route_workspace_words(int64_t T, int E, int k) {
  if (one_workgroup(T, E, k)) return 0;
  const int tokens = block_tokens(T);
  return (T + tokens - 1) / tokens * counts_pitch(E) / 2;
}

}  // namespace axe
