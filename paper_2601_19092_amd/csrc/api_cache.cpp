// Entry points of the paged cache: appending keys and values, attention over it.  Argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <vector>

#include "cache_ops.h"
#include "entry_points.h"

using namespace axe;

namespace {

constexpr int64_t kMost = int64_t(1) << 30;

int check_cache(const axe_cache_desc_t* g, const char* fn) {
  if (!g) return invalid(fn, "descriptor is NULL");
  if (g->T < 0 || g->S < 0 || g->pages < 0 || g->max_pages < 0 || g->q_heads <= 0 || g->kv_heads <= 0 || g->head_dim <= 0 || g->page_tokens <= 0)
    return invalid(fn, "needs T, S, pages, max_pages >= 0; heads, head_dim, page_tokens positive");
  if (!real_type(g->dtype) || !(real_type(g->cache_dtype) || g->cache_dtype == AXE_FP8_E4M3)) return invalid(fn, "unknown element type");
  if (g->q_heads % g->kv_heads) return invalid(fn, "q_heads must be a multiple of kv_heads");
  if (g->dtype == AXE_F32 || (g->cache_dtype != g->dtype && g->cache_dtype != AXE_FP8_E4M3)) return unsupported(fn, "rows in bf16 or fp16, the cache in the same or in e4m3");
  if (g->head_dim % (g->cache_dtype == AXE_FP8_E4M3 ? 16 : 8) || g->head_dim > 256) return unsupported(fn, "head_dim must be a multiple of 8 (of 16 with an e4m3 cache) up to 256");
  if (g->q_heads / g->kv_heads > kAttnMaxGroup || g->q_heads >= 65536 || g->S >= 1 << 20 || g->T > kMost || g->pages > kMost || (int64_t)g->max_pages * g->page_tokens > kMost)
    return unsupported(fn, "T, pages, max_pages page_tokens up to 2^30, S below 2^20, heads below 2^16, at most 128 query heads to a head of the cache");
  return AXE_OK;
}

// A layout of some dimensions with one stride each, none of them negative, 1 along the last.  Extents of 1 have stride 0.
struct Strided {
  int64_t s[4] = {0, 0, 0, 0};
  int64_t off = 0;
  MemLayout mem;
};
int plan_strided(const axe_layout_t& L, int mem_axis, std::initializer_list<int64_t> dims, int64_t elems, const char* fn, Strided& out) {
  if (elems > kMostElems) return invalid(fn, "a buffer of more than 2^58 elements");
  HLayout h;
  if (int rc = load_layout(&L, h, fn)) return rc;
  if (int rc = check_shape(h, (int32_t)dims.size(), dims.begin(), fn)) return rc;
  if (int rc = reduce_to_memory(h, mem_axis, out.mem, fn)) return rc;
  if (!out.mem.R.empty() || out.mem.swz.mask) return unsupported(fn, "replicated or swizzled operands are not supported");
  if (int rc = check_range(out.mem, elems, fn)) return rc;
  std::vector<HIter> D = out.mem.D;
  out.off = out.mem.off;
  for (int i = (int)dims.size() - 1; i >= 0; --i) {
    const int64_t e = dims.begin()[i];
    out.s[i] = 0;
    if (e == 1) continue;
    if (D.empty() || D.back().e % e) return unsupported(fn, "a dimension of an operand has more than one stride");
    out.s[i] = D.back().s;
    D.back().e /= e;
    if (D.back().e == 1) D.pop_back();
    else D.back().s *= e;                                          // (within the range that was checked)
    if (out.s[i] < 0) return unsupported(fn, "negative strides are not supported");
  }
  const int last = (int)dims.size() - 1;
  if (dims.begin()[last] > 1 && out.s[last] != 1) return unsupported(fn, "the columns of a head lie side by side");
  return AXE_OK;
}

struct CachePlan {
  Strided q, k, v, o, kc, vc;
};
// What a call uses: append q, k, v, out (with q), both caches; attention q, out, both caches.
struct Uses {
  bool q, kv, o;
};
int plan_cache(const axe_cache_desc_t* g, const char* fn, Uses u, CachePlan& p) {
  const int64_t D = g->head_dim;
  if (u.q)
    if (int rc = plan_strided(g->q, g->mem_axis, {g->T, g->q_heads, D}, g->q_elems, fn, p.q)) return rc;
  if (u.kv) {
    if (int rc = plan_strided(g->k, g->mem_axis, {g->T, g->kv_heads, D}, g->k_elems, fn, p.k)) return rc;
    if (int rc = plan_strided(g->v, g->mem_axis, {g->T, g->kv_heads, D}, g->v_elems, fn, p.v)) return rc;
  }
  if (u.o) {
    if (int rc = plan_strided(g->out, g->mem_axis, {g->T, g->q_heads, D}, g->out_elems, fn, p.o)) return rc;
    if (!provably_injective(p.o.mem)) {
      set_error("%s: two elements of out may share an address", fn);
      return AXE_EALIAS;
    }
  }
  if (g->pages == 0) return AXE_OK;
  if (int rc = plan_strided(g->k_cache, g->mem_axis, {g->pages, g->page_tokens, g->kv_heads, D}, g->k_cache_elems, fn, p.kc)) return rc;
  if (int rc = plan_strided(g->v_cache, g->mem_axis, {g->pages, g->page_tokens, g->kv_heads, D}, g->v_cache_elems, fn, p.vc)) return rc;
  for (const Strided* c : {&p.kc, &p.vc}) {
    if (!provably_injective(c->mem)) {
      set_error("%s: two elements of a cache may share an address", fn);
      return AXE_EALIAS;
    }
    const int unit = g->cache_dtype == AXE_FP8_E4M3 ? 16 : 8;
    if (c->s[0] % unit || c->s[1] % unit || c->s[2] % unit || c->off % unit) return unsupported(fn, "a cache's strides and offset must be multiples of 16 bytes");
  }
  return AXE_OK;
}
// (Where it lies until the thread's next call of this kind.)  What a call's strides have to be multiples of goes by the cache's type, so that is in the key too.
int kept_cache_plan(const axe_cache_desc_t* g, const char* fn, Uses u, const CachePlan*& out) {
  static thread_local LastPlan<CachePlan> last[2];
  LastPlan<CachePlan>& mine = last[u.kv];
  PlanKey key;
  for (int64_t v : {g->T, g->pages, (int64_t)g->q_heads, (int64_t)g->kv_heads, (int64_t)g->head_dim, (int64_t)g->page_tokens, (int64_t)g->cache_dtype, (int64_t)g->mem_axis, (int64_t)(4 * u.q + 2 * u.kv + u.o), g->q_elems,
                    g->k_elems, g->v_elems, g->out_elems, g->k_cache_elems, g->v_cache_elems})
    key.put(v);
  const bool keyed = (!u.q || key_of_layout(g->q, key)) && (!u.kv || (key_of_layout(g->k, key) && key_of_layout(g->v, key))) && (!u.o || key_of_layout(g->out, key)) &&
                     (!g->pages || (key_of_layout(g->k_cache, key) && key_of_layout(g->v_cache, key)));
  out = &mine.plan;
  if (keyed && mine.holds(key)) return AXE_OK;
  CachePlan p;
  if (int rc = plan_cache(g, fn, u, p)) return rc;
  mine.keep(key, p);
  mine.have = keyed;
  return AXE_OK;
}

// Two operands of one buffer's rows, each a range of columns of its own (the queries, keys and values of one product).
bool columns_apart(const void* a, const Strided& x, int64_t x_heads, const void* b, const Strided& y, int64_t y_heads, int64_t T, int64_t D, int eb) {
  const int64_t bytes = (const char*)b + y.off * eb - ((const char*)a + x.off * eb);
  if (bytes % eb) return false;
  const int64_t ld = x.s[0], xs = (x_heads - 1) * x.s[1] + D, ys = (y_heads - 1) * y.s[1] + D;
  int64_t delta = bytes / eb;
  if (T == 1) return delta >= xs || -delta >= ys;
  if (ld != y.s[0] || xs > ld || ys > ld) return false;
  delta = (delta % ld + ld) % ld;
  return xs <= delta && delta + ys <= ld;
}
// The two caches in one buffer: the same places, a distance apart that no two places of one have.
bool caches_apart(const void* a, const Strided& x, const void* b, const Strided& y, int eb) {
  const int64_t bytes = (const char*)b + y.off * eb - ((const char*)a + x.off * eb);
  if (bytes % eb || bytes == 0) return false;
  for (int i = 0; i < 4; ++i)
    if (x.s[i] != y.s[i]) return false;
  MemLayout both = x.mem;
  const int64_t delta = bytes / eb;
  both.D.push_back(HIter{2, delta < 0 ? -delta : delta, 0});
  return provably_injective(both);
}

CacheArgs cache_args(const axe_cache_desc_t* g, const CachePlan& p) {
  CacheArgs a = {};
  a.qs = {p.q.s[0], p.q.s[1]}, a.ks = {p.k.s[0], p.k.s[1]}, a.vs = {p.v.s[0], p.v.s[1]}, a.os = {p.o.s[0], p.o.s[1]};
  a.kp = {p.kc.s[0], p.kc.s[1], p.kc.s[2]}, a.vp = {p.vc.s[0], p.vc.s[1], p.vc.s[2]};
  a.T = g->T, a.pages = g->pages, a.S = g->S, a.q_heads = g->q_heads, a.kv_heads = g->kv_heads, a.D = g->head_dim;
  a.max_pages = g->max_pages, a.capacity = g->max_pages * g->page_tokens;
  a.page = divisor(g->page_tokens), a.group = divisor(g->q_heads / g->kv_heads);
  a.type = g->dtype, a.fp8 = g->cache_dtype == AXE_FP8_E4M3;
  return a;
}

struct Tables {
  Buf rows, lengths, pages;
};
Tables tables(const axe_cache_desc_t* g, const int32_t* seq_rows, const int32_t* lengths, const int32_t* table) {
  return {{seq_rows, ((int64_t)g->S + 1) * 4, 4, true}, {lengths, (int64_t)g->S * 4, 4, g->S > 0}, {table, (int64_t)g->S * g->max_pages * 4, 4, g->S > 0 && g->max_pages > 0}};
}
int64_t cache_scale_bytes(const axe_cache_desc_t* g) { return g->pages * g->page_tokens * g->kv_heads * 4; }
int check_scales(const axe_cache_desc_t* g, const char* fn, const float* ks, const float* vs) {
  if (g->cache_dtype != AXE_FP8_E4M3 && (ks || vs)) return invalid(fn, "scales go with an e4m3 cache");
  if (g->pages > kMostElems / 8 / g->page_tokens / g->kv_heads) return invalid(fn, "scales of more than 2^58 bytes");
  return AXE_OK;
}

}  // namespace

extern "C" {

int axe_cache_append(const axe_cache_desc_t* g, const void* d_q, const void* d_k, const void* d_v, const float* d_rotation, const int32_t* d_seq_rows, const int32_t* d_lengths,
                     const int32_t* d_page_table, void* d_q_out, void* d_k_cache, void* d_v_cache, float* d_k_scales, float* d_v_scales, void* stream) {
  const char* fn = "axe_cache_append";
  return guarded(fn, [&]() -> int {
    if (int rc = check_cache(g, fn)) return rc;
    if (g->rotary_dim < 0 || g->rotary_dim % 2 || g->rotary_dim > g->head_dim) return invalid(fn, "rotary_dim must be even, up to head_dim");
    if (g->rotary_style != AXE_ROTATE_HALVES && g->rotary_style != AXE_ROTATE_PAIRS) return invalid(fn, "unknown rotary_style");
    if (g->T == 0 || g->S == 0) return AXE_OK;
    if (!d_q != !d_q_out) return invalid(fn, "q and q_out are given together");
    if (int rc = check_scales(g, fn, d_k_scales, d_v_scales)) return rc;
    const bool has_q = d_q, fp8 = g->cache_dtype == AXE_FP8_E4M3, any = g->pages > 0;
    const CachePlan* kept;
    if (int rc = kept_cache_plan(g, fn, {has_q, true, has_q}, kept)) return rc;
    const CachePlan& p = *kept;
    const int eb = 2, cb = fp8 ? 1 : 2;
    const Tables t = tables(g, d_seq_rows, d_lengths, d_page_table);
    Buf q = {d_q, has_q ? g->q_elems * eb : 0, eb, false}, k = {d_k, g->k_elems * eb, eb, true}, v = {d_v, g->v_elems * eb, eb, true};
    Buf rot = {g->rotary_dim ? d_rotation : nullptr, (int64_t)g->max_pages * g->page_tokens * g->rotary_dim * 4, 4, g->rotary_dim && g->max_pages};
    Buf o = {d_q_out, has_q ? g->out_elems * eb : 0, eb, false};
    Buf kc = {any ? d_k_cache : nullptr, any ? g->k_cache_elems * cb : 0, 16, any}, vc = {any ? d_v_cache : nullptr, any ? g->v_cache_elems * cb : 0, 16, any};
    Buf sk = {any ? d_k_scales : nullptr, fp8 ? cache_scale_bytes(g) : 0, 4, fp8 && any}, sv = {any ? d_v_scales : nullptr, fp8 ? cache_scale_bytes(g) : 0, 4, fp8 && any};
    // q in place: a thread reads the elements that it writes, and those they are turned with, before the wave that holds them writes any
    Buf qi = q, ki = k, vi = v;
    if (has_q) {
      const bool on_q = d_q_out == d_q && p.q.off == p.o.off && (g->T == 1 || p.q.s[0] == p.o.s[0]) && p.q.s[1] == p.o.s[1];
      if (on_q || columns_apart(d_q_out, p.o, g->q_heads, d_q, p.q, g->q_heads, g->T, g->head_dim, eb)) qi.p = nullptr;
      if (columns_apart(d_q_out, p.o, g->q_heads, d_k, p.k, g->kv_heads, g->T, g->head_dim, eb)) ki.p = nullptr, ki.needed = false;
      if (columns_apart(d_q_out, p.o, g->q_heads, d_v, p.v, g->kv_heads, g->T, g->head_dim, eb)) vi.p = nullptr, vi.needed = false;
    }
    if (!d_k || !d_v) return invalid(fn, "NULL device pointer");
    if (int rc = check_buffers(fn, {qi, ki, vi, rot, t.rows, t.lengths, t.pages}, {o})) return rc;
    if (int rc = check_buffers(fn, {q, k, v, rot, t.rows, t.lengths, t.pages, o}, {kc, sk, sv})) return rc;
    if (int rc = check_buffers(fn, {q, k, v, rot, t.rows, t.lengths, t.pages, o, sk, sv}, {vc})) return rc;
    if (meet(kc, vc) && !caches_apart(d_k_cache, p.kc, d_v_cache, p.vc, cb)) return invalid(fn, "two outputs overlap");
    CacheArgs a = cache_args(g, p);
    a.q = at(d_q, p.q.off, eb), a.k = at(d_k, p.k.off, eb), a.v = at(d_v, p.v.off, eb), a.out = at(d_q_out, p.o.off, eb);
    a.k_cache = at(d_k_cache, p.kc.off, cb), a.v_cache = at(d_v_cache, p.vc.off, cb), a.k_scales = d_k_scales, a.v_scales = d_v_scales;
    a.rotation = d_rotation, a.seq_rows = d_seq_rows, a.lengths = d_lengths, a.table = d_page_table;
    a.rotary = g->rotary_dim, a.pairs = g->rotary_style == AXE_ROTATE_PAIRS;
    a.rows = divisor((has_q ? g->q_heads : 0) + 2 * (int64_t)g->kv_heads);
    return finish(launch_cache_append(a, (hipStream_t)stream), fn);
  });
}

int64_t axe_cache_attention_workspace(const axe_cache_desc_t* g) {
  return guarded("axe_cache_attention_workspace", [&]() -> int64_t {
    if (int rc = check_cache(g, "axe_cache_attention_workspace")) return rc;
    return attn_workspace_words(attn_shape(g->T, g->S, g->kv_heads, g->q_heads / g->kv_heads, g->head_dim, (int64_t)g->max_pages * g->page_tokens, g->causal ? g->window : 0), g->head_dim);
  });
}

int axe_cache_attention(const axe_cache_desc_t* g, const void* d_q, const void* d_k_cache, const void* d_v_cache, const float* d_k_scales, const float* d_v_scales, const int32_t* d_seq_rows,
                        const int32_t* d_lengths, const int32_t* d_page_table, void* d_out, int32_t* d_ws, int64_t ws_elems, void* stream) {
  const char* fn = "axe_cache_attention";
  return guarded(fn, [&]() -> int {
    if (int rc = check_cache(g, fn)) return rc;
    if (!(g->scale >= 0x1p-100f && g->scale <= 0x1p100f)) return invalid(fn, "scale must be positive, from 2^-100 to 2^100");
    if (g->window < 0) return invalid(fn, "window must not be negative");
    if (g->window && !g->causal) return unsupported(fn, "a window goes with causal attention");
    if (g->T == 0 || g->S == 0) return AXE_OK;
    if (int rc = check_scales(g, fn, d_k_scales, d_v_scales)) return rc;
    const bool fp8 = g->cache_dtype == AXE_FP8_E4M3, any = g->pages > 0;
    const CachePlan* kept;
    if (int rc = kept_cache_plan(g, fn, {true, false, true}, kept)) return rc;
    const CachePlan& p = *kept;
    const int G = g->q_heads / g->kv_heads, eb = 2, cb = fp8 ? 1 : 2;
    const AttnShape shape = attn_shape(g->T, g->S, g->kv_heads, G, g->head_dim, (int64_t)g->max_pages * g->page_tokens, g->causal ? g->window : 0);
    const int64_t words = attn_workspace_words(shape, g->head_dim);
    if (words > 0 && (!d_ws || ws_elems < words)) return invalid(fn, "the workspace is smaller than axe_cache_attention_workspace");
    const Tables t = tables(g, d_seq_rows, d_lengths, d_page_table);
    if (int rc = check_buffers(fn, {{d_q, g->q_elems * eb, eb, true}, {any ? d_k_cache : nullptr, any ? g->k_cache_elems * cb : 0, 16, any},
                                    {any ? d_v_cache : nullptr, any ? g->v_cache_elems * cb : 0, 16, any}, {any ? d_k_scales : nullptr, fp8 ? cache_scale_bytes(g) : 0, 4, fp8 && any},
                                    {any ? d_v_scales : nullptr, fp8 ? cache_scale_bytes(g) : 0, 4, fp8 && any}, t.rows, t.lengths, t.pages},
                               {{d_out, g->out_elems * eb, eb, true}, {words ? d_ws : nullptr, words * 4, 16, false}}))
      return rc;
    CacheArgs a = cache_args(g, p);
    a.q = at(d_q, p.q.off, eb), a.out = at(d_out, p.o.off, eb);
    a.k_cache = (void*)at(d_k_cache, p.kc.off, cb), a.v_cache = (void*)at(d_v_cache, p.vc.off, cb), a.k_scales = (float*)d_k_scales, a.v_scales = (float*)d_v_scales;
    a.seq_rows = d_seq_rows, a.lengths = d_lengths, a.table = d_page_table, a.ws = (float*)d_ws;
    a.causal = g->causal != 0, a.window = std::min<int64_t>(g->window, kMost);
    a.scale_log2 = (float)(g->scale * 1.4426950408889634);
    a.sixteens = g->page_tokens % 16 == 0 && std::max(p.kc.s[1], p.vc.s[1]) < (int64_t(1) << 26);
    a.reach31 = !any || std::max((p.kc.mem.hi - p.kc.off) * cb, (p.vc.mem.hi - p.vc.off) * cb) < (int64_t(1) << 31) - 1024;
    a.groups = shape.groups, a.tile_rows = shape.tile_rows, a.ws_rows = shape.ws_rows;
    return finish(launch_cache_attention(a, (hipStream_t)stream), fn);
  });
}

}  // extern "C"
