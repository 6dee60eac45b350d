// Entry points of what stands around the experts' products: norm, routing, rows in the experts' order.  Argument checks and launches.
#include <hip/hip_runtime.h>

#include <initializer_list>
#include <new>

#include "../../include/axe.h"
#include "host_layout.h"
#include "layer_ops.h"
#include "layer_shapes.h"
#include "plans.h"

using namespace axe;

namespace {

bool real_type(int t) { return t == AXE_BF16 || t == AXE_F16 || t == AXE_F32; }

int invalid(const char* fn, const char* what) {
  set_error("%s: %s", fn, what);
  return AXE_EINVAL;
}
int unsupported(const char* fn, const char* what) {
  set_error("%s: %s", fn, what);
  return AXE_EUNSUPPORTED;
}

// A buffer of a call: where, how many bytes, what it has to be aligned to, and whether the call may not do without it.
struct Buf {
  const void* p;
  int64_t bytes;
  int align;
  bool needed;
};
bool meet(const Buf& a, const Buf& b) {
  return a.p && b.p && (const char*)a.p < (const char*)b.p + b.bytes && (const char*)b.p < (const char*)a.p + a.bytes;
}
int check_buffers(const char* fn, std::initializer_list<Buf> in, std::initializer_list<Buf> out) {
  for (const auto& list : {in, out})
    for (const Buf& b : list) {
      if (b.needed && !b.p) return invalid(fn, "NULL device pointer");
      if (b.p && (uintptr_t)b.p % (uintptr_t)b.align) return invalid(fn, "a buffer is not aligned to its elements");
    }
  for (const Buf& o : out) {
    for (const Buf& i : in)
      if (meet(i, o)) return invalid(fn, "an output overlaps an input");
    for (const Buf& p : out)
      if (&p != &o && meet(p, o)) return invalid(fn, "two outputs overlap");
  }
  return AXE_OK;
}

// One matrix of a call: its layout on the memory axis, planned once per descriptor.  Bytes of its buffer are computed of a matrix that was planned (or is not there) only: 64 bits hold them.
struct Mat {
  int64_t ld = 0, off = 0;
};
constexpr int64_t kMostElems = int64_t(1) << 58;
int plan_matrix(const axe_layout_t& L, int mem_axis, int64_t rows, int64_t cols, int64_t elems, const char* fn, Mat& m) {
  if (elems > kMostElems) return invalid(fn, "a buffer of more than 2^58 elements");
  return strided_2d(&L, mem_axis, rows, cols, true, elems, fn, &m.ld, &m.off);
}
int64_t bytes_of(const void* p, int64_t elems, int eb) { return p ? elems * eb : 0; }

// The body of an entry point; planning allocates, and an entry point neither throws nor aborts.
template <class F>
auto guarded(const char* fn, F&& f) -> decltype(f()) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    set_error("%s: out of host memory", fn);
    return AXE_EINVAL;
  }
}

int finish(hipError_t e, const char* fn) { return e == hipSuccess ? AXE_OK : hip_fail(e, fn); }

// ---- norm -----------------------------------------------------------------------------------------------------------

struct NormPlan {
  Mat x, r, s, y;
};
int check_norm(const axe_rmsnorm_desc_t* g, const char* fn, bool backward) {
  if (!g) return invalid(fn, "descriptor is NULL");
  if (g->T < 0 || g->H <= 0) return invalid(fn, "H must be positive, T not negative");
  if (!real_type(g->x_dtype) || !(real_type(g->weight_dtype)) || !(real_type(g->y_dtype) || g->y_dtype == AXE_FP8_E4M3))
    return invalid(fn, "unknown element type");
  if (g->scale_dtype != AXE_SCALE_F32 && g->scale_dtype != AXE_SCALE_E8M0) return invalid(fn, "unknown scale_dtype");
  if (!(g->eps >= 0)) return invalid(fn, "eps must not be negative");
  if (g->y_dtype != g->x_dtype && g->x_dtype != AXE_F32 && (backward || g->y_dtype != AXE_FP8_E4M3))
    return unsupported(fn, "y has x's type, 16 bits of fp32 rows, or (forward) e4m3");
  if (backward && g->y_dtype == AXE_FP8_E4M3) return unsupported(fn, "the gradient of a quantised y is passed in 16 or 32 bits");
  if (g->H > kNormMaxH || g->T >= (int64_t(1) << 31)) return unsupported(fn, "H up to 32768, T below 2^31");
  return AXE_OK;
}
int plan_norm(const axe_rmsnorm_desc_t* g, const char* fn, bool res, bool sum, NormPlan& p) {
  if (int rc = plan_matrix(g->x, g->mem_axis, g->T, g->H, g->x_elems, fn, p.x)) return rc;
  if (int rc = plan_matrix(g->y, g->mem_axis, g->T, g->H, g->y_elems, fn, p.y)) return rc;
  if (res)
    if (int rc = plan_matrix(g->residual, g->mem_axis, g->T, g->H, g->residual_elems, fn, p.r)) return rc;
  if (sum)
    if (int rc = plan_matrix(g->sum, g->mem_axis, g->T, g->H, g->sum_elems, fn, p.s)) return rc;
  return AXE_OK;
}
int kept_norm_plan(const axe_rmsnorm_desc_t* g, const char* fn, bool res, bool sum, NormPlan& out) {
  static thread_local LastPlan<NormPlan> last;
  PlanKey key;
  for (int64_t v : {g->T, g->H, (int64_t)g->mem_axis, (int64_t)(2 * res + sum), g->x_elems, g->residual_elems, g->sum_elems, g->y_elems}) key.put(v);
  const bool keyed = key_of_layout(g->x, key) && key_of_layout(g->y, key) && (!res || key_of_layout(g->residual, key)) && (!sum || key_of_layout(g->sum, key));
  if (keyed && last.holds(key)) {
    out = last.plan;
    return AXE_OK;
  }
  if (int rc = plan_norm(g, fn, res, sum, out)) return rc;
  if (keyed) last.keep(key, out);
  return AXE_OK;
}
template <class V>
V* at(V* p, int64_t off, int eb) {
  using C = std::conditional_t<std::is_const<V>::value, const char, char>;
  return p ? (V*)((C*)p + off * eb) : nullptr;
}
// an output that is exactly an input: same buffer, same element size, same place of every element
bool same(const void* a, const Mat& m, int eb, const void* b, const Mat& n, int fb) { return a && a == b && m.ld == n.ld && m.off == n.off && eb == fb; }
int64_t scale_bytes(int64_t rows, int64_t H, int scale_dtype) { return rows * ((H + 127) / 128) * (scale_dtype == AXE_SCALE_E8M0 ? 1 : 4); }

// ---- routing ----------------------------------------------------------------------------------------------------------

int check_route(const axe_route_desc_t* g, const char* fn) {
  if (!g) return invalid(fn, "descriptor is NULL");
  if (g->T < 0 || g->E <= 0 || g->k <= 0 || g->k > g->E) return invalid(fn, "needs T >= 0, E >= 1, 1 <= k <= E");
  if (!real_type(g->logit_dtype)) return invalid(fn, "unknown element type");
  if ((g->score != AXE_ROUTE_SOFTMAX && g->score != AXE_ROUTE_SIGMOID) || (g->group_score != AXE_ROUTE_GROUP_MAX && g->group_score != AXE_ROUTE_GROUP_TOP2))
    return invalid(fn, "unknown score or group_score");
  if (g->groups < 1 || g->E % g->groups || g->groups_kept < 1 || g->groups_kept > g->groups || g->k > g->E / g->groups * g->groups_kept)
    return invalid(fn, "groups must divide E, 1 <= groups_kept <= groups, and k fit the experts of the groups kept");
  if (!(g->scale - g->scale == 0)) return invalid(fn, "scale must be finite");
  if ((uintptr_t)g->d_bias & 3) return invalid(fn, "a buffer is not aligned to its elements");
  if (g->E > kRouteMaxE || g->k > kRouteMaxK || g->groups > kRouteMaxGroups) return unsupported(fn, "E up to 1024, k up to 64, groups up to 64");
  if (g->T >= (int64_t(1) << 31) / g->k) return unsupported(fn, "T k below 2^31");
  return AXE_OK;
}
int kept_route_plan(const axe_route_desc_t* g, const char* fn, Mat& out) {
  static thread_local LastPlan<Mat> last;
  PlanKey key;
  for (int64_t v : {g->T, (int64_t)g->E, (int64_t)g->mem_axis, g->logits_elems}) key.put(v);
  const bool keyed = key_of_layout(g->logits, key);
  if (keyed && last.holds(key)) {
    out = last.plan;
    return AXE_OK;
  }
  if (int rc = plan_matrix(g->logits, g->mem_axis, g->T, g->E, g->logits_elems, fn, out)) return rc;
  if (keyed) last.keep(key, out);
  return AXE_OK;
}
RouteArgs route_args(const axe_route_desc_t* g, const Mat& m, const void* logits) {
  RouteArgs a = {};
  a.logits = at(logits, m.off, elem_bytes(g->logit_dtype));
  a.bias = g->d_bias;
  a.T = g->T, a.ld = m.ld, a.E = g->E, a.k = g->k, a.type = g->logit_dtype;
  a.sigmoid = g->score == AXE_ROUTE_SIGMOID, a.renorm = g->renorm != 0;
  // all groups kept: they decide nothing
  a.groups = g->groups_kept == g->groups ? 1 : g->groups, a.kept = a.groups == 1 ? 1 : g->groups_kept;
  a.top2 = g->group_score == AXE_ROUTE_GROUP_TOP2;
  a.per = g->E / a.groups;
  a.scale = g->scale;
  return a;
}

// ---- rows -------------------------------------------------------------------------------------------------------------

struct RowsPlan {
  Mat t, r;
};
int check_rows(const axe_rows_desc_t* g, const char* fn, bool dispatch) {
  if (!g) return invalid(fn, "descriptor is NULL");
  if (g->T < 0 || g->H <= 0 || g->k <= 0 || g->M < 0) return invalid(fn, "needs T, M >= 0, H and k positive");
  if (!(real_type(g->tokens_dtype) || g->tokens_dtype == AXE_FP8_E4M3) || !(real_type(g->rows_dtype) || g->rows_dtype == AXE_FP8_E4M3))
    return invalid(fn, "unknown element type");
  if (g->scale_dtype != AXE_SCALE_F32 && g->scale_dtype != AXE_SCALE_E8M0) return invalid(fn, "unknown scale_dtype");
  if (g->tokens_dtype != g->rows_dtype && !(dispatch && g->rows_dtype == AXE_FP8_E4M3)) return unsupported(fn, "tokens and rows have one type (dispatch: or the rows are e4m3)");
  if (!dispatch && g->rows_dtype == AXE_FP8_E4M3) return unsupported(fn, "rows in 16 or 32 bits");
  if (g->k > kRowsMaxK || g->H >= (int64_t(1) << 28) || g->M >= (int64_t(1) << 31) || g->T >= (int64_t(1) << 31) / g->k)
    return unsupported(fn, "k up to 64; M and T k below 2^31, H below 2^28");
  return AXE_OK;
}
int kept_rows_plan(const axe_rows_desc_t* g, const char* fn, RowsPlan& out) {
  static thread_local LastPlan<RowsPlan> last;
  PlanKey key;
  for (int64_t v : {g->T, g->M, g->H, (int64_t)g->mem_axis, g->tokens_elems, g->rows_elems}) key.put(v);
  const bool keyed = key_of_layout(g->tokens, key) && key_of_layout(g->rows, key);
  if (keyed && last.holds(key)) {
    out = last.plan;
    return AXE_OK;
  }
  if (int rc = plan_matrix(g->tokens, g->mem_axis, g->T, g->H, g->tokens_elems, fn, out.t)) return rc;
  if (int rc = plan_matrix(g->rows, g->mem_axis, g->M, g->H, g->rows_elems, fn, out.r)) return rc;
  if (keyed) last.keep(key, out);
  return AXE_OK;
}
RowsArgs rows_args(const axe_rows_desc_t* g, const RowsPlan& p) {
  RowsArgs a = {};
  a.T = g->T, a.M = g->M, a.ldt = p.t.ld, a.ldr = p.r.ld, a.H = (int32_t)g->H, a.k = g->k;
  a.t_type = g->tokens_dtype, a.r_type = g->rows_dtype, a.e8m0 = g->scale_dtype == AXE_SCALE_E8M0;
  return a;
}

}  // namespace

extern "C" {

int axe_rmsnorm(const axe_rmsnorm_desc_t* g, const void* d_x, const void* d_residual, const void* d_w, void* d_sum, void* d_y, void* d_scales, void* stream) {
  const char* fn = "axe_rmsnorm";
  return guarded(fn, [&]() -> int {
    if (int rc = check_norm(g, fn, false)) return rc;
    if (g->T == 0) return AXE_OK;
    NormPlan p;
    if (int rc = kept_norm_plan(g, fn, d_residual, d_sum, p)) return rc;
    const int xb = elem_bytes(g->x_dtype), yb = elem_bytes(g->y_dtype), wb = elem_bytes(g->weight_dtype);
    const bool fp8 = g->y_dtype == AXE_FP8_E4M3;
    if (!fp8 && d_scales) return invalid(fn, "scales go with an e4m3 y");
    Buf x = {d_x, g->x_elems * xb, xb, true}, r = {d_residual, bytes_of(d_residual, g->residual_elems, xb), xb, false}, w = {d_w, g->H * wb, wb, false};
    Buf s = {d_sum, bytes_of(d_sum, g->sum_elems, xb), xb, false}, y = {d_y, g->y_elems * yb, yb, true};
    Buf sc = {d_scales, scale_bytes(g->T, g->H, g->scale_dtype), g->scale_dtype == AXE_SCALE_E8M0 ? 1 : 4, fp8};
    // In place: a thread reads what it needs of its elements before it writes them (and one that is written twice gets both, so not both outputs).
    Buf xi = x, ri = r;
    const bool sum_x = same(d_sum, p.s, xb, d_x, p.x, xb), sum_r = same(d_sum, p.s, xb, d_residual, p.r, xb);
    const bool y_x = same(d_y, p.y, yb, d_x, p.x, xb), y_r = same(d_y, p.y, yb, d_residual, p.r, xb);
    if (!d_x) return invalid(fn, "NULL device pointer");
    if (sum_x || y_x) xi.p = nullptr, xi.needed = false;
    if (sum_r || y_r) ri.p = nullptr;
    if (int rc = check_buffers(fn, {xi, ri, w}, {s, y, sc})) return rc;
    // (an input left out above is the output itself; the other one must still be clear of it)
    if ((sum_x && meet(r, s)) || (y_x && meet(r, y)) || (sum_r && meet(x, s)) || (y_r && meet(x, y)) || (d_residual && meet(x, r) && (sum_x || y_x || sum_r || y_r)))
      return invalid(fn, "an output overlaps an input");
    NormArgs a = {};
    a.x = at(d_x, p.x.off, xb), a.r = at(d_residual, p.r.off, xb), a.w = d_w;
    a.sum = at(d_sum, p.s.off, xb), a.y = at(d_y, p.y.off, yb), a.scales = d_scales;
    a.T = g->T, a.H = (int32_t)g->H, a.ldx = p.x.ld, a.ldr = p.r.ld, a.lds = p.s.ld, a.ldy = p.y.ld;
    a.x_type = g->x_dtype, a.y_type = g->y_dtype, a.w_type = g->weight_dtype, a.e8m0 = g->scale_dtype == AXE_SCALE_E8M0, a.eps = g->eps;
    return finish(launch_rmsnorm(a, (hipStream_t)stream), fn);
  });
}

int64_t axe_rmsnorm_workspace(const axe_rmsnorm_desc_t* g) {
  return guarded("axe_rmsnorm_workspace", [&]() -> int64_t {
    if (int rc = check_norm(g, "axe_rmsnorm_workspace", g && g->y_dtype != AXE_FP8_E4M3)) return rc;
    return rmsnorm_workspace_words(g->T, g->H);
  });
}

int axe_rmsnorm_backward(const axe_rmsnorm_desc_t* g, const void* d_dy, const void* d_sum, const void* d_w, const void* d_dsum, void* d_dx, float* d_dweight,
                         int32_t* d_ws, int64_t ws_elems, void* stream) {
  const char* fn = "axe_rmsnorm_backward";
  return guarded(fn, [&]() -> int {
    if (int rc = check_norm(g, fn, true)) return rc;
    NormPlan p;
    if (g->T > 0)
      if (int rc = kept_norm_plan(g, fn, d_dsum, true, p)) return rc;
    const int xb = elem_bytes(g->x_dtype), yb = elem_bytes(g->y_dtype), wb = elem_bytes(g->weight_dtype);
    const int64_t words = d_dweight ? rmsnorm_workspace_words(g->T, g->H) : 0;
    if (words > 0 && (!d_ws || ws_elems < words)) return invalid(fn, "the workspace is smaller than axe_rmsnorm_workspace");
    const bool any = g->T > 0;
    Buf dy = {d_dy, any ? g->y_elems * yb : 0, yb, any}, h = {d_sum, any ? g->sum_elems * xb : 0, xb, any}, w = {d_w, g->H * wb, wb, false};
    Buf ds = {d_dsum, any ? bytes_of(d_dsum, g->residual_elems, xb) : 0, xb, false}, dx = {d_dx, any ? g->x_elems * xb : 0, xb, any};
    Buf dw = {d_dweight, g->H * 4, 4, false}, ws = {words ? d_ws : nullptr, words * 4, 4, false};
    const bool on_dy = same(d_dx, p.x, xb, d_dy, p.y, yb), on_ds = same(d_dx, p.x, xb, d_dsum, p.r, xb);
    Buf dyi = dy, dsi = ds;
    if (on_dy) dyi.p = nullptr, dyi.needed = false;
    if (on_ds) dsi.p = nullptr;
    if (int rc = check_buffers(fn, {dyi, h, w, dsi}, {dx, dw, ws})) return rc;
    if ((on_dy || on_ds) && (meet(dy, dw) || meet(ds, dw) || meet(dy, ws) || meet(ds, ws) || (d_dsum && meet(dy, ds)))) return invalid(fn, "an output overlaps an input");
    NormArgs a = {};
    a.x = at(d_dy, p.y.off, yb), a.h = at(d_sum, p.s.off, xb), a.r = at(d_dsum, p.r.off, xb), a.w = d_w, a.y = at(d_dx, p.x.off, xb);
    a.dw = d_dweight, a.ws = (float*)d_ws;
    a.T = g->T, a.H = (int32_t)g->H, a.ldx = p.y.ld, a.lds = p.s.ld, a.ldr = p.r.ld, a.ldy = p.x.ld;
    a.x_type = g->x_dtype, a.y_type = g->y_dtype, a.w_type = g->weight_dtype, a.eps = g->eps;
    if (!any && !d_dweight) return AXE_OK;
    return finish(launch_rmsnorm_backward(a, (hipStream_t)stream), fn);
  });
}

int64_t axe_route_workspace(const axe_route_desc_t* g) {
  return guarded("axe_route_workspace", [&]() -> int64_t {
    if (int rc = check_route(g, "axe_route_workspace")) return rc;
    return route_workspace_words(g->T, g->E, g->k);
  });
}

int axe_route(const axe_route_desc_t* g, const void* d_logits, int32_t* d_ids, float* d_weights, int32_t* d_group_rows, int32_t* d_row_of, int32_t* d_ws,
              int64_t ws_elems, void* stream) {
  const char* fn = "axe_route";
  return guarded(fn, [&]() -> int {
    if (int rc = check_route(g, fn)) return rc;
    Mat m;
    const bool any = g->T > 0;
    if (any)
      if (int rc = kept_route_plan(g, fn, m)) return rc;
    if ((d_group_rows == nullptr) != (d_row_of == nullptr) && any) return invalid(fn, "group_rows and row_of are given together");
    const int64_t words = d_group_rows ? route_workspace_words(g->T, g->E, g->k) : 0, pairs = g->T * g->k;
    if (words > 0 && (!d_ws || ws_elems < words)) return invalid(fn, "the workspace is smaller than axe_route_workspace");
    const int eb = elem_bytes(g->logit_dtype);
    if (int rc = check_buffers(fn, {{d_logits, any ? g->logits_elems * eb : 0, eb, any}, {g->d_bias, g->E * 4, 4, false}},
                               {{d_ids, pairs * 4, 4, any}, {d_weights, pairs * 4, 4, any}, {d_group_rows, (g->E + 1) * 4, 4, false}, {d_row_of, pairs * 4, 4, false},
                                {words ? d_ws : nullptr, words * 4, 4, false}}))
      return rc;
    if (!any && !d_group_rows) return AXE_OK;
    RouteArgs a = route_args(g, m, d_logits);
    a.ids = d_ids, a.weights = d_weights, a.group_rows = d_group_rows, a.row_of = d_row_of, a.ws = d_ws;
    return finish(launch_route(a, (hipStream_t)stream), fn);
  });
}

int axe_route_backward(const axe_route_desc_t* g, const void* d_logits, const int32_t* d_ids, const float* d_dweights, void* d_dlogits, void* stream) {
  const char* fn = "axe_route_backward";
  return guarded(fn, [&]() -> int {
    if (int rc = check_route(g, fn)) return rc;
    if (g->T == 0) return AXE_OK;
    Mat m;
    if (int rc = kept_route_plan(g, fn, m)) return rc;
    const int eb = elem_bytes(g->logit_dtype);
    const int64_t pairs = g->T * g->k;
    if (!d_logits) return invalid(fn, "NULL device pointer");
    const bool in_place = d_dlogits == d_logits;
    if (int rc = check_buffers(fn, {{in_place ? nullptr : d_logits, g->logits_elems * eb, eb, !in_place}, {d_ids, pairs * 4, 4, true}, {d_dweights, pairs * 4, 4, true}},
                               {{d_dlogits, g->logits_elems * eb, eb, true}}))
      return rc;
    RouteArgs a = route_args(g, m, d_logits);
    a.ids_in = d_ids, a.dweights = d_dweights, a.dlogits = at(d_dlogits, m.off, eb);
    return finish(launch_route_backward(a, (hipStream_t)stream), fn);
  });
}

int axe_rows_dispatch(const axe_rows_desc_t* g, const void* d_tokens, const void* d_token_scales, const int32_t* d_row_of, void* d_rows, void* d_scales, void* stream) {
  const char* fn = "axe_rows_dispatch";
  return guarded(fn, [&]() -> int {
    if (int rc = check_rows(g, fn, true)) return rc;
    if (g->T == 0 || g->M == 0) return AXE_OK;
    if (!d_row_of && (g->k != 1 || g->M != g->T)) return invalid(fn, "without row_of k is 1 and M is T");
    RowsPlan p;
    if (int rc = kept_rows_plan(g, fn, p)) return rc;
    const int tb = elem_bytes(g->tokens_dtype), rb = elem_bytes(g->rows_dtype), sb = g->scale_dtype == AXE_SCALE_E8M0 ? 1 : 4;
    const bool fp8 = g->rows_dtype == AXE_FP8_E4M3, copies = g->tokens_dtype == AXE_FP8_E4M3;
    if ((!fp8 && d_scales) || (!copies && d_token_scales)) return invalid(fn, "scales go with e4m3 rows, token_scales with e4m3 tokens");
    if (int rc = check_buffers(fn, {{d_tokens, g->tokens_elems * tb, tb, true}, {d_token_scales, scale_bytes(g->T, g->H, g->scale_dtype), sb, copies}, {d_row_of, g->T * g->k * 4, 4, false}},
                               {{d_rows, g->rows_elems * rb, rb, true}, {d_scales, scale_bytes(g->M, g->H, g->scale_dtype), sb, fp8}}))
      return rc;
    RowsArgs a = rows_args(g, p);
    a.tokens = at(d_tokens, p.t.off, tb), a.token_scales = d_token_scales, a.row_of = d_row_of;
    a.to_rows = at(d_rows, p.r.off, rb), a.scales = d_scales;
    return finish(launch_rows_dispatch(a, (hipStream_t)stream), fn);
  });
}

int axe_rows_combine(const axe_rows_desc_t* g, const void* d_rows, const int32_t* d_row_of, const float* d_weights, const void* d_add, void* d_tokens, void* stream) {
  const char* fn = "axe_rows_combine";
  return guarded(fn, [&]() -> int {
    if (int rc = check_rows(g, fn, false)) return rc;
    if (g->T == 0) return AXE_OK;
    if (g->M == 0) return invalid(fn, "M must be positive");
    RowsPlan p;
    if (int rc = kept_rows_plan(g, fn, p)) return rc;
    const int eb = elem_bytes(g->tokens_dtype);
    const int64_t pairs = g->T * g->k;
    if (int rc = check_buffers(fn, {{d_rows, g->rows_elems * eb, eb, true}, {d_row_of, pairs * 4, 4, true}, {d_weights, pairs * 4, 4, false},
                                    {d_add == d_tokens ? nullptr : d_add, g->tokens_elems * eb, eb, false}},
                               {{d_tokens, g->tokens_elems * eb, eb, true}}))
      return rc;
    RowsArgs a = rows_args(g, p);
    a.rows = at(d_rows, p.r.off, eb), a.row_of = d_row_of, a.weights = d_weights, a.add = at(d_add, p.t.off, eb), a.to_tokens = at(d_tokens, p.t.off, eb);
    return finish(launch_rows_combine(a, (hipStream_t)stream), fn);
  });
}

int axe_rows_combine_backward(const axe_rows_desc_t* g, const void* d_dtokens, const void* d_rows, const int32_t* d_row_of, const float* d_weights, void* d_drows,
                              float* d_dweights, void* stream) {
  const char* fn = "axe_rows_combine_backward";
  return guarded(fn, [&]() -> int {
    if (int rc = check_rows(g, fn, false)) return rc;
    if (g->T == 0) return AXE_OK;
    if (g->M == 0) return invalid(fn, "M must be positive");
    RowsPlan p;
    if (int rc = kept_rows_plan(g, fn, p)) return rc;
    const int eb = elem_bytes(g->tokens_dtype);
    const int64_t pairs = g->T * g->k;
    if (d_dweights && !d_rows) return invalid(fn, "NULL device pointer");
    if (int rc = check_buffers(fn, {{d_dtokens, g->tokens_elems * eb, eb, true}, {d_rows == d_drows ? nullptr : d_rows, g->rows_elems * eb, eb, false},
                                    {d_row_of, pairs * 4, 4, true}, {d_weights, pairs * 4, 4, false}},
                               {{d_drows, g->rows_elems * eb, eb, false}, {d_dweights, pairs * 4, 4, false}}))
      return rc;
    if (!d_drows && !d_dweights) return AXE_OK;
    RowsArgs a = rows_args(g, p);
    a.tokens = at(d_dtokens, p.t.off, eb), a.rows = d_dweights ? at(d_rows, p.r.off, eb) : nullptr, a.row_of = d_row_of, a.weights = d_weights;
    a.to_rows = at(d_drows, p.r.off, eb), a.dweights = d_dweights;
    return finish(launch_rows_combine_backward(a, (hipStream_t)stream), fn);
  });
}

}  // extern "C"
