// C entry points of the expert layer and of AdamW (include/imbd.h): argument checks on the host, then one
// call of the kernels' launch functions. No entry allocates, synchronises or throws.

#include <stdlib.h>

#include <algorithm>
#include <cmath>

#include "adamw.h"
#include "expert.h"

namespace imbd {
namespace {

#define FAIL(code, ...)     \
  do {                      \
    set_error(__VA_ARGS__); \
    return (code);          \
  } while (0)

// Row and column numbers plus a tile stay below 2^31.
constexpr int ROWS_MOST = 0x7fffffff - 1024, WIDTH_MOST = 1 << 30;

bool valid_dtype(int d) { return d == IMBD_F32 || d == IMBD_BF16; }

int check_route(int T, int E, int k) {
  if (T < 0 || E < 1 || k < 1) FAIL(IMBD_EINVAL, "bad router sizes: T = %d, E = %d, k = %d", T, E, k);
  if (k > E) FAIL(IMBD_EINVAL, "k = %d experts of E = %d", k, E);
  if (E > EXPERT_MAX || k > CHOICE_MAX)
    FAIL(IMBD_EUNSUPPORTED, "E = %d, k = %d: at most %d experts and %d a token", E, k, EXPERT_MAX, CHOICE_MAX);
  if (T > ROWS_MOST) FAIL(IMBD_EUNSUPPORTED, "T = %d", T);
  if ((int64_t)T * k >= (int64_t)1 << 31) FAIL(IMBD_EUNSUPPORTED, "T * k = %lld pairs", (long long)T * k);
  return IMBD_OK;
}

int check_layer(int dtype, int E, int d_out, int d_in, int n_rows, int n_x) {
  if (!valid_dtype(dtype)) FAIL(IMBD_EINVAL, "unknown dtype %d", dtype);
  if (E < 1 || d_out < 1 || d_in < 1 || n_rows < 0 || n_x < 0)
    FAIL(IMBD_EINVAL, "bad expert sizes: E = %d, d_out = %d, d_in = %d, n_rows = %d, n_x = %d", E, d_out, d_in,
         n_rows, n_x);
  if (E > EXPERT_MAX) FAIL(IMBD_EUNSUPPORTED, "E = %d: at most %d experts", E, EXPERT_MAX);
  if (n_rows > ROWS_MOST || n_x > ROWS_MOST || d_out > WIDTH_MOST || d_in > WIDTH_MOST)
    FAIL(IMBD_EUNSUPPORTED, "n_rows = %d, n_x = %d, d_out = %d, d_in = %d", n_rows, n_x, d_out, d_in);
  return IMBD_OK;
}

int check_weights(const char *what, const void *w, int64_t ldw, int64_t sw, int E, int d_out, int d_in) {
  if (!w) FAIL(IMBD_EINVAL, "%s must be set", what);
  if (ldw < d_in) FAIL(IMBD_EINVAL, "ld%s < d_in", what);
  if (E > 1 && sw < (int64_t)(d_out - 1) * ldw + d_in) FAIL(IMBD_EINVAL, "s%s: experts overlap", what);
  return IMBD_OK;
}

int check_combine(int dtype, int T, int k, int d, int n_rows) {
  if (!valid_dtype(dtype)) FAIL(IMBD_EINVAL, "unknown dtype %d", dtype);
  if (T < 0 || k < 1 || d < 1 || n_rows < 0)
    FAIL(IMBD_EINVAL, "bad sizes: T = %d, k = %d, d = %d, n_rows = %d", T, k, d, n_rows);
  if (k > CHOICE_MAX) FAIL(IMBD_EUNSUPPORTED, "k = %d: at most %d", k, CHOICE_MAX);
  if (T > ROWS_MOST || d > WIDTH_MOST) FAIL(IMBD_EUNSUPPORTED, "T = %d, d = %d", T, d);
  return IMBD_OK;
}

struct Range {
  uintptr_t from, to;
  int tensor;
  bool written;
};

// No tensor's memory in another's (or in its own twice): a step's workgroups run in any order.
int check_apart(const imbd_adamw_tensor *t, int n) {
  Range *r = static_cast<Range *>(malloc((size_t)n * 7 * sizeof(Range)));
  if (!r) FAIL(IMBD_EINVAL, "no host memory to check %d tensors", n);
  int count = 0;
  for (int i = 0; i < n; ++i) {
    const imbd_adamw_tensor &x = t[i];
    if (x.n == 0) continue;
    const size_t e = (size_t)x.n, s = x.state_bits == 8 ? 1 : 4, blocks = (e + 255) / 256;
    auto add = [&](const void *p, size_t bytes, bool written) {
      if (p) r[count++] = Range{(uintptr_t)p, (uintptr_t)p + bytes, i, written};
    };
    add(x.w, e * 4, true);
    add(x.w_lp, e * 2, true);
    add(x.grad, e * (x.grad_dtype == IMBD_BF16 ? 2 : 4), false);
    add(x.m, e * s, true);
    add(x.v, e * s, true);
    if (x.state_bits == 8) {
      add(x.m_scale, blocks * 4, true);
      add(x.v_scale, blocks * 4, true);
    }
  }
  std::sort(r, r + count, [](const Range &a, const Range &b) { return a.from < b.from; });
  // against the furthest end so far, of all ranges and of the written ones
  uintptr_t end = 0, end_written = 0;
  int at = 0, bad = -1;
  for (int i = 0; i < count && bad < 0; ++i) {
    if (r[i].from < (r[i].written ? end : end_written)) bad = r[i].tensor;
    if (r[i].to > end) end = r[i].to, at = r[i].tensor;
    if (r[i].written && r[i].to > end_written) end_written = r[i].to;
  }
  free(r);
  if (bad >= 0) FAIL(IMBD_EINVAL, "tensor %d shares memory with tensor %d", bad, at);
  return IMBD_OK;
}

int check_tensors(const imbd_adamw_tensor *t, int n, size_t *bytes) {
  *bytes = 0;
  if (n < 0 || (n > 0 && !t)) FAIL(IMBD_EINVAL, "n_tensors = %d", n);
  int64_t chunks = 0;
  for (int i = 0; i < n; ++i) {
    const imbd_adamw_tensor &x = t[i];
    if (x.n < 0) FAIL(IMBD_EINVAL, "tensor %d: n = %lld", i, (long long)x.n);
    if (!valid_dtype(x.grad_dtype)) FAIL(IMBD_EINVAL, "tensor %d: unknown grad_dtype %d", i, x.grad_dtype);
    if (x.state_bits != 32 && x.state_bits != 8) FAIL(IMBD_EINVAL, "tensor %d: state_bits = %d", i, x.state_bits);
    if (!(x.decay >= 0.f) || !std::isfinite(x.decay)) FAIL(IMBD_EINVAL, "tensor %d: decay must be finite and >= 0", i);
    if (x.n == 0) continue;
    if (!x.w || !x.grad || !x.m || !x.v) FAIL(IMBD_EINVAL, "tensor %d: w, grad, m and v must be set", i);
    if (x.state_bits == 8 && (!x.m_scale || !x.v_scale))
      FAIL(IMBD_EINVAL, "tensor %d: 8-bit state needs m_scale and v_scale", i);
    if (adamw_chunks(x.n) > 0xffffffffll) FAIL(IMBD_EUNSUPPORTED, "tensor %d: n = %lld", i, (long long)x.n);
    chunks += adamw_chunks(x.n);
  }
  if (chunks > WORKGROUPS_MOST) FAIL(IMBD_EUNSUPPORTED, "%lld chunks are more than one launch takes", (long long)chunks);
  if (chunks > 0) {
    const int rc = check_apart(t, n);
    if (rc != IMBD_OK) return rc;
  }
  if (chunks > 0) *bytes = (size_t)n * adamw_record_bytes() + (size_t)chunks * adamw_entry_bytes();
  return IMBD_OK;
}

int run_product(int pass, int dtype, const ExpertArgs &a, hipStream_t s, bool check = false) {
  if (expert_few_fits(pass, dtype, a)) return run_expert_few(a, s);  // (forward only: never with check)
  return expert_wide_fits(pass, dtype, a) ? run_expert_wide(pass, a, check, s) : run_expert_tile(pass, dtype, a, check, s);
}

hipStream_t stream_of(void *s) { return reinterpret_cast<hipStream_t>(s); }

}  // namespace
}  // namespace imbd

using namespace imbd;

#define TRY(expr)                   \
  do {                              \
    int rc_ = (expr);               \
    if (rc_ != IMBD_OK) return rc_; \
  } while (0)

extern "C" {

size_t expert_route_workspace_bytes(int T, int E, int k) {
  if (check_route(T, E, k) != IMBD_OK) return 0;
  return route_ws_bytes(T, E, k);
}

int expert_route(int T, int E, int k, int renorm, const float *logits, int64_t ldl, float *gates, int32_t *experts,
                 int32_t *offsets, int32_t *rows, int32_t *slots, void *ws, size_t ws_bytes, void *stream) {
  TRY(check_route(T, E, k));
  if (!offsets) FAIL(IMBD_EINVAL, "offsets must be set");
  if (T > 0) {
    if (!logits || !gates || !experts || !rows || !slots)
      FAIL(IMBD_EINVAL, "logits, gates, experts, rows and slots must be set");
    if (ldl < E) FAIL(IMBD_EINVAL, "ldl < E");
    const size_t need = route_ws_bytes(T, E, k);
    if (need && !ws) FAIL(IMBD_EWORKSPACE, "workspace is NULL (need %zu bytes)", need);
    if (need && (uintptr_t)ws % 256) FAIL(IMBD_EINVAL, "workspace must be 256-byte aligned");
    if (ws_bytes < need) FAIL(IMBD_EWORKSPACE, "workspace has %zu bytes, need %zu", ws_bytes, need);
  }
  return run_route(T, E, k, renorm, logits, ldl, gates, experts, offsets, rows, slots, ws, stream_of(stream));
}

int expert_route_bwd(int T, int E, int k, int renorm, const float *logits, int64_t ldl, const float *gates,
                     const int32_t *experts, const float *dgates, float *dlogits, int64_t lddl, void *stream) {
  TRY(check_route(T, E, k));
  if (T == 0) return IMBD_OK;
  if (!gates || !experts || !dgates || !dlogits) FAIL(IMBD_EINVAL, "gates, experts, dgates and dlogits must be set");
  if (!renorm && !logits) FAIL(IMBD_EINVAL, "logits must be set");
  if ((!renorm && ldl < E) || lddl < E) FAIL(IMBD_EINVAL, "leading dimension smaller than the row");
  return run_route_bwd(T, E, k, renorm, logits, ldl, gates, experts, dgates, dlogits, lddl, stream_of(stream));
}

int expert_fwd(int dtype, int relu, int E, int d_out, int d_in, int n_rows, int n_x, const void *w, int64_t ldw,
               int64_t sw, const float *bias, const void *x, int64_t ldx, const int32_t *rows, const int32_t *offsets,
               void *y, int64_t ldy, int y_dtype, void *stream) {
  TRY(check_layer(dtype, E, d_out, d_in, n_rows, n_x));
  if (!valid_dtype(y_dtype)) FAIL(IMBD_EINVAL, "unknown y dtype %d", y_dtype);
  if (n_rows == 0) return IMBD_OK;
  TRY(check_weights("w", w, ldw, sw, E, d_out, d_in));
  if (!offsets || !y || (!x && n_x > 0)) FAIL(IMBD_EINVAL, "x, offsets and y must be set");
  if (!rows && n_x != n_rows) FAIL(IMBD_EINVAL, "without rows, x has n_rows = %d rows, not %d", n_rows, n_x);
  if (ldx < d_in || ldy < d_out) FAIL(IMBD_EINVAL, "leading dimension smaller than the row");
  ExpertArgs a{};
  a.E = E; a.d_out = d_out; a.d_in = d_in; a.n_rows = n_rows; a.n_x = n_x;
  a.w = w; a.ldw = ldw; a.sw = sw; a.bias = bias; a.relu = relu != 0;
  a.x = x; a.ldx = ldx; a.rows = rows; a.offsets = offsets;
  a.out = y; a.ldo = ldy; a.out_dtype = y_dtype;
  return run_product(EXPERT_FWD, dtype, a, stream_of(stream));
}

int expert_bwd(int dtype, int E, int d_out, int d_in, int n_rows, int n_x, const void *w, int64_t ldw, int64_t sw,
               const void *dy, int64_t lddy, const void *x, int64_t ldx, const int32_t *rows, const int32_t *offsets,
               float *dw, int64_t lddw, int64_t sdw, float *db, void *dx, int64_t lddx, int dx_dtype, int mask_relu,
               void *stream) {
  TRY(check_layer(dtype, E, d_out, d_in, n_rows, n_x));
  if (!dw && !db && !dx) FAIL(IMBD_EINVAL, "one of dw, db and dx must be set");
  if (!offsets) FAIL(IMBD_EINVAL, "offsets must be set");
  const bool need_x = dw || (dx && mask_relu);
  if (n_rows > 0) {
    if (!dy) FAIL(IMBD_EINVAL, "dy must be set");
    if (lddy < d_out) FAIL(IMBD_EINVAL, "lddy < d_out");
    if (need_x) {
      if (!x && n_x > 0) FAIL(IMBD_EINVAL, "x must be set");
      if (ldx < d_in) FAIL(IMBD_EINVAL, "ldx < d_in");
      if (!rows && n_x != n_rows) FAIL(IMBD_EINVAL, "without rows, x has n_rows = %d rows, not %d", n_rows, n_x);
    }
  }
  if (dw) TRY(check_weights("dw", dw, lddw, sdw, E, d_out, d_in));
  if (dx) {
    if (!valid_dtype(dx_dtype)) FAIL(IMBD_EINVAL, "unknown dx dtype %d", dx_dtype);
    if (n_rows > 0) TRY(check_weights("w", w, ldw, sw, E, d_out, d_in));
    if (lddx < d_in) FAIL(IMBD_EINVAL, "lddx < d_in");
  }
  ExpertArgs a{};
  a.E = E; a.d_out = d_out; a.d_in = d_in; a.n_rows = n_rows; a.n_x = n_x;
  a.dy = dy; a.lddy = lddy; a.rows = rows; a.offsets = offsets; a.ldx = ldx;
  ExpertArgs g = a;  // the weights' gradient
  const bool grad = dw || db;
  g.x = x;
  if (!dw) g.n_x = 0;  // (db alone: x may be NULL and is not read)
  g.out = dw; g.ldo = lddw; g.so = sdw; g.out_dtype = IMBD_F32;
  g.db = db;
  if (dx && n_rows > 0) {
    if (grad) TRY(run_product(EXPERT_DW, dtype, g, stream_of(stream), true));
    a.w = w; a.ldw = ldw; a.sw = sw;
    a.x = mask_relu ? x : nullptr;
    a.mask = mask_relu != 0;
    a.out = dx; a.ldo = lddx; a.out_dtype = dx_dtype;
    TRY(run_product(EXPERT_DX, dtype, a, stream_of(stream)));
  }
  return grad ? run_product(EXPERT_DW, dtype, g, stream_of(stream)) : IMBD_OK;
}

int expert_combine(int dtype, int T, int k, int d, int n_rows, const void *ys, int64_t ldys, const int32_t *slots,
                   const float *gates, void *y, int64_t ldy, int y_dtype, void *stream) {
  TRY(check_combine(dtype, T, k, d, n_rows));
  if (!valid_dtype(y_dtype)) FAIL(IMBD_EINVAL, "unknown y dtype %d", y_dtype);
  if (T == 0) return IMBD_OK;
  if (!slots || !y || (!ys && n_rows > 0)) FAIL(IMBD_EINVAL, "ys, slots and y must be set");
  if (ldys < d || ldy < d) FAIL(IMBD_EINVAL, "leading dimension smaller than the row");
  return run_combine(dtype, T, k, d, n_rows, ys, ldys, slots, gates, y, ldy, y_dtype, stream_of(stream));
}

int expert_combine_bwd(int dtype, int T, int k, int d, int n_rows, const void *dy, int64_t lddy, const void *ys,
                       int64_t ldys, const int32_t *slots, const float *gates, void *dys, int64_t lddys,
                       float *dgates, void *stream) {
  TRY(check_combine(dtype, T, k, d, n_rows));
  if (T == 0) return IMBD_OK;
  if (!dy || !slots || !gates) FAIL(IMBD_EINVAL, "dy, slots and gates must be set");
  if (n_rows > 0 && (!dys || (dgates && !ys))) FAIL(IMBD_EINVAL, "ys and dys must be set");
  if (lddy < d || lddys < d || (dgates && ldys < d)) FAIL(IMBD_EINVAL, "leading dimension smaller than the row");
  return run_combine_bwd(dtype, T, k, d, n_rows, dy, lddy, ys, ldys, slots, gates, dys, lddys, dgates,
                         stream_of(stream));
}

size_t adamw_plan_bytes(const imbd_adamw_tensor *tensors, int n_tensors) {
  size_t bytes;
  return check_tensors(tensors, n_tensors, &bytes) == IMBD_OK ? bytes : 0;
}

int adamw_plan(const imbd_adamw_tensor *tensors, int n_tensors, void *plan, size_t plan_bytes) {
  size_t bytes;
  TRY(check_tensors(tensors, n_tensors, &bytes));
  if (bytes == 0) return IMBD_OK;
  if (!plan || (uintptr_t)plan % 8) FAIL(IMBD_EINVAL, "plan must be set and 8-byte aligned");
  if (plan_bytes < bytes) FAIL(IMBD_EWORKSPACE, "plan has %zu bytes, need %zu", plan_bytes, bytes);
  adamw_write_plan(tensors, n_tensors, plan);
  return IMBD_OK;
}

int adamw_step(const void *plan, size_t plan_bytes, int n_tensors, double lr, double beta1, double beta2, double eps,
               float grad_scale, int step, const int32_t *step_dev, void *stream) {
  if (n_tensors < 0) FAIL(IMBD_EINVAL, "n_tensors = %d", n_tensors);
  if (!std::isfinite(lr) || !std::isfinite(grad_scale)) FAIL(IMBD_EINVAL, "lr and grad_scale must be finite");
  if (!(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1)) FAIL(IMBD_EINVAL, "betas must lie in [0, 1)");
  if (!(eps >= 0) || !std::isfinite(eps)) FAIL(IMBD_EINVAL, "eps must be finite and >= 0");
  // what the kernel takes in fp32: 0 / 0 and 0 * infinity where an element has no gradient
  if (eps > 0 && (float)eps == 0.f) FAIL(IMBD_EINVAL, "eps = %g is zero in fp32", eps);
  if (!std::isfinite((float)(lr / (1 - beta1)))) FAIL(IMBD_EINVAL, "lr / (1 - beta1) = %g overflows fp32", lr / (1 - beta1));
  if (!step_dev && step < 1) FAIL(IMBD_EINVAL, "step = %d, need >= 1", step);
  if (plan_bytes == 0) return IMBD_OK;
  if (!plan || (uintptr_t)plan % 16) FAIL(IMBD_EINVAL, "plan must be set and 16-byte aligned");
  const size_t head = (size_t)n_tensors * adamw_record_bytes();
  if (plan_bytes <= head || (plan_bytes - head) % adamw_entry_bytes())
    FAIL(IMBD_EINVAL, "plan_bytes = %zu is no plan of %d tensors", plan_bytes, n_tensors);
  const size_t chunks = (plan_bytes - head) / adamw_entry_bytes();
  if (n_tensors == 0 || chunks > (size_t)WORKGROUPS_MOST) FAIL(IMBD_EINVAL, "plan_bytes = %zu is no plan", plan_bytes);
  return run_adamw(plan, n_tensors, (int64_t)chunks, lr, beta1, beta2, eps, grad_scale, step, step_dev,
                   stream_of(stream));
}

}  // extern "C"
