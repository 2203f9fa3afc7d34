// C entry points of a fully connected layer with activation and residual (include/imbd.h): argument checks on the host,
// then the launches. No entry allocates, synchronises or throws.

#include "dense.h"

namespace imbd {
namespace {

#define FAIL(code, ...)     \
  do {                      \
    set_error(__VA_ARGS__); \
    return (code);          \
  } while (0)
#define TRY(expr)                   \
  do {                              \
    int rc_ = (expr);               \
    if (rc_ != IMBD_OK) return rc_; \
  } while (0)

// Row and column numbers plus a tile stay below 2^31.
constexpr int ROWS_MOST = 0x7fffffff - 1024, WIDTH_MOST = 1 << 30;

bool valid_dtype(int d) { return d == IMBD_F32 || d == IMBD_BF16; }

int check_sizes(int dtype, int d_out, int d_in, int B) {
  if (!valid_dtype(dtype)) FAIL(IMBD_EINVAL, "unknown dtype %d", dtype);
  if (d_out < 1 || d_in < 1 || B < 0) FAIL(IMBD_EINVAL, "bad sizes: d_out = %d, d_in = %d, B = %d", d_out, d_in, B);
  if (B > ROWS_MOST || d_out > WIDTH_MOST || d_in > WIDTH_MOST)
    FAIL(IMBD_EUNSUPPORTED, "d_out = %d, d_in = %d, B = %d", d_out, d_in, B);
  return IMBD_OK;
}

int check_act(int act) {
  if (act < IMBD_ACT_NONE || act > IMBD_ACT_SILU) FAIL(IMBD_EINVAL, "unknown activation %d", act);
  return IMBD_OK;
}

int check_ws(size_t need, const void *ws, size_t ws_bytes) {
  if (need && !ws) FAIL(IMBD_EWORKSPACE, "workspace is NULL (need %zu bytes)", need);
  if (need && (uintptr_t)ws % 256) FAIL(IMBD_EINVAL, "workspace must be 256-byte aligned");
  if (ws_bytes < need) FAIL(IMBD_EWORKSPACE, "workspace has %zu bytes, need %zu", ws_bytes, need);
  return IMBD_OK;
}

hipStream_t stream_of(void *s) { return reinterpret_cast<hipStream_t>(s); }

}  // namespace
}  // namespace imbd

using namespace imbd;

extern "C" {

size_t linear_workspace_bytes(int which, int dtype, int d_out, int d_in, int B) {
  if ((which != 0 && which != 1) || check_sizes(dtype, d_out, d_in, B) != IMBD_OK) return 0;
  return linear_ws_bytes(which, dtype, d_out, d_in, B);
}

int linear_fwd(int dtype, int act, int d_out, int d_in, int B, const void *w, int64_t ldw, const float *bias,
               const void *x, int64_t ldx, const void *residual, int64_t ldr, void *y, int64_t ldy, int y_dtype, void *z,
               int64_t ldz, void *ws, size_t ws_bytes, void *stream) {
  TRY(check_sizes(dtype, d_out, d_in, B));
  TRY(check_act(act));
  if (!valid_dtype(y_dtype)) FAIL(IMBD_EINVAL, "unknown y dtype %d", y_dtype);
  if (B == 0) return IMBD_OK;
  if (!w || !x || !y) FAIL(IMBD_EINVAL, "w, x and y must be set");
  if (ldw < d_in || ldx < d_in || ldy < d_out || (residual && ldr < d_out) || (z && ldz < d_out))
    FAIL(IMBD_EINVAL, "leading dimension smaller than the row");
  if (residual == y && ldr != ldy) FAIL(IMBD_EINVAL, "a residual in the place of y has to have its leading dimension");
  if (z && (z == y || z == residual)) FAIL(IMBD_EINVAL, "z has to have memory of its own");
  TRY(check_ws(linear_ws_bytes(0, dtype, d_out, d_in, B), ws, ws_bytes));
  LinearArgs a{};
  a.dtype = dtype; a.d_out = d_out; a.d_in = d_in; a.B = B;
  a.w = w; a.ldw = ldw; a.bias = bias; a.x = x; a.ldx = ldx;
  a.act = act; a.z = z; a.ldz = ldz; a.res = residual; a.ldr = ldr;
  a.out = y; a.ldo = ldy; a.out_dtype = y_dtype;
  return run_linear_fwd(a, ws, stream_of(stream));
}

int linear_bwd(int dtype, int act, int d_out, int d_in, int B, const void *w, int64_t ldw, const void *dy, int64_t lddy,
               const void *x, int64_t ldx, float *dw, int64_t lddw, float *db, const void *z, int64_t ldz,
               const void *residual, int64_t ldr, void *dx, int64_t lddx, int dx_dtype, void *ws, size_t ws_bytes,
               void *stream) {
  TRY(check_sizes(dtype, d_out, d_in, B));
  TRY(check_act(act));
  if (!dw && !db && !dx) FAIL(IMBD_EINVAL, "one of dw, db and dx must be set");
  if (dx && !valid_dtype(dx_dtype)) FAIL(IMBD_EINVAL, "unknown dx dtype %d", dx_dtype);
  if (dw && lddw < d_in) FAIL(IMBD_EINVAL, "lddw < d_in");
  if (B > 0) {
    if (!dy || lddy < d_out) FAIL(IMBD_EINVAL, "dy must be set, rows of d_out apart at least");
    if (dw && (!x || ldx < d_in)) FAIL(IMBD_EINVAL, "x must be set, rows of d_in apart at least");
    if (dx) {
      if (!w) FAIL(IMBD_EINVAL, "w must be set");
      if (act != IMBD_ACT_NONE && !z) FAIL(IMBD_EINVAL, "z must be set");
      if (ldw < d_in || lddx < d_in || (act != IMBD_ACT_NONE && ldz < d_in) || (residual && ldr < d_in))
        FAIL(IMBD_EINVAL, "leading dimension smaller than the row");
      if (residual == dx && ldr != lddx) FAIL(IMBD_EINVAL, "a residual in the place of dx has to have its leading dimension");
    }
  }
  TRY(check_ws(linear_ws_bytes(1, dtype, d_out, d_in, B), ws, ws_bytes));
  LinearArgs a{};
  a.dtype = dtype; a.d_out = d_out; a.d_in = d_in; a.B = B;
  a.w = w; a.ldw = ldw; a.x = x; a.ldx = ldx; a.dy = dy; a.lddy = lddy;
  a.act = act; a.z = const_cast<void *>(z); a.ldz = ldz; a.res = residual; a.ldr = ldr;
  a.out = dx; a.ldo = lddx; a.out_dtype = dx_dtype;
  a.dw = dw; a.lddw = lddw; a.db = db;
  return run_linear_bwd(a, ws, stream_of(stream));
}

int act_bwd(int dtype, int act, int B, int d, const void *dy, int64_t lddy, const void *z, int64_t ldz, void *dz,
            int64_t lddz, void *stream) {
  TRY(check_sizes(dtype, d, 1, B));
  TRY(check_act(act));
  if (B == 0) return IMBD_OK;
  if (!dy || !z || !dz) FAIL(IMBD_EINVAL, "dy, z and dz must be set");
  if (lddy < d || ldz < d || lddz < d) FAIL(IMBD_EINVAL, "leading dimension smaller than the row");
  if ((dz == dy && lddz != lddy) || (dz == z && lddz != ldz))
    FAIL(IMBD_EINVAL, "dz in the place of an input has to have its leading dimension");
  return run_act_bwd(dtype, act, B, d, dy, lddy, z, ldz, dz, lddz, stream_of(stream));
}

}  // extern "C"
