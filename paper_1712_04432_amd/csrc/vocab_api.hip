// C entry points of what a vocabulary's logits are for (include/imbd.h): argument checks on the host, then one call of
// the kernels' launch functions. No entry allocates, synchronises or throws.

#include <cmath>

#include "vocab.h"

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

bool valid_dtype(int d) { return d == IMBD_F32 || d == IMBD_BF16; }

int check_rows(int B, int V) {
  if (B < 0 || V < 1) FAIL(IMBD_EINVAL, "bad sizes: B = %d, V = %d", B, V);
  if (B > VOCAB_ROWS_MOST || V > VOCAB_MOST) FAIL(IMBD_EUNSUPPORTED, "B = %d, V = %d", B, V);
  return IMBD_OK;
}

int check_distill(int B, int V, int K) {
  TRY(check_rows(B, V));
  if (K < 1) FAIL(IMBD_EINVAL, "K = %d", K);
  if (K > ENTRIES_MOST) FAIL(IMBD_EUNSUPPORTED, "K = %d: at most %d entries", K, ENTRIES_MOST);
  return IMBD_OK;
}

int check_top(int B, int V, int n) {
  TRY(check_rows(B, V));
  if (n < 0) FAIL(IMBD_EINVAL, "n = %d", n);
  if (n > TOP_MOST) FAIL(IMBD_EUNSUPPORTED, "n = %d: at most %d alternatives", n, TOP_MOST);
  return IMBD_OK;
}

int check_temperature(float t) {
  // (log2(e) / temperature has to be a number too)
  if (!(t > 0.f) || !std::isfinite(t) || !std::isfinite(2.0f / t) || 1.0f / t == 0.f)
    FAIL(IMBD_EINVAL, "temperature = %g has to be finite and above 0, and so its reciprocal", (double)t);
  return IMBD_OK;
}

int check_gradient(int dtype, const void *logits, int64_t ldz, const void *dlogits, int64_t lddl, int dl_dtype, int V) {
  if (!valid_dtype(dl_dtype)) FAIL(IMBD_EINVAL, "unknown dlogits dtype %d", dl_dtype);
  if (lddl < V) FAIL(IMBD_EINVAL, "lddl %lld < V %d", (long long)lddl, V);
  if (dlogits == logits && (lddl != ldz || dl_dtype != dtype))
    FAIL(IMBD_EINVAL, "dlogits in place of logits has to have their type and leading dimension");
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

size_t distill_workspace_bytes(int B, int V, int K) {
  return check_distill(B, V, K) == IMBD_OK ? distill_ws_bytes(B, V, K) : 0;
}

int distill_xent(int dtype, int B, int V, int K, const void *logits, int64_t ldz, const int32_t *ids,
                 const float *teacher, const float *lse, const float *weight, float temperature, float inv_batch,
                 float *loss, float *row_loss, void *dlogits, int64_t lddl, int dlogits_dtype, void *ws,
                 size_t ws_bytes, void *stream) {
  TRY(check_distill(B, V, K));
  if (!valid_dtype(dtype)) FAIL(IMBD_EINVAL, "unknown dtype %d", dtype);
  if (!loss) FAIL(IMBD_EINVAL, "loss must be set");
  if (B > 0 && (!logits || !ids || !teacher || !row_loss))
    FAIL(IMBD_EINVAL, "logits, ids, teacher and row_loss must be set");
  if (B > 0 && ldz < V) FAIL(IMBD_EINVAL, "ldz %lld < V %d", (long long)ldz, V);
  if (dlogits) TRY(check_gradient(dtype, logits, ldz, dlogits, lddl, dlogits_dtype, V));
  TRY(check_temperature(temperature));
  if (!std::isfinite(temperature * temperature)) FAIL(IMBD_EINVAL, "temperature = %g", (double)temperature);
  if (!std::isfinite(inv_batch)) FAIL(IMBD_EINVAL, "inv_batch must be finite");
  TRY(check_ws(distill_ws_bytes(B, V, K), ws, ws_bytes));
  return run_distill(dtype, B, V, K, logits, ldz, ids, teacher, lse, weight, temperature, inv_batch, loss, row_loss,
                     dlogits, lddl, dlogits_dtype, ws, stream_of(stream));
}

size_t token_logprobs_workspace_bytes(int B, int V, int n) {
  return check_top(B, V, n) == IMBD_OK ? logprobs_ws_bytes(B, V, n) : 0;
}

int token_logprobs(int dtype, int B, int V, int n, const void *logits, int64_t ldz, const int32_t *tokens,
                   float temperature, float *logp, float *entropy, float *lse, int32_t *top_ids, float *top_logp,
                   void *ws, size_t ws_bytes, void *stream) {
  TRY(check_top(B, V, n));
  if (!valid_dtype(dtype)) FAIL(IMBD_EINVAL, "unknown dtype %d", dtype);
  TRY(check_temperature(temperature));
  if (B == 0) return IMBD_OK;
  if (!logits || !tokens || !logp) FAIL(IMBD_EINVAL, "logits, tokens and logp must be set");
  if (n > 0 && (!top_ids || !top_logp)) FAIL(IMBD_EINVAL, "top_ids and top_logp must be set");
  if (ldz < V) FAIL(IMBD_EINVAL, "ldz %lld < V %d", (long long)ldz, V);
  TRY(check_ws(logprobs_ws_bytes(B, V, n), ws, ws_bytes));
  return run_logprobs(dtype, B, V, n, logits, ldz, tokens, temperature, logp, entropy, lse, top_ids, top_logp, ws,
                      stream_of(stream));
}

int token_logprobs_bwd(int dtype, int B, int V, const void *logits, int64_t ldz, const int32_t *tokens,
                       float temperature, const float *lse, const float *entropy, const float *dlogp,
                       const float *dentropy, void *dlogits, int64_t lddl, int dlogits_dtype, void *stream) {
  TRY(check_rows(B, V));
  if (!valid_dtype(dtype)) FAIL(IMBD_EINVAL, "unknown dtype %d", dtype);
  TRY(check_temperature(temperature));
  if (B == 0) return IMBD_OK;
  if (!logits || !tokens || !lse || !dlogits) FAIL(IMBD_EINVAL, "logits, tokens, lse and dlogits must be set");
  if (dentropy && !entropy) FAIL(IMBD_EINVAL, "entropy must be set where dentropy is");
  if (ldz < V) FAIL(IMBD_EINVAL, "ldz %lld < V %d", (long long)ldz, V);
  TRY(check_gradient(dtype, logits, ldz, dlogits, lddl, dlogits_dtype, V));
  return run_logprobs_bwd(dtype, B, V, logits, ldz, tokens, temperature, lse, entropy, dlogp, dentropy, dlogits, lddl,
                          dlogits_dtype, stream_of(stream));
}

}  // extern "C"
