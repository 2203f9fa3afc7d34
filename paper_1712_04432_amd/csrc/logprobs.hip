// Log probabilities of given tokens, with the entropy and the top alternatives of every row, and their gradient.
//
// A workgroup a row. The sums of the softmax are carried in one pass (RowSums in csrc/vocab.h); the alternatives
// are found one after another, each the largest (logit, lowest token) below the one before.

#include "order_key.h"
#include "vocab.h"

namespace imbd {
namespace {

struct LogprobsArgs {
  int B, V, n;
  const void *logits;
  int64_t ldz;
  const int32_t *tokens;
  float inv_t, c;
  float *logp, *entropy, *lse;
  int32_t *top_ids;
  float *top_logp;
};

// A logit and its token as one number: larger logits first, then lower tokens. 0: none.
__device__ __forceinline__ uint64_t choice_key(float z, int v) {
  const uint32_t k = order_key(z);
  if (z != z || k <= KEY_MINUS_INF) return 0;
  return ((uint64_t)k << 32) | (uint32_t)~v;
}

template <typename T>
__global__ void __launch_bounds__(256) logprobs_kernel(LogprobsArgs a) {
  __shared__ RowSums part[4];
  __shared__ uint64_t best[4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int64_t b = blockIdx.x;
  const T *z = reinterpret_cast<const T *>(a.logits) + b * a.ldz;
  RowSums r{LOWEST, 0.f, 0.f};
  for (int64_t v = tid; v < a.V; v += 256) {
    const float x = load_f32(z + v);
    if (x > r.m) r = moved(r, x, a.c);
    const float d = scaled(x, r.m, a.c), e = pow2(d);
    r.s += e;
    r.u += e * d;
  }
  r = wave_joined(r, a.c);
  if (lane == 0) part[wave] = r;
  __syncthreads();
  r = joined(joined(part[0], part[1], a.c), joined(part[2], part[3], a.c), a.c);
  const float ls = logf(r.s);
  if (tid == 0) {
    const int t = a.tokens[b];
    a.logp[b] = t < 0 ? 0.f : t >= a.V ? __builtin_nanf("") : (load_f32(z + t) - r.m) * a.inv_t - ls;
    if (a.entropy) a.entropy[b] = ls - LN2 * (r.u / r.s);
    if (a.lse) a.lse[b] = r.m * a.inv_t + ls;
  }
  uint64_t last = ~(uint64_t)0;
  for (int j = 0; j < a.n; ++j) {
    uint64_t k = 0;
    for (int64_t v = tid; v < a.V; v += 256) {
      const uint64_t x = choice_key(load_f32(z + v), (int)v);
      if (x < last && x > k) k = x;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t x = __shfl_xor((unsigned long long)k, o, 64);
      k = x > k ? x : k;
    }
    __syncthreads();
    if (lane == 0) best[wave] = k;
    __syncthreads();
    last = max(max(best[0], best[1]), max(best[2], best[3]));
    if (tid == 0) {
      a.top_ids[b * a.n + j] = last ? (int)~(uint32_t)last : -1;
      a.top_logp[b * a.n + j] = last ? (key_value((uint32_t)(last >> 32)) - r.m) * a.inv_t - ls : -INFINITY;
    }
    if (!last) last = 1;  // (nothing is below it)
  }
}

struct LogprobsBwdArgs {
  int V;
  const void *logits;
  int64_t ldz;
  const int32_t *tokens;
  float inv_t;
  const float *lse, *entropy, *dlogp, *dentropy;
  void *dlogits;
  int64_t lddl;
};

template <typename T, typename TO>
__global__ void __launch_bounds__(256) logprobs_bwd_kernel(LogprobsBwdArgs a) {
  const int64_t b = blockIdx.x;
  const T *z = reinterpret_cast<const T *>(a.logits) + b * a.ldz;
  TO *out = reinterpret_cast<TO *>(a.dlogits) + b * a.lddl;
  const int t = a.tokens[b];
  float g = a.dlogp && t >= 0 ? a.dlogp[b] : 0.f;
  const float h = a.dentropy ? a.dentropy[b] : 0.f;
  const bool none = g == 0.f && h == 0.f;
  if (t >= a.V && !none) g = __builtin_nanf("");
  const float lse = a.lse[b], add = h == 0.f ? 0.f : a.entropy[b];
  for (int64_t v = threadIdx.x; v < a.V; v += 256) {
    const float lq = __builtin_elementwise_maximum(load_f32(z + v) * a.inv_t - lse, -200.f), q = pow2(lq * LOG2E);
    const float d = (v == t ? g : 0.f) - q * (g + h * (lq + add));
    store_f32(out + v, none ? 0.f : d * a.inv_t);
  }
}

}  // namespace

size_t logprobs_ws_bytes(int B, int V, int n) { return 0; }

int run_logprobs(int dtype, int B, int V, int n, const void *logits, int64_t ldz, const int32_t *tokens,
                 float temperature, float *logp, float *entropy, float *lse, int32_t *top_ids, float *top_logp, void *ws,
                 hipStream_t s) {
  const float inv_t = 1.0f / temperature;
  LogprobsArgs a{B, V, n, logits, ldz, tokens, inv_t, inv_t * LOG2E, logp, entropy, lse, top_ids, top_logp};
  {
    LaunchTimer t(IMBD_K_LOGPROBS, 0, s);
    if (dtype == IMBD_BF16) hipLaunchKernelGGL(logprobs_kernel<uint16_t>, dim3(B), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(logprobs_kernel<float>, dim3(B), dim3(256), 0, s, a);
  }
  return check_launch("token_logprobs");
}

int run_logprobs_bwd(int dtype, int B, int V, const void *logits, int64_t ldz, const int32_t *tokens,
                     float temperature, const float *lse, const float *entropy, const float *dlogp,
                     const float *dentropy, void *dlogits, int64_t lddl, int dlogits_dtype, hipStream_t s) {
  LogprobsBwdArgs a{V, logits, ldz, tokens, 1.0f / temperature, lse, entropy, dlogp, dentropy, dlogits, lddl};
  const dim3 grid(B), wg(256);
  {
    LaunchTimer t(IMBD_K_LOGPROBS, 1, s);
    if (dtype == IMBD_BF16 && dlogits_dtype == IMBD_BF16)
      hipLaunchKernelGGL((logprobs_bwd_kernel<uint16_t, uint16_t>), grid, wg, 0, s, a);
    else if (dtype == IMBD_BF16) hipLaunchKernelGGL((logprobs_bwd_kernel<uint16_t, float>), grid, wg, 0, s, a);
    else if (dlogits_dtype == IMBD_BF16) hipLaunchKernelGGL((logprobs_bwd_kernel<float, uint16_t>), grid, wg, 0, s, a);
    else hipLaunchKernelGGL((logprobs_bwd_kernel<float, float>), grid, wg, 0, s, a);
  }
  return check_launch("token_logprobs_bwd");
}

}  // namespace imbd
