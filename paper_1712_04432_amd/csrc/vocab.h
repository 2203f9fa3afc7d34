// Rows of logits over a vocabulary (csrc/logprobs.hip, csrc/distill.hip): internal declarations and the pieces that
// their kernels share.
#pragma once

#include "cdna4.h"

namespace imbd {

constexpr int TOP_MOST = 64;         // alternatives
constexpr int ENTRIES_MOST = 256;    // a teacher's entries of a row
constexpr int VOCAB_MOST = 1 << 30;
constexpr int VOCAB_ROWS_MOST = (1 << 24) - 1;  // a workgroup each: 2^32 work-items are a launch's most

size_t logprobs_ws_bytes(int B, int V, int n);
int run_logprobs(int dtype, int B, int V, int n, const void *logits, int64_t ldz, const int32_t *tokens,
                 float temperature, float *logp, float *entropy, float *lse, int32_t *top_ids, float *top_logp, void *ws,
                 hipStream_t s);
int run_logprobs_bwd(int dtype, int B, int V, const void *logits, int64_t ldz, const int32_t *tokens,
                     float temperature, const float *lse, const float *entropy, const float *dlogp,
                     const float *dentropy, void *dlogits, int64_t lddl, int dlogits_dtype, hipStream_t s);
size_t distill_ws_bytes(int B, int V, int K);
int run_distill(int dtype, int B, int V, int K, const void *logits, int64_t ldz, const int32_t *ids,
                const float *teacher, const float *lse, const float *weight, float temperature, float inv_batch,
                float *loss, float *row_loss, void *dlogits, int64_t lddl, int dlogits_dtype, void *ws, hipStream_t s);

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

template <typename T>
__device__ __forceinline__ float load_f32(const T *p) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(*p);
  else return *p;
}
template <typename T>
__device__ __forceinline__ void store_f32(T *p, float v) {
  if constexpr (sizeof(T) == 2) *p = f32_to_bf16(v);
  else *p = v;
}

// What a softmax over a row needs, over part of it: m a reference (near the largest logit), s the sum of
// e = 2^d with d = (z - m) * c, c = log2(e) / temperature, and u the sum of e d, of which the entropy is made:
//   lse = m / temperature + ln s        entropy = ln s - ln 2 * u / s
// A part without a logit above -inf has s = 0; its m is the lowest finite value. A NaN or +inf makes s NaN.
struct RowSums {
  float m, s, u;
};
constexpr float LOWEST = -3.402823466e38f;

// 2^x to one unit in the last place; 0 where that is under the smallest normal number
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }
// d of a logit, so far down that 2^d is 0 instead of -inf (0 * -inf would be NaN); a NaN stays one
__device__ __forceinline__ float scaled(float z, float m, float c) {
  return __builtin_elementwise_maximum((z - m) * c, -200.f);
}
// The sums `r` with their reference moved to m >= r.m.
__device__ __forceinline__ RowSums moved(const RowSums &r, float m, float c) {
  const float d = scaled(r.m, m, c), f = pow2(d);
  return RowSums{m, f * r.s, f * (r.u + d * r.s)};
}
__device__ __forceinline__ RowSums joined(const RowSums &a, const RowSums &b, float c) {
  const float m = fmaxf(a.m, b.m);
  const RowSums x = moved(a, m, c), y = moved(b, m, c);
  return RowSums{m, x.s + y.s, x.u + y.u};
}
__device__ __forceinline__ RowSums wave_joined(RowSums r, float c) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const RowSums b{__shfl_xor(r.m, o, 64), __shfl_xor(r.s, o, 64), __shfl_xor(r.u, o, 64)};
    r = joined(r, b, c);
  }
  return r;
}

}  // namespace imbd
