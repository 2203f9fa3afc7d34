// Divergence of a student's softmax from a teacher of whose logits the top ones are known, and its gradient.
//
// A workgroup a row: the teacher's entries (one a thread), the sums of the student's softmax in one pass over the logits
// (RowSums in csrc/vocab.h), the row's loss, then the gradient in a second pass. The entries' tokens get theirs last,
// each from the sum over the entries that name the same token, so that two of them write the same value.

#include "loss_mean.h"
#include "vocab.h"

namespace imbd {
namespace {

struct DistillArgs {
  int B, V, K;
  const void *logits;
  int64_t ldz;
  const int32_t *ids;
  const float *teacher, *lse, *weight;
  float t, inv_t, c, inv_batch;
  float *row_loss;
  void *dlogits;
  int64_t lddl;
};

template <typename T, typename TO>
__global__ void __launch_bounds__(256) distill_kernel(DistillArgs a) {
  __shared__ RowSums part[4];
  __shared__ float red[4];
  __shared__ int id_of[ENTRIES_MOST];
  __shared__ float p_of[ENTRIES_MOST];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int64_t b = blockIdx.x;
  const T *z = reinterpret_cast<const T *>(a.logits) + b * a.ldz;
  TO *out = a.dlogits ? reinterpret_cast<TO *>(a.dlogits) + b * a.lddl : nullptr;
  auto all_max = [&](float v) {
    v = wave_maximum(v);
    __syncthreads();
    if (lane == 0) red[wave] = v;
    __syncthreads();
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(red[0], red[1]),
                                         __builtin_elementwise_maximum(red[2], red[3]));
  };
  auto all_sum = [&](float v) {
    v = wave_sum(v);
    __syncthreads();
    if (lane == 0) red[wave] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
  };
  // ---- the teacher
  const float w = a.weight ? a.weight[b] : 1.f;
  int id = -1;
  float t = -INFINITY;
  if (tid < a.K) {
    id = a.ids[b * a.K + tid];
    if (id >= 0) t = a.teacher[b * a.K + tid] * a.inv_t;
    if (t == -INFINITY) id = -1;
  }
  const bool outside = all_max(id >= a.V ? 1.f : 0.f) > 0.f;
  const float top = all_max(t);
  if (w == 0.f || top == -INFINITY) {  // nothing to learn from
    if (tid == 0) a.row_loss[b] = 0.f;
    if (out)
      for (int64_t v = tid; v < a.V; v += 256) store_f32(out + v, 0.f);
    return;
  }
  float lt;
  if (a.lse) lt = a.lse[b];
  else lt = top + logf(all_sum(id < 0 ? 0.f : expf(t - top)));
  const float lp = t - lt, p = id < 0 ? 0.f : expf(lp);
  const float mass = all_sum(p);
  float at = 0.f;  // the student's logit
  if (id >= 0 && id < a.V) at = load_f32(z + id);
  id_of[tid] = id;
  p_of[tid] = p;
  // ---- the student's sums
  RowSums r{LOWEST, 0.f, 0.f};
  for (int64_t v = tid; v < a.V; v += 256) {
    const float x = load_f32(z + v);
    if (x > r.m) r = moved(r, x, a.c);
    r.s += pow2(scaled(x, r.m, a.c));
  }
  r = wave_joined(r, a.c);
  if (lane == 0) part[wave] = r;
  __syncthreads();
  r = joined(joined(part[0], part[1], a.c), joined(part[2], part[3], a.c), a.c);
  const float ls = logf(r.s), bad = outside || r.s == 0.f ? __builtin_nanf("") : 0.f;
  const float kl = all_sum(p != 0.f ? p * (lp - ((at - r.m) * a.inv_t - ls)) : 0.f);
  if (tid == 0) a.row_loss[b] = w * (a.t * a.t) * kl + bad;
  if (!out) return;
  // ---- the gradient
  const float scale = a.inv_batch * w * a.t + bad, q1 = mass / r.s;
  auto slope = [&](float x, float pv) { return scale * (pow2(scaled(x, r.m, a.c)) * q1 - pv); };
  float same = 0.f;
  if (id >= 0)
    for (int j = 0; j < a.K; ++j) same += id_of[j] == id ? p_of[j] : 0.f;
  for (int64_t v = tid; v < a.V; v += 256) store_f32(out + v, slope(load_f32(z + v), 0.f));
  __syncthreads();
  if (id >= 0 && id < a.V) store_f32(out + id, slope(at, same));
}

__global__ void __launch_bounds__(256) distill_loss_kernel(int B, const float *row_loss, float inv_batch, float *loss) {
  __shared__ float part[256];
  block_loss_mean(B, row_loss, inv_batch, loss, part);
}

}  // namespace

size_t distill_ws_bytes(int B, int V, int K) { return 0; }

int run_distill(int dtype, int B, int V, int K, const void *logits, int64_t ldz, const int32_t *ids,
                const float *teacher, const float *lse, const float *weight, float temperature, float inv_batch,
                float *loss, float *row_loss, void *dlogits, int64_t lddl, int dlogits_dtype, void *ws, hipStream_t s) {
  const float inv_t = 1.0f / temperature;
  DistillArgs a{B, V, K, logits, ldz, ids, teacher, lse, weight, temperature, inv_t, inv_t * LOG2E, inv_batch,
                row_loss, dlogits, lddl};
  const dim3 grid(B), wg(256);
  if (B > 0) {
    LaunchTimer t(IMBD_K_DISTILL, 0, s);
    if (dtype == IMBD_BF16 && dlogits_dtype == IMBD_BF16)
      hipLaunchKernelGGL((distill_kernel<uint16_t, uint16_t>), grid, wg, 0, s, a);
    else if (dtype == IMBD_BF16) hipLaunchKernelGGL((distill_kernel<uint16_t, float>), grid, wg, 0, s, a);
    else if (dlogits_dtype == IMBD_BF16) hipLaunchKernelGGL((distill_kernel<float, uint16_t>), grid, wg, 0, s, a);
    else hipLaunchKernelGGL((distill_kernel<float, float>), grid, wg, 0, s, a);
  }
  const int rc = check_launch("distill_xent");
  if (rc != IMBD_OK) return rc;
  hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(256), 0, s, B, row_loss, inv_batch, loss);
  return check_launch("distill_xent (loss)");
}

}  // namespace imbd
