// The gated sum of the experts' outputs back into token order, and its backward pass:
//   y[t]       = sum_j g[t][j] ys[slot[t][j]]
//   dys[slot]  = g[t][j] dy[t],   dg[t][j] = dy[t] . ys[slot[t][j]]
// Both are streams: every row of ys is read (and of dys written) once, in whole 16-byte chunks where base
// and pitch allow, 0.5 flop a byte. Outputs are stored past the caches (nothing here reads them again; 16384
// tokens, k = 2, 4096 columns of bf16: 80 -> 59 us, backward 148 -> 130 us; reading past them too, 72 and 165). Elsewhere
// a thread takes one element: 4095 columns, 316 and 312 us (fp32 344 and 335, where 4096 take 147 and 286). The backward
// pass is one wave a token: 64 tokens, k = 8, 4096 columns 27 us, 16 tokens, k = 4, 14.

#include "expert.h"

namespace imbd {
namespace {

struct CombineArgs {
  int T, k, d, n_rows;
  const void *ys, *dy;
  int64_t ldys, lddy;
  const int32_t *slots;
  const float *gates;
  void *y, *dys;
  int64_t ldy, lddys;
  float *dgates;
};

// VEC consecutive elements as floats.
template <typename T, int VEC>
__device__ __forceinline__ void load_f32(const T *p, float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    if constexpr (sizeof(T) == 2) v[0] = bf16_to_f32(*p);
    else v[0] = *p;
  } else if constexpr (sizeof(T) == 2) {
    static_assert(VEC == 8, "");
    const u32x4 q = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = bf16_to_f32((uint16_t)(q[e >> 1] >> (16 * (e & 1))));
  } else {
    static_assert(VEC == 4 || VEC == 8, "");
#pragma unroll
    for (int h = 0; h < VEC / 4; ++h) {
      const f32x4 q = reinterpret_cast<const f32x4 *>(p)[h];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * h + e] = q[e];
    }
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_f32(T *p, const float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    if constexpr (sizeof(T) == 2) *p = f32_to_bf16(v[0]);
    else *p = v[0];
  } else if constexpr (sizeof(T) == 2) {
    u32x4 q;
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = cvt_pk_bf16(v[2 * e], v[2 * e + 1]);
    __builtin_nontemporal_store(q, reinterpret_cast<u32x4 *>(p));
  } else {
#pragma unroll
    for (int h = 0; h < VEC / 4; ++h)
      __builtin_nontemporal_store(f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]}, reinterpret_cast<f32x4 *>(p) + h);
  }
}

// One thread: VEC columns of one token, its k rows in the order of j.
template <typename T, typename O, int VEC>
__global__ void __launch_bounds__(256) combine_kernel(CombineArgs a, int64_t items, int per_row) {
  for (int64_t it = (int64_t)blockIdx.x * 256 + threadIdx.x; it < items; it += (int64_t)gridDim.x * 256) {
    const int t = (int)(it / per_row), c = (int)(it - (int64_t)t * per_row) * VEC;
    float sum[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum[e] = 0.f;
    for (int j = 0; j < a.k; ++j) {
      const int s = a.slots[(int64_t)t * a.k + j];
      if (s < 0 || s >= a.n_rows) continue;
      const float g = a.gates ? a.gates[(int64_t)t * a.k + j] : 1.f;
      float v[VEC];
      load_f32<T, VEC>(reinterpret_cast<const T *>(a.ys) + (int64_t)s * a.ldys + c, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] = fmaf(g, v[e], sum[e]);
    }
    store_f32<O, VEC>(reinterpret_cast<O *>(a.y) + (int64_t)t * a.ldy + c, sum);
  }
}

// One wave per token.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) combine_bwd_kernel(CombineArgs a) {
  const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= a.T) return;
  const T *dy = reinterpret_cast<const T *>(a.dy) + (int64_t)t * a.lddy;
  for (int j = 0; j < a.k; ++j) {
    const int64_t at = (int64_t)t * a.k + j;
    const int s = a.slots[at];
    float dot = 0.f;
    if (s >= 0 && s < a.n_rows) {
      const float g = a.gates[at];
      const T *ys = reinterpret_cast<const T *>(a.ys) + (int64_t)s * a.ldys;
      T *dys = reinterpret_cast<T *>(a.dys) + (int64_t)s * a.lddys;
      for (int c = lane * VEC; c < a.d; c += 64 * VEC) {
        float v[VEC], u[VEC];
        load_f32<T, VEC>(dy + c, v);
        if (a.dgates) {
          load_f32<T, VEC>(ys + c, u);
#pragma unroll
          for (int e = 0; e < VEC; ++e) dot = fmaf(v[e], u[e], dot);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[e] = g * v[e];
        store_f32<T, VEC>(dys + c, u);
      }
    }
    if (a.dgates) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o, 64);
      if (lane == 0) a.dgates[at] = dot;
    }
  }
}

bool al16(const void *p, int64_t ld, size_t es) { return (uintptr_t)p % 16 == 0 && ld * es % 16 == 0; }

}  // namespace

int run_combine(int dtype, int T, int k, int d, int n_rows, const void *ys, int64_t ldys, const int32_t *slots,
                const float *gates, void *y, int64_t ldy, int y_dtype, hipStream_t s) {
  CombineArgs a{};
  a.T = T; a.k = k; a.d = d; a.n_rows = n_rows;
  a.ys = ys; a.ldys = ldys; a.slots = slots; a.gates = gates; a.y = y; a.ldy = ldy;
  const size_t es = dtype == IMBD_BF16 ? 2 : 4, os = y_dtype == IMBD_BF16 ? 2 : 4;
  const bool vec = d % 8 == 0 && al16(ys, ldys, es) && al16(y, ldy, os);
  const int per_row = vec ? d / 8 : d;
  const int64_t items = (int64_t)T * per_row;
  const int64_t want = (items + 255) / 256;
  const dim3 grid((unsigned)(want < (1 << 20) ? want : (1 << 20))), wg(256);
  {
    LaunchTimer t(IMBD_K_COMBINE, 0, s);
#define GO(T_, O_)                                                                                   \
  do {                                                                                               \
    if (vec) hipLaunchKernelGGL((combine_kernel<T_, O_, 8>), grid, wg, 0, s, a, items, per_row);       \
    else hipLaunchKernelGGL((combine_kernel<T_, O_, 1>), grid, wg, 0, s, a, items, per_row);           \
  } while (0)
    if (dtype == IMBD_BF16 && y_dtype == IMBD_BF16) GO(uint16_t, uint16_t);
    else if (dtype == IMBD_BF16) GO(uint16_t, float);
    else if (y_dtype == IMBD_BF16) GO(float, uint16_t);
    else GO(float, float);
#undef GO
  }
  return check_launch("expert_combine");
}

int run_combine_bwd(int dtype, int T, int k, int d, int n_rows, const void *dy, int64_t lddy, const void *ys,
                    int64_t ldys, const int32_t *slots, const float *gates, void *dys, int64_t lddys, float *dgates,
                    hipStream_t s) {
  CombineArgs a{};
  a.T = T; a.k = k; a.d = d; a.n_rows = n_rows;
  a.ys = ys; a.ldys = ldys; a.slots = slots; a.gates = gates;
  a.dy = dy; a.lddy = lddy; a.dys = dys; a.lddys = lddys; a.dgates = dgates;
  const size_t es = dtype == IMBD_BF16 ? 2 : 4;
  const bool vec = d % 8 == 0 && al16(dy, lddy, es) && al16(dys, lddys, es) && (!dgates || al16(ys, ldys, es));
  const int64_t blocks = ((int64_t)T + 3) / 4;
  if (blocks > WORKGROUPS_MOST) {
    set_error("expert_combine_bwd: T = %d tokens are more than one launch takes", T);
    return IMBD_EUNSUPPORTED;
  }
  const dim3 grid((unsigned)blocks), wg(256);
  {
    LaunchTimer t(IMBD_K_COMBINE, 1, s);
    if (dtype == IMBD_BF16) {
      if (vec) hipLaunchKernelGGL((combine_bwd_kernel<uint16_t, 8>), grid, wg, 0, s, a);
      else hipLaunchKernelGGL((combine_bwd_kernel<uint16_t, 1>), grid, wg, 0, s, a);
    } else {
      if (vec) hipLaunchKernelGGL((combine_bwd_kernel<float, 8>), grid, wg, 0, s, a);
      else hipLaunchKernelGGL((combine_bwd_kernel<float, 1>), grid, wg, 0, s, a);
    }
  }
  return check_launch("expert_combine_bwd");
}

}  // namespace imbd
