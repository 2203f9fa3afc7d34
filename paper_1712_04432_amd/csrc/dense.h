// A fully connected layer's products with activation and residual (csrc/linear.hip) on the kernels of the expert layer: one
// expert that owns all rows. What those kernels take beside ExpertArgs, and the epilogue.
#pragma once

#include <type_traits>

#include "act.h"
#include "expert.h"

namespace imbd {

// E: ranges of `chunk` of the product's K, each a launch's own tiles. One range: the kernel finishes its outputs,
//   forward  z = sum + bias (stored where z is set), out = act(z) + residual
//   Delta_X  out = sum * act'(z) + residual
// More: it writes fp32 sums to out + e * so (ldo apart), which linear_reduce adds up in their order and finishes.
// w, x and dy are never split by expert (sw = 0), z is of the operands' type, the residual of the output's.
struct DenseArgs : ExpertArgs {
  int chunk;
  int act;
  void *z;
  int64_t ldz;
  const void *res;
  int64_t ldr;
  int width;  // operands padded to whole chunks (linear.hip): the outputs' own width
};

// N consecutive elements from p on, n of them real.
template <typename T, int N>
__device__ __forceinline__ void load_run(const T *p, int n, float (&v)[N]) {
  if (n >= N) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const f32x4 q = *reinterpret_cast<const f32x4_any *>(p + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i + j] = q[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const u32x2 q = *reinterpret_cast<const u32x2_any *>(p + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = q[j >> 1];
          v[i + j] = __builtin_bit_cast(float, j & 1 ? w & 0xffff0000u : w << 16);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.f;
      if (i < n) {
        if constexpr (sizeof(T) == 4) v[i] = p[i];
        else v[i] = bf16_to_f32(p[i]);
      }
    }
  }
}
template <typename T, int N>
__device__ __forceinline__ void store_run(T *p, int n, const float (&v)[N]) {
  if (n >= N) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4_any *>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
    } else if constexpr (N % 8 == 0) {
#pragma unroll
      for (int i = 0; i < N; i += 8)
        *reinterpret_cast<u32x4_any *>(p + i) = u32x4{cvt_pk_bf16(v[i], v[i + 1]), cvt_pk_bf16(v[i + 2], v[i + 3]),
                                                      cvt_pk_bf16(v[i + 4], v[i + 5]), cvt_pk_bf16(v[i + 6], v[i + 7])};
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 4)
        *reinterpret_cast<u32x2_any *>(p + i) = u32x2{cvt_pk_bf16(v[i], v[i + 1]), cvt_pk_bf16(v[i + 2], v[i + 3])};
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) {
        if constexpr (sizeof(T) == 4) p[i] = v[i];
        else p[i] = f32_to_bf16(v[i]);
      }
  }
}

// Outputs (m .. m + N - 1, n) from their sums (with the bias), cnt of them real. T: the operands' type.
template <typename T, int PASS, int N>
__device__ __forceinline__ void dense_finish(const DenseArgs &a, int n, int m, int cnt, float (&v)[N]) {
  if constexpr (PASS == EXPERT_FWD) {
    if (a.z) store_run(reinterpret_cast<T *>(a.z) + (int64_t)n * a.ldz + m, cnt, v);
    apply_act(a.act, v);
  }
  if constexpr (PASS == EXPERT_DX) {
    if (a.act != IMBD_ACT_NONE) {
      float z[N];
      load_run(reinterpret_cast<const T *>(a.z) + (int64_t)n * a.ldz + m, cnt, z);
      apply_slope(a.act, v, z);
    }
  }
  const int64_t at = (int64_t)n * a.ldo + m, rat = (int64_t)n * a.ldr + m;
  if (a.out_dtype == IMBD_BF16) {
    if (a.res) {
      float r[N];
      load_run(reinterpret_cast<const uint16_t *>(a.res) + rat, cnt, r);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += r[i];
    }
    store_run(reinterpret_cast<uint16_t *>(a.out) + at, cnt, v);
  } else {
    if (a.res) {
      float r[N];
      load_run(reinterpret_cast<const float *>(a.res) + rat, cnt, r);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += r[i];
    }
    store_run(reinterpret_cast<float *>(a.out) + at, cnt, v);
  }
}

// The products' launches (one range of K or several). check: as for the expert layer's.
// Any sizes, strides and alignments (csrc/expert_tile.hip).
int run_dense_tile(int pass, int dtype, const DenseArgs &a, bool check, hipStream_t s);
// ... and Delta_X and Delta_W in one launch, where both take the small tiles
bool dense_pair_fits(int dtype, const DenseArgs &dx, const DenseArgs &dw);
int run_dense_pair(int dtype, const DenseArgs &dx, const DenseArgs &dw, hipStream_t s);
// bf16, rows of whole 16-byte chunks (csrc/linear_wide.hip): whether it takes the call, the plan of M x N outputs (rows
// of a tile, ranges of K and their length, cycles), and the launch.
struct DensePlan {
  int bn, ranges, chunk;
  double cost;
};
bool dense_wide_fits(int pass, int dtype, const DenseArgs &a);
DensePlan dense_wide_plan(int pass, int64_t M, int64_t N, int64_t K);
int run_dense_wide(int pass, const DenseArgs &a, int bn, bool check, hipStream_t s);
// ... of operands that are padded to whole chunks, outputs of any width and alignment (forward and Delta_X, one range)
int run_dense_wide_any(int pass, const DenseArgs &a, int bn, bool check, hipStream_t s);

// Sums of ranges of K that a launch left: range s of output (n, m) at p + s*stride + (m / 64)*tile + n*ld + m % 64.
// Delta_W's bias sums: range s of db[o] at db + s*db_ld + o.
struct DensePartials {
  const float *p;
  int64_t ld, tile, stride;
  int ranges;
  const float *db;
  int db_ld;
};
// Forward and Delta_X of up to 256 rows (csrc/skinny.hip): whether it takes the call, the workspace that M x N outputs need,
// and the launch, which finishes the outputs (out->ranges == 1) or leaves its sums in ws.
bool skinny_dense_fits(int pass, const DenseArgs &a);
size_t skinny_dense_ws_bytes(int pass, int M, int N, int K);
int run_skinny_dense(int pass, const DenseArgs &a, void *ws, hipStream_t s, DensePartials *out);
// The forward product of up to 32 rows (csrc/linear_rows.hip), for what dense_wide_fits takes, and in fp32 for what this does.
bool linear_rows_f32_fits(const DenseArgs &a);
int run_linear_rows(int dtype, const DenseArgs &a, hipStream_t s);

// C entry points' launches (csrc/linear.hip).
struct LinearArgs {
  int dtype, d_out, d_in, B;
  const void *w;
  int64_t ldw;
  const float *bias;
  const void *x, *dy;
  int64_t ldx, lddy;
  int act;
  void *z;
  int64_t ldz;
  const void *res;
  int64_t ldr;
  void *out;  // y / dx
  int64_t ldo;
  int out_dtype;
  float *dw, *db;
  int64_t lddw;
};
size_t linear_ws_bytes(int which, int dtype, int d_out, int d_in, int B);
int run_linear_fwd(const LinearArgs &a, void *ws, hipStream_t s);
int run_linear_bwd(const LinearArgs &a, void *ws, hipStream_t s);
int run_act_bwd(int dtype, int act, int B, int d, const void *dy, int64_t lddy, const void *z, int64_t ldz, void *dz,
                int64_t lddz, hipStream_t s);

}  // namespace imbd
