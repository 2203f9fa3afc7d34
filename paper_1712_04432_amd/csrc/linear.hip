// A fully connected layer with activation and residual, forward and backward:
//   forward  z = W x + b, y = act(z) + r
//   Delta_X  dx = (W^T dy) * act'(z below) + dr;   Delta_W = dy^T x, db = sum dy
// The products run on the kernels of the expert layer (one expert that owns all rows), which finish their outputs
// themselves where K is whole. Where their tiles are too few to fill the GPU, K is cut into ranges: each writes its fp32 sums to the
// workspace, and linear_reduce adds them in their order and finishes the outputs the same way.

#include "dense.h"

namespace imbd {
namespace {

// Sums of ranges of K: range s of output (n, m) at p + s*stride + n*ld + m.
struct Partials {
  const float *p;
  int64_t ld, stride;
  int ranges;
};

// Eight outputs of one row a thread; Delta_W's bias sums in the row after the last.
template <typename T, int PASS>
__global__ void __launch_bounds__(256) linear_reduce_kernel(DenseArgs a, Partials q, const float *db, int M, int N, int per_row) {
  const unsigned i = blockIdx.x * 256u + threadIdx.x;
  const int n = (int)(i / (unsigned)per_row), m = 8 * (int)(i - (unsigned)n * (unsigned)per_row);
  float v[8] = {};
  if (n >= N) {
    const int o = (int)(i - (unsigned)N * (unsigned)per_row);
    if (PASS != EXPERT_DW || !a.db || o >= a.d_out) return;
    float s = 0.f;
    for (int e = 0; e < q.ranges; ++e) s += db[(int64_t)e * a.d_out + o];
    a.db[o] = s;
    return;
  }
  const int cnt = min(8, M - m);
  const float *p = q.p + (int64_t)n * q.ld + m;  // (rows of whole eights: what is past M is not used)
#pragma unroll 4
  for (int e = 0; e < q.ranges; ++e) {
    const f32x4 x = *reinterpret_cast<const f32x4 *>(p + e * q.stride), y = *reinterpret_cast<const f32x4 *>(p + e * q.stride + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += x[j], v[4 + j] += y[j];
  }
  if constexpr (PASS == EXPERT_FWD) {
    if (a.bias) {
      float bias[8];
      load_run(a.bias + m, cnt, bias);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += bias[j];
    }
  }
  if constexpr (PASS == EXPERT_DW) {
    if (a.out) store_run(reinterpret_cast<float *>(a.out) + (int64_t)n * a.ldo + m, cnt, v);
  } else {
    dense_finish<T, PASS>(a, n, m, cnt, v);
  }
}

template <typename T>
__global__ void __launch_bounds__(256) act_bwd_kernel(int act, int B, int d, const T *dy, int64_t lddy, const T *z, int64_t ldz,
                                                      T *dz, int64_t lddz, int64_t items, int per_row) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
    const int64_t b = i / per_row;
    const int m = 8 * (int)(i - b * per_row), cnt = min(8, d - m);
    float v[8], x[8];
    load_run(dy + b * lddy + m, cnt, v);
    load_run(z + b * ldz + m, cnt, x);
    apply_slope(act, v, x);
    store_run(dz + b * lddz + m, cnt, v);
  }
}

// ------------------------------------------------------------------------------ plans
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t partial_ld8(int M) { return ceil_div(M, 8) * 8; }

// Ranges of K of a product of M x N outputs on the any-size kernel's tiles, and their length.
struct Ranges {
  int n, chunk;
};
Ranges tile_ranges(int dtype, int64_t M, int64_t N, int64_t K) {
  const int64_t step = dtype == IMBD_BF16 ? 64 : 32;
  const int64_t tiles = ceil_div(M, 64) * ceil_div(N, 32);
  int64_t n = tiles > 0 ? 1024 / tiles : 1;
  if (n > K / (8 * step)) n = K / (8 * step);
  if (n < 1) n = 1;
  const int64_t chunk = ceil_div(ceil_div(K, n), step) * step;
  return Ranges{(int)(K > 0 ? ceil_div(K, chunk) : 1), (int)(K > 0 ? chunk : step)};
}

size_t range_bytes(const Ranges &r, int64_t M, int64_t N, bool db) {
  return r.n <= 1 ? 0 : (size_t)r.n * (size_t)(N * partial_ld8((int)M) + (db ? N : 0)) * 4;
}

// Whether the large tiles take a product that they can take: not while its rows are few (or, for Delta_W, its outputs).
bool wide_pays(int pass, int64_t M, int64_t N, int64_t K) { return pass == EXPERT_DW ? M >= 64 && N >= 64 : N > 64; }

size_t product_bytes(int pass, int dtype, int64_t M, int64_t N, int64_t K) {
  const bool db = pass == EXPERT_DW;
  size_t n = range_bytes(tile_ranges(dtype, M, N, K), M, N, db);
  if (dtype == IMBD_BF16 && wide_pays(pass, M, N, K)) {
    const DensePlan p = dense_wide_plan(pass, M, N, K);
    const size_t w = range_bytes(Ranges{p.ranges, p.chunk}, M, N, db);
    n = w > n ? w : n;
  }
  return n;
}

int product(int pass, int dtype, DenseArgs a, void *ws, bool check, hipStream_t s) {
  const int M = pass == EXPERT_FWD ? a.d_out : a.d_in, N = pass == EXPERT_DW ? a.d_out : a.n_rows;
  const int K = pass == EXPERT_FWD ? a.d_in : pass == EXPERT_DX ? a.d_out : a.n_rows;
  const bool wide = wide_pays(pass, M, N, K) && dense_wide_fits(pass, dtype, a);
  const DensePlan plan = wide ? dense_wide_plan(pass, M, N, K) : DensePlan{};
  const Ranges r = wide ? Ranges{plan.ranges, plan.chunk} : tile_ranges(dtype, M, N, K);
  auto run = [&](const DenseArgs &d) {
    return wide ? run_dense_wide(pass, d, plan.bn, check, s) : run_dense_tile(pass, dtype, d, check, s);
  };
  a.E = r.n;
  a.chunk = r.chunk;
  if (r.n == 1) return run(a);
  DenseArgs part = a;
  const Partials q{reinterpret_cast<float *>(ws), partial_ld8(M), (int64_t)N * partial_ld8(M), r.n};
  float *db = reinterpret_cast<float *>(ws) + r.n * q.stride;
  part.out = pass == EXPERT_DW && !a.out ? nullptr : ws;
  part.ldo = q.ld;
  part.so = q.stride;
  part.out_dtype = IMBD_F32;
  part.bias = nullptr;
  if (a.db) part.db = db;
  const int rc = run(part);
  if (rc != IMBD_OK || check) return rc;
  const int per_row = (int)(q.ld / 8);
  const int64_t rows = pass == EXPERT_DW && !a.out ? 0 : N, items = rows * per_row + (a.db ? a.d_out : 0);
  const dim3 grid((unsigned)ceil_div(items, 256)), wg(256);
  {
    LaunchTimer t(IMBD_K_LINEAR, 3, s);
#define GO(T)                                                                                                             \
  do {                                                                                                                    \
    if (pass == EXPERT_FWD) hipLaunchKernelGGL((linear_reduce_kernel<T, EXPERT_FWD>), grid, wg, 0, s, a, q, db, M, (int)rows, per_row); \
    else if (pass == EXPERT_DX) hipLaunchKernelGGL((linear_reduce_kernel<T, EXPERT_DX>), grid, wg, 0, s, a, q, db, M, (int)rows, per_row); \
    else hipLaunchKernelGGL((linear_reduce_kernel<T, EXPERT_DW>), grid, wg, 0, s, a, q, db, M, (int)rows, per_row);         \
  } while (0)
    if (dtype == IMBD_BF16) GO(uint16_t);
    else GO(float);
#undef GO
  }
  return check_launch("linear_reduce");
}

DenseArgs dense_args(const LinearArgs &l) {
  DenseArgs a{};
  a.d_out = l.d_out; a.d_in = l.d_in; a.n_rows = a.n_x = l.B;
  a.w = l.w; a.ldw = l.ldw;
  return a;
}

}  // namespace

size_t linear_ws_bytes(int which, int dtype, int d_out, int d_in, int B) {
  if (which == 0) return product_bytes(EXPERT_FWD, dtype, d_out, B, d_in);
  const size_t dx = product_bytes(EXPERT_DX, dtype, d_in, B, d_out), dw = product_bytes(EXPERT_DW, dtype, d_in, d_out, B);
  return dx > dw ? dx : dw;
}

int run_linear_fwd(const LinearArgs &l, void *ws, hipStream_t s) {
  DenseArgs a = dense_args(l);
  a.bias = l.bias;
  a.x = l.x; a.ldx = l.ldx;
  a.act = l.act;
  a.z = l.z; a.ldz = l.ldz;
  a.res = l.res; a.ldr = l.ldr;
  a.out = l.out; a.ldo = l.ldo; a.out_dtype = l.out_dtype;
  return product(EXPERT_FWD, l.dtype, a, ws, false, s);
}

int run_linear_bwd(const LinearArgs &l, void *ws, hipStream_t s) {
  DenseArgs g = dense_args(l);  // the weights' gradient
  g.dy = l.dy; g.lddy = l.lddy;
  g.x = l.dw ? l.x : nullptr; g.ldx = l.ldx;
  if (!l.dw) g.n_x = 0;  // (db alone: x is not read)
  g.out = l.dw; g.ldo = l.lddw; g.out_dtype = IMBD_F32;
  g.db = l.db;
  const bool grad = l.dw || l.db;
  if (l.out && l.B > 0) {
    DenseArgs a = dense_args(l);
    a.dy = l.dy; a.lddy = l.lddy;
    a.act = l.act;
    a.z = l.z; a.ldz = l.ldz;
    a.res = l.res; a.ldr = l.ldr;
    a.out = l.out; a.ldo = l.ldo; a.out_dtype = l.out_dtype;
    if (grad) {
      const int rc = product(EXPERT_DW, l.dtype, g, ws, true, s);
      if (rc != IMBD_OK) return rc;
    }
    const int rc = product(EXPERT_DX, l.dtype, a, ws, false, s);
    if (rc != IMBD_OK) return rc;
  }
  return grad ? product(EXPERT_DW, l.dtype, g, ws, false, s) : IMBD_OK;
}

int run_act_bwd(int dtype, int act, int B, int d, const void *dy, int64_t lddy, const void *z, int64_t ldz, void *dz,
                int64_t lddz, hipStream_t s) {
  const int per_row = (int)ceil_div(d, 8);
  const int64_t items = (int64_t)B * per_row, blocks = ceil_div(items, 256);
  if (items == 0) return IMBD_OK;
  const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20)), wg(256);
  {
    LaunchTimer t(IMBD_K_LINEAR, 4, s);
    if (dtype == IMBD_BF16)
      hipLaunchKernelGGL(act_bwd_kernel<uint16_t>, grid, wg, 0, s, act, B, d, static_cast<const uint16_t *>(dy), lddy,
                         static_cast<const uint16_t *>(z), ldz, static_cast<uint16_t *>(dz), lddz, items, per_row);
    else
      hipLaunchKernelGGL(act_bwd_kernel<float>, grid, wg, 0, s, act, B, d, static_cast<const float *>(dy), lddy,
                         static_cast<const float *>(z), ldz, static_cast<float *>(dz), lddz, items, per_row);
  }
  return check_launch("act_bwd");
}

}  // namespace imbd
