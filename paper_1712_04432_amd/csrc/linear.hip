// A fully connected layer with activation and residual, forward and backward:
//   forward  z = W x + b, y = act(z) + r
//   Delta_X  dx = (W^T dy) * act'(z below) + dr;   Delta_W = dy^T x, db = sum dy
// The products run on the kernels of the expert layer (one expert that owns all rows; csrc/expert_tile.hip and
// csrc/linear_wide.hip), on that of small batches (csrc/skinny.hip) and on one for few rows (csrc/linear_rows.hip), which all finish
// their outputs themselves where K is whole (dense_finish, in csrc/dense.h). Where their tiles are too few to fill the GPU, K
// is cut into ranges: each writes its fp32 sums to the workspace, and linear_reduce adds them in their order and finishes the
// outputs the same way. The backward products of small layers share one launch (paired).

#include "dense.h"

namespace imbd {
namespace {

// RN outputs of one row a thread; Delta_W's bias sums in the row after the last. (bf16 outputs: 4 ranges of 64 x 4096 3.8 us, 3 of 512
// x 4096 6.5, 4.5 TB/s of what the product has just left in the caches.)
constexpr int RN = 4;
template <typename T, int PASS>
__device__ __forceinline__ void linear_reduce(const DenseArgs &a, const DensePartials &q, int M, int N, int per_row, unsigned block) {
  const unsigned i = block * 256u + threadIdx.x;
  const int n = (int)(i / (unsigned)per_row), m = RN * (int)(i - (unsigned)n * (unsigned)per_row);
  float v[RN] = {};
  if (n >= N) {
    const int o = (int)(i - (unsigned)N * (unsigned)per_row);
    if (PASS != EXPERT_DW || !a.db || o >= a.d_out) return;
    float s = 0.f;
    for (int e = 0; e < q.ranges; ++e) s += q.db[(int64_t)e * q.db_ld + o];
    a.db[o] = s;
    return;
  }
  const int cnt = min(RN, M - m);
  const float *p = q.p + (int64_t)(m >> 6) * q.tile + (int64_t)n * q.ld + (m & 63);  // (whole fours: what is past M is not used)
#pragma unroll 8
  for (int e = 0; e < q.ranges; ++e) {
    const f32x4 x = *reinterpret_cast<const f32x4 *>(p + e * q.stride);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += x[j];
  }
  if constexpr (PASS == EXPERT_FWD) {
    if (a.bias) {
      float bias[RN];
      load_run(a.bias + m, cnt, bias);
#pragma unroll
      for (int j = 0; j < RN; ++j) v[j] += bias[j];
    }
  }
  if constexpr (PASS == EXPERT_DW) {
    if (a.out) store_run(reinterpret_cast<float *>(a.out) + (int64_t)n * a.ldo + m, cnt, v);
  } else {
    dense_finish<T, PASS>(a, n, m, cnt, v);
  }
}

template <typename T, int PASS>
__global__ void __launch_bounds__(256) linear_reduce_kernel(DenseArgs a, DensePartials q, int M, int N, int per_row) {
  linear_reduce<T, PASS>(a, q, M, N, per_row, blockIdx.x);
}
// Delta_X's and Delta_W's in one launch: the first `blocks` workgroups Delta_X's.
struct ReducePair {
  DenseArgs x, w;
  DensePartials qx, qw;
  int M, Nx, Nw, per_row;
  unsigned blocks;
};
template <typename T>
__global__ void __launch_bounds__(256) linear_reduce_pair_kernel(ReducePair p) {
  if (blockIdx.x < p.blocks) linear_reduce<T, EXPERT_DX>(p.x, p.qx, p.M, p.Nx, p.per_row, blockIdx.x);
  else linear_reduce<T, EXPERT_DW>(p.w, p.qw, p.M, p.Nw, p.per_row, blockIdx.x - p.blocks);
}

// Three tensors once. bf16, 8192 x 16384: silu 139 us (5.8 TB/s), bound by memory; gelu, with more arithmetic an element, 189; 64 x
// 4096 3.2 us.
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

// dst[r][c] (ld columns, a multiple of 8) = src[r][c], zeros past its rows and columns.
__global__ void __launch_bounds__(256) pad_kernel(const uint16_t *src, int64_t ld_src, int rows, int cols, uint16_t *dst, int ld,
                                                  int64_t items) {
  const int per_row = ld / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per_row;
    const int c = 8 * (int)(i - r * per_row), n = r < rows ? cols - c : 0;
    const uint16_t *p = src + r * ld_src + c;
    u32x4 v{};
    if (n >= 8) v = *reinterpret_cast<const u32x4_any *>(p);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) v[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
    *reinterpret_cast<u32x4 *>(dst + i * 8) = v;
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
  if (n > K / (10 * step)) n = K / (10 * step);
  if (n < 1) n = 1;
  const int64_t chunk = ceil_div(ceil_div(K, n), step) * step;
  return Ranges{(int)(K > 0 ? ceil_div(K, chunk) : 1), (int)(K > 0 ? chunk : step)};
}

size_t range_bytes(const Ranges &r, int64_t M, int64_t N, bool db) {
  return r.n <= 1 ? 0 : (size_t)r.n * (size_t)(N * partial_ld8((int)M) + (db ? N : 0)) * 4;
}

// Which kernel takes a product of M x N outputs over K (rows of x and dy: N, for Delta_W K) that may have any of them (bf16,
// rows of whole chunks). us, weights from memory.
//  ROWS    forward of up to 16 rows (4096 x 4096, 1 / 16 rows: 9.8 / 11.3; SKINNY 13.1 / 13.3) and up to 32 while K is short (1024 x
//          1024, 32 rows 5.4, SKINNY 6.7; 4096 x 4096 16.0 and 13.3), but for long K, which its workgroups walk alone (1000
//          outputs, 8 rows, K = 2048 / 4096 / 16384: ROWS 5.4 / 8.2 / 28.1, SKINNY 7.2 / 7.9 / 13.7; 2048 outputs, 4096 / 8192: 9.2 / 16.0
//          and 9.5 / 13.1; 4096 of 8192 18.0 and 20.9, 8192 of 8192 37.5 and 36.8). Up to 16 rows of weights past SKINNY's offsets (2^30
//          elements, 2.1 GB) go here at any K: 65536 outputs of 16384, 1 / 8 / 16 rows 411 / 433 / 474 (WIDE, 17 rows, 378), 16384 of
//          65536 357 / 360 / 430 (401), 4096 of 262144 394 / 428 / 497 (398); few outputs of very long K are slower here than they would
//          be in WIDE's ranges (1024 of 1048576 1528 / 2062 / 3130, and 591)
//  SKINNY  forward and Delta_X of up to 256 rows (4096 x 4096, 64 / 256 rows: forward 13.6 / 22.0, Delta_X 14.4 / 24.7; WIDE 20.6 / 30.7
//          and 17.9 / 28.0), but for long K of many outputs (4096 outputs of 16384: forward 45.0 / 58.2, WIDE 40.3 / 57.4; Delta_X 43.1 /
//          56.6 and 37.7 / 51.0; 1024 of 16384: 15.9 / 23.0, WIDE 25.1 / 31.5)
//  TILE    what is too little for the large tiles, whose start and end take 8 us (forward of 2048 x 2048, 512 / 2048 rows: TILE 22.4 /
//          36.1, WIDE 24.0 / 37.5; 1000 x 4096, 512 / 1024 rows 22.8 / 34.2 and 23.9 / 30.1. Delta_X, whose weights TILE transposes in
//          registers: 256 x 784, 1024 / 2048 rows 8.4 / 14.4 and 8.9 / 9.2; 512 x 512, 300 rows 11.8 and 9.9. Delta_W of 1024 x 1024,
//          512 / 1024 rows 14.8 / 31.7 and 19.3 / 24.5; 2048 x 2048, 300 / 512 rows 17.4 / 22.8 and 19.8 / 22.6)
//  WIDE    the rest
enum Route { ROWS, SKINNY, TILE, WIDE, PADDED };
bool few_rows(int dtype, int64_t M, int64_t N, int64_t K) {
  // (fp32 beside TILE: 8 rows, 300 x 700 4.3 / 11.0, 1000 x 2048 8.9 / 12.6, 4096 x 2048 13.3 / 18.4, 2048 x 4096 23.5 / 18.6, 8192 x 4096 35.7 /
  // 51.8; 32 rows, 1000 x 1024 8.6 / 11.7, 4096 x 1024 10.2 / 15.5, 4096 x 2048 18.8 / 18.7, 16384 x 1000 26.1 / 24.5)
  if (dtype == IMBD_F32) return N <= 16 ? K <= 2048 || (K <= 4096 && M >= 8192) : N <= 32 && K <= 1024 && M <= 8192;
  return (N <= 16 || (N <= 32 && K <= 1024)) && (K <= 2048 || (K <= 4096 && K <= 2 * M));
}
Route route(int pass, int64_t M, int64_t N, int64_t K) {
  const double flops = 2.0 * M * N * K;
  if (pass == EXPERT_DW) return M * N <= (8 << 20) && (K <= 320 || flops < 1.1e9) ? TILE : WIDE;
  const bool near = M * K < (1 << 30) - (1 << 24);  // (SKINNY: 32-bit offsets into W)
  if (pass == EXPERT_FWD && (few_rows(IMBD_BF16, M, N, K) || (N <= 16 && !near))) return ROWS;
  if (N <= 256 && near && !(K > 12288 && M * K > (32 << 20))) return SKINNY;
  return flops < (pass == EXPERT_FWD ? 6e9 : 0.15e9) ? TILE : WIDE;
}

// Products of bf16 layers whose widths are no whole chunks, where it pays: on the large tiles all the same, from copies with
// the rows padded by zeros (K too, so that no other row's elements meet them). us, padded / TILE: forward of 4099 x 4097, 64 /
// 256 rows 37.6 / 24.3 and 45.6 / 59.1, 8192 rows 349 / 623; 2047 x 2049, 2048 / 8192 rows 58.0 / 46.7 and 94.7 / 157. Delta_X of
// 517 x 513, 1024 / 2048 rows 21.5 / 15.2 and 23.1 / 27.9; 4099 x 4097, 64 / 8192 rows 34.6 / 42.0 and 325 / 1037. Delta_W of 1023 x
// 1025, 512 / 1024 rows 30.1 / 27.4 and 33.4 / 45.2; 4099 x 4097, 8192 rows 397 / 1329.
bool pads(int pass, int64_t M, int64_t N, int64_t K) {
  const double flops = 2.0 * M * N * K;
  if (M % 8 == 0 && (pass == EXPERT_DW ? N : K) % 8 == 0) return false;
  if (pass == EXPERT_DW) return K >= 1024 && flops >= 2e9 && M * N < ((int64_t)1 << 32);  // (linear_reduce's 32-bit items)
  return flops >= (pass == EXPERT_DX ? 1e9 : K >= 4096 ? 6e9 : 2e10);
}
int64_t pad8(int64_t n) { return ceil_div(n, 8) * 8; }
size_t pad_bytes(int64_t rows, int64_t cols) { return (size_t)(rows * pad8(cols) * 2 + 255) / 256 * 256; }
bool whole_chunks(const void *p, int64_t ld, int cols) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && cols % 8 == 0 && ld < (1 << 22); }

// The matrix itself, or its padded copy at *at, which moves on.
const void *padded(const void *src, int64_t *ld, int rows, int cols, int rows_out, char **at, bool check, hipStream_t s) {
  if (rows == rows_out && whole_chunks(src, *ld, cols)) return src;
  uint16_t *dst = reinterpret_cast<uint16_t *>(*at);
  const int64_t items = rows_out * (pad8(cols) / 8), blocks = ceil_div(items, 256);
  if (!check) {
    LaunchTimer t(IMBD_K_LINEAR, 5, s);
    hipLaunchKernelGGL(pad_kernel, dim3((unsigned)(blocks < (1 << 16) ? blocks : 1 << 16)), dim3(256), 0, s,
                       static_cast<const uint16_t *>(src), *ld, rows, cols, dst, (int)pad8(cols), items);
  }
  *at += pad_bytes(rows_out, cols);
  *ld = pad8(cols);
  return dst;
}

// The workspace of a product, whichever kernel its tensors' alignment leaves.
size_t product_bytes(int pass, int dtype, int64_t M, int64_t N, int64_t K) {
  const bool db = pass == EXPERT_DW;
  const size_t n = range_bytes(tile_ranges(dtype, M, N, K), M, N, db);
  if (dtype != IMBD_BF16 || M == 0 || N == 0 || K == 0) return n;
  size_t k = 0;
  if (pads(pass, M, N, K)) {
    if (pass == EXPERT_DW) {
      const DensePlan p = dense_wide_plan(pass, pad8(M), pad8(N), K);
      k = pad_bytes(K, M) + pad_bytes(K, N) + (size_t)p.ranges * (size_t)(pad8(N) * pad8(M) + pad8(N)) * 4;
    } else {
      const DensePlan p = dense_wide_plan(pass, pad8(M), N, pad8(K));
      k = pad_bytes(pad8(pass == EXPERT_FWD ? M : K), pass == EXPERT_FWD ? K : M) + pad_bytes(N, K);
      if (p.ranges > 1) k += (size_t)p.ranges * (size_t)(N * pad8(M)) * 4;
    }
  }
  const size_t padding = k > n ? k : n;
  k = 0;
  switch (route(pass, M, N, K)) {
    case SKINNY: k = skinny_dense_ws_bytes(pass, (int)M, (int)N, (int)K); break;
    case WIDE: {
      const DensePlan p = dense_wide_plan(pass, M, N, K);
      k = range_bytes(Ranges{p.ranges, p.chunk}, M, N, db);
      break;
    }
    default: break;
  }
  return k > padding ? k : padding;
}

int reduce(int pass, int dtype, const DenseArgs &a, const DensePartials &q, hipStream_t s) {
  const int M = pass == EXPERT_FWD ? a.d_out : a.d_in, N = pass == EXPERT_DW ? (a.out ? a.d_out : 0) : a.n_rows;
  const int per_row = (int)ceil_div(M, RN);
  const dim3 grid((unsigned)ceil_div((int64_t)N * per_row + (a.db ? a.d_out : 0), 256)), wg(256);
  {
    LaunchTimer t(IMBD_K_LINEAR, 3, s);
#define GO(T)                                                                                                                 \
  do {                                                                                                                        \
    if (pass == EXPERT_FWD) hipLaunchKernelGGL((linear_reduce_kernel<T, EXPERT_FWD>), grid, wg, 0, s, a, q, M, N, per_row); \
    else if (pass == EXPERT_DX) hipLaunchKernelGGL((linear_reduce_kernel<T, EXPERT_DX>), grid, wg, 0, s, a, q, M, N, per_row); \
    else hipLaunchKernelGGL((linear_reduce_kernel<T, EXPERT_DW>), grid, wg, 0, s, a, q, M, N, per_row);                   \
  } while (0)
    if (dtype == IMBD_BF16) GO(uint16_t);
    else GO(float);
#undef GO
  }
  return check_launch("linear_reduce");
}

int padded_product(int pass, const DenseArgs &a, void *ws, bool check, hipStream_t s) {
  char *at = static_cast<char *>(ws);
  DenseArgs b = a;
  b.E = 1;
  if (pass == EXPERT_DW) {
    if (a.out) b.x = padded(a.x, &b.ldx, a.n_rows, a.d_in, a.n_rows, &at, check, s);
    b.dy = padded(a.dy, &b.lddy, a.n_rows, a.d_out, a.n_rows, &at, check, s);
    b.d_in = (int)pad8(a.d_in);
    b.d_out = (int)pad8(a.d_out);
    const DensePlan p = dense_wide_plan(pass, b.d_in, b.d_out, a.n_rows);
    b.E = p.ranges;
    b.chunk = p.chunk;
    float *sums = reinterpret_cast<float *>(at);
    const int64_t stride = (int64_t)b.d_out * b.d_in;
    const DensePartials q{sums, b.d_in, 64, stride, p.ranges, sums + p.ranges * stride, b.d_out};
    b.out = a.out ? sums : nullptr;
    b.ldo = b.d_in;
    b.so = stride;
    if (a.db) b.db = sums + p.ranges * stride;
    const int rc = run_dense_wide(pass, b, p.bn, check, s);
    return rc != IMBD_OK || check ? rc : reduce(pass, IMBD_BF16, a, q, s);
  }
  const int M = pass == EXPERT_FWD ? a.d_out : a.d_in, K = pass == EXPERT_FWD ? a.d_in : a.d_out;
  const DensePlan p = dense_wide_plan(pass, pad8(M), a.n_rows, pad8(K));
  b.width = M;
  if (pass == EXPERT_FWD) {  // (sums are stored in whole chunks: then W has rows for them too)
    if (p.ranges > 1) b.d_out = (int)pad8(a.d_out);
    b.w = padded(a.w, &b.ldw, a.d_out, a.d_in, b.d_out, &at, check, s);
    b.x = padded(a.x, &b.ldx, a.n_rows, a.d_in, a.n_rows, &at, check, s);
    b.d_in = (int)pad8(a.d_in);
  } else {
    b.d_out = (int)pad8(a.d_out);
    b.w = padded(a.w, &b.ldw, a.d_out, a.d_in, b.d_out, &at, check, s);
    b.dy = padded(a.dy, &b.lddy, a.n_rows, a.d_out, a.n_rows, &at, check, s);
    b.d_in = (int)pad8(a.d_in);
  }
  b.E = p.ranges;
  b.chunk = p.chunk;
  if (p.ranges == 1) return run_dense_wide_any(pass, b, p.bn, check, s);
  const DensePartials q{reinterpret_cast<float *>(at), pad8(M), 64, (int64_t)a.n_rows * pad8(M), p.ranges, nullptr, 0};
  b.out = at;
  b.ldo = q.ld;
  b.so = q.stride;
  b.out_dtype = IMBD_F32;
  b.bias = nullptr;
  const int rc = run_dense_wide(pass, b, p.bn, check, s);
  return rc != IMBD_OK || check ? rc : reduce(pass, IMBD_BF16, a, q, s);
}

// Which kernel takes the product as its tensors lie.
Route product_route(int pass, int dtype, const DenseArgs &a) {
  const int M = pass == EXPERT_FWD ? a.d_out : a.d_in, N = pass == EXPERT_DW ? a.d_out : a.n_rows;
  const int K = pass == EXPERT_FWD ? a.d_in : pass == EXPERT_DX ? a.d_out : a.n_rows;
  if (dtype == IMBD_F32) return pass == EXPERT_FWD && few_rows(IMBD_F32, M, N, K) && linear_rows_f32_fits(a) ? ROWS : TILE;
  const bool fits = dense_wide_fits(pass, dtype, a);
  if (!fits && pads(pass, M, N, K) && a.n_rows < (1 << 29) && M < (1 << 22) && (pass == EXPERT_DW ? N : K) < (1 << 22))
    return PADDED;
  const Route to = fits ? route(pass, M, N, K) : TILE;
  return to == SKINNY && !skinny_dense_fits(pass, a) ? TILE : to;  // (past its 32-bit offsets)
}

// A product's arguments with its K in ranges, and where they leave their sums: from `ws` on.
DensePartials in_ranges(int pass, const Ranges &r, DenseArgs &a, void *ws) {
  const int M = pass == EXPERT_FWD ? a.d_out : a.d_in, N = pass == EXPERT_DW ? a.d_out : a.n_rows;
  a.E = r.n;
  a.chunk = r.chunk;
  if (r.n == 1) return DensePartials{};
  const int64_t stride = (int64_t)N * partial_ld8(M);
  float *db = reinterpret_cast<float *>(ws) + r.n * stride;
  const DensePartials q{reinterpret_cast<float *>(ws), partial_ld8(M), 64, stride, r.n, db, a.d_out};
  a.out = pass == EXPERT_DW && !a.out ? nullptr : ws;
  a.ldo = q.ld;
  a.so = q.stride;
  a.out_dtype = IMBD_F32;
  a.bias = nullptr;
  if (a.db) a.db = db;
  return q;
}

int product(int pass, int dtype, DenseArgs a, void *ws, bool check, hipStream_t s) {
  const int M = pass == EXPERT_FWD ? a.d_out : a.d_in, N = pass == EXPERT_DW ? a.d_out : a.n_rows;
  const int K = pass == EXPERT_FWD ? a.d_in : pass == EXPERT_DX ? a.d_out : a.n_rows;
  const Route to = product_route(pass, dtype, a);
  if (to == PADDED) return padded_product(pass, a, ws, check, s);
  a.E = 1;
  a.chunk = (K + 63) / 64 * 64;
  if (to == ROWS) return check ? IMBD_OK : run_linear_rows(dtype, a, s);
  if (to == SKINNY) {
    if (check) return IMBD_OK;
    DensePartials q;
    const int rc = run_skinny_dense(pass, a, ws, s, &q);
    return rc != IMBD_OK || q.ranges == 1 ? rc : reduce(pass, dtype, a, q, s);
  }
  const bool wide = to == WIDE;
  const DensePlan plan = wide ? dense_wide_plan(pass, M, N, K) : DensePlan{};
  const Ranges r = wide ? Ranges{plan.ranges, plan.chunk} : tile_ranges(dtype, M, N, K);
  DenseArgs part = a;
  const DensePartials q = in_ranges(pass, r, part, ws);
  const int rc = wide ? run_dense_wide(pass, part, plan.bn, check, s) : run_dense_tile(pass, dtype, part, check, s);
  return rc != IMBD_OK || check || r.n == 1 ? rc : reduce(pass, dtype, a, q, s);
}

// Delta_X and Delta_W of a layer on the any-size kernel's small tiles in one launch, and their sums in one: starts and ends
// overlap, and a second launch's are saved. Both are cut into ranges of L steps at most: 6 while they are too few to fill the
// GPU's 1024 places (bf16, whose transposes take more registers: 512), 12 where they do (what is left of long ranges at
// the end leaves CUs idle). us, in one / by themselves: rows x d_in to d_out in fp32 64 x 784 to 256 10.6 / 15.8, 300 x 512 to 512
// 14.8 / 31.5, 1000 x 1023 to 517 49 / 55, 2048 x 1024 to 1024 122 / 161; bf16 300 x 517 to 513 15.0 / 24.4, 200 x 255 to 1001 15.3 / 30.9.
// bf16 that has a faster kernel for one of them alone, too: 512 x 512 to 512 14.3 / 30.2, 1024 x 512 to 512 17.2 / 39.8, 1000
// x 1024 to 512 30.8 / 42.6 (1536 x 784 to 512 47.2 / 40.7, so up to 1.15 GFLOP a product); padded copies, 1000 x 1023 to 517 45.6 /
// 69.6, 2048 x 1023 to 517 68.9 / 77.6 (600 x 2001 to 1001 76.1 / 76.0, so up to 2.4). Not up to 256 rows on the small batches'
// kernel: 64 x 512 to 512 12.1 / 9.7, 256 x 1024 to 1024 18.5 / 15.7.
struct PairPlan {
  Ranges dx, dw;
  size_t dx_bytes, bytes;
};
PairPlan pair_plan(int dtype, int64_t d_out, int64_t d_in, int64_t B) {
  const int64_t step = dtype == IMBD_BF16 ? 64 : 32;
  const int64_t x_tiles = ceil_div(d_in, 64) * ceil_div(B, 32), w_tiles = ceil_div(d_in, 64) * ceil_div(d_out, 32);
  const int64_t x_steps = ceil_div(d_out, step), w_steps = ceil_div(B, step);
  const double each = ((double)x_tiles * x_steps + (double)w_tiles * w_steps) / (dtype == IMBD_BF16 ? 512 : 1024);
  const int64_t L = each <= 6 ? 6 : each >= 12 ? 12 : (int64_t)each;
  auto cut = [&](int64_t tiles, int64_t steps) {
    int64_t n = dtype == IMBD_BF16 && steps <= 8 ? 1 : ceil_div(steps, L);
    if (n > 1024 / tiles) n = 1024 / tiles;
    if (n < 1) n = 1;
    const int64_t len = ceil_div(steps, n);
    return Ranges{(int)ceil_div(steps, len), (int)(len * step)};
  };
  PairPlan p;
  p.dx = cut(x_tiles, x_steps);
  p.dw = cut(w_tiles, w_steps);
  p.dx_bytes = (range_bytes(p.dx, d_in, B, false) + 255) / 256 * 256;
  p.bytes = p.dx_bytes + range_bytes(p.dw, d_in, d_out, true);
  return p;
}

int reduce_pair(int dtype, const DenseArgs &x, const DenseArgs &w, const DensePartials &qx, const DensePartials &qw, hipStream_t s) {
  ReducePair p{x, w, qx, qw, x.d_in, x.n_rows, w.out ? w.d_out : 0, (int)ceil_div(x.d_in, RN), 0};
  p.blocks = (unsigned)ceil_div((int64_t)p.Nx * p.per_row, 256);
  const dim3 grid(p.blocks + (unsigned)ceil_div((int64_t)p.Nw * p.per_row + (w.db ? w.d_out : 0), 256)), wg(256);
  {
    LaunchTimer t(IMBD_K_LINEAR, 3, s);
    if (dtype == IMBD_BF16) hipLaunchKernelGGL(linear_reduce_pair_kernel<uint16_t>, grid, wg, 0, s, p);
    else hipLaunchKernelGGL(linear_reduce_pair_kernel<float>, grid, wg, 0, s, p);
  }
  return check_launch("linear_reduce");
}

// false: not one launch's. Else *rc is the call's result.
bool paired(int dtype, const DenseArgs &dx, const DenseArgs &dw, void *ws, hipStream_t s, int *rc) {
  const Route to_x = product_route(EXPERT_DX, dtype, dx), to_w = product_route(EXPERT_DW, dtype, dw);
  const double flops = 2.0 * dx.n_rows * dx.d_in * dx.d_out;
  if (to_x == SKINNY) return false;
  if ((to_x != TILE || to_w != TILE) && flops > (to_x == PADDED || to_w == PADDED ? 2.4e9 : 1.15e9)) return false;
  const PairPlan p = pair_plan(dtype, dx.d_out, dx.d_in, dx.n_rows);
  DenseArgs x = dx, w = dw;
  const DensePartials qx = in_ranges(EXPERT_DX, p.dx, x, ws), qw = in_ranges(EXPERT_DW, p.dw, w, static_cast<char *>(ws) + p.dx_bytes);
  if (!dense_pair_fits(dtype, x, w)) return false;
  *rc = run_dense_pair(dtype, x, w, s);
  if (*rc != IMBD_OK) return true;
  if (p.dx.n > 1 && p.dw.n > 1) *rc = reduce_pair(dtype, dx, dw, qx, qw, s);
  else if (p.dx.n > 1) *rc = reduce(EXPERT_DX, dtype, dx, qx, s);
  else if (p.dw.n > 1) *rc = reduce(EXPERT_DW, dtype, dw, qw, s);
  return true;
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
  const size_t one = dx > dw ? dx : dw, two = B > 0 ? pair_plan(dtype, d_out, d_in, B).bytes : 0;
  return one > two ? one : two;
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
      int rc;
      if (paired(l.dtype, a, g, ws, s, &rc)) return rc;
      rc = product(EXPERT_DW, l.dtype, g, ws, true, s);
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
