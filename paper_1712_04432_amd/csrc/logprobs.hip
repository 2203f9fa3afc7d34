// Log probabilities of given tokens, with the entropy and the top alternatives of every row, and their gradient.
//
// Forward. Bound by reading the logits, once: a workgroup walks a row, or a part of it (row_parts), with the sums of the
// softmax in registers (RowSums in csrc/vocab.h). A thread's reference m moves only when a group of its logits exceeds
// it by 16 octaves, so that the sums are rescaled a few times a row and not with every new maximum: fp32 holds 2^16
// times more than it needs to. Parts are joined in their order by a second launch.
//
// Alternatives cost the walk one comparison a chunk: every thread remembers its largest logit's chunk. The n-th largest
// of 64 disjoint groups' best is a bound that the row's n best reach; the threads whose best reaches it (hardly more than n)
// have their columns looked at once more, from the caches, and what reaches the bound there is put in order by counting.
// Where more than fit the list reach it (many equal columns of one thread), the n are found one after another.
//
// Measured, bf16: 2048 rows of 131072 with five alternatives 102 us (5.3 TB/s), 16 rows with twenty 7.3 + 4.8 us (their
// columns looked at again by a wave each, one after another, 12.6; parts joined by comparing all their lists, 28), forward
// and gradient of 8192 rows of 32768 311 us (5.2 TB/s).

#include "order_key.h"
#include "row_walk.h"
#include "vocab.h"

namespace imbd {
namespace {

constexpr int LP_NT = WALK_NT, LP_UNROLL = WALK_UNROLL;
constexpr int LP_LIST = 1024;  // candidates

struct LogprobsArgs {
  int V, n, parts, per;
  const void *logits;
  int64_t ldz;
  const int32_t *tokens;
  float inv_t, c;
  float *logp, *entropy, *lse;
  int32_t *top_ids;
  float *top_logp;
  RowSums *sums;   // more than one part: [b][part]
  uint64_t *keys;  // ... and the part's n best, in order, [b][part][n]
};

// A logit and its token as one number: larger logits first, then lower tokens. 0: none.
__device__ __forceinline__ uint64_t choice_key(float z, int v) {
  const uint32_t k = order_key(z);
  if (z != z || k <= KEY_MINUS_INF) return 0;
  return ((uint64_t)k << 32) | (uint32_t)~v;
}
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

// The n-th largest of the wave's keys (which differ, but for zeros), 1 where fewer are above 0.
__device__ __forceinline__ uint64_t nth_largest(uint64_t g, int n) {
  int rank = 0;
#pragma unroll
  for (int i = 0; i < 64; ++i) {
    const uint64_t k = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(g >> 32), i) << 32) |
                       (uint32_t)__builtin_amdgcn_readlane((int)g, i);
    rank += k > g;
  }
  const uint64_t at = __ballot(rank == n - 1 && g != 0);
  if (at == 0) return 1;
  const int src = __builtin_ctzll(at);
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(g >> 32), src) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)g, src);
}
// Puts the first n of `found` keys (all different) in order: put(place, key), key 0 past the last.
template <typename F>
__device__ __forceinline__ void put_in_order(const uint64_t *keys, int found, int n, F put) {
  for (int i = threadIdx.x; i < found; i += LP_NT) {
    const uint64_t key = keys[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < found; ++j) rank += keys[j] > key;
    if (rank < n) put(rank, key);
  }
  for (int j = found + threadIdx.x; j < n; j += LP_NT) put(j, 0);
}

// The row's results from its sums.
__device__ __forceinline__ void put_row(const LogprobsArgs &a, int64_t b, const RowSums &r, float zt, int t, float ls) {
  a.logp[b] = t < 0 ? 0.f : t >= a.V ? __builtin_nanf("") : (zt - r.m) * a.inv_t - ls;
  if (a.entropy) a.entropy[b] = ls - LN2 * (r.u / r.s);
  if (a.lse) a.lse[b] = r.m * a.inv_t + ls;
}
__device__ __forceinline__ void put_choice(const LogprobsArgs &a, int64_t b, int j, uint64_t key, const RowSums &r, float ls) {
  a.top_ids[b * a.n + j] = key ? (int)~(uint32_t)key : -1;
  a.top_logp[b * a.n + j] = key ? (key_value((uint32_t)(key >> 32)) - r.m) * a.inv_t - ls : -INFINITY;
}

template <typename T, bool ENT, bool TOP>
__global__ void __launch_bounds__(LP_NT) logprobs_kernel(LogprobsArgs a) {
  constexpr int N = chunk_elems<T>(), NW = LP_NT / 64;
  __shared__ RowSums part[NW];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int64_t b = blockIdx.x / (unsigned)a.parts;
  const int p = (int)(blockIdx.x - b * a.parts), c0 = p * a.per, cols = min(a.per, a.V - c0);
  const T *row = reinterpret_cast<const T *>(a.logits) + b * a.ldz, *z = row + c0;
  const RowChunks<T> chunks(z, cols);
  int t = -1;
  float zt = 0.f;
  if (a.parts == 1 && tid == 0) {
    t = a.tokens[b];
    if (t >= 0 && t < a.V) zt = load_f32(row + t);
  }
  float best = -INFINITY;
  int best_at = 0;
  const RowSums r = group_joined(walk<T, ENT, TOP>(chunks, a.c, &best, &best_at), a.c, part);
  const float ls = logf(r.s);
  if (tid == 0) {
    if (a.parts == 1) put_row(a, b, r, zt, t, ls);
    else a.sums[b * a.parts + p] = r;
  }
  if constexpr (TOP) {
    __shared__ uint64_t keys[LP_LIST];
    __shared__ int threads[LP_NT];
    __shared__ uint64_t bound_of, next[NW];
    __shared__ int n_threads, n_keys;
    auto put = [&](int j, uint64_t key) {
      if (a.parts == 1) put_choice(a, b, j, key, r, ls);
      else a.keys[(b * a.parts + p) * a.n + j] = key;
    };
    // keys that the thread's best does reach at least, and may reach at most
    const int at0 = chunks.column(best_at);
    const uint64_t some = choice_key(best, c0 + at0 + N - 1), most = choice_key(best, c0 + max(at0, 0));
    keys[tid] = some;
    if (tid == 0) n_threads = n_keys = 0;
    __syncthreads();
    if (wave == 0) {
      uint64_t g = some;
#pragma unroll
      for (int w = 1; w < NW; ++w) g = max64(g, keys[64 * w + lane]);
      const uint64_t at = nth_largest(g, a.n);
      if (lane == 0) bound_of = at;
    }
    __syncthreads();
    const uint64_t bound = bound_of;
    if (most >= bound) threads[atomicAdd(&n_threads, 1)] = tid;
    __syncthreads();
    auto look = [&](const u32x4 &v, int k) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const uint64_t key = choice_key(chunk_at<T>(v, j), c0 + chunks.column(k) + j);
        if (key >= bound) {
          const int at = atomicAdd(&n_keys, 1);
          if (at < LP_LIST) keys[at] = key;
        }
      }
    };
    // every thread looks at one chunk of one of them, several loads in flight (and at the cut chunks in any case)
    const int each = max(0, chunks.whole - chunks.first + LP_NT - 1) / LP_NT, all = n_threads * each;
    for (int i0 = tid; i0 < all; i0 += LP_UNROLL * LP_NT) {
      u32x4 v[LP_UNROLL];
      int k[LP_UNROLL];
#pragma unroll
      for (int q = 0; q < LP_UNROLL; ++q) {
        const int i = i0 + q * LP_NT, turn = i / n_threads;
        k[q] = i < all ? chunks.first + threads[i - turn * n_threads] + turn * LP_NT : chunks.whole;
        if (k[q] < chunks.whole) v[q] = chunks.load(k[q]);
      }
#pragma unroll
      for (int q = 0; q < LP_UNROLL; ++q)
        if (k[q] < chunks.whole) look(v[q], k[q]);
    }
    const bool head = chunks.skew > 0 && tid == LP_NT - 1;
    if (head || (chunks.tail && tid == 0)) look(chunks.load_cut(head ? 0 : chunks.whole), head ? 0 : chunks.whole);
    __syncthreads();
    const int found = n_keys;
    if (found <= LP_LIST) {
      put_in_order(keys, found, a.n, put);
      return;
    }
    uint64_t last = ~(uint64_t)0;
    for (int j = 0; j < a.n; ++j) {
      uint64_t k = 0;
      for (int v = tid; v < cols; v += LP_NT) {
        const uint64_t x = choice_key(load_f32(z + v), c0 + v);
        if (x < last) k = max64(k, x);
      }
      k = wave_max(k);
      __syncthreads();
      if (lane == 0) next[wave] = k;
      __syncthreads();
      last = max64(max64(next[0], next[1]), max64(next[2], next[3]));
      if (tid == 0) put(j, last);
    }
  }
}

// A row of several parts.
template <typename T>
__global__ void __launch_bounds__(LP_NT) logprobs_join_kernel(LogprobsArgs a) {
  __shared__ uint64_t keys[PARTS_MOST * TOP_MOST];
  __shared__ int n_keys;
  const int tid = threadIdx.x;
  const int64_t b = blockIdx.x;
  if (tid == 0) n_keys = 0;
  const int t = a.tokens[b];
  const float zt = t >= 0 && t < a.V ? load_f32(reinterpret_cast<const T *>(a.logits) + b * a.ldz + t) : 0.f;
  const RowSums r = joined_parts(a.sums + b * a.parts, a.parts, a.c);
  const float ls = logf(r.s);
  if (tid == 0) put_row(a, b, r, zt, t, ls);
  if (a.n == 0) return;
  const uint64_t *from = a.keys + b * a.parts * a.n;
  // the row's n best reach the n-th of 64 that are in the parts' lists: of the first few of each
  const int lane = tid & 63, some = min(a.n, 64 / a.parts), p = lane / some;
  const uint64_t bound = nth_largest(p < a.parts ? from[p * a.n + lane - p * some] : (uint64_t)0, a.n);
  __syncthreads();
  for (int i = tid; i < a.parts * a.n; i += LP_NT)
    if (from[i] >= bound) keys[atomicAdd(&n_keys, 1)] = from[i];
  __syncthreads();
  const int found = n_keys;
  put_in_order(keys, found, a.n, [&](int j, uint64_t key) { put_choice(a, b, j, key, r, ls); });
}

struct LogprobsBwdArgs {
  int V, parts, per;
  const void *logits;
  int64_t ldz;
  const int32_t *tokens;
  float inv_t;
  const float *lse, *entropy, *dlogp, *dentropy;
  void *dlogits;
  int64_t lddl;
};

// The gradient: one pass, a workgroup a part of a row.
template <typename T, typename TO>
__global__ void __launch_bounds__(LP_NT) logprobs_bwd_kernel(LogprobsBwdArgs a) {
  constexpr int N = chunk_elems<T>();
  const int64_t b = blockIdx.x / (unsigned)a.parts;
  const int p = (int)(blockIdx.x - b * a.parts), c0 = p * a.per, cols = min(a.per, a.V - c0);
  const T *z = reinterpret_cast<const T *>(a.logits) + b * a.ldz + c0;
  TO *out = reinterpret_cast<TO *>(a.dlogits) + b * a.lddl + c0;
  const int t = a.tokens[b], at = t - c0;
  float g = a.dlogp && t >= 0 ? a.dlogp[b] : 0.f;
  const float h = a.dentropy ? a.dentropy[b] : 0.f;
  const bool none = g == 0.f && h == 0.f;
  if (t >= a.V && !none) g = __builtin_nanf("");
  const float lse = a.lse[b], add = h == 0.f ? 0.f : a.entropy[b];
  g *= a.inv_t;
  const float hs = h * a.inv_t, base = g + hs * add;
  map_row<TO, LP_NT, LP_UNROLL>(RowChunks<T>(z, cols), out, [&](const u32x4 &v, int c, float(&d)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float lq = __builtin_elementwise_maximum(chunk_at<T>(v, i) * a.inv_t - lse, -200.f), q = pow2(lq * LOG2E);
      d[i] = -q * fmaf(hs, lq, base);
      if (none) d[i] = 0.f;
    }
    if (at >= c && at < c + N && at >= 0 && !none) {
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] += c + i == at ? g : 0.f;
    }
  });
}

}  // namespace

// Two workgroups a CU, of at least 4096 columns. 131072 columns in bf16 with 20 alternatives, 64 / 128 / 256 / 512 rows: 14.7
// / 17.3 / 26.4 / 38.0 us in 512 workgroups, 15.2 / 17.0 / 23.7 / 39.2 in 1024, 18.1 / 19.4 / 24.4 / 38.6 in 2048 (joining
// takes 4 to 5 of them; 512 rows of one part do without).
RowParts row_parts(int B, int V) {
  int parts = 512 / max(B, 1);
  parts = min(parts, min(PARTS_MOST, V / 4096));
  parts = max(parts, 1);
  const int per = (int)(((int64_t)V + parts - 1) / parts + 7) / 8 * 8;
  return RowParts{(int)(((int64_t)V + per - 1) / per), per};
}

size_t logprobs_ws_bytes(int B, int V, int n) {
  const RowParts cut = row_parts(B, V);
  return cut.parts == 1 ? 0 : (size_t)B * cut.parts * (sizeof(RowSums) + 8 * (size_t)n);
}

template <typename T>
static int launch_logprobs(const LogprobsArgs &a, int B, hipStream_t s) {
  const dim3 grid((unsigned)B * a.parts), wg(LP_NT);
  {
    LaunchTimer t(IMBD_K_LOGPROBS, 0, s);
    if (a.n > 0 && a.entropy) hipLaunchKernelGGL((logprobs_kernel<T, true, true>), grid, wg, 0, s, a);
    else if (a.n > 0) hipLaunchKernelGGL((logprobs_kernel<T, false, true>), grid, wg, 0, s, a);
    else if (a.entropy) hipLaunchKernelGGL((logprobs_kernel<T, true, false>), grid, wg, 0, s, a);
    else hipLaunchKernelGGL((logprobs_kernel<T, false, false>), grid, wg, 0, s, a);
  }
  const int rc = check_launch("token_logprobs");
  if (rc != IMBD_OK || a.parts == 1) return rc;
  {
    LaunchTimer t(IMBD_K_LOGPROBS, 1, s);
    hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3(B), wg, 0, s, a);
  }
  return check_launch("token_logprobs (join)");
}

int run_logprobs(int dtype, int B, int V, int n, const void *logits, int64_t ldz, const int32_t *tokens,
                 float temperature, float *logp, float *entropy, float *lse, int32_t *top_ids, float *top_logp, void *ws,
                 hipStream_t s) {
  const RowParts cut = row_parts(B, V);
  const float inv_t = 1.0f / temperature;
  LogprobsArgs a{V, n, cut.parts, cut.per, logits, ldz, tokens, inv_t, inv_t * LOG2E, logp, entropy, lse, top_ids, top_logp,
                 nullptr, nullptr};
  if (cut.parts > 1) {  // (the keys first: they are 8 bytes)
    a.keys = reinterpret_cast<uint64_t *>(ws);
    a.sums = reinterpret_cast<RowSums *>(a.keys + (size_t)B * cut.parts * n);
  }
  return dtype == IMBD_BF16 ? launch_logprobs<uint16_t>(a, B, s) : launch_logprobs<float>(a, B, s);
}

template <typename T>
static void launch_bwd(const LogprobsBwdArgs &a, int B, int dlogits_dtype, hipStream_t s) {
  const dim3 grid((unsigned)B * a.parts), wg(LP_NT);
  if (dlogits_dtype == IMBD_BF16) hipLaunchKernelGGL((logprobs_bwd_kernel<T, uint16_t>), grid, wg, 0, s, a);
  else hipLaunchKernelGGL((logprobs_bwd_kernel<T, float>), grid, wg, 0, s, a);
}

int run_logprobs_bwd(int dtype, int B, int V, const void *logits, int64_t ldz, const int32_t *tokens,
                     float temperature, const float *lse, const float *entropy, const float *dlogp,
                     const float *dentropy, void *dlogits, int64_t lddl, int dlogits_dtype, hipStream_t s) {
  const RowParts cut = row_parts(B, V);
  LogprobsBwdArgs a{V, cut.parts, cut.per, logits, ldz, tokens, 1.0f / temperature, lse, entropy, dlogp, dentropy, dlogits, lddl};
  {
    LaunchTimer t(IMBD_K_LOGPROBS, 2, s);
    if (dtype == IMBD_BF16) launch_bwd<uint16_t>(a, B, dlogits_dtype, s);
    else launch_bwd<float>(a, B, dlogits_dtype, s);
  }
  return check_launch("token_logprobs_bwd");
}

}  // namespace imbd
