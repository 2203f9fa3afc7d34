// Rows of logits over a vocabulary (csrc/logprobs.hip, csrc/distill.hip): internal declarations and the pieces that
// their kernels share.
#pragma once

#include "cdna4.h"
#include "lanes.h"

namespace imbd {

constexpr int TOP_MOST = 64;         // alternatives
constexpr int ENTRIES_MOST = 256;    // a teacher's entries of a row
constexpr int PARTS_MOST = 32;      // of a row
constexpr int VOCAB_MOST = 1 << 30;
constexpr int VOCAB_ROWS_MOST = (1 << 24) - 1;  // a workgroup of 256 each: a launch holds fewer than 2^32 work-items

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

template <typename T>
constexpr int chunk_elems() { return 16 / (int)sizeof(T); }

// The columns of a row (or part) from p on, walked in chunks that are aligned to 16 bytes wherever the row begins: chunk k holds
// columns k N - skew .. + N - 1. Chunks first .. whole - 1 are whole; chunk 0 before them (skew > 0) and chunk `whole` behind them
// (`tail`) are cut. (Chunks from the row's first column on read a bf16 row that begins in the middle of one 20% slower.)
template <typename T>
struct RowChunks {
  static constexpr int N = chunk_elems<T>();
  const T *p;
  int cols, skew, first, whole;
  bool tail;
  __device__ __forceinline__ RowChunks(const T *p_, int cols_) : p(p_), cols(cols_) {
    skew = (int)((uintptr_t)p_ & 15) / (int)sizeof(T);
    first = skew > 0;
    whole = (int)((uint32_t)(cols + skew) / N);
    tail = (cols + skew) % N != 0 && whole >= first;
  }
  __device__ __forceinline__ int column(int k) const { return k * N - skew; }
  __device__ __forceinline__ u32x4 load(int k) const { return *reinterpret_cast<const u32x4 *>(p + ((int64_t)k * N - skew)); }
  // what lies outside the row is -inf
  __device__ __forceinline__ u32x4 load_cut(int k) const {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      auto bits = [&](int j) -> uint32_t {
        const int c = column(k) + j;
        const bool in = c >= 0 && c < cols;
        if constexpr (sizeof(T) == 2) return in ? (uint32_t)p[c] : 0xff80u;
        else return in ? __builtin_bit_cast(uint32_t, p[c]) : 0xff800000u;
      };
      if constexpr (sizeof(T) == 2) v[i] = bits(2 * i) | bits(2 * i + 1) << 16;
      else v[i] = bits(i);
    }
    return v;
  }
};
template <typename T>
__device__ __forceinline__ float chunk_at(const u32x4 &v, int i) {
  const uint32_t w = v[sizeof(T) == 2 ? i >> 1 : i];  // (a copy: the cast of a vector's element itself takes the first)
  if constexpr (sizeof(T) == 2) return __builtin_bit_cast(float, i & 1 ? w & 0xffff0000u : w << 16);
  else return __builtin_bit_cast(float, w);
}
// Stores a chunk's N values, at any element alignment.
template <typename TO, int N>
__device__ __forceinline__ void store_chunk(TO *p, const float (&v)[N]) {
  if constexpr (sizeof(TO) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4_any *>(p + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
  } else if constexpr (N == 8) {
    *reinterpret_cast<u32x4_any *>(p) = u32x4{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]),
                                              cvt_pk_bf16(v[6], v[7])};
  } else {
    *reinterpret_cast<u32x2_any *>(p) = u32x2{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
  }
}
// Every chunk of the row through f(chunk, its values' results), which go to the same columns of out; UN chunks of a thread (of NT)
// in flight.
template <typename TO, int NT, int UN, typename T, typename F>
__device__ __forceinline__ void map_row(const RowChunks<T> &row, TO *out, F f) {
  constexpr int N = RowChunks<T>::N;
  const int tid = threadIdx.x;
  float d[N];
  int k = row.first + tid;
  for (; k + (UN - 1) * NT < row.whole; k += UN * NT) {
    u32x4 v[UN];
#pragma unroll
    for (int q = 0; q < UN; ++q) v[q] = row.load(k + q * NT);
#pragma unroll
    for (int q = 0; q < UN; ++q) {
      f(v[q], row.column(k + q * NT), d);
      store_chunk(out + row.column(k + q * NT), d);
    }
  }
  for (; k < row.whole; k += NT) {
    f(row.load(k), row.column(k), d);
    store_chunk(out + row.column(k), d);
  }
  const bool head = row.skew > 0 && tid == NT - 1;
  if (head || (row.tail && tid == 0)) {
    const int e = head ? 0 : row.whole, c = row.column(e);
    f(row.load_cut(e), c, d);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i >= 0 && c + i < row.cols) store_f32(out + c + i, d[i]);
  }
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
// All lanes' sums, in each of them.
__device__ __forceinline__ RowSums wave_joined(const RowSums &r, float c) {
  const RowSums x = moved(r, wave_max(r.m), c);
  return RowSums{x.m, wave_sum(x.s), wave_sum(x.u)};
}

// Long rows are cut into parts, a workgroup each, where the rows are too few to fill the GPU: `parts` of `per` columns (a
// multiple of 8; the last shorter).
struct RowParts {
  int parts, per;
};
RowParts row_parts(int B, int V);
// All parts of a row, joined by every wave for itself (PARTS_MOST <= 64).
__device__ __forceinline__ RowSums joined_parts(const RowSums *sums, int parts, float c) {
  const int lane = threadIdx.x & 63;
  return wave_joined(lane < parts ? sums[lane] : RowSums{LOWEST, 0.f, 0.f}, c);
}

}  // namespace imbd
