// A softmax's sums over a row of logits, by a workgroup in one pass.
#pragma once

#include "vocab.h"

namespace imbd {

constexpr int WALK_NT = 256;    // threads of a workgroup
constexpr int WALK_UNROLL = 4;  // chunks of a thread in flight

// One workgroup's part of a row. ENT: with u. TOP: remembers where the thread's largest logit is.
template <typename T, bool ENT, bool TOP>
__device__ __forceinline__ RowSums walk(const RowChunks<T> &row, float c, float *best, int *best_at) {
  constexpr int N = chunk_elems<T>();
  const int tid = threadIdx.x;
  const float slack = 16.f / c;
  RowSums r{LOWEST, 0.f, 0.f};
  auto take = [&](const auto &v, int first) {
    constexpr int M = sizeof(v) / 16;
    float top = -INFINITY;
#pragma unroll
    for (int q = 0; q < M; ++q) {
      float cm = chunk_at<T>(v[q], 0);
#pragma unroll
      for (int i = 1; i < N; ++i) cm = fmaxf(cm, chunk_at<T>(v[q], i));
      if constexpr (TOP) {
        const bool more = cm > *best;
        *best = more ? cm : *best;
        *best_at = more ? first + q * WALK_NT : *best_at;
      }
      top = fmaxf(top, cm);
    }
    if (top > r.m + slack) r = moved(r, top, c);
#pragma unroll
    for (int q = 0; q < M; ++q) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float x = chunk_at<T>(v[q], i);
        if constexpr (ENT) {
          const float d = scaled(x, r.m, c), e = pow2(d);
          r.s += e;
          r.u = fmaf(e, d, r.u);
        } else {
          r.s += pow2((x - r.m) * c);
        }
      }
    }
  };
  int k = row.first + tid;
  for (; k + (WALK_UNROLL - 1) * WALK_NT < row.whole; k += WALK_UNROLL * WALK_NT) {
    u32x4 v[WALK_UNROLL];
#pragma unroll
    for (int q = 0; q < WALK_UNROLL; ++q) v[q] = row.load(k + q * WALK_NT);
    take(v, k);
  }
  const bool head = row.skew > 0 && tid == WALK_NT - 1, tail = row.tail && tid == 0;
  for (; k < row.whole; k += WALK_NT) {
    const u32x4 v[1] = {row.load(k)};
    take(v, k);
  }
  if (head || tail) {
    const u32x4 v[1] = {row.load_cut(head ? 0 : row.whole)};
    take(v, head ? 0 : row.whole);
  }
  return r;
}

__device__ __forceinline__ RowSums group_joined(RowSums r, float c, RowSums *part) {
  const int tid = threadIdx.x;
  r = wave_joined(r, c);
  if ((tid & 63) == 0) part[tid >> 6] = r;
  __syncthreads();
  return joined(joined(part[0], part[1], c), joined(part[2], part[3], c), c);
}

}  // namespace imbd
