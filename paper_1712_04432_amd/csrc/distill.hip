// Divergence of a student's softmax from a teacher of whose logits the top ones are known, and its gradient.
//
// Bound by memory: the logits have to be read and the gradient written. Between the two lies the softmax's sum, so
//  * rows that fit a workgroup's registers (180224 logits in bf16, 176 registers of each of 512 threads) stay there between
//    the sum and the gradient, and memory sees them once;
//  * longer rows, and few rows, are cut into parts: one launch for the parts' sums, one that joins them and walks the
//    part again.
// The teacher's entries are one a thread; what they need of each other is exchanged while the row is on its way. Their
// tokens get their gradient after the row's others are written, each from the sum over the entries that name the same
// token, so that two of them write the same value.
//
// Measured: 4096 rows of 131072 in bf16 446 us (4.8 TB/s; a large copy reaches 4.9), in two passes over memory 1382; 500 rows
// of 50021 in fp32 54 us; 64 rows of 1000 11 us (two launches).

#include "loss_mean.h"
#include "row_walk.h"
#include "vocab.h"

namespace imbd {
namespace {

struct DistillArgs {
  int V, K, parts, per;
  const void *logits;
  int64_t ldz;
  const int32_t *ids;
  const float *teacher, *lse, *weight;
  float t, inv_t, c, inv_batch;
  float *row_loss;
  void *dlogits;
  int64_t lddl;
  RowSums *sums;  // parts: [b][part]
  float *zt;      // ... and the student's logits at the entries, [b][K]
};

// What the first ENTRIES_MOST threads of a workgroup exchange.
struct EntryRoom {
  float top[4], sum[4], outside[4], kl[4];
  int id[ENTRIES_MOST];
  float p[ENTRIES_MOST];
};

// One entry of a row's teacher (threads from K on: none) and what the whole row has of them.
struct Entry {
  int id;          // its token, -1: none
  float lp, p;     // log p, p
  float mass;      // the sum of all p
  bool none;       // the row has no entry
  float bad;       // NaN where an entry's token lies past the end
};

__device__ __forceinline__ void read_entry(const DistillArgs &a, int64_t b, int *id, float *t) {
  const int tid = threadIdx.x;
  *id = -1;
  *t = -INFINITY;
  if (tid < a.K) {
    *id = a.ids[b * a.K + tid];
    *t = a.teacher[b * a.K + tid];
  }
}

// (All threads of the workgroup call it; barriers leave loads under way.)
__device__ __forceinline__ Entry make_entry(const DistillArgs &a, int id, float t, float lse, EntryRoom &room) {
  const int tid = threadIdx.x, wave = tid >> 6;
  Entry e;
  t = id >= 0 ? t * a.inv_t : -INFINITY;
  if (t == -INFINITY) id = -1;
  e.id = id;
  if (wave < 4) {
    const float top = wave_maximum(t), outside = wave_max(id >= a.V ? 1.f : 0.f);
    if ((tid & 63) == 0) room.top[wave] = top, room.outside[wave] = outside;
    room.id[tid] = id;
  }
  lds_barrier();
  const float top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(room.top[0], room.top[1]),
                                                  __builtin_elementwise_maximum(room.top[2], room.top[3]));
  e.none = top == -INFINITY;
  e.bad = room.outside[0] + room.outside[1] + room.outside[2] + room.outside[3] > 0.f ? __builtin_nanf("") : 0.f;
  const float x = id >= 0 ? expf(t - top) : 0.f;
  if (wave < 4) {
    const float sum = wave_sum(x);
    if ((tid & 63) == 0) room.sum[wave] = sum;
  }
  lds_barrier();
  const float sum = (room.sum[0] + room.sum[1]) + (room.sum[2] + room.sum[3]);
  // with the teacher's own lse the entries' probabilities are exp(t - lse), else they sum to 1
  const float lt = a.lse ? lse : top + logf(sum);
  e.lp = t - lt;
  e.p = id >= 0 ? (a.lse ? expf(e.lp) : x / sum) : 0.f;
  e.mass = a.lse ? expf(top - lt) * sum : 1.f + 0.f * sum;  // (a NaN stays one)
  if (wave < 4) room.p[tid] = e.p;
  return e;
}

// The row's loss (thread 0 stores it): zt the student's logit at the entry.
__device__ __forceinline__ void put_loss(const DistillArgs &a, int64_t b, const Entry &e, float zt, const RowSums &r, float w,
                                         EntryRoom &room) {
  const int tid = threadIdx.x, wave = tid >> 6;
  if (wave < 4) {
    const float lq = (zt - r.m) * a.inv_t - logf(r.s);
    const float kl = wave_sum(e.p != 0.f ? e.p * (e.lp - lq) : 0.f);
    if ((tid & 63) == 0) room.kl[wave] = kl;
  }
  lds_barrier();
  if (tid == 0) {
    const float kl = (room.kl[0] + room.kl[1]) + (room.kl[2] + room.kl[3]);
    a.row_loss[b] = w * (a.t * a.t) * kl + e.bad + (r.s == 0.f ? __builtin_nanf("") : 0.f);
  }
}

// The sum of p over the entries that name this one's token.
__device__ __forceinline__ float same_token(const DistillArgs &a, const Entry &e, const EntryRoom &room) {
  float same = 0.f;
  if (e.id >= 0)
#pragma unroll 8
    for (int j = 0; j < a.K; ++j) same += room.id[j] == e.id ? room.p[j] : 0.f;
  return same;
}

// dz = scale (q1 2^((z - m) c) - p): the factors of a row.
struct Slope {
  float scale, q1, sq;
  __device__ __forceinline__ Slope(const DistillArgs &a, const Entry &e, const RowSums &r, float w) {
    scale = a.inv_batch * w * a.t + e.bad + (r.s == 0.f ? __builtin_nanf("") : 0.f);
    q1 = e.mass / r.s;
    sq = scale * q1;
  }
};

template <int NT, int N, typename TO>
__device__ __forceinline__ void put_zero_columns(TO *out, int cols) {
  const float zero[N] = {};
  const int whole = cols / N, c = whole * N + (int)threadIdx.x;
  for (int k = threadIdx.x; k < whole; k += NT) store_chunk(out + (int64_t)k * N, zero);
  if (c < cols && c < whole * N + N) store_f32(out + c, 0.f);
}

// A row in a workgroup's registers: NC chunks of each of NT threads, and the elements of the cut chunks one a thread.
template <typename T, int NT, int NC>
__global__ void __launch_bounds__(NT) distill_row_kernel(DistillArgs a) {
  constexpr int N = chunk_elems<T>(), NW = NT / 64;
  __shared__ EntryRoom room;
  __shared__ RowSums part[NW];
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t b = blockIdx.x;
  const T *z = reinterpret_cast<const T *>(a.logits) + b * a.ldz;
  T *out = a.dlogits ? reinterpret_cast<T *>(a.dlogits) + b * a.lddl : nullptr;
  const RowChunks<T> row(z, a.V);
  const float w = a.weight ? a.weight[b] : 1.f;
  auto put_zeros = [&] {
    if (tid == 0) a.row_loss[b] = 0.f;
    if (out) put_zero_columns<NT, N>(out, a.V);
  };
  if (w == 0.f) return put_zeros();
  int id;
  float t;
  read_entry(a, b, &id, &t);
  const float lse = a.lse ? a.lse[b] : 0.f;
  u32x4 v[NC];
  const uint32_t fill = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int k = row.first + tid + i * NT;
    v[i] = u32x4{fill, fill, fill, fill};
    if (k < row.whole) v[i] = row.load(k);
  }
  // threads 0 .. 15: a column of the cut chunk before the whole ones, or of that behind them
  int column = -1;
  if (tid < 8) column = row.skew > 0 && tid < min(N - row.skew, a.V) ? tid : -1;
  else if (tid < 8 + N && row.tail) column = row.column(row.whole) + tid - 8;
  if (column >= a.V) column = -1;
  const float last = column >= 0 ? load_f32(z + column) : -INFINITY;
  const Entry e = make_entry(a, id, t, lse, room);
  if (e.none) return put_zeros();
  const float zt = e.id >= 0 && e.id < a.V ? load_f32(z + e.id) : 0.f;
  // (the chunks stay packed between the passes: the compiler would keep what it unpacks)
  auto packed = [&] {
#pragma unroll
    for (int i = 0; i < NC; ++i) asm volatile("" : "+v"(v[i]));
  };
  // ---- the sum, each thread's over its own largest logit
  RowSums r{fmaxf(LOWEST, last), 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) r.m = fmaxf(r.m, chunk_at<T>(v[i], j));
  packed();
  r.s = pow2((last - r.m) * a.c);
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) r.s += pow2((chunk_at<T>(v[i], j) - r.m) * a.c);
  r = wave_joined(r, a.c);
  if (lane == 0) part[tid >> 6] = r;
  lds_barrier();
  r = joined_parts(part, NW, a.c);
  put_loss(a, b, e, zt, r, w, room);
  if (!out) return;
  // ---- the gradient
  packed();
  const Slope g(a, e, r, w);
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int k = row.first + tid + i * NT;
    float d[N];
#pragma unroll
    for (int j = 0; j < N; ++j) d[j] = g.sq * pow2((chunk_at<T>(v[i], j) - r.m) * a.c);
    if (k < row.whole) store_chunk(out + row.column(k), d);
  }
  if (column >= 0) store_f32(out + column, g.sq * pow2((last - r.m) * a.c));
  const float same = same_token(a, e, room);
  vm_barrier<0>();  // (every store of the row has landed)
  if (e.id >= 0 && e.id < a.V) store_f32(out + e.id, g.scale * (g.q1 * pow2((zt - r.m) * a.c) - same));
}

constexpr int DP_NT = WALK_NT;  // threads of a part's workgroup

// The sums of every part, and the logits at the entries (the gradient may take the logits' place, and its parts come in
// any order).
template <typename T>
__global__ void __launch_bounds__(DP_NT) distill_sums_kernel(DistillArgs a) {
  __shared__ RowSums part[DP_NT / 64];
  const int tid = threadIdx.x;
  const int64_t b = blockIdx.x / (unsigned)a.parts;
  const int p = (int)(blockIdx.x - b * a.parts), c0 = p * a.per, cols = min(a.per, a.V - c0);
  const T *row = reinterpret_cast<const T *>(a.logits) + b * a.ldz;
  if (p == 0 && tid < a.K) {
    const int id = a.ids[b * a.K + tid];
    a.zt[b * a.K + tid] = id >= 0 && id < a.V ? load_f32(row + id) : 0.f;
  }
  float best;
  int best_at;
  const RowSums r = group_joined(walk<T, false, false>(RowChunks<T>(row + c0, cols), a.c, &best, &best_at), a.c, part);
  if (tid == 0) a.sums[blockIdx.x] = r;
}

// A part of a row, of which the sums are known.
template <typename T, typename TO>
__global__ void __launch_bounds__(DP_NT) distill_part_kernel(DistillArgs a) {
  constexpr int N = chunk_elems<T>();
  __shared__ EntryRoom room;
  const int tid = threadIdx.x;
  const int64_t b = blockIdx.x / (unsigned)a.parts;
  const int p = (int)(blockIdx.x - b * a.parts), c0 = p * a.per, cols = min(a.per, a.V - c0);
  const T *z = reinterpret_cast<const T *>(a.logits) + b * a.ldz + c0;
  TO *out = a.dlogits ? reinterpret_cast<TO *>(a.dlogits) + b * a.lddl + c0 : nullptr;
  const RowChunks<T> chunks(z, cols);
  const float w = a.weight ? a.weight[b] : 1.f;
  int id;
  float t;
  read_entry(a, b, &id, &t);
  const Entry e = make_entry(a, id, t, a.lse ? a.lse[b] : 0.f, room);
  if (w == 0.f || e.none) {
    if (p == 0 && tid == 0) a.row_loss[b] = 0.f;
    if (out) put_zero_columns<DP_NT, N>(out, cols);
    return;
  }
  const RowSums r = joined_parts(a.sums + b * a.parts, a.parts, a.c);
  const float zt = tid < a.K ? a.zt[b * a.K + tid] : 0.f;
  if (p == 0) put_loss(a, b, e, zt, r, w, room);
  if (!out) return;
  const bool mine = e.id >= c0 && e.id < c0 + cols;
  lds_barrier();
  const Slope g(a, e, r, w);
  map_row<TO, DP_NT, WALK_UNROLL>(chunks, out, [&](const u32x4 &v, int, float(&d)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = g.sq * pow2((chunk_at<T>(v, i) - r.m) * a.c);
  });
  const float same = same_token(a, e, room);
  vm_barrier<0>();
  if (mine) store_f32(out + (e.id - c0), g.scale * (g.q1 * pow2((zt - r.m) * a.c) - same));
}

__global__ void __launch_bounds__(256) distill_loss_kernel(int B, const float *row_loss, float inv_batch, float *loss) {
  __shared__ float part[256];
  block_loss_mean(B, row_loss, inv_batch, loss, part);
}

// Chunks of a row that distill_row_kernel holds at most.
constexpr int64_t ROW_CHUNKS_MOST = 512 * 44;

// Long rows in parts while they are fewer than CUs to fill. bf16, 131072 columns (registers / parts, the loss's launch
// included): 8 rows 18.9 / 12.5 us, 64 21.7 / 17.7, 128 25.5 / 26.2, 512 61.8 / 70.5, 1024 134 / 170; 65536: 32 rows 13.9 / 13.3,
// 128 16.0 / 17.6; 32768: 8 rows 11.9 / 12.2, 512 22.0 / 26.4; 175000: 48 rows 28.5 / 19.8, 128 32.8 / 33.5, 512 122 / 108,
// 1024 201 / 250. fp32, 65536: 32 rows 14.6 / 13.5, 64 16.6 / 16.4, 128 20.6 / 24.8.
// (A launch holds fewer than 2^32 work-items, which rows of more than 256 threads can pass: those in parts have 256.)
bool in_registers(int dtype, int B, int V) {
  const int64_t chunks = V / (dtype == IMBD_BF16 ? 8 : 4), threads = chunks <= 2048 ? 256 : chunks <= 4096 ? 512 : 1024;
  return (chunks <= 4096 || (chunks <= ROW_CHUNKS_MOST && B >= 96)) && B * threads < (int64_t)1 << 32;
}

// Registers for both a row's logits and few idle threads: 512 threads hold 44 chunks each without spilling (48 spill).
// bf16, 4096 rows (us): 70000 columns with 1024 threads of 16 chunks 336, with 512 of 20 252; 81920: 341, 277; 98304: 368,
// with 512 of 24 379; 34000 to 65536 alike within 5% with 1024 of 8 and 512 of 12 or 16. 170000 in registers 617, 190000 in parts 1011.
template <typename T>
void launch_row(const DistillArgs &a, int B, hipStream_t s) {
  const int chunks = a.V / chunk_elems<T>();
#define GO(NT, NC) hipLaunchKernelGGL((distill_row_kernel<T, NT, NC>), dim3(B), dim3(NT), 0, s, a)
  if (chunks <= 512) GO(256, 2);
  else if (chunks <= 1024) GO(256, 4);
  else if (chunks <= 2048) GO(256, 8);
  else if (chunks <= 4096) GO(512, 8);
  else if (chunks <= 8192) GO(1024, 8);
  else if (chunks <= 10240) GO(512, 20);
  else if (chunks <= 16384) GO(1024, 16);
  else if (chunks <= 20480) GO(512, 40);
  else GO(512, 44);
#undef GO
}

template <typename T>
int launch_parts(const DistillArgs &a, int B, int dlogits_dtype, hipStream_t s) {
  {
    LaunchTimer t(IMBD_K_DISTILL, 1, s);
    hipLaunchKernelGGL(distill_sums_kernel<T>, dim3((unsigned)B * a.parts), dim3(DP_NT), 0, s, a);
  }
  const int rc = check_launch("distill_xent (sums)");
  if (rc != IMBD_OK) return rc;
  const dim3 grid((unsigned)B * a.parts);
  {
    LaunchTimer t(IMBD_K_DISTILL, 0, s);
    if (dlogits_dtype == IMBD_BF16) hipLaunchKernelGGL((distill_part_kernel<T, uint16_t>), grid, dim3(DP_NT), 0, s, a);
    else hipLaunchKernelGGL((distill_part_kernel<T, float>), grid, dim3(DP_NT), 0, s, a);
  }
  return check_launch("distill_xent");
}

}  // namespace

size_t distill_ws_bytes(int B, int V, int K) {
  const RowParts cut = row_parts(B, V);
  return (size_t)B * (cut.parts * sizeof(RowSums) + 4 * (size_t)K);
}

int run_distill(int dtype, int B, int V, int K, const void *logits, int64_t ldz, const int32_t *ids,
                const float *teacher, const float *lse, const float *weight, float temperature, float inv_batch,
                float *loss, float *row_loss, void *dlogits, int64_t lddl, int dlogits_dtype, void *ws, hipStream_t s) {
  const float inv_t = 1.0f / temperature;
  const RowParts cut = row_parts(B, V);
  DistillArgs a{V, K, cut.parts, cut.per, logits, ldz, ids, teacher, lse, weight, temperature, inv_t, inv_t * LOG2E, inv_batch,
                row_loss, dlogits, lddl, nullptr, nullptr};
  if (B > 0) {
    int rc;
    if (in_registers(dtype, B, V) && (!dlogits || dlogits_dtype == dtype)) {
      {
        LaunchTimer t(IMBD_K_DISTILL, 0, s);
        if (dtype == IMBD_BF16) launch_row<uint16_t>(a, B, s);
        else launch_row<float>(a, B, s);
      }
      rc = check_launch("distill_xent");
    } else {
      a.sums = reinterpret_cast<RowSums *>(ws);
      a.zt = reinterpret_cast<float *>(a.sums + (size_t)B * cut.parts);
      rc = dtype == IMBD_BF16 ? launch_parts<uint16_t>(a, B, dlogits_dtype, s) : launch_parts<float>(a, B, dlogits_dtype, s);
    }
    if (rc != IMBD_OK) return rc;
  }
  {
    LaunchTimer t(IMBD_K_DISTILL, 2, s);
    hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(256), 0, s, B, row_loss, inv_batch, loss);
  }
  return check_launch("distill_xent (loss)");
}

}  // namespace imbd
