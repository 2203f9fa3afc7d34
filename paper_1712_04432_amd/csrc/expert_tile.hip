// Products of an expert layer for any sizes, strides and alignments, fp32 and bf16: the kernel behind
// expert_fwd and expert_bwd wherever the large-tile kernels do not take the call.
//   forward  y[s][o]    = sum_i W_e[o][i] x[rows[s]][i]   (+ b_e[o], ReLU)     over the slots s of e
//   Delta_X  dx[s][i]   = sum_o W_e[o][i] dy[s][o]        (* [x > 0])
//   Delta_W  dw_e[o][i] = sum_s dy[s][o] x[rows[s]][i]    for every e; db_e[o] = sum_s dy[s][o]
// Written as D(m, n) = sum_k A(m, k) B(k, n) with m the output's contiguous index:
//   forward: m = o, n = s, k = i (both operands k-contiguous); Delta_X: m = i, n = s, k = o (W by k-rows);
//   Delta_W: m = i, n = o, k = s (both by k-rows).
//
// A workgroup of four waves owns a 128 x 64, 64 x 64 or 64 x 32 tile of D and walks K in steps of 128 bytes a row,
// double-buffered in LDS, with the loads of the next two steps (Delta_W, and the largest tile: one) in flight over the
// products; rows of 144 bytes make every fragment one conflict-free 16-byte read. Operands stored by k-rows are
// transposed in registers on their way.
// Addresses are 64-bit and loads are 16 bytes at any element alignment, so no size or stride is special. Whole
// steps load without conditions (rows that do not count from a row that exists, blocks cut by the last column earlier and
// whole); the last step of a K that is no whole number of them looks at each row, and k-rows of less than 16 bytes are
// read element by element.
// fp32 operands run on the fp32 matrix instruction: products and sums are fp32 for both types.
//
// Measured, 16384 rows, 8 experts of 2047 x 2049: bf16 forward 402 TFLOP/s, Delta_X 262, Delta_W 218 (116 with gathered
// rows), fp32 102, 88 and 93 (71); bound by the latency of the steps. The transposes of bf16 take 173 to 219 registers in
// Delta_W and 174 to 182 in Delta_X, which leaves two workgroups a CU; fp32 has four, on 128 x 64 tiles two.

#include <type_traits>

#include "expert.h"

namespace imbd {
namespace {

constexpr int XT_PITCH = 144;   // bytes per LDS row

// Elements pos .. pos + VEC - 1 of a run of `len` (those from len on are 0): the run's last VEC elements, moved down.
template <typename T>
__device__ __forceinline__ u32x4 chunk16(const T *run, int pos, int len) {
  constexpr int VEC = 16 / (int)sizeof(T), BITS = 8 * (int)sizeof(T);
  unsigned __int128 v = 0;
  if (len >= VEC) {
    const int at = min(pos, len - VEC), by = pos - at;
    v = __builtin_bit_cast(unsigned __int128, *reinterpret_cast<const u32x4_any *>(run + at));
    v = by < VEC ? v >> (by * BITS) : 0;
  } else {
#pragma unroll 1
    for (int e = len - 1; e >= pos; --e) {
      if constexpr (sizeof(T) == 2) v = (v << BITS) | run[e];
      else v = (v << BITS) | __builtin_bit_cast(uint32_t, run[e]);
    }
  }
  return __builtin_bit_cast(u32x4, v);
}

// k-contiguous operand: R rows x 128 bytes, R/32 chunks a thread. row(r) gives row r's first element, or
// null for a row of zeros; it does not change over k. `some`: any row that exists.
template <typename T, int R, int SETS>
struct KcTile {
  static constexpr int VEC = 16 / (int)sizeof(T), PER = R / 32;
  const T *p[PER];
  bool ok[PER];
  u32x4 v[SETS][PER];  // [register set][chunk]
  template <typename F>
  __device__ __forceinline__ void init(F row, const T *some, int tid) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      p[i] = row((tid + 256 * i) >> 3);
      ok[i] = p[i] != nullptr;
      if (!ok[i]) p[i] = some;
    }
  }
  // G: with the edges looked at
  template <bool G>
  __device__ __forceinline__ void load(int set, int k0, int K, int tid) {
    const int kk = k0 + (tid & 7) * VEC;
    if constexpr (G) asm volatile("" : "+v"(K));  // (its addresses are not worth registers in the steps before)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if constexpr (G) {
        v[set][i] = ok[i] && kk < K ? chunk16<T>(p[i], kk, K) : u32x4{0u, 0u, 0u, 0u};
        __builtin_amdgcn_sched_barrier(0);  // (one after another: their shifts take registers)
      } else v[set][i] = *reinterpret_cast<const u32x4_any *>(p[i] + kk);
    }
  }
  __device__ __forceinline__ void store(int set, char *lds, int tid) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      *reinterpret_cast<u32x4 *>(lds + ((tid + 256 * i) >> 3) * XT_PITCH + (tid & 7) * 16) =
          ok[i] ? v[set][i] : u32x4{0u, 0u, 0u, 0u};
  }
};

// Operand stored by k-rows: 128 bytes of k x R columns, in blocks of VEC x VEC transposed in registers, one a
// thread of the first 8 R / VEC (`tid` is rotated so that two such operands use different waves). A block that the
// matrix's last column cuts is read `by` columns earlier, whole, and its first `by` columns, which are another
// block's too, are not stored; what lies past the last column in LDS reaches only outputs that are not stored.
template <typename T, int R, int SETS>
struct TrTile {
  static constexpr int VEC = 16 / (int)sizeof(T);
  static constexpr int NB = 8 * R / VEC;
  u32x4 v[SETS][VEC];
  int col, first;  // first column of the matrix that this thread reads; that is its own
  __device__ __forceinline__ static int first_k(int tid) { return (tid & 7) * VEC; }
  __device__ __forceinline__ void init(int col0, int width, int tid) {
    first = col0 + (tid >> 3) * VEC;
    col = width >= VEC ? min(first, width - VEC) : first;  // (narrower matrices: load_edge)
  }
  // element by element. krow(j): the first element of the thread's k-row j, or null for zeros
  template <typename F>
  __device__ __forceinline__ void load_edge(int set, F krow, int width, int tid) {
    if (tid >= NB) return;
    asm volatile("" : "+v"(width));
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const T *p = krow(j);
      v[set][j] = p && col < width ? chunk16<T>(p, col, width) : u32x4{0u, 0u, 0u, 0u};
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // rows ld apart from p on (which points at this thread's first column)
  __device__ __forceinline__ void load_rows(int set, const T *p, int64_t ld, int tid) {
    if (tid >= NB) return;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      v[set][j] = *reinterpret_cast<const u32x4_any *>(p);
      p += ld;
    }
  }
  // each row by its own pointer (null: zeros, read from `some`)
  template <typename F>
  __device__ __forceinline__ void load_each(int set, F krow, const T *some, int tid) {
    if (tid >= NB) return;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const T *p = krow(j);
      v[set][j] = *reinterpret_cast<const u32x4_any *>((p ? p : some) + col);
      if (!p) v[set][j] = u32x4{0u, 0u, 0u, 0u};
    }
  }
  __device__ __forceinline__ void store(int set, char *lds, int tid) {
    if (tid >= NB) return;
    const int by = first - col;
#pragma unroll
    for (int r = 0; r < VEC; ++r) {
      u32x4 o;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if constexpr (VEC == 8) {
          const uint32_t x = v[set][2 * q][r >> 1], y = v[set][2 * q + 1][r >> 1];
          o[q] = (r & 1) ? ((x >> 16) | (y & 0xffff0000u)) : ((x & 0xffffu) | (y << 16));
        } else {
          o[q] = v[set][q][r];
        }
      }
      if (r >= by)
        *reinterpret_cast<u32x4 *>(lds + ((tid >> 3) * VEC + r - by) * XT_PITCH + (tid & 7) * 16) = o;
    }
  }
};

template <typename T>
__device__ __forceinline__ bool positive(T v) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(v) > 0.f;
  else return v > 0.f;
}

// TM, TN: columns (m) and rows (n) of a tile. GATHER: Delta_W with x's rows by index. (An instance for each way: with both
// in one, fp32 Delta_W took 141 registers instead of 117 and 127, and three waves a SIMD instead of four.)
template <typename T, int PASS, int TM, int TN, bool GATHER>
__global__ void __launch_bounds__(256, 2) expert_tile_kernel(ExpertArgs a, int tiles_m, int tiles_n) {
  constexpr int VEC = 16 / (int)sizeof(T);
  constexpr int BK = 8 * VEC;
  constexpr int STAGE = (TM + TN) * XT_PITCH;
  constexpr int FM = TM / 32, FN = TN / 32;  // 16-wide blocks of a wave (2 x 2 waves)
  constexpr int PT = TM + 4;                 // staging row pitch in floats
  static_assert(TN * PT * 4 <= 2 * STAGE, "the staged tile reuses the operand buffers");
  __shared__ __attribute__((aligned(16))) char smem[2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

  // the XCDs take 32 tiles of the launch order at a time by turns (experts of different length are spread over all);
  // column tiles run fastest, so that the tiles that share rows of x (or dy) follow each other
  const int turn = (int)(blockIdx.x >> 3), bid = ((turn >> 5) * 8 + (int)(blockIdx.x & 7)) * 32 + (turn & 31);
  const int tm = bid % tiles_m;
  int e, n0, n_end, r0 = 0, K;
  if constexpr (PASS == EXPERT_DW) {
    const int t = bid / tiles_m;
    e = t / tiles_n;
    if (e >= a.E) return;
    n0 = (t - e * tiles_n) * TN;
    n_end = a.d_out;
    expert_range(a, e, &r0, &K);
  } else {
    if (!find_row_tile<TN>(a, bid / tiles_m, &e, &n0, &n_end)) return;
    K = PASS == EXPERT_FWD ? a.d_in : a.d_out;
  }
  const int m0 = tm * TM, M = PASS == EXPERT_FWD ? a.d_out : a.d_in;
  const T *w = reinterpret_cast<const T *>(a.w) + (int64_t)e * a.sw;
  const T *x = reinterpret_cast<const T *>(a.x);
  const T *dy = reinterpret_cast<const T *>(a.dy);
  auto x_row = [&](int s) -> const T * {
    const int r = a.rows ? a.rows[s] : s;
    return r >= 0 && r < a.n_x ? x + (int64_t)r * a.ldx : nullptr;
  };

  constexpr int SETS = PASS == EXPERT_DW || TM == 128 ? 1 : 2;  // register sets: steps whose loads are in flight
  KcTile<T, TM, SETS> ka;
  KcTile<T, TN, SETS> kb;
  TrTile<T, TM, SETS> ta;
  TrTile<T, TN, SETS> tb;
  const int tid_b = tid ^ 128;  // (the k-row operand of n: the other half of the workgroup)
  const int ka0 = TrTile<T, TM, SETS>::first_k(tid), kb0 = TrTile<T, TN, SETS>::first_k(tid_b);
  // whether every block of the k-rows can be read whole
  bool inside = true;
  if constexpr (PASS == EXPERT_FWD) {
    ka.init([&](int r) { return m0 + r < M ? w + (int64_t)(m0 + r) * a.ldw : nullptr; }, w, tid);
    kb.init([&](int r) { return n0 + r < n_end ? x_row(n0 + r) : nullptr; }, a.n_x > 0 ? x : w, tid);
  } else if constexpr (PASS == EXPERT_DX) {
    kb.init([&](int r) { return n0 + r < n_end ? dy + (int64_t)(n0 + r) * a.lddy : nullptr; }, dy, tid);
    ta.init(m0, M, tid);
    inside = M >= VEC;
  } else {
    ta.init(m0, M, tid);
    tb.init(n0, n_end, tid_b);
    inside = M >= VEC && n_end >= VEC && a.n_x > 0 && x != nullptr;
  }
  // Delta_W: the rows of x of this thread's k-rows, read a step ahead of their use (read with it, every row's load
  // waited for its index and, loads coming back in order, for all loads before that)
  constexpr bool GATHER_W = PASS == EXPERT_DW && GATHER;
  int xrow[GATHER_W ? VEC : 1];
  auto next_rows = [&](int k0) {
    if constexpr (GATHER_W) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int k = k0 + ka0 + j;
        xrow[j] = k < K ? a.rows[r0 + k] : -1;
      }
    }
  };
  // the k-rows of the next step, for whole steps (which come in order)
  const T *wk = w + (int64_t)ka0 * a.ldw + ta.col, *yk = dy + (int64_t)(r0 + kb0) * a.lddy + tb.col;
  const T *xk = x + (int64_t)(r0 + ka0) * a.ldx + ta.col;
  // G: the step that holds the end of K
  auto load = [&](auto gtag, int set, int k0) {
    constexpr bool G = decltype(gtag)::value;
    if constexpr (PASS == EXPERT_FWD) ka.template load<G>(set, k0, K, tid);
    if constexpr (PASS != EXPERT_DW) kb.template load<G>(set, k0, K, tid);
    int k_end = K;
    if constexpr (G) asm volatile("" : "+s"(k_end), "+s"(k0));  // (as above)
    if constexpr (PASS == EXPERT_DX) {
      auto w_at = [&](int j) { return k0 + ka0 + j < k_end ? w + (int64_t)(k0 + ka0 + j) * a.ldw : nullptr; };
      if (!G && inside) ta.load_rows(set, wk, a.ldw, tid);
      else if (inside) ta.load_each(set, w_at, w, tid);
      else ta.load_edge(set, w_at, M, tid);
      wk += BK * a.ldw;
    }
    if constexpr (PASS == EXPERT_DW) {
      auto x_at = [&](int j) -> const T * {
        if constexpr (GATHER) return (uint32_t)xrow[j] < (uint32_t)a.n_x ? x + (int64_t)xrow[j] * a.ldx : nullptr;
        else return k0 + ka0 + j < k_end && a.n_x > 0 ? x + (int64_t)(r0 + k0 + ka0 + j) * a.ldx : nullptr;
      };
      auto y_at = [&](int j) { return k0 + kb0 + j < k_end ? dy + (int64_t)(r0 + k0 + kb0 + j) * a.lddy : nullptr; };
      if (!inside) {
        ta.load_edge(set, x_at, M, tid);
        tb.load_edge(set, y_at, n_end, tid_b);
      } else {
        if constexpr (!G && !GATHER) ta.load_rows(set, xk, a.ldx, tid);
        else ta.load_each(set, x_at, x, tid);
        if (!G) tb.load_rows(set, yk, a.lddy, tid_b);
        else tb.load_each(set, y_at, dy, tid_b);
      }
      xk += BK * a.ldx;
      yk += BK * a.lddy;
      next_rows(k0 + BK);
    }
  };
  auto store = [&](int set, char *buf) {
    if constexpr (PASS == EXPERT_FWD) ka.store(set, buf, tid);
    else ta.store(set, buf, tid);
    if constexpr (PASS != EXPERT_DW) kb.store(set, buf + TM * XT_PITCH, tid);
    else tb.store(set, buf + TM * XT_PITCH, tid_b);
  };

  const int wm = (wave & 1) * (TM / 2), wn = (wave >> 1) * (TN / 2), fr = lane & 15, fg = lane >> 4;
  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bool do_db = PASS == EXPERT_DW && a.db && tm == 0;
  float dbsum = 0.f;

  const int nk = (K + BK - 1) / BK, nw = K / BK;  // steps; whole ones
  const std::integral_constant<bool, false> plain{};
  const std::integral_constant<bool, true> guarded{};
  auto fetch = [&](int set, int kt) {
    if (kt < nw) load(plain, set, kt * BK);
    else if (kt < nk) load(guarded, set, kt * BK);
  };
  constexpr int DT = 256 / TN, DC = 8 / DT;  // db: threads a row, chunks a thread
  auto compute = [&](int kt) {
    const char *sa = smem + (kt & 1) * STAGE, *sb = sa + TM * XT_PITCH;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      u32x4 fa[FM], fb[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i)
        fa[i] = *reinterpret_cast<const u32x4 *>(sa + (wm + 16 * i + fr) * XT_PITCH + kk * 64 + fg * 16);
#pragma unroll
      for (int j = 0; j < FN; ++j)
        fb[j] = *reinterpret_cast<const u32x4 *>(sb + (wn + 16 * j + fr) * XT_PITCH + kk * 64 + fg * 16);
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fa[i]),
                                                                __builtin_bit_cast(bf16x8, fb[j]), acc[i][j], 0, 0, 0);
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
              const f32x4 af = __builtin_bit_cast(f32x4, fa[i]), bf = __builtin_bit_cast(f32x4, fb[j]);
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(af[q], bf[q], acc[i][j], 0, 0, 0);
            }
      }
    }
    if (do_db) {
      // chunks of row tid/DT of the dy tile, in the order of k
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        const u32x4 q = *reinterpret_cast<const u32x4 *>(sb + (tid / DT) * XT_PITCH + ((tid % DT) * DC + c) * 16);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int h = 0; h < 8; ++h) dbsum += bf16_to_f32((uint16_t)(q[h >> 1] >> (16 * (h & 1))));
        } else {
          const f32x4 f = __builtin_bit_cast(f32x4, q);
#pragma unroll
          for (int h = 0; h < 4; ++h) dbsum += f[h];
        }
      }
    }
  };
  // step kt computes from LDS buffer kt % 2 while the loads of the next SETS steps are in flight: step kt + 1's
  // (register set (kt + 1) % SETS) go to the other buffer at its end
  next_rows(0);
  fetch(0, 0);
  if constexpr (SETS == 2) fetch(1, 1);
  if (nk > 0) store(0, smem);
  __syncthreads();
  for (int kt = 0; kt < nk; kt += 2) {
    fetch(0, kt + SETS);
    compute(kt);
    if (kt + 1 < nk) store(SETS - 1, smem + STAGE);
    __syncthreads();
    if (kt + 1 >= nk) break;
    fetch(SETS - 1, kt + 1 + SETS);
    compute(kt + 1);
    if (kt + 2 < nk) store(0, smem);
    __syncthreads();
  }
  if (do_db) {
#pragma unroll
    for (int o = 1; o < DT; o <<= 1) dbsum += __shfl_xor(dbsum, o, 64);
    if (tid % DT == 0 && n0 + tid / DT < n_end) a.db[(int64_t)e * a.d_out + n0 + tid / DT] = dbsum;
  }
  if (PASS == EXPERT_DW && !a.out) return;

  // ---- the tile through LDS as [n][m], then rows of four outputs a thread
  float *stg = reinterpret_cast<float *>(smem);
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      *reinterpret_cast<f32x4 *>(stg + (wn + 16 * j + fr) * PT + wm + 16 * i + 4 * fg) = acc[i][j];
  __syncthreads();
  constexpr int TPR = TM / 4, RPP = 256 / TPR;  // threads a row, rows a pass
  const int m = m0 + (tid % TPR) * 4, cnt = min(4, M - m);
  if (cnt <= 0) return;
  float bias[4] = {0.f, 0.f, 0.f, 0.f};
  if (PASS == EXPERT_FWD && a.bias) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < cnt) bias[q] = a.bias[(int64_t)e * a.d_out + m + q];
  }
#pragma unroll 2
  for (int p = 0; p < TN / RPP; ++p) {
    const int nl = RPP * p + tid / TPR, n = n0 + nl;
    if (n >= n_end) continue;
    f32x4 v = *reinterpret_cast<const f32x4 *>(stg + nl * PT + (tid % TPR) * 4);
    if constexpr (PASS == EXPERT_FWD) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v[q] += bias[q];
        if (a.relu) v[q] = v[q] < 0.f ? 0.f : v[q];  // (a NaN stays one)
      }
    }
    if constexpr (PASS == EXPERT_DX) {
      if (a.mask) {
        const T *mk = x_row(n);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (!(mk && q < cnt && positive<T>(mk[m + q]))) v[q] = 0.f;
      }
    }
    const int64_t at = (PASS == EXPERT_DW ? (int64_t)e * a.so : 0) + (int64_t)n * a.ldo + m;
    if (a.out_dtype == IMBD_BF16) {
      uint16_t *o = reinterpret_cast<uint16_t *>(a.out) + at;
      if (cnt == 4) *reinterpret_cast<u32x2_any *>(o) = u32x2{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
      else
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q < cnt) o[q] = f32_to_bf16(v[q]);
    } else {
      float *o = reinterpret_cast<float *>(a.out) + at;
      if (cnt == 4) *reinterpret_cast<f32x4_any *>(o) = v;
      else
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q < cnt) o[q] = v[q];
    }
  }
}

}  // namespace

template <typename T, int PASS, int TM, int TN>
static int launch(const ExpertArgs &a, bool check, hipStream_t s) {
  const int M = PASS == EXPERT_FWD ? a.d_out : a.d_in;
  const int64_t tm = PASS == EXPERT_DW && !a.out ? 1 : (M + TM - 1) / TM;  // (db alone: the first column of tiles)
  const int64_t tn = (a.d_out + TN - 1) / TN;
  const int64_t blocks = (PASS == EXPERT_DW ? a.E * tn : row_tiles_most(a.n_rows, a.E, TN)) * tm;
  if (blocks > WORKGROUPS_MOST - 255) {
    set_error("expert product: %lld tiles are more than one launch takes", (long long)blocks);
    return IMBD_EUNSUPPORTED;
  }
  if (blocks == 0 || check) return IMBD_OK;
  const dim3 grid((unsigned)((blocks + 255) / 256 * 256)), wg(256);
  const int cm = (int)tm, cn = (int)tn;
  {
    LaunchTimer t(IMBD_K_EXPERT_FWD + PASS, 0, s);
    if (PASS == EXPERT_DW && a.rows)
      hipLaunchKernelGGL((expert_tile_kernel<T, PASS, TM, TN, PASS == EXPERT_DW>), grid, wg, 0, s, a, cm, cn);
    else
      hipLaunchKernelGGL((expert_tile_kernel<T, PASS, TM, TN, false>), grid, wg, 0, s, a, cm, cn);
  }
  return check_launch("expert_tile");
}

template <typename T, int PASS>
static int launch_sized(const ExpertArgs &a, bool check, hipStream_t s) {
  // The larger tile, 128 x 64 or 64 x 64, where it gives every CU two or four workgroups: a large one reads its operands
  // less often, small ones come out more even and hide each other's waits. bf16, 16384 rows, 8 experts of 2047 x 2049:
  // forward 346 us on 128 x 64 and 453 on 64 x 64, Delta_X 525 and 808, Delta_W 631 and 849; 4096 rows, 1031 x 1037: 47
  // and 42, 69 and 85, 63 and 76. fp32 forward and Delta_W are faster on 64 x 64 (those two sizes: forward 1320 and 1345,
  // 139 and 118); fp32 Delta_X is the better one way or the other by the last round of workgroups (1557 and 1592, 178 and
  // 152, 6400 rows of 1031 x 1037 183 and 202). 3000 rows, 13 experts of 517 x 1023, fp32 forward 54 us on 64 x 32, 74 on 64 x 64.
  constexpr int SIDE = sizeof(T) == 2 || PASS == EXPERT_DX ? 128 : 64;
  const int M = PASS == EXPERT_FWD ? a.d_out : a.d_in;
  const int64_t rows = PASS == EXPERT_DW ? (int64_t)a.E * ((a.d_out + SIDE - 1) / SIDE)
                                         : (int64_t)a.n_rows / SIDE + (a.n_rows < a.E ? a.n_rows : a.E) / 2;
  const int64_t squares = rows * ((M + SIDE - 1) / SIDE);
  return squares >= (SIDE == 128 ? 256 : 1024) ? launch<T, PASS, SIDE, 64>(a, check, s)
                                              : launch<T, PASS, 64, 32>(a, check, s);
}

template <typename T>
static int launch_pass(int pass, const ExpertArgs &a, bool check, hipStream_t s) {
  return pass == EXPERT_FWD  ? launch_sized<T, EXPERT_FWD>(a, check, s)
         : pass == EXPERT_DX ? launch_sized<T, EXPERT_DX>(a, check, s)
                             : launch_sized<T, EXPERT_DW>(a, check, s);
}

int run_expert_tile(int pass, int dtype, const ExpertArgs &a, bool check, hipStream_t s) {
  return dtype == IMBD_BF16 ? launch_pass<uint16_t>(pass, a, check, s) : launch_pass<float>(pass, a, check, s);
}

}  // namespace imbd
