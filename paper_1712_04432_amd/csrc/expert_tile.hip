// Products of an expert layer for any sizes, strides and alignments, fp32 and bf16: the kernel behind
// expert_fwd and expert_bwd wherever the large-tile kernels do not take the call.
//   forward  y[s][o]    = sum_i W_e[o][i] x[rows[s]][i]   (+ b_e[o], ReLU)     over the slots s of e
//   Delta_X  dx[s][i]   = sum_o W_e[o][i] dy[s][o]        (* [x > 0])
//   Delta_W  dw_e[o][i] = sum_s dy[s][o] x[rows[s]][i]    for every e; db_e[o] = sum_s dy[s][o]
// Written as D(m, n) = sum_k A(m, k) B(k, n) with m the output's contiguous index:
//   forward: m = o, n = s, k = i (both operands k-contiguous); Delta_X: m = i, n = s, k = o (W by k-rows);
//   Delta_W: m = i, n = o, k = s (both by k-rows).
//
// A workgroup of four waves owns a 64 x 64 (or 64 x 32) tile of D and walks K in steps of 128 bytes a row, double-buffered
// in LDS, with the loads of the next two steps (Delta_W: one) in flight over the products; rows of 144 bytes make every
// fragment one conflict-free 16-byte read. Operands stored by k-rows are transposed in registers on their way.
// Addresses are 64-bit and loads are 16 bytes at any element alignment, so no size or stride is special. Whole
// steps load without conditions (rows that do not count from a row that exists); the last step of a K that is
// no whole number of them, and k-rows at the edge of their matrix, chunk by chunk and element by element.
// fp32 operands run on the fp32 matrix instruction: products and sums are fp32 for both types.

#include <type_traits>

#include "expert.h"

namespace imbd {
namespace {

constexpr int XT = 64;          // columns (m) of a tile
constexpr int XT_PITCH = 144;   // bytes per LDS row
constexpr int XT_OUT = XT + 4;  // staging row pitch in floats

// 16 bytes from p; elements at index >= valid read as 0.
template <typename T>
__device__ __forceinline__ u32x4 chunk16(const T *p, int valid) {
  constexpr int VEC = 16 / (int)sizeof(T);
  if (valid >= VEC) return *reinterpret_cast<const u32x4_any *>(p);
  T tmp[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) tmp[e] = e < valid ? p[e] : T(0);
  u32x4 r;
  __builtin_memcpy(&r, tmp, 16);
  return r;
}

// k-contiguous operand: R rows x 128 bytes, R/32 chunks a thread. row(r) gives row r's first element, or
// null for a row of zeros; it does not change over k. `some`: any row that exists.
template <typename T, int R>
struct KcTile {
  static constexpr int VEC = 16 / (int)sizeof(T), PER = R / 32;
  const T *p[PER];
  bool ok[PER];
  u32x4 v[2][PER];  // [register set][chunk]
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
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if constexpr (G) v[set][i] = ok[i] && kk < K ? chunk16<T>(p[i] + kk, K - kk) : u32x4{0u, 0u, 0u, 0u};
      else v[set][i] = *reinterpret_cast<const u32x4_any *>(p[i] + kk);
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
// thread of the first 8 R / VEC (`tid` is rotated so that two such operands use different waves). krow(j) gives
// the first column of the tile in the thread's k-row j of the step, or null for zeros.
template <typename T, int R, int SETS>
struct TrTile {
  static constexpr int VEC = 16 / (int)sizeof(T);
  static constexpr int NB = 8 * R / VEC;
  u32x4 v[SETS][VEC];
  __device__ __forceinline__ static int first_k(int tid) { return (tid & 7) * VEC; }
  // G: with the columns' end looked at
  template <bool G, typename F>
  __device__ __forceinline__ void load(int set, F krow, const T *some, int cols, int tid) {
    if (tid >= NB) return;
    const int c = (tid >> 3) * VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const T *p = krow(j);
      if constexpr (G) {
        v[set][j] = p && c < cols ? chunk16<T>(p + c, cols - c) : u32x4{0u, 0u, 0u, 0u};
      } else {
        v[set][j] = *reinterpret_cast<const u32x4_any *>((p ? p : some) + c);
        if (!p) v[set][j] = u32x4{0u, 0u, 0u, 0u};
      }
    }
  }
  __device__ __forceinline__ void store(int set, char *lds, int tid) {
    if (tid >= NB) return;
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
      *reinterpret_cast<u32x4 *>(lds + ((tid >> 3) * VEC + r) * XT_PITCH + (tid & 7) * 16) = o;
    }
  }
};

template <typename T>
__device__ __forceinline__ bool positive(T v) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(v) > 0.f;
  else return v > 0.f;
}

// TN: rows (n) of a tile, 64 or 32.
template <typename T, int PASS, int TN>
__global__ void __launch_bounds__(256, 2) expert_tile_kernel(ExpertArgs a, int tiles_m, int tiles_n) {
  constexpr int VEC = 16 / (int)sizeof(T);
  constexpr int BK = 8 * VEC;
  constexpr int STAGE = (XT + TN) * XT_PITCH;
  constexpr int FN = TN / 32;  // 16-row blocks of a wave (2 x 2 waves of 32 columns x TN/2 rows)
  static_assert(TN * XT_OUT * 4 <= 2 * STAGE, "the staged tile reuses the operand buffers");
  __shared__ __attribute__((aligned(16))) char smem[2 * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

  // each XCD takes a contiguous range of the launch order; column tiles run fastest, so that the tiles
  // that share rows of x (or dy) follow each other
  int bid = blockIdx.x;
  if ((gridDim.x & 7) == 0) bid = (bid & 7) * (int)(gridDim.x >> 3) + (bid >> 3);
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
  const int m0 = tm * XT, M = PASS == EXPERT_FWD ? a.d_out : a.d_in;
  const T *w = reinterpret_cast<const T *>(a.w) + (int64_t)e * a.sw;
  const T *x = reinterpret_cast<const T *>(a.x);
  const T *dy = reinterpret_cast<const T *>(a.dy);
  auto x_row = [&](int s) -> const T * {
    const int r = a.rows ? a.rows[s] : s;
    return r >= 0 && r < a.n_x ? x + (int64_t)r * a.ldx : nullptr;
  };

  constexpr int SETS = PASS == EXPERT_DW ? 1 : 2;  // register sets: steps whose loads are in flight
  KcTile<T, XT> ka;
  KcTile<T, TN> kb;
  TrTile<T, XT, SETS> ta;
  TrTile<T, TN, SETS> tb;
  const int tid_b = tid ^ 128;  // (the k-row operand of n: the other half of the workgroup)
  const int ka0 = TrTile<T, XT, SETS>::first_k(tid), kb0 = TrTile<T, TN, SETS>::first_k(tid_b);
  // whether whole steps of k-rows may load without conditions: the tile's columns all exist
  bool inside = true;
  if constexpr (PASS == EXPERT_FWD) {
    ka.init([&](int r) { return m0 + r < M ? w + (int64_t)(m0 + r) * a.ldw : nullptr; }, w, tid);
    kb.init([&](int r) { return n0 + r < n_end ? x_row(n0 + r) : nullptr; }, a.n_x > 0 ? x : w, tid);
  } else if constexpr (PASS == EXPERT_DX) {
    kb.init([&](int r) { return n0 + r < n_end ? dy + (int64_t)(n0 + r) * a.lddy : nullptr; }, dy, tid);
    inside = m0 + XT <= M;
  } else {
    inside = m0 + XT <= M && n0 + TN <= n_end && a.n_x > 0 && x != nullptr;
  }
  // Delta_W: the rows of x of this thread's k-rows, read a step ahead of their use (read with it, every row's load
  // waited for its index and, loads coming back in order, for all loads before that)
  int xrow[PASS == EXPERT_DW ? VEC : 1];
  auto next_rows = [&](int k0) {
    if constexpr (PASS == EXPERT_DW) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int k = k0 + ka0 + j;
        xrow[j] = k < K ? (a.rows ? a.rows[r0 + k] : r0 + k) : -1;
      }
    }
  };
  auto load = [&](auto gtag, int set, int k0) {
    constexpr bool G = decltype(gtag)::value;
    if constexpr (PASS == EXPERT_FWD) ka.template load<G>(set, k0, K, tid);
    if constexpr (PASS != EXPERT_DW) kb.template load<G>(set, k0, K, tid);
    if constexpr (PASS == EXPERT_DX)
      ta.template load<G>(set, [&](int j) { return k0 + ka0 + j < K ? w + (int64_t)(k0 + ka0 + j) * a.ldw + m0 : nullptr; }, w,
                          M - m0, tid);
    if constexpr (PASS == EXPERT_DW) {
      ta.template load<G>(set, [&](int j) { return xrow[j] >= 0 && xrow[j] < a.n_x ? x + (int64_t)xrow[j] * a.ldx + m0 : nullptr; },
                          x + m0, M - m0, tid);
      tb.template load<G>(set, [&](int j) { return k0 + kb0 + j < K ? dy + (int64_t)(r0 + k0 + kb0 + j) * a.lddy + n0 : nullptr; },
                          dy, n_end - n0, tid_b);
      next_rows(k0 + BK);
    }
  };
  auto store = [&](int set, char *buf) {
    if constexpr (PASS == EXPERT_FWD) ka.store(set, buf, tid);
    else ta.store(set, buf, tid);
    if constexpr (PASS != EXPERT_DW) kb.store(set, buf + XT * XT_PITCH, tid);
    else tb.store(set, buf + XT * XT_PITCH, tid_b);
  };

  const int wm = (wave & 1) * 32, wn = (wave >> 1) * (TN / 2), fr = lane & 15, fg = lane >> 4;
  f32x4 acc[2][FN];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bool do_db = PASS == EXPERT_DW && a.db && tm == 0;
  float dbsum = 0.f;

  const int nk = (K + BK - 1) / BK, nw = inside ? K / BK : 0;  // steps; whole ones
  const std::integral_constant<bool, false> plain{};
  const std::integral_constant<bool, true> guarded{};
  auto fetch = [&](int set, int kt) {
    if (kt < nw) load(plain, set, kt * BK);
    else if (kt < nk) load(guarded, set, kt * BK);
  };
  constexpr int DT = 256 / TN, DC = 8 / DT;  // db: threads a row, chunks a thread
  auto compute = [&](int kt) {
    const char *sa = smem + (kt & 1) * STAGE, *sb = sa + XT * XT_PITCH;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      u32x4 fa[2], fb[FN];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        fa[i] = *reinterpret_cast<const u32x4 *>(sa + (wm + 16 * i + fr) * XT_PITCH + kk * 64 + fg * 16);
#pragma unroll
      for (int j = 0; j < FN; ++j)
        fb[j] = *reinterpret_cast<const u32x4 *>(sb + (wn + 16 * j + fr) * XT_PITCH + kk * 64 + fg * 16);
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fa[i]),
                                                                __builtin_bit_cast(bf16x8, fb[j]), acc[i][j], 0, 0, 0);
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < 2; ++i)
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
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      *reinterpret_cast<f32x4 *>(stg + (wn + 16 * j + fr) * XT_OUT + wm + 16 * i + 4 * fg) = acc[i][j];
  __syncthreads();
  const int m = m0 + (tid & 15) * 4, cnt = min(4, M - m);
  if (cnt <= 0) return;
  float bias[4] = {0.f, 0.f, 0.f, 0.f};
  if (PASS == EXPERT_FWD && a.bias) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < cnt) bias[q] = a.bias[(int64_t)e * a.d_out + m + q];
  }
#pragma unroll
  for (int p = 0; p < TN / 16; ++p) {
    const int nl = 16 * p + (tid >> 4), n = n0 + nl;
    if (n >= n_end) continue;
    f32x4 v = *reinterpret_cast<const f32x4 *>(stg + nl * XT_OUT + (tid & 15) * 4);
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

template <typename T, int TN>
static int launch(int pass, const ExpertArgs &a, hipStream_t s) {
  const int M = pass == EXPERT_FWD ? a.d_out : a.d_in;
  const int64_t tm = pass == EXPERT_DW && !a.out ? 1 : (M + XT - 1) / XT;  // (db alone: the first column of tiles)
  const int64_t tn = (a.d_out + TN - 1) / TN;
  const int64_t blocks = (pass == EXPERT_DW ? a.E * tn : row_tiles_most(a.n_rows, a.E, TN)) * tm;
  if (blocks >= ((int64_t)1 << 31) - 8) {
    set_error("expert product: %lld tiles are more than one launch takes", (long long)blocks);
    return IMBD_EUNSUPPORTED;
  }
  if (blocks == 0) return IMBD_OK;
  const dim3 grid((unsigned)((blocks + 7) / 8 * 8)), wg(256);
  const int cm = (int)tm, cn = (int)tn;
  {
    LaunchTimer t(IMBD_K_EXPERT_FWD + pass, 0, s);
    if (pass == EXPERT_FWD) hipLaunchKernelGGL((expert_tile_kernel<T, EXPERT_FWD, TN>), grid, wg, 0, s, a, cm, cn);
    else if (pass == EXPERT_DX) hipLaunchKernelGGL((expert_tile_kernel<T, EXPERT_DX, TN>), grid, wg, 0, s, a, cm, cn);
    else hipLaunchKernelGGL((expert_tile_kernel<T, EXPERT_DW, TN>), grid, wg, 0, s, a, cm, cn);
  }
  return check_launch("expert_tile");
}

int run_expert_tile(int pass, int dtype, const ExpertArgs &a, hipStream_t s) {
  // 32-row tiles where those of 64 do not give every CU four: whole workgroups come out more even, and more of them
  // hide each other's waits. (The sums' order in K does not depend on the tile.)
  const int M = pass == EXPERT_FWD ? a.d_out : a.d_in;
  const int64_t rows = pass == EXPERT_DW ? (int64_t)a.E * ((a.d_out + 63) / 64) : (int64_t)a.n_rows / 64 + a.E / 2;
  const bool small = rows * ((M + XT - 1) / XT) < 1024;
  if (dtype == IMBD_BF16) return small ? launch<uint16_t, 32>(pass, a, s) : launch<uint16_t, 64>(pass, a, s);
  return small ? launch<float, 32>(pass, a, s) : launch<float, 64>(pass, a, s);
}

}  // namespace imbd
