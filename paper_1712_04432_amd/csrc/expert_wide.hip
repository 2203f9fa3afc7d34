// The large-tile products of an expert layer (bf16 operands, fp32 accumulation), for whole 16-byte rows:
//   forward  y[s][o]    = sum_i W_e[o][i] x[rows[s]][i]   (+ b_e[o], ReLU)
//   Delta_X  dx[s][i]   = sum_o W_e[o][i] dy[s][o]        (* [x > 0])
//   Delta_W  dw_e[o][i] = sum_s dy[s][o] x[rows[s]][i];   db_e[o] = sum_s dy[s][o]
// as D(m, n) = sum_k A(m, k) B(k, n), m the output's contiguous index (o, i, i) and n its row (s, s, o).
//
// These products are bound by the matrix cores, and the tile is chosen for what feeds them: with 128 x 128
// outputs a wave, a k-step of 32 costs 16 KB of LDS reads and 64 matrix instructions (1024 cycles), so the
// four waves of a 256 x 256 tile read LDS half the time and its 160 KB hold the slabs of several k-steps.
// One wave a SIMD: nothing but its own instruction order hides its waits, so
//  * slabs of 32 k travel straight from memory to LDS through a ring of NS slots, NS - 1 k-steps ahead;
//  * the fragments of k-step S + 1 are read between the products of k-step S, into a second register set;
//  * one barrier a k-step, at which the wave's next products already have their operands in registers.
// Every load of a slab is issued by every wave in every step (past the last slab with an empty buffer
// descriptor, which fills zeros), so the number of loads in flight is the same everywhere and a wait is a
// constant.
//
// Slabs in LDS. An operand with k contiguous: rows of 64 bytes, the four 16-byte chunks XORed with 0, 2, 3, 1
// for rows 0-3, 4-7, 8-11, 12-15 of sixteen. (A 16-byte read serves lanes 0-3, 12-15, 20-27 and 4-11, 16-19,
// 28-31 of each half wave together; with these four, each such set covers all banks. 0, 1, 2, 3: twice the time.) By k-rows: quarters of 64 columns, 32 k-rows of 128
// bytes, read with the LDS transpose read; its swizzle is that of the weight-gradient kernel.
//
// Ragged edges. Rows of an expert's last tile, output columns past the width and k past the end read as
// zero: by lane (an offset past the buffer descriptor) or because the descriptor ends there. An expert's
// neighbours never enter a sum, not even times zero: their rows may hold infinities.

#include <type_traits>
#include <utility>

#include "expert.h"

namespace imbd {
namespace {

constexpr int XW_KS = 32;                     // k per slab
constexpr int XW_GM = 8;                      // m tiles per launch-order group
constexpr uint32_t XW_OOB = 0xffff0000u;      // past every buffer descriptor
constexpr uint32_t XW_MOST = 0xfffe0000u;     // bytes that a descriptor covers at most

__device__ __forceinline__ int xw_swz_tr(int r) { return 2 * ((r >> 1) & 1) + 4 * ((r >> 3) & 1); }

// f(0), f(1), .. f(N-1) with the number as a compile-time constant.
template <typename F, int... q>
__device__ __forceinline__ void static_for_seq(F &f, std::integer_sequence<int, q...>) {
  (f(std::integral_constant<int, q>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F f) {
  static_for_seq(f, std::make_integer_sequence<int, N>{});
}

__device__ __forceinline__ int xw_swz_kc(int v) { return 2 * ((v ^ (v >> 1)) & 1) + (v >> 1); }  // 0, 2, 3, 1

// One wave writes 64 x 16 bytes to LDS at lds_base + 16*lane, from byte offsets voff + IMM of the buffer. (The
// instruction's own offset counts on both sides, so it is taken off the LDS base.)
template <int IMM>
__device__ __forceinline__ void dma16_at(const i32x4 &rsrc, uint32_t voff, uint32_t lds_base) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen offset:%3 lds"
               :
               : "v"(voff), "s"(rsrc), "{m0}"(lds_base - IMM), "n"(IMM)
               : "memory");
}

// acc += A B on accumulation registers. A wave's 256 accumulators fill that half of the register file
// exactly, and only named as such do they stay there: left to itself the compiler moved them through the
// other half (500 moves in a k-step pair, and spills).
__device__ __forceinline__ void mfma(f32x4 &acc, const bf16x8 &a, const bf16x8 &b) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
// The same on plain registers; the operand `a` may be a constant that the compiler writes just before (wait
// states between a vector write and a matrix instruction's read are not its business in inline assembly; the
// fragments of the other form come from LDS and are waited for).
__device__ __forceinline__ void mfma_v(f32x4 &acc, const bf16x8 &a, const bf16x8 &b) {
  asm volatile("s_nop 3\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "v"(b));
}
// Wait states between the last product and the first read of its result (the compiler does not see them).
__device__ __forceinline__ void mfma_drain() { asm volatile("s_nop 15\n\ts_nop 15" : : : "memory"); }

// A buffer descriptor that moves by `step` bytes a slab: `most` bytes on every slab, `last` on the one that
// holds the end of k, none past it.
struct Window {
  uint64_t base;
  int64_t step;
  uint32_t most, last;
  __device__ __forceinline__ i32x4 next(bool live, bool ends) {
    const i32x4 r = buf_rsrc(reinterpret_cast<const void *>(base), live ? (ends ? last : most) : 0u);
    base += (uint64_t)step;
    return r;
  }
};

// One operand's slab: R rows (or columns) of the tile, loaded by four waves. KC: k contiguous (R rows of 64
// bytes); else by k-rows (32 k-rows of R columns).
template <int R, bool KC>
struct Slab {
  static constexpr int BYTES = R * 64;
  static constexpr int PER = R / 64;  // loads a wave
  uint32_t voff[KC ? PER : 1];        // k-rows: one offset, the quarters 128 bytes apart
};

template <int PASS, int BM, int BN, int NS>
struct Shape {
  static constexpr bool A_KC = PASS == EXPERT_FWD, B_KC = PASS != EXPERT_DW;
  static constexpr int FM = BM / 32, FN = BN / 32;  // 16-wide blocks of a wave (2 x 2 waves)
  static constexpr int SLAB = (BM + BN) * 64;
  static constexpr int RING = NS * SLAB;
  static constexpr int LOADS = BM / 64 + BN / 64;   // a wave, a slab
};

template <int PASS, int BM, int BN, int NS, bool GATHER>
constexpr int xw_lds_bytes() {
  // the ring; Delta_W with gathered x: the row indices of 2*NS slabs, 256 bytes a wave each
  constexpr int ring = Shape<PASS, BM, BN, NS>::RING + (PASS == EXPERT_DW && GATHER ? 2 * NS * 1024 : 0);
  constexpr int stage = 4 * 16 * (BM / 2 * 4 + 16);  // the epilogue: 16 rows of each wave
  return ring > stage ? ring : stage;
}

template <int PASS, int BM, int BN, int NS, bool GATHER, int WGS>
__global__ void __launch_bounds__(256, WGS) expert_wide_kernel(ExpertArgs a, int tiles_m, int tiles_n) {
  using Sh = Shape<PASS, BM, BN, NS>;
  constexpr bool A_KC = Sh::A_KC, B_KC = Sh::B_KC;
  constexpr int FM = Sh::FM, FN = Sh::FN;
  constexpr bool GATHER_W = PASS == EXPERT_DW && GATHER;  // x by k-rows, each from its own row
  constexpr int LOADS = Sh::LOADS + (GATHER_W ? 1 : 0);
  __shared__ __attribute__((aligned(1024))) char smem[xw_lds_bytes<PASS, BM, BN, NS, GATHER>()];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;

  // ---- the tile. The launch order has tiles in groups of XW_GM m tiles x all n tiles (Delta_W: of one expert);
  // the XCDs take 32 of it at a time by turns, so the workgroups resident on an XCD share slabs in its L2, and
  // experts of different length are spread over all XCDs (a contiguous range for each: Delta_W of 8 experts,
  // one to an XCD, waited for the longest twice as long as it worked).
  const int turn = (int)(blockIdx.x >> 3);
  int L = ((turn >> 5) * 8 + (int)(blockIdx.x & 7)) * 32 + (turn & 31);
  int e = 0, m0, n0, n_end, r0 = 0, K;
  const int M = PASS == EXPERT_FWD ? a.d_out : a.d_in;
  if constexpr (PASS == EXPERT_DW) {
    e = L / (tiles_m * tiles_n);
    L -= e * (tiles_m * tiles_n);
  }
  const int mg = L / (XW_GM * tiles_n);
  const int gsz = min(XW_GM, tiles_m - mg * XW_GM);
  if (e >= a.E || gsz <= 0) return;
  L -= mg * XW_GM * tiles_n;
  const int tn = L / gsz;
  m0 = (mg * XW_GM + L - tn * gsz) * BM;
  if constexpr (PASS == EXPERT_DW) {
    n0 = tn * BN;
    n_end = a.d_out;
    expert_range(a, e, &r0, &K);
    r0 = __builtin_amdgcn_readfirstlane(r0);
    K = __builtin_amdgcn_readfirstlane(K);
  } else {
    if (!find_row_tile<BN>(a, tn, &e, &n0, &n_end)) return;
    K = PASS == EXPERT_FWD ? a.d_in : a.d_out;
  }
  const int nsl = (K + XW_KS - 1) / XW_KS;
  const uint16_t *w = reinterpret_cast<const uint16_t *>(a.w) + (int64_t)e * a.sw;
  const uint16_t *x = reinterpret_cast<const uint16_t *>(a.x);
  const uint16_t *dy = reinterpret_cast<const uint16_t *>(a.dy);

  // ---- sources: a window on each operand and every lane's offsets in it
  Slab<BM, A_KC> sa;
  Slab<BN, B_KC> sb;
  Window wa, wb;
  const int kc = 8 * ((lane & 3) ^ xw_swz_kc(lane >> 4));            // k-contiguous: this lane's first k in a slab
  const int kr = 8 * wave + (lane >> 3);                           // k-rows: this lane's row of a slab
  const uint32_t kcol = (uint32_t)(16 * ((lane & 7) ^ xw_swz_tr(kr)));  // ... and byte column of a quarter
  const int k_last = K - (nsl - 1) * XW_KS;                        // k of the last slab
  // rows of k: 32 of them (k_last in the last slab) of `cols` columns from the window's base on
  auto k_rows = [&](const uint16_t *p, int64_t ld, int cols) {
    return Window{(uint64_t)(uintptr_t)p, XW_KS * ld * 2, (uint32_t)(((XW_KS - 1) * ld + cols) * 2),
                  (uint32_t)(((k_last - 1) * ld + cols) * 2)};
  };
  // k contiguous: `rows` rows (what lies past k in the last slab is masked by lane)
  auto k_cols = [&](const uint16_t *p, int64_t ld, int64_t rows) {
    const uint32_t n = rows > 0 ? (uint32_t)(((rows - 1) * ld + min(K, XW_KS)) * 2) : 0u;
    return Window{(uint64_t)(uintptr_t)p, XW_KS * 2, n, rows > 0 ? (uint32_t)(((rows - 1) * ld + k_last) * 2) : 0u};
  };
  if constexpr (A_KC) {
    wa = k_cols(w + (int64_t)m0 * a.ldw, a.ldw, min(BM, M - m0));
#pragma unroll
    for (int q = 0; q < BM / 64; ++q) {
      const int r = 16 * (BM / 64 * wave + q) + (lane >> 2);
      sa.voff[q] = m0 + r < M ? (uint32_t)(((int64_t)r * a.ldw + kc) * 2) : XW_OOB;
    }
  } else if constexpr (PASS == EXPERT_DX) {
    wa = k_rows(w + m0, a.ldw, M - m0);
    sa.voff[0] = (uint32_t)((int64_t)kr * a.ldw * 2) + kcol;
  } else if constexpr (!GATHER) {
    wa = k_rows(x + (int64_t)r0 * a.ldx + m0, a.ldx, M - m0);
    sa.voff[0] = (uint32_t)((int64_t)kr * a.ldx * 2) + kcol;
  } else {
    // (any row of x: the rows that do not exist are masked by lane)
    const uint32_t n = a.n_x > 0 ? (uint32_t)(((int64_t)(a.n_x - 1) * a.ldx + M - m0) * 2) : 0u;
    wa = Window{(uint64_t)(uintptr_t)(x + m0), 0, n, n};
    sa.voff[0] = XW_OOB;
  }
  if constexpr (B_KC) {
    constexpr bool G = PASS == EXPERT_FWD && GATHER;
    const int64_t ld = PASS == EXPERT_FWD ? a.ldx : a.lddy;
    const uint16_t *src = PASS == EXPERT_FWD ? x : dy;
    wb = k_cols(G ? src : src + (int64_t)n0 * ld, ld, G ? a.n_x : min(BN, n_end - n0));
#pragma unroll
    for (int q = 0; q < BN / 64; ++q) {
      const int r = 16 * (BN / 64 * wave + q) + (lane >> 2);
      bool ok = n0 + r < n_end;
      int row = r;
      if constexpr (G) {
        row = ok ? a.rows[n0 + r] : -1;
        ok = row >= 0 && row < a.n_x;
      }
      sb.voff[q] = ok ? (uint32_t)row * (uint32_t)(ld * 2) + (uint32_t)(kc * 2) : XW_OOB;
    }
  } else {
    wb = k_rows(dy + (int64_t)r0 * a.lddy + n0, a.lddy, n_end - n0);
    sb.voff[0] = (uint32_t)((int64_t)kr * a.lddy * 2) + kcol;
  }

  // the row indices of gathered k-rows: lane l's of slab X at idx0 + (X % 2NS)*1024 + 4l
  const uint32_t idx0 = lds0 + (uint32_t)(Sh::RING + wave * 256);
  const i32x4 ri = GATHER_W ? buf_rsrc(a.rows + r0, (uint32_t)K * 4u) : i32x4{0, 0, 0, 0};
  auto load_index = [&](int X) {
    if constexpr (GATHER_W)
      dma4(ri, (uint32_t)(X * XW_KS + kr) * 4u, idx0 + (uint32_t)((X % (2 * NS)) * 1024));
  };
  auto index_of = [&](int X) {  // (its indices have landed)
    return *(const __attribute__((address_space(3))) int *)(uintptr_t)(idx0 + (uint32_t)((X % (2 * NS)) * 1024 + 4 * lane));
  };
  auto gather = [&](int X, int row) {  // the offsets of slab X
    const bool ok = X * XW_KS + kr < K && row >= 0 && row < a.n_x;
    sa.voff[0] = ok ? (uint32_t)row * (uint32_t)(a.ldx * 2) + kcol : XW_OOB;
  };

  // ---- loads of slab X, in LOADS pieces (slabs in order: the windows move on)
  i32x4 ra, rb;
  uint32_t slot_w = 0;
  bool past = false;  // this lane's k lies past the end (k contiguous)
  auto open_a = [&](int X) {
    ra = wa.next(X < nsl, X == nsl - 1);
    slot_w = lds0 + (uint32_t)((X % NS) * Sh::SLAB);
  };
  auto open_b = [&](int X) {
    rb = wb.next(X < nsl, X == nsl - 1);
    if constexpr (A_KC || B_KC) past = X * XW_KS + kc >= K;
  };
  auto piece = [&](auto qtag) {
    constexpr int q = decltype(qtag)::value;
    if constexpr (q < BM / 64) {
      if constexpr (A_KC) dma16_at<0>(ra, past ? XW_OOB : sa.voff[q], slot_w + (uint32_t)((BM / 64 * wave + q) * 1024));
      else dma16_at<128 * q>(ra, sa.voff[0], slot_w + (uint32_t)(q * 4096 + wave * 1024));
    } else if constexpr (q < Sh::LOADS) {
      constexpr int p = q - BM / 64;
      const uint32_t to = slot_w + (uint32_t)(BM * 64);
      if constexpr (B_KC) dma16_at<0>(rb, past ? XW_OOB : sb.voff[p], to + (uint32_t)((BN / 64 * wave + p) * 1024));
      else dma16_at<128 * p>(rb, sb.voff[0], to + (uint32_t)(p * 4096 + wave * 1024));
    }
  };

  // ---- fragments
  const int fi = lane & 15, kg = lane >> 4, wm = wave & 1, wn = wave >> 1;
  const int tr = 8 * kg + (fi >> 2);
  uint32_t fa[A_KC ? 1 : 4], fb[B_KC ? 1 : 4];
  {
    const uint32_t kcl = (uint32_t)(fi * 64 + ((kg ^ xw_swz_kc(fi >> 2)) * 16));
    if constexpr (A_KC) fa[0] = lds0 + (uint32_t)(wm * FM * 1024) + kcl;
    if constexpr (B_KC) fb[0] = lds0 + (uint32_t)(BM * 64 + wn * FN * 1024) + kcl;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t c = (uint32_t)(((2 * j + ((fi >> 1) & 1)) ^ xw_swz_tr(tr)) * 16 + tr * 128 + 8 * (fi & 1));
      // (a wave's blocks start on a quarter or, 32-wide waves, in the middle of one)
      if constexpr (!A_KC) fa[j] = lds0 + (uint32_t)(wm * FM / 4 * 4096) + c;
      if constexpr (!B_KC) fb[j] = lds0 + (uint32_t)(BM * 64 + wn * FN / 4 * 4096) + c;
    }
  }
  static_assert(FM % 4 == 0 && FN % 4 == 0, "k-row fragments come in whole quarters");
  auto lds16 = [](uint32_t p) {
    return __builtin_bit_cast(bf16x8, *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)p);
  };
  auto lds_tr = [](uint32_t p) {
    lds_i16x4 *q = (lds_i16x4 *)(uintptr_t)p;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(q + 4 * 128 / 8);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto read_a = [&](uint32_t slot, int i) {
    if constexpr (A_KC) return lds16(fa[0] + slot + (uint32_t)(i * 1024));
    else return lds_tr(fa[i & 3] + slot + (uint32_t)((i >> 2) * 4096));
  };
  auto read_b = [&](uint32_t slot, int j) {
    if constexpr (B_KC) return lds16(fb[0] + slot + (uint32_t)(j * 1024));
    else return lds_tr(fb[j & 3] + slot + (uint32_t)((j >> 2) * 4096));
  };

  f32x4 acc[FM][FN], accd[PASS == EXPERT_DW ? FN : 1];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // db: the products with a row of ones, by the waves of the first m tile's first half
  const bool do_db = PASS == EXPERT_DW && a.db && m0 == 0 && wm == 0;
  if constexpr (PASS == EXPERT_DW)
#pragma unroll
    for (int j = 0; j < FN; ++j) accd[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});

  // ---- the first NS slabs (and the indices of 2 NS)
  if constexpr (GATHER_W) {
#pragma unroll
    for (int X = 0; X < 2 * NS; ++X) load_index(X);
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
  }
  // (a slab's loads end with the index load of the slab NS after it; the first NS slabs repeat one instead,
  // which keeps their number)
#pragma unroll
  for (int X = 0; X < NS; ++X) {
    if constexpr (GATHER_W) gather(X, index_of(X));
    open_a(X);
    open_b(X);
    static_for<Sh::LOADS>(piece);
    load_index(X);
  }

  bf16x8 av[2][FM], bv[2][FN];
  vm_barrier<LOADS * (NS - 1)>();  // slab 0
#pragma unroll
  for (int i = 0; i < FM; ++i) av[0][i] = read_a(0, i);
#pragma unroll
  for (int j = 0; j < FN; ++j) bv[0][j] = read_b(0, j);

  auto step = [&](int S, auto ctag) {
    constexpr int c = decltype(ctag)::value;
    // slab S + 1 has landed everywhere, and every wave has slab S in registers: its slot is free
    vm_barrier<LOADS * (NS - 2)>();
    const uint32_t slot = (uint32_t)(((S + 1) % NS) * Sh::SLAB);
    const int X = S + NS;
    int row = 0;
    // The step's FM * FN products in pairs, and before each pair what fits its 32 cycles: the reads of k-step
    // S + 1 in the first half, then the windows and the loads of slab S + NS. (All the scalar work of a slab in
    // one place left the matrix cores idle for 15% of the step.)
    constexpr int NP = FM * FN / 2, RP = NP / 2, NR = FM + FN, LP = NP - RP - 4;
    static_for<NP>([&](auto ptag) {
      constexpr int p = decltype(ptag)::value;
      if constexpr (p < RP) {
        if constexpr (GATHER_W && p == 0) row = index_of(X);
#pragma unroll
        for (int r = p * NR / RP; r < (p + 1) * NR / RP; ++r) {
          // (a and b by turns, then what is left of the longer)
          constexpr int both = 2 * (FM < FN ? FM : FN);
          const bool is_a = r < both ? r % 2 == 0 : FM > FN;
          const int at = r < both ? r / 2 : r - both / 2;
          if (is_a) av[c ^ 1][at < FM ? at : 0] = read_a(slot, at);
          else bv[c ^ 1][at < FN ? at : 0] = read_b(slot, at);
        }
      } else if constexpr (p == RP) {
        open_a(X);
      } else if constexpr (p == RP + 2) {
        open_b(X);
        if constexpr (GATHER_W) gather(X, row);
      } else if constexpr (p >= RP + 4) {
        constexpr int l = p - RP - 4, lo = l * Sh::LOADS / LP, hi = (l + 1) * Sh::LOADS / LP;
        static_for<hi - lo>([&](auto q) { piece(std::integral_constant<int, lo + decltype(q)::value>{}); });
        if constexpr (p == NP - 1) load_index(X + NS);
      }
      mfma(acc[2 * p / FN][2 * p % FN], av[c][2 * p / FN], bv[c][2 * p % FN]);
      mfma(acc[2 * p / FN][2 * p % FN + 1], av[c][2 * p / FN], bv[c][2 * p % FN + 1]);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (PASS == EXPERT_DW) {
      if (do_db) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
          mfma_v(accd[j], ones, bv[c][j]);
      }
    }
  };
  int S = 0;
  for (; S + 2 <= nsl; S += 2) {
    step(S, std::integral_constant<int, 0>{});
    step(S + 1, std::integral_constant<int, 1>{});
  }
  if (S < nsl) step(S, std::integral_constant<int, 0>{});
  vm_barrier<0>();  // LDS is free: nothing is in flight and every wave is done reading
  mfma_drain();
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[i][j]));  // (read behind the wait states)
  if constexpr (PASS == EXPERT_DW)
#pragma unroll
    for (int j = 0; j < FN; ++j) asm volatile("" : "+v"(accd[j]));

  if constexpr (PASS == EXPERT_DW) {
    if (do_db && kg == 0) {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int n = n0 + 16 * (wn * FN + j) + fi;
        if (n < n_end) a.db[(int64_t)e * a.d_out + n] = accd[j][0];
      }
    }
    if (!a.out) return;
  }

  // ---- epilogue: each wave puts 16 rows of its outputs at a time through its own part of LDS ([n][m]) and
  // stores whole rows, 16 bytes a lane
  constexpr int WM = BM / 2;  // outputs of a row
  char *stg = smem + wave * (16 * (WM * 4 + 16));
  const int mw = m0 + wm * WM;
  f32x4 bias[PASS == EXPERT_FWD ? FM : 1];
  if constexpr (PASS == EXPERT_FWD) {
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = mw + 16 * i + 4 * kg;  // (the width is a multiple of 8: all four or none)
      bias[i] = a.bias && m < M ? *reinterpret_cast<const f32x4_any *>(a.bias + (int64_t)e * a.d_out + m)
                                : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  const bool half = a.out_dtype == IMBD_BF16;
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int nb = n0 + 16 * (wn * FN + j);
    if (nb >= n_end) break;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      f32x4 v = acc[i][j];
      if constexpr (PASS == EXPERT_FWD) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v[q] += bias[i][q];
          if (a.relu) v[q] = v[q] < 0.f ? 0.f : v[q];  // (a NaN stays one)
        }
      }
      if (PASS != EXPERT_DW && half)
        *reinterpret_cast<u32x2 *>(stg + fi * (WM * 2 + 16) + (16 * i + 4 * kg) * 2) =
            u32x2{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3])};
      else
        *reinterpret_cast<f32x4 *>(stg + fi * (WM * 4 + 16) + (16 * i + 4 * kg) * 4) = v;
    }
    if (PASS != EXPERT_DW && half) {
      constexpr int LPR = WM / 8, RPI = 64 / LPR;  // lanes a row, rows an instruction
#pragma unroll
      for (int p = 0; p < 16 / RPI; ++p) {
        const int r = p * RPI + lane / LPR, m = mw + (lane % LPR) * 8, n = nb + r;
        u32x4 v = *reinterpret_cast<const u32x4 *>(stg + r * (WM * 2 + 16) + (lane % LPR) * 16);
        if (n < n_end && m < M) {
          if constexpr (PASS == EXPERT_DX) {
            if (a.mask) {
              const int row = a.rows ? a.rows[n] : n;
              u32x4 mk = {0u, 0u, 0u, 0u};
              if (row >= 0 && row < a.n_x) mk = *reinterpret_cast<const u32x4 *>(x + (int64_t)row * a.ldx + m);
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                if (!(bf16_to_f32((uint16_t)mk[q]) > 0.f)) v[q] &= 0xffff0000u;
                if (!(bf16_to_f32((uint16_t)(mk[q] >> 16)) > 0.f)) v[q] &= 0xffffu;
              }
            }
          }
          *reinterpret_cast<u32x4 *>(reinterpret_cast<uint16_t *>(a.out) + (int64_t)n * a.ldo + m) = v;
        }
      }
    } else {
      constexpr int LPR = WM / 4, RPI = 64 / LPR;
#pragma unroll
      for (int p = 0; p < 16 / RPI; ++p) {
        const int r = p * RPI + lane / LPR, m = mw + (lane % LPR) * 4, n = nb + r;
        f32x4 v = *reinterpret_cast<const f32x4 *>(stg + r * (WM * 4 + 16) + (lane % LPR) * 16);
        if (n < n_end && m < M) {
          if constexpr (PASS == EXPERT_DX) {
            if (a.mask) {
              const int row = a.rows ? a.rows[n] : n;
              u32x2 mk = {0u, 0u};
              if (row >= 0 && row < a.n_x) mk = *reinterpret_cast<const u32x2 *>(x + (int64_t)row * a.ldx + m);
#pragma unroll
              for (int q = 0; q < 4; ++q)
                if (!(bf16_to_f32((uint16_t)(mk[q >> 1] >> (16 * (q & 1)))) > 0.f)) v[q] = 0.f;
            }
          }
          *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out) +
                                     (PASS == EXPERT_DW ? (int64_t)e * a.so : 0) + (int64_t)n * a.ldo + m) = v;
        }
      }
    }
  }
}

bool al16(const void *p, int64_t ld, int es) { return (uintptr_t)p % 16 == 0 && ld * es % 16 == 0; }

}  // namespace

bool expert_wide_fits(int pass, int dtype, const ExpertArgs &a) {
  const int es = a.out_dtype == IMBD_BF16 ? 2 : 4;
  const int64_t ld_most = (int64_t)1 << 22;  // 256 rows of a tile within one descriptor
  if (dtype != IMBD_BF16 || a.d_in % 8 || a.d_out % 8) return false;
  if (a.out && (!al16(a.out, a.ldo, es) || (pass == EXPERT_DW && a.so % 4))) return false;
  if (pass != EXPERT_DW && (!al16(a.w, a.ldw, 2) || a.sw % 8 || a.ldw >= ld_most)) return false;
  if (pass != EXPERT_FWD && (!al16(a.dy, a.lddy, 2) || a.lddy >= ld_most)) return false;
  if (pass != EXPERT_DX || a.mask) {
    if (!al16(a.x, a.ldx, 2) || a.ldx >= ld_most) return false;
    // gathered rows lie anywhere in x: all of it within one descriptor
    if (a.rows && pass != EXPERT_DX && (int64_t)a.n_x * a.ldx * 2 > (int64_t)XW_MOST) return false;
  }
  return a.n_rows < (1 << 29);  // byte offsets into rows
}

template <int PASS, int BM, int BN, int NS, int WGS>
static int launch(const ExpertArgs &a, hipStream_t s) {
  const int M = PASS == EXPERT_FWD ? a.d_out : a.d_in;
  const int64_t tm = PASS == EXPERT_DW && !a.out ? 1 : (M + BM - 1) / BM;
  const int64_t tn = (a.d_out + BN - 1) / BN;
  const int64_t rows = row_tiles_most(a.n_rows, a.E, BN), blocks = (PASS == EXPERT_DW ? a.E * tn : rows) * tm;
  if (blocks >= ((int64_t)1 << 31) - 256) {
    set_error("expert product: %lld tiles are more than one launch takes", (long long)blocks);
    return IMBD_EUNSUPPORTED;
  }
  const dim3 grid((unsigned)((blocks + 255) / 256 * 256));
  {
    LaunchTimer t(IMBD_K_EXPERT_FWD + PASS, 0, s);
    if (a.rows && PASS != EXPERT_DX)
      hipLaunchKernelGGL((expert_wide_kernel<PASS, BM, BN, NS, true, WGS>), grid, dim3(256), 0, s, a, (int)tm,
                         (int)(PASS == EXPERT_DW ? tn : rows));
    else
      hipLaunchKernelGGL((expert_wide_kernel<PASS, BM, BN, NS, false, WGS>), grid, dim3(256), 0, s, a, (int)tm,
                         (int)(PASS == EXPERT_DW ? tn : rows));
  }
  return check_launch("expert_wide");
}

int run_expert_wide(int pass, const ExpertArgs &a, hipStream_t s) {
  if (pass == EXPERT_FWD) return launch<EXPERT_FWD, 256, 256, 4, 1>(a, s);
  if (pass == EXPERT_DX) return launch<EXPERT_DX, 256, 256, 4, 1>(a, s);
  return launch<EXPERT_DW, 256, 256, 4, 1>(a, s);
}

}  // namespace imbd
